"""A whole decoder layer chained from the C-ABI operators (no compute here:
each step is one library call; this module only allocates the intermediate
tensors and passes views).

The dataflow is the operator graph of one Llama-style layer (the paper's unit
of profiling and scaling, Section 2.2):

    [residual +] RMS Norm -> QKV linear -> RoPE(q, k) -> KV-cache write(k, v)
    -> attention (prefill: causal ragged; decode: paged) -> O linear
    -> residual + RMS Norm -> gate-up linear -> SiLU-mul -> down linear

`residual` follows the usual convention: None for the first layer (the input
is its own residual), otherwise the running residual, which the two fused
norms update in place to x + residual.  The layer returns the MLP output `y`
and the residual to pass to the next layer together with `y`.

A layer whose weights hold `inv_freq` (of opscale_rope_frequencies) turns,
normalises (`w_q_norm` and `w_k_norm` [head_dim], both or neither) and caches its
heads in one call.  One whose shape has a softcap or a window, or whose step has
`rules` (slopes, prefix_lens, doc_starts), attends with them.
"""
from __future__ import annotations

import dataclasses
import math

from . import _lib as L


@dataclasses.dataclass(frozen=True)
class LayerShape:
    hidden: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    ffn: int
    eps: float = 1e-5
    rope_theta: float = 500000.0
    # with weights that hold inv_freq
    rope_interleaved: bool = False
    rope_magnitude: float = 1.0
    head_eps: float = 1e-6
    # attention's cap of the scores and its reach in keys (0: none)
    softcap: float = 0.0
    window: int = 0


def _front(shape: LayerShape, w, x, residual, stream):
    """[residual +] norm and the QKV projection; returns (qkv, residual)."""
    import torch
    if residual is None:
        residual = x.clone()
        h1 = L.opscale_rmsnorm(x, w["w_norm1"], eps=shape.eps, stream=stream)
    else:
        h1 = torch.empty_like(x)
        L.opscale_add_rmsnorm(x, residual, w["w_norm1"], y=h1, eps=shape.eps, stream=stream)
    qkv = L.opscale_linear(h1, w["w_qkv"], stream=stream)
    return h1, qkv, residual


def _split(shape: LayerShape, qkv):
    T = qkv.shape[0]
    Hq, Hkv, D = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    q = qkv[:, : Hq * D].view(T, Hq, D)
    k = qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
    v = qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
    return q, k, v


def _place(shape: LayerShape, w, q, k, v, positions, k_cache, v_cache, slot_mapping, stream):
    """Turn q and k to their positions, in place, and write k and v to the cache."""
    if "inv_freq" in w:
        L.opscale_qk_norm_rope(q, k, positions, w["inv_freq"], w.get("w_q_norm"), w.get("w_k_norm"), shape.head_eps,
                               shape.rope_interleaved, shape.rope_magnitude, v, k_cache, v_cache, slot_mapping,
                               stream=stream)
        return
    if "w_q_norm" in w or "w_k_norm" in w or shape.rope_interleaved or shape.rope_magnitude != 1.0:
        raise L.OpscaleError(L.OPSCALE_ERR_INVALID_ARG, "head norms and rotations other than the plain one take inv_freq")
    L.opscale_rope(q, k, positions, shape.rope_theta, stream=stream)
    L.opscale_reshape_and_cache(k, v, k_cache, v_cache, slot_mapping, stream=stream)


def _rules(shape: LayerShape, rules):
    """The modifiers of the layer's attention, empty for the plain one."""
    r = {n: t for n, t in (rules or {}).items() if t is not None}
    if shape.softcap:
        r["softcap"] = shape.softcap
    if shape.window:
        r["window"] = shape.window
    return r


def _back(shape: LayerShape, w, attn, residual, stream):
    import torch
    T = attn.shape[0]
    o = L.opscale_linear(attn.view(T, -1), w["w_o"], stream=stream)
    h2 = torch.empty_like(o)
    L.opscale_add_rmsnorm(o, residual, w["w_norm2"], y=h2, eps=shape.eps, stream=stream)
    gu = L.opscale_linear(h2, w["w_gate_up"], stream=stream)
    act = L.opscale_swiglu(gu, stream=stream)
    y = L.opscale_linear(act, w["w_down"], stream=stream)
    return {"o": o, "h2": h2, "gate_up": gu, "act": act, "y": y}


def prefill_layer(shape: LayerShape, w, x, residual, positions, cu_seqlens, max_seqlen: int, k_cache, v_cache,
                  slot_mapping, stream=None, rules=None):
    """One layer over a ragged prefill batch x [T, H].  positions / slot_mapping:
    int32 [T] on the GPU (position of each token in its prompt, cache slot of
    each token); cu_seqlens int32 [B + 1].  Attention sees the step's own tokens
    only, so each prompt is whole: one whose beginning is in the cache already
    would lose those keys.  rules: a dict of the step's slopes, prefix_lens and
    doc_starts, each as in opscale_attn_prefill_mod."""
    h1, qkv, residual = _front(shape, w, x, residual, stream)
    q, k, v = _split(shape, qkv)
    _place(shape, w, q, k, v, positions, k_cache, v_cache, slot_mapping, stream)
    mods = _rules(shape, rules)
    attend = L.opscale_attn_prefill_mod if mods else L.opscale_attn_prefill
    attn = attend(q, k, v, cu_seqlens, max_seqlen, 1.0 / math.sqrt(shape.head_dim), True, stream=stream, **mods)
    out = _back(shape, w, attn, residual, stream)
    out.update(h1=h1, qkv=qkv, attn=attn, residual=residual)
    return out


def decode_layer(shape: LayerShape, w, x, residual, positions, slot_mapping, k_cache, v_cache, block_table,
                 context_lens, max_context_len: int, workspace=None, stream=None, rules=None):
    """One decode step of the layer for B sequences, x [B, H] (one new token
    each at positions[b] = context_lens[b] - 1, written to cache slot
    slot_mapping[b] before attention reads the whole context).  rules: as in
    prefill_layer, doc_starts [B].  workspace: of the attention call's own
    workspace_size (opscale_attn_decode_mod_workspace_size with modifiers)."""
    h1, qkv, residual = _front(shape, w, x, residual, stream)
    q, k, v = _split(shape, qkv)
    _place(shape, w, q, k, v, positions, k_cache, v_cache, slot_mapping, stream)
    mods = _rules(shape, rules)
    attend = L.opscale_attn_decode_mod if mods else L.opscale_attn_decode
    attn = attend(q, k_cache, v_cache, block_table, context_lens, max_context_len, 1.0 / math.sqrt(shape.head_dim),
                  workspace=workspace, stream=stream, **mods)
    out = _back(shape, w, attn, residual, stream)
    out.update(h1=h1, qkv=qkv, attn=attn, residual=residual)
    return out
