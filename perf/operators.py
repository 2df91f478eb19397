"""The attention path beyond one fixed layer shape: calls whose speed counts, with a plain form of each.

Operators (the "kind" of a case):
  qk_rope   RMS Norm of every query and key head, position rotation (half or interleaved pairs, the whole head or its
            first part, scaled frequencies) and, where a cache is given, its K and V rows, in one pass
  tables    block tables, slots, positions, offsets and lengths of a step, from the requests' lengths
  prefill   ragged grouped-query attention whose scores may be capped by a tanh or lowered with distance, under any
            of a causal, window, document and prefix mask
  decode    one new token a sequence under the same rules, over a paged cache

With `own` false, run() is elementary torch in 32 bits (angles in 64); with it true, the package's entry points.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
BF16, F32 = "bf16", "f32"


def _dtype(c):
    return torch.bfloat16 if c["dt"] == BF16 else torch.float32


# ------------------------------------------------------------------ lengths --
def _lens(dist, batch, lo, hi, seed=0):
    return {"dist": dist, "batch": batch, "lo": lo, "hi": hi, "len_seed": seed}


def lengths(c):
    """Prompt, context or new-token lengths of a case, from the case alone."""
    rng = np.random.default_rng(c["len_seed"])
    if c["dist"] == "lognormal":
        v = np.rint(rng.lognormal(0.5 * (math.log(c["lo"]) + math.log(c["hi"])), 1.0, c["batch"]))
    elif c["dist"] == "uniform":
        v = rng.integers(c["lo"], c["hi"], size=c["batch"], endpoint=True)
    else:  # "equal"
        v = np.full(c["batch"], c["hi"])
    return np.clip(v, c["lo"], c["hi"]).astype(np.int64)


def _rules(cap=0.0, bias=False, window=0, prefix=0, docs=0, causal=True):
    """cap: of the tanh; window: keys back; prefix: tokens that all see, at most; docs: mean document length."""
    return {"cap": cap, "bias": bias, "window": window, "prefix": prefix, "docs": docs, "causal": causal}


def listed():
    return [
        # One user's next token: norm, rotation and cache write of an 8B-shaped layer.  The smallest call.
        dict(name="qk_rope_b1", kind="qk_rope", dt=BF16, t=1, hq=32, hkv=8, d=128, rot=128, norm=True, pairs="half",
             scaling="none", maxpos=8192, block=16),
        # A ragged prefill batch with 70B-shaped heads, frequencies scaled for a long context.
        dict(name="qk_rope_prefill_t8871", kind="qk_rope", dt=BF16, t=8871, hq=64, hkv=8, d=128, rot=128, norm=True,
             pairs="half", scaling="bands", maxpos=131072, block=16),
        # One chunk of a chunked prefill in fp32: half of each head turned, neighbouring elements as pairs, no norm.
        dict(name="qk_rope_chunk_f32_t1023", kind="qk_rope", dt=F32, t=1023, hq=28, hkv=4, d=128, rot=64, norm=False,
             pairs="neighbours", scaling="ramp", maxpos=33000, block=0),
        # The tables of a decode step: 256 sequences of 128 to 8192 tokens, one new one each.
        dict(name="tables_decode_b256", kind="tables", block=16, new="one", **_lens("uniform", 256, 128, 8192)),
        # Admission of a burst: 1024 ragged prompts, some with a cached beginning, padded to a captured graph's size.
        dict(name="tables_prefill_b1024", kind="tables", block=16, new="prompt", **_lens("lognormal", 1024, 4, 4096)),
        # Sixteen ragged prompts through a layer with capped scores.
        dict(name="prefill_cap_ragged16", kind="prefill", dt=BF16, hq=32, hkv=8, d=128, **_rules(cap=50.0),
             **_lens("lognormal", 16, 16, 4096)),
        # Long prompts through a layer with capped scores that looks 4096 keys back.  The largest call.
        dict(name="prefill_cap_window_long2", kind="prefill", dt=BF16, hq=64, hkv=8, d=128,
             **_rules(cap=50.0, window=4096), **_lens("equal", 2, 8192, 8192)),
        # Rows of packed documents behind a common instruction that all of them see, scores lowered with distance.
        dict(name="prefill_bias_docs_b3", kind="prefill", dt=BF16, hq=16, hkv=16, d=64,
             **_rules(bias=True, prefix=200, docs=700), **_lens("uniform", 3, 2000, 4096)),
        # The tiny layer's attention in fp32 with a bidirectional prefix and a cap.
        dict(name="prefill_prefix_f32_b2", kind="prefill", dt=F32, hq=4, hkv=4, d=64, **_rules(cap=30.0, prefix=64),
             **_lens("uniform", 2, 96, 160)),
        # A 256-sequence decode step with capped scores, contexts of 128 to 8192.
        dict(name="decode_cap_b256", kind="decode", dt=BF16, hq=32, hkv=8, d=128, block=16, **_rules(cap=50.0),
             **_lens("uniform", 256, 128, 8192)),
        # A few long conversations, 4096 keys back and the opening tokens, scores lowered with distance, seven query
        # heads to a key head.
        dict(name="decode_window_b4_long", kind="decode", dt=BF16, hq=28, hkv=4, d=128, block=16,
             **_rules(bias=True, window=4096, prefix=100), **_lens("uniform", 4, 8192, 32768)),
        # One short conversation in fp32.
        dict(name="decode_f32_b1", kind="decode", dt=F32, hq=8, hkv=1, d=128, block=16, **_rules(cap=30.0),
             **_lens("equal", 1, 700, 700)),
    ]


# --------------------------------------------------------------------- draw --
def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_rules(rng, hi):
    return _rules(cap=rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]), bias=rng.random() < 0.4,
                  window=_log(rng, 1, hi) if rng.random() < 0.4 else 0,
                  prefix=_log(rng, 1, hi) if rng.random() < 0.3 else 0,
                  docs=_log(rng, 8, hi) if rng.random() < 0.3 else 0, causal=rng.random() < 0.85)


def _some_lengths(rng, batch, lo, hi):
    return _lens(rng.choice(["uniform", "lognormal"]), batch, lo, hi, rng.randrange(1 << 30))


def _draw(rng):
    kind = rng.choice(["qk_rope", "tables", "prefill", "prefill", "decode", "decode"])
    heads = [(32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 16, 64), (8, 1, 128), (12, 3, 64), (32, 8, 64), (40, 8, 128)]
    hq, hkv, d = rng.choice(heads)
    dt = BF16 if rng.random() < 0.8 else F32
    if kind == "qk_rope":
        d = rng.choice([64, 96, 128, 256])
        return dict(kind=kind, dt=dt, t=_log(rng, 1, 8871), hq=hq, hkv=hkv, d=d,
                    rot=rng.choice([d, d, d // 2, 32]), norm=rng.random() < 0.7,
                    pairs=rng.choice(["half", "neighbours"]), scaling=rng.choice(["none", "linear", "bands", "ramp"]),
                    maxpos=_log(rng, 16, 131072), block=rng.choice([0, 16, 64]))
    if kind == "tables":
        if rng.random() < 0.5:
            hi = _log(rng, 8, 8192)
            return dict(kind=kind, block=rng.choice([1, 16, 16, 64, 256]), new="one",
                        **_some_lengths(rng, _log(rng, 1, 4096), max(1, hi // 64), hi))
        hi = _log(rng, 8, 16384)
        return dict(kind=kind, block=rng.choice([1, 16, 16, 64, 256]), new="prompt",
                    **_some_lengths(rng, max(1, min(_log(rng, 1, 4096), 1_000_000 // hi)), max(1, hi // 64), hi))
    if kind == "prefill":
        if dt == F32:
            hi = _log(rng, 16, 1024)
            return dict(kind=kind, dt=dt, hq=hkv, hkv=hkv, d=d, **_draw_rules(rng, hi),
                        **_some_lengths(rng, rng.randint(1, 4), max(1, hi // 16), hi))
        hi = _log(rng, 32, 8192)
        return dict(kind=kind, dt=dt, hq=hq, hkv=hkv, d=d, **_draw_rules(rng, hi),
                    **_some_lengths(rng, max(1, min(_log(rng, 1, 48), 16384 // hi)), max(1, hi // 32), hi))
    hi = _log(rng, 16, 32768) if dt == BF16 else _log(rng, 16, 2048)
    batch = max(1, min(_log(rng, 1, 512), (600_000 if dt == BF16 else 8192) // hi))
    return dict(kind=kind, dt=dt, hq=hq, hkv=hkv, d=d, block=rng.choice([16, 16, 32, 64]),
                **{**_draw_rules(rng, hi), "causal": True}, **_some_lengths(rng, batch, max(1, hi // 32), hi))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (5e13 if c.get("dt") == F32 else 1e15))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


# ------------------------------------------------------------------- inputs --
class _Draws:
    """Normal tensors from one seed, in the order they are asked for."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def __call__(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=self.g)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def _scaled(c):
    """The rotation's arguments of a case: (base, factor, low, high, original context)."""
    return {"none": (500000.0, 1.0, 1.0, 4.0, 8192), "linear": (10000.0, 4.0, 1.0, 4.0, 8192),
            "bands": (500000.0, 8.0, 1.0, 4.0, 8192), "ramp": (10000.0, 16.0, 1.0, 32.0, 4096)}[c["scaling"]]


def _frequencies(c):
    """Radians a position of each pair, and the factor on sine and cosine, in 64 bits."""
    theta, factor, low, high, orig = _scaled(c)
    rot = c["rot"]
    i = np.arange(rot // 2, dtype=np.float64)
    f = theta ** (-2.0 * i / rot)
    if c["scaling"] == "linear":
        return f / factor, 1.0
    if c["scaling"] == "bands":  # by turns within the original context: few of them, slowed by the factor
        t = np.clip((orig * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return (1 - t) * f / factor + t * f, 1.0
    if c["scaling"] == "ramp":  # the same by pair index between the pairs that turn `high` and `low` times
        at = [rot * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(theta)) for turns in (high, low)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        r = np.clip((i - first) / max(last - first, 0.001), 0.0, 1.0)
        return f / factor * r + f * (1 - r), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _doc_starts(c, lens, seed, rows):
    """Each row's document start within its prompt; the last rows of a prompt may be padding (a start past its end)."""
    rng = np.random.default_rng([int(seed), c["len_seed"], 17])
    out = []
    for n in (int(n) for n in lens):
        cuts = np.cumsum(np.maximum(1, rng.geometric(1.0 / c["docs"], size=n // c["docs"] * 3 + 4)))
        start = np.zeros(n, np.int64)
        for k in cuts[cuts < n]:
            start[k:] = k
        pad = int(rng.integers(0, 4)) if n > 8 else 0
        start[n - pad:] = n
        out.append(start if rows else start[n - pad - 1:n - pad])
    return np.concatenate(out)


def _rule_inputs(c, s, dr, lens, seed, rows):
    rng = np.random.default_rng([int(seed), 19])
    s["slopes"] = s["prefix"] = s["starts"] = None
    if c["bias"]:
        h = torch.arange(1, c["hq"] + 1, dtype=torch.float32, device=DEV)
        s["slopes"] = torch.exp2(-8.0 * h / c["hq"]) * (1.0 + 0.1 * dr(c["hq"]).abs())
    if c["prefix"]:
        s["prefix"] = _i32(np.minimum(rng.integers(0, c["prefix"], size=len(lens), endpoint=True), lens))
    if c["docs"]:
        s["starts"] = _i32(_doc_starts(c, lens, seed, rows))


def _kept(c, lens, new):
    """Tokens that a prompt's request has in the cache already (a shared beginning), for some of them."""
    rng = np.random.default_rng([c["len_seed"], 23])
    return np.where(rng.random(len(lens)) < 0.25, rng.integers(0, 600, size=len(lens)), 0) if new == "prompt" else lens - 1


def _cdiv(a, b):
    return (a + b - 1) // b


def _tables_shape(c):
    """Of a table case: tokens in the cache, new ones, table columns, pages in use, free pages, token slots."""
    lens = lengths(c)
    kept = _kept(c, lens, c["new"])
    new = np.ones_like(lens) if c["new"] == "one" else lens
    pages = int(_cdiv(kept, c["block"]).sum())
    want = int((_cdiv(kept + new, c["block"]) - _cdiv(kept, c["block"])).sum())
    return kept, new, int(_cdiv(kept + new, c["block"]).max()) + 2, pages, want + 5, _cdiv(int(new.sum()), 256) * 256


def prepare(c, seed):
    if own:
        import paper_2608_13499_amd as ops
    dr, kind, s, rng = _Draws(seed), c["kind"], {"c": c}, np.random.default_rng([int(seed), 11])
    if kind == "tables":
        kept, new, cols, pages, free, slots = _tables_shape(c)
        perm = rng.permutation(pages + free).astype(np.int32)  # pages scattered, as after a long serving run
        table, at = np.full((len(kept), cols), -1, np.int32), 0
        for b, n in enumerate(_cdiv(kept, c["block"])):
            table[b, :n] = perm[at:at + n]
            at += n
        begin = int(rng.integers(0, 4))
        s.update(kept=_i32(kept), new=_i32(new), table=_i32(table), free=_i32(perm[pages:]), begin=_i32([begin]))
        s["tokens"] = slots
        return s
    dt = _dtype(c)
    if kind == "qk_rope":
        t, hq, hkv, d = c["t"], c["hq"], c["hkv"], c["d"]
        s["qkv"] = dr(t, (hq + 2 * hkv) * d).to(dt)
        s["pos"] = _i32(np.sort(rng.integers(0, c["maxpos"], size=t)))
        s["wq"] = s["wk"] = s["k_cache"] = s["v_cache"] = s["slots"] = None
        if c["norm"]:
            s["wq"], s["wk"] = (dr(d, std=0.1, mean=1.0).to(dt) for _ in range(2))
        if c["block"]:
            pages = _cdiv(t, c["block"]) + 3
            s["k_cache"], s["v_cache"] = (dr(pages, c["block"], hkv, d).to(dt) for _ in range(2))
            s["slots"] = _i32(rng.permutation(pages * c["block"])[:t])
        s["q_out"], s["k_out"] = (torch.empty(t, h, d, dtype=dt, device=DEV) for h in (hq, hkv))
        if own:
            theta, factor, low, high, orig = _scaled(c)
            s["freq"], s["magnitude"] = ops.opscale_rope_frequencies(c["rot"], theta, c["scaling"], factor, low, high,
                                                                     orig)
        else:
            f, s["magnitude"] = _frequencies(c)
            s["freq"] = torch.from_numpy(f).to(DEV)
        return s
    lens = lengths(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    s["lens"], s["maxlen"] = [int(n) for n in lens], int(lens.max())
    s["scale"] = 1.0 / math.sqrt(d)
    # queries and keys with a share in common, so that scores spread over -10 to 20 as a trained layer's do
    if kind == "prefill":
        t = int(lens.sum())
        qkv = dr(t, hq + 2 * hkv, d)
        qkv[:, :hq + hkv] = 1.5 * qkv[:, :hq + hkv] + 0.6 * dr(d)
        s["qkv"] = qkv.to(dt).view(t, -1)
        s["cu"] = _i32(np.concatenate([[0], np.cumsum(lens)]))
        _rule_inputs(c, s, dr, lens, seed, True)
        return s
    pages = _cdiv(lens, c["block"])
    perm, at = rng.permutation(int(pages.sum())), 0
    table = np.zeros((len(lens), int(pages.max())), np.int32)
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    common = 0.6 * dr(d)
    s["k"] = (1.5 * dr(at, c["block"], hkv, d) + common).to(dt)
    s["v"] = dr(at, c["block"], hkv, d).to(dt)
    s["q"] = (1.5 * dr(len(lens), hq, d) + common).to(dt)
    s["table"], s["ctx"] = _i32(table), _i32(lens)
    _rule_inputs(c, s, dr, lens, seed, False)
    if own:  # the scratch a serving loop keeps between steps
        s["ws"] = torch.empty(ops.opscale_attn_decode_mod_workspace_size(len(lens), hq, d, s["maxlen"]),
                              dtype=torch.uint8, device=DEV)
    return s


def _split(qkv, c):
    t, hq, hkv, d = qkv.shape[0], c["hq"], c["hkv"], c["d"]
    return (qkv[:, :hq * d].view(t, hq, d), qkv[:, hq * d:(hq + hkv) * d].view(t, hkv, d),
            qkv[:, (hq + hkv) * d:].view(t, hkv, d))


# -------------------------------------------------------------- plain forms --
def _turn(x, cos, sin, c):
    """The first `rot` elements of each head turned, pair by pair."""
    rot = c["rot"]
    y = x.clone()
    if c["pairs"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_qk_rope(s):
    c = s["c"]
    q, k, v = _split(s["qkv"], c)
    ang = s["pos"].double()[:, None] * s["freq"]
    cos, sin = ((f(ang) * s["magnitude"]).float()[:, None, :] for f in (torch.cos, torch.sin))

    def one(x, w, out):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        out.copy_(_turn(x, cos, sin, c))
        return out

    q, k = one(q, s["wq"], s["q_out"]), one(k, s["wk"], s["k_out"])
    if s["slots"] is None:
        return q, k
    rows = s["slots"].long()
    s["k_cache"].view(-1, *k.shape[1:])[rows] = k
    s["v_cache"].view(-1, *k.shape[1:])[rows] = v
    return q, k, s["k_cache"], s["v_cache"]


def _plain_tables(s):
    c, table, tokens = s["c"], s["table"], s["tokens"]
    block, cols = c["block"], table.shape[1]
    kept, new = s["kept"].long(), s["new"].long()
    cu = torch.zeros(len(kept) + 1, dtype=torch.int64, device=DEV)
    cu[1:] = torch.cumsum(new, 0)
    have, need = (kept + block - 1) // block, (kept + new + block - 1) // block
    taken = torch.cumsum(need - have, 0)
    col = torch.arange(cols, device=DEV)[None, :]
    at = s["begin"].long() + (taken - (need - have))[:, None] + col - have[:, None]
    fresh = (col >= have[:, None]) & (col < need[:, None])
    table.copy_(torch.where(fresh, s["free"][at.clamp(0, len(s["free"]) - 1)], table))
    t = torch.arange(tokens, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    live = t < cu[-1]
    b = b.clamp(max=len(kept) - 1)
    pos = torch.where(live, kept[b] + t - cu[b], 0)
    page = table[b, (pos // block).clamp(max=cols - 1)].long()
    slots = torch.where(live, page * block + pos % block, -1)
    i32 = [x.to(torch.int32) for x in (cu, pos, slots, kept + new, s["begin"] + taken[-1:])]
    return (*i32, table)


def _visible(i, j, last, prefix, start, c):
    """Whether the query at i sees the key at j (broadcast)."""
    ok = (j <= i) if c["causal"] else (j <= last)
    if c["window"]:
        ok = ok & (i - j < c["window"]) & (j - i < c["window"])
    if start is not None:
        ok = ok & (j >= start)
    if prefix is not None:
        ok = ok | (j < prefix)
    return ok


def _attend(q, k, v, i, j, seen, s, heads):
    """q [h, m, d], k and v [h, n, d], in 32 bits: the masked softmax over n; rows that see nothing are zero."""
    c = s["c"]
    sc = torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"]
    if c["cap"]:
        sc = c["cap"] * torch.tanh(sc / c["cap"])
    if s["slopes"] is not None:
        sc = sc - s["slopes"][heads][:, None, None] * (i - j).abs().float()
    sc = sc.masked_fill(~seen, -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True).clamp(min=-1e30))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_prefill(s):
    c = s["c"]
    q, k, v = _split(s["qkv"], c)
    group = c["hq"] // c["hkv"]
    out, at = torch.empty(q.shape, dtype=q.dtype, device=DEV), 0
    for b, n in enumerate(s["lens"]):
        j = torch.arange(n, device=DEV)
        seen = _visible(j[:, None], j[None, :], n - 1, None if s["prefix"] is None else s["prefix"][b],
                        None if s["starts"] is None else s["starts"][at:at + n, None], c)
        step = max(1, min(c["hkv"], (1 << 28) // (group * n * n)))  # KV heads at a time
        for g in range(0, c["hkv"], step):
            kv, h = slice(g, min(g + step, c["hkv"])), slice(g * group, min(g + step, c["hkv"]) * group)
            kk, vv = (x[at:at + n, kv].float().transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
            o = _attend(q[at:at + n, h].float().transpose(0, 1), kk, vv, j[:, None], j[None, :], seen, s, h)
            out[at:at + n, h] = o.transpose(0, 1)
        at += n
    return out


def _plain_decode(s):
    c = s["c"]
    q, (B, hq, d), hkv = s["q"].float(), s["q"].shape, c["hkv"]
    out = torch.empty_like(s["q"])
    rows = s["table"].shape[1] * c["block"]
    j = torch.arange(rows, device=DEV)
    step = max(1, (1 << 29) // (rows * hkv * d))  # sequences at a time
    for b0 in range(0, B, step):
        b = slice(b0, min(B, b0 + step))
        n = s["ctx"][b].long()[:, None]
        seen = (j < n) & _visible(n - 1, j, n - 1, None if s["prefix"] is None else s["prefix"][b].long()[:, None],
                                  None if s["starts"] is None else s["starts"][b].long()[:, None], c)
        kk, vv = (x[s["table"][b].long()].reshape(-1, rows, hkv, d).float().transpose(1, 2) for x in (s["k"], s["v"]))
        sc = torch.matmul(kk, q[b].view(-1, hkv, hq // hkv, d).transpose(2, 3).contiguous()).transpose(2, 3)
        sc = sc.reshape(-1, hq, rows) * s["scale"]
        if c["cap"]:
            sc = c["cap"] * torch.tanh(sc / c["cap"])
        if s["slopes"] is not None:
            sc = sc - s["slopes"][:, None] * (n - 1 - j).abs().float()[:, None]
        sc = sc.masked_fill(~seen[:, None], -math.inf)
        p = torch.exp(sc - sc.amax(-1, keepdim=True).clamp(min=-1e30))
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
        out[b] = torch.matmul(p.view(-1, hkv, hq // hkv, rows), vv).reshape(-1, hq, d)
    return out


# --------------------------------------------------------------------- run ---
def run(s):
    c = s["c"]
    kind = c["kind"]
    if not own:
        return {"qk_rope": _plain_qk_rope, "tables": _plain_tables, "prefill": _plain_prefill,
                "decode": _plain_decode}[kind](s)
    import paper_2608_13499_amd as ops
    if kind == "tables":
        return (*ops.opscale_block_tables(s["kept"], s["new"], s["table"], s["free"], s["begin"], c["block"],
                                          s["tokens"]), s["table"])
    if kind == "qk_rope":
        q, k, v = _split(s["qkv"], c)
        ops.opscale_qk_norm_rope(q, k, s["pos"], s["freq"], s["wq"], s["wk"], EPS, c["pairs"] == "neighbours",
                                 s["magnitude"], v, s["k_cache"], s["v_cache"], s["slots"], s["q_out"], s["k_out"])
        out = s["q_out"], s["k_out"]
        return out if s["slots"] is None else (*out, s["k_cache"], s["v_cache"])
    rules = dict(softcap=c["cap"], slopes=s["slopes"], window=c["window"], prefix_lens=s["prefix"],
                 doc_starts=s["starts"])
    if kind == "prefill":
        q, k, v = _split(s["qkv"], c)
        return ops.opscale_attn_prefill_mod(q, k, v, s["cu"], s["maxlen"], s["scale"], c["causal"], **rules)
    return ops.opscale_attn_decode_mod(s["q"], s["k"], s["v"], s["table"], s["ctx"], s["maxlen"], s["scale"], **rules,
                                       workspace=s["ws"])


# -------------------------------------------------------------------- work ---
def _seen_keys(c, lens, seed=0):
    """(query, key) pairs that see each other and keys that any query sees, over the prompts or sequences, with the
    mean prefix and whole documents of the mean length (what the seed draws differs a little)."""
    pairs, keys = 0, 0
    w, p = c["window"] or 1 << 60, c["prefix"] // 2
    for n in (int(n) for n in lens):
        i = np.arange(n, dtype=np.int64) if c["kind"] == "prefill" else np.array([n - 1], np.int64)
        start = i // c["docs"] * c["docs"] if c["docs"] else np.zeros_like(i)
        lo = np.maximum(start, i - w + 1)
        hi = i if c["causal"] else np.minimum(n - 1, i + w - 1)
        pre = min(p, n)
        pairs += int((np.maximum(0, hi - np.maximum(lo, pre) + 1) + pre).sum())
        keys += n if c["kind"] == "prefill" else int(hi[0] - max(lo[0], pre) + 1 + pre)
    return pairs, keys


def work(c):
    if c["kind"] == "tables":
        kept, new, cols, pages, free, tokens = _tables_shape(c)
        b, used = len(kept), int(new.sum())
        # lengths read, offsets and lengths written, a position and a slot a token, the pages taken copied, and the
        # half-filled page of a request that goes on read
        return {"bytes": 4 * (2 * b + 2 * b + 2 + 2 * tokens + 2 * (free - 5) + b), "flops": 4 * used}
    size = 2 if c["dt"] == BF16 else 4
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "qk_rope":
        t, qk = c["t"], c["t"] * (hq + hkv) * d
        cache = 3 * t * hkv * d if c["block"] else 0  # v read, k and v rows written
        return {"bytes": size * (2 * qk + cache) + 4 * t + 4 * c["rot"], "flops": (4 * qk if c["norm"] else 0) + 3 * qk}
    lens = lengths(c)
    pairs, keys = _seen_keys(c, lens)
    rows = int(lens.sum()) if c["kind"] == "prefill" else len(lens)
    pages = 0 if c["kind"] == "prefill" else keys // c["block"]
    return {"bytes": size * (2 * rows * hq + 2 * keys * hkv) * d + 4 * (pages + len(lens)), "flops": 4 * hq * d * pairs}


# ------------------------------------------------------------------- exact ---
def _exact_qk_rope(c, s):
    q, k, v = (x.double() for x in _split(s["qkv"], c))
    if s["wq"] is not None:
        q, k = (x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["d"] + EPS) * w.double()
                for x, w in ((q, s["wq"]), (k, s["wk"])))
    f, mag = _frequencies(c)
    ang = torch.outer(s["pos"].double(), torch.from_numpy(f).to(DEV))
    rotor = torch.polar(torch.full_like(ang, mag), ang)[:, None, :]  # a pair is a complex number
    rot = c["rot"]

    def turn(x):
        pair = x[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2) if c["pairs"] == "half" else \
            x[..., :rot].unflatten(-1, (-1, 2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * rotor)
        z = z.transpose(-1, -2) if c["pairs"] == "half" else z
        return torch.cat([z.reshape(*x.shape[:-1], rot), x[..., rot:]], -1)

    q, k = turn(q), turn(k)
    if s["slots"] is None:
        return q, k
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    kc.view(-1, c["hkv"], c["d"])[s["slots"].long()] = k
    vc.view(-1, c["hkv"], c["d"])[s["slots"].long()] = v
    return q, k, kc, vc


def _exact_tables(c, s):
    kept, new, table, free = (s[n].cpu().numpy() for n in ("kept", "new", "table", "free"))
    block, at = c["block"], int(s["begin"])
    pos, slots = np.zeros(s["tokens"], np.int32), np.full(s["tokens"], -1, np.int32)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    for b in range(len(kept)):
        for col in range(_cdiv(int(kept[b]), block), _cdiv(int(kept[b] + new[b]), block)):
            table[b, col] = free[at]
            at += 1
        p = np.arange(kept[b], kept[b] + new[b])
        pos[cu[b]:cu[b + 1]] = p
        slots[cu[b]:cu[b + 1]] = table[b, p // block] * block + p % block
    return tuple(_i32(x) for x in (cu, pos, slots, kept + new, [at], table))


def _exact_row_block(q, k, v, i, j, seen, slope, c, scale):
    sc = (q @ k.t()) * scale
    if c["cap"]:
        sc = torch.tanh(sc / c["cap"]) * c["cap"]
    sc = sc - slope * (i[:, None] - j[None, :]).abs().double()
    sc = torch.where(seen, sc, -torch.inf)
    return torch.nan_to_num(torch.softmax(sc, -1)) @ v


def _exact_seen(i, j, n, prefix, start, c):
    late = (j[None, :] > i[:, None]) if c["causal"] else torch.zeros(len(i), len(j), dtype=torch.bool, device=DEV)
    far = (i[:, None] - j[None, :]).abs() >= (c["window"] or 1 << 40)
    return ~(late | far | (j[None, :] < start[:, None])) | (j[None, :] < prefix)


def _exact_attention(c, s):
    """Head by head, some query rows at a time."""
    decode = c["kind"] == "decode"
    if not decode:
        q, k, v = _split(s["qkv"], c)
    else:
        q = s["q"]
    out, at, group = torch.zeros(q.shape, dtype=torch.float64, device=DEV), 0, c["hq"] // c["hkv"]
    for b, n in enumerate(s["lens"]):
        rows = 1 if decode else n
        j = torch.arange(n, device=DEV)
        prefix = 0 if s["prefix"] is None else int(s["prefix"][b])
        start = torch.zeros(rows, dtype=torch.int64, device=DEV) if s["starts"] is None else s["starts"][at:at + rows].long()
        if decode:
            pages = s["table"][b, :_cdiv(n, c["block"])].long()
            kb, vb = (x[pages].reshape(-1, c["hkv"], c["d"])[:n] for x in (s["k"], s["v"]))
        else:
            kb, vb = k[at:at + n], v[at:at + n]
        for r in range(0, rows, 4096):
            i = torch.tensor([n - 1], device=DEV) if decode else j[r:r + 4096]
            seen = _exact_seen(i, j, n, prefix, start[r:r + 4096], c)
            for g in range(c["hkv"]):
                kk, vv = kb[:, g].double().contiguous(), vb[:, g].double().contiguous()
                for h in range(g * group, (g + 1) * group):
                    slope = 0.0 if s["slopes"] is None else s["slopes"][h].double()
                    qq = q[at + r:at + r + len(i), h].double()
                    out[at + r:at + r + len(i), h] = _exact_row_block(qq, kk, vv, i, j, seen, slope, c, s["scale"])
        at += rows
    return out


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "qk_rope":
        return _exact_qk_rope(c, s)
    if c["kind"] == "tables":
        return _exact_tables(c, s)
    return _exact_attention(c, s)
