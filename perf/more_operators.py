"""The layer in fewer bits: an fp8 linear and a KV cache in 4 bits, calls whose speed counts, with a plain form of each.

Operators (the "kind" of a case):
  quantize  activations to e4m3 (8 bits) with a power-of-two scale for each token and 128 of its elements
  linear    y = x W^T (+ bias) of e4m3 operands, a scale for each token and 128 of K and for each 128 x 128 of W
  store     K and V rows of new tokens written to a paged cache of e2m1 elements (4 bits) with a power-of-two scale for
            each 32, and those tokens read back
  load      the keys of some requests read back from such a cache, packed
  decode    attention of one new token a sequence over such a cache

With `own` false, run() is elementary torch in 32 bits; with it true, the package's entry points.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BF16, F32 = "bf16", "f32"
BLOCK = 128  # elements of K that share a scale, and rows of W
GROUP = 32  # elements of a head that share a scale in the cache


def _dtype(c):
    return torch.bfloat16 if c["dt"] == BF16 else torch.float32


def _cdiv(a, b):
    return (a + b - 1) // b


# ------------------------------------------------------------------ lengths --
def _lens(dist, batch, lo, hi, seed=0):
    return {"dist": dist, "batch": batch, "lo": lo, "hi": hi, "len_seed": seed}


def lengths(c):
    """Prompt or context lengths of a case, from the case alone."""
    rng = np.random.default_rng(c["len_seed"])
    if c["dist"] == "lognormal":
        v = np.rint(rng.lognormal(0.5 * (math.log(c["lo"]) + math.log(c["hi"])), 1.0, c["batch"]))
    elif c["dist"] == "uniform":
        v = rng.integers(c["lo"], c["hi"], size=c["batch"], endpoint=True)
    else:  # "equal"
        v = np.full(c["batch"], c["hi"])
    return np.clip(v, c["lo"], c["hi"]).astype(np.int64)


def _rules(cap=0.0, bias=False, window=0, prefix=0):
    """cap: of the tanh; bias: scores lowered with distance; window: keys back; prefix: tokens that all see, at most."""
    return {"cap": cap, "bias": bias, "window": window, "prefix": prefix}


def listed():
    return [
        # The next token of one user on its way into an 8B-shaped layer.  The smallest call.
        dict(name="quantize_b1", kind="quantize", dt=BF16, m=1, k=4096),
        # A ragged prefill batch of 16 prompts before the down projection.
        dict(name="quantize_prefill_t8871", kind="quantize", dt=BF16, m=8871, k=14336),
        # The down projection of a decode step of 48 sequences: the weights' bytes count.
        dict(name="linear_down_m48", kind="linear", dt=BF16, m=48, n=4096, k=14336, bias=False),
        # The QKV projection, with a bias, of one chunk of a chunked prefill.
        dict(name="linear_qkv_m1023", kind="linear", dt=BF16, m=1023, n=6144, k=4096, bias=True),
        # Gate and up of the same 16 prompts: the matrix cores count.  The largest call.
        dict(name="linear_gate_up_t8871", kind="linear", dt=BF16, m=8871, n=28672, k=4096, bias=False),
        # The tiny layer's down projection with an fp32 result: K ends inside a block of scales.
        dict(name="linear_tiny_f32", kind="linear", dt=F32, m=128, n=256, k=688, bias=True),
        # The cache rows of a decode step: the last token of each of 256 sequences.
        dict(name="store_decode_b256", kind="store", dt=BF16, hkv=8, d=128, block=16, new="one",
             **_lens("uniform", 256, 128, 8192)),
        # The cache rows of 16 ragged prompts, and the prompts as later chunks will see them.
        dict(name="store_prefill_ragged16", kind="store", dt=BF16, hkv=8, d=128, block=16, new="prompt",
             **_lens("lognormal", 16, 16, 4096)),
        # Four long conversations leave the 4-bit cache, from the 100th key on.
        dict(name="load_b4_long", kind="load", dt=BF16, hkv=4, d=128, block=16, first=100,
             **_lens("uniform", 4, 8192, 32768)),
        # A decode step of 256 sequences.
        dict(name="decode_b256", kind="decode", dt=BF16, hq=32, hkv=8, d=128, block=16, **_rules(),
             **_lens("uniform", 256, 128, 8192)),
        # A few long conversations, 4096 keys back and the opening tokens, scores lowered with distance, seven query
        # heads to a key head.
        dict(name="decode_window_b4_long", kind="decode", dt=BF16, hq=28, hkv=4, d=128, block=16,
             **_rules(bias=True, window=4096, prefix=100), **_lens("uniform", 4, 8192, 32768)),
        # One short conversation with an fp32 query and capped scores.
        dict(name="decode_f32_b1", kind="decode", dt=F32, hq=8, hkv=1, d=128, block=16, **_rules(cap=30.0),
             **_lens("equal", 1, 700, 700)),
    ]


# --------------------------------------------------------------------- draw --
def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _some_lengths(rng, batch, lo, hi):
    return _lens(rng.choice(["uniform", "lognormal"]), batch, lo, hi, rng.randrange(1 << 30))


def _draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear", "store", "load", "decode", "decode"])
    dt = BF16 if rng.random() < 0.8 else F32
    if kind == "quantize":
        k = rng.choice([4096, 4096, 3584, 8192, 14336, 28672, 688, 16 * _log(rng, 1, 1024)])
        return dict(kind=kind, dt=dt, m=_log(rng, 1, 8871), k=k)
    if kind == "linear":
        n, k = rng.choice([(6144, 4096), (4096, 4096), (28672, 4096), (4096, 14336), (10240, 8192), (8192, 8192),
                           (57344, 8192), (8192, 28672), (4608, 3584), (2816, 1024), (256, 688),
                           (8 * _log(rng, 1, 1024), 16 * _log(rng, 1, 512))])
        return dict(kind=kind, dt=dt, m=_log(rng, 1, 8871), n=n, k=k, bias=rng.random() < 0.3)
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 16, 64), (8, 1, 128), (12, 3, 64),
                             (32, 8, 64), (40, 8, 128)])
    block = rng.choice([16, 16, 32, 64, 128])
    if kind == "store":
        one = rng.random() < 0.5
        hi = _log(rng, 8, 8192)
        batch = _log(rng, 1, 1024) if one else max(1, min(_log(rng, 1, 64), 32768 // hi))
        return dict(kind=kind, dt=dt, hkv=hkv, d=d, block=block, new="one" if one else "prompt",
                    **_some_lengths(rng, batch, max(1, hi // 32), hi))
    if kind == "load":
        hi = _log(rng, 8, 32768)
        return dict(kind=kind, dt=dt, hkv=hkv, d=d, block=block, first=rng.choice([0, 0, _log(rng, 1, hi)]),
                    **_some_lengths(rng, max(1, min(_log(rng, 1, 64), 131072 // hi)), max(1, hi // 32), hi))
    hi = _log(rng, 16, 32768)
    batch = max(1, min(_log(rng, 1, 512), 600_000 // hi))
    rules = _rules(cap=rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]), bias=rng.random() < 0.3,
                   window=_log(rng, 1, hi) if rng.random() < 0.3 else 0,
                   prefix=_log(rng, 1, hi) if rng.random() < 0.2 else 0)
    return dict(kind=kind, dt=dt, hq=hq, hkv=hkv, d=d, block=block, **rules,
                **_some_lengths(rng, batch, max(1, hi // 32), hi))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 2e15)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


# ------------------------------------------------------- the formats, plain --
def _exponent(most, top, lowest, highest):
    """The smallest e with `most` <= 1.75 * 2^(top + e), within [lowest, highest]."""
    m, x = torch.frexp(most)  # m in [1/2, 1)
    e = torch.where(m <= 0.875, x - top - 1, x - top)
    return torch.where(most > 0, e, lowest).clamp(lowest, highest)


def _power(e):
    """2^e in fp32, of integers e in [-126, 127]."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _to_e4m3(x):
    """x [M, K] in fp32 as e4m3 elements, and the scales [blocks of K, M]."""
    m, k = x.shape
    blocks = _cdiv(k, BLOCK)
    most = torch.nn.functional.pad(x.abs(), (0, blocks * BLOCK - k)).view(m, blocks, BLOCK).amax(-1)
    e = _exponent(most, 8, -100, 120)
    codes = (x * _power(-e).repeat_interleave(BLOCK, 1)[:, :k]).to(torch.float8_e4m3fn)
    return codes, _power(e).t().contiguous()


def _round_e2m1(y):
    """The e2m1 value (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) nearest to y, ties to the even one, as y's type."""
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(y.dtype)
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), y)


def _to_e2m1(x):
    """x [..., D] in fp32 as (e2m1 values [..., D], exponents [..., D / 32])."""
    g = x.unflatten(-1, (-1, GROUP))
    e = _exponent(g.abs().amax(-1), 2, -100, 125)
    return _round_e2m1(g * _power(-e)[..., None]).flatten(-2), e


def _pack(x, k_rows):
    """Pages of a cache, as bytes, from x [pages, block, hkv, D]: of each page and head, the codes of its rows (element
    2 i of a row in the low four bits of its byte i, 2 i + 1 in the high ones), then a byte of e + 127 for each group
    and row."""
    v, e = _to_e2m1(x.transpose(1, 2).float())
    a = v.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(v).to(torch.uint8) << 3)
    both = code[..., 0::2] | (code[..., 1::2] << 4)
    flat = torch.cat([both.flatten(-2), (e + 127).to(torch.uint8).transpose(-1, -2).flatten(-2)], -1)
    return flat.view(k_rows)


def _unpack(pages, d, values):
    """fp32 [..., block, D] of the bytes [..., block, D / 2 + D / 32] of pages and heads."""
    block, lead = pages.shape[-2], pages.shape[:-2]
    flat = pages.reshape(*lead, -1)
    codes, e = flat[..., :block * d // 2], flat[..., block * d // 2:]
    x = torch.stack([values[(codes & 15).long()], values[(codes >> 4).long()]], -1).view(*lead, block, d // GROUP, GROUP)
    e = e.to(torch.int32).view(*lead, d // GROUP, block).transpose(-1, -2)
    return (x * _power(e - 127)[..., None]).flatten(-2)


def _values():
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    return torch.cat([v, -v])


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


def _activations(c, dr):
    """Tokens with a few channels that are much larger than the others, as a trained layer's have."""
    return dr(c["m"], c["k"]) * torch.exp(1.0 * dr(c["k"]))


def _table(c, lens, rng):
    """Pages scattered over the cache, as after a long serving run."""
    pages = _cdiv(lens, c["block"])
    perm, at = rng.permutation(int(pages.sum())), 0
    table = np.zeros((len(lens), int(pages.max())), np.int32)
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, at


def prepare(c, seed):
    dr, kind, s, rng = _Draws(seed), c["kind"], {"c": c}, np.random.default_rng([int(seed), 11])
    dt = _dtype(c)
    if kind == "quantize":
        s["x"] = _activations(c, dr).to(dt)
        return s
    if kind == "linear":
        s["xq"], s["xs"] = _to_e4m3(_activations(c, dr))
        n, k = c["n"], c["k"]
        # trained weights as they are stored: e4m3 elements that fill their range, fp32 scales of a block's own
        s["wq"] = (dr(n, k) * 90.0).clamp(-448, 448).to(torch.float8_e4m3fn)
        s["ws"] = torch.exp(0.3 * dr(_cdiv(n, BLOCK), _cdiv(k, BLOCK))) * (0.02 / 90.0)
        s["bias"] = dr(n).to(dt) if c["bias"] else None
        if own:
            import paper_2608_13499_amd as ops  # the scratch that a serving loop keeps between steps
            s["scratch"] = torch.empty(ops.opscale_linear_fp8_workspace_size(c["m"], n, k, dt), dtype=torch.uint8,
                                       device=DEV)
        return s
    lens = lengths(c)
    hkv, d, block = c["hkv"], c["d"], c["block"]
    table, pages = _table(c, lens, rng)
    shape = (hkv, block, d // 2 + d // GROUP)
    s["table"], s["values"] = _i32(table), _values()
    if kind == "store":
        new = np.ones_like(lens) if c["new"] == "one" else lens
        first = lens - new
        s["t"] = int(new.sum())
        s["cu"], s["first"] = _i32(np.concatenate([[0], np.cumsum(new)])), _i32(first)
        s["slots"] = _i32(np.concatenate([table[b, np.arange(f, n) // block].astype(np.int64) * block +
                                          np.arange(f, n) % block for b, (f, n) in enumerate(zip(first, lens))]))
        s["kv"] = (1.5 * dr(s["t"], 2 * hkv, d) + 0.6 * dr(2 * hkv, d)).to(dt)
        s["k"], s["v"] = (torch.zeros(pages, *shape, dtype=torch.uint8, device=DEV) for _ in range(2))
        return s
    # keys with a share in common with each other and the queries, so that scores spread over -10 to 20 as a trained
    # layer's do; some pages at a time
    common = 0.6 * dr(d)
    s["k"], s["v"] = (torch.empty(pages, *shape, dtype=torch.uint8, device=DEV) for _ in range(2))
    for p in range(0, pages, 8192):
        n = min(8192, pages - p)
        s["k"][p:p + n] = _pack(1.5 * dr(n, block, hkv, d) + common, (n, *shape))
        s["v"][p:p + n] = _pack(dr(n, block, hkv, d), (n, *shape))
    if kind == "load":
        first = np.minimum(c["first"], lens)
        s["t"] = int((lens - first).sum())
        s["cu"], s["first"] = _i32(np.concatenate([[0], np.cumsum(lens - first)])), _i32(first)
        return s
    hq = c["hq"]
    s["lens"], s["maxlen"], s["ctx"] = [int(n) for n in lens], int(lens.max()), _i32(lens)
    s["scale"] = 1.0 / math.sqrt(d)
    s["q"] = (1.5 * dr(len(lens), hq, d) + common).to(dt)
    s["slopes"] = s["prefix"] = None
    if c["bias"]:
        h = torch.arange(1, hq + 1, dtype=torch.float32, device=DEV)
        s["slopes"] = torch.exp2(-8.0 * h / hq) * (1.0 + 0.1 * dr(hq).abs())
    if c["prefix"]:
        s["prefix"] = _i32(np.minimum(rng.integers(0, c["prefix"], size=len(lens), endpoint=True), lens))
    if own:
        import paper_2608_13499_amd as ops
        s["scratch"] = torch.empty(ops.opscale_attn_decode_fp4_workspace_size(len(lens), hq, d, s["maxlen"]),
                                   dtype=torch.uint8, device=DEV)
    return s


def _kv(s):
    """K and V of the new tokens, as views."""
    hkv = s["c"]["hkv"]
    return s["kv"][:, :hkv], s["kv"][:, hkv:]


# -------------------------------------------------------------- plain forms --
def _plain_quantize(s):
    return _to_e4m3(s["x"].float())


def _plain_linear(s):
    c = s["c"]
    n, k = c["n"], c["k"]
    x = s["xq"].float() * s["xs"].t().repeat_interleave(BLOCK, 1)[:, :k]
    w = s["wq"].float() * s["ws"].repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
    y = torch.matmul(x, w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(_dtype(c))


def _plain_store(s):
    """The tokens' values as the cache holds them; the cache's bytes are written too, row by row."""
    c = s["c"]
    slots, block, d = s["slots"].long(), c["block"], c["d"]
    out = []
    for x, cache in zip(_kv(s), (s["k"], s["v"])):
        rows = _pack(x.float()[:, None], (len(slots), c["hkv"], d // 2 + d // GROUP))  # pages of one row
        flat = cache.view(cache.shape[0], c["hkv"], -1)
        page, row = slots // block, slots % block
        flat[:, :, :block * d // 2].unflatten(-1, (block, d // 2))[page, :, row] = rows[..., :d // 2]
        flat[:, :, block * d // 2:].unflatten(-1, (d // GROUP, block))[page, :, :, row] = rows[..., d // 2:]
        out.append(_unpack(rows[:, :, None], d, s["values"])[:, :, 0].to(_dtype(c)))
    return tuple(out)


def _plain_load(s):
    c, t = s["c"], torch.arange(s["t"], device=DEV)
    cu = s["cu"].long()
    b = torch.searchsorted(cu, t, right=True) - 1
    j = s["first"].long()[b] + t - cu[b]
    page, row = s["table"].long()[b, j // c["block"]], j % c["block"]
    out = []
    for cache in (s["k"], s["v"]):
        x = _unpack(cache, c["d"], s["values"])
        out.append(x[page, :, row].to(_dtype(c)))
    return tuple(out)


def _plain_decode(s):
    c = s["c"]
    q, (B, hq, d), hkv = s["q"].float(), s["q"].shape, c["hkv"]
    out = torch.empty_like(s["q"])
    rows = s["table"].shape[1] * c["block"]
    j = torch.arange(rows, device=DEV)
    step = max(1, (1 << 28) // (rows * hkv * d))  # sequences at a time
    for b0 in range(0, B, step):
        b = slice(b0, min(B, b0 + step))
        n = s["ctx"][b].long()[:, None]
        seen = j < n
        if c["window"]:
            seen = seen & (n - 1 - j < c["window"])
        if s["prefix"] is not None:
            seen = (seen | (j < s["prefix"][b].long()[:, None])) & (j < n)
        kk, vv = (_unpack(x[s["table"][b].long()], d, s["values"]).transpose(1, 2).reshape(-1, hkv, rows, d)
                  for x in (s["k"], s["v"]))
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
        return {"quantize": _plain_quantize, "linear": _plain_linear, "store": _plain_store, "load": _plain_load,
                "decode": _plain_decode}[kind](s)
    import paper_2608_13499_amd as ops
    if kind == "quantize":
        return ops.opscale_quantize_fp8(s["x"])
    if kind == "linear":
        return ops.opscale_linear_fp8(s["xq"], s["xs"], s["wq"], s["ws"], s["bias"], _dtype(c), workspace=s["scratch"])
    if kind == "store":
        k, v = _kv(s)
        ops.opscale_kv_write_fp4(k, v, s["k"], s["v"], s["slots"])
    if kind in ("store", "load"):
        return ops.opscale_kv_read_fp4(s["k"], s["v"], s["table"], s["cu"], s["t"], s["first"], _dtype(c))
    return ops.opscale_attn_decode_fp4(s["q"], s["k"], s["v"], s["table"], s["ctx"], s["maxlen"], s["scale"],
                                       softcap=c["cap"], slopes=s["slopes"], window=c["window"],
                                       prefix_lens=s["prefix"], workspace=s["scratch"])


# -------------------------------------------------------------------- work ---
def _seen_keys(c, lens):
    """Keys that the queries see, over the sequences, with the mean prefix (what the seed draws differs a little)."""
    far = np.maximum(0, lens - c["window"]) if c["window"] else np.zeros_like(lens)
    return int((lens - np.maximum(far - c["prefix"] // 2, 0)).sum())


def work(c):
    size = 2 if c["dt"] == BF16 else 4
    if c["kind"] == "quantize":
        m, k = c["m"], c["k"]
        return {"bytes": m * k * (size + 1) + 4 * m * _cdiv(k, BLOCK), "flops": 2 * m * k}
    if c["kind"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        scales = 4 * _cdiv(k, BLOCK) * (m + _cdiv(n, BLOCK))
        return {"bytes": m * k + n * k + size * m * n + scales + (size * n if c["bias"] else 0), "flops": 2 * m * n * k}
    lens = lengths(c)
    hkv, d = c["hkv"], c["d"]
    held = d // 2 + d // GROUP  # bytes of a row of a head in the cache
    if c["kind"] == "decode":
        keys, b = _seen_keys(c, lens), len(lens)
        return {"bytes": 2 * keys * hkv * held + 2 * size * b * c["hq"] * d + 4 * (keys // c["block"] + b),
                "flops": 4 * c["hq"] * d * keys}
    if c["kind"] == "store":  # rows read, written to the cache, read from it, written
        t = len(lens) if c["new"] == "one" else int(lens.sum())
        return {"bytes": 2 * t * hkv * (2 * size * d + 2 * held) + 8 * t, "flops": 6 * t * hkv * d}
    t = int((lens - np.minimum(c["first"], lens)).sum())
    return {"bytes": 2 * t * hkv * (size * d + held) + 4 * (t // c["block"] + 2 * len(lens)), "flops": 2 * t * hkv * d}


# ------------------------------------------------------------------- exact ---
def _exact_power(most, largest, lowest, highest):
    """2^e, e the least integer in [lowest, highest] with `most` <= largest * 2^e, or the highest."""
    p = torch.exp2(torch.arange(lowest, highest + 1, dtype=torch.float64, device=DEV))
    return p[torch.searchsorted(p * largest, most.contiguous()).clamp(max=len(p) - 1)]


def _exact_quantize(x):
    m, k = x.shape
    codes = torch.empty(m, k, dtype=torch.float64, device=DEV)
    scales = torch.empty(_cdiv(k, BLOCK), m, dtype=torch.float64, device=DEV)
    for i in range(len(scales)):
        at = slice(i * BLOCK, min(k, (i + 1) * BLOCK))
        b = x[:, at].double()
        scales[i] = _exact_power(b.abs().amax(1), 448.0, -100, 120)
        y = b / scales[i][:, None]
        # 3 bits behind the first one, whose place is 2^-6 at the least
        place = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        codes[:, at] = torch.round(y / place) * place
    return codes, scales


def _exact_cached(x):
    """What the cache holds for x [..., D]: the borders between e2m1 values counted."""
    g = x.double().unflatten(-1, (-1, GROUP))
    scale = _exact_power(g.abs().amax(-1), 7.0, -100, 125)[..., None]
    y = g.abs() / scale
    at = torch.zeros_like(g)
    for low, high, even in ((0, .5, 0), (.5, 1, 1), (1, 1.5, 0), (1.5, 2, 1), (2, 3, 0), (3, 4, 1), (4, 6, 0)):
        border = 0.5 * (low + high)
        at += ((y >= border) if even else (y > border)).double() * (high - low)
    return (torch.sign(g) * at * scale).flatten(-2)


def _exact_linear(c, s):
    y = torch.zeros(c["m"], c["n"], dtype=torch.float64, device=DEV)
    for i in range(_cdiv(c["k"], BLOCK)):
        at = slice(i * BLOCK, min(c["k"], (i + 1) * BLOCK))
        w = s["wq"][:, at].double() * s["ws"][:, i].double().repeat_interleave(BLOCK)[:c["n"], None]
        y += (s["xq"][:, at].double() @ w.t().contiguous()) * s["xs"][i].double()[:, None]
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_rows(cache, pages, d, first, n):
    """Rows first .. n - 1 in 64 bits of the keys on these pages, [hkv, n - first, d]."""
    p = cache[pages].flatten(2).to(torch.int64)  # page, head, byte
    block, row = cache.shape[2], torch.arange(d, device=DEV)
    key = torch.arange(first, n, device=DEV)
    page, at = (key // block)[:, None], (key % block)[:, None]
    nib = p[page, :, at * (d // 2) + row // 2] >> (4 * (row % 2))[:, None]  # key, element, head
    e = p[page, :, block * d // 2 + row // GROUP * block + at] - 127
    frac, exp = (nib & 1).double(), (nib >> 1) & 3
    size = torch.where(exp == 0, 0.5 * frac, torch.ldexp(1.0 + 0.5 * frac, exp - 1))
    return torch.ldexp(torch.where(nib & 8 != 0, -size, size), e).permute(2, 0, 1).contiguous()


def _exact_load(c, s):
    lens, first, parts = lengths(c), s["first"].tolist(), ([], [])
    for b, n in enumerate(int(n) for n in lens):
        pages = s["table"][b, :_cdiv(n, c["block"])].long()
        for part, cache in zip(parts, (s["k"], s["v"])):
            part.append(_exact_rows(cache, pages, c["d"], first[b], n))
    return tuple(torch.cat(p, 1).transpose(0, 1) for p in parts)


def _exact_decode(c, s):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    out = torch.zeros(len(s["lens"]), hkv, hq // hkv, d, dtype=torch.float64, device=DEV)
    slopes = torch.zeros(hq, dtype=torch.float64, device=DEV) if s["slopes"] is None else s["slopes"].double()
    for b, n in enumerate(s["lens"]):
        pages = s["table"][b, :_cdiv(n, c["block"])].long()
        k, v = (_exact_rows(x, pages, d, 0, n) for x in (s["k"], s["v"]))
        back = n - 1 - torch.arange(n, device=DEV)
        hidden = back >= (c["window"] or 1 << 40)
        if s["prefix"] is not None:
            hidden &= back <= n - 1 - s["prefix"][b]
        for g in range(hkv):
            qq = s["q"][b].view(hkv, hq // hkv, d)[g].double()
            sc = (qq @ k[g].t().contiguous()) * s["scale"]
            if c["cap"]:
                sc = torch.tanh(sc / c["cap"]) * c["cap"]
            sc = sc - slopes.view(hkv, -1)[g][:, None] * back.double()
            sc[:, hidden] = -torch.inf
            out[b, g] = torch.softmax(sc, -1) @ v[g]
    return out.view(-1, hq, d)


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "quantize":
        return _exact_quantize(s["x"])
    if c["kind"] == "linear":
        return _exact_linear(c, s)
    if c["kind"] == "store":
        return tuple(_exact_cached(x) for x in _kv(s))
    return _exact_load(c, s) if c["kind"] == "load" else _exact_decode(c, s)
