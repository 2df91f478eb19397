"""The bounds of attn_error, checked on the CPU: they hold for a plain computation in
fp32, and operands or probabilities with some bits fewer exceed them."""
import numpy as np
import pytest

from attn_error import cut, row
from oracle import step

D, N = 128, 150


def _inputs(seed, std=1.5):
    rng = np.random.default_rng(seed)
    q, k = (np.float64(np.float32(std * rng.standard_normal(s))) for s in ((24, D), (N, D)))
    return q, k, np.float64(np.float32(rng.standard_normal((N, D))))


def _fp32(q, k, v, keys, scale, softcap, slope, i):
    """One row in fp32 throughout, sums in order."""
    f = np.float32
    x = np.array([f(scale) * np.add.accumulate(f(q) * f(kk), dtype=f)[-1] for kk in k], f)
    s = f(softcap) * np.tanh(x / f(softcap)) if softcap else x
    s = s - f(slope) * f(np.abs(i - keys))
    w = np.exp(s - s.max(), dtype=f)
    o = np.add.accumulate(w[:, None] * f(v), axis=0, dtype=f)[-1]
    return np.float64(o / np.add.accumulate(w, dtype=f)[-1])


RULES = [dict(), dict(softcap=5.0), dict(softcap=50.0), dict(slope=0.1)]


def _worst(change, rule, seed=3):
    """The largest share of the bound that `change` of (q, k, v) uses up over 24 rows."""
    q, k, v = _inputs(seed)
    worst = 0.0
    for i in range(24):
        n = 6 * (i + 1)
        keys, scale = np.arange(n), 1 / np.sqrt(D)
        o, bound = row(q[i], k[:n], v[:n], n - 1, keys, scale, **rule)
        got = change(q[i], k[:n], v[:n], keys, scale, n - 1, rule)
        worst = max(worst, float((np.abs(got - o) / bound).max()))
    return worst


@pytest.mark.parametrize("rule", RULES)
def test_the_rows_are_the_oracle_s(rule):
    q, k, v = _inputs(4)
    for n in (1, 7, 150):
        o, _ = row(q[0], k[:n], v[:n], n - 1, np.arange(n), 0.09, **rule)
        ref = step._row(q[0], k[:n], v[:n], 0.09, n - 1, np.arange(n), rule.get("softcap", 0.0), rule.get("slope", 0.0))
        np.testing.assert_allclose(o, ref, rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("rule", RULES)
def test_fp32_is_within(rule):
    assert _worst(lambda q, k, v, keys, scale, i, r: _fp32(q, k, v, keys, scale, r.get("softcap", 0.0),
                                                           r.get("slope", 0.0), i), rule) < 1.0


@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("bits", [(14, 14, 14), (14, 24, 24), (24, 14, 24), (24, 24, 15)])
def test_fewer_bits_are_not(rule, bits):
    def change(q, k, v, keys, scale, i, r):
        q, k, v = (cut(a, b) for a, b in zip((q, k, v), bits))
        return row(q, k, v, i, keys, scale, **r)[0]

    assert _worst(change, rule) > 1.0


@pytest.mark.parametrize("bits", [8, 12, 15])
def test_rounded_probabilities_are_not(bits):
    """Probabilities cut for V, and not for their sum."""
    def change(q, k, v, keys, scale, i, r):
        s = scale * (k @ q)
        w = np.exp(s - s.max())
        return cut(w, bits) @ v / w.sum()

    assert _worst(change, {}) > 1.0
