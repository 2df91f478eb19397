"""Pins of oracle.step: values worked by hand, closed forms and the plain operators
they reduce to, each with a planted mistake that the pin has to catch."""
import math

import numpy as np
import pytest

import oracle
from oracle import step


# ------------------------------------------------------ rotation and norm ---
def test_frequencies_by_hand():
    # rot 4, base 100: f = 1, 0.1; over 63 tokens they turn 10.03 and 1.003 times
    f, m = step.rope_frequencies(4, 100.0)
    assert np.allclose(f, [1.0, 0.1]) and m == 1.0
    f, _ = step.rope_frequencies(4, 100.0, "linear", 4.0)
    assert np.allclose(f, [0.25, 0.025])
    turns = 63 * 0.1 / (2 * math.pi)
    f, m = step.rope_frequencies(4, 100.0, "bands", 4.0, 0.5, 8.0, 63)
    kept = (turns - 0.5) / 7.5
    assert np.allclose(f, [1.0, 0.1 * (kept + (1 - kept) / 4)]) and m == 1.0
    # ramp, from the pair that turns 8 times (index 0.098 -> 0) to the one that turns 0.5 times (1.30 -> 2)
    f, m = step.rope_frequencies(4, 100.0, "ramp", 4.0, 0.5, 8.0, 63)
    assert np.allclose(f, [1.0, 0.1 * (0.5 + 0.5 / 4)]) and math.isclose(m, 1 + 0.1 * math.log(4))


def test_turned_pairs_keep_length_and_relative_angle():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 8))
    f, _ = step.rope_frequencies(4, 50.0)
    for inter in (False, True):
        y = step.qk_norm_rope(x, None, 0.0, [0, 5, 9], f, inter)
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 4:], x[..., 4:])
        pairs = [(0, 1), (2, 3)] if inter else [(0, 2), (1, 3)]
        for i, (a, b) in enumerate(pairs):
            z0, z1 = x[1, 0, a] + 1j * x[1, 0, b], y[1, 0, a] + 1j * y[1, 0, b]
            assert np.isclose(z1, z0 * np.exp(1j * 5 * f[i]))
    # the half layout over the whole head is the plain rotary embedding
    f, _ = step.rope_frequencies(8, 10000.0)
    assert np.allclose(step.qk_norm_rope(x, None, 0.0, [1, 2, 3], f, False), oracle.rope(x, np.array([1, 2, 3]), 1e4))
    assert not np.allclose(step.qk_norm_rope(x, None, 0.0, [1, 2, 3], f, True), oracle.rope(x, np.array([1, 2, 3]), 1e4))


def test_head_norm_is_rmsnorm_of_each_head():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((4, 3, 16)), rng.standard_normal(16)
    y = step.qk_norm_rope(x, w, 1e-3, None, None, False)
    assert np.allclose(y.reshape(12, 16), oracle.rmsnorm(x.reshape(12, 16), w, 1e-3))


# ------------------------------------------------------------- step tables --
def test_tables_by_hand():
    # pages of 4: request 0 has 3 tokens and brings 3 (one slot left, one new page), request 1 brings none,
    # request 2 starts with 5 (two pages)
    table = [[7, -1, -1], [8, 9, -1], [-1, -1, -1]]
    cu, pos, slots, kv, nxt, t = step.block_tables([3, 8, 0], [3, 0, 5], table, [90, 91, 92, 93], 1, 4, 10)
    assert cu == [0, 3, 3, 8] and kv == [6, 8, 5] and nxt == 4
    assert pos == [3, 4, 5, 0, 1, 2, 3, 4, 0, 0]
    assert slots == [31, 364, 365, 368, 369, 370, 371, 372, -1, -1]
    assert t.tolist() == [[7, 91, -1], [8, 9, -1], [92, 93, -1]]
    # six tokens fit: request 2 gets three of its five and one page
    cu, pos, slots, kv, nxt, t = step.block_tables([3, 8, 0], [3, 0, 5], table, [90, 91, 92, 93], 1, 4, 6)
    assert cu == [0, 3, 3, 6] and kv == [6, 8, 3] and nxt == 3 and t[2].tolist() == [92, -1, -1]
    # the free list is one page short; then rows of one page
    cu, pos, slots, kv, nxt, t = step.block_tables([3, 8, 0], [3, 0, 5], table, [90, 91, 92], 1, 4, 10)
    assert nxt == 4 and t[2].tolist() == [92, -1, -1] and slots[7] == -1 and slots[6] == 371
    cu, pos, slots, kv, nxt, t = step.block_tables([3], [3], [[7]], [90], 0, 4, 3)
    assert slots == [31, -1, -1] and kv == [4] and nxt == 0 and pos == [3, 4, 5]


# ---------------------------------------------- attention with modifiers ----
def test_visible_by_hand():
    def see(*a):
        return step.visible(*a).tolist()

    assert see(3, 6, True, 0, 0, 0) == [0, 1, 2, 3]
    assert see(3, 6, False, 0, 0, 0) == [0, 1, 2, 3, 4, 5]
    assert see(3, 6, True, 2, 0, 0) == [2, 3]
    assert see(3, 6, False, 2, 0, 0) == [2, 3, 4]
    assert see(3, 6, True, 2, 1, 0) == [0, 2, 3]
    assert see(1, 6, True, 0, 4, 0) == [0, 1, 2, 3]        # the prefix is seen ahead too
    assert see(4, 6, True, 0, 0, 3) == [3, 4]
    assert see(4, 6, True, 0, 0, 6) == []                  # padding
    assert see(4, 6, True, 0, 2, 6) == [0, 1]


def _qkv(seed, T, Hq, Hkv, D):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((T, h, D)) for h in (Hq, Hkv, Hkv))


def test_without_modifiers_it_is_plain_attention():
    q, k, v = _qkv(2, 11, 4, 2, 8)
    cu = [0, 4, 4, 11]
    for causal in (True, False):
        assert np.allclose(step.attn_prefill_mod(q, k, v, cu, 0.3, causal), oracle.attn_prefill(q, k, v, cu, 0.3, causal))
    # a document mask is a ragged batch of the documents
    starts = [0, 1, 2, 3, 0, 0, 0, 3, 3, 5, 5]
    got = step.attn_prefill_mod(q, k, v, cu, 0.3, doc_starts=starts)
    ref = oracle.attn_prefill(q, k, v, [0, 1, 2, 3, 4, 7, 9, 11], 0.3, True)
    assert np.allclose(got, ref)
    assert not np.allclose(got, oracle.attn_prefill(q, k, v, cu, 0.3, True))


def test_modifiers_by_hand():
    # one query, keys giving s = 2 and -1 (D = 1, scale 1); values 1 and 0: the first one's probability
    k = np.array([[[2.0]], [[-1.0]]])
    v = np.array([[[1.0]], [[0.0]]])
    q = np.array([[[0.0]], [[1.0]]])

    def p(**kw):
        return step.attn_prefill_mod(q, k, v, [0, 2], 1.0, **kw)[1, 0, 0]

    def logistic(d):
        return 1 / (1 + math.exp(-d))

    assert math.isclose(p(), logistic(3.0))
    assert math.isclose(p(softcap=1.5), logistic(1.5 * (math.tanh(2 / 1.5) + math.tanh(1 / 1.5))))
    assert math.isclose(p(slopes=[0.25]), logistic(3.0 - 0.25))
    assert math.isclose(p(softcap=1.5, slopes=[0.25]), logistic(1.5 * (math.tanh(2 / 1.5) + math.tanh(1 / 1.5)) - 0.25))
    assert p(window=1) == 0.0 and p(doc_starts=[0, 2]) == 0.0
    # ahead in a prefix the distance counts as well
    ahead = step.attn_prefill_mod(q[::-1], k, v, [0, 2], 1.0, slopes=[0.25], prefix_lens=[2])[0, 0, 0]
    assert math.isclose(ahead, logistic(3.0 + 0.25))


@pytest.mark.parametrize("n", [1, 5, 8])
def test_decode_is_the_last_row_of_prefill(n):
    rng = np.random.default_rng(3)
    q, k, v = _qkv(4, n, 4, 2, 8)
    table = np.array([[2, 0]])
    kc, vc = np.zeros((3, 4, 2, 8)), np.zeros((3, 4, 2, 8))
    for j in range(n):
        kc[table[0, j // 4], j % 4], vc[table[0, j // 4], j % 4] = k[j], v[j]
    slopes = rng.random(4)
    for kw in (dict(), dict(softcap=2.0), dict(slopes=slopes), dict(window=3), dict(window=2, prefix_lens=[2]),
               dict(prefix_lens=[1], doc_starts=[n])):
        pre = dict(kw, doc_starts=[n] * n) if "doc_starts" in kw else kw
        got = step.attn_decode_mod(q[-1:], kc, vc, table, [n], 0.5, **kw)
        assert np.allclose(got, step.attn_prefill_mod(q, k, v, [0, n], 0.5, **pre)[-1:]), kw
    # a page that is not there takes its keys away
    if n > 4:
        gone = step.attn_decode_mod(q[-1:], kc, vc, np.array([[2, 3]]), [n], 0.5)
        assert np.allclose(gone, step.attn_decode_mod(q[-1:], kc, vc, table, [4], 0.5))
