"""What attention with score modifiers may be off by, element by element.

A row's output is o = sum w_j v_j / sum w_j over the keys it sees (w = e^s), and a
relative error d_j of w_j moves it by sum p_j d_j (v_j - o), p = w / sum w: nothing
where all v_j are equal.  In u = 2^-24, half a step of fp32:

  * scale q . k is a sum of D products, D roundings of partial sums.  Products of
    independent signs reach about sqrt(D) of their size: a partial sum lies within
    3 r + |x|, r = scale sqrt(sum (q_d k_d)^2), x the score.  A rounding is off by
    u / sqrt(3) of that (rms), D of them by sqrt(D) as much; six times that is
    3.5 sqrt(D) u (3 r + |x|), independent from key to key, so that the keys' shares add
    up as squares.
  * the same way for all keys (a constant's rounding): the factor scale, the units of the
    exponential, the cap, the bias, eight roundings of |x| + slope |i - j| and, with a
    cap, ten of the capped score (its polynomial's 5.5e-7 is 9.2 u); four of the exponential.
  * the sums over n keys, n roundings of partial sums of at most A = sum p |v|, six times
    their rms: 3.5 sqrt(n) u A, and as much of |o| for sum w; four more for the merge.
  * bf16: w_j for its product with V in one piece, the same in sum w (2^-8, half a step of
    bf16: 2^-8 sum p |v - o|), or in two (2^-16 sum p |v|, the sum unrounded); the result
    2^-8 |o|.  fp32: the result u |o|.
"""
import numpy as np

U = 2.0 ** -24


def row(q, k, v, i, keys, scale, softcap=0.0, slope=0.0, dtype="f32", pieces=1):
    """(output, bound) of one query q [D] at position i over the keys at positions
    `keys`, k and v [len(keys), D], all float64."""
    D, n = q.shape[-1], len(keys)
    if n == 0:
        return np.zeros(D), np.zeros(D)
    x = scale * (k @ q)
    r = scale * np.sqrt((k * k) @ (q * q))
    s = softcap * np.tanh(x / softcap) if softcap else x
    far = slope * np.abs(i - np.asarray(keys, np.float64))
    w = np.exp(s - far - (s - far).max())
    p = w / w.sum()
    o = p @ v
    dev, mass = np.abs(v - o), p @ np.abs(v)
    scattered = 3.5 * np.sqrt(D) * U * (3 * r + np.abs(x))
    common = U * (8 * (np.abs(x) + np.abs(far)) + (10 * np.abs(s) if softcap else 0.0) + 4)
    bound = np.sqrt((p * scattered) ** 2 @ dev ** 2) + (p * common) @ dev
    bound = bound + U * (3.5 * np.sqrt(n) + 4) * (mass + np.abs(o))
    if dtype == "bf16":
        bound = bound + (2.0 ** -8 * (p @ dev) if pieces == 1 else 2.0 ** -16 * mass) + 2.0 ** -8 * np.abs(o)
    else:
        bound = bound + U * np.abs(o)
    return o, bound + 1e-30


def cut(a, bits):
    """a rounded to `bits` bits of mantissa (the leading one counted)."""
    m, e = np.frexp(np.asarray(a, np.float64))
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)
