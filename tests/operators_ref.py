"""Plain evaluations of the rotary positions and of attention over rows held in 8 bits, in 64 bits (angles in 80), written
from the definitions in include/videoscan.h."""
import numpy as np


def quantise(x):
    """[..., 128] fp64 -> (whole numbers, scales [..., 1])."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(np.abs(x).max(-1, keepdims=True) / 127.0)
    s = np.maximum(np.ldexp(np.ceil(m * 256.0), e - 8), 2.0 ** -126)
    return np.rint(x / s), s


def stands_for(x):
    q, s = quantise(x)
    return q * s


def attend(q, k, v, seen, scale):
    """q [T][Hq][D] over k, v [L][Hkv][D], token t over the first seen[t] rows.  Returns out, sum p |v| and sum p max_j |v_j| (the last
    for every value of a row)."""
    T, hq, d = q.shape
    g = hq // k.shape[1]
    out, absolute, most = (np.zeros((T, hq, d)) for _ in range(3))
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        for t in range(T):
            n = seen[t]
            z = kh[:n] @ q[t, h] * scale
            w = np.exp(z - z.max())
            w /= w.sum()
            out[t, h], absolute[t, h], most[t, h] = w @ vh[:n], w @ np.abs(vh[:n]), w @ np.abs(vh[:n]).max(-1)
    return out, absolute, most


def decode_bound(q, k, v, ref, absolute, most, scale):
    """How far a value of a decoding step over rows in 8 bits may be off, q [Hq][D], k [L][Hkv][D] (what the rows stand for), v likewise.
    * sums of (code + 1152) q over 128 dims in fp32 that start at -1152 sum q: what has come together is at most 1280 sum|q| s, s at most
      max|k| / 126, and rounded to 2^-24 of that by each of 16 additions of eight products and what they start at: a score at most
      e = 2^-24 17 (1280 / 126) sum|q| max|k| scale < 2^-16.5 of the rest (the query in fp16 gives up 2^-39 of its largest entry, far
      less), and four roundings and the exponential of fp32 2^-21 of itself; a weight then by a factor of exp(2 e) at most, on top
      and below the fraction; and whatever the weights are, they are fractions of one: no value leaves the range of the keys' values, so it is
      at most twice the largest of their magnitudes off (which is less where scores are large: e grows with them);
    * a probability below 2^-126 may be 0 in fp32, beside a sum of at least 1 (the reference never passes the largest score): at most
      2^-126 of a key's value;
    * p times the scale of V in bf16: 2^-8 of every term; the output in bf16: 2^-8 of itself;
    * sums of p s (code + 128), up to 255 p s each where max|v| is over 126 / 127 * 127 p s: an fp32 rounding per 32 keys of what
      has come together (2^-24 of at most 2.02 * 2 sum p max|v|), and as many for what is taken off."""
    g = q.shape[0] // k.shape[1]
    z = np.abs(q).sum(-1) * np.repeat(np.abs(k).max((0, 2)), g) * scale  # [Hq]
    e = 2.0 ** -16.5 * z + 2.0 ** -21 * (z + 1.0)
    with np.errstate(over="ignore", invalid="ignore"):
        weights = np.fmin(np.expm1(2.0 * e)[:, None] * 1.01 * absolute, 2.0 * np.repeat(np.abs(v).max(0), g, 0))
    steps = k.shape[0] // 32 + 8
    return 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * 1.01 * absolute + weights + 2.0 ** -24 * steps * 8.1 * most + 2.0 ** -126 * np.repeat(np.abs(v).sum(0), g, 0)


def prefill_bound(q, k, v, ref, absolute, most, scale):
    """The same for a token of a prefill, q [Hq][D], k and v its rows: on top of decode_bound
    * partial results of splits are fp16, scaled so that the largest of 32 dims is in [2^14, 2^15): 2^-11 of a value, or 2^-25 where it is under
      2^-14, 2^-39 of the largest; weighted by the splits' shares, 2^-11 of the terms' magnitudes and 2^-39 of the rows' largest;
    * weights in fp16 instead of bf16: 2^-11 of a term (decode_bound has 2^-8), but 2^-25 under 2^-14, where the largest weight is at least 2^6
      when the reference is set and the reference only goes up: 2^-31 of a row of its size, for each key;
    * their sums go up to 1279 and back by 1152 a unit of weight, where a row's largest code is 126 at least: a rounding of 2^-24 of 2431 / 126 = 19.3
      instead of 8.1 of the rows' largest, per 32 keys;
    * a product of a probability and a scale of V that is under 2^-126 may be 0, beside a sum of at least 1: 2^-126 of a key's whole number, which is
      at most 127 (decode_bound has 2^-126 of the value, which for scales under 1 is less)."""
    n = k.shape[0]
    return decode_bound(q, k, v, ref, absolute, most, scale) + 2.0 ** -11 * 1.01 * absolute + (2.0 ** -39 + 2.0 ** -31 * n + 2.0 ** -24 * (n // 32 + 8) * 11.2) * most + 2.0 ** -126 * 127 * n


def rotate(x, positions, sections, theta, halves, inverse=False):
    """x [T][H][D] fp64, positions [3][T]."""
    n = sum(sections)
    axis = np.repeat(np.arange(3), sections)
    rate = np.power(np.longdouble(theta), -np.arange(n, dtype=np.longdouble) / n)
    angle = positions.astype(np.longdouble)[axis].T * rate              # [T][n]
    c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
    s = -s if inverse else s
    y = x.copy()
    a, b = (slice(0, n), slice(n, 2 * n)) if halves else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y
