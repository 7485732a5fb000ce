"""The definitions of the 8-bit floating-point operators in 64 bits (numpy), for the tests."""
import numpy as np

E4M3 = np.array([(-1 if b & 128 else 1) * (np.ldexp(1 + (b & 7) / 8, (b >> 3 & 15) - 7) if b >> 3 & 15 else np.ldexp((b & 7) / 8, -6))
                 if b & 127 != 127 else np.nan for b in range(256)])
MAGNITUDES = E4M3[:127]


def up(f):
    return -(-f // 128) * 128


def blocks(x, block_rows):
    r, c = x.shape
    out = np.zeros((-(-r // block_rows) * block_rows, up(c)))
    out[:r, :c] = x
    return out.reshape(-1, block_rows, up(c) // 128, 128)


def quantize(x, block_rows):
    """(bytes of E4M3, bytes of E8M0): the nearest number by search, ties to the even code."""
    x = np.asarray(x, np.float64)
    b = blocks(x, block_rows)
    top = np.where(np.isfinite(b), np.abs(b), 0).max(axis=(1, 3))
    s = np.full(top.shape, 0)
    some = top > 0
    guess = np.frexp(top[some])[1] - 12
    while True:                                               # the smallest s with top <= 448 2^s
        more = top[some] > np.ldexp(448.0, guess)
        if not more.any():
            break
        guess = guess + more
    s[some] = np.maximum(guess, -126)
    y = np.ldexp(b, -s[:, None, :, None]).reshape(-1, b.shape[2] * 128)[: x.shape[0], : x.shape[1]]
    with np.errstate(invalid="ignore"):
        a = np.abs(y)
        hi = np.clip(np.searchsorted(MAGNITUDES, np.where(np.isfinite(a), a, 0)), 1, 126)
        below, above = a - MAGNITUDES[hi - 1], MAGNITUDES[hi] - a
        code = np.where(below < above, hi - 1, np.where(below > above, hi, hi - 1 + (hi - 1) % 2))
    code = np.where(np.signbit(y), code + 128, code)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8), (s + 127).astype(np.uint8)


def numbers(q, scale, block_rows):
    """What bytes stand for."""
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(int) - 127))
    return E4M3[q] * np.repeat(np.repeat(s, block_rows, 0)[: q.shape[0]], 128, 1)[:, : q.shape[1]]


def act(g, kind):
    """(activation, slope); kind 0: SiLU, 1: GELU in tanh form."""
    if kind == 0:
        p = 1 / (1 + np.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    c = np.sqrt(2 / np.pi)
    t = np.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
