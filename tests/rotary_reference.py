"""Multi-axis rotary positions in 64 bits (numpy), written from the formula: test infrastructure."""
import numpy as np


def coordinates(dims, N, offset=0):
    return np.stack(np.unravel_index(np.arange(offset, offset + N), dims)).astype(np.int64)


def angles(positions, sections, base, per_axis_ladder):
    """positions [axes, B, N] -> angles [B, N, pairs], reduced modulo a turn in long double."""
    P = sum(sections)
    out = np.empty(positions.shape[1:] + (P,))
    turn = np.longdouble(2) * np.longdouble("3.14159265358979323846264338327950288")
    c = 0
    for a, size in enumerate(sections):
        for i in range(size):
            expo = np.longdouble(i) / size if per_axis_ladder else np.longdouble(c) / P
            freq = np.longdouble(base) ** -expo
            out[..., c] = np.fmod(positions[a].astype(np.longdouble) * freq, turn).astype(np.float64)
            c += 1
    return out


def rotate(x, ang, parts, interleaved, inverse=False):
    """x [B, heads, N, D] (float64) turned by ang [B, N, P]."""
    B, heads, N, D = x.shape
    P = ang.shape[-1]
    y = x.reshape(B, heads, N, parts, D // parts).copy()
    c, s = np.cos(ang)[:, None, :, None, :], np.sin(ang)[:, None, :, None, :] * (-1 if inverse else 1)
    i1, i2 = (np.arange(0, 2 * P, 2), np.arange(1, 2 * P, 2)) if interleaved else (np.arange(P), np.arange(P, 2 * P))
    x1, x2 = y[..., i1].copy(), y[..., i2].copy()
    y[..., i1] = x1 * c - x2 * s
    y[..., i2] = x2 * c + x1 * s
    return y.reshape(B, heads, N, D)


def tolerance(x, ref, P, parts, interleaved, bf16):
    """Per element.  fp32: sine and cosine are off by the angle's rounding (half a step of a 32-bit half-turn fraction,
    then of an fp32 number below 1: under 2^-23.3 in all) and the function's own error (2 ulp: 2^-23), together under
    4 * 2^-24; the two products and their sum add at most 2 * 2^-24 of |x1| + |x2|.  8 * 2^-24 covers that.  bf16 adds
    the final rounding, half a step: 2^-8 of the value."""
    B, heads, N, D = x.shape
    y = np.abs(x).reshape(B, heads, N, parts, D // parts)
    t = np.zeros_like(y)
    i1, i2 = (np.arange(0, 2 * P, 2), np.arange(1, 2 * P, 2)) if interleaved else (np.arange(P), np.arange(P, 2 * P))
    pair = y[..., i1] + y[..., i2]
    t[..., i1], t[..., i2] = pair, pair
    t = t.reshape(x.shape) * 8 * 2.0 ** -24
    return t + np.abs(ref) * 2.0 ** -8 if bf16 else t
