"""Block-scaled 8-bit floats, the norm in them, their products and the layer of experts in them, in float64 from the definitions.

A block is 128 elements along the last axis, or 128 rows of 128 elements (block_rows 128); its scale is the smallest power of two, at
least 2^-127, of which its largest magnitude is at most 448 times; a block that is not finite is NaN."""
import numpy as np

BLOCK, MOST = 128, 448.0
STEP = 2.0 ** -23          # of a sum in fp32, by its magnitude
# magnitudes of the codes 0 .. 126, ascending (127 is NaN): exponent field c // 8, fraction c % 8
E4M3 = np.array([(c % 8) * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])


def _blocks(x, block_rows):
    """[.., n, K] -> [.., n', r, K', 128], zeros behind n and K."""
    n, K = x.shape[-2:]
    pad = [(0, 0)] * (x.ndim - 2) + [(0, -n % block_rows), (0, -K % BLOCK)]
    p = np.pad(np.asarray(x, dtype=np.float64), pad)
    return p.reshape(*p.shape[:-2], p.shape[-2] // block_rows, block_rows, p.shape[-1] // BLOCK, BLOCK)


def _per_row(s, n):
    """[.., n', r, K', 1] -> [.., n, K']"""
    return s.reshape(*s.shape[:-4], -1, s.shape[-2])[..., :n, :]


def scale_bytes(x, block_rows=1):
    """[.., n, K] -> [.., n, K']"""
    b = np.abs(_blocks(x, block_rows))
    bad = ~np.isfinite(b).all((-1, -3), keepdims=True)
    amax = np.where(np.isfinite(b), b, 0.0).max((-1, -3), keepdims=True)
    m, e = np.frexp(amax / MOST)                         # (a quotient that rounds to a power of two: checked below)
    e = np.where(m == 0.5, e - 1, e)
    e = np.where(amax > np.ldexp(MOST, e), e + 1, e)
    e = np.where(amax <= np.ldexp(MOST, e - 1), e - 1, e)
    byte = np.where(bad, 255, np.where(amax > 0, np.maximum(e + 127, 0), 0))
    byte = np.broadcast_to(byte, (*b.shape[:-1], 1))
    return _per_row(byte, x.shape[-2]).astype(np.int64)


def codes(x, byte):
    """Codes 0..255 [.., n, K] for given scales [.., n, K']: the nearest magnitude, the even code of two equally near ones."""
    at = np.arange(x.shape[-1]) // BLOCK
    s = byte[..., at]
    v = np.where(s == 255, 0.0, np.asarray(x, dtype=np.float64)) / np.ldexp(1.0, np.where(s == 255, 127, s) - 127)
    a = np.minimum(np.abs(v), MOST)
    hi = np.minimum(np.searchsorted(E4M3, a), 126)        # the first that is not below
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return c + 128 * (np.signbit(v) & (s != 255))


def values(c, byte):
    mag = np.where(c & 127 == 127, np.nan, E4M3[np.minimum(c & 127, 126)]) * np.where(c & 128, -1.0, 1.0)
    s = byte[..., np.arange(c.shape[-1]) // BLOCK]
    return mag * np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))


def rounded(x, block_rows=1):
    b = scale_bytes(x, block_rows)
    return values(codes(x, b), b)


def pack(c, byte):
    """Bytes as the library lays them out."""
    last = [(0, 0)] * (c.ndim - 1)
    padded = np.pad(c, last + [(0, -c.shape[-1] % BLOCK)]), np.pad(byte, last + [(0, -byte.shape[-1] % 16)])
    return tuple(np.ascontiguousarray(v, dtype=np.uint8) for v in padded)


def near(x, err):
    """How far the rounding of values within err of x can be from that of x: it is monotone for each scale, and the scale is one of
    those of the block's largest magnitude, less and plus err."""
    far, exact = np.zeros_like(x), rounded(x)
    for s in (scale_bytes(np.maximum(np.abs(x) - err, 0.0)), scale_bytes(np.abs(x) + err)):
        for v in (x - err, x + err):
            far = np.maximum(far, np.abs(values(codes(v, s), s) - exact))
    return far


def rmsnorm(total, gain, eps):
    """(xn, rstd) of the rows of the rounded sum."""
    v = np.asarray(total, dtype=np.float64)
    rstd = 1.0 / np.sqrt((v * v).mean(-1) + eps)
    return np.asarray(gain, dtype=np.float64) * v * rstd[:, None], rstd


def sums_error(a, b, exact=False):
    """How far a b^T may be off.  The sums are in fp32: a rounding for every 128 products (exact: 32 of them), and for the partial sums of up
    to 24 pieces.  Unless `exact` (results in fp32, whose codes are multiplied as bf16 values), the 8-bit matrix instruction first brings 8
    neighbouring products to the exponent of the largest, ea + eb <= log2 |a b|, and drops their bits from 2^-14 of that on: 2^-13 of the
    group's largest product at most for each of the 7 others; the largest itself has 6 bits of fraction and keeps them.  The largest
    product of a group is at most the product of the largest factors."""
    err = (a.shape[-1] / (32 if exact else BLOCK) + 24) * STEP * (np.abs(a) @ np.abs(b).T)
    if not exact:
        most = [np.pad(np.abs(v), [(0, 0), (0, -v.shape[-1] % 8)]).reshape(v.shape[0], -1, 8).max(-1) for v in (a, b)]
        err += 7 * 2.0 ** -13 * (most[0] @ most[1].T)
    return err


def ff_forward(x, W1, W3, W2, topk_idx, gates, inv_pos=None, residual=None, small=False):
    """(out, bound) of the layer.  x [T,d], W1, W3 [E,f,d] and W2 [E,d,f]: the values that the 8 bits stand for.  bound: how far the layer may
    be off whose products sum in fp32, whose activations may therefore fall on the other side of a rounding, and which rounds an
    expert's output and the result to bf16; small: whose activations are of exact products and whose experts' outputs stay in fp32."""
    T, d = x.shape
    out = np.zeros((T, d)) if residual is None else np.asarray(residual, dtype=np.float64).copy()
    bound, mag = np.zeros((T, d)), np.abs(out)
    for e in range(W1.shape[0]):
        t, j = np.nonzero((topk_idx == e) & (True if inv_pos is None else inv_pos >= 0))
        if t.size == 0:
            continue
        g, xs = np.asarray(gates, dtype=np.float64)[t, j][:, None], x[t]
        h1, h3, e1, e3 = xs @ W1[e].T, xs @ W3[e].T, sums_error(xs, W1[e], small), sums_error(xs, W3[e], small)
        with np.errstate(over="ignore"):
            silu = h1 / (1.0 + np.exp(-h1))
        act = silu * h3
        # |silu'| <= 1.1; the sigmoid in fp32 is 2 + |h1| steps off
        ea = (1.1 * e1 + (4 + np.abs(h1)) * STEP * np.abs(silu)) * (np.abs(h3) + e3) + np.abs(silu) * e3 + 2 * STEP * np.abs(act)
        aq, far = rounded(act), near(act, ea)
        y = aq @ W2[e].T
        ey = far @ np.abs(W2[e]).T + sums_error(np.abs(aq) + far, W2[e])
        if not small:
            ey += 2.0 ** -8 * (np.abs(y) + ey)
        np.add.at(out, t, g * y)
        np.add.at(bound, t, np.abs(g) * ey)
        np.add.at(mag, t, np.abs(g) * (np.abs(y) + ey))
    bound += (topk_idx.shape[1] + 1) * STEP * mag
    return out, bound + 2.0 ** -8 * (np.abs(out) + bound)
