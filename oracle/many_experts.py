"""Plain float64 oracle of routing from logits for many experts, of microscaled 4-bit floats and of the layer of 4-bit
experts, written from their definitions: loops and numpy, no grouping, no tiling.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


# ---- routing -------------------------------------------------------------------------------------------------


def clean_logits(logits):
    l = np.asarray(logits, dtype=np.float64).copy()
    l[np.isnan(l)] = -np.inf
    l[l == np.inf] = np.float64(np.float32(3.402823e38))
    return l


def scores(logits, score):
    l = clean_logits(logits)
    with np.errstate(over="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-l))
        s = np.zeros_like(l)
        for t in range(l.shape[0]):
            m = l[t].max()
            if m > -np.inf:
                z = np.exp(l[t] - m)
                s[t] = z / z.sum()
        return s


def _first_largest(values, n):
    """Indices of the n largest, one after another, the lowest of equal ones."""
    left = list(range(len(values)))
    out = []
    for _ in range(n):
        best = left[0]
        for i in left[1:]:
            if values[i] > values[best]:
                best = i
        out.append(best)
        left.remove(best)
    return out


def group_route(logits, k, score="sigmoid", bias=None, n_groups=1, topk_groups=1, group_score="top2", renorm=True, scale=1.0):
    s = scores(logits, score)
    T, E = s.shape
    v = s + (np.asarray(bias, dtype=np.float64) if bias is not None else 0.0)
    v[np.isneginf(clean_logits(logits))] = -np.inf
    v[np.isnan(v)] = -np.inf
    per = E // n_groups
    idx = np.zeros((T, k), dtype=np.int64)
    for t in range(T):
        allowed = list(range(E))
        if n_groups > 1:
            value = []
            for g in range(n_groups):
                best = sorted(v[t, g * per:(g + 1) * per], reverse=True)
                total = best[0]
                if group_score == "top2" and per > 1 and best[1] > -np.inf:
                    total = best[0] + best[1]
                value.append(total)
            kept = set(_first_largest(value, topk_groups))
            allowed = [e for e in range(E) if e // per in kept]
        idx[t] = [allowed[i] for i in _first_largest([v[t, e] for e in allowed], k)]
    w = np.take_along_axis(s, idx, 1)
    gates = scale * (w / (w.sum(1, keepdims=True) + 1e-20) if renorm else w)
    counts = np.zeros(E, dtype=np.int64)
    groups = [[] for _ in range(E)]
    for t in range(T):
        for j in range(k):
            groups[idx[t, j]].append(t * k + j)
            counts[idx[t, j]] += 1
    perm = np.array([p for g in groups for p in g], dtype=np.int64)
    inv = np.empty(T * k, dtype=np.int64)
    inv[perm] = np.arange(T * k)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    return dict(topk_idx=idx, gates=gates, scores=s, counts=counts, offsets=offsets, perm=perm, inv_pos=inv.reshape(T, k))


def group_route_backward(logits, topk_idx, dgates, score="sigmoid", renorm=True, scale=1.0, dscores=None):
    l, s = clean_logits(logits), scores(logits, score)
    T, E = s.shape
    dl = np.zeros((T, E))
    for t in range(T):
        w = s[t, topk_idx[t]]
        z = w.sum() + 1e-20
        if renorm:   # g_j = scale w_j / z
            dw = np.array([sum(dgates[t, j] * scale * ((i == j) / z - w[j] / z ** 2) for j in range(len(w))) for i in range(len(w))])
        else:
            dw = scale * np.asarray(dgates[t], dtype=np.float64)
        ds = np.zeros(E) if dscores is None else np.asarray(dscores[t], dtype=np.float64).copy()
        for i, e in enumerate(topk_idx[t]):
            ds[e] += dw[i]
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                dl[t] = ds * s[t] * (1.0 / (1.0 + np.exp(l[t])))
        else:
            dl[t] = s[t] * (ds - (ds * s[t]).sum())
    return dl


# ---- microscaled 4-bit floats ---------------------------------------------------------------------------------


def mx4_scale_bytes(x):
    """[.., K] -> [.., K/32]: floor(log2(largest magnitude)) - 2 + 127, at least 0; 255 where a block is not finite."""
    b = np.abs(np.asarray(x, dtype=np.float64)).reshape(*x.shape[:-1], -1, BLOCK)
    bad = ~np.isfinite(b).all(-1)
    amax = np.where(bad, 1.0, np.where(np.isfinite(b), b, 0.0).max(-1))
    exponent = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 1, -10000)
    return np.where(bad, 255, np.maximum(exponent - 2 + 127, 0)).astype(np.int64)


def mx4_codes(x, scale_bytes):
    """Codes 0..15 of [.., K] for given scales: the nearest magnitude, the even code of two equally near ones."""
    v = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, BLOCK)
    bad = (scale_bytes == 255)[..., None]
    v = np.where(bad, 0.0, v) / np.ldexp(1.0, np.where(scale_bytes == 255, 127, scale_bytes) - 127)[..., None]
    dist = np.abs(np.minimum(np.abs(v), 6.0)[..., None] - E2M1)
    near = dist.min(-1, keepdims=True)
    candidates = np.where(dist == near, np.arange(8), 99)
    even = np.where((dist == near) & (np.arange(8) % 2 == 0), np.arange(8), 99).min(-1)
    code = np.where(even < 99, even, candidates.min(-1))
    return (code + 8 * np.signbit(v) * ~bad).astype(np.int64).reshape(x.shape)


def mx4_values(codes, scale_bytes):
    mag = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(scale_bytes == 255, np.nan, np.ldexp(1.0, scale_bytes - 127))
    return (mag.reshape(*scale_bytes.shape, BLOCK) * scale[..., None]).reshape(codes.shape)


def mx4_round(x):
    b = mx4_scale_bytes(x)
    return mx4_values(mx4_codes(x, b), b)


def mx4_pack(codes, scale_bytes):
    """Bytes as the library lays them out."""
    lo, hi = codes[..., 0::2], codes[..., 1::2]
    pad = -scale_bytes.shape[-1] % 16
    return (lo | hi << 4).astype(np.uint8), np.pad(scale_bytes, [(0, 0)] * (scale_bytes.ndim - 1) + [(0, pad)]).astype(np.uint8)


def mx4_near(act, err):
    """How far MXFP4 rounding of a value within err of act can be from that of act: the rounding is monotone for each scale, and the
    scale is one of those of the block's largest magnitude, less and plus err."""
    b = act.reshape(*act.shape[:-1], -1, BLOCK)
    e = err.reshape(b.shape)
    lo = mx4_scale_bytes((np.maximum(np.abs(b) - e, 0.0)).reshape(act.shape))
    hi = mx4_scale_bytes((np.abs(b) + e).reshape(act.shape))
    exact = mx4_round(act)
    far = np.zeros_like(act)
    for scale in (lo, hi):
        for v in (act - err, act + err):
            far = np.maximum(far, np.abs(mx4_values(mx4_codes(v, scale), scale) - exact))
    return far


# ---- the layer ------------------------------------------------------------------------------------------------

STEP = 2.0 ** -23          # of a sum in fp32, by its magnitude


def ff_forward_mx4(x, W1, W3, W2, topk_idx, gates, inv_pos=None, residual=None):
    """(out, bound).  W1, W3 [E, f, d] and W2 [E, d, f]: the values that the 4 bits stand for.  bound: how far the layer may be off whose
    products sum in fp32 (one rounding for every 128 elements, the partial sums of up to 24 pieces, silu), whose activations may
    therefore fall on the other side of a rounding, and which rounds an expert's output and the result to bf16."""
    T, d = x.shape
    f = W1.shape[1]
    xq = mx4_round(np.asarray(x, dtype=np.float64))
    out = np.zeros((T, d)) if residual is None else np.asarray(residual, dtype=np.float64).copy()
    bound = np.zeros((T, d))
    mag = np.abs(out)
    for t in range(T):
        for j in range(topk_idx.shape[1]):
            if inv_pos is not None and inv_pos[t, j] < 0:
                continue
            e, g = topk_idx[t, j], float(gates[t, j])
            h1, h3 = W1[e] @ xq[t], W3[e] @ xq[t]
            e1 = (d / 128 + 24) * STEP * (np.abs(W1[e]) @ np.abs(xq[t]))
            e3 = (d / 128 + 24) * STEP * (np.abs(W3[e]) @ np.abs(xq[t]))
            with np.errstate(over="ignore"):
                sig = 1.0 / (1.0 + np.exp(-h1))
            silu = h1 * sig
            act = silu * h3
            # |silu'| <= 1.1; the sigmoid in fp32 is 2 + |h1| steps off
            ea = (1.1 * e1 + (4 + np.abs(h1)) * STEP * np.abs(silu)) * (np.abs(h3) + e3) + np.abs(silu) * e3 + 2 * STEP * np.abs(act)
            aq, far = mx4_round(act), mx4_near(act, ea)
            y = W2[e] @ aq
            ey = np.abs(W2[e]) @ far + (f / 128 + 24) * STEP * (np.abs(W2[e]) @ (np.abs(aq) + far))
            ey += 2.0 ** -8 * (np.abs(y) + ey)
            out[t] += g * y
            bound[t] += abs(g) * ey
            mag[t] += abs(g) * (np.abs(y) + ey)
    bound += (topk_idx.shape[1] + 1) * STEP * mag
    return out, bound + 2.0 ** -8 * (np.abs(out) + bound)
