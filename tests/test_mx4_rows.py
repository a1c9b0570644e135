"""The layer of 4-bit experts with every row looked at, tensors past 32-bit offsets, and what NaN and infinities reach."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import many_experts as O
from paper_2403_07816_amd import binding as B

from test_mx4 import DEV, experts, rng_of, routing_of

gpu = pytest.mark.gpu


def grouped(x, V1, V3, V2, idx, gates, inv, residual):
    """(out, bound) as the oracle's ff_forward_mx4, an expert's rows at a time."""
    d, f, step = x.shape[1], V1.shape[1], O.STEP
    xq = O.mx4_round(x)
    out = np.zeros_like(x) if residual is None else residual.copy()
    bound, mag = np.zeros_like(x), np.abs(out)
    for e in range(V1.shape[0]):
        t, j = np.nonzero((idx == e) & (inv >= 0))
        if not t.size:
            continue
        rows, g = xq[t], gates[t, j].astype(np.float64)[:, None]
        h1, h3 = rows @ V1[e].T, rows @ V3[e].T
        e1, e3 = ((d / 128 + 24) * step * (np.abs(rows) @ np.abs(V[e]).T) for V in (V1, V3))
        silu = h1 / (1 + np.exp(-h1))
        act = silu * h3
        ea = (1.1 * e1 + (4 + np.abs(h1)) * step * np.abs(silu)) * (np.abs(h3) + e3) + np.abs(silu) * e3 + 2 * step * np.abs(act)
        aq, far = O.mx4_round(act), O.mx4_near(act, ea)
        y = aq @ V2[e].T
        ey = far @ np.abs(V2[e]).T + (f / 128 + 24) * step * ((np.abs(aq) + far) @ np.abs(V2[e]).T)
        ey += 2.0 ** -8 * (np.abs(y) + ey)
        for sums, part in ((out, g * y), (bound, g * ey), (mag, g * (np.abs(y) + ey))):
            np.add.at(sums, t, part)
    bound += (idx.shape[1] + 1) * step * mag
    return out, bound + 2.0 ** -8 * (np.abs(out) + bound)


def test_grouped_is_the_oracle():
    rng = rng_of("grouped")
    T, d, f, E, k = 12, 64, 96, 4, 2
    V1, V3, V2 = (0.1 * rng.standard_normal(s) for s in ((E, f, d), (E, f, d), (E, d, f)))
    x, res, gates = rng.standard_normal((T, d)), rng.standard_normal((T, d)), rng.random((T, k)).astype(np.float32)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    inv = np.where(rng.random((T, k)) < 0.2, -1, 0)
    for a, b in zip(grouped(x, V1, V3, V2, idx, gates, inv, res), O.ff_forward_mx4(x, V1, V3, V2, idx, gates, inv, res)):
        assert np.allclose(a, b, rtol=1e-9, atol=1e-12)


@gpu
@pytest.mark.parametrize("T,d,f,E,k,favour,cap", [
    (63, 256, 160, 4, 2, None, 0), (300, 288, 416, 5, 2, None, 0),                                         # few rows
    (1300, 512, 1056, 6, 2, None, 0), (840, 2336, 768, 2, 1, None, 0), (2500, 96, 1824, 14, 1, None, 0),   # tall tiles
    (350, 288, 4384, 2, 1, None, 0), (900, 96, 4384, 4, 2, 3, 300),                                        # DOWN cut along its sums
    (1500, 416, 544, 8, 2, 7, 0), (1200, 416, 544, 4, 3, 2, 257),                                          # uneven, and dropped pairs
    (2048, 64, 2080, 8, 4, None, 0), (4096, 1056, 96, 8, 4, None, 0)])                                     # more tiles than a round
def test_every_row_of_the_layer(T, d, f, E, k, favour, cap):
    rng = rng_of("every", T, d, f, E, k)
    (W1, V1), (W3, V3), (W2, V2) = experts(rng, E, d, f), experts(rng, E, d, f), experts(rng, E, f, d)
    x, res = (torch.from_numpy(rng.standard_normal((T, d))).bfloat16() for _ in range(2))
    r, idx, gates, inv = routing_of(rng, T, E, k, favour, cap)
    out = B.btx_moe_ff_forward_mx4(x.to(DEV), W1, W3, W2, r, residual=res.to(DEV)).cpu().double().numpy()
    want, bound = grouped(x.double().numpy(), V1, V3, V2, idx, gates, inv, res.double().numpy())
    wrong = np.argwhere(~(np.abs(out - want) <= bound))
    assert not wrong.size, (len(wrong), wrong[:4])
    assert np.linalg.norm(bound) < 0.06 * np.linalg.norm(want)


@gpu
@pytest.mark.parametrize("T,d,f,E,k", [(70, 416, 544, 4, 2), (900, 416, 544, 4, 2), (400, 96, 4384, 4, 2)])
def test_nan_and_infinity_stay_with_their_rows(T, d, f, E, k):
    """Few rows, tall tiles, DOWN cut: a row with an infinity, an expert with a NaN scale, a column of an expert with one."""
    rng = rng_of("stay", T, d, f)
    W1, W3, W2 = experts(rng, E, d, f)[0], experts(rng, E, d, f)[0], experts(rng, E, f, d)[0]
    r, idx, _, _ = routing_of(rng, T, E, k)
    x = torch.from_numpy(rng.standard_normal((T, d))).bfloat16().to(DEV)
    clean = B.btx_moe_ff_forward_mx4(x, W1, W3, W2, r)
    assert torch.isfinite(clean).all()
    bad = x.clone()
    for t, at, junk in ((0, 0, float("inf")), (T // 2 + 1, d - 1, float("nan")), (T - 1, d // 2, -float("inf"))):
        bad[t, at] = junk
    hit = (~torch.isfinite(bad)).any(1)
    out = B.btx_moe_ff_forward_mx4(bad, W1, W3, W2, r)
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], clean[~hit])
    for e, W, block in ((2, W1, d // 32 - 1), (0, W3, 0)):
        keep = W.scales[e, 5, block].clone()
        W.scales[e, 5, block] = 255
        out = B.btx_moe_ff_forward_mx4(x, W1, W3, W2, r)
        W.scales[e, 5, block] = keep
        hit = torch.from_numpy((idx == e).any(1)).to(DEV)
        assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], clean[~hit])
    W2.scales[1, 37, f // 32 - 1] = 255
    out = B.btx_moe_ff_forward_mx4(x, W1, W3, W2, r)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[:, 37] = torch.from_numpy((idx == 1).any(1)).to(DEV)
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], clean[~hit])


# ---- past 32-bit offsets: as many times the rows of a small batch, which takes the same kernels -------------------


def device_routing(idx, E, gates):
    """idx [T] on the GPU: one expert a token."""
    T = idx.numel()
    perm = torch.sort(idx, stable=True).indices
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T, device=DEV)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.bincount(idx, minlength=E).cumsum(0)
    return SimpleNamespace(topk_idx=idx.int().view(T, 1), gates=gates.view(T, 1), offsets=offsets, perm=perm.int(), inv_pos=inv.int().view(T, 1))


@gpu
@pytest.mark.parametrize("T,n,d", [((1 << 20) + 3, 350, 8192), ((1 << 23) - 3, 3000, 1024), ((1 << 23) - 1, 2000, 1024)])
def test_token_rows_past_32_bits(T, n, d):
    """4 GiB of x's codes with 64-bit addresses; the most that the tall tiles find with 32 bits; the first batch that is too large for them."""
    rng = rng_of("tokens", T)
    f, E = 32, 2
    W1, W3, W2 = experts(rng, E, d, f)[0], experts(rng, E, d, f)[0], experts(rng, E, f, d)[0]
    few = torch.from_numpy(rng.standard_normal((n, d))).bfloat16().to(DEV)
    idx, gates = torch.from_numpy(rng.integers(0, E, n)).to(DEV), torch.from_numpy(rng.random(n)).float().to(DEV)
    want = B.btx_moe_ff_forward_mx4(few, W1, W3, W2, device_routing(idx, E, gates))
    times = -(-T // n)
    out = B.btx_moe_ff_forward_mx4(few.repeat(times, 1)[:T], W1, W3, W2, device_routing(idx.repeat(times)[:T], E, gates.repeat(times)[:T]))
    whole = T // n * n
    assert torch.equal(out[:whole].view(-1, n, d), want.expand(whole // n, n, d)) and torch.equal(out[whole:], want[:T - whole])


@gpu
@pytest.mark.parametrize("T", [40, 2100])
def test_experts_past_32_bits(T):
    """65 experts of 4096 x 32768, more than 4 GiB of codes a matrix: the last of them, and a layer of two experts that are those."""
    rng = rng_of("stack", T)
    E, d, f, pick = 65, 4096, 32768, [3, 64]
    g = torch.Generator(device=DEV).manual_seed(T)
    lib = B.load_library()

    def stack(n, K):
        codes = torch.randint(0, 256, (E, n, K // 2), dtype=torch.uint8, device=DEV, generator=g)
        return B.Mx4(codes, torch.full((E, n, lib.btx_mx4_scale_pitch(K)), 127 - int(np.log2(4 * np.sqrt(K))), dtype=torch.uint8, device=DEV), K)

    W1, W3, W2 = stack(f, d), stack(f, d), stack(d, f)
    x = torch.from_numpy(rng.standard_normal((T, d))).bfloat16().to(DEV)
    which, gates = torch.from_numpy(rng.integers(0, 2, T)).to(DEV), torch.from_numpy(rng.random(T)).float().to(DEV)
    out = B.btx_moe_ff_forward_mx4(x, W1, W3, W2, device_routing(torch.tensor(pick, device=DEV)[which], E, gates))
    two = [B.Mx4(W.codes[pick], W.scales[pick], W.K) for W in (W1, W3, W2)]
    want = B.btx_moe_ff_forward_mx4(x, *two, device_routing(which, 2, gates))
    assert torch.isfinite(want).all() and torch.equal(out, want)


@gpu
@pytest.mark.parametrize("shape,axis", [((131075, 32768), -1), ((3, 32768, 43720), -2)])
def test_tensors_past_32_bits(shape, axis):
    """More than 2^32 elements there and back: 8 rows (or columns) again and again."""
    rng = rng_of("elements", axis)
    n = 8
    few = torch.from_numpy(rng.standard_normal((n, shape[-1]) if axis == -1 else (shape[-2], n))).bfloat16().to(DEV)
    q = B.btx_mx4_quantize(few, axis)
    back = B.btx_mx4_dequantize(q, torch.bfloat16, axis)
    times = -(-shape[0] // n) if axis == -1 else shape[-1] // n
    x = few.repeat(times, 1)[:shape[0]] if axis == -1 else few.repeat(1, times).expand(shape).contiguous()
    Q = B.btx_mx4_quantize(x, axis)
    for got, want in ((Q.codes, q.codes), (Q.scales, q.scales)):
        m = got.reshape(-1, got.shape[-1])
        whole = m.shape[0] // n * n
        assert torch.equal(m[:whole].view(-1, n, m.shape[1]), want.expand(whole // n, n, m.shape[1])) and torch.equal(m[whole:], want[:len(m) - whole])
    x = B.btx_mx4_dequantize(Q, torch.bfloat16, axis)
    if axis == -1:
        whole = shape[0] // n * n
        assert torch.equal(x[:whole].view(-1, n, shape[1]), back.expand(whole // n, n, shape[1])) and torch.equal(x[whole:], back[:shape[0] - whole])
    else:
        assert torch.equal(x.view(*shape[:2], times, n), back.unsqueeze(1).expand(*shape[:2], times, n))
