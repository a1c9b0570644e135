"""Block-scaled 8-bit floats where the kernels of many rows, the matrix cores' own 8-bit product and sums that are cut along K can go wrong."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import fp8 as O
from paper_2403_07816_amd import binding as B

import test_fp8
from test_fp8 import BF, DEV, F32, check_layer, check_product, make_layer, rng_of
from test_mx4 import experts, routing_of

gpu = pytest.mark.gpu


def rest_of(call):
    """call(residual) of a layer that weighs one slot of a token by 1, the others by 0: what the residual leaves of y that is what y rounds to in bf16.  Zeros
    wherever y itself was rounded."""
    return call(-call(None)).float().abs()


@gpu
@pytest.mark.parametrize("T,d,f,E,k,rounded", [(1, 256, 128, 4, 1, False), (40, 264, 128, 4, 2, False), (2048, 2048, 128, 2, 1, False), (2049, 2048, 128, 2, 1, True),
                                               (70, 64, 128, 16, 8, False), (70, 64, 128, 16, 9, True), (8191, 64, 128, 8, 5, False), (8192, 64, 128, 8, 4, False),
                                               (8192, 64, 128, 8, 5, True)])
def test_which_experts_outputs_are_rounded(T, d, f, E, k, rounded):
    x, _, W, routing, _, _, _ = make_layer(T, d, f, E, k, 21)
    routing.gates.zero_()
    routing.gates[:, 0] = 1.0
    rest = rest_of(lambda r: B.btx_moe_ff_forward_fp8(x, *[w for w, _ in W], routing, residual=r))
    # (a sum of 128 products of 8 bits each has a rest but for one in a hundred)
    assert not rest.any() if rounded else (rest > 0).float().mean() > 0.9


@gpu
@pytest.mark.parametrize("T,d,f,E,k", [(1, 256, 128, 4, 1), (40, 288, 128, 4, 2), (70, 64, 128, 16, 8)])
def test_outputs_of_4_bit_experts_that_are_not_cut_are_rounded(T, d, f, E, k):
    rng = rng_of("rounded", T, d, f, E, k)
    (W1, _), (W3, _), (W2, _) = experts(rng, E, d, f), experts(rng, E, d, f), experts(rng, E, f, d)
    x = torch.from_numpy(rng.standard_normal((T, d))).to(BF).to(DEV)
    r, _, _, _ = routing_of(rng, T, E, k)
    r.gates.zero_()
    r.gates[:, 0] = 1.0
    assert not rest_of(lambda res: B.btx_moe_ff_forward_mx4(x, W1, W3, W2, r, residual=res)).any()


# ---- products --------------------------------------------------------------------------------------------------

# rows, columns, depth; the kernels of bf16 and of fp32 results (test_launches_fp8.py holds them to it)
EDGE_PRODUCTS = [(5, 136, 700, "few16", "few16"), (40, 136, 700, "few16", "few16"), (5, 33000, 136, "few64", "few16"), (30, 33000, 300, "few64", "few16"), (300, 136, 2304, "mid64", "mid64"), (1100, 4104, 264, "mid128", "mid128"),
                 (700, 2080, 8300, "mid64", "mid128"), (16500, 2048, 130, "tall", "mid128"), (500, 16600, 2040, "tall apart", "mid128"), (3001, 64, 1024, "few16", "few16")]
SHAPES = [s[:3] for s in EDGE_PRODUCTS]


def on_device(rows, K, seed, block_rows=1, scale=1.0):
    """(operand, the values that it stands for)"""
    g = torch.Generator(device=DEV).manual_seed(1000 * seed + rows + K)
    v = torch.randn((rows, K), generator=g, device=DEV) * torch.exp(0.5 * torch.randn((rows, 1), generator=g, device=DEV)) * scale
    q = B.btx_fp8_quantize(v, block_rows=block_rows)
    return q, B.btx_fp8_dequantize(q, F32).double().cpu().numpy()


def some_rows(M):
    return np.arange(M) if M <= 400 else np.unique(np.concatenate([np.arange(20), np.arange(M - 20, M), rng_of("rows", M).integers(0, M, 100)]))


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_nan_stays_with_its_row_and_column(M, N, K, dtype):
    """Scales that are NaN, over codes and over the zeros that a block with a NaN is quantised to, and the code that is NaN."""
    (a, av), (b, bv) = on_device(M, K, 1), on_device(N, K, 2, 128)
    last = (K - 1) // 128
    rows, columns = [2, 3, 4, M - 1], [0, 33, 50, N - 1]
    for q, at in ((a, rows), (b, columns)):
        q.scales[at[0], 0] = 255
        q.scales[at[1], last] = 255
        q.codes[at[1], 128 * last:128 * last + 128] = 0
        q.codes[at[2], K - 1] = 127
        q.codes[at[3], 1] = 255
    out = B.btx_fp8_matmul(a, b, dtype=dtype).cpu()
    nan = torch.zeros((M, N), dtype=torch.bool)
    nan[rows] = True
    nan[:, columns] = True
    assert torch.equal(torch.isnan(out), nan)
    keep, kept = np.setdiff1d(some_rows(M), rows), np.setdiff1d(np.arange(N), columns)
    check_product(out[keep][:, kept], av[keep], bv[kept])


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_scales_from_the_smallest(M, N, K, dtype):
    """Every code under scales from 2^-127 on, which no other test has in front of the matrix cores' own 8-bit product; none of a result that leaves fp32."""
    g = torch.Generator(device=DEV).manual_seed(M + N + K)

    def made(rows, lo, hi):
        q = B.alloc_fp8((rows, K), -1, DEV)
        q.codes.copy_(torch.randint(0, 127, q.codes.shape, generator=g, device=DEV) + 128 * torch.randint(0, 2, q.codes.shape, generator=g, device=DEV))
        q.codes[:, K:] = 0
        q.scales.zero_()
        n = (K + 127) // 128
        q.scales[:, :n] = torch.randint(lo, hi, (rows, n), generator=g, device=DEV).to(torch.uint8)
        q.scales[:4, :n] = torch.tensor([[lo], [lo], [hi - 1], [lo + 1]], dtype=torch.uint8, device=DEV)
        return q

    a, b = made(M, 0, 60), made(N, 120, 200)
    rows = some_rows(M)
    av = O.values(a.codes[rows, :K].cpu().numpy().astype(np.int64), a.scales[rows].cpu().numpy().astype(np.int64))
    bv = O.values(b.codes[:, :K].cpu().numpy().astype(np.int64), b.scales.cpu().numpy().astype(np.int64))
    want, err = av @ bv.T, O.sums_error(av, bv, exact=dtype == F32)
    # Below 2^-126 values are 2^-149 apart in fp32 and 2^-133 in bf16: sums of K products, results, and, in front of fp32 results, the values of a.
    err = err + K * 2.0 ** -149 + (2.0 ** -134 * np.abs(bv).sum(1) if dtype == F32 else 0)
    bound = err + torch.finfo(dtype).eps / 2 * (np.abs(want) + err) + (0 if dtype == F32 else 2.0 ** -134)
    off = np.abs(B.btx_fp8_matmul(a, b, dtype=dtype)[rows].double().cpu().numpy() - want)
    assert np.all(off <= bound), float((off / bound).max())
    assert (np.abs(want) > 2 * bound).mean() > 0.9


# cut along K, and the kernel that does: bf16 results, fp32 results
CUT_PRODUCTS = [(33, 2048, 11008, "mid64", "mid64"), (513, 264, 18000, "mid64", "mid64"), (200, 2080, 8300, "mid64", "mid128"), (2048, 4096, 8300, "tall", None),
                (16, 512, 8192, "mid64", "mid64"), (301, 1032, 2177, "mid64", "mid64")]


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K", [s[:3] for s in CUT_PRODUCTS])
def test_sums_that_are_cut_lose_nothing(M, N, K, dtype):
    """Whole numbers whose sums stay below 2^24: exact in fp32 in whatever order (and their products, 1 to 64, to the matrix cores' 8-bit product too); a bf16
    result is that, rounded once."""
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    whole = lambda rows: torch.randint(-8, 9, (rows, K), generator=g, device=DEV).float()  # noqa: E731
    av, bv = whole(M), whole(N)
    a, b = B.btx_fp8_quantize(av), B.btx_fp8_quantize(bv)
    assert torch.equal(B.btx_fp8_dequantize(a, F32), av) and torch.equal(B.btx_fp8_dequantize(b, F32), bv)
    residual = torch.randint(-64, 65, (M, N), generator=g, device=DEV).to(dtype)
    rows = torch.from_numpy(some_rows(M)).to(DEV)
    want = av[rows].double() @ bv.double().T
    assert torch.equal(B.btx_fp8_matmul(a, b, dtype=dtype)[rows], want.float().to(dtype))
    assert torch.equal(B.btx_fp8_matmul(a, b, dtype=dtype, residual=residual)[rows], (want + residual[rows].double()).float().to(dtype))


@gpu
@pytest.mark.parametrize("T,d,n", [(190, 264, 136), (2100, 1032, 2056)])
def test_training_of_a_linear_layer_in_bf16(T, d, n):
    """y = x W^T and dx = dy W with results in bf16: against the values that the codes stand for, and dx against differences of the loss of exact products."""
    rng = rng_of("training in bf16", T, d, n)
    x, W, dY = (torch.tensor(rng.standard_normal(s)).to(BF) for s in ((T, d), (n, d), (T, n)))
    q = {name: (B.btx_fp8_quantize(v.to(DEV), axis, rows), axis) for name, v, axis, rows in
         (("x", x, -1, 1), ("W", W, -1, 128), ("Wt", W, -2, 128), ("dY", dY, -1, 1), ("dYt", dY, -2, 1), ("xt", x, -2, 1))}
    v = {}
    for name, (t, axis) in q.items():
        back = B.btx_fp8_dequantize(t, F32, axis).double().cpu().numpy()
        v[name] = back if axis == -1 else back.T
    check_product(B.btx_fp8_matmul(q["x"][0], q["W"][0]), v["x"], v["W"])
    dx = B.btx_fp8_matmul(q["dY"][0], q["Wt"][0])
    check_product(dx, v["dY"], v["Wt"])
    check_product(B.btx_fp8_matmul(q["dYt"][0], q["xt"][0], dtype=F32), v["dYt"], v["xt"])
    step = rng.standard_normal((T, d))
    x0, W0, dY0 = (t.double().numpy() for t in (x, W, dY))
    loss = lambda m: float((dY0 * (m @ W0.T)).sum())  # noqa: E731
    slope = (loss(x0 + 1e-5 * step) - loss(x0 - 1e-5 * step)) / 2e-5
    got = dx.double().cpu().numpy()
    # every factor of a product is off by half an e4m3 step, 2^-4 of it at most, at random: two factors
    assert abs((got * step).sum() - slope) <= 2 * 2.0 ** -4 * np.linalg.norm(got) * np.linalg.norm(step)


# ---- the layer in tall tiles -------------------------------------------------------------------------------------

# T, d, f, E, k; the kernels of UP and DOWN, whether DOWN's sums are cut (test_launches_fp8.py holds the sizes to them)
TALL_LAYERS = [((9000, 520, 776, 4, 2), "tall", "tall", False), ((900, 2040, 1096, 4, 2), "tall apart", "mid64", True), ((1600, 520, 8200, 4, 1), "tall", "tall", True)]
TALL_EXPERTS = (2200, 8192, 16400, 33, 1)
tall = pytest.mark.parametrize("T,d,f,E,k", [s[0] for s in TALL_LAYERS])


@pytest.fixture
def made(monkeypatch):
    """make_layer() with operands from the device."""
    monkeypatch.setattr(test_fp8, "operand", on_device)
    return make_layer


def poisoned(T, d, f, E, k):
    return torch.full((B.load_library().btx_moe_ff_forward_fp8_workspace_bytes(T, d, f, E, k),), 255, dtype=torch.uint8, device=DEV)


@gpu
@tall
@pytest.mark.parametrize("skew,drop", [(True, 0.0), (False, 0.4), (True, 0.9), (False, 1.0)])
def test_tall_layer_of_a_favoured_expert_and_dropped_pairs(made, T, d, f, E, k, skew, drop):
    x, xv, W, routing, idx, gates, inv = made(T, d, f, E, k, 3, skew, drop)
    residual = torch.tensor(rng_of("dres", T).standard_normal((T, d))).to(BF).to(DEV)
    out = torch.full((T + 1, d), 77.0, dtype=BF, device=DEV)
    B.btx_moe_ff_forward_fp8(x, *[w for w, _ in W], routing, out=out[:T], residual=residual, workspace=poisoned(T, d, f, E, k))
    check_layer(out[:T], xv, W, idx, gates, inv, residual)
    assert (out[T] == 77.0).all()                          # rows behind the last token are left
    if drop == 1.0:
        assert torch.equal(out[:T], residual)


@gpu
@tall
def test_tall_layer_of_one_expert_twice(made, T, d, f, E, k):
    """A routing that names an expert in all of a token's slots and has one without tokens, and a workspace that holds NaN."""
    x, xv, W, routing, _, gates, _ = made(T, d, f, E, k, 6)
    idx = np.repeat(rng_of("twice", T).integers(0, E - 1, (T, 1)), k, 1)
    perm = np.argsort(idx.reshape(-1), kind="stable")
    inv = np.argsort(perm).reshape(T, k)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(idx.reshape(-1), minlength=E))])
    for name, v in (("topk_idx", idx), ("perm", perm), ("inv_pos", inv), ("offsets", offsets)):
        setattr(routing, name, torch.tensor(v, dtype=torch.int32, device=DEV))
    ws = poisoned(T, d, f, E, k)
    out = B.btx_moe_ff_forward_fp8(x, *[w for w, _ in W], routing, workspace=ws)
    check_layer(out, xv, W, idx, gates, inv)
    assert torch.equal(B.btx_moe_ff_forward_fp8(x, *[w for w, _ in W], routing, workspace=ws), out)


@gpu
@tall
def test_tall_layer_keeps_nan_to_its_tokens(made, T, d, f, E, k):
    """A token's scale, a block of W1 of one expert (whose tokens' block of activations is quantised to NaN in the kernel), a column of another's output."""
    x, xv, W, routing, idx, gates, inv = made(T, d, f, E, k, 4)
    q = [w for w, _ in W]
    clean = B.btx_moe_ff_forward_fp8(x, *q, routing).cpu()
    check_layer(clean, xv, W, idx, gates, inv)
    x.scales[3, 1] = 255
    x.scales[T - 1, (d - 1) // 128] = 255
    q[0].scales[0, f - 1, 1] = 255
    q[2].scales[1, 10, 2] = 255
    out = B.btx_moe_ff_forward_fp8(x, *q, routing, workspace=poisoned(T, d, f, E, k)).cpu()
    nan = torch.zeros(T, d, dtype=torch.bool)
    nan[[3, T - 1]] = True
    nan[torch.tensor((idx == 0).any(1))] = True
    nan[torch.tensor((idx == 1).any(1)), 10] = True
    assert torch.equal(torch.isnan(out), nan) and not nan.all(1).all()
    assert torch.equal(out[~nan], clean[~nan])


@gpu
def test_tall_layer_of_weights_past_32_bit_offsets():
    """The last of experts of more than 4 GiB in all; the others are zero."""
    T, d, f, E, _ = TALL_EXPERTS
    lib = B.load_library()
    q, last = [], []
    for n, K in ((f, d), (f, d), (d, f)):
        w = B.Fp8(torch.zeros((E, n, lib.btx_fp8_code_pitch(K)), dtype=torch.uint8, device=DEV),
                  torch.full((E, n, lib.btx_fp8_scale_pitch(K)), 127, dtype=torch.uint8, device=DEV), K)
        part = B.btx_fp8_quantize(torch.randn((n, K), generator=torch.Generator(device=DEV).manual_seed(n + K), device=DEV) * K ** -0.5)
        w.codes[E - 1], w.scales[E - 1] = part.codes, part.scales
        q.append(w)
        last.append(B.btx_fp8_dequantize(part, F32).double())
    x = B.btx_fp8_quantize(torch.randn((T, d), generator=torch.Generator(device=DEV).manual_seed(T), device=DEV))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    half = T // 2                                          # tokens of expert 0, and of the last
    routing = SimpleNamespace(topk_idx=i32([[0]] * half + [[E - 1]] * (T - half)), gates=torch.ones((T, 1), device=DEV), perm=i32(range(T)),
                              offsets=i32([0] + [half] * (E - 1) + [T]), inv_pos=i32([[t] for t in range(T)]))
    out = B.btx_moe_ff_forward_fp8(x, *q, routing).double()
    assert not out[:half].any()
    xv = B.btx_fp8_dequantize(x, F32).double()[half:]
    h1, h3 = xv @ last[0].T, xv @ last[1].T
    act = B.btx_fp8_dequantize(B.btx_fp8_quantize((h1 * torch.sigmoid(h1) * h3).float()), F32).double()
    want = act @ last[2].T
    # codes on the other side of a rounding, and two roundings to bf16: 2^-8 of the norm each at most
    assert (out[half:] - want).norm() <= 2 * 2.0 ** -8 * want.norm()


@gpu
@tall
def test_tall_layer_in_a_graph_and_on_two_streams(made, T, d, f, E, k):
    _, _, W, routing, _, _, _ = made(T, d, f, E, k, 5)
    q = [w for w, _ in W]
    g = torch.Generator(device=DEV).manual_seed(T)
    tokens = [torch.randn((T, d), generator=g, device=DEV) for _ in range(3)]
    B.btx_init()

    def buffers():
        return SimpleNamespace(x=B.alloc_fp8((T, d), -1, DEV), out=torch.empty((T, d), dtype=BF, device=DEV), ws=poisoned(T, d, f, E, k))

    def layer(b):
        return B.btx_moe_ff_forward_fp8(b.x, *q, routing, out=b.out, workspace=b.ws)

    def fill(b, i):
        B.btx_fp8_quantize(tokens[i], out=b.x)
        b.out.fill_(3.0)

    eager, b = buffers(), buffers()
    fill(b, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(b)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(b)
    for i in (1, 2, 1, 0):
        fill(b, i)
        graph.replay()
        fill(eager, i)
        assert torch.equal(layer(eager), b.out)
        torch.cuda.synchronize()
    want = []
    for x, i in ((b, 1), (eager, 2)):
        fill(x, i)
        want.append(layer(x).clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for x in (b, eager):
            x.out.zero_()
        torch.cuda.synchronize()
        for stream, x in zip(streams, (b, eager)):
            with torch.cuda.stream(stream):
                layer(x)
        torch.cuda.synchronize()
        assert all(torch.equal(x.out, w) for x, w in zip((b, eager), want))


@gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_values_past_fp32(M, N, K):
    """448 * 2^127 (a scale that no tensor of finite floats is quantised to) times 2^-127: in front of fp32 results a value is a bf16 value, and that one infinite;
    bf16 results are of codes and scales as they are."""
    a, b = (B.Fp8(torch.zeros((n, (K + 127) // 128 * 128), dtype=torch.uint8, device=DEV), torch.full((n, 16 * (((K + 127) // 128 + 15) // 16)), s, dtype=torch.uint8, device=DEV), K)
            for n, s in ((M, 254), (N, 0)))
    a.codes[2, K - 1] = 126
    b.codes[:, K - 1] = 56
    out = B.btx_fp8_matmul(a, b), B.btx_fp8_matmul(a, b, dtype=F32)
    assert (out[0][2] == 448).all() and (out[1][2] == float("inf")).all()
    assert all(int(o.count_nonzero()) == N for o in out)
    q = B.btx_fp8_quantize(torch.full((1, 8), torch.finfo(F32).max, device=DEV))
    assert int(q.scales[0, 0]) == 247 and torch.isinf(B.btx_fp8_dequantize(q, F32)).all()
