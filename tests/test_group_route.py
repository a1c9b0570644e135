"""Routing from logits for many experts and its gradient: against the float64 oracle, whose selection it has to make exactly."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import many_experts as O
from paper_2403_07816_amd import binding as B

gpu = pytest.mark.gpu
DEV = "cuda:0"
SCORE = {"sigmoid": B.BTX_SCORE_SIGMOID, "softmax": B.BTX_SCORE_SOFTMAX}
GROUP = {"top2": B.BTX_GROUP_TOP2, "max": B.BTX_GROUP_MAX}


def rng_of(*key):
    return np.random.default_rng(sum(ord(c) * (i + 1) for i, c in enumerate(str(key))))


# ---- the oracle -----------------------------------------------------------------------------------------------


def test_oracle_agrees_with_a_sort():
    rng = rng_of("sort")
    l = rng.standard_normal((50, 24))
    bias = 0.1 * rng.standard_normal(24)
    r = O.group_route(l, 5, "sigmoid", bias, 4, 2, "top2")
    v = 1 / (1 + np.exp(-l)) + bias
    value = np.sort(v.reshape(50, 4, 6), 2)[:, :, -2:].sum(2)
    kept = np.argsort(-value, 1)[:, :2]
    mask = np.zeros((50, 4), bool)
    np.put_along_axis(mask, kept, True, 1)
    v = np.where(np.repeat(mask, 6, 1), v, -np.inf)
    assert np.array_equal(r["topk_idx"], np.argsort(-v, 1)[:, :5])
    assert np.allclose(r["gates"].sum(1), 1.0)
    assert np.array_equal(r["perm"][r["inv_pos"].reshape(-1)], np.arange(250))


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("with_scores", [True, False])
def test_oracle_backward_against_differences(score, renorm, with_scores):
    rng = rng_of(score, renorm, with_scores)
    T, E, k = 3, 9, 4
    l = rng.standard_normal((T, E))
    r = O.group_route(l, k, score, renorm=renorm, scale=2.5)
    dg = rng.standard_normal((T, k))
    ds = rng.standard_normal((T, E)) if with_scores else None

    def loss(x):
        s = O.scores(x, score)
        w = np.take_along_axis(s, r["topk_idx"], 1)
        g = 2.5 * (w / (w.sum(1, keepdims=True) + 1e-20) if renorm else w)
        return (g * dg).sum() + (0.0 if ds is None else (s * ds).sum())

    dl = O.group_route_backward(l, r["topk_idx"], dg, score, renorm, 2.5, ds)
    h = 1e-5
    for t in range(T):
        for e in range(E):
            d = np.zeros_like(l)
            d[t, e] = h
            assert abs((loss(l + d) - loss(l - d)) / (2 * h) - dl[t, e]) < 1e-8


# ---- refusals -------------------------------------------------------------------------------------------------


def test_refusals():
    lib = B.load_library()
    p, q, null = ctypes.c_void_p(256), ctypes.c_void_p(264), None

    def fwd(l=p, dt=0, T=100, E=64, k=8, score=0, G=8, keep=4, gs=0, scale=1.0, idx=p, gates=p, scores=p, perm=p, ws=p, nbytes=1 << 20):
        return lib.btx_moe_group_route(l, dt, null, T, E, k, score, G, keep, gs, 1, scale, idx, gates, scores, p, p, perm, p, ws, nbytes, null)

    assert fwd(T=0) == 0 and fwd(T=0, l=null, ws=null) == 0
    for bad in (dict(dt=2), dict(T=-1), dict(E=0), dict(E=257, G=1, keep=1), dict(k=0), dict(k=17), dict(k=9, keep=1), dict(G=0), dict(G=17, E=68),
                dict(G=7), dict(keep=0), dict(keep=9), dict(score=2), dict(gs=2), dict(scale=float("inf")), dict(scale=float("nan")),
                dict(l=null), dict(idx=null), dict(gates=null), dict(perm=null), dict(ws=null), dict(l=q), dict(scores=q), dict(ws=q),
                dict(T=1 << 28, k=8)):
        assert fwd(**bad) == 1, bad
    assert fwd(T=1 << 30, E=8, k=1, G=1, keep=1) == 1
    assert fwd(nbytes=16) == 3

    def bwd(l=p, dt=0, idx=p, dg=p, ds=null, T=100, E=64, k=8, score=0, scale=1.0, dl=p):
        return lib.btx_moe_group_route_backward(l, dt, idx, dg, ds, T, E, k, score, 1, scale, dl, null)

    assert bwd(T=0, l=null) == 0
    for bad in (dict(dt=2), dict(T=-1), dict(E=257), dict(k=0), dict(k=17), dict(E=4, k=5), dict(score=2), dict(scale=float("nan")), dict(l=null),
                dict(idx=null), dict(dg=null), dict(dl=null), dict(l=q), dict(ds=q), dict(dl=q), dict(T=1 << 28)):
        assert bwd(**bad) == 1, bad
    assert bwd(T=(1 << 30) - 1, k=1) == 2 and bwd(T=1 << 30, k=1) == 1

    def gates(dt=1, dwt=1, dY=p, dg=p, dW=(p, p, p), s13=64 * 64, T=8, ws=p, nbytes=1 << 30, f=64):
        return lib.btx_moe_ff_backward_gates(dY, p, p, p, p, dt, s13, 64 * 64, T, 64, f, 4, 2, p, p, p, p, p, p, p, dg, *dW, dwt, ws, nbytes, null)

    assert gates(T=0) == 0
    for bad in (dict(dt=3), dict(dt=0, dwt=1), dict(dY=null), dict(dg=null), dict(dW=(p, null, p)), dict(s13=8), dict(ws=null), dict(f=60), dict(dY=q)):
        assert gates(**bad) == 1, bad
    assert gates(nbytes=0) == 3 and gates(T=1 << 26) == 2


def test_workspace_never_falls():
    lib = B.load_library()
    for E in (1, 60, 256):
        sizes = [lib.btx_moe_group_route_workspace_bytes(T, E, 1) for T in [0, 1, 64, 65, 128, 4000, 32768, 32769, 40000, 65536, 65537, 1 << 20]]
        assert sizes == sorted(sizes) and sizes[2] == 0 and sizes[3] > 0


def test_host_tensors_are_refused():
    with pytest.raises(AssertionError):
        B.btx_moe_group_route(torch.zeros(4, 8), 2)


# ---- the kernels ----------------------------------------------------------------------------------------------


def route_both(l, k, score="sigmoid", bias=None, G=1, keep=1, gs="top2", renorm=True, scale=1.0, with_scores=True):
    """l: torch tensor on the host."""
    T, E = l.shape
    o = O.group_route(l.double().numpy(), k, score, None if bias is None else bias.double().numpy(), G, keep, gs, renorm, scale)
    out = B.alloc_group_routing(T, E, k, DEV, scores=with_scores)
    for t in vars(out).values():
        if t is not None:
            t.view(torch.uint8).fill_(0xFF)              # nothing may depend on what was there
    ws = torch.full((max(B.load_library().btx_moe_group_route_workspace_bytes(T, E, k), 16),), 0xFF, dtype=torch.uint8, device=DEV)
    r = B.btx_moe_group_route(l.to(DEV), k, SCORE[score], None if bias is None else bias.to(DEV), G, keep, GROUP[gs], renorm, scale, out=out,
                              workspace=ws)
    return r, o


def check_route(r, o, scale=1.0):
    for name in ("topk_idx", "counts", "offsets", "perm", "inv_pos"):
        assert np.array_equal(getattr(r, name).cpu().numpy(), o[name]), name
    # exp's argument is rounded to (|l| + |max|) 2^-24; at |l| <= 8 with the sums and quotients under 48 steps
    assert np.all(np.abs(r.gates.cpu().double().numpy() - o["gates"]) <= 48 * 2.0 ** -23 * np.abs(o["gates"]) + 1e-37 * scale)
    if r.scores is not None:
        assert np.all(np.abs(r.scores.cpu().double().numpy() - o["scores"]) <= 48 * 2.0 ** -23 * np.abs(o["scores"]) + 1e-37)


SHAPES = [  # T, E, k, groups, kept
    (1, 1, 1, 1, 1), (1, 256, 16, 1, 1), (2, 5, 5, 1, 1), (3, 256, 8, 8, 4), (63, 60, 6, 4, 2), (64, 64, 8, 8, 4), (65, 64, 8, 8, 4),
    (67, 33, 7, 3, 2), (129, 255, 16, 15, 9), (130, 144, 8, 9, 1), (200, 250, 10, 5, 3), (301, 16, 2, 16, 5), (77, 32, 1, 16, 1),
    (500, 160, 6, 8, 3), (1000, 7, 3, 7, 5), (2049, 128, 8, 2, 1), (333, 252, 9, 14, 14), (90, 12, 4, 6, 3),
]


@gpu
@pytest.mark.parametrize("T,E,k,G,keep", SHAPES)
@pytest.mark.parametrize("score,gs,bias,renorm,dtype", [
    ("sigmoid", "top2", True, True, torch.float32), ("softmax", "max", False, False, torch.bfloat16),
    ("softmax", "top2", True, True, torch.bfloat16), ("sigmoid", "max", False, True, torch.float32)])
def test_route(T, E, k, G, keep, score, gs, bias, renorm, dtype):
    rng = rng_of(T, E, k, score)
    l = torch.from_numpy(rng.standard_normal((T, E)) * 1.3).to(dtype)
    b = torch.from_numpy(0.1 * rng.standard_normal(E)).float() if bias else None
    check_route(*route_both(l, k, score, b, G, keep, gs, renorm, 2.5))


@gpu
def test_route_more_tokens_than_one_pass_of_a_block():
    rng = rng_of("many")
    l = torch.from_numpy(rng.standard_normal((32900, 8))).float()       # 128 tokens a block
    check_route(*route_both(l, 3, "softmax", None, 4, 2, "top2"))


@gpu
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("G,keep", [(1, 1), (4, 2)])
def test_route_ties_go_to_the_lower_index(score, G, keep):
    rng = rng_of("ties", score, G)
    for values in ([0.0], [0.0, 1.0], [-1.0, 0.5, 0.5, 2.0]):
        l = torch.from_numpy(rng.choice(values, (70, 48))).float()
        check_route(*route_both(l, 8, score, None, G, keep))
    # one step apart in float: the order of the scores in double
    one = np.float32(1.0)
    steps = np.array([one, np.nextafter(one, np.float32(2)), np.nextafter(one, np.float32(0))])
    check_route(*route_both(torch.from_numpy(rng.choice(steps, (70, 48))), 8, score, None, G, keep))
    # the bias decides between equal scores, by one step of double's sum only
    bias = torch.from_numpy(rng.choice([0.25, np.nextafter(np.float32(0.25), np.float32(1))], 48)).float()
    check_route(*route_both(torch.zeros(70, 48), 8, score, bias, G, keep))


@gpu
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,k", [(256, 8), (60, 16)])
def test_route_ties_at_the_last_slot(score, E, k):
    """Equal logits for the last slot and behind it, and some that differ from them by a step of float."""
    rng = rng_of("last", score, E)
    one = np.float32(1.0)
    values = np.array([one, np.nextafter(one, np.float32(2)), np.nextafter(one, np.float32(0)), 2.0, -1.0], dtype=np.float32)
    rare = min(k / E, 0.2)                                  # so that the k-th largest is now the one value, now the other
    for p in ([rare, rare / 2, rare, rare / 4], [rare / 2, rare / 3, rare / 2, rare / 2], [rare / 4, rare, 3 * rare, 0.0]):
        l = torch.from_numpy(rng.choice(values, (130, E), p=[*p, 1 - sum(p)]))
        check_route(*route_both(l, k, score, None))
        check_route(*route_both(l, k, score, None, 4, 3, "max"))
    check_route(*route_both(torch.from_numpy(rng.standard_normal((130, E))).bfloat16(), k, score, None))


@gpu
@pytest.mark.parametrize("G,keep,gs", [(1, 1, "max"), (4, 2, "max"), (4, 2, "top2")])
def test_route_of_scores_about_the_least_normal_float(G, keep, gs):
    """Logits a few steps of float apart whose scores are 0 in float, or nearly: the order of double still."""
    rng = rng_of("least", G, gs)
    for base in (-87.33655, -80.0, -95.0, -103.0):
        step = np.spacing(np.float32(abs(base)))
        l = base + step * rng.integers(-6, 7, (150, 64))
        r, o = route_both(torch.from_numpy(l).float(), 8, "sigmoid", None, G, keep, gs, renorm=False)
        assert np.array_equal(r.topk_idx.cpu().numpy(), o["topk_idx"]), base
        l[:, 5] = 0.0                                      # the row's largest, and far below it the others
        r, o = route_both(torch.from_numpy(l).float(), 8, "softmax", None, G, keep, gs, renorm=False)
        assert np.array_equal(r.topk_idx.cpu().numpy(), o["topk_idx"]), base


@gpu
@pytest.mark.parametrize("gs", ["top2", "max"])
def test_route_under_a_bias_that_outweighs_the_scores(gs):
    """Values near 1 of scores near 1 and of scores near 0: what is behind the last slot may be the less exact one."""
    rng = rng_of("outweighs", gs)
    one = rng.random(64) < 0.5
    l = rng.uniform(9, 12, (200, 64)) * np.where(one, -1, 1)
    bias = torch.from_numpy(np.where(one, 1.0, 0.0)).float()
    check_route(*route_both(torch.from_numpy(l).float(), 9, "sigmoid", bias))
    check_route(*route_both(torch.from_numpy(l).float(), 9, "sigmoid", bias, 8, 3, gs))
    least = torch.from_numpy(rng.choice([0.0, 0.1, -1e30, -1e35, np.finfo(np.float32).min, -np.inf], 64)).float()
    for k in (4, 14):                                      # experts that a bias all but masks, and the sums with theirs
        check_route(*route_both(torch.from_numpy(l).float(), k, "sigmoid", least, 16, 6, gs))
    inf = torch.zeros(64)
    inf[[3, 5, 20, 21, 50]] = float("inf")                 # more groups of an infinite value than are kept
    check_route(*route_both(torch.from_numpy(l).float(), 4, "sigmoid", inf, 4, 1, gs))


@gpu
def test_route_with_a_bias_on_any_boundary():
    l = torch.randn(70, 64, generator=torch.Generator().manual_seed(8)).to(DEV)
    wide = 0.1 * torch.randn(67, generator=torch.Generator().manual_seed(9)).to(DEV)
    for at in range(4):
        want = B.btx_moe_group_route(l, 6, bias=wide[at:at + 64].clone(), n_groups=4, topk_groups=2)
        got = B.btx_moe_group_route(l, 6, bias=wide[at:at + 64], n_groups=4, topk_groups=2)
        assert all(torch.equal(getattr(got, n), getattr(want, n)) for n in vars(want)), at


@gpu
def test_routes_on_two_streams_at_once():
    """Two calls in flight, each with its own workspace and outputs."""
    T, E, k = 5000, 128, 6
    ls = [torch.randn(T, E, generator=torch.Generator().manual_seed(i)).to(DEV) for i in (1, 2)]
    want = [B.btx_moe_group_route(l, k, n_groups=4, topk_groups=2) for l in ls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for l, s in zip(ls, streams):
            with torch.cuda.stream(s):
                got.append(B.btx_moe_group_route(l, k, n_groups=4, topk_groups=2))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert all(torch.equal(getattr(r, n), getattr(want[i % 2], n)) for n in vars(r)), i


@gpu
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("gs", ["top2", "max"])
def test_route_masked_experts(score, gs):
    rng = rng_of("masked", score, gs)
    l = rng.standard_normal((90, 40))
    l[rng.random((90, 40)) < 0.5] = -np.inf
    l[3] = -np.inf                                        # nothing left
    l[4, :] = -np.inf
    l[4, 17] = 0.5                                        # one expert, in a group of its own value
    l[5, 10:20] = -np.inf                                 # a whole group
    bias = torch.from_numpy(0.2 * rng.standard_normal(40)).float()
    for b in (None, bias):
        r, o = route_both(torch.from_numpy(l).float(), 6, score, b, 4, 2, gs)
        check_route(r, o)
        assert np.all(r.gates.cpu().numpy()[3] == 0.0)
        check_route(*route_both(torch.from_numpy(l).float(), 6, score, b))


@gpu
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_route_of_anything_stays_in_range(score):
    rng = rng_of("anything", score)
    l = rng.standard_normal((100, 64)).astype(np.float32) * 200
    l[rng.random(l.shape) < 0.1] = np.nan
    l[rng.random(l.shape) < 0.1] = np.inf
    l[rng.random(l.shape) < 0.1] = -np.inf
    l[7] = np.nan
    l[8] = 3.4e38
    r, o = route_both(torch.from_numpy(l), 8, score, None, 8, 3)
    idx = r.topk_idx.cpu().numpy()
    assert idx.min() >= 0 and idx.max() < 64 and all(len(set(row)) == 8 for row in idx)
    assert np.array_equal(np.sort(r.perm.cpu().numpy()), np.arange(800))
    for name in ("topk_idx", "counts", "perm"):
        assert np.array_equal(getattr(r, name).cpu().numpy(), o[name]), name
    assert torch.isfinite(r.gates).all() and torch.isfinite(r.scores).all()
    bias = torch.full((64,), float("nan"))
    idx = route_both(torch.from_numpy(l), 8, score, bias, 8, 3)[0].topk_idx.cpu().numpy()
    assert idx.min() >= 0 and idx.max() < 64 and all(len(set(row)) == 8 for row in idx)


@gpu
def test_route_without_scores_and_unaligned_rows():
    rng = rng_of("plain")
    l = torch.from_numpy(rng.standard_normal((70, 22))).bfloat16()      # rows of 44 bytes
    check_route(*route_both(l, 4, "softmax", None, 2, 1, with_scores=False))


@gpu
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 256, 16), (17, 60, 6), (65, 33, 4), (300, 64, 8), (5, 250, 3)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm,with_scores,dtype", [(True, False, torch.float32), (False, False, torch.bfloat16), (True, True, torch.float32),
                                                      (False, True, torch.float32)])
def test_route_backward(T, E, k, score, renorm, with_scores, dtype):
    rng = rng_of("bwd", T, E, k, score)
    l = torch.from_numpy(rng.standard_normal((T, E)) * 2).to(dtype)
    if T > 3:
        l[2, 1] = float("-inf")
    o = O.group_route(l.double().numpy(), k, score, renorm=renorm)
    dg = torch.from_numpy(rng.standard_normal((T, k))).float()
    ds = torch.from_numpy(0.1 * rng.standard_normal((T, E))).float() if with_scores else None
    want = O.group_route_backward(l.double().numpy(), o["topk_idx"], dg.double().numpy(), score, renorm, 2.5,
                                  None if ds is None else ds.double().numpy())
    from types import SimpleNamespace
    r = SimpleNamespace(topk_idx=torch.from_numpy(o["topk_idx"]).int().to(DEV))
    out = torch.full((T, E), float("nan"), dtype=dtype, device=DEV)
    got = B.btx_moe_group_route_backward(l.to(DEV), r, dg.to(DEV), SCORE[score], renorm, 2.5, None if ds is None else ds.to(DEV), out=out)
    # terms of size scale |dg| / z (+ |ds|) times s that cancel, each 64 steps off at most; bf16: one rounding more
    s = O.scores(l.double().numpy(), score)
    w = np.take_along_axis(s, o["topk_idx"], 1)
    size = 2.5 * np.abs(dg.double().numpy()).max(1) / ((w.sum(1)) if renorm else 1.0) + (0 if ds is None else np.abs(ds.numpy()).max(1))
    tol = 64 * 2.0 ** -23 * size[:, None] * 2 * s + 1e-37
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(got.cpu().double().numpy() - want) <= tol)
    again = l.to(DEV)                                     # in place
    B.btx_moe_group_route_backward(again, r, dg.to(DEV), SCORE[score], renorm, 2.5, None if ds is None else ds.to(DEV), out=again)
    assert torch.equal(again, got)


@gpu
def test_route_backward_passes_over_experts_out_of_range():
    from types import SimpleNamespace
    l = torch.randn(20, 12, generator=torch.Generator().manual_seed(3)).to(DEV)
    idx = torch.tensor([[1, 12], [-1, 3]] * 10, dtype=torch.int32, device=DEV)
    dl = B.btx_moe_group_route_backward(l, SimpleNamespace(topk_idx=idx), torch.ones(20, 2, device=DEV))
    assert torch.isfinite(dl).all()


# ---- the experts' gradients under another router ----------------------------------------------------------------


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d,f,E,k", [(1, 64, 64, 4, 2), (37, 64, 96, 8, 3), (300, 128, 264, 16, 4), (700, 256, 384, 4, 2)])
def test_backward_gates_is_the_layers_backward(T, d, f, E, k, dtype):
    """Beside btx_moe_ff_backward on the same routing: the same weight gradients bit for bit, and its dX where the router adds nothing."""
    from paper_2403_07816_amd import synth
    L = synth.make_layer(T, d, f, E, dtype=dtype, seed=5, device=DEV, unit_rms=True, with_dY=True)
    r = B.btx_moe_route(L["x"], L["W_router"], k=k)
    out, h1, h3 = B.btx_moe_ff_forward(L["x"], L["W1"], L["W3"], L["W2"], r)
    zero = torch.zeros_like(L["W_router"])
    a = B.btx_moe_ff_backward(L["dY"], L["x"], zero, L["W1"], L["W3"], L["W2"], r, h1, h3)
    b = B.btx_moe_ff_backward_gates(L["dY"], L["x"], L["W1"], L["W3"], L["W2"], r, h1, h3)
    for name in ("dW1", "dW3", "dW2"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    # (two sums of k terms in fp32, rounded to the rows' type)
    eps = torch.finfo(dtype).eps
    assert ((a.dX.float() - b.dX.float()).abs() <= eps * a.dX.float().abs() + k * 2.0 ** -22 * a.dX.float().abs().max()).all()
    frozen = B.btx_moe_ff_backward_gates(L["dY"], L["x"], L["W1"], L["W3"], L["W2"], r, h1, h3, frozen_experts=True)
    assert torch.equal(frozen.dX, b.dX) and torch.equal(frozen.dgates, b.dgates) and frozen.dW1 is None
    # <dY, FF_e(x)>, in float64 on the host; the kernel sums bf16 activations of a row of f, and products in fp32
    x, dY = L["x"].double().cpu(), L["dY"].double().cpu()
    W1, W3, W2 = (L[n].double().cpu() for n in ("W1", "W3", "W2"))
    idx = r.topk_idx.cpu().long()
    for t in range(0, T, max(1, T // 16)):
        for j in range(k):
            e = int(idx[t, j])
            a1, a3 = x[t] @ W1[e], x[t] @ W3[e]
            act = torch.nn.functional.silu(a1) * a3
            D = W2[e] @ dY[t]
            want, size = float(D @ act), float((D * act).norm()) + 1e-30
            # every term off by the roundings of h1, h3, D and the sums: 8 half steps of the rows' type, adding up at worst like their norm
            assert abs(float(b.dgates[t, j]) - want) <= (8 * eps / 2) * size * 2 + f * 2.0 ** -23 * size, (t, j)


@gpu
def test_training_step_of_a_layer_routed_from_logits():
    """Router product, routing, experts, and back, in fp32: against torch's gradients of the same step in float64."""
    T, d, f, E, k = 50, 64, 96, 12, 3
    g = torch.Generator().manual_seed(11)
    x, Wr, dY = torch.randn(T, d, generator=g), torch.randn(d, E, generator=g) / 8, torch.randn(T, d, generator=g)
    W1, W3 = torch.randn(E, d, f, generator=g) / 8, torch.randn(E, d, f, generator=g) / 8
    W2, bias = torch.randn(E, f, d, generator=g) / 10, torch.randn(E, generator=g) / 10
    X, WR, A, C, D = (t.to(DEV) for t in (x, Wr, W1, W3, W2))
    logits = X @ WR
    r = B.btx_moe_group_route(logits, k, bias=bias.to(DEV), n_groups=4, topk_groups=2, scale=2.5)
    out, h1, h3 = B.btx_moe_ff_forward(X, A, C, D, r)
    grads = B.btx_moe_ff_backward_gates(dY.to(DEV), X, A, C, D, r, h1, h3)
    dl = B.btx_moe_group_route_backward(logits, r, grads.dgates, scale=2.5)
    dX, dWr = grads.dX + dl @ WR.T, X.T @ dl

    leaves = [t.double().requires_grad_(True) for t in (x, Wr, W1, W3, W2)]
    xx, wr, a, c, b2 = leaves
    s = torch.sigmoid(xx @ wr)
    idx = r.topk_idx.cpu().long()
    w = s.gather(1, idx)
    gates = 2.5 * w / (w.sum(1, keepdim=True) + 1e-20)
    y = torch.zeros(T, d, dtype=torch.float64)
    for t in range(T):
        y[t] = sum(gates[t, j] * ((torch.nn.functional.silu(xx[t] @ a[e]) * (xx[t] @ c[e])) @ b2[e]) for j, e in enumerate(idx[t].tolist()))
    want = torch.autograd.grad((y * dY.double()).sum(), leaves)
    for name, got, exact in zip(("out", "x", "Wr", "W1", "W3", "W2"), (out, dX, dWr, grads.dW1, grads.dW3, grads.dW2), (y.detach(),) + want):
        err = (got.cpu().double() - exact).norm() / exact.norm()
        # fp32 sums of up to d, f or T terms: (depth of three products) sqrt(100) steps of 2^-24, with room for the cancelling ones
        assert err < 2e-5, (name, float(err))


@gpu
def test_route_on_another_stream_and_in_a_graph():
    lib = B.load_library()
    T, E, k = 300, 64, 8
    l = torch.randn(T, E, generator=torch.Generator().manual_seed(1)).to(DEV)
    bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(2)).to(DEV)
    kw = dict(bias=bias, n_groups=8, topk_groups=4)
    want = B.btx_moe_group_route(l, k, **kw)
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(4)).to(DEV)
    want_dl = B.btx_moe_group_route_backward(l, want, dg)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r = B.btx_moe_group_route(l, k, **kw)
    s.synchronize()
    assert all(torch.equal(getattr(r, n), getattr(want, n)) for n in vars(want))
    out, ws = B.alloc_group_routing(T, E, k, DEV), torch.empty(lib.btx_moe_group_route_workspace_bytes(T, E, k), dtype=torch.uint8, device=DEV)
    inp, dl = l.clone(), torch.empty_like(l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.btx_moe_group_route(inp, k, out=out, workspace=ws, **kw)
        B.btx_moe_group_route_backward(inp, out, dg, out=dl)
    for i in range(4):
        inp.copy_(torch.roll(l, i, 0))
        graph.replay()
        torch.cuda.synchronize()
        eager = B.btx_moe_group_route(inp, k, **kw)
        assert all(torch.equal(getattr(out, n), getattr(eager, n)) for n in vars(eager)), i
        assert torch.equal(dl, B.btx_moe_group_route_backward(inp, eager, dg)), i
        if i == 0:
            assert torch.equal(dl, want_dl)


@gpu
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,renorm,dtype", [(12, True, torch.float32), (33, False, torch.bfloat16), (256, True, torch.float32)])
def test_route_backward_takes_nothing_from_masked_experts(score, E, renorm, dtype):
    """Whatever reaches the scores or gates of masked experts (a loss of log s has an infinite gradient there): their gradients are 0 and
    the others' what they are without it."""
    from types import SimpleNamespace
    rng = rng_of("nothing", score, E)
    T, k = 40, 6
    l = rng.standard_normal((T, E))
    l[rng.random((T, E)) < 0.4] = -np.inf
    l[3] = -np.inf
    l[4] = -np.inf
    l[4, :2] = (0.5, np.nan)                               # fewer than k are left
    l = torch.from_numpy(l).to(dtype)
    masked = ~(l > -np.inf)
    idx = torch.from_numpy(O.group_route(l.double().numpy(), k, score, renorm=renorm)["topk_idx"])
    r = SimpleNamespace(topk_idx=idx.int().to(DEV))
    dg, ds = torch.from_numpy(rng.standard_normal((T, k))).float(), torch.from_numpy(rng.standard_normal((T, E))).float()
    at_gates = masked.gather(1, idx)
    assert at_gates.any()
    plain = [torch.where(at_gates, 0.0, dg), torch.where(masked, 0.0, ds)]
    for junk in (float("inf"), -float("inf"), float("nan"), 3e38):
        got = [torch.where(at_gates, junk, dg), torch.where(masked, junk, ds)]
        for with_scores in (False, True):
            want, have = (B.btx_moe_group_route_backward(l.to(DEV), r, a.to(DEV), SCORE[score], renorm, 2.5, b.to(DEV) if with_scores else None)
                          for a, b in (plain, got))
            assert torch.equal(have, want) and torch.isfinite(have).all() and (have.cpu()[masked] == 0).all(), (junk, with_scores)


@gpu
def test_route_past_32_bits():
    """More than 2^31 logits: the tokens of a small batch again and again."""
    T, n, E, k = (1 << 23) + 77, 1000, 256, 3
    few = torch.randn(n, E, generator=torch.Generator().manual_seed(6)).to(DEV)
    dg = torch.randn(n, k, generator=torch.Generator().manual_seed(7)).to(DEV)
    kw = dict(score_fn=B.BTX_SCORE_SOFTMAX, n_groups=8, topk_groups=4)
    want = B.btx_moe_group_route(few, k, **kw)
    times, whole = -(-T // n), T // n * n
    l = few.repeat(times, 1)[:T]
    r = B.btx_moe_group_route(l, k, **kw)

    def again(got, of):
        return torch.equal(got[:whole].view(-1, n, got.shape[1]), of.expand(whole // n, n, got.shape[1])) and torch.equal(got[whole:], of[:T - whole])

    for name in ("topk_idx", "gates", "scores"):
        assert again(getattr(r, name), getattr(want, name)), name
    flat = r.topk_idx.view(-1).long()
    assert torch.equal(r.counts.long(), torch.bincount(flat, minlength=E))
    perm = torch.sort(flat, stable=True).indices
    assert torch.equal(r.perm.long(), perm) and torch.equal(r.perm[r.inv_pos.view(-1).long()].long(), torch.arange(T * k, device=DEV))
    back = dict(score_fn=B.BTX_SCORE_SOFTMAX)
    assert again(B.btx_moe_group_route_backward(l, r, dg.repeat(times, 1)[:T], **back), B.btx_moe_group_route_backward(few, want, dg, **back))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d,f,E,k,cap", [(300, 128, 96, 64, 4, 0.5), (500, 64, 96, 4, 2, 0.7), (40, 64, 64, 5, 1, 1.0)])
def test_backward_gates_of_dropped_pairs(T, d, f, E, k, cap, dtype):
    """Pairs that a capacity limit has dropped have a gradient of 0, and the rest is as in the layer's own backward pass."""
    from paper_2403_07816_amd import synth
    L = synth.make_layer(T, d, f, E, dtype=dtype, seed=7, device=DEV, unit_rms=True, with_dY=True)
    r = B.btx_moe_route(L["x"], L["W_router"], k=k, capacity_factor=cap)
    dropped = r.inv_pos < 0
    assert dropped.any() and not dropped.all()
    _, h1, h3 = B.btx_moe_ff_forward(L["x"], L["W1"], L["W3"], L["W2"], r)
    args = (L["W1"], L["W3"], L["W2"], r, h1, h3)
    out = B.ExpertGrads(torch.empty_like(L["x"]), torch.full((T, k), float("nan"), device=DEV), *(torch.empty_like(w) for w in args[:3]))
    b = B.btx_moe_ff_backward_gates(L["dY"], L["x"], *args, out=out)
    a = B.btx_moe_ff_backward(L["dY"], L["x"], torch.zeros_like(L["W_router"]), *args)
    assert (b.dgates[dropped] == 0).all() and torch.isfinite(b.dgates).all() and (b.dgates[~dropped] != 0).any()
    for name in ("dW1", "dW3", "dW2"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    eps = torch.finfo(dtype).eps
    assert ((a.dX.float() - b.dX.float()).abs() <= eps * a.dX.float().abs() + k * 2.0 ** -22 * a.dX.float().abs().max()).all()
