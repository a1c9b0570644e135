"""What the calls of block-scaled 8-bit floats launch for given sizes, without a GPU (see launches.py)."""
import math
import os
import random

import pytest

from paper_2403_07816_amd import binding as B

from launches import P, PLENTY, compiled, launches
from test_fp8 import LAYERS, MATMULS
from test_fp8_edges import CUT_PRODUCTS, EDGE_PRODUCTS, TALL_EXPERTS, TALL_LAYERS

MAX_THREADS = (1 << 32) - 1     # of one launch and direction of the grid
UP_FEW, FEW16, FEW64 = "f8_few_kernel<true, 2, 2, 2, float>", "f8_few_kernel<false, {}, 1, 4, {}>", "f8_few_kernel<false, {}, 4, 2, {}>"
MID, TALL = "f8_mid_kernel<(MidMode){}, {}>", "f8_tile_kernel<(TileMode){}, {}>"


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    if not os.path.exists(B.LIB_PATH):
        from paper_2403_07816_amd.build import build
        build(verbose=False)
    folder = tmp_path_factory.mktemp("launches")
    return lambda *calls: launches(list(calls), str(folder))


def name(launch):
    return launch.kernel.replace("btx::", "")


def fits(launch):
    return all(0 < g and g * b <= MAX_THREADS for g, b in zip(launch.grid, launch.block)) and launch.lds <= 160 * 1024 and launch.grid[1] <= 65535


def tensor(fn, batch, rows, cols, axis, dtype=B.BTX_BF16, block_rows=1):
    if fn == "q":
        return ("btx_fp8_quantize", [P, dtype, batch, rows, cols, axis, block_rows, P, P, 0])
    return ("btx_fp8_dequantize", [P, P, dtype, batch, rows, cols, axis, P, 0])


def matmul(M, N, K, dtype=B.BTX_BF16):
    return ("btx_fp8_matmul", [P] * 4 + [M, N, K, 0, P, dtype, P, PLENTY, 0])


def layer(T, d, f, E, k):
    return ("btx_moe_ff_forward_fp8", [P] * 8 + [T, d, f, E, k] + [P] * 7 + [PLENTY, 0])


@pytest.mark.parametrize("fn", ["q", "d"])
def test_tensors(record, fn):
    for batch, rows, cols, axis, br in ((1, 1, 1, 1, 1), (3, 301, 4096, 1, 1), (1, 1 << 20, 1 << 15, 1, 1), (1, 32, 1, 0, 1), (4, 4096, 11008, 0, 128),
                                        (65535, 32, 65, 0, 1), (65535, 5, 1000, 1, 128), (1, 1 << 19, 1 << 18, 0, 1), (1, 1 << 28, 100, 1, 128)):
        (rc, found), = record(tensor(fn, batch, rows, cols, axis, block_rows=br))
        assert rc == 0 and len(found) == 1 and fits(found[0]), (batch, rows, cols, axis)
        if axis == 0:
            assert found[0].grid[:2] == (math.ceil(rows / 128) * math.ceil(cols / 128), batch)


def test_norm(record):
    for T in (1, 5, 16384, (1 << 26) - 1):
        for d, per in ((8, 1), (512, 1), (520, 1), (2056, 2), (4104, 4), (8200, 8), (16384, 8)):
            for dtype in (B.BTX_F32, B.BTX_BF16):
                if T * d > 1 << 38:
                    continue
                (rc, found), = record(("btx_rmsnorm_fp8", [P, P, dtype, P, 1e-5, T, d, P, 2 * P, P, P, P, 0]))
                rows = 4 if d <= 512 else 1
                assert rc == 0 and all(fits(x) for x in found) and sum(x.grid[0] for x in found) == math.ceil(T / rows)
                assert len(found) == (1 if T < 1 << 22 else math.ceil(T / rows / (1 << 22)))
                assert name(found[0]).endswith(f"{64 if d <= 512 else 256}, {per}>")


# rows, columns, depth; the kernel of bf16 results and that of fp32 ones; whether either is cut along K
PATHS = [
    (1, 11008, 4096, "few16", "few16", False), (12, 11008, 4096, "few16", "few16", False), (16, 11008, 4096, "mid64", "few16", True),
    (33, 11008, 1024, "few16", "few16", False), (16, 4096, 11008, "few16", "few16", False), (17, 4096, 11008, "mid64", "mid64", True),
    (24, 4096, 4096, "few16", "few16", False), (32, 4096, 4096, "few16", "few16", False), (33, 4096, 4096, "mid64", "mid64", True),
    (16, 512, 8192, "mid64", "mid64", True), (16, 1024, 8192, "few16", "few16", False), (5, 33000, 136, "few64", "few16", False),
    (30, 33000, 300, "few64", "few16", False), (40, 33000, 520, "mid64", "few16", False), (128, 1024, 1024, "few16", "few16", False), (129, 1024, 1024, "few16", "few16", False), (256, 1024, 2048, "few16", "few16", False),
    (257, 1024, 2048, "mid64", "mid64", True), (256, 1024, 2056, "mid64", "mid64", True), (700, 4096, 8300, "mid64", "mid128", False),
    (64, 4096, 11008, "mid64", "mid64", True), (1024, 4096, 4096, "mid64", "mid64", False), (1025, 4096, 4096, "mid128", "mid128", False),
    (2049, 4096, 4096, "tall", "mid128", False), (1376, 4096, 4001, "mid128", "mid128", False), (16384, 11008, 4096, "tall", "mid128", False),
    (2048, 4096, 11008, "tall", "mid128", True), (1000, 4000, 4090, "mid64", "mid64", False), (1100, 4104, 2040, "mid128", "mid128", False),
    (500, 16600, 4096, "tall", "mid128", False),
    # of few columns and many rows
    (65, 16, 2048, "few16", "few16", False), (4095, 64, 2048, "few16", "few16", False), (4095, 64, 2304, "mid64", "mid64", True),
    (4096, 64, 2048, "few16", "few16", False), (4097, 64, 2048, "mid64", "mid64", True), (5000, 16, 8192, "few16", "few16", False), (16384, 8, 520, "few64", "few16", False),
    (64, 8, 8192, "mid64", "mid64", True), (65, 8, 8192, "mid64", "mid64", True)]


def kind(launch):
    n = name(launch)
    if n.startswith("f8_few_kernel<false"):
        return {"1, 4": "few16", "4, 2": "few64"}[", ".join(n.split(", ")[2:4])]
    return f"mid{n.split(', ')[1][:-1]}" if n.startswith("f8_mid") else "tall"


@pytest.mark.parametrize("M,N,K,bf16,f32,cut", PATHS)
def test_products(record, M, N, K, bf16, f32, cut):
    for dtype, want in ((B.BTX_BF16, bf16), (B.BTX_F32, f32)):
        (rc, found), = record(matmul(M, N, K, dtype))
        assert rc == 0 and all(fits(x) for x in found) and kind(found[0]) == want, name(found[0])
        sums = len(found) == 2
        assert sums == (cut and (want == bf16 or dtype == B.BTX_BF16)), (name(found[0]), len(found))
        assert not sums or name(found[1]).startswith("f8_add_slices_kernel")


def all_kernels():
    ot = ("float", "unsigned short")
    few = {FEW16.format(rb, t) for rb in (2, 4) for t in ot} | {FEW64.format(rb, ot[1]) for rb in (2, 4)} | {UP_FEW}
    return few | {MID.format(m, bm) for m in range(3) for bm in (64, 128)} | {TALL.format(m, a) for m in range(2) for a in ("false", "true")}


def test_the_shapes_of_the_parity_tests_reach_every_kernel(record):
    calls = [matmul(*c, dtype) for c in MATMULS for dtype in (B.BTX_BF16, B.BTX_F32)] + [layer(*c) for c in LAYERS]
    reached, cut = set(), set()
    for rc, found in record(*calls):
        assert rc == 0 and all(fits(x) for x in found)
        names = [name(x) for x in found]
        reached |= set(names)
        if any(n.startswith("f8_add") for n in names) or any(n.startswith("combine_kernel") and n.endswith("false, true>") for n in names):
            cut |= {n for n in names if "mid" in n or "tile" in n}
    assert all_kernels() <= reached, all_kernels() - reached
    assert cut >= {MID.format(1, 64), MID.format(2, 64), TALL.format(1, "false")}, cut


def test_any_sizes_fit_their_launches_and_workspaces(record):
    rng, lib = random.Random(7), B.load_library()
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    shapes = [(log(1, 1 << 20), 8 * log(1, 1 << 17), log(1, 1 << 20), rng.randint(0, 1)) for _ in range(300)]
    shapes = [s for s in shapes if s[0] * s[1] < 1 << 37 and s[0] * s[2] < 1 << 39 and s[1] * s[2] < 1 << 39]
    for (M, N, K, dtype), (rc, found) in zip(shapes, record(*[matmul(*s) for s in shapes])):
        assert rc == 0 and all(fits(x) for x in found), (M, N, K, dtype)
        assert len(found) == 1 or lib.btx_fp8_matmul_workspace_bytes(M, N, K) >= 2 * M * N * 4, (M, N, K)
    shapes = []
    while len(shapes) < 300:
        E = rng.choice([1, 2, 4, 8, 33, 64, 256])
        k, d, f, T = rng.randint(1, min(E, 16)), 8 * log(1, 1 << 14), 8 * log(1, 1 << 14), log(1, 1 << 20)
        if T * (d + 127) // 128 * 128 < (1 << 32) - 2048 and T * k * max(d, f) < 1 << 38 and E * d * f < 1 << 38 and T * k < (1 << 28) - 256:
            shapes.append((T, d, f, E, k))
    for (T, d, f, E, k), (rc, found) in zip(shapes, record(*[layer(*s) for s in shapes])):
        assert rc == 0 and all(fits(x) for x in found), (T, d, f, E, k)
        names, R = [name(x) for x in found], T * k
        kept = R * (lib.btx_fp8_code_pitch(f) + lib.btx_fp8_scale_pitch(f))
        ws = lib.btx_moe_ff_forward_fp8_workspace_bytes(T, d, f, E, k)
        assert len(found) == (3 if names[0].startswith("f8_tile") else 4)
        assert ws >= kept + R * d * 2
        if len(found) == 4:                                # the activations in fp32, in front of y
            assert names[1].startswith("f8_quantize_rows_kernel<float") and ws >= kept + R * f * 4, (T, d, f, E, k)
        if names[-1].endswith("false, true>"):             # sums of at least two ranges
            assert ws >= kept + 2 * R * d * 4, (T, d, f, E, k)


def test_limits(record):
    (rc, found), = record(matmul((1 << 28) - 257, 8, 64))
    assert rc == 0 and fits(found[0])
    for call, want in ((matmul(1 << 28, 8, 64), 2), (matmul(1 << 20, 1 << 19, 64, B.BTX_F32), 2), (matmul(1 << 20, 1 << 19, 64), 0)):
        (rc, found), = record(call)
        assert rc == want and (rc or all(fits(x) for x in found)) and (not rc or not found)
    (rc, found), = record(layer((1 << 25) - 64, 128, 8, 8, 8))
    assert rc == 0 and all(fits(x) for x in found)


def test_layers_of_whole_16_blocks_take_each_kernel(record):
    """(whose workgroups begin at different places of K there)"""
    ups = ((5, 2048, 200, 4, 2), UP_FEW), ((90, 2040, 520, 4, 2), MID.format(0, 64)), ((150, 4096, 264, 1, 1), MID.format(0, 128)), ((900, 2048, 1200, 2, 2), TALL.format(0, "true"))
    for (shape, up), (rc, found) in zip(ups, record(*[layer(*s) for s, _ in ups])):
        assert shape in LAYERS and rc == 0 and name(found[0]) == up, (shape, name(found[0]))


def norm(T, d, dtype):
    return ("btx_rmsnorm_fp8", [P, P, dtype, P, 1e-5, T, d, P, 2 * P, P, P, P, 0])


def test_every_kernel_that_is_compiled_can_be_launched(record, tmp_path):
    types = (B.BTX_F32, B.BTX_BF16)
    calls = [matmul(*c, dtype) for c in MATMULS for dtype in types] + [layer(*c) for c in LAYERS]
    calls += [tensor(fn, 2, 301, cols, axis, dtype, br) for fn in "qd" for cols in (129, 264) for axis in (0, 1) for dtype in types for br in (1, 128)]
    calls += [norm(3, d, dtype) for d in range(8, 16385, 8) for dtype in types]
    reached = {name(x) for rc, found in record(*calls) for x in found}
    have = {k for k in compiled(str(tmp_path)) if k.startswith("f8_")}
    assert len(have) > 20 and have <= reached, sorted(have - reached)


def test_the_largest_turned_product(record):
    """A workgroup of 256 threads for 16 rows, with fp32 results: the largest launch of all."""
    (rc, found), = record(matmul((1 << 28) - 257, 8, 64, B.BTX_F32))
    assert rc == 0 and name(found[0]) == FEW16.format(2, "float") and fits(found[0]) and found[0].grid[0] * found[0].block[0] == (1 << 32) - 4096


def test_layers_of_the_most_columns_and_experts(record):
    """64 rows of each in tiles of 64 rows and 64 columns would be 2^24 workgroups of 256 threads, which no launch has."""
    for T, tall in ((2047, False), (2048, True)):
        (rc, found), = record(layer(T, 8, 2097120, 256, 8))
        assert rc == 0 and name(found[0]).startswith("f8_tile_kernel") == tall and all(fits(x) for x in found), T


def test_the_shapes_of_the_edge_tests_reach_the_kernels_that_they_are_for(record):
    seen = set()
    for M, N, K, *kinds in EDGE_PRODUCTS:
        for dtype, want in zip((B.BTX_BF16, B.BTX_F32), kinds):
            (rc, found), = record(matmul(M, N, K, dtype))
            got = kind(found[0]) + (" apart" if name(found[0]) == TALL.format(1, "true") else "")
            assert rc == 0 and got == want, (M, N, K, dtype, got)
            seen.add(name(found[0]))
    assert all_kernels() - seen == {UP_FEW, MID.format(0, 64), MID.format(0, 128), TALL.format(0, "false"), TALL.format(0, "true")}
    for M, N, K, *kinds in CUT_PRODUCTS:
        for dtype, want in zip((B.BTX_BF16, B.BTX_F32), kinds):
            (rc, found), = record(matmul(M, N, K, dtype))
            if want:
                assert rc == 0 and kind(found[0]) == want and len(found) == 2 and name(found[1]).startswith("f8_add_slices_kernel"), (M, N, K, dtype, name(found[0]))


def test_the_edge_tests_of_tall_layers_take_tall_tiles(record):
    ups = {"tall": TALL.format(0, "false"), "tall apart": TALL.format(0, "true")}
    downs = {"tall": TALL.format(1, "false"), "mid64": MID.format(1, 64)}
    for (shape, up, down, cut) in TALL_LAYERS + [(TALL_EXPERTS, "tall", "tall", False)]:
        (rc, found), = record(layer(*shape))
        assert rc == 0 and [name(x) for x in found[:2]] == [ups[up], downs[down]], (shape, found)
        assert name(found[2]).startswith("combine_kernel") and name(found[2]).endswith("false, true>") == cut, (shape, name(found[2]))
