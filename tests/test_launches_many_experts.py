"""What the calls of many experts and of 4-bit experts launch for given sizes, without a GPU (see launches.py)."""
import math
import os

import pytest

from paper_2403_07816_amd import binding as B

from launches import P, PLENTY, launches

MAX_THREADS = (1 << 32) - 1     # of one launch and direction of the grid


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    if not os.path.exists(B.LIB_PATH):
        from paper_2403_07816_amd.build import build
        build(verbose=False)
    folder = tmp_path_factory.mktemp("launches")
    return lambda *calls: launches(list(calls), str(folder))


def fits(launch):
    return all(0 < g and g * b <= MAX_THREADS for g, b in zip(launch.grid, launch.block)) and launch.lds <= 160 * 1024


def route(T, E, k, G=1, keep=1, dtype=B.BTX_F32):
    return ("btx_moe_group_route", [P, dtype, P, T, E, k, B.BTX_SCORE_SIGMOID, G, keep, B.BTX_GROUP_TOP2, 1, 1.0] + [P] * 8 + [PLENTY, 0])


def route_backward(T, E, k, dtype=B.BTX_F32):
    return ("btx_moe_group_route_backward", [P, dtype, P, P, P, T, E, k, B.BTX_SCORE_SOFTMAX, 1, 1.0, P, 0])


def tensor(fn, batch, rows, cols, axis, dtype=B.BTX_BF16):
    if fn == "btx_mx4_quantize":
        return (fn, [P, dtype, batch, rows, cols, axis, P, P, 0])
    return (fn, [P, P, dtype, batch, rows, cols, axis, P, 0])


def layer(T, d, f, E, k):
    return ("btx_moe_ff_forward_mx4", [P] * 7 + [T, d, f, E, k] + [P] * 7 + [PLENTY, 0])


@pytest.mark.parametrize("T,tokens", [(1, 64), (64, 64), (65, 16), (301, 16), (4096, 16), (4097, 32), (8192, 32), (8193, 64), (32768, 64),
                                      (32769, 128), (1 << 20, 2048), ((1 << 30) - 1, 1 << 21)])
def test_route_workgroups(record, T, tokens):
    """As many as there are compute units before a workgroup takes more tokens; never more than 512."""
    (rc, found), = record(route(T, 64, 1))
    assert rc == 0 and len(found) == (1 if T <= 64 else 2) and all(fits(x) for x in found)
    assert found[0].kernel.startswith("group_select_kernel") and found[0].grid[0] == math.ceil(T / tokens) <= 512
    assert found[0].block[0] == min(1024, 64 * math.ceil(min(T, tokens) / 4))
    if T > 64:
        assert found[1].kernel == "group_scatter_kernel" and found[1].grid == found[0].grid
        assert B.load_library().btx_moe_group_route_workspace_bytes(T, 64, 1) >= found[0].grid[0] * 64 * 4


@pytest.mark.parametrize("E,G,most", [(1, 1, 4), (64, 1, 4), (65, 1, 8), (256, 1, 16), (256, 8, 16), (64, 8, 4), (256, 16, 16), (252, 9, 32), (250, 10, 32),
                                      (255, 15, 32), (60, 4, 4)])
def test_route_experts_of_a_lane(record, E, G, most):
    (rc, found), = record(route(100, E, 1, G))
    assert rc == 0 and found[0].kernel == f"group_select_kernel<float, {most}, 1>"


def test_route_backward_workgroups(record):
    for T in (1, 16, 17, 16384, (1 << 28) - 16):
        (rc, found), = record(route_backward(T, 8, 1))
        assert rc == 0 and len(found) == 1 and fits(found[0]) and found[0].grid[0] == math.ceil(T / 16)


@pytest.mark.parametrize("fn", ["btx_mx4_quantize", "btx_mx4_dequantize"])
def test_tensor_workgroups(record, fn):
    for batch, rows, cols, axis in ((1, 1, 32, 1), (3, 301, 4096, 1), (1, 1 << 20, 1 << 15, 1), (1, 32, 1, 0), (4, 4096, 11008, 0), (65535, 32, 65, 0),
                                    (1, 1 << 24, 16320, 0), (2, 64, 4194240, 0)):
        (rc, found), = record(tensor(fn, batch, rows, cols, axis))
        assert rc == 0 and len(found) == 1 and fits(found[0]), (batch, rows, cols, axis)
        if axis == 0:
            pieces = math.ceil(cols / 64)
            assert found[0].grid[0] % pieces == 0 and found[0].grid[0] // pieces * 256 >= rows and found[0].grid[1] == batch
            assert found[0].kernel.endswith(", true>" if cols % 8 == 0 else ", false>")


def tile_rows(found):
    up = found[1].kernel
    assert up.startswith(("mx4_few_kernel<true, ", "mx4_tile_kernel<true>"))
    return 256 if "tile" in up else 16 * int(up.split(", ")[1])


@pytest.mark.parametrize("T,d,f,E,k,rows", [
    (1, 4096, 11008, 4, 2, 32), (48, 4096, 11008, 4, 2, 32), (49, 4096, 11008, 4, 2, 32), (50, 4096, 11008, 4, 2, 64), (63, 4096, 11008, 4, 2, 64),
    (64, 4096, 11008, 4, 2, 256), (301, 4096, 11008, 4, 2, 256), (64, 4096, 1376, 32, 8, 32), (128, 4096, 1376, 32, 8, 256),
    (51, 4096, 11008, 1, 1, 64), (52, 4096, 11008, 1, 1, 256), (999, 1024, 1024, 2, 1, 64), (1000, 1024, 1024, 2, 1, 256), (3000, 128, 64, 2, 1, 64),
    (16384, 4096, 11008, 4, 2, 256), (1 << 18, 65536, 32, 1, 1, 64)])
def test_layer_tile_height(record, T, d, f, E, k, rows):
    (rc, found), = record(layer(T, d, f, E, k))
    assert rc == 0 and len(found) == 4 and all(fits(x) for x in found)
    assert found[0].kernel == ("layer_begin_kernel<true>" if rows == 256 else "layer_begin_kernel<false>")
    assert tile_rows(found) == rows and found[3].kernel.startswith("combine_kernel")
    down = found[2].kernel
    assert down == "mx4_tile_kernel<false>" if rows == 256 else down.startswith(f"mx4_few_kernel<false, {rows // 16}, ")
    if rows < 256:                                          # one for every tile that there may be and 32 columns
        tiles = min(T * k // rows + min(E, T * k), T * k)
        assert found[1].grid[:2] == (tiles, f // 32) and found[2].grid[:2] == (tiles, d // 32)
        assert [x.block[0] for x in found[1:3]] == [512 if K >= 8192 else 256 for K in (d, f)]


@pytest.mark.parametrize("T,d,f,E,k,up,down,cut", [
    (301, 4096, 11008, 4, 2, 6 * 86 + 8, (6 * 16 + 8) * 4, True),       # two rounds of tiles have a workgroup each
    (301, 4096, 8192, 4, 2, 6 * 64 + 8, (6 * 16 + 8) * 4, True),
    (301, 4096, 2048, 4, 2, 6 * 16 + 8, 6 * 16 + 8, False),             # sums of fewer than 16 k tiles
    (16384, 4096, 11008, 4, 2, 256, 256, False), (16384, 4096, 1376, 32, 8, 256, 256, False)])
def test_layer_tiles(record, T, d, f, E, k, up, down, cut):
    (rc, found), = record(layer(T, d, f, E, k))
    assert rc == 0 and tile_rows(found) == 256
    want = [min(n, 256) if n > 512 else n for n in (up, down)]
    assert [x.grid[0] for x in found[1:3]] == want
    assert found[3].kernel.endswith("true>" if cut else "false>")


def test_layer_limits(record):
    """What is refused is refused before anything is launched, and what is not can be launched."""
    cases = [((1 << 26) - 1, 32, 32, 4, 4), ((1 << 26) - 1, 32, 32, 1, 1), (1 << 26, 32, 32, 1, 1), (1 << 24, 32, 32, 16, 16), (1 << 19, 2097120, 32, 1, 1),
             (4, 2097120, 2097120, 1, 1), (4, 32, 2097152, 1, 1), (4, 2097152, 32, 1, 1), (1 << 18, 2097120, 64, 2, 2), (1 << 19, 32, 2097120, 1, 1)]
    for case, (rc, found) in zip(cases, record(*[layer(*c) for c in cases])):
        assert (rc == 0 and len(found) == 4 and all(fits(x) for x in found)) or (rc in (1, 2) and not found), (case, rc, found)


@pytest.mark.parametrize("T,d,rows", [
    ((1 << 23) - 3, 1024, 256), ((1 << 23) - 2, 1024, 64), ((1 << 23) - 1, 1024, 64),
    ((1 << 24) - 8, 512, 256), ((1 << 24) - 2, 512, 64), ((1 << 25) - 16, 256, 256), ((1 << 25) - 3, 256, 64), ((1 << 20) - 1, 8192, 256), (1 << 20, 8192, 64)])
def test_token_rows_of_tall_tiles_have_offsets_of_32_bits(record, T, d, rows):
    """A tall tile's lane finds 16 bytes of a token row at row * d/2 + chunk (112 at most) + 1024 from its base."""
    (rc, found), = record(layer(T, d, 32, 2, 1))
    assert rc == 0 and len(found) == 4 and all(fits(x) for x in found)
    assert tile_rows(found) == rows
    if rows == 256:
        assert (T - 1) * (d // 2) + 112 + 1024 < 1 << 32


MOST_TOKENS = (1 << 26) - 4     # the combining kernel has a wavefront for a token


@pytest.mark.parametrize("T,d,f,E,k,status", [
    (MOST_TOKENS, 32, 32, 1, 1, 0), (MOST_TOKENS, 32, 32, 256, 1, 0), ((1 << 26) - 65, 32, 32, 4, 4, 0), (MOST_TOKENS - 1, 512, 32, 1, 1, 0),
    (MOST_TOKENS + 1, 32, 32, 1, 1, 1), ((1 << 26) - 1, 32, 32, 1, 1, 1), (MOST_TOKENS, 544, 32, 1, 1, 2),
    ((1 << 14) - 1, 2097120, 32, 1, 1, 0), (1 << 14, 2097120, 32, 1, 1, 2), ((1 << 26) - 64, 32, 32, 4, 4, 1)])
def test_layer_takes_what_its_limits_allow(record, T, d, f, E, k, status):
    """T <= 2^26 - 4, T k < 2^28 - 256 (refused as arguments), T * scale pitch of d < 2^30 (not supported)."""
    (rc, found), = record(layer(T, d, f, E, k))
    assert rc == status and len(found) == (4 if status == 0 else 0) and all(fits(x) for x in found)


def backward_gates(T, d, f, E, k, dtype=B.BTX_F32):
    return ("btx_moe_ff_backward_gates", [P] * 5 + [dtype, d * f, d * f, T, d, f, E, k] + [P] * 11 + [dtype, P, PLENTY, 0])


def test_backward_gates_limits(record):
    (most, _), (more, found) = record(backward_gates(MOST_TOKENS, 8, 8, 1, 1), backward_gates(MOST_TOKENS + 1, 8, 8, 1, 1))
    assert (most, more, found) == (2, 2, [])               # (the experts' products refuse the former)


def test_experts_that_a_layer_takes(record):
    """Routing from logits and the layer of 4-bit experts: 256; the experts' gradients and the bf16 and fp32 layers: 64."""
    def forward(E):
        return ("btx_moe_ff_forward", [P] * 4 + [B.BTX_BF16, 4096, 4096, 100, 64, 64, E, 4] + [P] * 8 + [P, PLENTY, 0])

    calls = [route(100, 256, 4), layer(100, 64, 64, 256, 4), forward(64), backward_gates(100, 64, 64, 64, 4),
             route(100, 257, 4), layer(100, 64, 64, 257, 4), forward(65), backward_gates(100, 64, 64, 65, 4)]
    for i, (rc, found) in enumerate(record(*calls)):
        assert (rc, bool(found)) == ((0, True) if i < 4 else (1, False)), i
