"""What binding.py hands to the library: sizes that have 32 bits there, workspaces of any dtype, outputs that nothing else fills."""
from types import SimpleNamespace

import pytest
import torch

from paper_2403_07816_amd import binding as B

gpu = pytest.mark.gpu
DEV = "cuda:0"


@gpu
@pytest.mark.parametrize("dtype", [torch.uint8, torch.float32, torch.int64])
def test_workspace_of_any_dtype(dtype):
    """A workspace is as long as its bytes are."""
    lib = B.load_library()
    T, d, f, E, k = 100, 64, 96, 4, 2
    g = torch.Generator().manual_seed(1)
    x, W, b = (torch.randn(s, generator=g).to(DEV) for s in ((T, d), (d, E), (T, E)))
    W1, W3, W2 = (torch.randn(s, generator=g).to(DEV) / 8 for s in ((E, d, f), (E, d, f), (E, f, d)))

    def ws(nbytes):
        size = torch.empty(0, dtype=dtype).element_size()
        return torch.empty(-(-nbytes // size), dtype=dtype, device=DEV)

    def same(a, c):
        return all(torch.equal(u, v) for u, v in zip(vars(a).values(), vars(c).values()))

    r = B.btx_moe_route(x, W, k=k, workspace=ws(lib.btx_moe_route_workspace_bytes(T, d, E, k)))
    assert same(r, B.btx_moe_route(x, W, k=k))
    out, h1, h3 = B.btx_moe_ff_forward(x, W1, W3, W2, r, workspace=ws(lib.btx_moe_ff_forward_workspace_bytes(T, d, f, E, k, B.BTX_F32)))
    assert torch.equal(out, B.btx_moe_ff_forward(x, W1, W3, W2, r)[0])
    back = ws(lib.btx_moe_ff_backward_workspace_bytes(T, d, f, E, k, B.BTX_F32))
    assert same(B.btx_moe_ff_backward(x, x, W, W1, W3, W2, r, h1, h3, workspace=back), B.btx_moe_ff_backward(x, x, W, W1, W3, W2, r, h1, h3))
    assert same(B.btx_moe_ff_backward_gates(x, x, W1, W3, W2, r, h1, h3, workspace=back), B.btx_moe_ff_backward_gates(x, x, W1, W3, W2, r, h1, h3))
    assert same(B.btx_moe_group_route(b, k, workspace=ws(lib.btx_moe_group_route_workspace_bytes(T, E, k))), B.btx_moe_group_route(b, k))
    gain, xb = torch.ones(d, device=DEV), x.bfloat16()
    rn, xn, rstd = B.btx_moe_norm_route(x, gain, 1e-5, W, k=k, workspace=ws(lib.btx_moe_route_workspace_bytes(T, d, E, k)))
    assert same(rn, B.btx_moe_norm_route(x, gain, 1e-5, W, k=k)[0])
    for a, c in zip(B.btx_rmsnorm_backward(x, x, gain, rstd, workspace=ws(lib.btx_rmsnorm_backward_workspace_bytes(T, d))),
                    B.btx_rmsnorm_backward(x, x, gain, rstd)):
        assert torch.equal(a, c)
    Q = [B.btx_mx4_quantize(w, axis=-2) for w in (W1, W3, W2)]
    assert torch.equal(B.btx_moe_ff_forward_mx4(xb, *Q, r, workspace=ws(lib.btx_moe_ff_forward_mx4_workspace_bytes(T, d, f, E, k))),
                       B.btx_moe_ff_forward_mx4(xb, *Q, r))


def shaped(*shape, dtype=torch.float32):
    """Of any size, in no memory."""
    return torch.zeros(1, dtype=dtype).expand(shape)


def group_out(T, E, k):
    i32 = torch.int32
    return B.GroupRouting(shaped(T, k, dtype=i32), shaped(T, k), None, shaped(E, dtype=i32), shaped(E + 1, dtype=i32), shaped(T * k, dtype=i32),
                          shaped(T, k, dtype=i32))


def route_out(T, E, k):
    i32 = torch.int32
    return B.Routing(shaped(T, k, dtype=i32), shaped(T, k), shaped(T, E), shaped(E, dtype=i32), shaped(E + 1, dtype=i32), shaped(T * k, dtype=i32),
                     shaped(T, k, dtype=i32), shaped(E), shaped(E), shaped(1))


MANY = 2 ** 32 + 8         # rows: 8 in 32 bits
EXPERTS = [torch.zeros(4, 16, 32), torch.zeros(4, 16, 32), torch.zeros(4, 32, 16)]
H = shaped(2 * MANY, 32)


def mx4(E, n, K):
    return B.Mx4(shaped(E, n, K // 2, dtype=torch.uint8), shaped(E, n, 16, dtype=torch.uint8), K)


@pytest.mark.parametrize("call", [
    lambda: B.btx_moe_group_route(shaped(MANY, 4), 2, out=group_out(MANY, 4, 2)),
    lambda: B.btx_moe_group_route(shaped(8, 4), 2 ** 32 + 2, out=group_out(8, 4, 2)),
    lambda: B.btx_moe_group_route(shaped(8, 4), 2, score_fn=2 ** 32, out=group_out(8, 4, 2)),
    lambda: B.btx_moe_group_route(shaped(8, 4), 2, n_groups=2 ** 32 + 1, out=group_out(8, 4, 2)),
    lambda: B.btx_moe_group_route(shaped(8, 4), 2, n_groups=1 - 2 ** 32, out=group_out(8, 4, 2)),
    lambda: B.btx_moe_group_route_backward(shaped(MANY, 4), group_out(MANY, 4, 2), shaped(MANY, 2), out=shaped(MANY, 4)),
    lambda: B.btx_moe_ff_forward_mx4(shaped(MANY, 32, dtype=torch.bfloat16), mx4(4, 64, 32), mx4(4, 64, 32), mx4(4, 32, 64), group_out(MANY, 4, 2),
                                     out=shaped(MANY, 32, dtype=torch.bfloat16)),
    lambda: B.btx_moe_ff_backward_gates(shaped(MANY, 16), shaped(MANY, 16), *EXPERTS, group_out(MANY, 4, 2), H, H,
                                        out=B.ExpertGrads(shaped(MANY, 16), shaped(MANY, 2), None, None, None)),
    lambda: B.btx_moe_route(shaped(MANY, 16), shaped(16, 4), out=route_out(MANY, 4, 2)),
    lambda: B.btx_moe_route(shaped(8, 16), shaped(16, 4), k=2 ** 32 + 2, out=route_out(8, 4, 2)),
    lambda: B.btx_moe_route_noalloc(shaped(MANY, 16), shaped(16, 4), route_out(MANY, 4, 2)),
    lambda: B.btx_moe_norm_route(shaped(MANY, 16), shaped(16), 1e-5, shaped(16, 4), out=route_out(MANY, 4, 2), xn=shaped(MANY, 16), rstd=shaped(MANY)),
    lambda: B.btx_rmsnorm_backward(shaped(MANY, 16), shaped(MANY, 16), shaped(16), shaped(MANY), dH=shaped(MANY, 16)),
    lambda: B.btx_mix_experts(*EXPERTS, B.BTX_MIX_SPLIT, C=2 ** 32 + 2),
    lambda: B.btx_moe_ff_forward(shaped(MANY, 16), *EXPERTS, route_out(MANY, 4, 2), out=shaped(MANY, 16), save=False),
    lambda: B.btx_moe_ff_backward(shaped(MANY, 16), shaped(MANY, 16), shaped(16, 4), *EXPERTS, route_out(MANY, 4, 2), H, H, frozen_experts=True,
                                  out=B.Grads(shaped(MANY, 16), shaped(16, 4), shaped(4), None, None, None))])
def test_sizes_past_32_bits_are_refused(call):
    """The library's sizes are ints: what does not fit one would be another size there."""
    with pytest.raises(ValueError, match="32 bits"):
        call()


def test_outputs_of_routing_from_logits_are_not_filled_first():
    """The call writes every entry of them; only without tokens it writes none, and counts and offsets are 0 already."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Calls(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            names.append(func.overloadpacket.__name__)
            return func(*args, **(kwargs or {}))

    names = []
    with Calls():
        B.alloc_group_routing(5, 8, 2, "cpu")
    assert set(names) == {"empty"}
    r = B.alloc_group_routing(0, 8, 2, "cpu")
    assert r.counts.tolist() == [0] * 8 and r.offsets.tolist() == [0] * 9 and r.topk_idx.shape == (0, 2)
