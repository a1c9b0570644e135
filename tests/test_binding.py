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
