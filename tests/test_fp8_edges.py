"""Block-scaled 8-bit floats where the kernels of many rows, the matrix cores' own 8-bit product and sums that are cut along K can go wrong."""
import pytest
import torch

from paper_2403_07816_amd import binding as B

from test_fp8 import BF, DEV, make_layer, rng_of
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
