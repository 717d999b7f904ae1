"""Layers of at most 128 output rows with more than 128 tokens: a long reduction is split instead of walked by a handful of CTAs."""
import pytest
import torch

import paper_2302_06058_b200 as bm
from test_gpu_linear import test_forward_exact_on_small_integers as exact_on_small_integers
from test_gpu_linear_sums import positive_operand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,I,J,N,M", [(129, 64, 4096, 2, 4), (129, 128, 16384, 2, 4), (1001, 128, 4128, 2, 4), (700, 96, 8192, 1, 4),
                                       (300, 32, 4096, 2, 4), (2048, 96, 8192, 2, 4), (129, 128, 4096, 4, 8), (515, 96, 8224, 4, 8),
                                       (9000, 128, 384, 2, 4), (9000, 64, 1184, 4, 8)])
def test_exact(T, I, J, N, M):
    exact_on_small_integers(T, I, J, N, M)


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("T", [129, 1000, 8192])
def test_long_reductions_are_split(T, dense):
    for I in (32, 64, 128):
        for J in (4096, 16384):
            assert bm.bimask_debug_linear_plan(T, I, J, dense)[0] == 0, (I, J)
        assert bm.bimask_debug_linear_plan(T, I, 384, dense)[0] == 1, I


@pytest.mark.parametrize("dense", [False, True])
def test_their_sums_are_as_near_as_those_of_few_tokens(dense):
    """129 tokens and 128 share the kernel: the bias takes the exact sum of positive products away, the result is the error.
    Allowed: what chains of 32 MMAs may be off, one addition per chain and per CTA, the rounding of the bias."""
    T, I, J = 129, 128, 16384
    vals, hw, Wm = positive_operand(I, J, dense, 5)
    x = (torch.rand(J, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda") + 0.5).to(torch.bfloat16)
    exact = Wm.double() @ x.double()
    bias = -exact.float()
    Y = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bimask_linear_fwd(x.expand(T, J).contiguous(), vals, hw, bias, bm.ACT_NONE, None, T, I, J, Y, None, None, st)
    off = (Y.double() - (exact + bias.double())).abs() / exact
    assert int(st.item()) == 0
    assert float(off.max()) <= ((32 + 32) * 2.0 ** -23 + (J / 512 + 9) * 2.0 ** -24) * (1 + 2.0 ** -8)
