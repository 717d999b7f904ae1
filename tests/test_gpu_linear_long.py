"""Reductions that the CTA-pair kernel cuts into several tensor-core chains: exact results where sums are exact (two to six
chains, even and uneven ones, one accumulator and two, one and several tiles per pair), and the same bytes with and without
residual, in place and again."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from test_gpu_linear import bf, cuda, operand, run_linear
from test_gpu_linear import test_forward_exact_on_small_integers as exact_on_small_integers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,I,J,N,M", [(512, 2560, 3104, 2, 4), (512, 2560, 4128, 2, 4), (2495, 512, 6816, 2, 4), (900, 4096, 4096, 2, 4),
                                       (900, 2080, 16384, 1, 4), (131, 8224, 4096, 2, 4), (11521, 1184, 3104, 2, 4), (6001, 1536, 9248, 2, 4),
                                       (3101, 1184, 1696, 4, 8), (300, 8192, 4128, 4, 8), (11521, 1184, 1568, 4, 8), (2100, 2080, 6144, 4, 8)])
def test_exact(T, I, J, N, M):
    assert bm.bimask_debug_linear_plan(T, I, J, N > 2)[0] == 2 and (J + 127) // 128 > (12 if N > 2 else 24)
    exact_on_small_integers(T, I, J, N, M)


@pytest.mark.parametrize("act", [bm.ACT_GELU, bm.ACT_SILU])
@pytest.mark.parametrize("T,I,J,N,M", [(5003, 1536, 4096, 2, 4), (2495, 512, 6816, 2, 4), (700, 2080, 3104, 4, 8)])
def test_repeated_and_in_place(T, I, J, N, M, act):
    rng = np.random.default_rng(T)
    vals, hw, _ = operand(rng.standard_normal((I, J)), N, M)
    X, _ = bf(rng.standard_normal((T, J)))
    R, _ = bf(rng.standard_normal((T, I)))
    bias = cuda(rng.standard_normal(I), torch.float32)
    Y, q, s = run_linear(vals, hw, X, bias, act, R, T, I, J, True)
    for _ in range(3):
        same = R.clone()
        Y2, q2, s2 = run_linear(vals, hw, X, bias, act, same, T, I, J, True, Y=same)
        assert torch.equal(Y, Y2) and torch.equal(q, q2) and torch.equal(s, s2)
    Y3, _, _ = run_linear(vals, hw, X, bias, act, None, T, I, J, False)
    assert bool(((Y3.float() + R.float() - Y.float()).abs() <= 2.0 ** -7 * (Y3.float().abs() + R.float().abs()) + 1e-6).all())
