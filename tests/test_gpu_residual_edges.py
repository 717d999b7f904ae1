"""The residual junction where it is easily wrong: ties, values that are not finite, results in the place of inputs, the ends of
the range of magnitudes.  Statements, tolerances and random problems are those of test_gpu_residual.py."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
import test_gpu_residual as R
from test_gpu_residual import TYPES, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alpha", [1.7, 0.3, 1.0])
@pytest.mark.parametrize("stream", TYPES)
@pytest.mark.parametrize("T,C", [(24, 4096), (31, 96), (3, 16384)])
def test_the_scaled_stream_is_a_product_of_its_own(T, C, stream, alpha):
    """alpha x is rounded to fp32 before the branch is added.  A decimal alpha has an fp32 neighbour beside it; the rounding takes the
    neighbour's excess off again where alpha x has few bits, so that x' lies on a tie where alpha x + y does, and goes to the even side
    (in one fused step the excess decides every tie the same way)."""
    q = Problem(T, C, 0, 2, stream, scale=False, alpha=alpha)
    f = q.forward()
    want = (q.d["x"].float() * q.alpha + q.d["y"].float()).to(q.dt)
    assert torch.equal(f["xo"], want)
    q.check_forward(f)
