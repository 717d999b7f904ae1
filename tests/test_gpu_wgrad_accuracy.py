"""The accuracy that the weight gradient from a checkpoint promises: no more than 512 tokens (32 MMAs of 16) in one tensor-core
chain, the rest added in fp32 with rounding to nearest.  One chain over all tokens would be off by 9e-6 (8192 tokens, mixed
signs) and by several 1e-5 (positive products)."""
import pytest
import torch

import paper_2302_06058_b200 as bm

pytestmark = pytest.mark.gpu


def operands(T, I, J, positive):
    """(dY, q, s, the checkpoint's values)."""
    g = torch.Generator(device="cuda").manual_seed(T + I)
    if positive:
        dY = (torch.rand(T, I, generator=g, device="cuda") + 0.5).to(torch.bfloat16)
        q = torch.randint(40, 128, (T, J), generator=g, device="cuda", dtype=torch.int8)
    else:
        dY = torch.randn(T, I, generator=g, device="cuda").to(torch.bfloat16)
        q = (torch.randn(T, J, generator=g, device="cuda") * 40).clamp(-127, 127).round().to(torch.int8)
    s = torch.randint(120, 123, (T, J // 32), generator=g, device="cuda", dtype=torch.uint8)
    x = q.double() * torch.exp2(s.double() - 127.0).repeat_interleave(32, 1)
    return dY, q, s, x


def weight_gradient(dY, q, s, T, I, J):
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, I, J), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dW = torch.empty(I, J, device="cuda")
    bm.bimask_wgrad_ckpt(dY, q, s, T, I, J, dW, ws, ws.numel(), st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return dW.double()


# 81 output tiles of 256 x 256: one work item over all tokens; few tiles: the tokens are cut into pieces as well
@pytest.mark.parametrize("T,I,J", [(8192, 2304, 2304), (9000, 2304, 2304), (16500, 2304, 2304), (16500, 512, 4608), (12608, 384, 1536)])
def test_mixed_signs(T, I, J):
    """A chain of T tokens is off by about 1.1e-9 T relative: 0.6e-6 at 512, and independent chains add up to no more; the
    fp32 additions add at most sqrt(T / 512) 2^-24 = 0.35e-6."""
    dY, q, s, x = operands(T, I, J, False)
    want = dY.double().t() @ x
    off = float((weight_gradient(dY, q, s, T, I, J) - want).norm() / want.norm())
    print(f"{T} {I} {J}: {off:.2e}")
    assert off <= 1e-6


@pytest.mark.parametrize("T,I,J", [(8192, 2304, 2304), (16500, 2304, 2304), (16500, 512, 4608), (12608, 384, 1536)])
def test_positive_products(T, I, J):
    """Allowed: one unit of the last place per MMA of a chain and 32 for the products inside them (2^-23 of the segment's sum
    each), an addition rounded to nearest per segment and per piece of the tokens."""
    dY, q, s, x = operands(T, I, J, True)
    want = dY.double().t() @ x
    off = float(((weight_gradient(dY, q, s, T, I, J) - want).abs() / want).max())
    allowed = (32 + 32) * 2.0 ** -23 + (T / 512 + 64 + 1) * 2.0 ** -24
    print(f"{T} {I} {J}: {off:.2e} of {allowed:.2e}")
    assert off <= allowed
