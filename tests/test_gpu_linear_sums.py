"""How far the sums of the linear-layer operators are from exact ones.

A result in bf16 hides the error of the sum behind it; here the bias takes the exact sum away, so that the result IS the
error.  All products are positive (the worst case of sums that are cut off instead of rounded)."""
import pytest
import torch

import paper_2302_06058_b200 as bm

pytestmark = pytest.mark.gpu


def positive_operand(I, J, dense, seed):
    """(vals, hw_meta, the same matrix in fp64 on the GPU), all kept weights in [0.5, 2]."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = torch.rand(I, J, generator=g, device="cuda") * 1.5 + 0.5
    b = bm.alloc_layer_buffers(1, I, J, 1, dense=dense)
    N, M = (4, 8) if dense else (2, 4)
    bm.bimask_fwd_mask(W, I, J, N, M, b["maskbits_f"], b["vals_f"], None if dense else b["meta_f"], None if dense else b["hw_meta_f"])
    if dense:
        return b["vals_f"], None, b["vals_f"].view(I, J)
    words = b["maskbits_f"].view(I, -1)
    bits = ((words.unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=words.dtype)) & 1).view(I, -1)[:, :J]
    return b["vals_f"], b["hw_meta_f"], W.to(torch.bfloat16) * bits.to(torch.bfloat16)


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("T", [3, 24, 50, 100])
def test_few_tokens_sum_long_reductions_in_short_chains(T, dense):
    """75 row tiles: no split, one CTA adds up all 16384 products.  Allowed: what a chain of 512 products may be off (one unit
    of the last place per MMA of 16 and 32 for the products inside them, 2^-23 of the segment's sum each), 32 additions
    rounded to nearest, and the rounding of the bias.  One chain over everything is off by more."""
    I, J = 9504, 16384
    vals, hw, Wm = positive_operand(I, J, dense, 5)
    x = (torch.rand(J, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda") + 0.5).to(torch.bfloat16)
    exact = torch.cat([Wm[i:i + 1056].double() @ x.double() for i in range(0, I, 1056)])
    X = x.expand(T, J).contiguous()
    Y = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bias = -exact.float()
    bm.bimask_linear_fwd(X, vals, hw, bias, bm.ACT_NONE, None, T, I, J, Y, None, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    off = (Y.double() - (exact + bias.double())).abs() / exact
    allowed = ((512 / 16 + 32) * 2.0 ** -23 + (J / 512 + 1) * 2.0 ** -24) * (1 + 2.0 ** -8)
    print(f"T {T} dense {dense}: worst {off.max().item():.2e}, mean {off.mean().item():.2e}, allowed {allowed:.2e}")
    assert float(off.max()) <= allowed


@pytest.mark.parametrize("T,I,J,dense", [(700, 2048, 16384, False), (900, 4096, 16384, False), (8192, 1536, 16384, False), (1200, 4096, 16384, True)])
def test_pairs_sum_long_reductions_in_several_chains(T, I, J, dense):
    """CTA pairs: chains of at most 96 MMAs.  Allowed: one unit of the last place per MMA of a chain and 32 for the products inside
    them (2^-23 of the chain's sum each), an addition per chain, the rounding of the bias.  One chain over everything is off by more."""
    assert bm.bimask_debug_linear_plan(T, I, J, dense)[0] == 2
    vals, hw, Wm = positive_operand(I, J, dense, 5)
    x = (torch.rand(J, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda") + 0.5).to(torch.bfloat16)
    exact = torch.cat([Wm[i:i + 1024].double() @ x.double() for i in range(0, I, 1024)])
    bias = -exact.float()
    Y = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bimask_linear_fwd(x.expand(T, J).contiguous(), vals, hw, bias, bm.ACT_NONE, None, T, I, J, Y, None, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    off = (Y.double() - (exact + bias.double())).abs() / exact
    chains = -(-J // (12 * 128 if dense else 24 * 128))
    allowed = ((96 + 32) * 2.0 ** -23 + (chains + 1) * 2.0 ** -24) * (1 + 2.0 ** -8)
    print(f"{T} {I} {J} dense {dense}: worst {off.max().item():.2e}, allowed {allowed:.2e}")
    assert float(off.max()) <= allowed
