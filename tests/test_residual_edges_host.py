"""CPU checks of the arguments of dropout and the residual junction that only a caller can get right (no GPU is touched)."""
import pytest
import torch


@pytest.fixture(scope="module")
def bm():
    from paper_2302_06058_b200 import build
    build.build()
    import paper_2302_06058_b200 as m
    m.lib()
    return m


def test_status_word_and_limits_of_the_debug_helper(bm):
    L, inval = bm.lib(), bm.binding.BIMASK_EINVAL
    a = {k: 256 for k in bm.binding._RESIDUAL_POINTERS}
    a["ws_bytes"] = 1 << 24
    n0 = bm.bimask_launch_count()
    assert bm.make_residual_args(4, 64, a).status_word is None and bm.make_residual_args(4, 64, {**a, "status_word": 260}).status_word == 260
    odd = bm.make_residual_args(4, 64, {**a, "status_word": 258}, post=bm.NORM_RMS, pre=bm.NORM_LAYER)
    for call in (L.bimask_residual_norm_fwd, L.bimask_residual_norm_bwd):
        assert call(odd, None) == inval and "status_word" in bm.bimask_last_error()
    good = bm.make_residual_args(4, 64, a, post=bm.NORM_RMS, pre=bm.NORM_LAYER)
    for limits in ((-1, -1, 0), (1 << 33, -1, 0), (0, -2, 0), (0, 32, 0), (0, 3, -1), (0, 3, 4)):
        for backward in (0, 1):
            assert L.bimask_debug_residual_give_up(good, backward, *limits, None) == inval and "out of range" in bm.bimask_last_error()
    assert L.bimask_debug_residual_give_up(None, 0, 0, -1, 0, None) == inval
    assert bm.bimask_launch_count() == n0


def test_a_counter_is_one_64_bit_number_on_the_device(bm):
    """Another type would be read as eight bytes of something else, host memory faults when the kernel runs."""
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(1), torch.zeros(2, dtype=torch.int64), torch.zeros(0, dtype=torch.int64)):
        with pytest.raises(ValueError, match="counter"):
            bm.make_dropout(0.1, 1, 0, bad)
    with pytest.raises(ValueError, match="device"):
        bm.make_dropout(0.1, 1, 0, torch.zeros(1, dtype=torch.int64))
    assert bm.make_dropout(0.1, 1, 0, 4096).counter == 4096 and bm.make_dropout(0.1, 1).counter is None


def test_parameters_are_tensors_like_any_other(bm):
    """A gate of three dimensions and a workspace that are registered parameters of a module."""
    def parameter(*shape, dtype=torch.bfloat16):
        return torch.nn.Parameter(torch.zeros(*shape, dtype=dtype), requires_grad=False)

    gate = parameter(4, 1, 64)
    a = bm.make_residual_args(4, 64, {"gate": gate, "dgate": gate.detach().clone(), "ws": parameter(1000, dtype=torch.float32)})
    assert (a.gate_pitch, a.ws_bytes, a.gate) == (64, 4000, gate.data_ptr())
    assert bm.make_residual_args(4, 64, {"gate": parameter(4, 128).detach()[:, :64]}).gate_pitch == 128
