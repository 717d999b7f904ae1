"""Workspace queries on the CPU: a buffer sized for the largest batch has to serve every smaller one."""
import pytest

SIZES = [(32, 32), (64, 96), (96, 4128), (128, 512), (128, 16384), (256, 512), (256, 1536), (384, 384), (384, 1536), (1152, 384),
         (1536, 384), (32, 16384), (4096, 1024), (1024, 4096), (16384, 4096)]


@pytest.fixture(scope="module")
def bm():
    from paper_2302_06058_b200 import build
    build.build()
    import paper_2302_06058_b200 as m
    m.lib()
    return m


@pytest.mark.parametrize("I,J", SIZES)
def test_a_buffer_for_the_largest_batch_serves_smaller_ones(bm, I, J):
    queries = (lambda T: bm.bimask_linear_workspace_bytes(T, I, J), lambda T: bm.bimask_workspace_bytes(T, I, J, 32),
               lambda T: bm.bimask_linear_workspace_bytes(T, J, I))
    for q in queries:
        last = 0
        for T in list(range(1, 700)) + list(range(700, 24000, 61)):
            n = q(T)
            assert n >= last, T
            last = n


def test_the_query_of_a_larger_batch_covers_more_splits_of_a_smaller_one(bm):
    """5632 tokens are cut into more pieces than 5696: a buffer for 5696 holds them, and less than they need is refused (on
    the host, before any launch)."""
    L, a = bm.lib(), 256                                     # an address that is never dereferenced
    T, I, J = 5632, 256, 1536
    need = 2 * T * J + 11 * I * J * 4                        # 88 token tiles of 64 in 11 pieces of eight
    assert bm.bimask_linear_workspace_bytes(5696, I, J) >= need
    assert L.bimask_wgrad_ckpt(a, a, a, T, I, J, a, a, need - 1, a, None) == bm.binding.BIMASK_EINVAL
    assert f"workspace too small ({need - 1} bytes, need {need})" in bm.bimask_last_error()
