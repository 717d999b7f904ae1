"""Which kernel bimask_linear_fwd takes and how it cuts the reduction, on the device at hand, and exact results at sizes that the
rules treat differently."""
import pytest

import paper_2302_06058_b200 as bm
from test_gpu_linear import test_forward_exact_on_small_integers as exact_on_small_integers

pytestmark = pytest.mark.gpu

WIDTHS = (128, 512, 1024, 1536, 1920, 2048, 2304, 2560, 3584, 4096, 4608, 5120, 6144, 9472, 9600, 16384)


@pytest.mark.parametrize("J", [384, 1024, 2048, 4096, 16384])
@pytest.mark.parametrize("T", [1, 24, 128])
def test_a_split_reduction_fits_the_device_in_one_round(T, J):
    """The clusters of all tiles are resident at once, with as many CTAs each as that allows (at most eight, four 128-wide pieces
    of the reduction or more for each)."""
    for I in WIDTHS:
        kernel, splits, tiles, fit = bm.bimask_debug_linear_plan(T, I, J)
        assert kernel == 0 and tiles == (I + 127) // 128
        pieces = (J + 127) // 128
        assert splits == 1 or (tiles <= fit and 4 * splits <= pieces), (I, splits, fit)
        if pieces >= 32 and 8 * tiles <= 100:                # room for clusters of eight on any device of 148 SMs
            assert splits == 8, (I, splits)


# 16 to 48 row tiles: clusters of 6, 5, 4, 3 and 2 CTAs
@pytest.mark.parametrize("T,I,J,N,M", [(3, 2048, 4096, 2, 4), (9, 2560, 4128, 2, 4), (24, 3584, 4096, 2, 4), (24, 4608, 4096, 4, 8),
                                       (40, 3040, 2080, 2, 4), (100, 6144, 2048, 2, 4)])
def test_exact_at_every_cluster_size(T, I, J, N, M):
    exact_on_small_integers(T, I, J, N, M)
