"""zo_paged_attention of 17 to 32 rows for a key head, two groups of 16 in one workgroup, and of one more: lengths around tiles
and pages, ranges that are joined, padding, and values that are not finite."""
import numpy as np
import pytest

from _paged import attend, check_attention
from test_gpu_paged_attention import test_values_that_are_not_finite_stay_with_the_rows_that_see_them as not_finite

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kvh,dh", [(5, 1, 128), (8, 8, 128), (4, 2, 64), (32, 1, 64), (33, 1, 128)])
@pytest.mark.parametrize("rows", [17, 31, 32, 33])
def test_rows(rows, heads, kvh, dh, dt, cache):
    rng = np.random.default_rng(rows + heads)
    most = -(-rows // (heads // kvh))
    news = [most, 1, 0, most - 1, most, most, 1]
    lens = [most, 40, 0, 65, 300 + most, most // 2, 1100]     # the sixth begins before position 0
    got, ref, mag = attend(rng, dt, lens, news, 16, heads, kvh, dh, cache, pad=8, rows_behind=2)
    check_attention(got, ref, mag, dt, (rows, heads))


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("news,heads", [([10], 2), ([8], 4), ([31], 1), ([16], 2)])
def test_values_that_are_not_finite(news, heads, cache):
    not_finite(news, heads, cache)
