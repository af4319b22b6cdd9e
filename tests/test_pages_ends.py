"""The page format at the ends of its range (CPU): what append writes of finite numbers reads back finite."""
import numpy as np
import pytest
import torch

from oracle import pages as P

F32_MAX, BF16_MAX = float(np.finfo(np.float32).max), 255 * 2.0 ** 120
TOPS = [F32_MAX, BF16_MAX, 248 * 2.0 ** 120, 240 * 2.0 ** 120, 232 * 2.0 ** 120, 224 * 2.0 ** 120]


@pytest.mark.parametrize("top", TOPS)
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_values_read_back_finite(top, sign):
    """As float32 and bf16, and within a half step (2^-4) of what was appended; what is not finite is NaN beside them."""
    x = np.zeros((1, 64, 4))
    x[0, :4] = [[sign * top, 1.0, -sign * top / 2, 0], [np.inf, -np.inf, np.nan, 2.0 ** 120], [0, 0, 0, 0], [1e30, 0, 0, 0]]
    pages = P.Pages(np.zeros((1, 1, 1, 2, 256), np.uint8), np.ones((1, 1, 1, 2)))
    pages.append(0, [0], 0, x, x)
    k, v, _ = pages.read(0, [0], 64)
    assert np.array_equal(k, v, equal_nan=True)
    assert np.array_equal(np.isnan(k), ~np.isfinite(x))
    ok = np.isfinite(x)
    half = pages.scales[0, 0, 0, 0] * 2.0 ** -10  # of the subnormal codes
    assert np.all(np.abs(k - x)[ok] <= np.maximum(2.0 ** -4 * np.abs(x), half)[ok])
    for dt in (torch.float32, torch.bfloat16):
        assert torch.from_numpy(k[ok]).to(dt).isfinite().all()
        assert np.array_equal(torch.from_numpy(k[ok]).to(dt).double().numpy(), k[ok])


def test_growing_to_the_last_scale():
    """Codes of a page whose scale grows to 2^120 stay below the last value."""
    x = np.full((1, 1, 4), 448 * 2.0 ** 119)
    pages = P.Pages(np.zeros((1, 1, 1, 2, 256), np.uint8), np.ones((1, 1, 1, 2)))
    pages.append(0, [0], 0, x, x)
    assert np.all(pages.scales == 2.0 ** 119)
    pages.append(0, [0], 1, np.full((1, 1, 4), F32_MAX), -x)
    k, v, _ = pages.read(0, [0], 2)
    assert np.array_equal(k[0], np.array([[224.0], [240.0]]).repeat(4, 1) * 2.0 ** 120) and np.array_equal(v[0, 1], -x[0, 0])


def test_page_sets_of_other_types_are_refused():
    """Codes in other 8-bit types would be taken for e4m3."""
    tadm = pytest.importorskip("paper_2609_37924_amd")
    scale = torch.zeros(4, 2, 3, 2)
    for dt in (torch.float8_e5m2, torch.int8, torch.bool, torch.float8_e4m3fnuz):
        with pytest.raises(ValueError, match="float8_e4m3fn codes"):
            tadm.page_set(torch.zeros(4, 2, 3, 2, 64 * 16, dtype=dt), scale)
    for dt in (torch.uint8, torch.float8_e4m3fn):
        assert tadm.page_set(torch.zeros(4, 2, 3, 2, 64 * 16, dtype=dt), scale).head_dim == 16
