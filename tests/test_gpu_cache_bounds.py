"""Selection by bounds whose ends lie the wrong way round, against the 64-bit oracle."""

import numpy as np
import pytest

from test_gpu_cache import HEADS, Select, bf16

pytestmark = pytest.mark.gpu


def _turned(s, share):
    """``share`` of the features of all bounds with lo and hi exchanged."""
    b = s.bounds.float().numpy()
    turn = s.rng.random(b[:, :, 0].shape) < share
    lo, hi = b[:, :, 0].copy(), b[:, :, 1].copy()
    b[:, :, 0], b[:, :, 1] = np.where(turn, hi, lo), np.where(turn, lo, hi)
    s.bounds = bf16(b)
    return s


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("share", [0.3, 1.0])
def test_select_takes_the_larger_product_of_either_bound(hq, hkv, d, share):
    rows = [(400, 3), (0, 5), (1023, 2), (9000, 1), (159, 1)]
    s = _turned(Select(hq, hkv, d, 16, rows, 100 * hq + hkv + d), share)
    s.check(9)
    s.check(40, 0, 0)


def test_select_does_not_see_which_bound_comes_first():
    s = Select(8, 2, 128, 16, [(30000, 1), (700, 2)], 3)
    want = s.run(50).cpu().numpy()
    assert np.array_equal(_turned(s, 1.0).run(50).cpu().numpy(), want)
    assert np.array_equal(_turned(s, 0.5).run(50).cpu().numpy(), want)
