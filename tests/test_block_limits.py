"""Sizes at the ends of their types in the operators around attention, on the CPU: the library's checks (with pointers that are never
followed) and the binding's."""
import pytest
import torch

from tests import test_block_refusals as R
from tests.test_block_refusals import lib, on_cpu  # noqa: F401
from paper_2605_08962_amd import binding

INT_MAX = 2 ** 31 - 1


@pytest.mark.parametrize("inverse", [False, True])
def test_numbers_of_pairs_beyond_the_head(lib, inverse):  # noqa: F811
    """Their double does not fit the type they come in."""
    for pairs in (33, 1 << 29, 1 << 30, (1 << 30) + 32, INT_MAX):
        assert R._rotary(lib, None, inverse, num_pairs=pairs) == R.SHAPE, pairs
    for d in (2, 3, 65, 512):
        wide = dict(head_dim=d, q_stride=4 * d, k_stride=2 * d, v_stride=2 * d, q_out_stride=4 * d, k_out_stride=2 * d, v_out_stride=2 * d)
        assert R._rotary(lib, None, inverse, num_pairs=d // 2 + 1, **wide) == R.SHAPE
        assert R._rotary(lib, None, inverse, num_pairs=d // 2, total_tokens=0, **wide) == R.OK
