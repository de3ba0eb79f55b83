"""The feed-forward's tile kernel where a pair of CTAs has several tiles, wide and
narrow, element by element against the float64 oracle with the bounds of
test_gpu_ffn.py; which tiles each size gets is checked in test_ffn_tiles.py."""
import pytest

from ffn_tiling import SIZES
from test_gpu_ffn import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [c[0] for c in SIZES], ids=str)
def test_ffn_several_tiles_to_a_pair(case):
    check(*make(case, 20 + case[0]), case[3])
