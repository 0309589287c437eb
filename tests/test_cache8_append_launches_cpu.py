"""What appending to the cache of 8-bit blocks launches where C_max is a bound far above the rows that there are, without a GPU."""
import pytest

from test_launches_cpu import BF16, F32, launches, recorder   # noqa: F401 (a fixture)
from test_serving_launches_cpu import SHAPE, append


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("U,T,C,L,Hkv,block", [(1, 100, 1 << 27, 1 << 27, 1, 8), (128, 128, 65000, 65000, 2, 16), (1, 1, (1 << 30) - 1, (1 << 30) - 1, 1, 8),
                                               (3, 1000, 500, 1 << 20, 4, 16), (3, 1000, 1 << 20, 70, 4, 16)])
def test_blocks_that_the_rows_can_touch(recorder, U, T, C, L, Hkv, block, dt):
    """A user has at most T rows, C_max and L_max: no workgroup for blocks that so many rows do not reach."""
    (one,) = launches(recorder, append(U, T, C, L, Hkv, 16, dt, block=block))
    rows = min(T, C, L)
    assert one.grid == (rows + 2 * block - 2) // block


@pytest.mark.parametrize("over", [0, 1])
def test_the_most_blocks(recorder, over):
    """2^23 - 1 blocks times heads are a launch, one more are refused."""
    rows = 8 * ((1 << 23) - 1) - 14 + 7 + over      # touch 2^23 - 1 blocks of 8, and one more
    call = append(1, rows, rows, rows, 1, 16, BF16)
    recorder.launch_clear()
    assert call(recorder) == (SHAPE if over else 0) and recorder.launch_count() == (0 if over else 1)
