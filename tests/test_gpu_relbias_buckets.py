"""The bias table's gradient where a bucket has about as many keys as one pair of lanes sums: the first bucket after the query
has a key less than the one before it (distance 0 is before), so the two sides of one distance may be summed in different ways."""
import pytest

from test_gpu_relbias import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("s", [1, 20, 33, 34, 66, 100, 300, 700])
@pytest.mark.parametrize("starts", [[0, 33], [0, 34], [0, 32, 65], [0, 33, 66], [0, 0, 33], [0, 0, 33, 33, 66], [0, 33, 34, 67]])
def test_both_sides(s, starts):
    check(2, 3, s, s, starts, True, causal=False)
    check(1, 2, s, s, starts, True, causal=False, window=40)
    check(1, 2, s, s, starts, False, causal=False)
    check(1, 2, s, s, starts, False, causal=True)


@pytest.mark.parametrize("q,k", [(20, 1100), (12, 2050), (6, 4099), (900, 1100), (500, 2300)])
@pytest.mark.parametrize("starts", [[0, 33], [0, 33, 66]])
def test_rows_over_several_wavefronts(q, k, starts):
    check(1, 2, q, k, starts, True, causal=False, q_starts=[k // 2])
    check(1, 2, q, k, starts, True, causal=False, q_starts=[k - q])
