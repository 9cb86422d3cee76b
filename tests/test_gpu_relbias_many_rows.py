"""Relative bias rows that are many more than are on the chip at once, dealt forth and back over the workgroups: rows of every
way that they are held."""
import pytest

from test_gpu_relbias import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,h,q,k", [(4, 16, 1201, 30), (2, 8, 1500, 300), (1, 4, 5003, 516), (1, 2, 7001, 1001), (1, 1, 13000, 1028),
                                     (1, 1, 5600, 2050), (1, 1, 2900, 4097), (1, 1, 2600, 5000), (1, 1, 1700, 8200)])
@pytest.mark.parametrize("bidirectional", [False, True])
def test_many_rows(b, h, q, k, bidirectional):
    check(b, h, q, k, [0, 1, 3, 9], bidirectional, causal=not bidirectional, window=0 if q < 3000 else 700, q_starts=[max(0, k - q)] * b)
