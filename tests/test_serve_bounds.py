"""The stated bounds of products with a step per token: what lies within them is taken, what passes one of them is refused.  Checked on
the host before anything is enqueued; a call within the bounds ends at a check behind them."""
import pytest

import paper_2609_17380_amd.canon as C

BASE = 1 << 44


def gemm(m, n, k=0, lda=None, ldb=None, ldc=None):
    """The status of a product whose y overlaps sa: CANON_EINVAL, if its sizes are taken."""
    far = [BASE + (i << 56) for i in range(5)]
    return C.lib().canon_gemm_i8_tokens(m, n, k, far[0], k if lda is None else lda, far[4], far[2], k if ldb is None else ldb, far[3],
                                        C.F32, far[4], n if ldc is None else ldc, None)


@pytest.mark.parametrize("m,n", [(64 << 23, 1), (64 << 23, 8), (64 << 13, 8 << 10), (1, 8 << 23), (64, 8 << 23), (64 << 3, 8 << 20)])
def test_sizes_at_the_bound(m, n):
    assert gemm(m, n) == C.EINVAL


@pytest.mark.parametrize("m,n", [((64 << 23) + 1, 1), (64 << 23, 9), (1, (8 << 23) + 1), (65, 8 << 23), ((64 << 13) + 1, 8 << 10),
                                 ((1 << 31) + 1, 1), (1, (1 << 31) + 1)])
def test_sizes_behind_it(m, n):
    assert gemm(m, n) == C.EUNSUPPORTED


def test_strides():
    assert gemm(1 << 20, 8, lda=1 << 20) == C.EINVAL and gemm(1 << 20, 8, lda=(1 << 20) + 1) == C.EUNSUPPORTED
    assert gemm(8, 1 << 20, ldb=1 << 20) == C.EINVAL and gemm(8, 1 << 20, ldb=(1 << 20) + 1) == C.EUNSUPPORTED
    assert gemm(1 << 20, 8, ldc=1 << 20) == C.EINVAL and gemm(1 << 20, 8, ldc=(1 << 20) + 1) == C.EUNSUPPORTED
