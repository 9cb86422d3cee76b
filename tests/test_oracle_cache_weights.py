"""R26 against the formula where the tokens' values, or the channels of a query, are of very different sizes: a key counts by what
it adds to the row."""
import numpy as np
import pytest

import oracle
from serve_bounds import OUTLIERS, SPREADS, attention_bound, outlier_case, spread_case
from serve_util import from_bf16


@pytest.mark.parametrize("kind,size", SPREADS)
def test_values_of_different_sizes(kind, size):
    c, q = spread_case(kind, size)
    K, Q = 1024, q.shape[1]
    got = from_bf16(c.attention(q, K, 0.125, [K - Q], [Q], [K])).astype(np.float64)
    want, bound = attention_bound(c, q, 0.125, [K - Q], [Q], [K])
    assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / bound)
    if kind == "none":  # the row is one of the other keys': rounding to bf16 alone leaves 1.7e-3
        rms = np.sqrt(((got - want) ** 2).mean(-1) / (want ** 2).mean(-1))
        assert (rms <= 2.5e-3).all()


@pytest.mark.parametrize("times,bf16", OUTLIERS)
def test_channels_of_different_sizes(times, bf16):
    c, q = outlier_case(times, bf16)
    K, Q = 700, q.shape[1]
    got = from_bf16(c.attention(q, K, 0.125, [K - Q], [Q], [K])).astype(np.float64)
    want, bound = attention_bound(c, q, 0.125, [K - Q], [Q], [K])
    assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / bound)
    # rounding to bf16 alone leaves 1.7e-3; at 10^4 the largest channel passes 2^15, the others come as multiples of 2^-7, and 0.29 of
    # that on 63 channels, times a key's 1 and the scale, leaves a score off by 2.2e-3 more
    if times <= 1e3:
        assert (np.sqrt(((got - want) ** 2).mean(-1) / (want ** 2).mean(-1)) <= 2.5e-3).all()


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_scores_are_products_of_query_and_scale(scale):
    # a query and a scale of sizes whose product is an ordinary score's
    c, q = spread_case("all", 1.0, K=300)
    plain = c.attention(q, 300, 0.125, [297], [3], [300])
    other = c.attention(q * np.float32(2.0 ** -100 if scale > 1 else 2.0 ** 100), 300,
                        0.125 * (2.0 ** 100 if scale > 1 else 2.0 ** -100), [297], [3], [300])
    assert np.array_equal(plain, other)


def test_exp2():
    # the polynomial within 9.4e-8 with its coefficients rounded, and five fused steps, each off by 2^-24 of at most 1.42; p, which
    # they are parts of, at least 0.7: the last by 2^-24 / 0.7, those before it by a half, a quarter, .. of as much
    x = np.concatenate((np.linspace(-127, 0, 2000001), -np.linspace(0, 1, 400001))).astype(np.float32)
    e, want = oracle.exp2(x).astype(np.float64), 2.0 ** x.astype(np.float64)
    tiny = x < -126
    assert (np.abs(e / want - 1.0)[~tiny] <= 9.4e-8 + 2 * 2.0 ** -24 / 0.7).all()
    assert (e[x < -126.001] == 0).all() and e[x == 0].min() == e.max() == 1.0 and oracle.exp2(np.float32([-127.0]))[0] == 0
    # 1.5e-7 relative either side of a step: never falls by more than both
    x = np.sort(x)
    assert (np.diff(oracle.exp2(x).astype(np.float64)) >= -3e-7 * 2.0 ** x[1:].astype(np.float64)).all()
