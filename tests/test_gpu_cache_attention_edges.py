"""canon_cache_attention at the ends of its range: a cache of no pages, values and channels of very different sizes."""
import numpy as np
import pytest
import torch

import paper_2609_17380_amd.canon as C
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, dev_i32, host_u16, poisoned_workspace
from serve_bounds import OUTLIERS, SPREADS, attention_bound, outlier_case, spread_case
from serve_util import device_cache, from_bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("pages,table_len", [(0, 0), (0, 3), (2, 0), (2, 3)])
def test_no_keys(D, pages, table_len):
    # a cache of no pages has no address at all; with pages and k_len 0 nothing of it is to be read either
    B, KV, page = 2, 2, 16
    codes = lambda *s: torch.full(s, 77, dtype=torch.int8, device=DEV)  # noqa: E731
    steps = lambda: torch.full((pages, KV, page), float("nan"), device=DEV)  # noqa: E731
    table = torch.full((B, table_len), 1 << 30, dtype=torch.int32, device=DEV)
    cache = C.KVCache(page, KV, D, codes(pages, KV, page, D), codes(pages, KV, page // 16, D, 16), steps(), steps(), table)
    assert cache.n_pages == pages and (pages > 0 or not cache.k_codes)
    for Q, G in ((1, 1), (3, 2), (16, 1), (17, 3), (70, 1), (400, 1)):
        H = KV * G
        for lens in (None, dev_i32(np.array([5, 0]))):
            rows = C.AttnRows(B, H, Q, 0, scale=0.125, k_lens=lens)
            q = torch.full((B * Q, H * D), 3.0, device=DEV)
            out = torch.full((B * Q, H * D), 7.0, dtype=torch.bfloat16, device=DEV)
            C.cache_attention(cache, rows, q, out, poisoned_workspace(C.cache_attention_workspace_bytes(cache, rows)))
            torch.cuda.synchronize()
            assert (host_u16(out) == 0).all(), (Q, G)


def attend(c, q, k_len, scale, starts, bf16=False):
    B, Q, H, D = q.shape
    cache = device_cache(c)
    rows = C.AttnRows(B, H, Q, k_len, scale=scale, q_starts=dev_i32(np.asarray(starts)))
    out = torch.full((B * Q, H * D), 7.0, dtype=torch.bfloat16, device=DEV)
    x = dev_bf16((np.ascontiguousarray(q).view(np.uint32) >> 16).astype(np.uint16)) if bf16 else dev_f32(q)
    C.cache_attention(cache, rows, x.view(B * Q, H * D), out,
                      poisoned_workspace(C.cache_attention_workspace_bytes(cache, rows)))
    torch.cuda.synchronize()
    return host_u16(out).reshape(q.shape)


@pytest.mark.parametrize("kind,size", SPREADS)
@pytest.mark.parametrize("prompt", [False, True])
def test_values_of_different_sizes(kind, size, prompt):
    # a workgroup for a tile, and (a prompt) wavefronts that take all keys
    K = 1024
    c, q = spread_case(kind, size, KV=8, Q=K) if prompt else spread_case(kind, size)
    first = K - q.shape[1]
    got = attend(c, q, K, 0.125, [first])
    for at in ((0, 96, 255, 500, K - 3) if prompt else (0,)):
        few = np.ascontiguousarray(q[:, at:at + 3])
        assert_bits(got[:, at:at + 3], c.attention(few, K, 0.125, [first + at], [3], [K]), f"rows from {at}")
        want, bound = attention_bound(c, few, 0.125, [first + at], [3], [K])
        assert (np.abs(from_bf16(got[:, at:at + 3]) - want) <= bound).all(), at


@pytest.mark.parametrize("times,bf16", OUTLIERS)
@pytest.mark.parametrize("prompt", [False, True])
def test_channels_of_different_sizes(times, bf16, prompt):
    K = 700
    c, q = outlier_case(times, bf16, KV=8, K=K, Q=K) if prompt else outlier_case(times, bf16)
    first = K - q.shape[1]
    got = attend(c, q, K, 0.125, [first], bf16)
    for at in ((0, 255, 400, K - 3) if prompt else (0,)):
        few = np.ascontiguousarray(q[:, at:at + 3])
        assert_bits(got[:, at:at + 3], c.attention(few, K, 0.125, [first + at], [3], [K]), f"rows from {at}")
        want, bound = attention_bound(c, few, 0.125, [first + at], [3], [K])
        assert (np.abs(from_bf16(got[:, at:at + 3]) - want) <= bound).all(), at


@pytest.mark.parametrize("Q", [3, 300])
def test_queries_at_the_ends_of_their_digits(Q):
    """The largest element just below and above what three digits hold at one step, the smallest and largest numbers, subnormal
    parts, ties; the scale's sign."""
    c, q = spread_case("all", 1.0, KV=8, K=300, Q=Q)
    tops = np.array([8355711.0, 8355711.5, 8355712.0, 8388607.0, 8388608.0, 8322815.0], np.float32)
    for h, top in enumerate(tops):
        q[0, 0, h] = np.float32(0.5) + np.arange(64, dtype=np.float32)  # halves of the step
        q[0, 0, h, 9] = -top if h % 2 else top
    for h, e in enumerate((-126, -125, -104, 127, 100, -149)):
        q[0, 1, h] = np.ldexp(q[0, 1, h], e).astype(np.float32)
        q[0, 1, h, 3] = np.float32(1.9999999) * np.float32(2.0) ** e if e > -149 else np.float32(1e-45)
    for scale in (0.125, -0.125, 2.0 ** -20, 2.0 ** 100, 2.0 ** -120):
        got = attend(c, q, 300, scale, [300 - Q])
        want = c.attention(q[:, :2].copy(), 300, scale, [300 - Q], [2], [300])
        nan = np.isnan(from_bf16(want))
        assert (np.isnan(from_bf16(got[:, :2])) == nan).all()
        assert_bits(np.where(nan, 0, got[:, :2]).astype(np.uint16), np.where(nan, 0, want).astype(np.uint16), f"scale {scale}")
