"""The workspace of canon_cache_attention: that of a window does not grow with the keys behind it, and no more of it than the call asks for
is written."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_17380_amd.canon as C
from serve_util import device_cache, host_cache


def raw(cls, *fields):
    r = cls.__new__(cls)
    ctypes.Structure.__init__(r, *fields)
    return r


def workspace(batch, heads, kv, dim, q_len, k_len, window, causal=1, page=64):
    p = 1 << 40
    cache = raw(C.KVCache, 100, page, kv, dim, p, p, p, p, batch, -(-k_len // page), p)
    rows = raw(C.AttnRows, batch, heads, q_len, k_len, 0, 0, window, causal, 0.125, None, None, None)
    return C.lib().canon_cache_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(rows))


def test_a_window_bounds_it():
    # 512 keys and the positions of a block of 16 columns: four tiles of 256 at the most
    for k_len in (1100, 32768, 1 << 21):
        assert workspace(32, 64, 8, 256, 1, k_len, 512) == 4 * 32 * 64 * 4 * (256 + 4)
    assert workspace(32, 64, 8, 256, 1, 600, 512) == 4 * 32 * 64 * 3 * (256 + 4)
    assert workspace(32, 64, 8, 256, 1, 32768, 0) == 4 * 32 * 64 * 128 * (256 + 4)
    both = workspace(2, 4, 4, 64, 3, 32768, 512, causal=0)
    assert both == 4 * 2 * 4 * 3 * 6 * (64 + 4)  # 1023 keys, and 16 positions more


@pytest.mark.gpu
@pytest.mark.parametrize("H,KV,D,Q", [(4, 4, 64, 1), (6, 2, 96, 5), (7, 1, 128, 9), (16, 2, 32, 3), (40, 1, 64, 2)])
@pytest.mark.parametrize("window,causal", [(1, True), (255, True), (257, False), (700, True), (512, False)])
def test_a_window_far_into_the_keys(H, KV, D, Q, window, causal):
    from gpu_util import DEV, assert_bits, dev_f32, dev_i32, host_u16
    import paper_2609_17380_amd.inputs as I

    B, K = 3, 5000
    c = host_cache(B, KV, D, 64, K, seed=window)
    cache = device_cache(c)
    q = I.normal_f32((B, Q, H, D), window, 111) * np.float32(2)
    for starts in ([K - Q, 2047, 255], [-2, 4095 - Q, 3 * 256 - 1], [K + 5, 0, 1300]):
        lens = [K, K - 9, K - 600]
        rows = C.AttnRows(B, H, Q, K, causal=causal, window=window, scale=0.125, q_starts=dev_i32(np.asarray(starts)),
                          k_lens=dev_i32(np.asarray(lens)))
        need = C.cache_attention_workspace_bytes(cache, rows)
        ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device=DEV)
        out = torch.full((B * Q, H * D), 7.0, dtype=torch.bfloat16, device=DEV)
        C.cache_attention(cache, rows, dev_f32(q).view(B * Q, H * D), out, ws[:need])
        torch.cuda.synchronize()
        assert need > 0 and (ws[need:] == 255).all()
        assert_bits(host_u16(out).reshape(q.shape), c.attention(q, K, 0.125, starts, [Q] * B, lens, causal, window), str(starts))
