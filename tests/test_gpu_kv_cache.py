"""canon_cache_append and canon_cache_read: codes, steps and untouched slots bit for bit as the oracle's, over head sizes, pages,
lengths and positions; the four operators of a decoding step run together."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, dev_i32, host_f32, host_u16, poisoned_workspace
from serve_util import device_cache, from_bf16, permuted_table, tables

pytestmark = pytest.mark.gpu


def fresh(B, KV, D, page, positions, seed=0):
    n, table = permuted_table(B, max(1, -(-positions // page)), seed=seed)
    return oracle.KVCache(n, page, KV, D, table, 55, np.nan)


def new_tokens(B, Q, KV, D, seed, bf16):
    k, v = (I.normal_f32((B, Q, KV, D), seed, s) * np.float32(3) for s in (41, 42))
    if bf16:
        k, v = (from_bf16(x.view(np.uint32) >> 16) for x in (k, v))
    return k, v


def to_dev(x, bf16, stride=0):
    rows, width = x.shape[0] * x.shape[1], x.shape[2] * x.shape[3]
    t = dev_bf16((np.ascontiguousarray(x).view(np.uint32) >> 16).astype(np.uint16)) if bf16 else dev_f32(x)
    t = t.view(rows, width)
    if stride:
        wide = torch.full((rows, stride), float("nan"), dtype=t.dtype, device=DEV)
        wide[:, 3:3 + width] = t
        t = wide[:, 3:3 + width]
    return t


def same(cache, c):
    torch.cuda.synchronize()
    for name, t, want in zip(("k_codes", "v_codes", "k_steps", "v_steps"), cache.tensors, c.arrays()):
        got = t.cpu().numpy()
        if want.dtype == np.float32:
            nan = np.isnan(want)
            assert (np.isnan(got) == nan).all(), name
            assert_bits(np.where(nan, 0, got).astype(np.float32), np.where(nan, 0, want).astype(np.float32), name)
        else:
            assert (got == want).all(), (name, np.argwhere(got != want)[:3])


def append(cache, c, k, v, starts, lens, rot=0, inter=False, positions=0, bf16=False, stride=0, q_start=None):
    B, Q = k.shape[:2]
    turn, cos, sin = None, None, None
    if rot:
        cos, sin = tables(rot, positions)
        turn = C.Rotation(dev_f32(cos), dev_f32(sin), rot, interleaved=inter)
    rows = C.CacheRows(B, Q, q_start=q_start or 0, q_starts=None if q_start is not None else dev_i32(np.asarray(starts)),
                       q_lens=dev_i32(np.asarray(lens)))
    C.cache_append(cache, rows, to_dev(k, bf16, stride), to_dev(v, bf16, stride), rotation=turn)
    c.append(k, v, starts, lens, cos, sin, rot, inter)
    return rows


@pytest.mark.parametrize("D,KV,page", [(32, 1, 16), (64, 3, 32), (96, 2, 64), (128, 4, 128), (160, 1, 16), (192, 2, 256),
                                       (224, 1, 64), (256, 2, 32)])
@pytest.mark.parametrize("bf16", [False, True])
def test_prompts_and_tokens(D, KV, page, bf16):
    B, P = 3, 300
    for rot, inter in ((0, False), (D, False), (D, True), (D // 2, False), (6, True), (6, False), (2, True)):
        c = fresh(B, KV, D, page, P)
        cache = device_cache(c)
        at = np.zeros(B, np.int64)
        for step, lens in enumerate(([37, 1, 0], [1, 1, 1], [16, 47, 100], [1, 0, 1], [5, 15, 31], [1, 1, 1])):
            k, v = new_tokens(B, max(lens), KV, D, seed=step, bf16=bf16)
            append(cache, c, k, v, at, lens, rot, inter, P, bf16, stride=KV * D + 11 if step % 2 else 0)
            at += lens
        same(cache, c)


def test_tokens_that_the_cache_has_no_place_for():
    B, KV, D, page = 4, 2, 64, 16
    c = fresh(B, KV, D, page, 64)
    c.table[1, 1], c.table[2, 0], c.table[2, 3] = -1, int(c.dims[0]), 1 << 30
    cache = device_cache(c)
    k, v = new_tokens(B, 70, KV, D, 1, False)
    append(cache, c, k, v, [-20, 0, 0, 60], [70, 70, 99, 70], D, False, 50)  # positions from 50 on have no angle: NaN steps
    same(cache, c)
    append(cache, c, k, v, [1 << 30, -(1 << 31), (1 << 31) - 1, 63], [70, 70, 70, 2])
    same(cache, c)


def test_special_values():
    B, KV, D = 1, 1, 64
    c = fresh(B, KV, D, 16, 64)
    cache = device_cache(c)
    k, v = new_tokens(B, 20, KV, D, 2, False)
    k[0, 1], v[0, 2] = 0.0, 0.0
    k[0, 3, 0, 5], v[0, 4, 0, 6], k[0, 5, 0, 7] = np.inf, np.nan, -np.inf
    v[0, 6] *= 1e-38
    k[0, 7] *= 1e-44
    v[0, 8] *= 1e38
    k[0, 9, 0, 0] = 3e38
    v[0, 10] = np.float32(127) * np.where(np.arange(D) % 2, 0.5, 1)  # halves of a step
    append(cache, c, k, v, [0], [20])
    same(cache, c)
    cos, sin = tables(D, 64)
    c2, = (fresh(B, KV, D, 16, 64),)
    cache2 = device_cache(c2)
    append(cache2, c2, k, v, [3], [20], D, True, 64)
    same(cache2, c2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_read(dtype):
    B, KV, D, page, Q = 3, 2, 96, 32, 50
    c = fresh(B, KV, D, page, 128)
    c.table[2, 1] = -7
    cache = device_cache(c)
    k, v = new_tokens(B, Q, KV, D, 3, False)
    starts, lens = [0, 17, 20], [Q, 30, Q]
    rows = append(cache, c, k, v, starts, lens)
    out = [torch.full((B, Q, KV, D), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
    C.cache_read(cache, rows, *out)
    only = torch.full((B * Q, KV * D), 7.0, dtype=dtype, device=DEV)
    C.cache_read(cache, rows, v=only)
    torch.cuda.synchronize()
    f = lambda x: x.float().cpu().numpy()  # noqa: E731
    assert np.array_equal(f(only).reshape(B, Q, KV, D), f(out[1]), equal_nan=True)
    for x, got in zip((k, v), out):
        codes, steps = oracle.act8_pack(x.reshape(-1, D), D)
        want = (codes.astype(np.float32) * steps).reshape(x.shape)
        want[1, 30:] = 0.0
        pos = 20 + np.arange(Q)
        want[2, (pos >= 32) & (pos < 64)] = np.nan
        if dtype == torch.bfloat16:
            want = torch.from_numpy(want).bfloat16().float().numpy()
        assert np.array_equal(f(got), want, equal_nan=True)


def test_a_decoding_step():
    """Prompts of different lengths, then tokens one at a time: rotation, append, attention; captured and replayed, every
    result as the oracle's, and the last tokens as a single prompt over all of them gives."""
    B, H, KV, D, page, P = 3, 8, 2, 64, 16, 400
    rot, scale = 32, 0.125
    cos, sin = tables(rot, P)
    turn = C.Rotation(dev_f32(cos), dev_f32(sin), rot, interleaved=True)
    c = fresh(B, KV, D, page, P)
    cache = device_cache(c)
    lens = np.array([300, 5, 77])
    k, v = new_tokens(B, 300, KV, D, 5, True)
    append(cache, c, k, v, [0] * B, lens, rot, True, P, True)
    starts, keys = dev_i32(lens), dev_i32(lens + 1)
    qkv = torch.zeros(B, (H + 2 * KV) * D, dtype=torch.bfloat16, device=DEV)
    q, kk, vv = qkv[:, :H * D], qkv[:, H * D:(H + KV) * D], qkv[:, (H + KV) * D:]
    out = torch.zeros(B, H * D, dtype=torch.bfloat16, device=DEV)
    rows, arows = C.CacheRows(B, 1, q_starts=starts), C.AttnRows(B, H, 1, P, scale=scale, q_starts=starts, k_lens=keys)
    ws = poisoned_workspace(C.cache_attention_workspace_bytes(cache, arows))

    def step():
        C.rope(B, H, D, turn, q, q, positions=starts)
        C.cache_append(cache, rows, kk, vv, rotation=turn)
        C.cache_attention(cache, arows, q, out, ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        x = from_bf16(I.normal_f32((B, 1, H + 2 * KV, D), 60 + i, 43).view(np.uint32) >> 16)
        qkv.copy_(to_dev(x, True))
        starts.copy_(dev_i32(lens))
        keys.copy_(dev_i32(lens + 1))
        if i % 2:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        turned = oracle.rope(x[:, 0, :H], lens, cos, sin, rot, True)
        turned = from_bf16(torch.from_numpy(turned).bfloat16().view(torch.int16).numpy().view(np.uint16))
        c.append(x[:, :, H:H + KV], x[:, :, H + KV:], lens, [1] * B, cos, sin, rot, True)
        ref = c.attention(turned[:, None], P, scale, lens, [1] * B, lens + 1)
        same(cache, c)
        assert_bits(host_u16(out).reshape(ref.shape), ref, f"step {i}")
        lens = lens + 1
