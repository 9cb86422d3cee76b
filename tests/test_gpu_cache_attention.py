"""canon_cache_attention: bit-identical to the oracle over head sizes, groups, pages, lengths and masks, rows without keys,
junk in every place that is not seen; near the formula in 64 bits; the same row alone and in a prompt; under capture."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, dev_i32, host_u16, poisoned_workspace
from serve_util import attention_64, device_cache, from_bf16, host_cache

pytestmark = pytest.mark.gpu


def queries(B, Q, H, D, seed=0, scale=2.0, bf16=False):
    q = I.normal_f32((B, Q, H, D), seed, 31) * np.float32(scale)
    return from_bf16(q.view(np.uint32) >> 16) if bf16 else q


def run(c, q, k_len, scale=0.125, starts=None, q_lens=None, k_lens=None, causal=True, window=0, bf16=False, q_start=0,
        stride=0):
    B, Q, H, D = q.shape
    cache = device_cache(c)
    i32 = lambda x: None if x is None else dev_i32(np.asarray(x))  # noqa: E731
    rows = C.AttnRows(B, H, Q, k_len, causal=causal, window=window, scale=scale, q_start=q_start, q_starts=i32(starts),
                      q_lens=i32(q_lens), k_lens=i32(k_lens))
    x = dev_bf16((np.ascontiguousarray(q).view(np.uint32) >> 16).astype(np.uint16)) if bf16 else dev_f32(q)
    x = x.view(B * Q, H * D)
    if stride:
        wide = torch.full((B * Q, stride), float("nan"), dtype=x.dtype, device=DEV)
        wide[:, 8:8 + H * D] = x
        x = wide[:, 8:8 + H * D]
    out = torch.full((B * Q, H * D), 7.0, dtype=torch.bfloat16, device=DEV)
    C.cache_attention(cache, rows, x, out, poisoned_workspace(C.cache_attention_workspace_bytes(cache, rows)))
    torch.cuda.synchronize()
    return host_u16(out).reshape(q.shape)


def want(c, q, k_len, scale=0.125, starts=None, q_lens=None, k_lens=None, causal=True, window=0, q_start=0):
    B, Q = q.shape[:2]
    return c.attention(q, k_len, scale, [q_start] * B if starts is None else starts, [Q] * B if q_lens is None else q_lens,
                       [k_len] * B if k_lens is None else k_lens, causal, window)


def check(c, q, k_len, bf16=False, stride=0, **k):
    got, ref = run(c, q, k_len, bf16=bf16, stride=stride, **k), want(c, q, k_len, **k)
    nan = np.isnan(from_bf16(ref))
    assert (np.isnan(from_bf16(got)) == nan).all()
    assert_bits(np.where(nan, 0, got).astype(np.uint16), np.where(nan, 0, ref).astype(np.uint16), "attention")
    return got


SIZES = [  # batch, heads, kv heads, dim, page, queries, keys
    (1, 1, 1, 32, 16, 1, 1), (2, 2, 1, 64, 16, 1, 15), (1, 4, 4, 128, 64, 1, 16), (3, 6, 2, 96, 32, 1, 255),
    (2, 16, 2, 128, 64, 1, 256), (2, 17, 1, 128, 128, 1, 257), (1, 8, 8, 256, 256, 1, 1000), (2, 5, 1, 160, 16, 3, 700),
    (1, 3, 3, 192, 64, 17, 530), (1, 2, 2, 224, 32, 33, 300), (2, 4, 2, 64, 16, 70, 513), (1, 40, 1, 64, 64, 5, 300),
]


@pytest.mark.parametrize("B,H,KV,D,page,Q,K", SIZES)
@pytest.mark.parametrize("mask", ["causal", "window", "both sides"])
def test_matches_the_oracle(B, H, KV, D, page, Q, K, mask):
    c = host_cache(B, KV, D, page, K, seed=K)
    q = queries(B, Q, H, D, seed=K + 1, bf16=Q == 1)
    lens = [max(1, K - 7 * b) for b in range(B)]
    new = [min(Q, n) for n in lens]
    check(c, q, K, bf16=Q == 1, stride=H * D + 24, starts=[n - m for n, m in zip(lens, new)], q_lens=new, k_lens=lens,
          causal=mask != "both sides", window=37 if mask == "window" else 0)


@pytest.mark.parametrize("D,KV,H", [(128, 8, 16), (64, 4, 4), (96, 16, 16), (256, 8, 8), (32, 8, 8), (160, 8, 8), (192, 8, 8),
                                    (224, 8, 8)])
@pytest.mark.parametrize("window,causal", [(0, True), (100, True), (300, False)])
def test_prompts(D, KV, H, window, causal):
    # enough blocks of queries that a wavefront takes all keys of its queries
    K = Q = 1100 if KV >= 8 else 2100
    B = 2
    c = host_cache(B, KV, D, 64, K, seed=D)
    q = queries(B, Q, H, D, seed=D, bf16=True)
    rows = np.r_[0:3, 250:260, 500, Q - 300:Q - 297, Q - 2:Q]
    got = run(c, q, K, k_lens=[K, K - 77], q_lens=[Q, Q - 77], causal=causal, window=window, bf16=True)
    for i in rows:  # the oracle's rows one at a time
        for b in range(B):
            one = want_row(c, q, K, b, i, [K, K - 77][b], [Q, Q - 77][b], causal, window)
            assert_bits(got[b, i], one, f"row {b} {i}")
    assert (got[1, Q - 77:] == 0).all()


def want_row(c, q, K, b, i, k_len, q_len, causal, window):
    """Row i of sequence b, asked for alone."""
    one = oracle.KVCache.__new__(oracle.KVCache)
    one.__dict__.update(c.__dict__)
    one.table = np.ascontiguousarray(c.table[b:b + 1])
    one.dims = c.dims.copy()
    one.dims[4] = 1
    return one.attention(np.ascontiguousarray(q[b:b + 1, i:i + 1]), K, 0.125, [i], [1 if i < q_len else 0], [k_len], causal,
                         window)[0, 0]


def test_many_short_prompts():
    # one tile of keys, and enough blocks of queries for wavefronts that take all of it
    B, H, KV, D, K = 8, 16, 8, 64, 200
    c = host_cache(B, KV, D, 32, K, seed=30)
    q = queries(B, K, H, D, seed=31, bf16=True)
    lens = [K - 23 * b for b in range(B)]
    check(c, q, K, q_lens=lens, k_lens=lens, bf16=True)


def test_many_sequences():
    # a batch that fills the chip with single tokens: a workgroup for every tile all the same
    B, H, KV, D, K = 40, 8, 4, 64, 700
    c = host_cache(B, KV, D, 64, K, seed=32)
    lens = [1 + 17 * b for b in range(B)]
    check(c, queries(B, 1, H, D, seed=33), K, starts=[n - 1 for n in lens], k_lens=lens)


def test_a_row_is_the_same_alone_and_in_a_prompt():
    B, H, KV, D, K = 2, 16, 8, 128, 1500
    c = host_cache(B, KV, D, 64, K, seed=3)
    q = queries(B, K, H, D, seed=4)
    full = run(c, q, K)
    for i in (0, 1, 255, 256, 700, K - 1):
        alone = run(c, np.ascontiguousarray(q[:, i:i + 1]), i + 1, starts=[i, i])
        assert_bits(alone[:, 0], full[:, i], f"row {i}")
        part = run(c, np.ascontiguousarray(q[:, i:i + 3]), K, starts=[i, i])
        assert_bits(part[:, :len(full[0, i:i + 3])], full[:, i:i + 3], f"rows from {i}")


@pytest.mark.parametrize("Q,K,D", [(1, 3000, 128), (40, 900, 64)])
def test_near_the_formula(Q, K, D):
    # bf16's rounding is 2^-8 of a value (half a step of 8 significant bits); what the digits of 16 bits leave is reckoned below
    B, H, KV = 2, 8, 2
    c = host_cache(B, KV, D, 64, K, seed=9)
    q = queries(B, Q, H, D, seed=10)
    starts = [K - Q] * B
    got = from_bf16(run(c, q, K, starts=starts)).astype(np.float64)
    ref = attention_64(c, q, 0.125, starts, [Q] * B, [K] * B, True, 0)
    # score: |q16/2^16 error| sum |k| scale <= 2^-16 amax_q sum_d |k_d| / 8; with amax_q < 11 and |k| < 8 on D <= 128 elements
    # < 2^-16 * 11 * 8 * 128 / 8 = 0.022 at the very worst, and 4e-4 at six standard deviations of its random signs; a weight
    # is off by that part, a value by 2^-16 of the largest of its tile: 1e-3 |v|max in all
    assert (np.abs(got - ref) <= np.abs(ref) * 2.0 ** -8 + 1e-3 * np.abs(kept_max(c))).all()


def kept_max(c):
    return 127.0 * np.nanmax(np.where(np.isfinite(c.v_steps), c.v_steps, 0.0))


def test_rows_without_keys_and_lengths_of_any_value():
    B, H, KV, D, K, Q = 4, 4, 2, 64, 300, 5
    c = host_cache(B, KV, D, 16, K, seed=5)
    q = queries(B, Q, H, D, seed=6)
    for starts, q_lens, k_lens in (([-3, -5, 0, 10], [Q, Q, 0, -1], [K, K, K, K]),
                                   ([0, 300, 290, 1 << 30], [Q, 99, 3, Q], [0, -5, 1 << 30, 7]),
                                   ([0, -(1 << 30), 5, 299], [1, Q, 2, Q], [1, K, 5, 299])):
        for causal, window in ((True, 0), (False, 0), (False, 4), (True, 1)):
            check(c, q, K, starts=starts, q_lens=q_lens, k_lens=[max(-9, k) for k in k_lens], causal=causal, window=window)
    none = np.zeros((B, 1, H, D), np.float32)
    assert (run(c, none, 0) == 0).all()


def test_extreme_scores_and_values():
    B, H, KV, D, K = 1, 8, 2, 64, 600
    c = host_cache(B, KV, D, 16, K, seed=7)
    q = queries(B, 3, H, D, seed=8)
    q[0, 0, 0] *= 1e30     # one key takes all
    q[0, 0, 1] *= 1e-37    # subnormal parts, flat weights
    q[0, 0, 2] = 0.0
    q[0, 0, 3] *= 200.0
    q[0, 1, 4, 5] = np.inf
    q[0, 1, 5, 6] = np.nan
    q[0, 2, 6] *= 3e38
    for scale in (0.125, 1e30, 0.0, -0.5):
        check(c, q, K, starts=[K - 3], scale=scale)
    keys = I.normal_f32((B, K, KV, D), 3, 23) * np.exp(6 * I.normal_f32((B, K, 1, 1), 3, 24))
    vals = I.normal_f32((B, K, KV, D), 3, 25) * np.exp(9 * I.normal_f32((B, K, KV, 1), 3, 26))
    check(host_cache(B, KV, D, 16, K, k=keys.astype(np.float32), v=vals.astype(np.float32)), queries(B, 3, H, D), K,
          starts=[K - 3])
    tiny = host_cache(B, KV, D, 16, K, v=(vals * 1e-38).astype(np.float32))
    check(tiny, queries(B, 3, H, D), K, starts=[K - 3])
    zero = host_cache(B, KV, D, 16, K, v=np.zeros_like(vals, dtype=np.float32))
    assert (check(zero, queries(B, 3, H, D), K, starts=[K - 3]) & 0x7FFF == 0).all()


@pytest.mark.parametrize("Q", [1, 600])
def test_infinities_and_nan_reach_only_the_rows_that_see_them(Q):
    B, H, KV, D, K = 2, 16, 8, 64, 900
    k, v = (I.normal_f32((B, K, KV, D), 1, s) for s in (27, 28))
    k[0, 700, 3, 5] = np.inf
    v[0, 850, 6, 9] = np.nan
    v[1, 320, 0, 0] = -np.inf
    c = host_cache(B, KV, D, 16, K, k=k, v=v)
    q = queries(B, Q, H, D, seed=2)
    got = from_bf16(check(c, q, K, starts=[K - Q] * B))
    pos = np.arange(Q) + K - Q
    bad = np.isnan(got).any(-1)
    want_bad = np.zeros((B, Q, H), bool)
    want_bad[0, pos >= 700, 6:8] = True
    want_bad[0, pos >= 850, 12:14] = True
    want_bad[1, pos >= 320, 0:2] = True
    assert (bad == want_bad).all()


def test_pages_that_the_cache_does_not_have():
    B, H, KV, D, K = 3, 4, 2, 64, 200
    c = host_cache(B, KV, D, 16, K, seed=11)
    for value in (-1, int(c.dims[0]), 1 << 30, -(1 << 31)):
        c.table[1, 5] = value  # keys 80 .. 95 of the second sequence
        c.table[2, 12] = value  # keys 192 .. of the third, which has 190
        q = queries(B, 1, H, D, seed=12)
        out = from_bf16(check(c, q, K, starts=[K - 1] * B, k_lens=[K, K, 190], causal=False))
        assert not np.isnan(out[[0, 2]]).any() and np.isnan(out[1]).all()
        out = from_bf16(check(c, q, K, starts=[K - 1, 79, K - 1], k_lens=[K, K, 190]))
        assert not np.isnan(out).any()
        out = from_bf16(check(c, q, K, starts=[K - 1] * B, k_lens=[K, K, 190], window=100))
        assert not np.isnan(out).any()


def test_a_captured_call_and_a_stream_of_its_own():
    B, H, KV, D, K = 4, 16, 2, 128, 2000
    c = host_cache(B, KV, D, 64, K, seed=13)
    cache = device_cache(c)
    starts, lens = dev_i32(np.array([K - 1] * B)), dev_i32(np.array([K] * B))
    rows = C.AttnRows(B, H, 1, K, scale=0.125, q_starts=starts, k_lens=lens)
    q = torch.zeros(B, H * D, device=DEV)
    out = torch.zeros(B, H * D, dtype=torch.bfloat16, device=DEV)
    ws = poisoned_workspace(C.cache_attention_workspace_bytes(cache, rows))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        C.cache_attention(cache, rows, q, out, ws)
    for i in range(4):
        x = queries(B, 1, H, D, seed=40 + i)
        n = K - 300 * i
        q.copy_(dev_f32(x).view(B, H * D))
        starts.fill_(n - 1)
        lens.fill_(n)
        ref = want(c, x, K, starts=[n - 1] * B, k_lens=[n] * B)
        graph.replay()
        torch.cuda.synchronize()
        assert_bits(host_u16(out).reshape(ref.shape), ref, f"replay {i}")
        out.zero_()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            C.cache_attention(cache, rows, q, out, ws)
        side.synchronize()
        assert_bits(host_u16(out).reshape(ref.shape), ref, f"stream {i}")
