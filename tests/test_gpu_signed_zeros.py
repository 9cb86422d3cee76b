"""Row and column sums that end at -0.  A result below 2^-126 is flushed to the zero of its own sign, so a chain, a fold or a
whole sum can be -0; what the order does not add (chunks, columns and rows that are not there) leaves it -0, and a term of +0
does not.  Bit-identical to the oracle, in which absent terms are not there at all."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, dev_i32, host_f32, host_u16, poisoned_workspace
from test_gpu_layernorm import host_bf16

pytestmark = pytest.mark.gpu

ONE = 0x3F80
TINY = np.float32(2.0 ** -126)  # the least magnitude that is not flushed


def last_split(n):
    """The term at which the last addition of a sum of n terms in chunks of 32 splits them (of one chunk: none, 0)."""
    chunks = (n + 31) // 32
    return 32 << ((chunks - 1).bit_length() - 1) if chunks > 1 else 0


def tiny_rows(rows, n, seed, kinds=(0, 1, 2)):
    """Rows of -0 with a few terms of 1 to 1.75 times 2^-126 of either sign, many of whose sums are flushed: a third of the rows
    with the terms anywhere, a third with them near the row's end, both with a +0 now and then; a third with 1 and -1.5 on
    the two sides of the sum's last addition (or of its last chunk's), which ends at -0."""
    rng = np.random.default_rng(seed)
    x = np.full((rows, n), -0.0, np.float32)
    kind, r, k = rng.choice(kinds, rows) if n > 1 else np.zeros(rows, int), np.arange(rows), 6
    near = n - 1 - rng.integers(0, min(n, 40), (rows, k))
    at = np.where(kind[:, None] == 1, near, rng.integers(0, n, (rows, k)))
    v = (rng.choice([1, 1.25, 1.5, 1.75], (rows, k)) * rng.choice([-1, 1], (rows, k))).astype(np.float32) * TINY
    live = np.where(kind == 2, 0, rng.integers(2, k + 1, rows))
    for i in range(k):
        m = i < live
        x[r[m], at[m, i]] = v[m, i]
    z = (rng.random(rows) < 0.2) & (kind < 2)
    x[r[z], rng.integers(0, n, rows)[z]] = 0.0
    m = r[kind == 2]
    cut = last_split(n) or n - 1
    x[m, rng.integers(0, cut, len(m))] = TINY
    x[m, rng.integers(cut, n, len(m))] = -1.5 * TINY
    return x


def minus_zeros(x):
    return int((np.ascontiguousarray(x).view(np.uint32) == 0x80000000).sum())


def rms_backward(x, g, rstd, dy):
    rows, cols = x.shape
    dx = torch.full((rows, cols), float("nan"), device=DEV)
    C.rownorm(C.BWD, rows, cols, dev_f32(x), dev_bf16(g), np.float32(1e-5), rstd=dev_f32(rstd), dy=dev_f32(dy), dx=dx)
    torch.cuda.synchronize()
    return host_f32(dx)


def test_the_norm_gradient_of_a_dot_of_minus_zero():
    # the dot is flushed from -2^-127 to -0, so that dx[2] = RN(-0 - -0) = +0; of a dot of +0 it is -0
    x, g, rstd = np.ones((1, 3), np.float32), np.full(3, ONE, np.uint16), np.ones(1, np.float32)
    dy = np.array([[TINY, -1.5 * TINY, -0.0]], np.float32)
    got = rms_backward(x, g, rstd, dy)
    assert got.view(np.uint32)[0, 2] == 0
    assert_bits(got, oracle.rownorm_bwd(x, g, rstd, dy)[0], "dx")


LENGTHS = [1, 2, 3, 31, 32, 33, 63, 64, 65, 100, 255, 257, 511, 513, 700, 1024, 1025, 1500, 2047, 2048]


@pytest.mark.parametrize("cols", LENGTHS + [2049, 4100])
def test_norm_rows(cols):
    print(f"norm 96x{cols}", flush=True)
    rows = 96
    dy, g = tiny_rows(rows, cols, 1), np.full(cols, ONE, np.uint16)
    x = np.where(np.arange(rows)[:, None] % 2, I.normal_f32((rows, cols), 1, 3), np.float32(1)).astype(np.float32)
    rstd = np.ones(rows, np.float32)
    assert_bits(rms_backward(x, g, rstd, dy), oracle.rownorm_bwd(x, g, rstd, dy)[0], "dx")
    y, r = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV), torch.empty(rows, device=DEV)
    C.rownorm(C.FWD, rows, cols, dev_f32(dy), dev_bf16(g), np.float32(1e-5), y=y, rstd=r)
    torch.cuda.synchronize()
    want_y, want_r = oracle.rownorm_fwd(dy, g, np.float32(1e-5))
    assert_bits(host_u16(y), want_y, "y")
    assert_bits(host_f32(r), want_r, "rstd")


@pytest.mark.parametrize("cols", LENGTHS + [2049, 4096, 4100, 5001, 8192, 8195, 16390, 32767])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_norm_rows(cols, dtype):
    # few rows (spread over wavefronts from 1025 columns on) and many
    for rows in (64, 3000) if cols in (1500, 2047) else (64,):
        print(f"layer norm {rows}x{cols} {dtype}", flush=True)
        x, g, b = tiny_rows(rows, cols, 2), np.full(cols, ONE, np.uint16), np.full(cols, 0x8000, np.uint16)
        want_y, want_m, want_r = oracle.layernorm_fwd(x, g, b, 1e-5)
        assert cols == 1 or minus_zeros(want_m) > rows // 5
        on = dev_f32 if dtype == torch.float32 else lambda v: dev_bf16(host_bf16(v))  # their values have 3 bits
        y, m, r = torch.empty((rows, cols), device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        C.layernorm(rows, cols, on(x), dev_bf16(g), dev_bf16(b), 1e-5, y, m, r)
        torch.cuda.synchronize()
        assert_bits(host_f32(m), want_m, "mean")
        assert_bits(host_f32(r), want_r, "rstd")
        assert_bits(host_f32(y), want_y, "y")


def layer_norm_backward(x, dy, group=None):
    """dx, dgain and dbias of rows whose mean is taken as 0 and whose rstd as 1 (arguments of the call), and the oracle's."""
    rows, cols = x.shape
    g, m, r = np.full(cols, ONE, np.uint16), np.zeros(rows, np.float32), np.ones(rows, np.float32)
    xd = dev_f32(x)
    if group:
        codes, steps = oracle.act8_pack(x, group)
        xd = C.Act8(group, torch.from_numpy(codes).to(DEV), dev_f32(steps))
        x = oracle.act8_unpack(codes, steps, group)
    dx, dg, db = torch.empty((rows, cols), device=DEV), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    ws = poisoned_workspace(C.layernorm_bwd_workspace_bytes(rows, cols))
    C.layernorm_bwd(rows, cols, xd, dev_bf16(g), dev_f32(m), dev_f32(r), dev_f32(dy), dx, ws, dgain=dg, dbias=db)
    torch.cuda.synchronize()
    return [host_f32(t) for t in (dx, dg, db)], oracle.layernorm_bwd(x, g, m, r, dy)


@pytest.mark.parametrize("cols", LENGTHS + [2049, 4096, 4100, 5001, 8195, 16390])
def test_layer_norm_gradient_rows(cols):
    print(f"layer norm backward 64x{cols}", flush=True)
    rows = 64
    dy = tiny_rows(rows, cols, 3)
    x = np.where(np.arange(rows)[:, None] % 2, I.normal_f32((rows, cols), 1, 3), np.float32(1)).astype(np.float32)
    for group in (None, 64):
        got, want = layer_norm_backward(x, dy, group)
        assert_bits(got[0], want[0], "dx")


@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 64, 65, 100, 512, 513, 1000, 1057, 5000, 16500])
def test_sums_over_rows(rows):
    # chains of 32 rows, blocks of chunks and folds of 16, some of each absent
    cols = 200
    print(f"rows {rows}", flush=True)
    dy = np.ascontiguousarray(tiny_rows(cols, rows, 4).T)
    got, want = layer_norm_backward(np.ones((rows, cols), np.float32), dy)
    assert rows == 1 or minus_zeros(want[2]) > cols // 5
    assert_bits(got[2], want[2], "dbias")
    assert_bits(got[1], want[1], "dgain")


@pytest.mark.parametrize("rows,cols", [(4096, 2048), (4099, 2050), (4097, 4095), (4100, 4097), (4096, 8190), (8200, 1021), (16400, 257),
                                       (32769, 4), (32800, 5), (32770, 33), (32771, 255), (32800, 31), (32768 + 40, 64), (32800, 100)])
@pytest.mark.parametrize("group", [None, 32])
def test_one_pass_over_many_rows(rows, cols, group):
    # the backward of enough rows is one pass, with columns and whole wavefronts that the row does not have
    print(f"layer norm backward {rows}x{cols} group {group}", flush=True)
    dy = tiny_rows(rows, cols, 5)
    dy[:, ::3] = tiny_rows(cols, rows, 6, (2,))[::3].T  # so that sums over the rows are -0 as well
    x = np.where(np.arange(rows)[:, None] % 2, np.float32(-1), np.float32(1)) * np.ones((1, cols), np.float32)
    got, want = layer_norm_backward(np.ascontiguousarray(x), dy, group)
    assert minus_zeros(want[2]) > cols // 5
    assert_bits(got[0], want[0], "dx")
    assert_bits(got[1], want[1], "dgain")
    assert_bits(got[2], want[2], "dbias")


LOG32 = list(C.relbias_log(32, 128).start)[:32]
LOG16 = list(C.relbias_log(32, 128, True).start)[:16]
WIDE = [0, 1, 34, 70, 200]


KEYS = [1, 2, 5, 31, 32, 33, 63, 64, 65, 96, 97, 128, 129, 200, 255, 256, 300, 511, 512, 700, 1024, 1100, 2047, 2500, 5000]
BUCKETS = [(LOG32, False), (LOG16, True), (WIDE, False), (WIDE, True), ([0], False), ([0], True), ([0, 32], True),
           ([0, 1, 2, 3], True)]


def relative_bias_backward(p, dp, starts, bidirectional, pos, causal=False, window=0, k_len=None):
    """dscores and dtable of queries from position pos on, and the oracle's."""
    B, H, Q, k = p.shape
    lens = None if k_len is None else [k_len] * B
    rows = C.AttnRows(B, H, Q, k, scale=1.0, causal=causal, q_start=pos, window=window, k_lens=None if lens is None else dev_i32(lens))
    bias = C.RelBias(starts, bidirectional)
    ds, dt = torch.empty(p.shape, dtype=torch.bfloat16, device=DEV), torch.empty((bias.buckets, H), device=DEV)
    ws = poisoned_workspace(C.softmax_relbias_bwd_workspace_bytes(rows, bias))
    C.softmax_relbias_bwd(rows, bias, dev_bf16(p), dev_f32(dp), ds, ws, dtable=dt)
    torch.cuda.synchronize()
    return (host_u16(ds), host_f32(dt)), oracle.relbias_bwd(p, dp, starts, bidirectional, scale=1.0, causal=causal, window=window,
                                                            q_starts=[pos] * B, k_lens=lens)


@pytest.mark.parametrize("k", KEYS)
@pytest.mark.parametrize("starts,bidirectional", BUCKETS)
def test_relative_bias_gradient(k, starts, bidirectional):
    print(f"relbias backward {k} keys {len(starts)} starts bidirectional={bidirectional}", flush=True)
    rng = np.random.default_rng(6)
    dp = tiny_rows(64, k, 7).reshape(1, 16, 4, k)
    p = np.where((rng.random(dp.shape) < 0.5) & (dp == 0), 0, ONE).astype(np.uint16)
    got, want = relative_bias_backward(p, dp, starts, bidirectional, k // 2)
    assert_bits(got[0], want[0], "dscores")
    assert_bits(got[1], want[1], "dtable")


@pytest.mark.parametrize("k", KEYS[1:])
@pytest.mark.parametrize("starts,bidirectional", BUCKETS)
def test_relative_bias_table_gradient(k, starts, bidirectional):
    # Every head is a trial: its first two rows leave the chain of one bucket at -0 (ds of 1 and -1.5 times 2^-126 in one key of
    # it, and zeros), and the third row's sum of that bucket, of two keys with ds of 1.19 and -1.31, decides whether it stays.
    print(f"relbias table gradient {k} keys {len(starts)} starts bidirectional={bidirectional}", flush=True)
    H, cut, rng = 48, last_split(k), np.random.default_rng(8)
    for pos in sorted({max(0, v) for v in (0, cut - 3, cut, cut + 5, cut + 37, cut + 190, k // 2, k - 1)}):
        p, dp = np.zeros((1, H, 3, k), np.uint16), np.full((1, H, 3, k), -0.0, np.float32)
        for h in range(H):
            if cut and h % 2:   # the last addition's two sides
                a, b = max(0, cut - 1 - rng.integers(0, 4)), min(k - 1, cut + rng.integers(0, 4))
            else:               # the row's end
                b = k - 1 - rng.integers(0, min(3, k - 1))
                a = max(0, b - 1 - rng.integers(0, 3))
            p[0, h, :2, a], dp[0, h, :2, a] = 0x3F00, (4 * TINY, -6 * TINY)
            p[0, h, 2, [a, b]], dp[0, h, 2, [a, b]] = 0x3E80, (3 * TINY, -7 * TINY)
        got, want = relative_bias_backward(p, dp, starts, bidirectional, pos)
        if starts == [0] and (not bidirectional or pos == 0):
            assert minus_zeros(want[1]) > H // 8
        assert_bits(got[0], want[0], "dscores")
        assert_bits(got[1], want[1], "dtable")


@pytest.mark.parametrize("k", [2, 31, 32, 33, 64, 65, 97, 256, 300, 700, 1100, 2500])
@pytest.mark.parametrize("starts,bidirectional", BUCKETS)
def test_relative_bias_gradient_of_unseen_keys(k, starts, bidirectional):
    # keys that are not seen are terms of +0, unlike those that are not there: a -0 before them does not stay
    print(f"relbias masked {k} keys {len(starts)} starts bidirectional={bidirectional}", flush=True)
    rng = np.random.default_rng(9)
    for masks in (dict(causal=True), dict(window=max(1, k // 3)), dict(k_len=k - 1), dict(causal=True, window=20, k_len=k // 2 + 1)):
        dp = tiny_rows(64, k, 10).reshape(1, 8, 8, k)
        p = np.where((rng.random(dp.shape) < 0.5) & (dp == 0), 0, ONE).astype(np.uint16)
        for pos in sorted({0, k // 2, k - 1}):
            got, want = relative_bias_backward(p, dp, starts, bidirectional, pos, **masks)
            assert_bits(got[0], want[0], "dscores")
            assert_bits(got[1], want[1], "dtable")
