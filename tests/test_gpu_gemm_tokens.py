"""canon_quant_tokens and canon_gemm_i8_tokens: bit-identical to the oracle over sizes around every kernel's tiles, types,
leading dimensions off any alignment, and special values."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, host_f32, host_u16
from serve_util import from_bf16

pytestmark = pytest.mark.gpu


def bf16_bits(x):
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().view(torch.int16).numpy().view(np.uint16)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 3), (2, 255), (3, 256), (2, 257), (3, 512), (2, 1001), (2, 1024),
                                       (3, 2048), (2, 2051), (2, 4096), (3, 5632), (2, 8192), (2, 8193), (2, 16384), (2, 16387),
                                       (1, 65536), (300, 64), (4, 0)])
@pytest.mark.parametrize("bf16", [False, True])
def test_quant_tokens(rows, cols, bf16):
    x = I.normal_f32((rows, max(cols, 1)), rows, 61)[:, :cols] * np.float32(4)
    if cols > 2 and rows > 1:
        x[1, 1] = np.nan
        x[0] = np.where(np.arange(cols) % 3 == 0, 127, 63.5) if rows > 2 else x[0]
        if rows > 2:
            x[2] = 0
    if bf16:
        x = from_bf16(bf16_bits(x)).reshape(rows, cols)
    codes = torch.full((rows * cols + 1,), 99, dtype=torch.int8, device=DEV)
    steps = torch.full((rows,), 7.0, device=DEV)
    d = (dev_bf16(bf16_bits(x)) if bf16 else dev_f32(x)).view(rows, cols)
    odd = torch.empty(rows * cols + 1, dtype=d.dtype, device=DEV)
    odd[1:] = d.reshape(-1)
    C.quant_tokens(rows, cols, odd[1:].view(rows, cols), codes[1:], steps)
    torch.cuda.synchronize()
    assert codes[0].item() == 99
    if cols == 0:
        assert (steps == 0).all()
        return
    wc, ws = oracle.act8_pack(x, cols)
    got = steps.cpu().numpy()
    assert (np.isnan(got) == np.isnan(ws[:, 0])).all()
    assert_bits(np.nan_to_num(got), np.nan_to_num(ws[:, 0]), "steps")
    assert (codes[1:].cpu().numpy().reshape(rows, cols) == wc).all()


def codes(shape, seed):
    return np.random.default_rng(seed).integers(-128, 128, shape).astype(np.int8)


def product(a, sa, b, sb, dtype, pads=(0, 0, 0)):
    (m, k), n = a.shape, b.shape[0]

    def lay(x, pad):
        t = torch.full((x.shape[0], x.shape[1] + pad), 77, dtype=torch.int8, device=DEV)
        t[:, :x.shape[1]] = torch.from_numpy(x).to(DEV)
        return t

    y = torch.full((m, n + pads[2]), 7.0, dtype=dtype, device=DEV)
    C.gemm_i8_tokens(m, n, k, lay(a, pads[0]), k + pads[0], dev_f32(sa), lay(b, pads[1]), k + pads[1], dev_f32(sb), y, ldc=n + pads[2])
    torch.cuda.synchronize()
    assert (y[:, n:] == 7.0).all()
    return y[:, :n].contiguous()


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 7, 15), (1, 16, 16), (2, 17, 17), (3, 40, 63), (15, 33, 64), (16, 8, 65),
                                   (17, 100, 500), (31, 64, 512), (33, 65, 1030), (64, 2056, 2048), (64, 48, 8192), (65, 130, 72),
                                   (1, 5001, 2056), (100, 300, 129), (129, 257, 640), (256, 256, 64), (256, 512, 192), (300, 200, 0),
                                   (5, 9, 0), (1, 300, 65536), (66, 70, 4000), (700, 1300, 260), (70, 2500, 140), (1290, 3300, 130),
                                   (130, 12400, 300), (650, 1300, 12), (650, 1300, 700),
                                   (3584, 3584, 64)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_product(m, n, k, dtype):
    a, b = codes((m, k), m + k), codes((n, k), n)
    sa, sb = (np.exp(I.normal_f32((x,), x, 62)).astype(np.float32) for x in (m, n))
    want = oracle.gemm_i8_tokens(a, sa, b, sb)
    for pads in ((0, 0, 0), (3, 1, 5), (16, 32, 8)):
        y = product(a, sa, b, sb, dtype, pads)
        if dtype == torch.float32:
            assert_bits(host_f32(y), want, f"product {pads}")
        else:
            assert_bits(host_u16(y), bf16_bits(want), f"product {pads}")


def test_extreme_codes_and_steps():
    # the largest sums: -128 x -128 over 65536 terms is 2^30
    for m in (2, 70):
        a, b = np.full((m, 65536), -128, np.int8), np.full((9, 65536), -128, np.int8)
        b[1] = 127
        sa, sb = np.ones(m, np.float32), np.array([1, 2, np.nan, np.inf, 1e-38, 1e-45, 3e38, 0, -1], np.float32)
        sa[1] = np.inf
        want = oracle.gemm_i8_tokens(a, sa, b, sb)
        for dtype in (torch.float32, torch.bfloat16):
            y = product(a, sa, b, sb, dtype).float().cpu().numpy()
            ref = want if dtype == torch.float32 else torch.from_numpy(want).bfloat16().float().numpy()
            assert np.array_equal(y, ref, equal_nan=True)


def test_a_projection_of_tokens():
    """Activations into 8 bits and through weights kept in 8 bits: near the product of the values that they stand for."""
    for m in (1, 40, 256):
        x = I.normal_f32((m, 512), 1, 63)
        w = I.normal_f32((256, 512), 2, 64)
        wc, ws = oracle.act8_pack(w, 512)
        q, s = torch.empty(m, 512, dtype=torch.int8, device=DEV), torch.empty(m, device=DEV)
        y = torch.empty(m, 256, device=DEV)
        C.quant_tokens(m, 512, dev_f32(x), q, s)
        C.gemm_i8_tokens(m, 256, 512, q, 512, s, torch.from_numpy(wc).to(DEV), 512, dev_f32(ws[:, 0].copy()), y)
        torch.cuda.synchronize()
        ref = (q.cpu().numpy().astype(np.float64) * host_f32(s)[:, None]) @ (wc.astype(np.float64) * ws).T
        # three roundings of 2^-24: the sum's, and one for each step
        assert (np.abs(y.cpu().numpy() - ref) <= 3 * 2.0 ** -24 * np.abs(ref) + 1e-30).all()
