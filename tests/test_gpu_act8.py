"""Activations kept in 8 bits, and SwiGLU that keeps and reads them: bit-identical to the oracle, near 64 bits, and special
values, from pointers off any alignment."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, host_f32, host_u16
from test_gpu_layernorm import host_bf16, keep_for, new, off, on_device

pytestmark = pytest.mark.gpu


def activations(rows, cols, dtype, seed=0):
    x = I.normal_f32((rows, cols), seed, 5) * np.exp2(np.arange(rows) % 7 - 3).astype(np.float32)[:, None]
    return I.bf16_bits_to_f32(host_bf16(x)) if dtype == torch.bfloat16 else x


def pack(x, dtype, group):
    rows, cols = x.shape
    kept = keep_for(rows, cols, group)
    C.act8_pack(rows, cols, on_device(x, dtype), kept)
    torch.cuda.synchronize()
    return kept


SHAPES = [(1, 1), (1, 5), (7, 31), (3, 32), (5, 33), (4, 255), (3, 256), (9, 257), (2, 1023), (2, 1024), (3, 1025), (40, 704),
          (1, 70001), (300, 100)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pack_and_unpack_match_the_oracle(rows, cols, group, dtype):
    print(f"act8 {rows}x{cols} group {group} {dtype}", flush=True)
    x = activations(rows, cols, dtype)
    codes, steps = oracle.act8_pack(x, group)
    kept = pack(x, dtype, group)
    assert np.array_equal(kept.tensors[0].cpu().numpy(), codes)
    assert_bits(host_f32(kept.tensors[1]), steps, "steps")
    want = oracle.act8_unpack(codes, steps, group)
    f, h = new(rows, cols), new(rows, cols, dtype=torch.bfloat16)
    C.act8_unpack(rows, cols, kept, f)
    C.act8_unpack(rows, cols, kept, h)
    torch.cuda.synchronize()
    assert_bits(host_f32(f), want, "fp32")
    assert_bits(host_u16(h), host_bf16(want), "bf16")
    # the nearest multiple of the step, the quotient rounded to binary32 before (at most 127 (1 + 2^-23) steps)
    s = np.repeat(steps, group, 1)[:, :cols].astype(np.float64)
    assert np.all(np.abs(want.astype(np.float64) - x) <= s * (0.5 + 128 * 2.0 ** -24) + np.abs(x) * 2.0 ** -23)


def test_special_groups():
    group, cols = 32, 160
    x = activations(3, cols, torch.float32, seed=1)
    x[0, :32] = 0.0
    x[0, 40], x[0, 70], x[0, 100] = np.nan, np.inf, -np.inf
    x[1, 32:64] = 1e-39      # subnormal
    x[1, 64:96] = 3e-38      # its step is flushed
    x[2, 3] = 3e38
    codes, steps = oracle.act8_pack(x, group)
    kept = pack(x, torch.float32, group)
    got_codes, got_steps = kept.tensors[0].cpu().numpy(), host_f32(kept.tensors[1])
    assert np.array_equal(got_codes, codes)
    assert np.array_equal(np.isnan(got_steps), np.isnan(steps)) and np.isnan(steps[0, 1])
    assert np.array_equal(got_steps[~np.isnan(steps)].view(np.uint32), steps[~np.isnan(steps)].view(np.uint32))
    f = new(3, cols)
    C.act8_unpack(3, cols, kept, f)
    torch.cuda.synchronize()
    f = host_f32(f)
    assert not f[0, :32].any() and not f[1, 32:96].any()
    assert np.isnan(f[0, 32:128]).all()
    assert np.isfinite(f[1:]).all() and np.isfinite(f[0, 128:]).all()


def test_ties_and_borders():
    # every half step of a group whose step is a power of two: exact quotients, ties to even
    k = np.arange(-254, 255, dtype=np.float32) * np.float32(0.5)
    x = np.zeros((2, 512), np.float32)
    x[0, :254], x[1, :255] = k[:254], k[254:]
    x[:, 256:], x[:, 255] = 127.0, 127.0
    x[0, 256] = -127.0
    codes, steps = oracle.act8_pack(x, 256)
    kept = pack(x, torch.float32, 256)
    assert np.array_equal(kept.tensors[0].cpu().numpy(), codes)
    assert codes.min() == -127 and codes.max() == 127


def test_a_long_row():
    # more than 2^31 bytes of fp32 in one row of whole groups; first, middle and last elements against the oracle
    rows, cols, group = 3, 1 << 28, 128
    print("act8 3 x 2^28", flush=True)
    x = torch.randn(rows * cols, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).view(rows, cols)
    kept = C.Act8(group, torch.empty((rows, cols), dtype=torch.int8, device=DEV),
                  torch.empty((rows, cols // group), dtype=torch.float32, device=DEV))
    C.act8_pack(rows, cols, x, kept)
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    C.act8_unpack(rows, cols, kept, y)
    torch.cuda.synchronize()
    for r, c in ((0, 0), (1, 12345 * group), (2, cols - 1024)):
        part = host_f32(x[r, c:c + 1024])[None]
        codes, steps = oracle.act8_pack(part, group)
        assert np.array_equal(kept.tensors[0][r, c:c + 1024].cpu().numpy(), codes[0])
        assert_bits(host_u16(y[r, c:c + 1024]), host_bf16(oracle.act8_unpack(codes, steps, group))[0], "values")
    # a value v is at most s (1/2 + 2^-17) from x, its bf16 rounding at most 2^-8 |v| <= 2^-8 (|x| + s (1/2 + 2^-17)) from v:
    # together s (1/2 + 2^-17) (1 + 2^-8) + 2^-8 |x|, 0.50197 s
    worst = ((y.float() - x).abs() - kept.tensors[1].repeat_interleave(group, 1) * 0.502 - x.abs() * 2.0 ** -8).max()
    assert float(worst) <= 0


def swiglu_wanted(gu, da, F):
    g, u = np.ascontiguousarray(gu[:, :F]), np.ascontiguousarray(gu[:, F:])
    lib = oracle._load()
    n = g.size
    a, dg, du = (np.empty(g.shape, np.uint16) for _ in range(3))
    assert lib.cref_swiglu(n, oracle._p(g), oracle._p(u), oracle._p(np.ascontiguousarray(da)), oracle._p(a), oracle._p(dg),
                           oracle._p(du)) == 0
    return a, np.concatenate((dg, du), 1)


@pytest.mark.parametrize("T,F", [(1, 1), (3, 31), (2, 64), (5, 255), (4, 512), (3, 513), (2, 1100), (192, 704)])
@pytest.mark.parametrize("group,dtype", [(32, torch.bfloat16), (64, torch.float32), (128, torch.bfloat16), (256, torch.float32)])
def test_swiglu_matches_the_oracle(T, F, group, dtype):
    print(f"swiglu {T}x{F} group {group} {dtype}", flush=True)
    gu = activations(T, 2 * F, dtype, seed=2)
    da = I.normal_f32((T, F), 2, 9)
    x, dad = on_device(gu, dtype), off(dev_f32(da))
    kept = keep_for(2 * T, F, group)
    bf = torch.bfloat16
    a, a2, a8 = (new(T, F, dtype=bf) for _ in range(3))
    dgu, dgu8 = new(T, 2 * F, dtype=bf), new(T, 2 * F, dtype=bf)
    C.swiglu(T, F, x, a, keep=kept)
    C.swiglu(T, F, x, a2)
    C.swiglu_bwd(T, F, x, dad, dgu)
    C.swiglu_bwd(T, F, kept, dad, dgu8, a=a8)
    torch.cuda.synchronize()
    want_a, want_d = swiglu_wanted(gu, da, F)
    assert_bits(host_u16(a), want_a, "a with keep")
    assert_bits(host_u16(a2), want_a, "a")
    assert_bits(host_u16(dgu), want_d, "dgu")
    codes, steps = oracle.act8_pack(gu.reshape(2 * T, F), group)
    assert np.array_equal(kept.tensors[0].cpu().numpy(), codes)
    assert_bits(host_f32(kept.tensors[1]), steps, "steps")
    a_w, d_w = swiglu_wanted(oracle.act8_unpack(codes, steps, group).reshape(T, 2 * F), da, F)
    assert_bits(host_u16(a8), a_w, "a from 8 bits")
    assert_bits(host_u16(dgu8), d_w, "dgu from 8 bits")


def test_swiglu_near_64_bits_and_against_differences():
    T, F = 7, 100
    gu = activations(T, 2 * F, torch.float32, seed=3)
    da = I.normal_f32((T, F), 3, 9)
    a, dgu = new(T, F, dtype=torch.bfloat16), new(T, 2 * F, dtype=torch.bfloat16)
    C.swiglu(T, F, dev_f32(gu), a)
    C.swiglu_bwd(T, F, dev_f32(gu), dev_f32(da), dgu)
    torch.cuda.synchronize()
    g, u, d = gu[:, :F].astype(np.float64), gu[:, F:].astype(np.float64), da.astype(np.float64)

    def f(g, u):
        return g / (1 + np.exp(-g)) * u

    # half a bf16 unit (2^-8 relative at most half of 2^-7), and a few units of 2^-24 of what the sums of the sigmoid's
    # derivative cancel
    tol = 2.0 ** -8 + 2.0 ** -18
    assert np.all(np.abs(I.bf16_bits_to_f32(host_u16(a)) - f(g, u)) <= tol * np.abs(f(g, u)) + 1e-37)
    h = 1e-5  # the third derivatives are below 2 |u| and |g|: an error of h^2
    got = I.bf16_bits_to_f32(host_u16(dgu)).astype(np.float64)
    dg = d * (f(g + h, u) - f(g - h, u)) / (2 * h)
    du = d * (f(g, u + h) - f(g, u - h)) / (2 * h)
    assert np.all(np.abs(got[:, :F] - dg) <= tol * np.abs(dg) + 1e-6 * np.abs(d * u))
    assert np.all(np.abs(got[:, F:] - du) <= tol * np.abs(du) + 1e-6 * np.abs(d * g) + 1e-9)


def test_swiglu_special_values():
    gu = np.array([[0.0, -0.0, np.inf, -200.0, 200.0, np.nan, 1.0, -90.0] + [1.0] * 8], np.float32)
    da = np.ones((1, 8), np.float32)
    a, dgu = new(1, 8, dtype=torch.bfloat16), new(1, 16, dtype=torch.bfloat16)
    C.swiglu(1, 8, dev_f32(gu), a)
    C.swiglu_bwd(1, 8, dev_f32(gu), dev_f32(da), dgu)
    torch.cuda.synchronize()
    wa, wd = swiglu_wanted(gu, da, 8)

    def same(x, y):
        x, y = I.bf16_bits_to_f32(x), I.bf16_bits_to_f32(y)
        assert np.array_equal(np.isnan(x), np.isnan(y)) and np.array_equal(x[~np.isnan(x)], y[~np.isnan(y)])

    same(host_u16(a), wa)
    same(host_u16(dgu), wd)
