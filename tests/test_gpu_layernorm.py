"""canon_layernorm and canon_layernorm_bwd: bit-identical to the oracle at row lengths around their vectors, chunks and
workgroup shapes, from pointers off any alignment, and near the formula in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, host_f32, host_u16, poisoned_workspace

pytestmark = pytest.mark.gpu

EPS = float(np.float32(1e-5))


def off(t):
    """A copy of t that starts one element off the allocation's alignment."""
    u = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)[1:].view(t.shape)
    u.copy_(t)
    return u


def new(*shape, dtype=torch.float32):
    """An output off any alignment, NaN (or 255) all over."""
    return off(torch.full(shape, float("nan"), dtype=dtype, device=DEV) if dtype.is_floating_point
               else torch.full(shape, -1, dtype=dtype, device=DEV))


def inputs(rows, cols, dtype, seed=0):
    x = I.normal_f32((rows, cols), seed, 3) * np.float32(2) + np.float32(0.5)
    if dtype == torch.bfloat16:
        x = I.bf16_bits_to_f32(host_bf16(x))
    return (x, I.normal_bf16((cols,), seed, 200, std=0.1, mean=1.0), I.normal_bf16((cols,), seed, 201, std=0.1),
            I.normal_f32((rows, cols), seed, 7))


def host_bf16(x):
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def on_device(x, dtype):
    return off(dev_f32(x) if dtype == torch.float32 else dev_bf16(host_bf16(x)))


def keep_for(rows, cols, group):
    return C.Act8(group, new(rows, cols, dtype=torch.int8), new(rows, C.act8_groups(cols, group)))


def run(x, gain, bias, dy, dtype, y_dtype, group=None):
    """Forward (keeping x in 8 bits if a group is given) and backward; every output as numpy."""
    rows, cols = x.shape
    xd, gd, bd, dyd = on_device(x, dtype), off(dev_bf16(gain)), None if bias is None else off(dev_bf16(bias)), off(dev_f32(dy))
    y, mean, rstd = new(rows, cols, dtype=y_dtype), new(rows), new(rows)
    kept = None if group is None else keep_for(rows, cols, group)
    C.layernorm(rows, cols, xd, gd, bd, EPS, y, mean, rstd, keep=kept)
    dx, dg, db = new(rows, cols), new(cols), new(cols)
    ws = poisoned_workspace(C.layernorm_bwd_workspace_bytes(rows, cols))
    C.layernorm_bwd(rows, cols, xd if kept is None else kept, gd, mean, rstd, dyd, dx, ws, dgain=dg, dbias=db)
    torch.cuda.synchronize()
    out = {"y": host_u16(y) if y_dtype == torch.bfloat16 else host_f32(y), "mean": host_f32(mean), "rstd": host_f32(rstd),
           "dx": host_f32(dx), "dgain": host_f32(dg), "dbias": host_f32(db)}
    if kept is not None:
        out |= {"codes": kept.tensors[0].cpu().numpy(), "steps": host_f32(kept.tensors[1])}
    return out


def wanted(x, gain, bias, dy, y_dtype, group=None):
    y, mean, rstd = oracle.layernorm_fwd(x, gain, bias, EPS)
    out = {"y": host_bf16(y) if y_dtype == torch.bfloat16 else y, "mean": mean, "rstd": rstd}
    if group is not None:
        out["codes"], out["steps"] = oracle.act8_pack(x, group)
        x = oracle.act8_unpack(out["codes"], out["steps"], group)
    out["dx"], out["dgain"], out["dbias"] = oracle.layernorm_bwd(x, gain, mean, rstd, dy)
    return out


def same(got, want):
    for name in want:
        if name == "codes":
            assert np.array_equal(got[name], want[name]), name
        else:
            assert_bits(got[name], want[name], name)


SHAPES = [(1, 1), (1, 7), (5, 33), (33, 64), (3, 255), (40, 2047), (32, 2048), (65, 2049), (9, 2052), (7, 4096), (5, 4097),
          (3, 8192), (2, 8195), (3, 16384), (2, 16388), (2, 32767), (1, 32768)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matches_the_oracle(rows, cols, dtype):
    print(f"layer norm {rows}x{cols} {dtype}", flush=True)
    x, g, b, dy = inputs(rows, cols, dtype)
    for y_dtype in (torch.float32, torch.bfloat16):
        same(run(x, g, b, dy, dtype, y_dtype), wanted(x, g, b, dy, y_dtype))
    same(run(x, g, None, dy, dtype, torch.float32), wanted(x, g, None, dy, torch.float32))


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128, 256])
def test_from_8_bits_matches_the_oracle(rows, cols, group):
    print(f"layer norm in 8 bits {rows}x{cols} group {group}", flush=True)
    dtype = torch.float32 if group in (32, 256) else torch.bfloat16
    x, g, b, dy = inputs(rows, cols, dtype, seed=1)
    same(run(x, g, b, dy, dtype, torch.bfloat16, group), wanted(x, g, b, dy, torch.bfloat16, group))


@pytest.mark.parametrize("rows", [31, 32, 33, 1023, 1024, 1057, 4100])
def test_reductions_over_rows(rows):
    # around a chain of 32 rows and the 16 blocks of the fold
    cols = 37
    print(f"rows {rows}", flush=True)
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=2)
    same(run(x, g, b, dy, torch.float32, torch.float32), wanted(x, g, b, dy, torch.float32))


@pytest.mark.parametrize("cols", [3, 512, 516, 1021, 1024, 1500, 2048, 2050, 4093, 4096, 4099, 5000, 8189, 8192, 8200])
@pytest.mark.parametrize("rows,dtype,group", [(4096, torch.float32, None), (4101, torch.bfloat16, None), (4127, torch.float32, 128)])
def test_one_pass_over_many_rows(rows, cols, dtype, group):
    # from 4096 rows on the backward is one pass (up to 8192 columns); a whole and a cut last chain, rows that four at a time
    # do not divide
    print(f"layer norm {rows}x{cols} {dtype} group {group}", flush=True)
    x, g, b, dy = inputs(rows, cols, dtype, seed=9)
    same(run(x, g, b, dy, dtype, torch.bfloat16, group), wanted(x, g, b, dy, torch.bfloat16, group))


@pytest.mark.parametrize("rows,cols", [(8193, 1021), (8200, 1024), (16390, 510), (16384, 511), (32769, 4), (32800, 5), (32771, 6),
                                       (32800, 7), (32800, 3), (32770, 254)])
@pytest.mark.parametrize("dtype,group", [(torch.float32, None), (torch.bfloat16, None), (torch.float32, 32), (torch.bfloat16, 64)])
def test_one_pass_over_narrow_rows(rows, cols, dtype, group):
    # narrower rows are one pass from more of them on, and every cut of the last vector, rows of one vector among them; of
    # rows of three columns there is no whole vector
    print(f"layer norm {rows}x{cols} {dtype} group {group}", flush=True)
    x, g, b, dy = inputs(rows, cols, dtype, seed=10)
    same(run(x, g, b, dy, dtype, torch.bfloat16, group), wanted(x, g, b, dy, torch.bfloat16, group))


@pytest.mark.parametrize("rows,cols", [(256, 2048), (512, 2047), (513, 2048), (1023, 2048), (2048, 1030), (2050, 1025), (300, 8191),
                                       (600, 8190)])
def test_row_counts_around_the_shapes(rows, cols):
    # rows spread over more wavefronts up to eight to a CU of 2048 columns each
    print(f"layer norm {rows}x{cols}", flush=True)
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=10)
    same(run(x, g, b, dy, torch.float32, torch.float32, 64), wanted(x, g, b, dy, torch.float32, 64))


def test_no_rows():
    cols = 50
    z = torch.empty(0, dtype=torch.float32, device=DEV)
    g = dev_bf16(np.full(cols, 0x3F80, np.uint16))
    dg, db = new(cols), new(cols)
    C.layernorm(0, cols, z, g, None, EPS, z, z, z)
    C.layernorm_bwd(0, cols, z, g, z, z, z, z, poisoned_workspace(C.layernorm_bwd_workspace_bytes(0, cols)), dgain=dg,
                    dbias=db)
    torch.cuda.synchronize()
    assert not host_f32(dg).view(np.uint32).any() and not host_f32(db).view(np.uint32).any()


def test_one_gradient_alone():
    rows, cols = 70, 300
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=3)
    want = wanted(x, g, b, dy, torch.float32)
    xd, gd, dyd = dev_f32(x), dev_bf16(g), dev_f32(dy)
    m, r = dev_f32(want["mean"]), dev_f32(want["rstd"])
    for name in ("dgain", "dbias", None):
        dx, part = new(rows, cols), new(cols)
        ws = poisoned_workspace(C.layernorm_bwd_workspace_bytes(rows, cols)) if name else None
        C.layernorm_bwd(rows, cols, xd, gd, m, r, dyd, dx, ws, **({name: part} if name else {}))
        torch.cuda.synchronize()
        assert_bits(host_f32(dx), want["dx"], "dx")
        if name:
            assert_bits(host_f32(part), want[name], name)


def sum_error(n):
    """Relative error, against the sum of magnitudes, of an R1 sum of n terms: at most 32 additions of a chain and
    log2(n / 32) + 1 of the fold, half a unit of 2^-23 each, and one rounding per term before."""
    return (34 + max(0, int(np.ceil(np.log2(max(n, 1) / 32)))) + 1) * 2.0 ** -24


@pytest.mark.parametrize("rows,cols", [(4, 33), (70, 1000), (3, 2500)])
def test_near_the_formula_in_64_bits(rows, cols):
    print(f"64 bits {rows}x{cols}", flush=True)
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=4)
    got = run(x, g, b, dy, torch.float32, torch.float32)
    X, G, B, DY = x.astype(np.float64), I.bf16_bits_to_f32(g).astype(np.float64), I.bf16_bits_to_f32(b).astype(np.float64), dy.astype(np.float64)
    mean, var = X.mean(1), X.var(1)
    rstd = 1 / np.sqrt(var + EPS)
    xh = (X - mean[:, None]) * rstd[:, None]
    u, su = 2.0 ** -24, sum_error(cols)
    # mean: the sum's error and a rounding (and that of 1/n) more
    tol_mean = (su + 2 * u) * np.abs(X).mean(1)
    assert np.all(np.abs(got["mean"] - mean) <= tol_mean)
    # variance: squares of differences that are tol_mean and a rounding off; the root halves it, plus four roundings
    tol_r = 0.5 * (su + 4 * u + 2 * (tol_mean[:, None] + u * np.abs(X - mean[:, None])).max(1) * np.abs(xh).mean(1) * rstd) + 4 * u
    assert np.all(np.abs(got["rstd"] / rstd - 1) <= tol_r)
    tol_xh = np.abs(xh) * (tol_r[:, None] + 3 * u) + (tol_mean * rstd)[:, None]
    assert np.all(np.abs(got["y"] - (xh * G + B)) <= tol_xh * np.abs(G) + 2 * u * (np.abs(xh * G) + np.abs(B)) + 1e-30)
    gy = DY * G
    m1, m2 = gy.mean(1), (gy * xh).mean(1)
    want = rstd[:, None] * (gy - m1[:, None] - xh * m2[:, None])
    tol_m1 = (su + 3 * u) * np.abs(gy).mean(1)
    tol_m2 = (su + 4 * u) * np.abs(gy * xh).mean(1) + (np.abs(gy) * tol_xh).mean(1)
    inner = (u * 3 * (np.abs(gy) + np.abs(m1[:, None]) + np.abs(xh * m2[:, None])) + tol_m1[:, None]
             + np.abs(xh) * tol_m2[:, None] + tol_xh * np.abs(m2[:, None]))
    assert np.all(np.abs(got["dx"] - want) <= rstd[:, None] * inner * (1 + 1e-5) + np.abs(want) * (tol_r[:, None] + 2 * u))
    rows_err = sum_error(rows)
    assert np.all(np.abs(got["dbias"] - DY.sum(0)) <= rows_err * np.abs(DY).sum(0))
    assert np.all(np.abs(got["dgain"] - (DY * xh).sum(0)) <= (rows_err + 2 * u) * np.abs(DY * xh).sum(0) * 1.01
                  + (np.abs(DY) * tol_xh).sum(0) * 1.01)


def test_gradients_against_differences():
    # central differences in 64 bits of the loss sum(w y): a step h leaves an error of third derivatives, h^2 / 6 of them,
    # all of order 1 here
    rows, cols = 3, 40
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=5)
    got = run(x, g, b, dy, torch.float32, torch.float32)
    G, B, W = (v.astype(np.float64) for v in (I.bf16_bits_to_f32(g), I.bf16_bits_to_f32(b), dy))

    def loss(X, gain, bias):
        d = X - X.mean(1, keepdims=True)
        return float((W * (d / np.sqrt((d * d).mean(1, keepdims=True) + EPS) * gain + bias)).sum())

    X, h = x.astype(np.float64), 1e-4
    rng = np.random.default_rng(0)
    for r, c in zip(rng.integers(0, rows, 12), rng.integers(0, cols, 12)):
        e = np.zeros_like(X)
        e[r, c] = h
        assert abs((loss(X + e, G, B) - loss(X - e, G, B)) / (2 * h) - got["dx"][r, c]) < 2e-5
        v = np.zeros(cols)
        v[c] = h
        assert abs((loss(X, G + v, B) - loss(X, G - v, B)) / (2 * h) - got["dgain"][c]) < 2e-5
        assert abs((loss(X, G, B + v) - loss(X, G, B - v)) / (2 * h) - got["dbias"][c]) < 2e-5


def test_special_rows():
    # constant rows (variance 0), a NaN and an infinity: their rows alone are NaN, and no other row changes
    rows, cols = 6, 96
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=6)
    x[1], x[2] = 3.0, 0.0
    x[3, 5], x[4, 90] = np.nan, np.inf
    got = run(x, g, b, dy, torch.float32, torch.float32, 32)
    want = wanted(x, g, b, dy, torch.float32, 32)
    ok = [0, 1, 2, 5]
    for name in ("y", "dx"):
        assert_bits(got[name][ok], want[name][ok], name)
        assert np.isnan(got[name][3]).all() and np.isnan(got[name][4]).all()
    assert np.array_equal(got["codes"], want["codes"])


def test_captured_with_an_eager_call_between():
    rows, cols = 100, 2048
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=7)
    want = wanted(x, g, b, dy, torch.bfloat16, 128)
    xd, gd, bd, dyd = torch.zeros((rows, cols), device=DEV), dev_bf16(g), dev_bf16(b), dev_f32(dy)
    y, mean, rstd, kept = new(rows, cols, dtype=torch.bfloat16), new(rows), new(rows), keep_for(rows, cols, 128)
    dx, dg, db = new(rows, cols), new(cols), new(cols)
    ws = poisoned_workspace(C.layernorm_bwd_workspace_bytes(rows, cols))

    def both():
        C.layernorm(rows, cols, xd, gd, bd, EPS, y, mean, rstd, keep=kept)
        C.layernorm_bwd(rows, cols, kept, gd, mean, rstd, dyd, dx, ws, dgain=dg, dbias=db)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        xd.zero_()
        both()
        xd.copy_(dev_f32(x))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same({"y": host_u16(y), "mean": host_f32(mean), "rstd": host_f32(rstd), "dx": host_f32(dx), "dgain": host_f32(dg),
              "dbias": host_f32(db)}, {n: want[n] for n in ("y", "mean", "rstd", "dx", "dgain", "dbias")})


def test_another_stream():
    rows, cols = 64, 1000
    x, g, b, dy = inputs(rows, cols, torch.float32, seed=8)
    want = wanted(x, g, b, dy, torch.float32)
    s = torch.cuda.Stream()
    xd, gd, bd = dev_f32(x), dev_bf16(g), dev_bf16(b)
    y, mean, rstd = new(rows, cols), new(rows), new(rows)
    s.wait_stream(torch.cuda.current_stream())
    C.layernorm(rows, cols, xd, gd, bd, EPS, y, mean, rstd, stream=s)
    s.synchronize()
    assert_bits(host_f32(y), want["y"], "y")
