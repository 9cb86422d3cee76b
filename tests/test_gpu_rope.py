"""canon_rope: bit-identical to the oracle over layouts, types, strides and positions, in place, and its gradient; a block's
rotation through it."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_17380_amd.canon as C
import paper_2609_17380_amd.inputs as I
from gpu_util import DEV, assert_bits, dev_bf16, dev_f32, dev_i32, host_f32, host_u16
from serve_util import from_bf16, tables

pytestmark = pytest.mark.gpu


def bf16_bits(x):
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().view(torch.int16).numpy().view(np.uint16)


def check(tokens, heads, dim, rot, inter, xb, yb, backward, pos, cos, sin, x=None, pad=0, in_place=False, positions=None):
    if x is None:
        x = I.normal_f32((tokens, heads, dim), tokens + dim, 51)
    if xb:
        x = from_bf16(bf16_bits(x)).reshape(x.shape)
    d = (dev_bf16(bf16_bits(x)) if xb else dev_f32(x)).view(tokens, heads * dim)
    if pad:
        wide = torch.full((tokens, heads * dim + pad), float("nan"), dtype=d.dtype, device=DEV)
        wide[:, 1:1 + heads * dim] = d
        d = wide[:, 1:1 + heads * dim]
    y = d if in_place else torch.full((tokens, heads * dim + pad), 7.0, dtype=torch.bfloat16 if yb else torch.float32,
                                      device=DEV)[:, pad:]
    turn = C.Rotation(dev_f32(cos), dev_f32(sin), rot, interleaved=inter)
    C.rope(tokens, heads, dim, turn, d, y, positions=None if pos is None else dev_i32(pos), backward=backward)
    torch.cuda.synchronize()
    want = oracle.rope(x, np.arange(tokens) if pos is None else pos, cos, sin, rot, inter, backward)
    y = y.contiguous()
    if yb:
        got = host_u16(y).reshape(want.shape)
        nan = np.isnan(want)
        assert (np.isnan(from_bf16(got)) == nan).all()
        assert_bits(np.where(nan, 0, got).astype(np.uint16), np.where(nan, 0, bf16_bits(want)).astype(np.uint16), "rope")
    else:
        got = host_f32(y).reshape(want.shape)
        nan = np.isnan(want)
        assert (np.isnan(got) == nan).all()
        assert_bits(np.where(nan, 0, got).astype(np.float32), np.where(nan, 0, want).astype(np.float32), "rope")
    return want


@pytest.mark.parametrize("tokens,heads,dim,rot", [(1, 1, 2, 2), (1, 16, 128, 128), (5, 3, 64, 32), (33, 12, 96, 24), (7, 2, 50, 48),
                                                  (3, 5, 7, 6), (3, 5, 7, 0), (129, 2, 256, 64), (4, 1, 1024, 1024), (9, 4, 80, 40)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("backward", [False, True])
def test_matches_the_oracle(tokens, heads, dim, rot, inter, backward):
    cos, sin = tables(max(rot, 2), 200)
    cos, sin = cos[:, :max(rot // 2, 1)], sin[:, :max(rot // 2, 1)]
    pos = np.random.default_rng(tokens).integers(0, 200, tokens).astype(np.int32)
    for xb, yb in ((False, False), (True, True), (False, True), (True, False)):
        for p, pad in ((pos, 0), (None, 13)):
            check(tokens, heads, dim, rot, inter, xb, yb, backward, p, cos, sin, pad=pad)
        if xb == yb:
            check(tokens, heads, dim, rot, inter, xb, yb, backward, pos, cos, sin, in_place=True, pad=5)


def test_positions_without_an_angle_and_special_values():
    cos, sin = tables(32, 10)
    pos = np.array([0, 9, 10, -1, 1 << 30, -(1 << 31), 5], np.int32)
    x = I.normal_f32((7, 2, 48), 1, 52)
    x[0, 0, :8] = [np.inf, -np.inf, np.nan, 1e-40, -1e-40, 0.0, -0.0, 3e38]
    x[1, 1, 40:44] = [np.inf, np.nan, 1e-40, -1e-40]  # kept elements
    x[6, 0] *= np.float32(1e-38)
    for inter in (False, True):
        for yb in (False, True):
            want = check(7, 2, 48, 32, inter, False, yb, False, pos, cos, sin, x=x)
            assert np.isnan(want[2:6, :, :32]).all() and not np.isnan(want[2:6, :, 32:]).any()


def test_backward_is_the_gradient():
    # <dy, R x> = <R^T dy, x> in 64 bits up to the roundings: 6 of 2^-24 of each term's size
    tokens, heads, dim, rot = 40, 4, 64, 48
    cos, sin = tables(rot, 4096)
    pos = np.random.default_rng(0).integers(0, 4096, tokens).astype(np.int32)
    x, dy = (I.normal_f32((tokens, heads, dim), s, 53) for s in (1, 2))
    for inter in (False, True):
        y = check(tokens, heads, dim, rot, inter, False, False, False, pos, cos, sin, x=x).astype(np.float64)
        dx = check(tokens, heads, dim, rot, inter, False, False, True, pos, cos, sin, x=dy).astype(np.float64)
        a, b = (dy * y).sum(-1), (dx * x).sum(-1)
        assert (np.abs(a - b) <= 6 * 2.0 ** -24 * (np.linalg.norm(x, axis=-1) * np.linalg.norm(dy, axis=-1)) * 2).all()


def test_many_tokens():
    tokens, heads, dim = 70000, 4, 128
    cos, sin = tables(128, 512)
    pos = (np.arange(tokens) % 512).astype(np.int32)
    check(tokens, heads, dim, 128, False, False, True, False, pos, cos, sin)
