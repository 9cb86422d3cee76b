"""Refusals of layer norm, activations kept in 8 bits, SwiGLU and attention rows with a relative position bias: checked on
the host before anything is enqueued, so no GPU is needed and no pointer below is followed."""
import ctypes

import pytest
import torch

import paper_2609_17380_amd.canon as C

BASE = 1 << 32
ORDER = ctypes.byref(C.ORDER_V1)


def p(k):
    """A device address of its own, 2^28 bytes from the next."""
    return BASE + (k << 28)


def act8(group=64, codes=p(20), steps=p(21)):
    r = C.Act8.__new__(C.Act8)
    ctypes.Structure.__init__(r, group, codes, steps)
    return r


def pack(rows=4, cols=100, dtype=C.F32, x=p(0), kept=None, **k):
    kept = kept if kept is not None else act8(**k)
    return C.lib().canon_act8_pack(rows, cols, dtype, x, ctypes.byref(kept), None)


def unpack(rows=4, cols=100, dtype=C.F32, out=p(0), **k):
    return C.lib().canon_act8_unpack(rows, cols, ctypes.byref(act8(**k)), dtype, out, None)


@pytest.mark.parametrize("call", [pack, unpack])
def test_act8(call):
    for bad in (dict(rows=-1), dict(cols=-1), dict(dtype=2), dict(dtype=-1), dict(group=0), dict(group=16), dict(group=96),
                dict(group=512), dict(group=-32), dict(codes=None), dict(steps=None), dict(steps=p(21) + 2)):
        assert call(**bad) == C.EINVAL, bad
    assert call(rows=1 << 21, cols=(1 << 20)) == C.EUNSUPPORTED
    assert call(rows=1 << 62, cols=1 << 62) == C.EUNSUPPORTED
    assert call(rows=0) == C.OK and call(cols=0) == C.OK


def test_act8_overlap_and_alignment():
    n = 4 * 100
    assert pack(x=None) == C.EINVAL and unpack(out=None) == C.EINVAL
    assert pack(x=p(0) + 2) == C.EINVAL and pack(dtype=C.BF16, x=p(0) + 1) == C.EINVAL
    assert pack(codes=p(0) + 4 * n - 1) == C.EINVAL          # the last byte of x
    assert pack(steps=p(0)) == C.EINVAL and pack(codes=p(21)) == C.EINVAL
    assert unpack(out=p(20)) == C.EINVAL and unpack(out=p(21) - 4 * n + 4) == C.EINVAL
    lib = C.lib()
    assert lib.canon_act8_pack(4, 100, C.F32, p(0), None, None) == C.EINVAL
    assert lib.canon_act8_unpack(4, 100, None, C.F32, p(0), None) == C.EINVAL
    assert C.act8_groups(0, 32) == 0 and C.act8_groups(1, 32) == 1 and C.act8_groups(33, 32) == 2
    assert C.act8_groups(-1, 32) == 0 and C.act8_groups(64, 48) == 0


def test_swiglu():
    lib = C.lib()

    def fwd(T=4, F=100, dtype=C.F32, gu=p(0), a=p(1), kept=None):
        return lib.canon_swiglu(T, F, dtype, gu, a, ctypes.byref(kept) if kept else None, None)

    def bwd(T=4, F=100, dtype=C.F32, gu=p(0), kept=None, da=p(1), dgu=p(2), a=p(3)):
        return lib.canon_swiglu_bwd(T, F, dtype, gu, ctypes.byref(kept) if kept else None, da, dgu, a, None)

    for bad in (dict(T=-1), dict(F=-1), dict(dtype=2), dict(gu=None), dict(gu=p(0) + 2), dict(a=None), dict(a=p(1) + 1),
                dict(a=p(0) + 3199), dict(kept=act8(group=5)), dict(kept=act8(codes=None)), dict(kept=act8(codes=p(1) + 10)),
                dict(kept=act8(steps=p(20)))):
        assert fwd(**bad) == C.EINVAL, bad
    assert fwd(T=1 << 30, F=1 << 30) == C.EUNSUPPORTED and bwd(T=1 << 30, F=1 << 30) == C.EUNSUPPORTED
    assert fwd(T=0) == C.OK and bwd(F=0) == C.OK
    for bad in (dict(T=-1), dict(F=-1), dict(dtype=7), dict(gu=None), dict(kept=act8()), dict(da=None), dict(da=p(1) + 2),
                dict(dgu=None), dict(dgu=p(2) + 1), dict(a=p(3) + 1), dict(dgu=p(1) + 1598), dict(a=p(2)), dict(a=p(0)),
                dict(gu=None, kept=act8(group=0)), dict(gu=None, kept=act8(), dgu=p(20)), dict(gu=None, kept=act8(), a=p(21))):
        assert bwd(**bad) == C.EINVAL, bad


def test_layernorm():
    lib = C.lib()

    def fwd(order=ORDER, rows=4, cols=100, xt=C.F32, x=p(0), gain=p(1), bias=p(2), yt=C.BF16, y=p(3), mean=p(4), rstd=p(5),
            kept=None):
        return lib.canon_layernorm(order, rows, cols, xt, x, gain, bias, 1e-5, yt, y, mean, rstd,
                                   ctypes.byref(kept) if kept else None, None)

    assert fwd(order=None) == C.EINVAL and fwd(order=ctypes.byref(C.Order(1, 31, 0, 1))) == C.EUNSUPPORTED
    for bad in (dict(rows=-1), dict(cols=0), dict(xt=2), dict(yt=2), dict(x=None), dict(gain=None), dict(y=None), dict(mean=None),
                dict(rstd=None), dict(x=p(0) + 1), dict(gain=p(1) + 1), dict(bias=p(2) + 1), dict(y=p(3) + 1),
                dict(yt=C.F32, y=p(3) + 2), dict(mean=p(4) + 2), dict(rstd=p(5) + 1), dict(y=p(0)), dict(y=p(0) + 1598),
                dict(mean=p(3)), dict(rstd=p(4) + 12), dict(mean=p(2)), dict(kept=act8(group=33)), dict(kept=act8(codes=p(0))),
                dict(kept=act8(steps=p(5)))):
        assert fwd(**bad) == C.EINVAL, bad
    assert fwd(cols=32769) == C.EUNSUPPORTED and fwd(rows=(1 << 26) + 1) == C.EUNSUPPORTED
    assert fwd(rows=0) == C.OK

    size = C.layernorm_bwd_workspace_bytes(4, 100)
    assert size >= 2 * 100 * 4
    for rows, cols in ((-1, 4), (4, 0), (4, 32769), ((1 << 26) + 1, 4)):
        assert C.layernorm_bwd_workspace_bytes(rows, cols) == 0

    def bwd(order=ORDER, rows=4, cols=100, xt=C.F32, x=p(0), kept=None, gain=p(1), mean=p(2), rstd=p(3), dy=p(4), dx=p(5),
            dg=p(6), db=p(7), ws=p(8), n=size):
        return lib.canon_layernorm_bwd(order, rows, cols, xt, x, ctypes.byref(kept) if kept else None, gain, mean, rstd, dy, dx,
                                       dg, db, ws, n, None)

    assert bwd(order=None) == C.EINVAL
    for bad in (dict(rows=-1), dict(cols=0), dict(xt=2), dict(x=None), dict(kept=act8()), dict(x=None, kept=act8(group=1)),
                dict(gain=None), dict(mean=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(dx=p(5) + 2),
                dict(dg=p(6) + 1), dict(db=p(7) + 2), dict(ws=None), dict(ws=p(8) + 128), dict(dx=p(0)), dict(dx=p(4) + 4),
                dict(dg=p(5)), dict(db=p(6) + 396), dict(dg=p(1)), dict(ws=p(5)), dict(x=None, kept=act8(codes=p(5)))):
        assert bwd(**bad) == C.EINVAL, bad
    assert bwd(n=size - 1) == C.EWORKSPACE and bwd(cols=32769) == C.EUNSUPPORTED


def rows(batch=2, heads=3, q=10, k=10, ld=0, q_start=0, window=0, causal=1, q_starts=None, q_lens=None, k_lens=None):
    r = C.AttnRows(batch, heads, q, k, ld=ld, q_start=q_start, window=window)
    r.causal, r.q_starts, r.q_lens, r.k_lens = causal, q_starts, q_lens, k_lens
    return r


def test_relbias():
    lib = C.lib()

    def fwd(order=ORDER, bias=C.RelBias([0, 1, 4]), table=p(0), x=p(1), y=p(2), **k):
        return lib.canon_softmax_relbias(order, ctypes.byref(rows(**k)), ctypes.byref(bias), table, x, y, None)

    def bwd(order=ORDER, bias=C.RelBias([0, 1, 4]), pr=p(1), dp=p(2), ds=p(3), dt=p(4), ws=p(5), n=1 << 20, **k):
        return lib.canon_softmax_relbias_bwd(order, ctypes.byref(rows(**k)), ctypes.byref(bias), pr, dp, ds, dt, ws, n, None)

    def starts(*s, n=None, bidirectional=0):
        r = C.RelBias(s)
        r.n_starts, r.bidirectional = len(s) if n is None else n, bidirectional
        return r

    for call in (fwd, bwd):
        assert call(order=None) == C.EINVAL and call(order=ctypes.byref(C.Order(2, 32, 0, 1))) == C.EUNSUPPORTED
        for bad in (dict(batch=-1), dict(heads=-1), dict(q=-1), dict(k=-1), dict(ld=9), dict(ld=-1), dict(window=-1),
                    dict(causal=2), dict(q_start=(1 << 30) + 1), dict(q_start=-(1 << 30) - 1), dict(q_starts=p(9) + 2),
                    dict(q_lens=p(9) + 1), dict(k_lens=p(9) + 3), dict(bias=starts()), dict(bias=starts(1, 2)),
                    dict(bias=starts(0, 2, 1)), dict(bias=starts(0, -1)), dict(bias=starts(0, n=129)),
                    dict(bias=starts(0, n=-1)), dict(bias=starts(0, 1, bidirectional=2))):
            assert call(**bad) == C.EINVAL, bad
        for bad in (dict(k=32769), dict(ld=(1 << 31) + 1), dict(batch=1 << 16, heads=1 << 10, q=1 << 6),
                    dict(batch=1 << 40, heads=1 << 40, q=1 << 40),
                    dict(q=1 << 20, ld=1 << 31), dict(bias=starts(0, 1025))):
            assert call(**bad) == C.EUNSUPPORTED, bad
    for bad in (dict(table=None), dict(x=None), dict(y=None), dict(table=p(0) + 1), dict(x=p(1) + 2), dict(y=p(2) + 1),
                dict(y=p(1) + 2398), dict(y=p(0)), dict(k_lens=p(2) + 4), dict(q_starts=p(2))):
        assert fwd(**bad) == C.EINVAL, bad
    for bad in (dict(pr=None), dict(dp=None), dict(ds=None), dict(pr=p(1) + 1), dict(dp=p(2) + 2), dict(ds=p(3) + 1),
                dict(dt=p(4) + 2), dict(ws=None), dict(ws=p(5) + 64), dict(ds=p(1)), dict(ds=p(2) + 2398), dict(dt=p(3)),
                dict(ws=p(3) - 256), dict(q_lens=p(3))):
        assert bwd(**bad) == C.EINVAL, bad
    need = C.softmax_relbias_bwd_workspace_bytes(rows(), C.RelBias([0, 1, 4]))
    assert need > 0 and bwd(n=need - 1) == C.EWORKSPACE
    assert C.softmax_relbias_bwd_workspace_bytes(rows(q=-1), C.RelBias([0])) == 0
    assert fwd(batch=0) == C.OK and fwd(k=0) == C.OK and fwd(q=0, table=None, x=None, y=None) == C.OK


def test_relbias_log():
    for bad in ((0, 0, 8), (1, 0, 8), (3, 1, 8), (2, 1, 8), (8, 2, 64), (8, 0, 4), (8, 0, -1)):
        assert C.lib().canon_relbias_log(*bad, ctypes.byref(C.RelBias())) == C.EINVAL, bad
    assert C.lib().canon_relbias_log(130, 0, 500, ctypes.byref(C.RelBias())) == C.EUNSUPPORTED
    assert C.lib().canon_relbias_log(8, 0, 1025, ctypes.byref(C.RelBias())) == C.EUNSUPPORTED
    assert C.lib().canon_relbias_log(8, 0, 64, None) == C.EINVAL
    with pytest.raises(C.CanonError):
        C.relbias_log(8, 4)
    with pytest.raises(ValueError):
        C.RelBias(range(129))


def test_the_binding_refuses_other_tensors():
    # of a type, a place or a size that the call does not take (here: not on a GPU)
    f, h, q = torch.zeros(400), torch.zeros(400, dtype=torch.bfloat16), torch.zeros(400, dtype=torch.int8)
    kept = C.Act8(64, q, torch.zeros(8))
    for call in (lambda: C.act8_pack(4, 100, f, kept), lambda: C.act8_unpack(4, 100, kept, f.double()),
                 lambda: C.layernorm(4, 100, f.half(), h, None, 1e-5, f, f, f),
                 lambda: C.layernorm_bwd(4, 100, kept, h, f, f, f, f),
                 lambda: C.swiglu(4, 50, f, h), lambda: C.swiglu_bwd(4, 50, kept, f, h),
                 lambda: C.act8_pack(4, 100, None, kept), lambda: C.layernorm(4, 100, None, h, None, 1e-5, f, f, f),
                 lambda: C.AttnRows(4, 1, 1, 1, k_lens=torch.zeros(4, dtype=torch.int32)),
                 lambda: C.AttnRows(4, 1, 1, 1, k_lens=[1, 2, 3, 4]),
                 lambda: C.softmax_relbias(C.AttnRows(1, 1, 20, 20), C.RelBias([0]), h, f, h)):
        with pytest.raises(ValueError):
            call()


def test_relbias_table_is_bounded():
    # the sums of the rows have a column to a head's bucket, and one launch folds at most 2^24 of them
    lib, bias = C.lib(), C.RelBias(range(128), bidirectional=True)
    for heads, refused in ((1 << 16, False), ((1 << 16) + 1, True), (1 << 26, True)):
        r = rows(batch=1, heads=heads, q=1, k=1)
        st = lib.canon_softmax_relbias(ORDER, ctypes.byref(r), ctypes.byref(bias), None, p(1), p(2), None)
        assert st == (C.EUNSUPPORTED if refused else C.EINVAL), heads  # EINVAL: no table
        assert (C.softmax_relbias_bwd_workspace_bytes(r, bias) == 0) == refused


def test_a_record_is_checked_where_it_is_used(monkeypatch):
    lens = torch.tensor([1, 2], dtype=torch.int32)
    with monkeypatch.context() as m:
        m.setattr(C, "_device", lambda: -1)  # where the record's tensors are
        r = C.AttnRows(2, 1, 1, 4, k_lens=lens)
        other = C.AttnRows(2, 1, 1, 4, k_lens=lens)
        other.batch = 3  # more sequences than lengths
        t, x, y = torch.zeros(1, dtype=torch.bfloat16), torch.zeros(12), torch.zeros(12, dtype=torch.bfloat16)
        with pytest.raises(ValueError, match="k_lens"):
            C.softmax_relbias(other, C.RelBias([0]), t, x, y)
        with pytest.raises(ValueError, match="k_lens"):
            C.softmax_relbias_bwd(other, C.RelBias([0]), y, x, y)
    with pytest.raises(ValueError, match="k_lens"):  # the current device is another
        C.softmax_relbias(r, C.RelBias([0]), t, x[:8], y[:8])
    with pytest.raises(ValueError, match="k_lens"):
        C.softmax_relbias_bwd(r, C.RelBias([0]), y[:8], x[:8], y[:8])


def test_records_follow_their_tensors(monkeypatch):
    monkeypatch.setattr(C, "_device", lambda: -1)
    codes, steps, lens = torch.zeros(64, dtype=torch.int8), torch.zeros(1), torch.zeros(2, dtype=torch.int32)
    kept, r = C.Act8(64, codes, steps), C.AttnRows(2, 1, 1, 4, k_lens=lens)
    codes.set_(torch.zeros(128, dtype=torch.int8)[64:])  # other memory under the same tensors
    lens.set_(torch.zeros(4, dtype=torch.int32)[2:])
    kept._of(1, 64, -1)
    r._of(-1)
    assert kept.codes == codes.data_ptr() and r.k_lens == lens.data_ptr()


def test_the_binding_refuses_what_is_no_tensor():
    f, h = torch.zeros(400), torch.zeros(400, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        C.layernorm_bwd(4, 100, f, h, f, f, f, f, workspace=1 << 20)
    with pytest.raises(ValueError, match="workspace"):
        C._scratch(1 << 20, 0)
    with pytest.raises(ValueError):
        C.act8_pack(4, 100, f, C.Act8(64, None, None))
