"""Refusals of products with a step per token, rotary positions, the paged cache and attention over it: checked on the host
before anything is enqueued, so no GPU is needed and no pointer below is followed."""
import ctypes

import pytest
import torch

import paper_2609_17380_amd.canon as C

BASE = 1 << 40
ORDER = ctypes.byref(C.ORDER_V1)


def p(k):
    """A device address of its own, 2^30 bytes from the next."""
    return BASE + (k << 30)


def raw(cls, *fields):
    r = cls.__new__(cls)
    ctypes.Structure.__init__(r, *fields)
    return r


# ---- products ----------------------------------------------------------------------------------------------------

def quant(rows=4, cols=100, dtype=C.F32, x=p(0), codes=p(1), steps=p(2)):
    return C.lib().canon_quant_tokens(rows, cols, dtype, x, codes, steps, None)


def test_quant_tokens():
    for bad in (dict(rows=-1), dict(cols=-1), dict(dtype=2), dict(x=None), dict(codes=None), dict(steps=None), dict(x=p(0) + 2),
                dict(steps=p(2) + 2), dict(dtype=C.BF16, x=p(0) + 1), dict(codes=p(0) + 1599), dict(steps=p(1) + 396),
                dict(steps=p(0))):
        assert quant(**bad) == C.EINVAL, bad
    assert quant(cols=65537) == C.EUNSUPPORTED and quant(rows=(1 << 31) + 1) == C.EUNSUPPORTED
    assert quant(rows=0, x=None, codes=None, steps=None) == C.OK


def gemm(m=8, n=16, k=32, a=p(0), lda=32, sa=p(1), b=p(2), ldb=32, sb=p(3), dtype=C.F32, y=p(4), ldc=16):
    return C.lib().canon_gemm_i8_tokens(m, n, k, a, lda, sa, b, ldb, sb, dtype, y, ldc, None)


def test_gemm_i8_tokens():
    for bad in (dict(m=-1), dict(n=-1), dict(k=-1), dict(lda=31), dict(ldb=31), dict(ldc=15), dict(dtype=3), dict(a=None),
                dict(b=None), dict(sa=None), dict(sb=None), dict(y=None), dict(y=p(4) + 2), dict(sa=p(1) + 1), dict(sb=p(3) + 2),
                dict(dtype=C.BF16, y=p(4) + 1), dict(y=p(0) + 252), dict(y=p(2)), dict(y=p(1) + 28), dict(sa=p(4)),
                dict(sb=p(4) + 500)):
        assert gemm(**bad) == C.EINVAL, bad
    assert gemm(k=65537, lda=65537, ldb=65537) == C.EUNSUPPORTED
    assert gemm(m=1 << 30, n=1 << 20, ldc=1 << 20) == C.EUNSUPPORTED
    assert gemm(m=1 << 25, n=1 << 10, ldc=1 << 10, y=p(64)) == C.EUNSUPPORTED
    assert gemm(m=0, a=None, y=None) == C.OK and gemm(n=0, b=None, y=None) == C.OK


# ---- rotary positions --------------------------------------------------------------------------------------------

def turn(rot=64, inter=0, positions=100, cos=p(20), sin=p(21)):
    return raw(C.Rotation, rot, inter, positions, cos, sin)


def rope(backward=0, tokens=4, heads=3, dim=64, positions=None, xd=C.F32, x=p(0), xs=192, yd=C.BF16, y=p(1), ys=192, rotation=True, **k):
    return C.lib().canon_rope(backward, tokens, heads, dim, ctypes.byref(turn(**k)) if rotation else None, positions, xd, x, xs, yd,
                              y, ys, None)


def test_rope():
    for bad in (dict(backward=2), dict(tokens=-1), dict(heads=-1), dict(dim=-1), dict(rotation=False), dict(xd=2), dict(yd=-1),
                dict(rot=63), dict(rot=66), dict(rot=-2), dict(inter=2), dict(positions=p(3) + 1), dict(cos=None), dict(sin=None),
                dict(cos=p(20) + 2), dict(x=None), dict(y=None), dict(x=p(0) + 2), dict(y=p(1) + 1), dict(xs=191), dict(ys=100),
                dict(y=p(0) + 400), dict(y=p(20)), dict(y=p(21) + 128), dict(x=p(1)),              # in place, but of another type
                dict(xd=C.BF16, x=p(1), xs=200), dict(positions=p(1) + 8)):
        assert rope(**bad) == C.EINVAL, bad
    assert rope(dim=1025, xs=9999, ys=9999) == C.EUNSUPPORTED
    assert rope(tokens=1 << 40) == C.EUNSUPPORTED
    assert rope(tokens=0, x=None, y=None) == C.OK and rope(heads=0, xs=0, ys=0, x=None, y=None) == C.OK


def tabs(rot=8, theta=1e4, scaling=None, first=0, n=4, cos=True, sin=True):
    out = [(ctypes.c_float * 64)() for _ in range(2)]
    return C.lib().canon_rope_tables(rot, theta, ctypes.byref(scaling) if scaling else None, first, n, out[0] if cos else None,
                                     out[1] if sin else None)


def test_rope_tables():
    S, inf, nan = C.RopeScaling, float("inf"), float("nan")
    assert tabs() == C.OK and tabs(n=0, cos=False, sin=False) == C.OK
    for bad in (dict(rot=0), dict(rot=7), dict(rot=1026), dict(theta=0.0), dict(theta=-1.0), dict(theta=inf), dict(theta=nan),
                dict(first=-1), dict(n=-1), dict(cos=False), dict(sin=False), dict(scaling=S(4)), dict(scaling=S(-1)),
                dict(scaling=S(1, 0.5)), dict(scaling=S(1, nan)), dict(scaling=S(2, inf)), dict(scaling=S(2, 2.0), rot=2),
                dict(scaling=S(3, 2.0, 4.0, 4.0, 100.0)), dict(scaling=S(3, 2.0, -1.0, 4.0, 100.0)),
                dict(scaling=S(3, 2.0, 1.0, 4.0, 0.0)), dict(scaling=S(0, amplitude=nan))):
        assert tabs(**bad) == C.EINVAL, bad
    assert tabs(first=1 << 31, n=1) == C.EUNSUPPORTED


# ---- the cache ---------------------------------------------------------------------------------------------------

CACHE = dict(n_pages=10, page=16, kv=2, dim=64, kc=p(8), vc=p(9), ks=p(10), vs=p(11), batch=3, table_len=4, table=p(12))


def cache(**k):
    c = CACHE | k
    return raw(C.KVCache, c["n_pages"], c["page"], c["kv"], c["dim"], c["kc"], c["vc"], c["ks"], c["vs"], c["batch"], c["table_len"],
               c["table"])


BAD_CACHES = [dict(n_pages=-1), dict(page=8), dict(page=48), dict(page=512), dict(page=0), dict(kv=0), dict(dim=0), dict(batch=-1),
              dict(table_len=-1), dict(kc=None), dict(vc=None), dict(ks=None), dict(vs=None), dict(kc=p(8) + 8), dict(vc=p(9) + 1),
              dict(ks=p(10) + 4), dict(vs=p(11) + 8), dict(table=None), dict(table=p(12) + 2)]
WIDE_CACHES = [dict(dim=48), dict(dim=288), dict(dim=16), dict(n_pages=1 << 31), dict(kv=65536), dict(batch=65536)]


def append(q_len=5, q_start=0, starts=None, lens=None, dtype=C.F32, k=p(0), k_row=128, v=p(1), v_row=128, rotation=None, none=False, **c):
    rows = raw(C.CacheRows, q_len, q_start, starts, lens)
    return C.lib().canon_cache_append(None if none else ctypes.byref(cache(**c)), ctypes.byref(rows), dtype, k, k_row, v, v_row,
                                      ctypes.byref(rotation) if rotation else None, None)


def read(q_len=5, q_start=0, starts=None, lens=None, dtype=C.F32, k=p(0), v=p(1), **c):
    rows = raw(C.CacheRows, q_len, q_start, starts, lens)
    return C.lib().canon_cache_read(ctypes.byref(cache(**c)), ctypes.byref(rows), dtype, k, v, None)


@pytest.mark.parametrize("call", [append, read])
def test_append_and_read(call):
    for bad in BAD_CACHES + [dict(q_len=-1), dict(starts=p(13) + 2), dict(lens=p(13) + 1), dict(dtype=2), dict(k=p(0) + 2),
                             dict(v=p(1) + 2), dict(dtype=C.BF16, k=p(0) + 1)]:
        assert call(**bad) == C.EINVAL, bad
    for wide in WIDE_CACHES + [dict(q_start=(1 << 30) + 1), dict(q_start=-(1 << 30) - 1), dict(q_len=(1 << 27) + 1)]:
        assert call(**wide) == C.EUNSUPPORTED, wide
    assert call(q_len=0, k=None, v=None) == C.OK and call(batch=0, k=None, v=None) == C.OK


def test_append_and_read_overlap():
    for bad in (dict(none=True), dict(k=None), dict(v=None), dict(k_row=127), dict(v_row=100), dict(k=p(8) + 4096), dict(v=p(9)),
                dict(k=p(11)), dict(kc=p(9)), dict(kc=p(1)), dict(table=p(10)), dict(starts=p(10)), dict(lens=p(11) + 8),
                dict(rotation=turn(rot=66)), dict(rotation=turn(rot=64, cos=p(8))), dict(rotation=turn(cos=None))):
        assert append(**bad) == C.EINVAL, bad
    for bad in (dict(k=p(8)), dict(v=p(11)), dict(v=p(0) + 400), dict(k=p(12)), dict(starts=p(0)), dict(lens=p(1))):
        assert read(**bad) == C.EINVAL, bad
    assert read(k=None, v=None) == C.OK


# ---- attention ---------------------------------------------------------------------------------------------------

ROWS = dict(batch=3, heads=4, q_len=5, k_len=60, ld=0, q_start=0, window=0, causal=1, scale=0.125, starts=None, q_lens=None, k_lens=None)


def attn(order=ORDER, dtype=C.F32, q=p(0), qs=256, out=p(1), ws=p(2), ws_bytes=1 << 28, none=False, **k):
    r = ROWS | {x: k.pop(x) for x in list(k) if x in ROWS and x != "batch"} | ({"batch": k["rows_batch"]} if "rows_batch" in k else {})
    k.pop("rows_batch", None)
    rows = raw(C.AttnRows, *(r[x] for x in ROWS))
    c = cache(**k)
    return C.lib().canon_cache_attention(order, None if none else ctypes.byref(c), ctypes.byref(rows), dtype, q, qs, out, ws, ws_bytes, None)


def test_attention():
    for bad in BAD_CACHES + [dict(order=None), dict(none=True), dict(rows_batch=2), dict(heads=0), dict(heads=3), dict(q_len=-1),
                             dict(k_len=-1), dict(k_len=65), dict(ld=60), dict(window=-1), dict(causal=2), dict(starts=p(13) + 2),
                             dict(q_lens=p(13) + 1), dict(k_lens=p(13) + 3), dict(dtype=5), dict(q=None), dict(q=p(0) + 2),
                             dict(qs=255), dict(out=None), dict(out=p(1) + 1), dict(out=p(0) + 100), dict(out=p(8)),
                             dict(out=p(11) + 64), dict(out=p(12)), dict(starts=p(1)), dict(n_pages=0)]:
        assert attn(**bad) == C.EINVAL, bad
    for wide in WIDE_CACHES + [dict(heads=1 << 24), dict(q_len=1 << 21), dict(q_start=(1 << 30) + 1),
                               dict(k_len=(1 << 21) + 1, table_len=1 << 20)]:
        assert attn(**wide) == C.EUNSUPPORTED, wide
    assert attn(order=ctypes.byref(C.Order(1, 31, 0, 1))) == C.EUNSUPPORTED
    assert attn(q_len=0, q=None, out=None) == C.OK and attn(rows_batch=0, batch=0, q=None, out=None) == C.OK


def test_attention_workspace():
    rows = raw(C.AttnRows, *(ROWS | dict(k_len=4000)).values())
    c = cache(table_len=300)
    need = C.lib().canon_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(rows))
    assert need == 4 * 3 * 5 * 4 * 16 * (64 + 4)  # rows, tiles of 256 keys, elements and what joins them
    k = dict(k_len=4000, table_len=300)
    assert attn(ws_bytes=need - 1, **k) == C.EWORKSPACE
    for bad in (dict(ws=None), dict(ws=p(2) + 128), dict(ws=p(0) - 256), dict(ws=p(8))):
        assert attn(**bad, **k) == C.EINVAL, bad
    assert C.lib().canon_cache_attention_workspace_bytes(ctypes.byref(cache(page=17)), ctypes.byref(rows)) == 0
    one = raw(C.AttnRows, *ROWS.values())
    assert C.lib().canon_cache_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(one)) == 0
    many = raw(C.AttnRows, *(ROWS | dict(k_len=4000, q_len=4000, heads=16)).values())
    assert C.lib().canon_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(many)) == 0


# ---- the binding -------------------------------------------------------------------------------------------------

def test_binding(monkeypatch):
    """On tensors of the host, taken for the current device's: what is wrong is told before the library is called."""
    monkeypatch.setattr(C, "_device", lambda: -1)
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)  # noqa: E731
    parts = dict(k_codes=z(4, 2, 16, 64, t=torch.int8), v_codes=z(4, 2, 1, 64, 16, t=torch.int8), k_steps=z(4, 2, 16),
                 v_steps=z(4, 2, 16), table=z(2, 3, t=torch.int32))
    make = lambda **k: C.KVCache(16, 2, 64, **(parts | k))  # noqa: E731
    c = make()
    for bad in (dict(k_codes=z(4, 2, 16, 63, t=torch.int8)), dict(v_codes=z(4, 2, 1, 64, 15, t=torch.int8)), dict(k_steps=z(4, 2, 15)),
                dict(v_steps=z(4, 2, 16, t=torch.bfloat16)), dict(table=z(6, t=torch.int32)), dict(table=z(2, 3, t=torch.int64)),
                dict(k_codes=None), dict(v_codes=None), dict(k_steps=None), dict(table=None),
                dict(table=z(3, 2, t=torch.int32).T)):
        with pytest.raises(ValueError):
            make(**bad)
    with pytest.raises(ValueError, match="sequences"):
        C.cache_append(c, C.CacheRows(3, 1), z(2, 128), z(2, 128))
    for k, v in ((z(2, 127), z(2, 128)), (z(2, 128), z(2, 128, t=torch.bfloat16)), (z(2, 128, t=torch.float64), z(2, 128)),
                 (None, z(2, 128)), (z(128, 2).T, z(2, 128))):
        with pytest.raises(ValueError):
            C.cache_append(c, C.CacheRows(2, 1), k, v)
    with pytest.raises(ValueError):
        C.cache_read(c, C.CacheRows(2, 1))
    with pytest.raises(ValueError):
        C.cache_read(c, C.CacheRows(2, 1), z(2, 128), z(2, 128, t=torch.bfloat16))
    with pytest.raises(ValueError):
        C.Rotation(z(5, 4), z(5, 3), 8)
    with pytest.raises(ValueError):
        C.rope(2, 2, 64, C.Rotation(z(5, 32), z(5, 32), 64), z(2, 128), z(2, 128), positions=z(2))
    for ld in (31, 0):
        with pytest.raises(ValueError):
            C.gemm_i8_tokens(4, 8, 32, z(4, 32, t=torch.int8), ld, z(4), z(8, 32, t=torch.int8), 32, z(8), z(4, 8))
    with pytest.raises(ValueError):
        C.quant_tokens(2, 8, z(2, 8, t=torch.int32), z(2, 8, t=torch.int8), z(2))
    monkeypatch.setattr(C, "_device", lambda: 0)  # another device than the tensors'
    for call in (lambda: C.cache_append(c, C.CacheRows(2, 1), z(2, 128), z(2, 128)),
                 lambda: C.quant_tokens(2, 8, z(2, 8), z(2, 8, t=torch.int8), z(2))):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(C.CanonError):
        C.rope_tables(7, 4)
