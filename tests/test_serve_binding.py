"""The binding's records of a cache and of a rotation: their tensors are looked at again by every call, as they may have been resized
or given other memory since.  On tensors of the host, taken for the current device's: nothing reaches the library."""
import pytest
import torch

import paper_2609_17380_amd.canon as C


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(C, "_device", lambda: -1)

    class Library:
        def __getattr__(self, name):
            def call(*_):
                raise AssertionError(f"{name} was called")
            return call

    monkeypatch.setattr(C, "_lib", Library)


def z(*s, t=torch.float32):
    return torch.zeros(*s, dtype=t)


def parts():
    return dict(k_codes=z(4, 2, 16, 64, t=torch.int8), v_codes=z(4, 2, 1, 64, 16, t=torch.int8), k_steps=z(4, 2, 16),
                v_steps=z(4, 2, 16), table=z(2, 3, t=torch.int32))


def calls(c):
    rows = C.CacheRows(2, 1)
    return (lambda: C.cache_append(c, rows, z(2, 128), z(2, 128)), lambda: C.cache_read(c, rows, z(2, 128)),
            lambda: C.cache_attention(c, C.AttnRows(2, 2, 1, 1), z(2, 128), z(2, 128, t=torch.bfloat16)))


@pytest.mark.parametrize("name", ["k_codes", "v_codes", "k_steps", "v_steps", "table"])
def test_a_cache_whose_tensors_changed(host, name):
    def shorter(t):
        t.resize_(1)

    def longer(t):
        t.resize_(t.numel() * 2)

    def turned(t):
        t.transpose_(0, -1)

    def freed(t):
        t.set_(torch.zeros(0, dtype=t.dtype))

    def type_of(t):
        t.data = t.data.to(torch.float64)

    for change in (shorter, longer, turned, freed, type_of):
        p = parts()
        c = C.KVCache(16, 2, 64, *p.values())
        change(p[name])
        for call in calls(c):
            with pytest.raises(ValueError, match=name):
                call()


@pytest.mark.parametrize("which", [0, 1])
def test_a_rotation_whose_tables_changed(host, which):
    for change in (lambda t: t.resize_(3), lambda t: t.resize_(1000), lambda t: t.t_(), lambda t: t.set_(torch.zeros(0))):
        tables = z(5, 32), z(5, 32)
        turn = C.Rotation(*tables, 64)
        change(tables[which])
        for call in (lambda: C.rope(2, 2, 64, turn, z(2, 128), z(2, 128)),
                     lambda: C.cache_append(C.KVCache(16, 2, 64, *parts().values()), C.CacheRows(2, 1), z(2, 128), z(2, 128),
                                            rotation=turn)):
            with pytest.raises(ValueError, match="cos" if which == 0 else "sin"):
                call()


def test_other_memory_of_the_same_kind(host):
    p, tables = parts(), (z(5, 32), z(5, 32))
    c, turn = C.KVCache(16, 2, 64, *p.values()), C.Rotation(*tables, 64)
    for t in (*p.values(), *tables):
        t.set_(torch.ones_like(t))
    c._of(-1), turn._of(-1)
    assert [c.k_codes, c.v_codes, c.k_steps, c.v_steps, c.table] == [t.data_ptr() for t in p.values()]
    assert [turn.cos, turn.sin] == [t.data_ptr() for t in tables]
    assert c._of(-1) and c.kept and c.k_steps == p["k_steps"].data_ptr()
    with pytest.raises(ValueError, match="device"):
        c._of(0)
    with pytest.raises(ValueError, match="device"):
        turn._of(0)


def test_a_refusal_leaves_nothing_half_taken(host):
    p = parts()
    c = C.KVCache(16, 2, 64, *p.values())
    first = p["k_codes"].data  # the memory that it had
    p["k_codes"].set_(torch.ones_like(first))
    steps = p["k_steps"].data
    p["k_steps"].set_(torch.ones(3))
    with pytest.raises(ValueError, match="k_steps"):
        c._of(-1)
    p["k_codes"].set_(first)
    p["k_steps"].set_(steps)
    c._of(-1)
    assert c.k_codes == first.data_ptr() and c.k_steps == steps.data_ptr()
    p["v_steps"].resize_(1)
    longer = z(7, 9, t=torch.int32)
    c.set_table(longer)
    for _ in range(2):
        with pytest.raises(ValueError, match="v_steps"):
            c._of(-1)
    longer = z(7, 9, t=torch.int32)
    c.set_table(longer)
    p["v_steps"].resize_(4, 2, 16)
    c._of(-1)
    assert (c.batch, c.table_len, c.table) == (7, 9, longer.data_ptr())
    with pytest.raises(ValueError, match="table"):
        c.set_table(z(3, 2, t=torch.int64))
    c._of(-1)
    assert (c.batch, c.table_len, c.table) == (7, 9, longer.data_ptr())
