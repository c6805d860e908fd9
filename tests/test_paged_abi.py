"""What the entry points of the paged K/V cache refuse: on the host, with nothing enqueued (no GPU needed)."""
import pytest
import torch

from paper_2601_21896_amd import binding as B

A = 0x10000  # a fake, 16-byte aligned "device address": validation must fail before it is ever used
MB = 0x100000


def _call(f, ok, **kw):
    a = dict(ok)
    a.update(kw)
    return f(None, *a.values())


def test_tables_refuse_bad_arguments():
    ok = dict(kv=A, new=A + MB, B=4, free=A + 2 * MB, nf=100, fs=A + 3 * MB, ps=16, table=A + 4 * MB, mp=8, ld=8,
              slots=A + 5 * MB, ms=64, rs=A + 6 * MB, out=A + 7 * MB, fe=A + 8 * MB)
    call = lambda **kw: _call(B.library().pafu_paged_tables, ok, **kw)  # noqa: E731
    for name in ("kv", "new", "free", "table", "slots", "rs", "out", "fe"):
        assert call(**{name: None}) == -1, name
    for name in ("kv", "new", "free", "table", "slots", "rs", "out"):
        assert call(**{name: ok[name] + 4}) == -4, name
    assert call(fe=ok["fe"] + 2) == -4
    for kw in (dict(B=-1), dict(B=8193), dict(nf=-1), dict(ps=0), dict(ps=4), dict(ps=24), dict(ps=8192), dict(ps=-16),
               dict(mp=0), dict(ld=7), dict(ms=-1), dict(ms=2 ** 30 + 1)):
        assert call(**kw) == -2, kw
    # in place is not allowed, nor are outputs over inputs or over each other
    for kw in (dict(out=A), dict(rs=A + MB), dict(fe=A + 3 * MB), dict(slots=A + 4 * MB), dict(table=A + 2 * MB),
               dict(out=A + 6 * MB + 16)):
        assert call(**kw) == -6, kw
    assert call(B=0, kv=None) == 0


def test_slots_refuse_bad_arguments():
    ok = dict(table=A, mp=8, ld=8, start=A + MB, count=A + 2 * MB, B=4, ps=16, slots=A + 3 * MB, ms=64, rs=A + 4 * MB)
    call = lambda **kw: _call(B.library().pafu_paged_slots, ok, **kw)  # noqa: E731
    for name in ("table", "start", "count", "slots", "rs"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ok[name] + 8}) == -4, name
    for kw in (dict(B=-1), dict(B=8193), dict(ps=12), dict(mp=0), dict(ld=7), dict(ms=-1), dict(ms=2 ** 30 + 1)):
        assert call(**kw) == -2, kw
    for kw in (dict(slots=A), dict(rs=A + 2 * MB), dict(rs=A + 3 * MB)):
        assert call(**kw) == -6, kw
    assert call(B=0, table=None) == 0


POOL = dict(Kp=A + 0x10000000, Vp=A + 0x20000000, np=10, ps=16, ldp=16 * 256, ldt=256, ldh=128)
BAD_POOLS = (dict(np=0), dict(ps=7), dict(ps=0), dict(ps=24), dict(ps=8192), dict(ldh=64), dict(ldt=64), dict(ldt=128),
             dict(ldp=16 * 256 - 8), dict(ldt=1 << 41), dict(ldp=1 << 41),
             dict(ldh=128 * 8, ldt=128, ldp=2 * 16 * 128),   # heads closer than a head's 16 tokens
             dict(np=2 ** 31 - 1, ldp=1 << 40))


def test_append_refuses_bad_arguments():
    ok = dict(K=A, V=A + MB, ld=256, rows=20, slots=A + 2 * MB, N=2, D=128, **POOL, dt=0, ks=0, vs=0)
    call = lambda **kw: _call(B.library().pafu_paged_append, ok, **kw)  # noqa: E731
    for name in ("K", "V", "slots", "Kp", "Vp"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ok[name] + 8}) == -4, name
    for kw in (dict(rows=-1), dict(N=0), dict(D=96), dict(ld=255), dict(ks=65), dict(vs=-65)) + BAD_POOLS:
        assert call(**kw) == -2, kw
    for kw in (dict(dt=1), dict(dt=3)):
        assert call(**kw) == -3, kw
    for kw in (dict(ld=260), dict(ldp=16 * 256 + 4), dict(ldt=260, ldp=16 * 260), dict(dt=2, ldp=16 * 256 + 8)):
        assert call(**kw) == -4, kw
    assert call(Vp=ok["Kp"]) == -6                                   # K and V pages at one place
    assert call(Vp=ok["Kp"] + 128 * 2) == -6                         # half a token apart
    assert call(K=ok["Kp"] + 512) == -6
    assert call(slots=ok["Vp"]) == -6
    assert call(rows=0, K=None, slots=None) == 0


def test_attention_refuses_bad_arguments():
    ok = dict(Q=A, ldq=1024, **POOL, dt=0, ks=0, vs=0, table=A + MB, mp=8, ld=8, kv=A + 2 * MB, B=4, N=8, Nkv=2, D=128,
              pin=0, win=0, sc=0.0, O=A + 3 * MB, ldo=1024, od=0, ws=None, wsb=0)
    call = lambda **kw: _call(B.library().pafu_paged_attention, ok, **kw)  # noqa: E731
    for name in ("Q", "Kp", "Vp", "table", "kv", "O"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ok[name] + 8}) == -4, name
    for kw in (dict(B=-1), dict(B=8193), dict(N=0), dict(N=7), dict(Nkv=0), dict(D=96), dict(pin=-1), dict(win=-1),
               dict(ldq=1023), dict(ldo=1000), dict(ks=65), dict(mp=0), dict(ld=7)) + BAD_POOLS:
        assert call(**kw) == -2, kw
    assert call(dt=1) == -3 and call(od=2) == -3
    assert call(B=4096, N=4096, ldq=4096 * 128, ldo=4096 * 128) == -2  # a launch's threads are counted in 32 bits
    # and so are the tiles of all requests
    assert call(B=8192, mp=1 << 20, ld=1 << 20, ps=4096, ldp=4096 * 256) == -2
    for kw in (dict(ldq=1028), dict(ldo=1028), dict(ws=A + 4 * MB + 8, wsb=1024)):
        assert call(**kw) == -4, kw
    for kw in (dict(O=A), dict(O=ok["Kp"] + 4096), dict(O=A + MB), dict(ws=A, wsb=64), dict(ws=ok["Vp"], wsb=64),
               dict(ws=A + 3 * MB, wsb=64), dict(ws=A + 2 * MB, wsb=64)):
        assert call(**kw) == -6, kw
    assert call(B=0, Q=None) == 0
    size = B.pafu_paged_attention_workspace_bytes
    assert size(4, 7, 2, 128) == size(0, 8, 2, 128) == size(4, 8, 0, 128) == size(4, 8, 2, 96) == 0


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    i, more = torch.zeros(4, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    pages = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    rows = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        B.pafu_paged_tables(i, i, i, 16, i.view(4, 1), i, more, i, i[:1])
    with pytest.raises(ValueError, match="GPU"):
        B.pafu_paged_slots(i.view(4, 1), i, i, 16, i, more)
    with pytest.raises(ValueError, match="GPU"):
        B.pafu_paged_append(rows, rows, i, pages, pages)
    with pytest.raises(ValueError, match="GPU"):
        B.pafu_paged_attention(rows, pages, pages, i.view(4, 1), i, rows)


def test_binding_refuses_types_and_shapes_that_the_library_cannot_see():
    i = torch.zeros(6, dtype=torch.int32)
    pages = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    rows = torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    table = i.view(6, 1)
    bad_lists = ((i.long(), TypeError), (i[::2], ValueError), (i.view(2, 3), ValueError), (i[:3], ValueError), (None, TypeError),
                 ([0] * 6, TypeError))
    for bad, error in bad_lists:
        with pytest.raises(error):
            B.pafu_paged_tables(i, bad, i, 16, table, i, torch.zeros(7, dtype=torch.int32), i, i[:1])
        with pytest.raises(error):
            B.pafu_paged_slots(table, i, bad, 16, i, torch.zeros(7, dtype=torch.int32))
        with pytest.raises(error):
            B.pafu_paged_append(rows, rows, bad, pages, pages)
        with pytest.raises(error):
            B.pafu_paged_attention(rows, pages, pages, table, bad, rows)
    for bad in (i, i[:5]):                                           # row_start holds one more than there are requests
        with pytest.raises(ValueError, match="row_start"):
            B.pafu_paged_slots(table, i, i, 16, i, bad)
    for bad, error in ((table.long(), TypeError), (i, ValueError), (i.view(3, 2), ValueError),
                       (torch.zeros(2, 6, dtype=torch.int32).t(), ValueError)):
        with pytest.raises(error, match="block table"):
            B.pafu_paged_attention(rows, pages, pages, bad, i, rows)
    for K, V, error in ((pages, pages[:1], ValueError), (pages[0], pages[0], ValueError), (pages, pages.half(), TypeError),
                        (pages.float(), pages.float(), TypeError), (pages.transpose(2, 3), pages.transpose(2, 3), ValueError),
                        (pages, pages.transpose(0, 1).contiguous().transpose(0, 1), ValueError)):
        with pytest.raises(error, match="page tensors"):
            B.pafu_paged_attention(rows, K, V, table, i, rows)
        with pytest.raises(error, match="page tensors"):
            B.pafu_paged_append(rows, rows, i, K, V)
    wide = torch.zeros(6, 4, 128, dtype=torch.bfloat16)
    for bad, error in ((rows.half(), TypeError), (rows[0], ValueError), (wide[:, ::2, :64], ValueError), (wide[:, :2, ::2], ValueError),
                       (rows[:, :, :32], ValueError)):
        with pytest.raises(error):
            B.pafu_paged_attention(bad, pages, pages, table, i, rows)
        with pytest.raises(error):
            B.pafu_paged_append(bad, rows, i, pages, pages)
    with pytest.raises(ValueError, match="one stride"):
        B.pafu_paged_append(rows, wide.view(6, 8, 64)[:, :2], i, pages, pages)
    with pytest.raises(ValueError, match="Q and O"):
        B.pafu_paged_attention(rows, pages, pages, table, i, rows[:, :1])
    with pytest.raises(ValueError, match="workspace"):
        B.pafu_paged_attention(rows, pages, pages, table, i, rows, workspace=torch.zeros(8, dtype=torch.uint8)[::2])
    with pytest.raises(OverflowError):
        B.pafu_paged_attention(rows, pages, pages, table, i, rows, window=2 ** 31)
    for bad in ("16", 1.5):
        with pytest.raises(TypeError):
            B.pafu_paged_slots(table, i, i, bad, i, torch.zeros(7, dtype=torch.int32))


def test_the_module_takes_the_entry_points_of_the_loaded_library():
    call = B._paged()
    assert B._paged() is call
    assert call.torch_version == torch.__version__.split("+")[0]
    with pytest.raises(TypeError):
        call.attention(1, 2)
    with pytest.raises(TypeError):
        call.bind(1)
