"""What the entry points of the paged cache refuse, and what they ask for; nothing is launched."""
import ctypes

import pytest

import paper_2503_01873_amd as P

A = 1 << 20                       # addresses that are never followed
OK = dict(k=A, v=2 * A, kscale=3 * A, vscale=4 * A, table=5 * A, length=6 * A, S=2, Hkv=2, d=64, page=64, pages=8, table_width=4,
          format=P.CACHE_I8, kmean=7 * A, kshift=8 * A)


def cache(**kw):
    return P.pasa_cache(**{**OK, **kw})


def write(c, **kw):
    a = dict(k=9 * A, v=10 * A, R=2, row_stride=128, row_start=11 * A, io_dtype=P.IO_F16, check=False)
    return P.pasa_cache_write(c, **{**a, **kw})


def read(c, **kw):
    a = dict(k=9 * A, v=10 * A, first=11 * A, N=5, io_dtype=P.IO_F16, check=False)
    return P.pasa_cache_read(c, **{**a, **kw})


def choose(c, **kw):
    a = dict(q=9 * A, R=2, row_stride=256, row_start=11 * A, Hq=4, blocks=12 * A, count=2, head=0, tail=1, workspace=13 * A,
             workspace_bytes=1, io_dtype=P.IO_F16, check=False)
    return P.pasa_cache_choose(c, **{**a, **kw})


def attend(c, **kw):
    a = dict(q=9 * A, o=10 * A, R=2, row_stride=256, row_start=11 * A, Hq=4, scale=0.125, workspace=13 * A, workspace_bytes=1, check=False)
    return P.pasa_attn_cache(c, **{**a, **kw})


# write and read have no workspace that would stop a good call: they are refused for one more thing each time
CALLS = [("write", lambda c: write(c, R=0)), ("read", lambda c: read(c, N=0)), ("choose", choose), ("attend", attend)]


@pytest.mark.parametrize("name,call", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(kscale=None), 1), (dict(vscale=0), 1), (dict(table=None), 1), (dict(length=None), 1),
    (dict(k=A + 8), 1), (dict(v=2 * A + 4), 1), (dict(kscale=3 * A + 4), 1), (dict(kmean=7 * A + 8), 1), (dict(kshift=8 * A + 2), 1),
    (dict(table=5 * A + 2), 1), (dict(length=6 * A + 1), 1), (dict(v=A), 1), (dict(vscale=3 * A), 1),
    (dict(S=0), 1), (dict(Hkv=-1), 1), (dict(pages=0), 1), (dict(table_width=0), 1), (dict(d=0), 1), (dict(page=0), 1), (dict(format=2), 1),
    (dict(format=-1), 1), (dict(d=96), 2), (dict(d=256), 2), (dict(page=8), 2), (dict(page=48), 2), (dict(page=256), 2),
    (dict(table_width=4097), 2), (dict(table_width=16385, page=16), 2), (dict(S=1 << 30, Hkv=4), 2),
])
def test_caches_that_are_refused(name, call, kw, status):
    assert call(cache(**kw)) == status
    if name == "choose":
        assert P.pasa_cache_choose_workspace(cache(**kw)) == 0
    if name == "attend":
        assert P.pasa_attn_cache_workspace(cache(**kw), 2, 4) == 0


def test_no_cache_at_all():
    assert write(None) == 1 and read(None) == 1 and choose(None) == 1 and attend(None) == 1
    assert P.pasa_cache_choose_workspace(None) == 0 and P.pasa_attn_cache_workspace(None, 1, 4) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(row_start=None), 1), (dict(k=9 * A + 8), 1), (dict(v=10 * A + 2), 1), (dict(row_start=11 * A + 2), 1),
    (dict(R=0), 1), (dict(R=-3), 1), (dict(row_stride=127), 1), (dict(row_stride=132), 1), (dict(row_stride=120), 1), (dict(row_stride=-128), 1),
    (dict(io_dtype=2), 1), (dict(R=0x7FFFFFFF), 2),
])
def test_writes_that_are_refused(kw, status):
    assert write(cache(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k=10 * A), 1), (dict(k=9 * A + 8), 1), (dict(first=11 * A + 2), 1), (dict(N=0), 1), (dict(N=-1), 1),
    (dict(io_dtype=-1), 1), (dict(N=262145), 2),
])
def test_reads_that_are_refused(kw, status):
    assert read(cache(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(), 4), (dict(q=None), 1), (dict(row_start=None), 1), (dict(blocks=None), 1), (dict(blocks=12 * A + 2), 1), (dict(R=0), 1),
    (dict(Hq=3), 1), (dict(Hq=0), 1), (dict(count=0), 1), (dict(head=-1), 1), (dict(tail=-1), 1), (dict(row_stride=248), 1), (dict(io_dtype=3), 1),
    (dict(workspace=None, workspace_bytes=1 << 30), 4), (dict(workspace=13 * A + 128, workspace_bytes=1 << 30), 4), (dict(workspace_bytes=255), 4),
    (dict(count=262145), 2),
])
def test_choices_that_are_refused(kw, status):
    assert choose(cache(), **kw) == status


def test_a_choice_needs_the_means():
    assert choose(cache(kmean=None)) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(), 4), (dict(q=None), 1), (dict(o=None), 1), (dict(o=9 * A), 1), (dict(o=10 * A + 8), 1), (dict(row_start=None), 1), (dict(R=-1), 1),
    (dict(Hq=3), 1), (dict(Hq=-4), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(tree=14 * A + 4), 1), (dict(tree=14 * A), 4), (dict(blocks=12 * A, count=0), 1), (dict(blocks=12 * A + 1, count=2), 1),
    (dict(blocks=12 * A, count=2), 4), (dict(row_stride=255), 1), (dict(io_dtype=9), 1), (dict(workspace=None, workspace_bytes=1 << 40), 4),
    (dict(workspace=13 * A + 16, workspace_bytes=1 << 40), 4), (dict(blocks=12 * A, count=262145), 2), (dict(R=0x7FFFFFF0), 2),
])
def test_attention_that_is_refused(kw, status):
    assert attend(cache(), **kw) == status


def test_units_beyond_31_bits_are_refused():
    big = cache(S=1 << 20, Hkv=8, table_width=4096)
    assert attend(big, Hq=8, row_stride=8 * 64) == 2 and P.pasa_attn_cache_workspace(big, 2, 8) == 0


def test_workspaces():
    assert P.pasa_cache_choose_workspace(cache()) == 256                     # 2 x 2 x 4 words of 8 bytes, rounded up
    assert P.pasa_cache_choose_workspace(cache(table_width=4096)) == 2 * 2 * 4096 * 8
    # 2 KV heads x (2 sequences + 0 more blocks) x 4 units = 16 units of 64 keys, four at a time: 4 workgroups of two slots
    assert P.pasa_attn_cache_workspace(cache(), 2, 4) % 256 == 0
    small, large = P.pasa_attn_cache_workspace(cache(), 2, 4), P.pasa_attn_cache_workspace(cache(table_width=4096), 2, 4)
    assert 0 < small < large < 64 << 20
    assert attend(cache(), workspace_bytes=small - 1) == 4


def test_errors_name_the_entry_point():
    for name, call in (("pasa_cache_write:", lambda: write(cache(), R=0, check=True)), ("pasa_cache_read:", lambda: read(cache(), N=0, check=True)),
                       ("pasa_cache_choose:", lambda: choose(cache(), check=True)), ("pasa_attn_cache:", lambda: attend(cache(), check=True))):
        with pytest.raises(P.PasaError, match=name):
            call()


def test_the_description_is_laid_out_as_in_c():
    c = cache()
    assert c.data_ptr() == ctypes.addressof(c) and ctypes.sizeof(c) == 8 * 8 + 7 * 4 + 4
    words = (ctypes.c_uint64 * 8).from_address(c.data_ptr())
    assert list(words) == [A, 2 * A, 3 * A, 4 * A, 7 * A, 8 * A, 5 * A, 6 * A]
    assert list((ctypes.c_int * 7).from_address(c.data_ptr() + 64)) == [2, 2, 64, 64, 8, 4, P.CACHE_I8]
