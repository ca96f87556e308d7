"""The arguments of the cache's calls reach the library in their places, through the extension in C and through ctypes; nothing is launched."""
import ctypes
import functools

import numpy as np
import pytest

import paper_2503_01873_amd as P

VP, CI, CF, SZ, LL = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_longlong
# entry point: its marshaller, the names of its arguments in C's order and their types
ENTRIES = {
    "pasa_cache_write": ("cache_write", "cache k v R row_stride row_start io_dtype stream", [VP, VP, VP, CI, LL, VP, CI, VP]),
    "pasa_cache_read": ("cache_read", "cache k v first N io_dtype stream", [VP, VP, VP, VP, CI, CI, VP]),
    "pasa_cache_choose": ("cache_choose", "cache q R row_stride row_start Hq blocks count head tail io_dtype workspace workspace_bytes stream",
                          [VP, VP, CI, LL, VP, CI, VP, CI, CI, CI, CI, VP, SZ, VP]),
    "pasa_attn_cache": ("attn_cache", "cache q o R row_stride row_start Hq scale tree blocks count io_dtype workspace workspace_bytes stream",
                        [VP, VP, VP, CI, LL, VP, CI, CF, VP, VP, CI, CI, VP, SZ, VP]),
}


class At:
    def __init__(self, address):
        self.address = self.cuda_stream = address

    def data_ptr(self):
        return self.address


def _given(names, types):
    given = {}
    for i, (n, t) in enumerate(zip(names, types)):
        given[n] = At((i + 1) << 40 | 0x10) if t is VP else 100 + i if t is CI else 0.375 if t is CF else (5 << 32) + 3 + i
    return given


@pytest.mark.parametrize("route", ["C", "ctypes"])
@pytest.mark.parametrize("entry", ENTRIES)
def test_every_argument_arrives_in_its_place(entry, route, monkeypatch):
    from paper_2503_01873_amd import _calls, binding
    marshaller, names, types = ENTRIES[entry]
    names = names.split()
    came = {}

    def stand_in(*args):
        came.update(zip(names, args))
        return 7

    f = ctypes.CFUNCTYPE(CI, *types)(stand_in)
    call = functools.partial(getattr(binding, "_" + marshaller), f)
    if route == "C":
        def refused(*args):
            raise AssertionError("ordinary arguments went through ctypes")
        call = functools.partial(getattr(_calls, marshaller), ctypes.cast(f, VP).value, refused)
    monkeypatch.setattr(P.lib(), "call_" + entry, call)
    given = _given(names, types)
    assert getattr(P, entry)(**given, check=False) == 7
    for n, x in given.items():
        assert came[n] == (x.address if isinstance(x, At) else x), n


A = 1 << 20


def _cache():
    return P.pasa_cache(A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, S=2, Hkv=2, d=64, page=64, pages=8, table_width=4, kmean=7 * A)


def _attend(**kw):
    a = dict(cache=_cache(), q=9 * A, o=10 * A, R=2, row_stride=256, row_start=11 * A, Hq=4, scale=0.125, workspace=13 * A, workspace_bytes=1, check=False)
    return P.pasa_attn_cache(**{**a, **kw})


@pytest.mark.parametrize("size", [np.int64(4), np.uint8(4), ctypes.c_int(4)])
def test_sizes_are_whatever_ctypes_takes_for_an_integer(size):
    assert _attend(Hq=size) == 4 and _attend(R=size) == 4
    assert P.pasa_cache_choose(_cache(), 9 * A, size, 256, 11 * A, size, 12 * A, size, 0, 1, 13 * A, 1, check=False) == 4


@pytest.mark.parametrize("kw,error", [({"R": 2.0}, ctypes.ArgumentError), ({"q": "x"}, AttributeError), ({"scale": "x"}, ValueError),
                                      ({"row_stride": 256.0}, ctypes.ArgumentError), ({"stream": "x"}, AttributeError)])
def test_what_is_no_argument_is_refused(kw, error):
    with pytest.raises(error):
        _attend(**kw)


def test_a_description_keeps_its_buffers():
    class Buffer:
        def data_ptr(self):
            return A

    b = Buffer()
    c = P.pasa_cache(b, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 1, 1, 64, 64, 1, 1)
    assert c.k == A and c.buffers[0] is b and c.kmean is None and c.format == P.CACHE_I8
