"""The arguments of the calls for rotary positions and pages reach the library in their places, through the extension in C and through ctypes; nothing is launched."""
import ctypes
import functools

import numpy as np
import pytest

import paper_2503_01873_amd as P

VP, CI, SZ, LL = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_longlong
# entry point: its marshaller, the names of its arguments in C's order and their types
ENTRIES = {
    "pasa_rotate": ("rotate", "rotary x y B H N d x_strides y_strides positions row0 transposed io_dtype stream", [VP, VP, VP, CI, CI, CI, CI, VP, VP, VP, CI, CI, CI, VP]),
    "pasa_cache_rotate": ("cache_rotate", "cache rotary x y heads R x_stride y_stride row_start tree transposed io_dtype stream",
                          [VP, VP, VP, VP, CI, CI, LL, LL, VP, VP, CI, CI, VP]),
    "pasa_cache_fork": ("cache_fork", "cache refs source workspace workspace_bytes stream", [VP, VP, VP, VP, SZ, VP]),
    "pasa_cache_room": ("cache_room", "cache refs R row_start lacking workspace workspace_bytes stream", [VP, VP, CI, VP, VP, VP, SZ, VP]),
}


class At:
    def __init__(self, address):
        self.address = self.cuda_stream = address

    def data_ptr(self):
        return self.address


def _call(entry, route, monkeypatch, came, look=lambda n, x: x):
    from paper_2503_01873_amd import _calls, binding
    marshaller, names, types = ENTRIES[entry]

    def stand_in(*args):
        came.update({n: look(n, x) for n, x in zip(names.split(), args)})
        return 7

    f = ctypes.CFUNCTYPE(CI, *types)(stand_in)
    call = functools.partial(getattr(binding, "_" + marshaller), f)
    if route == "C":
        def refused(*args):
            raise AssertionError("ordinary arguments went through ctypes")
        call = functools.partial(getattr(_calls, marshaller), ctypes.cast(f, VP).value, refused)
    monkeypatch.setattr(P.lib(), "call_" + entry, call)
    return f


@pytest.mark.parametrize("route", ["C", "ctypes"])
@pytest.mark.parametrize("entry", ENTRIES)
def test_every_argument_arrives_in_its_place(entry, route, monkeypatch):
    came, given = {}, {}
    keep = _call(entry, route, monkeypatch, came)
    _, names, types = ENTRIES[entry]
    for i, (n, t) in enumerate(zip(names.split(), types)):
        given[n] = At((i + 1) << 40 | 0x10) if t is VP else 100 + i if t is CI else (5 << 32) + 3 + i
        if n.endswith("strides"):
            given[n] = given[n].address
    assert getattr(P, entry)(**given, check=False) == 7
    for n, x in given.items():
        assert came[n] == (x.address if isinstance(x, At) else x), n
    del keep


@pytest.mark.parametrize("route", ["C", "ctypes"])
def test_strides_arrive(route, monkeypatch):
    came = {}
    keep = _call("pasa_rotate", route, monkeypatch, came,
                 lambda n, x: list((LL * 3).from_address(x)) if n.endswith("strides") and x else x)
    P.pasa_rotate(None, 16, 32, 1, 2, 3, 64, x_strides=(1 << 40, 64, 8), y_strides=(0, 8, 1 << 33), transposed=True, check=False)
    assert came["x_strides"] == [1 << 40, 64, 8] and came["y_strides"] == [0, 8, 1 << 33] and came["transposed"] == 1 and came["stream"] is None
    P.pasa_rotate(None, 16, 32, 1, 2, 3, 64, check=False)
    assert came["x_strides"] is None and came["y_strides"] is None and came["rotary"] is None and came["row0"] == 0 and came["transposed"] == 0
    P.pasa_rotate(None, 16, 32, 1, 2, 3, 64, row0=-5, check=False)
    assert came["row0"] == -5
    del keep


def test_sizes_and_strides_are_whatever_ctypes_takes():
    r = P.pasa_rotary(magnitude=1.0, rot=64)
    for size in (np.int64(5), ctypes.c_int(5)):
        assert P.pasa_rotate(r, 16, 32, size, size, size, 63, check=False) == 1
    assert P.pasa_rotate(r, 16, 32, 1, 1, 1, 64, x_strides=[8, 8, 7], check=False) == 1
    assert P.pasa_rotate(r, 16, 32, 1, 1, 1, 64, x_strides=np.array([8, 8, 7]), check=False) == 1
    with pytest.raises(ctypes.ArgumentError):
        P.pasa_rotate(r, 16, 32, 1.0, 1, 1, 64)
    with pytest.raises(AttributeError):
        P.pasa_rotate(r, "x", 32, 1, 1, 1, 64)
    with pytest.raises(AttributeError):
        P.pasa_cache_fork(P.pasa_cache(16, 32, 48, 64, 16, 16, 1, 1, 64, 64, 1, 1), 16, 16, 256, 256, "stream")
