"""Helpers for the tests of the calls on pages: a pool with small contents that tell pages apart, the same on the GPU."""
from __future__ import annotations

import numpy as np

import paper_2503_01873_amd as P
from oracle import pages_oracle as po
from tests import cache_harness as ch

FORMATS = {"i8": P.CACHE_I8, "e4m3": P.CACHE_E4M3, "i4": P.CACHE_I4}


def pool(g, S, Hkv, d, page, width, pages, format="i4", mean=True):
    """Nobody holds anything; contents are random bytes."""
    raw = page * d * 17 // 32 if format == "i4" else page * d
    c = {"k": g.integers(0, 256, (pages, Hkv, raw), np.uint8), "v": g.integers(0, 256, (pages, Hkv, raw), np.uint8),
         "kscale": g.standard_normal((pages, Hkv, page)).astype(np.float32), "vscale": g.standard_normal((pages, Hkv, page)).astype(np.float32),
         "kmean": g.standard_normal((pages, Hkv, d)).astype(np.float32) if mean else None,
         "table": np.full((S, width), -1, np.int32), "length": np.zeros(S, np.int32), "refs": np.zeros(pages, np.int32), "format": format, "d": d}
    return c


def hold(g, c, lengths, shared=0.0):
    """Sequences get pages, out of order; a part of them those of the sequence before."""
    page = c["kscale"].shape[2]
    free = list(g.permutation(len(c["refs"])))
    for b, n in enumerate(lengths):
        c["length"][b] = n
        for i in range(-(-n // page)):
            if b and g.random() < shared and c["table"][b - 1, i] >= 0:
                c["table"][b, i] = c["table"][b - 1, i]
            else:
                c["table"][b, i] = free.pop()
    c["refs"][:] = po.counts(c)


class OnGpu:
    def __init__(self, c, device="cuda:0"):
        import torch
        self.t = {n: torch.from_numpy(np.ascontiguousarray(x)).to(device) for n, x in c.items() if isinstance(x, np.ndarray)}
        self.device = torch.device(device)
        pages, Hkv, page = c["kscale"].shape
        self.c = P.pasa_cache(*(self.t[n] for n in ("k", "v", "kscale", "vscale", "table", "length")), S=len(c["length"]), Hkv=Hkv, d=c["d"], page=page,
                              pages=pages, table_width=c["table"].shape[1], format=FORMATS[c["format"]], kmean=self.t.get("kmean"))

    def _workspace(self, need):
        import torch
        assert need > 0
        self.need = need
        self.ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=self.device)
        return self.ws, need

    def _done(self):
        import torch
        torch.cuda.synchronize(self.device)
        assert bool((self.ws[self.need:] == 0xFF).all()), "written behind the workspace"

    def stream(self):
        import torch
        return torch.cuda.current_stream(self.device)

    def fork(self, source):
        P.pasa_cache_fork(self.c, self.t["refs"], ch.ints(source, self.device), *self._workspace(P.pasa_cache_fork_workspace(self.c)), self.stream())
        self._done()

    def room(self, row_start, R):
        lacking = ch.ints([-7], self.device)
        P.pasa_cache_room(self.c, self.t["refs"], R, ch.ints(row_start, self.device), lacking, *self._workspace(P.pasa_cache_room_workspace(self.c, R)), self.stream())
        self._done()
        return int(lacking[0])

    def compact(self):
        used = ch.ints([-7], self.device)
        P.pasa_cache_compact(self.c, self.t["refs"], used, *self._workspace(P.pasa_cache_compact_workspace(self.c)), self.stream())
        self._done()
        return int(used[0])

    def free(self):
        P.pasa_cache_free(self.c, self.t["refs"], self.stream())

    def same(self, c):
        for n, x in c.items():
            if isinstance(x, np.ndarray):
                got = self.t[n].cpu().numpy()
                assert np.array_equal(got, x, equal_nan=x.dtype == np.float32), (n, np.argwhere(got != x)[:5])
