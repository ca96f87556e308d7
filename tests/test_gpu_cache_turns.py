"""The cache's calls together, as a server makes them: whole steps, graphs, streams, long chunks, large pools."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import cache_oracle as co
from oracle import pasa_oracle as po
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu


class Server:
    """Sequences that grow, on the GPU and in the oracle."""

    def __init__(self, g, S, Hq, Hkv, d, page, width, format="i8", dtype="f16", count=0):
        import torch
        self.g, self.S, self.Hq, self.Hkv, self.d, self.dtype, self.count = g, S, Hq, Hkv, d, dtype, count
        self.c = ch.empty(g, S, Hkv, d, page, width, format, shift=True)
        self.gpu = ch.OnGpu(self.c)
        self.scale = float(np.float32(d ** -0.5))
        self.type = torch.float16 if dtype == "f16" else torch.bfloat16

    def buffers(self, R):
        """What a step reads and writes, allocated once."""
        import torch
        dev = "cuda:0"
        self.R = R
        self.qkv = torch.zeros((R, (self.Hq + 2 * self.Hkv) * self.d), dtype=self.type, device=dev)
        self.row_start = torch.zeros(self.S + 1, dtype=torch.int32, device=dev)
        self.o = torch.full((R, self.Hq, self.d), float("nan"), dtype=self.type, device=dev)
        self.blocks = torch.zeros((self.S, self.Hkv, max(self.count, 1)), dtype=torch.int32, device=dev)
        self.choose_bytes = P.pasa_cache_choose_workspace(self.gpu.cache)
        self.choose_ws = torch.empty(self.choose_bytes, dtype=torch.uint8, device=dev)
        self.attn_bytes = P.pasa_attn_cache_workspace(self.gpu.cache, R, self.Hq)
        self.attn_ws = torch.empty(self.attn_bytes, dtype=torch.uint8, device=dev)

    def inputs(self, length, rows):
        """New tokens of the sequences, and their rows; on the GPU by copies into the buffers."""
        import torch
        R = self.R
        q = ch.rounded(2 * self.g.standard_normal((R, self.Hq, self.d)), self.dtype)
        k = ch.rounded(self.g.standard_normal((R, self.Hkv, self.d)) + self.c["kshift"], self.dtype)
        v = ch.rounded(self.g.standard_normal((R, self.Hkv, self.d)), self.dtype)
        self.c["length"][:] = length
        self.starts = ch.starts(rows)
        self.gpu.t["length"].copy_(ch.ints(length))
        self.row_start.copy_(ch.ints(self.starts))
        self.qkv.copy_(torch.from_numpy(np.concatenate([x.reshape(R, -1) for x in (q, k, v)], 1)).to(self.type))
        self.q, self.k, self.v = q.astype(np.float64), k, v

    def calls(self, stream):
        n, m = self.Hq * self.d, self.Hkv * self.d
        q, k, v = self.qkv[:, :n], self.qkv[:, n:n + m], self.qkv[:, n + m:]
        io, stride = ch.IO[self.dtype], self.qkv.stride(0)
        P.pasa_cache_write(self.gpu.cache, k, v, self.R, stride, self.row_start, stream, io_dtype=io)
        if self.count:
            P.pasa_cache_choose(self.gpu.cache, q, self.R, stride, self.row_start, self.Hq, self.blocks, self.count, 1, 1, self.choose_ws,
                                self.choose_bytes, stream, io_dtype=io)
        P.pasa_attn_cache(self.gpu.cache, q, self.o, self.R, stride, self.row_start, self.Hq, self.scale, self.attn_ws, self.attn_bytes, stream,
                          blocks=self.blocks if self.count else None, count=self.count, io_dtype=io)

    def check(self):
        """The step just taken, against the oracle, which takes it too."""
        import torch
        torch.cuda.synchronize()
        co.write(self.c, self.k, self.v, self.starts)
        blocks = None
        if self.count:
            # the means on the GPU: their last bits could make another choice
            self.c["kmean"] = self.gpu.back("kmean")
            blocks = co.choose(self.c, self.q, self.starts, self.count, 1, 1)
            assert np.array_equal(self.blocks.cpu().numpy(), blocks)
        got = self.o.double().cpu().numpy()
        rows = slice(self.starts[0], self.starts[-1])
        ref = co.attend(self.c, self.q, self.starts, self.scale, blocks=blocks)
        ch.check_attend(self.c, got[rows], [x[rows] for x in ref], self.dtype, int(self.c["length"].max()))


@pytest.mark.parametrize("format,dtype,count,Hq,Hkv,d,page", [("i8", "f16", 0, 28, 4, 128, 64), ("e4m3", "bf16", 5, 28, 4, 128, 32), ("i8", "bf16", 3, 5, 5, 64, 16)])
def test_prompts_and_steps(format, dtype, count, Hq, Hkv, d, page):
    """Prompts of ragged length, then steps, one of them with a sequence that pauses, one after drafted tokens were taken back."""
    import torch
    g = np.random.default_rng([d, page])
    s = Server(g, 4, Hq, Hkv, d, page, -(-400 // page), format, dtype, count)
    length = np.array([333, 1, 70, 128])
    s.buffers(int(length.sum()))
    s.inputs(length, length)
    s.calls(torch.cuda.current_stream())
    s.check()
    s.buffers(4 + 3)
    for rows in ([1, 1, 1, 1], [1, 0, 1, 1], [2, 1, 3, 1]):
        length = length + rows
        s.inputs(length, rows)
        s.calls(torch.cuda.current_stream())
        s.check()
    length = length - [1, 0, 2, 0]                  # the drafted ones that were not accepted
    length = length + 1
    s.inputs(length, [1, 1, 1, 1])
    s.calls(torch.cuda.current_stream())
    s.check()


@pytest.mark.parametrize("count", [0, 4])
def test_a_captured_step_follows_lengths_and_rows(count):
    """One graph, replayed for sequences that grow; the program's own work and an eager call with the same workspace in between."""
    import torch
    g = np.random.default_rng(3)
    s = Server(g, 3, 8, 2, 128, 32, 40, count=count)
    length = np.array([500, 31, 900])
    s.buffers(int(length.sum()))
    s.inputs(length, length)
    s.calls(torch.cuda.current_stream())
    torch.cuda.synchronize()
    co.write(s.c, s.k, s.v, s.starts)
    s.buffers(5)
    length = length + 1
    s.inputs(length, [1, 1, 1])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s.calls(stream)
    torch.cuda.current_stream().wait_stream(stream)
    s.check()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    for x in (graph, other):                        # two graphs that share buffers and workspaces
        with torch.cuda.graph(x):
            s.calls(torch.cuda.current_stream())
    for turn, rows in enumerate([[1, 1, 1], [1, 0, 2], [0, 3, 1], [1, 1, 1], [2, 2, 1]]):
        length = length + rows
        s.inputs(length, rows)
        s.o.fill_(float("nan"))
        (other if turn == 3 else graph).replay()
        torch.cuda.synchronize()
        first = s.o.clone()
        s.check()
        s.o.fill_(float("nan"))
        s.calls(torch.cuda.current_stream())        # the same step again, eager: the same bits
        torch.cuda.synchronize()
        assert torch.equal(first.view(torch.int16), s.o.view(torch.int16))
        _ = torch.randn(1000, 1000, device="cuda:0").sum().item()


def test_a_stream_of_its_own():
    """Everything on another stream than the current one, behind work that it has to wait for."""
    import torch
    g = np.random.default_rng(4)
    s = Server(g, 2, 4, 2, 64, 16, 30)
    s.buffers(300)
    s.inputs([200, 100], [200, 100])
    right = s.qkv.clone()
    s.qkv.zero_()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        a = torch.randn(4096, 4096, device="cuda:0")
        for _ in range(8):
            a = (a @ a) * 1e-3
        s.qkv.copy_(right)
    s.calls(stream)
    stream.synchronize()
    s.check()


def test_a_long_chunk_goes_through_the_prepared_keys():
    """Read back, prepared, attended to by the calls for long chunks: what the cache holds, with the shift it was written with."""
    import torch
    g = np.random.default_rng(5)
    N, Nq, Hq, Hkv, d = 700, 200, 4, 2, 128
    c = ch.filled(g, [N], Hkv, d, 64, "i8", shift=True)
    gpu = ch.OnGpu(c)
    k, v = (torch.empty((1, Hkv, N, d), dtype=torch.float16, device="cuda:0") for _ in range(2))
    stream = torch.cuda.current_stream()
    P.pasa_cache_read(gpu.cache, k, v, None, N, stream)
    q = torch.from_numpy(g.standard_normal((1, Hq, Nq, d)).astype(np.float16)).to("cuda:0")
    o = torch.empty_like(q)
    size = P.pasa_attn_fwd_workspace(1, Hq, Hkv, N, d)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda:0")
    scale = float(np.float32(d ** -0.5))
    P.pasa_prepare_kv(k, v, 1, Hkv, N, d, scale, ws, size, stream)
    P.pasa_attn_fwd_chunk(q, o, 1, Hq, Hkv, Nq, N - Nq, N, d, True, scale, ws, size, stream)
    # the rows of the chunk through the cache itself: the same attention
    rows = q[0].transpose(0, 1).contiguous()
    o2 = torch.empty_like(rows)
    size = P.pasa_attn_cache_workspace(gpu.cache, Nq, Hq)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda:0")
    P.pasa_attn_cache(gpu.cache, rows, o2, Nq, Hq * d, ch.ints([0, Nq]), Hq, scale, ws, size, stream)
    torch.cuda.synchronize()
    want_k, want_v = co.read(c, None, N)
    assert np.abs(k.double().cpu().numpy() - want_k).max() <= 2.0 ** -10 * np.abs(want_k).max()
    pad = np.zeros((1, Hq, N - Nq, d), np.float16)
    ref = po.pasa_bhnd(np.concatenate([pad, q.cpu().numpy()], 2), k.cpu().numpy(), v.cpu().numpy(), scale, True, po.default_beta(), 128, po.MIXED)
    assert np.abs(o.double().cpu().numpy() - ref[:, :, N - Nq:].astype(np.float64)).max() <= 2e-3
    rows = rows.double().cpu().numpy()
    ch.check_attend(c, o2.double().cpu().numpy(), co.attend(c, rows, ch.starts([Nq]), scale), "f16", N)


def test_a_pool_beyond_4_gib_and_rows_far_apart():
    """Pages whose bytes lie beyond 2^32, rows whose elements do."""
    import torch
    g = np.random.default_rng(6)
    Hq, Hkv, d, page, pages = 4, 2, 128, 128, 140000                     # 4.6 GB of keys
    small = ch.empty(g, 2, Hkv, d, page, 3, "i8", spare=0)
    ids = np.array([[139999, 5, 131073], [0, 139998, 70000]], np.int32)
    dev = "cuda:0"
    t = {n: torch.empty((pages, Hkv, page, d), dtype=torch.uint8, device=dev) for n in ("k", "v")}
    t |= {n: torch.full((pages, Hkv, page), float("nan"), device=dev) for n in ("kscale", "vscale")}
    t["kmean"] = torch.zeros((pages, Hkv, d), device=dev)
    length, table = ch.ints([300, 257]), ch.ints(ids)
    cache = P.pasa_cache(t["k"], t["v"], t["kscale"], t["vscale"], table, length, 2, Hkv, d, page, pages, 3, kmean=t["kmean"])
    R, stride = 557, 1 << 22                                             # 2.3 G elements
    flat = torch.empty(R * stride, dtype=torch.float16, device=dev)
    x = ch.rounded(g.standard_normal((R, Hq + 2 * Hkv, d)), "f16")
    flat.view(R, stride)[:, :x[0].size] = torch.from_numpy(x.reshape(R, -1)).to(dev).half()
    q, k, v = flat, flat[Hq * d:], flat[(Hq + Hkv) * d:]
    stream = torch.cuda.current_stream()
    row_start = ch.ints([0, 300, 557])
    P.pasa_cache_write(cache, k, v, R, stride, row_start, stream)
    out = [torch.empty((2, Hkv, 300, d), dtype=torch.float16, device=dev) for _ in range(2)]
    P.pasa_cache_read(cache, out[0], out[1], None, 300, stream)
    o = torch.empty((R, Hq, d), dtype=torch.float16, device=dev)
    size = P.pasa_attn_cache_workspace(cache, R, Hq)
    ws = torch.empty(size, dtype=torch.uint8, device=dev)
    P.pasa_attn_cache(cache, q, o, R, stride, row_start, Hq, 0.088, ws, size, stream)
    torch.cuda.synchronize()
    # the same tokens in a small pool, in the oracle
    small["length"][:] = [300, 257]
    co.write(small, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], ch.starts([300, 257]))
    want = co.read(small, None, 300)
    for a, b in zip(out, want):
        assert np.abs(a.double().cpu().numpy() - b).max() <= 2.0 ** -11 * np.abs(b).max() * (1 + 2.0 ** -10) + 2.0 ** -24
    ref = co.attend(small, x[:, :Hq].astype(np.float64), ch.starts([300, 257]), float(np.float32(0.088)))
    ch.check_attend(small, o.double().cpu().numpy(), ref, "f16", 300)
    got = t["kmean"][torch.from_numpy(ids.reshape(-1)).long().to(dev)].cpu().numpy()
    want = small["kmean"][small["table"].reshape(-1)]
    there = ~np.isnan(want)
    assert np.abs(got[there] - want[there]).max() <= 1e-5


def test_shared_pages_and_rows_before_the_first_sequence():
    """Two sequences that share a prefix they do not write, and rows that belong to nobody before the first and behind the last."""
    import torch
    g = np.random.default_rng(7)
    Hq, Hkv, d, page = 4, 2, 64, 32
    c = ch.filled(g, [96 + 10, 0], Hkv, d, page, "e4m3", width=5)
    c["table"][1, :3] = c["table"][0, :3]
    c["length"][:] = [96 + 11, 96 + 2]
    gpu = ch.OnGpu(c)
    row_start = np.array([2, 3, 5], np.int32)
    k, v = (ch.rounded(g.standard_normal((7, Hkv, d)), "f16") for _ in range(2))
    q = ch.rounded(g.standard_normal((7, Hq, d)), "f16").astype(np.float64)
    tk, st = ch.tensor(k, "f16")
    tv, _ = ch.tensor(v, "f16")
    P.pasa_cache_write(gpu.cache, tk, tv, 7, st, ch.ints(row_start), torch.cuda.current_stream())
    co.write(c, k, v, row_start)
    got = ch.run_attend(gpu, q, row_start, 0.125, "f16")
    ref = co.attend(c, q, row_start, 0.125)
    assert np.isnan(got[:2]).all() and np.isnan(got[5:]).all()
    ch.check_attend(c, got, ref, "f16", 107)
    for n in ("k", "kscale", "v", "vscale"):
        assert np.array_equal(gpu.back(n), c[n], equal_nan=True)
