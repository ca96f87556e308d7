"""The paged 8-bit cache on the GPU against the oracle: tokens in, tokens back, pages chosen, attention."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import cache_oracle as co
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu

FORMATS = ["i8", "e4m3"]


def _gpu(c):
    return ch.OnGpu(c)


def _write(gpu, k, v, row_start, dtype, stride=None):
    import torch
    R, Hkv, d = k.shape
    tk, st = ch.tensor(k, dtype, stride)
    tv, _ = ch.tensor(v, dtype, stride)
    P.pasa_cache_write(gpu.cache, tk, tv, R, st, ch.ints(row_start), torch.cuda.current_stream(), io_dtype=ch.IO[dtype])
    torch.cuda.synchronize()


def _same_cache(gpu, c):
    """Scales bit for bit, codes by value (zero has two in e4m3), means to their last bits."""
    for n in ("k", "v"):
        s = gpu.back(n + "scale")
        assert np.array_equal(s, c[n + "scale"], equal_nan=True)
        a, b = gpu.back(n), c[n]
        if c["format"] == "e4m3":
            a, b = co.E4M3[a], co.E4M3[b]
        assert np.array_equal(a, b, equal_nan=True)
    if c["kmean"] is not None:
        # a product and an addition a token in fp32 (128 tokens at most), and the quotient
        m = gpu.back("kmean")
        assert np.array_equal(np.isnan(m), np.isnan(c["kmean"]))
        with np.errstate(invalid="ignore"):
            x = np.abs(co.values(c["k"], c["kscale"], c["format"]))
            wide = np.where(np.isnan(x), 0.0, x).max(axis=2)
            assert not (np.abs(m.astype(np.float64) - c["kmean"]) > 132 * 2.0 ** -24 * wide).any()


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,Hkv,page", [(128, 4, 64), (64, 5, 16), (128, 1, 128), (64, 2, 32)])
def test_tokens_enter_in_steps(d, Hkv, page, dtype, format):
    """Prompts, single tokens, none, and a step that is taken back; sequences without tokens; rows behind the last sequence; strides."""
    g = np.random.default_rng([d, page, FORMATS.index(format)])
    S, width = 4, 5
    c = ch.empty(g, S, Hkv, d, page, width, format, shift=page != 16, mean=page != 128)
    gpu = _gpu(c)
    for step, (length, rows, behind) in enumerate([
        ([2 * page + 3, 1, 0, page], [2 * page + 3, 1, 0, page], 2),
        ([2 * page + 4, 2, 1, page + 1], [1, 1, 1, 1], 0),
        ([2 * page + 4, 2 + page, 1, 3 * page], [0, page, 0, 2 * page - 1], 1),
        ([2 * page + 1, 3, 2, 3 * page - 2], [2, 1, 1, 5], 0),             # shorter than before: what was behind is overwritten
    ]):
        R = sum(rows) + behind
        k = ch.rounded(g.standard_normal((R, Hkv, d)) * 2.0 ** g.integers(-12, 8, (R, Hkv, 1)), dtype)
        v = ch.rounded(g.standard_normal((R, Hkv, d)) * 2.0 ** g.integers(-12, 8, (R, Hkv, 1)), dtype)
        k[0, 0], v[R - 1, 0] = 0.0, 0.0
        c["length"][:] = length
        gpu.t["length"].copy_(ch.ints(length))
        co.write(c, k, v, ch.starts(rows))
        _write(gpu, k, v, ch.starts(rows), dtype, None if step % 2 else (Hkv + 3) * d + 8)
        _same_cache(gpu, c)


@pytest.mark.parametrize("format", FORMATS)
def test_every_tie_and_border_of_the_codes(format):
    """All finite fp16 values as one channel beside a largest one: quotients that are ties, or nearly."""
    g = np.random.default_rng(5)
    bits = np.arange(1 << 16, dtype=np.uint16).view(np.float16).astype(np.float32)
    bits = bits[np.isfinite(bits)]
    tops = np.array([127.0, 448.0, 1.0, 254.0, 0.0999755859375, 60000.0, 3.0, 2.0 ** -24], np.float32)
    rows = []
    for top in tops:
        x = bits[np.abs(bits) <= top]
        x = np.concatenate([x, np.zeros(-len(x) % 63, np.float32)]).reshape(-1, 63)
        rows.append(np.concatenate([np.full((len(x), 1), top, np.float32), x], 1))
    x = np.concatenate(rows)
    x = x[g.permutation(len(x))[:4000]] if len(x) > 4000 else x
    n = len(x)
    c = ch.empty(g, 1, 1, 64, 128, -(-n // 128), format)
    c["length"][:] = n
    gpu = _gpu(c)
    k, v = x[:, None], np.ascontiguousarray(x[::-1, None])
    co.write(c, k, v, ch.starts([n]))
    _write(gpu, k, v, ch.starts([n]), "f16")
    _same_cache(gpu, c)


@pytest.mark.parametrize("format", FORMATS)
def test_values_that_are_not_finite_and_the_smallest(format):
    """A token that holds one gets the scale NaN and finite codes; other tokens and heads keep theirs."""
    g = np.random.default_rng(6)
    c = ch.empty(g, 2, 2, 64, 16, 2, format, shift=True)
    n = [20, 7]
    c["length"][:] = n
    k, v = (ch.rounded(g.standard_normal((27, 2, 64)), "bf16") for _ in range(2))
    k[3, 1, 5], k[4, 0, 63], v[9, 1, 0], v[26, 0, 8] = np.nan, np.inf, -np.inf, np.nan
    v[10, 0] = ch.rounded(np.full(64, 2.0 ** -101), "bf16")              # below what a scale is made for: rounds to zero
    v[11, 0] = ch.rounded(np.linspace(-1, 1, 64) * 2.0 ** -99, "bf16")
    v[12, 1] = ch.rounded(np.linspace(-1, 1, 64) * 2.0 ** 127, "bf16")
    gpu = _gpu(c)
    co.write(c, k, v, ch.starts(n))
    _write(gpu, k, v, ch.starts(n), "bf16")
    _same_cache(gpu, c)
    assert np.isnan(c["kscale"]).sum() - np.isnan(gpu.back("kscale")).sum() == 0
    codes = gpu.back("k")[c["table"][0, 0], 1, 3]
    assert (codes == (128 if format == "i8" else 0)).all()


def test_tokens_without_a_page_are_dropped_and_nothing_else_is_touched():
    """Table entries outside the pool, lengths and row numbers beyond their range, rows before position 0."""
    g = np.random.default_rng(7)
    c = ch.empty(g, 4, 2, 64, 16, 3, "i8")
    c["table"][0, 1], c["table"][1, 0], c["table"][2, 2] = -5, 1 << 30, c["k"].shape[0]
    c["length"][:] = [40, 20, 1000, 2]
    rows = ch.starts([30, 20, 48, 5])
    rows[4] = 5000                                                        # beyond R
    R = 103
    k, v = (ch.rounded(g.standard_normal((R, 2, 64)), "f16") for _ in range(2))
    gpu = _gpu(c)
    co.write(c, k, v, rows)
    _write(gpu, k, v, rows, "f16")
    _same_cache(gpu, c)


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,page,N", [(128, 64, 1), (64, 16, 200), (128, 32, 300), (64, 128, 129)])
def test_tokens_come_back(d, page, N, dtype, format):
    import torch
    g = np.random.default_rng([d, N])
    c = ch.filled(g, [300, 1, 0, 170], 3, d, page, format, dtype, shift=N != 300, wild=True)
    c["table"][3, 0] = c["k"].shape[0] + 3
    gpu = _gpu(c)
    n = 4 * 3 * N * d
    for first in (None, [0, 0, 0, 0], [299, -1, 5, 100], [-3, 2, 0, 2 ** 31 - 1]):
        out = [torch.full((n + 1024,), float("nan"), dtype=torch.float16 if dtype == "f16" else torch.bfloat16, device="cuda:0") for _ in range(2)]
        P.pasa_cache_read(gpu.cache, out[0], out[1], None if first is None else ch.ints(first), N, torch.cuda.current_stream(), io_dtype=ch.IO[dtype])
        torch.cuda.synchronize()
        for t, want, shift in zip(out, co.read(c, first, N), (c["kshift"], None)):
            assert bool(torch.isnan(t[n:]).all())
            got = t[:n].view(4, 3, N, d).double().cpu().numpy()
            extra = 0 if shift is None else 2.0 ** -23 * (np.abs(want) + 2 * np.abs(shift)[None, :, None])      # the sum in fp32
            bound = ch.HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -10) + ch.TINY[dtype] + extra + 2.0 ** -23 * np.abs(want)
            assert not (np.abs(got - want) > bound).any() and np.isfinite(got).all()
            assert not got[want == 0].any()


def _queries(g, R, Hq, d, dtype, size=1.5):
    return ch.rounded(size * g.standard_normal((R, Hq, d)), dtype).astype(np.float64)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,Hq,Hkv,page,count,head,tail", [
    (128, 28, 4, 64, 8, 1, 1), (64, 5, 5, 16, 40, 0, 2), (128, 2, 2, 32, 1, 0, 0), (64, 16, 2, 128, 3, 2, 2), (128, 8, 1, 16, 16, 16, 1)])
def test_pages_are_chosen(d, Hq, Hkv, page, count, head, tail, dtype):
    import torch
    g = np.random.default_rng([d, Hq, page])
    lengths = [1500, 7, 0, page * count, 1200, 3 * page * count + 1]
    rows = [3, 1, 1, 2, 0, 1]
    c = ch.filled(g, [min(n, 1500) for n in lengths], Hkv, d, page, "i8", width=-(-1500 // page) + 1)
    R = sum(rows) + 1
    q = _queries(g, R, Hq, d, dtype)
    ids = c["table"][0]
    c["kmean"][ids[5]] = c["kmean"][ids[3]]                       # equal scores: the first is taken
    if len(ids) > 12:
        c["kmean"][ids[9]], c["kmean"][ids[7], :, 2] = 0.0, np.nan
        c["table"][5, 2] = -1
    gpu = _gpu(c)
    need = P.pasa_cache_choose_workspace(gpu.cache)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda:0")
    out = torch.full((6 * Hkv * count + 16,), -7, dtype=torch.int32, device="cuda:0")
    tq, st = ch.tensor(q, dtype, (Hq + 1) * d)
    P.pasa_cache_choose(gpu.cache, tq, R, st, ch.ints(ch.starts(rows)), Hq, out, count, head, tail, ws, need, torch.cuda.current_stream(), io_dtype=ch.IO[dtype])
    torch.cuda.synchronize()
    assert bool((out[-16:] == -7).all()) and bool((ws[need:] == 0xFF).all())
    want = co.choose(c, q, ch.starts(rows), count, head, tail)
    assert np.array_equal(out[:-16].cpu().numpy().reshape(want.shape), want)


@pytest.mark.parametrize("width,count", [(1024, 100), (1025, 300), (4096, 4095), (4097, 7), (16384, 256)])
def test_pages_of_long_sequences_are_chosen(width, count):
    """Every size of the kernel that picks, up to the largest table; many equal scores at the border."""
    import torch
    g = np.random.default_rng(width)
    d, Hkv, page, S = 64, 2, 16, 2
    c = ch.empty(g, S, Hkv, d, page, 1, "i8")
    pool = 50
    c["table"] = g.integers(0, c["k"].shape[0], (S, width)).astype(np.int32)      # few different pages: equal scores
    c["kmean"] = g.standard_normal(c["kmean"].shape).astype(np.float32)
    c["length"][:] = [width * page, width * page - 17]
    gpu = _gpu(c)
    q = _queries(g, 2, 4, d, "f16")
    ws = torch.empty(P.pasa_cache_choose_workspace(gpu.cache), dtype=torch.uint8, device="cuda:0")
    out = torch.empty((S, Hkv, count), dtype=torch.int32, device="cuda:0")
    tq, st = ch.tensor(q, "f16")
    P.pasa_cache_choose(gpu.cache, tq, 2, st, ch.ints([0, 1, 2]), 4, out, count, 1, 1, ws, ws.numel(), torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert np.array_equal(out.cpu().numpy(), co.choose(c, q, ch.starts([1, 1]), count, 1, 1))


LAYOUTS = [(28, 4, 128), (5, 5, 64), (8, 1, 128), (16, 2, 64), (3, 1, 64)]


@pytest.mark.parametrize("format,dtype", [("i8", "f16"), ("e4m3", "bf16"), ("i8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("Hq,Hkv,d", LAYOUTS)
@pytest.mark.parametrize("page", [16, 64, 128])
def test_a_decoding_step(page, Hq, Hkv, d, format, dtype):
    """One row per sequence; lengths from nothing to several units of work, around their borders."""
    g = np.random.default_rng([page, Hq, d])
    lengths = [1, 0, 63, 64, 65, 700, 128, 1345]
    c = ch.filled(g, lengths, Hkv, d, page, format, dtype, shift=page == 64, wild=True)
    q = _queries(g, len(lengths), Hq, d, dtype)
    scale = float(np.float32(d ** -0.5))
    row_start = ch.starts([1] * len(lengths))
    got = ch.run_attend(_gpu(c), q, row_start, scale, dtype)
    ref = co.attend(c, q, row_start, scale)
    assert not ref[0][1].any()
    ch.check_attend(c, got, ref, dtype, max(lengths))


@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (16, 16, 64), (4, 4, 128)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("format", FORMATS)
def test_chains_and_trees(Hq, Hkv, d, tree, format):
    """Rows per sequence from none to 64 (chains: more), sequences that consist of nothing else, rows before position 0, rows behind the last sequence."""
    g = np.random.default_rng([Hq, d, tree])
    lengths, rows = [300, 64, 5, 90, 1, 200], [7, 64, 9, 0, 1, 40 if tree else 90]
    c = ch.filled(g, lengths, Hkv, d, 32, format, wild=True)
    R = sum(rows) + 3
    q = _queries(g, R, Hq, d, "f16")
    bits = None
    if tree:
        bits = np.zeros(R, np.uint64)
        for r0, m in zip(ch.starts(rows), rows):
            for t in range(m):
                parent = int(g.integers(0, t)) if t and g.random() < 0.9 else None
                bits[r0 + t] = np.uint64(1 << t) | (bits[r0 + parent] if parent is not None else np.uint64(0))
        bits[0] = 0                                                     # does not see itself
        bits[3] = np.uint64(2 ** 64 - 1)                                # bits of tokens that are not there
        bits[ch.starts(rows)[1] + 5] = 0                                # sees nothing at all
    scale = float(np.float32(d ** -0.5))
    got = ch.run_attend(_gpu(c), q, ch.starts(rows), scale, "f16", tree=bits, stride=(Hq + 2 * Hkv) * d)
    ref = co.attend(c, q, ch.starts(rows), scale, tree=bits)
    assert np.isnan(got[-3:]).all()
    ch.check_attend(c, got, ref, "f16", max(lengths))


@pytest.mark.parametrize("page,count", [(16, 9), (64, 4), (128, 2), (32, 100)])
@pytest.mark.parametrize("rows", [1, 5])
def test_only_chosen_pages_are_seen(page, count, rows):
    g = np.random.default_rng([page, rows])
    lengths = [900, 33, 0, 640, 1000]
    Hq, Hkv, d = 12, 2, 128
    c = ch.filled(g, lengths, Hkv, d, page, "i8", wild=True)
    blocks = np.full((5, Hkv, count), -1, np.int32)
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            pages = -(-n // page)
            at = np.sort(g.permutation(pages)[:count - (h and b == 3)])
            blocks[b, h, :len(at)] = at
    blocks[4, 1, :] = -1                                                # nothing chosen: zeros
    if count == 9:
        blocks[0, 0, 2] = 10 ** 6                                       # outside the table
    q = _queries(g, 5 * rows, Hq, d, "f16")
    scale = float(np.float32(d ** -0.5))
    got = ch.run_attend(_gpu(c), q, ch.starts([rows] * 5), scale, "f16", blocks=blocks)
    ref = co.attend(c, q, ch.starts([rows] * 5), scale, blocks=blocks)
    ch.check_attend(c, got, ref, "f16", max(lengths))


@pytest.mark.parametrize("S,L,Hq,Hkv,d,rows", [(1, 4999, 28, 4, 128, 1), (1, 40000, 8, 1, 64, 1), (2, 9000, 4, 2, 128, 20), (40, 500, 5, 5, 64, 1),
                                               (300, 90, 2, 1, 64, 1)])
def test_work_that_many_workgroups_share(S, L, Hq, Hkv, d, rows):
    """Long sequences are swept by several workgroups, many short ones by few; a workgroup's range crosses sequences."""
    g = np.random.default_rng([S, L])
    lengths = [L] + [int(n) for n in g.integers(0 if S > 10 else L // 2, L + 1, S - 1)]
    c = ch.filled(g, lengths, Hkv, d, 64, "i8")
    q = _queries(g, S * rows, Hq, d, "f16", 4.0)
    scale = float(np.float32(d ** -0.5))
    got = ch.run_attend(_gpu(c), q, ch.starts([rows] * S), scale, "f16")
    ref = co.attend(c, q, ch.starts([rows] * S), scale)
    ch.check_attend(c, got, ref, "f16", L)


@pytest.mark.parametrize("format", FORMATS)
def test_what_is_not_finite_stays_where_it_is_seen(format):
    """Tokens that are NaN make NaN of the rows that see them, and of no others; infinite queries make NaN of theirs."""
    g = np.random.default_rng(11)
    lengths, rows = [200, 130], [6, 6]
    Hq, Hkv, d = 4, 2, 64
    c = ch.filled(g, lengths, Hkv, d, 64, format)
    i, at = c["table"][0, 197 // 64], 197 % 64                          # the fourth of the first sequence's rows
    c["kscale"][i, 0, at] = np.nan
    i, at = c["table"][1, 128 // 64], 128 % 64                          # the fifth of the second's
    c["vscale"][i, 1, at] = np.nan
    q = _queries(g, 12, Hq, d, "f16")
    q[1, 0, 3] = np.inf
    q[8, 3] = np.nan
    ref = co.attend(c, q, ch.starts(rows), 0.125)
    got = ch.run_attend(_gpu(c), q, ch.starts(rows), 0.125, "f16")
    nan = np.isnan(ref[0]).all(2)
    assert nan[3:6, :2].all() and not nan[2, :2].any() and nan[10:, 2:].all() and not nan[9].any() and nan[8, 3] and nan[1, 0]
    ch.check_attend(c, got, ref, "f16", 200)


def test_scores_of_any_size_and_values_of_any_scale():
    """Large scores (one key decides), a row whose scores are all -inf, values whose scales span 2^40, keys that rise all the way."""
    g = np.random.default_rng(12)
    Hq, Hkv, d, L = 4, 2, 64, 777
    c = ch.filled(g, [L, L, L], Hkv, d, 64, "i8", dtype="bf16")
    c["vscale"] = np.where(np.isfinite(c["vscale"]), c["vscale"] * 2.0 ** g.integers(-20, 21, c["vscale"].shape), c["vscale"]).astype(np.float32)
    q = _queries(g, 3, Hq, d, "bf16", 60.0)
    for n in range(L):                                                  # sequence 1: keys in the direction of the queries, ever longer
        i, at = c["table"][1, n // 64], n % 64
        code, _ = co.encode(q[1, ::2].astype(np.float32), "i8")
        c["k"][i, :, at], c["kscale"][i, :, at] = code, 0.002 * (1 + n)
    q[2, 0, :], q[2, 1, :] = 0.0, 0.0                                   # all scores equal
    got = ch.run_attend(_gpu(c), q, ch.starts([1, 1, 1]), 0.125, "bf16")
    ref = co.attend(c, q, ch.starts([1, 1, 1]), 0.125)
    ch.check_attend(c, got, ref, "bf16", L)
    # scores of -inf only: scales of keys that overflow
    c["kscale"][:] = 3e38
    c["k"][:] = 128 - 127
    q[:] = 60000.0
    got = ch.run_attend(_gpu(c), q, ch.starts([1, 1, 1]), 0.125, "bf16")
    assert not got.any()


def test_bad_pages_are_not_seen():
    g = np.random.default_rng(13)
    lengths = [300, 120, 64, 10 ** 6]
    Hq, Hkv, d = 4, 2, 64
    c = ch.filled(g, [300, 120, 64, 320], Hkv, d, 16, "e4m3")
    c["length"][3] = 10 ** 6                                            # taken as the table's width
    c["table"][0, 3], c["table"][0, 18], c["table"][1, 0] = -1, c["k"].shape[0], 2 ** 31 - 1
    c["table"][2, :] = -2 ** 31
    q = _queries(g, 4, Hq, d, "f16")
    row_start = np.array([0, 1, 2, 3, 900], np.int32)                   # beyond R
    got = ch.run_attend(_gpu(c), q, row_start, 0.125, "f16")
    ref = co.attend(c, q, row_start, 0.125)
    assert not ref[0][2].any()
    ch.check_attend(c, got, ref, "f16", 320)


# Sequences, KV heads, table in pages of 64, and lengths (drawn between the two, some of them the third): a workgroup a block of rows, cut or not;
# groups of wavefronts; a line that is cut; more sequences than a wavefront has lanes, than a workgroup has threads
SHARES = [
    (1, 1, 80, (5000, 5001), 5000), (3, 4, 16, (1, 1024), 900), (40, 8, 16, (1, 700), 1000), (40, 8, 160, (30, 600), 9000), (70, 1, 80, (1000, 5000), 17),
    (90, 3, 80, (40, 300), 5000), (200, 2, 16, (0, 1000), 0), (300, 2, 40, (0, 100), 2500), (520, 1, 24, (1, 200), 1500), (30, 32, 2, (1, 128), 128),
    (64, 16, 3, (1, 190), 64), (17, 16, 20, (200, 1280), 64),
]


@pytest.mark.parametrize("S,Hkv,width,between,some", SHARES)
@pytest.mark.parametrize("rows", [1, 3])
def test_every_way_to_share_out(S, Hkv, width, between, some, rows):
    g = np.random.default_rng([S, Hkv, rows])
    d, Hq = 64, 2 * Hkv
    lengths = [some if g.random() < 0.06 or b == S // 2 else int(g.integers(*between)) for b in range(S)]
    c = ch.filled(g, lengths, Hkv, d, 64, "i8", width=width)
    n = [0 if g.random() < 0.1 else rows for _ in range(S)]
    n[S // 2] = rows * 9 if rows > 1 else 1                              # more than a block of rows of one sequence
    R = sum(n)
    q = _queries(g, R, Hq, d, "f16", 3.0)
    scale = float(np.float32(d ** -0.5))
    got = ch.run_attend(_gpu(c), q, ch.starts(n), scale, "f16")
    ref = co.attend(c, q, ch.starts(n), scale)
    ch.check_attend(c, got, ref, "f16", max(lengths))


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (16, 16, 64)])
@pytest.mark.parametrize("listed", [False, True])
def test_tables_of_which_little_is_used(Hq, Hkv, d, format, listed):
    """Tables as wide as they may be (keys that may be more than any cache holds are read another way), short sequences in them."""
    g = np.random.default_rng([d, listed])
    lengths = [1500, 3, 400, 0, 65]
    c = ch.filled(g, lengths, Hkv, d, 64, format, wild=True)
    table = np.full((5, 4096), -1, np.int32)
    table[:, :c["table"].shape[1]] = c["table"]
    c["table"] = table
    blocks = None
    if listed:
        blocks = np.full((5, Hkv, 2000), -1, np.int32)
        blocks[0, :, :9], blocks[2, :, :3], blocks[4, :, 0] = [0, 2, 3, 5, 7, 11, 13, 17, 23], [0, 4, 6], 1
    q = _queries(g, 5, Hq, d, "f16")
    scale = float(np.float32(d ** -0.5))
    got = ch.run_attend(_gpu(c), q, ch.starts([1] * 5), scale, "f16", blocks=blocks)
    ch.check_attend(c, got, co.attend(c, q, ch.starts([1] * 5), scale, blocks=blocks), "f16", 1500)


@pytest.mark.parametrize("S", [64, 65, 256, 300, 700])
def test_many_sequences_write_and_attend(S):
    """As many sequences as a wavefront has lanes, as a workgroup has threads, and more; some without rows."""
    import torch
    g = np.random.default_rng(S)
    Hkv, Hq, d, page = 2, 4, 64, 16
    lengths = g.integers(0, 40, S)
    c = ch.filled(g, [int(n) for n in lengths], Hkv, d, page, "i8", width=5, shift=True)
    rows = g.integers(0, 4, S)
    c["length"] = (c["length"] + rows).astype(np.int32)
    R = int(rows.sum()) + 2
    k, v = (ch.rounded(g.standard_normal((R, Hkv, d)), "f16") for _ in range(2))
    q = _queries(g, R, Hq, d, "f16")
    gpu = _gpu(c)
    co.write(c, k, v, ch.starts(rows))
    _write(gpu, k, v, ch.starts(rows), "f16")
    _same_cache(gpu, c)
    blocks = np.full((S, Hkv, 3), -1, np.int32)
    for b in range(S):
        pages = min(3, -(-int(c["length"][b]) // page))
        blocks[b, :, :pages] = np.arange(pages)
    for chosen in (None, blocks):
        got = ch.run_attend(gpu, q, ch.starts(rows), 0.125, "f16", blocks=chosen)
        ch.check_attend(c, got, co.attend(c, q, ch.starts(rows), 0.125, blocks=chosen), "f16", 80)
    out = torch.empty((S, Hkv, 2), dtype=torch.int32, device="cuda:0")
    ws = torch.empty(P.pasa_cache_choose_workspace(gpu.cache), dtype=torch.uint8, device="cuda:0")
    tq, st = ch.tensor(q, "f16")
    c["kmean"] = gpu.back("kmean")
    P.pasa_cache_choose(gpu.cache, tq, R, st, ch.ints(ch.starts(rows)), Hq, out, 2, 0, 1, ws, ws.numel(), torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert np.array_equal(out.cpu().numpy(), co.choose(c, q, ch.starts(rows), 2, 0, 1))


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,d,rows", [(8, 2, 128, 1), (4, 4, 64, 1), (8, 2, 128, 7), (16, 4, 64, 5)])
def test_tokens_without_a_value_do_not_blur_the_others(Hq, Hkv, d, rows, format):
    """The first token, and a few others, have values of zeros (and so the scale 1) and half of the weight; the others' values are small."""
    g = np.random.default_rng([13, d, rows])
    L, S, page = 5000, 2, 64
    c = ch.filled(g, [0, 0], Hkv, d, page, format, width=-(-L // page))
    c["length"][:] = [L, 700]
    q = _queries(g, 1, Hq, d, "f16", 0.3).repeat(S * rows, 0)
    k, v = 0.3 * g.standard_normal((L + 700, Hkv, d)), 0.01 * (1 + 0.25 * g.standard_normal((L + 700, Hkv, d)))
    for n in (0, 77, 78, L, L + 699):
        v[n] = 0.0
    scale = float(np.float32(d ** -0.5))
    for n in (0, L):                                                    # a key whose scores are about log(L)
        for h in range(Hkv):
            t = q[0, h * Hq // Hkv:(h + 1) * Hq // Hkv].T
            k[n, h] = np.linalg.lstsq(t.T, np.full(t.shape[1], np.log(L) / scale), rcond=None)[0]
    co.write(c, ch.rounded(k, "f16"), ch.rounded(v, "f16"), np.array([0, L, L + 700], np.int32))
    zeros = c["vscale"] == 1.0
    assert zeros.any()
    ref = co.attend(c, q, ch.starts([rows] * S), scale)
    got = ch.run_attend(_gpu(c), q, ch.starts([rows] * S), scale, "f16")
    c["vscale"] = np.where(zeros, 0.0, c["vscale"]).astype(np.float32)       # no part of what a row's largest product may be
    ch.check_attend(c, got, ref, "f16", L)
    # nothing but such tokens: zeros
    c["vscale"] = np.ones_like(c["vscale"])
    c["v"][:] = 128 if format == "i8" else 0x80
    assert not ch.run_attend(_gpu(c), q, ch.starts([rows] * S), scale, "f16").any()


@pytest.mark.parametrize("share", [0.3, 0.5, 0.83])
@pytest.mark.parametrize("rows", [1, 9])
def test_many_keys_of_little_weight(rows, share):
    """One key has a share of the weight, 100000 others the rest, all alike, and values of one sign: what P's rounding takes from each adds up.  P keeps 2^-25 of
    a level that is at least 2^7 below the row's largest product."""
    g = np.random.default_rng([14, rows])
    L, Hq, Hkv, d, page = 100000, 2, 1, 64, 128
    c = ch.filled(g, [0], Hkv, d, page, "i8", width=-(-L // page))
    c["length"][:] = L
    q = ch.rounded(g.standard_normal((1, 1, d)), "f16").astype(np.float64).repeat(Hq, 1).repeat(rows, 0)
    k, v = np.zeros((L, Hkv, d)), 1 + 0.1 * g.standard_normal((L, Hkv, d))
    k[0] = q[0, 0] / (q[0, 0] @ q[0, 0]) * np.log(L * share / (1 - share)) / 0.125
    co.write(c, ch.rounded(k, "f16"), ch.rounded(v, "f16"), np.array([0, L], np.int32))
    ref = co.attend(c, q, ch.starts([rows]), 0.125)
    got = ch.run_attend(_gpu(c), q, ch.starts([rows]), 0.125, "f16")
    ch.check_attend(c, got, ref, "f16", L / 128)
