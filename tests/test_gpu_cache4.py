"""The paged cache in 4 bits on the GPU against the oracle: tokens in, tokens back, pages chosen, attention."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import cache4_oracle as c4
from oracle import cache_oracle as co
from tests import cache4_harness as h4
from tests import cache_harness as ch

pytestmark = pytest.mark.gpu


def _write(gpu, k, v, row_start, dtype, stride=None):
    import torch
    tk, st = ch.tensor(k, dtype, stride)
    tv, _ = ch.tensor(v, dtype, stride)
    P.pasa_cache_write(gpu.cache, tk, tv, len(k), st, ch.ints(row_start), torch.cuda.current_stream(), io_dtype=ch.IO[dtype])
    torch.cuda.synchronize()


def _same_cache(gpu, c):
    """Codes, factors and scales bit for bit, means to their last bits."""
    for n in ("k", "v"):
        assert np.array_equal(gpu.back(n + "scale"), c[n + "scale"], equal_nan=True)
        assert np.array_equal(gpu.back(n), c[n])
    if c["kmean"] is not None:
        # a product and an addition a token in fp32 (128 tokens at most), and the quotient
        m = gpu.back("kmean")
        assert np.array_equal(np.isnan(m), np.isnan(c["kmean"]))
        with np.errstate(invalid="ignore"):
            x = np.abs(co.values(c4.numbers(c, "k"), c["kscale"], "i4"))
            wide = np.where(np.isnan(x), 0.0, x).max(axis=2)
            assert not (np.abs(m.astype(np.float64) - c["kmean"]) > 132 * 2.0 ** -24 * wide).any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,Hkv,page", [(128, 4, 64), (64, 5, 16), (128, 1, 128), (64, 2, 32)])
def test_tokens_enter_in_steps(d, Hkv, page, dtype):
    """Prompts, single tokens, none, and a step that is taken back; sequences without tokens; rows behind the last sequence; strides."""
    g = np.random.default_rng([d, page])
    S, width = 4, 5
    c = h4.empty(g, S, Hkv, d, page, width, shift=page != 16, mean=page != 128)
    gpu = h4.OnGpu(c)
    for step, (length, rows, behind) in enumerate([
        ([2 * page + 3, 1, 0, page], [2 * page + 3, 1, 0, page], 2),
        ([2 * page + 4, 2, 1, page + 1], [1, 1, 1, 1], 0),
        ([2 * page + 4, 2 + page, 1, 3 * page], [0, page, 0, 2 * page - 1], 1),
        ([2 * page + 1, 3, 2, 3 * page - 2], [2, 1, 1, 5], 0),             # shorter than before: what was behind is overwritten
    ]):
        R = sum(rows) + behind
        k = g.standard_normal((R, Hkv, d)) * 2.0 ** g.integers(-12, 8, (R, Hkv, 1)) * np.repeat(2.0 ** g.integers(-9, 1, (R, Hkv, d // 32)), 32, 2)
        v = g.standard_normal((R, Hkv, d)) * 2.0 ** g.integers(-12, 8, (R, Hkv, 1)) * np.repeat(2.0 ** g.integers(-9, 1, (R, Hkv, d // 32)), 32, 2)
        k, v = ch.rounded(k, dtype), ch.rounded(v, dtype)
        k[0, 0], v[R - 1, 0] = 0.0, 0.0
        c["length"][:] = length
        gpu.t["length"].copy_(ch.ints(length))
        c4.write(c, k, v, ch.starts(rows))
        _write(gpu, k, v, ch.starts(rows), dtype, None if step % 2 else (Hkv + 3) * d + 8)
        _same_cache(gpu, c)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_tie_and_border(dtype):
    """Values that are halves of steps, groups whose largest is half of a step of the factor, and largest values around those where a scale is just met."""
    g = np.random.default_rng(5)
    x = []
    for i in range(1500):
        s = 2.0 ** int(g.integers(-20, 5)) * int(g.integers(128, 256)) / 128           # a scale
        m = [int(g.integers(1, 225)), int(g.choice([1, 2, 223, 224, 100]))]
        row = np.concatenate([g.integers(-15, 16, 32) / 2 * f * s for f in m])
        row[0] = 1568 * s * (1 if i % 3 == 0 else 1 - 2.0 ** -int(g.integers(7, 20)) if i % 3 == 1 else 1 + 2.0 ** -int(g.integers(7, 12)))
        if i % 2:
            row[32] = (m[1] + 0.5) * 7 * s
        x.append(row)
    x = ch.rounded(np.array(x), dtype)
    n = len(x)
    c = h4.empty(g, 1, 1, 64, 128, -(-n // 128), mean=False)
    c["length"][:] = n
    gpu = h4.OnGpu(c)
    k, v = x[:, None], np.ascontiguousarray(x[::-1, None])
    c4.write(c, k, v, ch.starts([n]))
    _write(gpu, k, v, ch.starts([n]), dtype)
    _same_cache(gpu, c)


def test_values_that_are_not_finite_and_the_smallest_and_largest():
    """A token that holds one gets the scale NaN and codes of zero; other tokens and heads keep theirs."""
    g = np.random.default_rng(6)
    c = h4.empty(g, 2, 2, 64, 16, 2, shift=True)
    n = [20, 7]
    c["length"][:] = n
    k, v = (ch.rounded(g.standard_normal((27, 2, 64)), "bf16") for _ in range(2))
    k[3, 1, 5], k[4, 0, 63], v[9, 1, 0], v[26, 0, 8] = np.nan, np.inf, -np.inf, np.nan
    v[10, 0] = ch.rounded(np.full(64, 2.0 ** -99), "bf16")               # below what a scale is made for: rounds to zero
    v[11, 0] = ch.rounded(np.linspace(-1, 1, 64) * 2.0 ** -97, "bf16")
    v[12, 1] = ch.rounded(np.linspace(-1, 1, 64) * 2.0 ** 127, "bf16")
    v[13, 1] = 3.3895313892515355e38                                      # the largest of the type
    v[14, 0], v[14, 0, 3] = 0.0, 2.0 ** -98
    gpu = h4.OnGpu(c)
    c4.write(c, k, v, ch.starts(n))
    _write(gpu, k, v, ch.starts(n), "bf16")
    _same_cache(gpu, c)
    assert (gpu.back("k")[c["table"][0, 0], 1, 3 * 32:4 * 32] == 0x88).all()


def test_tokens_without_a_page_are_dropped_and_nothing_else_is_touched():
    """Table entries outside the pool, lengths and row numbers beyond their range, rows before position 0."""
    g = np.random.default_rng(7)
    c = h4.empty(g, 4, 2, 64, 16, 3)
    c["table"][0, 1], c["table"][1, 0], c["table"][2, 2] = -5, 1 << 30, c["k"].shape[0]
    c["length"][:] = [40, 20, 1000, 2]
    rows = ch.starts([30, 20, 48, 5])
    rows[4] = 5000                                                        # beyond R
    R = 103
    k, v = (ch.rounded(g.standard_normal((R, 2, 64)), "f16") for _ in range(2))
    gpu = h4.OnGpu(c)
    c4.write(c, k, v, rows)
    _write(gpu, k, v, rows, "f16")
    _same_cache(gpu, c)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,page,N", [(128, 64, 1), (64, 16, 200), (128, 32, 300), (64, 128, 129)])
def test_tokens_come_back(d, page, N, dtype):
    import torch
    g = np.random.default_rng([d, N])
    c = h4.filled(g, [300, 1, 0, 170], 3, d, page, dtype, shift=N != 300, wild=True)
    c["table"][3, 0] = c["k"].shape[0] + 3
    gpu = h4.OnGpu(c)
    n = 4 * 3 * N * d
    for first in (None, [0, 0, 0, 0], [299, -1, 5, 100], [-3, 2, 0, 2 ** 31 - 1]):
        out = [torch.full((n + 1024,), float("nan"), dtype=torch.float16 if dtype == "f16" else torch.bfloat16, device="cuda:0") for _ in range(2)]
        P.pasa_cache_read(gpu.cache, out[0], out[1], None if first is None else ch.ints(first), N, torch.cuda.current_stream(), io_dtype=ch.IO[dtype])
        torch.cuda.synchronize()
        for t, want, shift in zip(out, co.read(c4.plain(c), first, N), (c["kshift"], None)):
            assert bool(torch.isnan(t[n:]).all())
            got = t[:n].view(4, 3, N, d).double().cpu().numpy()
            # a value has 19 bits; the sum with the shift is rounded to fp32, then to the type
            extra = 0 if shift is None else 2.0 ** -24 * np.abs(want)
            assert not (np.abs(got - want) > ch.HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -20) + ch.TINY[dtype] + extra).any() and np.isfinite(got).all()


def test_large_outputs_come_back_past_the_caches():
    """More than 32 MiB of output, which is stored another way."""
    import torch
    g = np.random.default_rng(8)
    Hkv, d, page, N, S = 4, 128, 128, 4200, 4
    c = h4.filled(g, [100, 256, 0, 7], Hkv, d, page)
    table = np.full((S, 40), -1, np.int32)
    table[:, :c["table"].shape[1]] = c["table"]
    c["table"] = table
    gpu = h4.OnGpu(c)
    out = [torch.full((S, Hkv, N, d), float("nan"), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    P.pasa_cache_read(gpu.cache, out[0], out[1], None, N, torch.cuda.current_stream(), io_dtype=P.IO_BF16)
    for t, want in zip(out, co.read(c4.plain(c), None, 256)):
        got = t[:, :, :256].double().cpu().numpy()
        assert not (np.abs(got - want) > 2.0 ** -8 * np.abs(want)).any() and not bool(t[:, :, 256:].any())


@pytest.mark.parametrize("d,Hq,Hkv,page,count", [(128, 28, 4, 64, 8), (64, 5, 5, 16, 40)])
def test_pages_are_chosen(d, Hq, Hkv, page, count):
    import torch
    g = np.random.default_rng([d, Hq, page])
    lengths, rows = [1500, 7, 0, page * count], [3, 1, 1, 2]
    c = h4.filled(g, [min(n, 1500) for n in lengths], Hkv, d, page)
    q = ch.rounded(g.standard_normal((7, Hq, d)), "f16").astype(np.float64)
    gpu = h4.OnGpu(c)
    need = P.pasa_cache_choose_workspace(gpu.cache)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda:0")
    out = torch.full((4, Hkv, count), -7, dtype=torch.int32, device="cuda:0")
    tq, st = ch.tensor(q, "f16")
    P.pasa_cache_choose(gpu.cache, tq, 7, st, ch.ints(ch.starts(rows)), Hq, out, count, 1, 1, ws, need, torch.cuda.current_stream())
    want = co.choose({**c4.plain(c)}, q, ch.starts(rows), count, 1, 1)
    assert np.array_equal(out.cpu().numpy(), want)


def _queries(g, R, Hq, d, dtype, size=1.5):
    return ch.rounded(size * g.standard_normal((R, Hq, d)), dtype).astype(np.float64)


def _attend(c, q, row_start, scale, dtype, **kw):
    got = ch.run_attend(h4.OnGpu(c), q, row_start, scale, dtype, **kw)
    kw.pop("stride", None)
    ref = h4.attend(c, q, row_start, scale, dtype, **kw)
    h4.check(got, ref)
    return got, ref


LAYOUTS = [(28, 4, 128), (5, 5, 64), (8, 1, 128), (16, 2, 64), (3, 1, 64), (40, 1, 128)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", LAYOUTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_a_decoding_step(page, Hq, Hkv, d, dtype):
    """One row per sequence; lengths from nothing to several units of work, around their borders."""
    g = np.random.default_rng([page, Hq, d])
    lengths = [1, 0, 63, 64, 65, 700, 128, 1345]
    c = h4.filled(g, lengths, Hkv, d, page, dtype, shift=page == 64, wild=True)
    q = _queries(g, len(lengths), Hq, d, dtype)
    _, ref = _attend(c, q, ch.starts([1] * len(lengths)), float(np.float32(d ** -0.5)), dtype)
    assert not ref[0][1].any()


@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (16, 16, 64), (4, 4, 128)])
@pytest.mark.parametrize("tree", [False, True])
def test_chains_and_trees(Hq, Hkv, d, tree):
    """Rows per sequence from none to 64 (chains: more), sequences that consist of nothing else, rows before position 0, rows behind the last sequence."""
    g = np.random.default_rng([Hq, d, tree])
    lengths, rows = [300, 64, 5, 90, 1, 200], [7, 64, 9, 0, 1, 40 if tree else 90]
    c = h4.filled(g, lengths, Hkv, d, 32, wild=True)
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
    got, _ = _attend(c, q, ch.starts(rows), float(np.float32(d ** -0.5)), "f16", tree=bits, stride=(Hq + 2 * Hkv) * d)
    assert np.isnan(got[-3:]).all()


@pytest.mark.parametrize("page,count", [(16, 9), (64, 4), (128, 2), (32, 100)])
@pytest.mark.parametrize("rows", [1, 5])
def test_only_chosen_pages_are_seen(page, count, rows):
    g = np.random.default_rng([page, rows])
    lengths = [900, 33, 0, 640, 1000]
    Hq, Hkv, d = 12, 2, 128
    c = h4.filled(g, lengths, Hkv, d, page, wild=True)
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
    _attend(c, q, ch.starts([rows] * 5), float(np.float32(d ** -0.5)), "f16", blocks=blocks)


@pytest.mark.parametrize("S,L,Hq,Hkv,d,rows", [(1, 4999, 28, 4, 128, 1), (1, 20000, 8, 1, 64, 1), (2, 5000, 4, 2, 128, 20), (40, 500, 5, 5, 64, 1),
                                               (300, 90, 2, 1, 64, 1), (520, 40, 2, 1, 128, 1)])
def test_work_that_many_workgroups_share(S, L, Hq, Hkv, d, rows):
    """Long sequences are swept by several workgroups, many short ones by few; a workgroup's range crosses sequences."""
    g = np.random.default_rng([S, L])
    lengths = [L] + [int(n) for n in g.integers(0 if S > 10 else L // 2, L + 1, S - 1)]
    c = h4.filled(g, lengths, Hkv, d, 64)
    q = _queries(g, S * rows, Hq, d, "f16", 4.0)
    _attend(c, q, ch.starts([rows] * S), float(np.float32(d ** -0.5)), "f16")


def test_what_is_not_finite_stays_where_it_is_seen():
    """Tokens that are NaN make NaN of the rows that see them, and of no others; infinite queries make NaN of theirs."""
    g = np.random.default_rng(11)
    lengths, rows = [200, 130], [6, 6]
    Hq, Hkv, d = 4, 2, 64
    c = h4.filled(g, lengths, Hkv, d, 64)
    i, at = c["table"][0, 197 // 64], 197 % 64                          # the fourth of the first sequence's rows
    c["kscale"][i, 0, at] = np.nan
    i, at = c["table"][1, 128 // 64], 128 % 64                          # the fifth of the second's
    c["vscale"][i, 1, at] = np.nan
    q = _queries(g, 12, Hq, d, "f16")
    q[1, 0, 3] = np.inf
    q[8, 3] = np.nan
    ref = co.attend(c4.plain(c), q, ch.starts(rows), 0.125)[0]
    got = ch.run_attend(h4.OnGpu(c), q, ch.starts(rows), 0.125, "f16")
    nan = np.isnan(ref).all(2)
    assert nan[3:6, :2].all() and not nan[2, :2].any() and nan[10:, 2:].all() and not nan[9].any() and nan[8, 3] and nan[1, 0]
    assert np.array_equal(np.isnan(got), np.isnan(ref))


@pytest.mark.parametrize("d", [64, 128])
def test_tokens_whose_value_is_zero_and_scores_of_any_size(d):
    """A first token without a value that has most of the weight; large scores; rows whose scores are all equal."""
    g = np.random.default_rng([12, d])
    Hq, Hkv, L = 4, 2, 333
    c = h4.filled(g, [L, L, L], Hkv, d, 64, dtype="bf16")
    q = _queries(g, 3, Hq, d, "bf16", 30.0)
    q[2, 0, :], q[2, 1, :] = 0.0, 0.0
    i = c["table"][0, 0]
    for h in range(Hkv):
        code, factor, scale = c4.encode(ch.rounded(q[0, 2 * h] / 8, "bf16"))
        c4.put(c, "k", i, h, 0, code, factor)
        c["kscale"][i, h, 0] = scale
        c4.put(c, "v", i, h, 0, np.zeros(d, np.int8), np.ones(d // 32, np.uint8))
        c["vscale"][i, h, 0] = 1.0
    _attend(c, q, ch.starts([1, 1, 1]), 0.125, "bf16")


def test_values_of_any_scale():
    """The least scales that tokens may have, and the largest, each in a sequence of its own."""
    g = np.random.default_rng(14)
    Hq, Hkv, d, L = 4, 2, 64, 300
    c = h4.filled(g, [L, L], Hkv, d, 64)
    for b, e in ((0, -108), (1, 116)):
        ids = c["table"][b]
        c["vscale"][ids] = np.where(np.isfinite(c["vscale"][ids]), 2.0 ** e, c["vscale"][ids]).astype(np.float32)
    q = _queries(g, 2, Hq, d, "bf16")
    _attend(c, q, ch.starts([1, 1]), 0.125, "bf16")


@pytest.mark.parametrize("d", [64, 128])
def test_keys_of_any_scale(d):
    """Scales of keys up to the largest that tokens may have: queries of zero see them all alike, small ones choose by them."""
    g = np.random.default_rng([16, d])
    Hq, Hkv, L = 4, 2, 200
    c = h4.filled(g, [L, L, L], Hkv, d, 64)
    q = _queries(g, 3, Hq, d, "bf16")
    q[1], q[2] = 0.0, ch.rounded(q[2] * 2.0 ** -24, "f16")
    for b in (1, 2):
        for n in range(0, L, 7):
            c["kscale"][c["table"][b, n // 64], :, n % 64] = 2.0 ** int(g.integers(100, 118))
    scale = float(np.float32(d ** -0.5))
    got = ch.run_attend(h4.OnGpu(c), q, ch.starts([1, 1, 1]), scale, "f16")
    assert np.isfinite(got).all()
    o, bound = h4.attend(c, q, ch.starts([1, 1, 1]), scale, "f16")
    h4.check(got[:2], (o[:2], bound[:2]))
    # the third: scores of 2^80 and more, of which one key has the largest by far more than their rounding; its value is the output
    for h in range(Hq):
        x = np.concatenate([(co.values(c4.numbers(c, "k")[i, h // 2], c["kscale"][i, h // 2], "i4") @ q[2, h])[:min(64, L - 64 * j)] for j, i in enumerate(c["table"][2])]) * scale
        top, second = np.sort(x)[::-1][:2]
        assert top > second * (1 + 2.0 ** -12) and top > 2.0 ** 60
        n = int(np.argmax(x))
        v = co.values(c4.numbers(c, "v")[c["table"][2, n // 64], h // 2, n % 64], c["vscale"][c["table"][2, n // 64], h // 2, n % 64], "i4")
        assert (np.abs(got[2, h] - v) <= 2.0 ** -10 * np.abs(v) + 2.0 ** -24).all()


def test_bad_pages_are_not_seen():
    g = np.random.default_rng(13)
    Hq, Hkv, d = 4, 2, 64
    c = h4.filled(g, [300, 120, 64, 320], Hkv, d, 16)
    c["length"][3] = 10 ** 6                                            # taken as the table's width
    c["table"][0, 3], c["table"][0, 18], c["table"][1, 0] = -1, c["k"].shape[0], 2 ** 31 - 1
    c["table"][2, :] = -2 ** 31
    q = _queries(g, 4, Hq, d, "f16")
    _, ref = _attend(c, q, np.array([0, 1, 2, 3, 900], np.int32), 0.125, "f16")          # beyond R
    assert not ref[0][2].any()


# as in the tests of 8 bits: a workgroup a block of rows, cut or not; groups of wavefronts; a line that is cut
SHARES = [
    (1, 1, 80, (5000, 5001), 5000), (3, 4, 16, (1, 1024), 900), (40, 8, 160, (30, 300), 3000), (70, 1, 80, (1000, 2000), 17), (200, 2, 16, (0, 300), 0),
    (30, 32, 2, (1, 128), 128),
]


@pytest.mark.parametrize("S,Hkv,width,between,some", SHARES)
@pytest.mark.parametrize("rows", [1, 3])
def test_every_way_to_share_out(S, Hkv, width, between, some, rows):
    g = np.random.default_rng([S, Hkv, rows])
    d, Hq = 64, 2 * Hkv
    lengths = [some if g.random() < 0.06 or b == S // 2 else int(g.integers(*between)) for b in range(S)]
    c = h4.filled(g, lengths, Hkv, d, 64, width=width, mean=False)
    n = [0 if g.random() < 0.1 else rows for _ in range(S)]
    n[S // 2] = rows * 9 if rows > 1 else 1                              # more than a block of rows of one sequence
    q = _queries(g, sum(n), Hq, d, "f16", 3.0)
    _attend(c, q, ch.starts(n), float(np.float32(d ** -0.5)), "f16")


@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (16, 16, 64)])
@pytest.mark.parametrize("listed", [False, True])
def test_tables_of_which_little_is_used(Hq, Hkv, d, listed):
    """Tables as wide as they may be (keys that may be more than any cache holds are read another way), short sequences in them."""
    g = np.random.default_rng([d, listed])
    lengths = [1500, 3, 400, 0, 65]
    c = h4.filled(g, lengths, Hkv, d, 64, wild=True)
    table = np.full((5, 4096), -1, np.int32)
    table[:, :c["table"].shape[1]] = c["table"]
    c["table"] = table
    blocks = None
    if listed:
        blocks = np.full((5, Hkv, 2000), -1, np.int32)
        blocks[0, :, :9], blocks[2, :, :3], blocks[4, :, 0] = [0, 2, 3, 5, 7, 11, 13, 17, 23], [0, 4, 6], 1
    q = _queries(g, 5, Hq, d, "f16")
    _attend(c, q, ch.starts([1] * 5), float(np.float32(d ** -0.5)), "f16", blocks=blocks)


def test_pools_beyond_4_GiB():
    """Pages whose codes lie more than 2^32 bytes into the pool."""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = np.random.default_rng(15)
    Hq, Hkv, d, page = 8, 8, 128, 128
    c = h4.filled(g, [200, 90], Hkv, d, page, mean=False)
    raw = c["k"].shape[2]
    pages = (1 << 32) // (Hkv * raw) + 60
    table = np.full((2, 2), -1, np.int64)
    gpu = h4.OnGpu(c)
    big = {n: torch.zeros((pages,) + tuple(gpu.t[n].shape[1:]), dtype=gpu.t[n].dtype, device="cuda:0") for n in ("k", "v", "kscale", "vscale")}
    for b in range(2):
        for p in range(-(-int(c["length"][b]) // page)):
            table[b, p] = pages - 1 - 7 * b - 3 * p
            for n in big:
                big[n][int(table[b, p])] = gpu.t[n][int(c["table"][b, p])]
    gpu.t["table"].copy_(torch.from_numpy(table.astype(np.int32)))
    gpu.cache = P.pasa_cache(big["k"], big["v"], big["kscale"], big["vscale"], gpu.t["table"], gpu.t["length"], S=2, Hkv=Hkv, d=d, page=page, pages=pages,
                             table_width=2, format=P.CACHE_I4)
    q = _queries(g, 2, Hq, d, "f16")
    got = ch.run_attend(gpu, q, ch.starts([1, 1]), 0.088388346, "f16")
    h4.check(got, h4.attend(c, q, ch.starts([1, 1]), 0.088388346, "f16"))
    out = [torch.empty((2, Hkv, 200, d), dtype=torch.float16, device="cuda:0") for _ in range(2)]
    P.pasa_cache_read(gpu.cache, out[0], out[1], None, 200, torch.cuda.current_stream())
    want = co.read(c4.plain(c), None, 200)
    for t, w in zip(out, want):
        assert not (np.abs(t.double().cpu().numpy() - w) > 2.0 ** -11 * np.abs(w) + 2.0 ** -25).any()
    # a token written there, and read back
    k, v = (ch.rounded(g.standard_normal((2, Hkv, d)), "f16") for _ in range(2))
    _write(gpu, k, v, ch.starts([1, 1]), "f16")
    c4.write(c, k, v, ch.starts([1, 1]))
    for b in range(2):
        p = (int(c["length"][b]) - 1) // page
        for n in ("k", "v"):
            assert np.array_equal(big[n][int(table[b, p])].cpu().numpy(), c[n][int(c["table"][b, p])])
