"""The calls that share, give out, take back and pack the pages of a cache, on the GPU against the oracle: everything that they write has to be equal."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import pages_oracle as po
from tests import cache_harness as ch
from tests import pages_harness as ph

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("format", ["i8", "e4m3", "i4"])
@pytest.mark.parametrize("Hkv,d,page,mean", [(4, 128, 64, True), (1, 64, 16, False), (5, 64, 32, True), (3, 128, 128, False)])
def test_pages_are_copied_between_pools(Hkv, d, page, mean, format):
    import torch
    g = np.random.default_rng([Hkv, d, page])
    a, b = (ph.pool(g, 1, Hkv, d, page, 1, pages, format, mean) for pages in (40, 23))
    ga, gb = ph.OnGpu(a), ph.OnGpu(b)
    of, to = g.permutation(40)[:15], g.permutation(23)[:15]
    of[3], to[5], of[7], to[8] = -1, 23, 40, -2 ** 31                     # outside: passed over
    P.pasa_cache_copy(gb.c, ga.c, ch.ints(to), ch.ints(of), 15, torch.cuda.current_stream())
    po.copy(b, a, to, of)
    gb.same(b)
    ga.same(a)
    # within a pool
    of, to = np.split(g.permutation(40)[:30], 2)
    P.pasa_cache_copy(ga.c, ga.c, ch.ints(to), ch.ints(of), 15, torch.cuda.current_stream())
    po.copy(a, a, to, of)
    ga.same(a)


def test_a_pool_without_means_takes_pages_of_one_with():
    import torch
    g = np.random.default_rng(2)
    a, b = ph.pool(g, 1, 2, 64, 16, 1, 9), ph.pool(g, 1, 2, 64, 16, 1, 9, mean=False)
    ga, gb = ph.OnGpu(a), ph.OnGpu(b)
    P.pasa_cache_copy(gb.c, ga.c, ch.ints([1, 8]), ch.ints([0, 3]), 2, torch.cuda.current_stream())
    po.copy(b, a, [1, 8], [0, 3])
    gb.same(b)


@pytest.mark.parametrize("S,width,page", [(5, 7, 16), (1, 1, 128), (64, 40, 32), (300, 3, 16), (7, 700, 16), (1500, 2, 16), (64, 128, 16), (40, 300, 16),
                                          (9000, 1, 16)])
def test_sequences_go_on_as_others(S, width, page):
    g = np.random.default_rng([S, width])
    c = ph.pool(g, S, 1, 64, page, width, S * width + 3, mean=False)
    lengths = g.integers(0, width * page + 1, S)
    lengths[0], lengths[-1] = width * page, 0
    ph.hold(g, c, lengths, 0.5)
    c["table"][S // 2, width - 1] = 2 ** 30 if c["table"][S // 2, width - 1] < 0 else c["table"][S // 2, width - 1]
    for b in (0, S // 4):                                                 # entries that hold nothing go on as they are
        i = (c["length"][b] + page - 1) // page // 2
        if S > 4 and i < width and c["table"][b, i] >= 0:
            c["table"][b, i] = -5
    c["refs"][:] = po.counts(c)
    gpu = ph.OnGpu(c)
    for source in (np.arange(S), np.roll(np.arange(S), 1), g.integers(0, S, S), np.where(g.random(S) < 0.3, -1, np.arange(S)),
                   g.integers(-2, S + 2, S), np.full(S, S // 3), np.full(S, 2 ** 31 - 1)):
        po.fork(c, source)
        gpu.fork(source)
        gpu.same(c)
        assert np.array_equal(c["refs"], po.counts(c))


def test_lengths_beyond_the_table_are_taken_as_its_end():
    g = np.random.default_rng(4)
    c = ph.pool(g, 4, 1, 64, 16, 3, 20, mean=False)
    ph.hold(g, c, [48, 10, 30, 48])
    c["length"][:] = [10 ** 6, -3, 30, 48]
    gpu = ph.OnGpu(c)
    for source in ([0, 0, 1, 3], [3, 1, 0, 1]):
        po.fork(c, source)
        gpu.fork(source)
        gpu.same(c)
    c["length"][:] = [-1, 10 ** 6, 17, 16]
    gpu.t["length"].copy_(ch.ints(c["length"]))
    po.free(c)
    gpu.free()
    gpu.same(c)


@pytest.mark.parametrize("S,width,page", [(6, 9, 16), (64, 5, 64), (2, 4000, 16), (1100, 2, 128)])
def test_pages_behind_the_lengths_are_let_go(S, width, page):
    g = np.random.default_rng([S, width])
    c = ph.pool(g, S, 1, 64, page, width, S * width + 2, mean=False)
    ph.hold(g, c, g.integers(0, width * page + 1, S), 0.4)
    c["length"] = g.integers(0, c["length"] + 1).astype(np.int32)
    c["length"][0] = 0
    gpu = ph.OnGpu(c)
    po.free(c)
    gpu.free()
    gpu.same(c)
    assert np.array_equal(c["refs"], po.counts(c))


@pytest.mark.parametrize("format,mean", [("i4", True), ("i8", False)])
@pytest.mark.parametrize("S,Hkv,d,page,width", [(5, 2, 64, 16, 6), (40, 4, 128, 64, 3), (1, 1, 128, 128, 2), (300, 1, 64, 32, 3)])
def test_rows_get_pages_of_their_own(S, Hkv, d, page, width, format, mean):
    """Steps, prompts, none; beams that go on from one page, all of them or not; a sequence that was taken back into what others hold."""
    g = np.random.default_rng([S, d, page])
    c = ph.pool(g, S, Hkv, d, page, width, S * width + 5, format, mean)
    gpu = ph.OnGpu(c)

    def step(n):
        n = np.minimum(n, width * page - c["length"])
        rows = ch.starts(n)
        c["length"] += n.astype(np.int32)
        gpu.t["length"].copy_(ch.ints(c["length"]))
        R = int(rows[-1]) + 3
        assert gpu.room(rows, R) == po.room(c, rows, R) == 0
        gpu.same(c)

    step(g.integers(0, page * (width - 1), S))
    step(np.ones(S, np.int64))
    for turn in range(4):
        source = g.integers(0, S, S) if turn % 2 else np.arange(S) // 4 * 4
        po.fork(c, source)
        gpu.fork(source)
        if turn == 2:
            c["length"] = np.maximum(0, c["length"] - g.integers(0, page + 3, S)).astype(np.int32)        # back into what is shared
        step(np.where(g.random(S) < 0.8, 1, 0))
        step(g.integers(0, page + 2, S))
    assert np.array_equal(c["refs"], po.counts(c))


def test_prompts_of_many_pages_and_many_sequences():
    """More places than the workgroup has threads; more sequences than that."""
    g = np.random.default_rng(8)
    for S, width, lengths in ((3, 3000, [3000 * 16, 0, 1500 * 16 + 1]), (2100, 3, g.integers(0, 49, 2100))):
        c = ph.pool(g, S, 1, 64, 16, width, int(sum(-(-n // 16) for n in lengths)) + 40, mean=False)
        gpu = ph.OnGpu(c)
        c["refs"][g.permutation(len(c["refs"]))[:30]] = 2                 # held by somebody else
        gpu.t["refs"].copy_(ch.ints(c["refs"]))
        c["length"] += np.array(lengths, np.int32)
        gpu.t["length"].copy_(ch.ints(c["length"]))
        rows = ch.starts(lengths)
        assert gpu.room(rows, int(rows[-1])) == po.room(c, rows, int(rows[-1])) == 0
        gpu.same(c)


@pytest.mark.parametrize("pages", [1, 3, 5, 16, 17, 16383, 16384, 16385, 40001])
def test_the_lowest_free_pages_are_found_wherever_they_are(pages):
    g = np.random.default_rng(pages)
    S, width = 6, 4
    c = ph.pool(g, S, 1, 64, 16, width, pages, mean=False)
    c["refs"][:] = 1
    free = g.permutation(pages)[:11]
    free = np.union1d(free, [pages - 1])
    c["refs"][free] = 0
    gpu = ph.OnGpu(c)
    n = np.array([33, 1, 0, 16, 47, 17])                                  # 3 + 1 + 1 + 3 + 2 = 10 places
    c["length"] += n.astype(np.int32)
    gpu.t["length"].copy_(ch.ints(c["length"]))
    lacking = po.room(c, ch.starts(n), int(n.sum()))
    assert gpu.room(ch.starts(n), int(n.sum())) == lacking == max(0, 10 - len(free))
    gpu.same(c)


def test_where_no_page_is_left():
    """Places without a page count and are without; what was shared is let go of, so that nobody writes to it; row numbers beyond their range."""
    g = np.random.default_rng(9)
    c = ph.pool(g, 5, 1, 64, 16, 4, 9, mean=False)
    ph.hold(g, c, [20, 20, 20, 16, 0])
    gpu = ph.OnGpu(c)
    po.fork(c, [0, 0, 0, 3, 3])
    gpu.fork([0, 0, 0, 3, 3])
    c["refs"][(c["refs"] == 0) & (np.cumsum(c["refs"] == 0) > 2)] = 1     # two free ones are left
    gpu.t["refs"].copy_(ch.ints(c["refs"]))
    c["length"] += 3
    gpu.t["length"].copy_(ch.ints(c["length"]))
    rows = [0, 3, 6, 9, 12, 900]
    assert gpu.room(rows, 15) == po.room(c, rows, 15) == 2
    gpu.same(c)
    assert (c["table"][2, 1] >= 0) and c["table"][3, 1] == c["table"][4, 1] == -1
    c["length"][:] = [10 ** 6, 5, 2, -4, 64]
    gpu.t["length"].copy_(ch.ints(c["length"]))
    rows = [-5, 2, 2, 15, 15, 15]
    assert gpu.room(rows, 15) == po.room(c, rows, 15)
    gpu.same(c)


def test_holders_that_are_not_the_counts_harm_nothing_else():
    """Whatever refs, tables and row numbers hold: the calls end, keep to the buffers and leave no page number outside the pool."""
    import torch
    g = np.random.default_rng(10)
    for seed in range(6):
        c = ph.pool(g, 9, 1, 64, 16, 5, 30, mean=False)
        c["table"] = g.integers(-3, 33, c["table"].shape).astype(np.int32)
        c["refs"] = g.integers(-4, 4, 30).astype(np.int32)
        c["length"] = g.integers(-9, 100, 9).astype(np.int32)
        gpu = ph.OnGpu(c)
        rows = g.integers(-5, 60, 10)
        gpu.room(rows, 50)
        gpu.fork(g.integers(-3, 12, 9))
        gpu.free()
        gpu.compact()
        table = gpu.t["table"].cpu().numpy()
        assert ((table < 30) | np.isin(table, c["table"])).all()
        assert bool(torch.isfinite(gpu.t["kscale"]).all())


@pytest.mark.parametrize("format,mean", [("i4", True), ("e4m3", False)])
@pytest.mark.parametrize("pages,live", [(1, 0), (1, 1), (40, 17), (40, 0), (40, 40), (1000, 999), (1000, 1), (16384, 16384), (16384, 8000), (16385, 16384), (33000, 20000), (50000, 16384),
                                        (50000, 40000)])
def test_a_pool_is_packed(pages, live, format, mean):
    g = np.random.default_rng([pages, live])
    S = 4
    width = max(1, -(-live // S) + 2)
    c = ph.pool(g, S, 1, 64, 16, width, pages, format, mean and pages < 20000)
    held = g.permutation(pages)[:live]
    if live == 8000:
        held = np.arange(pages)[-live:]                                  # all of them move
    for i, p in enumerate(held):
        c["table"][i % S, i // S] = p
    if live > 10:
        c["table"][3, -1], c["table"][2, -1] = c["table"][0, 0], 2 ** 31 - 1                # held twice; outside
    c["refs"][:] = po.counts(c)
    gpu = ph.OnGpu(c)
    for again in range(2):
        assert gpu.compact() == po.compact(c) == live
        gpu.same(c)
        assert (c["refs"][:live] != 0).all() and not c["refs"][live:].any()


def test_pages_that_are_held_outside_the_tables_move_too():
    """A count above what the tables hold (another table of the caller's) keeps a page in use; entries without a count stay."""
    g = np.random.default_rng(12)
    c = ph.pool(g, 2, 2, 64, 16, 4, 30)
    ph.hold(g, c, [50, 33])
    c["refs"][29] += 1
    c["table"][1, 3] = 28 if c["refs"][28] == 0 else 27
    c["refs"][c["table"][1, 3]] = 0
    gpu = ph.OnGpu(c)
    assert gpu.compact() == po.compact(c)
    gpu.same(c)


def test_pools_beyond_4_GiB():
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    Hkv, d, page = 8, 128, 128
    raw = page * d * 17 // 32
    pages = (1 << 32) // (Hkv * raw) + 50
    t = {n: torch.zeros((pages, Hkv, raw), dtype=torch.uint8, device="cuda:0") for n in ("k", "v")}
    t.update({n: torch.zeros((pages, Hkv, page), device="cuda:0") for n in ("kscale", "vscale")})
    high = [pages - 1, pages - 20, pages - 3]
    for i, p in enumerate(high):
        t["k"][p], t["v"][p], t["kscale"][p], t["vscale"][p] = i + 1, i + 11, i + 21, i + 31
    table, length, refs = ch.ints([high]), ch.ints([3 * page]), torch.zeros(pages, dtype=torch.int32, device="cuda:0")
    refs[high] = 1
    c = P.pasa_cache(t["k"], t["v"], t["kscale"], t["vscale"], table, length, S=1, Hkv=Hkv, d=d, page=page, pages=pages, table_width=3, format=P.CACHE_I4)
    stream = torch.cuda.current_stream()
    P.pasa_cache_copy(c, c, ch.ints([pages - 2]), ch.ints([high[1]]), 1, stream)
    assert int(t["k"][pages - 2].min()) == 2 == int(t["k"][pages - 2].max()) and float(t["vscale"][pages - 2].min()) == 32
    ws = torch.empty(P.pasa_cache_compact_workspace(c), dtype=torch.uint8, device="cuda:0")
    P.pasa_cache_compact(c, refs, None, ws, ws.numel(), stream)
    assert table.cpu().numpy().tolist() == [[2, 0, 1]] and refs[:3].cpu().numpy().tolist() == [1, 1, 1] and int(refs.sum()) == 3
    for i, p in enumerate([2, 0, 1]):
        assert int(t["k"][p].min()) == i + 1 == int(t["k"][p].max()) and int(t["v"][p].min()) == i + 11 and float(t["kscale"][p].max()) == i + 21
