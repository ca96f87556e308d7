"""A cache of keys and values in 8 bits, in pages, and the attention that reads it: calls as a server makes them, with their plain forms.

Kinds of work:

  append   tokens of several sequences enter the cache (pasa_cache_write) and come back as attention will see them (pasa_cache_read)
  read     a stretch of every sequence comes back in 16 bits, laid out for pasa_prepare_kv (pasa_cache_read)
  choose   the pages that the queries' pseudo-averages point at (pasa_cache_choose)
  attend   a few rows of every sequence against the cache: decoding steps, trees of drafted tokens, over all keys or over chosen pages
           (pasa_attn_cache)
  turn     a whole decoding step of one layer: the new token enters, pages are chosen, attention reads them

The head layouts are those of `workloads/` (28 query heads on 4 with d = 128, 8 heads with d = 128, 5 heads with d = 64) and generic ones.
Lengths of a ragged batch are spread evenly between nothing and the longest.
"""
import math

import torch

own = False


def _case(name, work, S, Hq, Hkv, d, L, rows=1, page=64, format="i8", dtype="f16", ragged=True, tree=False, count=0, shift=False):
    """S sequences of up to L tokens, the last `rows` of them new (fewer where ragged).  count: pages that are chosen, 0 for all."""
    return {"name": name, "work": work, "S": S, "Hq": Hq, "Hkv": Hkv, "d": d, "L": L, "rows": rows, "page": page, "format": format,
            "dtype": dtype, "ragged": ragged, "tree": tree, "count": count, "shift": shift}


def listed():
    return [
        # the tokens of one decoding step: the smallest call, all latency
        _case("append_step_b16", "append", 16, 28, 4, 128, 8192, shift=True),
        # four prompts of ragged length, in the type models are stored in
        _case("append_prompts_bf16", "append", 4, 28, 4, 128, 8192, rows=8192, page=128, format="e4m3", dtype="bf16"),
        # frames of a video: d = 64, one KV head per query head, small pages
        _case("append_d64", "append", 14, 5, 5, 64, 2500, rows=2304, page=32, shift=True),
        # two long prompts read back for a chunk that is prepared anew
        _case("read_long_b2", "read", 2, 28, 4, 128, 32768, rows=32768, format="e4m3", dtype="bf16", ragged=False, shift=True),
        # pages for a decoding step of sixteen sequences
        _case("choose_b16", "choose", 16, 28, 4, 128, 32768, count=64),
        # pages for a step of the longest sequence that the library takes
        _case("choose_long", "choose", 1, 28, 4, 128, 262144, count=256, dtype="bf16"),
        # a decoding step of one sequence of no round length
        _case("step_one_4999", "attend", 1, 28, 4, 128, 4999),
        # a decoding step of sixteen sequences of ragged length
        _case("step_b16_ragged", "attend", 16, 28, 4, 128, 32768, shift=True),
        # a decoding step of the longest sequence
        _case("step_long", "attend", 1, 28, 4, 128, 262144, page=128, dtype="bf16"),
        # trees of drafted tokens behind eight sequences
        _case("tree_b8", "attend", 8, 28, 4, 128, 8192, rows=48, format="e4m3", dtype="bf16", tree=True),
        # a decoding step over the pages that were chosen
        _case("chosen_b16", "attend", 16, 28, 4, 128, 32768, count=64),
        # what a layer does in a decoding step: the token written, pages chosen, attention over them
        _case("turn_b16", "turn", 16, 28, 4, 128, 32768, count=64, shift=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        work = rng.choice(["append", "append", "read", "choose", "attend", "attend", "attend", "turn"])
        Hq, Hkv, d = rng.choice([(28, 4, 128), (28, 4, 128), (32, 8, 128), (8, 8, 128), (12, 2, 128), (5, 5, 64), (16, 16, 64), (16, 2, 64)])
        S, L, page = _log(rng, 1, 64), _log(rng, 16, 262144), rng.choice([16, 32, 64, 64, 128])
        rows, tree, count = 1, False, 0
        if work == "append":
            rows = rng.choice([1, _log(rng, 2, L)])
        elif work == "read":
            rows = _log(rng, 1, L)
        elif work == "attend":
            rows = rng.choice([1, 1, 1, _log(rng, 2, 64)])
            tree = rows > 1 and rng.random() < 0.7
        if work in ("choose", "turn") or (work == "attend" and rows == 1 and rng.random() < 0.3):
            count = _log(rng, 4, 256)
        c = _case("", work, S, Hq, Hkv, d, L, rows=min(rows, L), page=page, format=rng.choice(["i8", "i8", "e4m3"]),
                  dtype=rng.choice(["f16", "bf16"]), ragged=rng.random() < 0.6, tree=tree, count=count, shift=rng.random() < 0.5)
        del c["name"]
        # within what the largest listed ones hold and compute
        if S * L * Hkv * d <= 16 * 32768 * 4 * 128 and work_flops(c) <= 5e10 and S * L * Hq * c["rows"] <= (1 << 30 if work == "attend" else 1 << 62):
            return c


def _lengths(c):
    """Tokens of every sequence with the new ones, and new ones among them."""
    if not c["ragged"]:
        return [c["L"]] * c["S"], [c["rows"]] * c["S"]
    part = [(0.618033988749895 * b) % 1.0 for b in range(c["S"])]
    lengths = [c["L"] - int(p * c["L"]) for p in part]
    spread = [(0.414213562373095 * b) % 1.0 for b in range(c["S"])]
    return lengths, [min(n, c["rows"] - int(p * c["rows"])) for n, p in zip(lengths, spread)]


def _width(c):
    return (c["L"] + c["page"] - 1) // c["page"]


def _tail(c):
    """Last pages that are always chosen: those that the new tokens lie in."""
    return 1 + (c["rows"] + c["page"] - 2) // c["page"]


# ---- plain forms ----

def _type(c):
    return torch.float16 if c["dtype"] == "f16" else torch.bfloat16


def _codes(x, format):
    """8-bit codes of x [..., d] in 32 bits, and the scales, one for the d values of a token and head.  In 64 bits: ties."""
    x = x.double()
    top = x.abs().amax(-1)
    scale = (top / (127.0 if format == "i8" else 448.0)).float()
    scale = torch.where(top < 2.0 ** -100, torch.ones_like(scale), scale)
    y = x / scale.double()[..., None]
    if format == "i8":
        return (y.round().clamp(-127, 127) + 128).to(torch.uint8), scale
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp(min=-6) - 3)     # of an e4m3 value near y
    y = ((y / step).round() * step).clamp(-448, 448)
    return y.float().to(torch.float8_e4m3fn).view(torch.uint8), scale


def _values(codes, scale, format):
    x = codes.float() - 128 if format == "i8" else codes.view(torch.float8_e4m3fn).float()
    return x * scale[..., None]


def _rows(s):
    """Of every row: its sequence, its number among that sequence's new tokens, its position."""
    start, length = s["row_start"].long(), s["length"].long()
    row = torch.arange(s["R"], device=start.device)
    b = torch.searchsorted(start, row, right=True) - 1
    t = row - start[b]
    return b, t, length[b] - (start[b + 1] - start[b]) + t


def _plain_write(s):
    c = s["c"]
    b, t, pos = _rows(s)
    page, at = s["table"].long()[b, pos // c["page"]], pos % c["page"]
    k = s["k_new"].float()
    if c["shift"]:
        k = k - s["kshift"]
    for_k, for_v = _codes(k, c["format"]), _codes(s["v_new"].float(), c["format"])
    s["k"][page, :, at], s["kscale"][page, :, at] = for_k
    s["v"][page, :, at], s["vscale"][page, :, at] = for_v
    # the mean keys of the pages that were written to; a sequence's places beyond its last such page stand for the last one again
    start, length = s["row_start"].long(), s["length"].long()
    first = (length - (start[1:] - start[:-1])) // c["page"]
    place = first[:, None] + torch.arange(_tail(c), device=first.device)
    place = torch.minimum(place, ((length - 1) // c["page"])[:, None])
    page = s["table"].long().gather(1, place)
    left = (length[:, None] - place * c["page"]).clamp(max=c["page"])
    there = (torch.arange(c["page"], device=first.device) < left[..., None]).double()
    x = _values(s["k"][page], s["kscale"][page], c["format"]).double()              # [S, pages, Hkv, page, d]
    s["kmean"][page] = ((x * there[:, :, None, :, None]).sum(3) / left[..., None, None]).float()


def _plain_read(s):
    c = s["c"]
    N = c["rows"]
    pos = s["first"].long()[:, None] + torch.arange(N, device=s["k"].device)
    there = pos < s["length"].long()[:, None]
    pos = torch.where(there, pos, torch.zeros_like(pos))
    page, at = s["table"].long().gather(1, pos // c["page"]), pos % c["page"]
    out = []
    for_k = _values(s["k"][page, :, at], s["kscale"][page, :, at], c["format"])    # [S, N, Hkv, d]
    if c["shift"]:
        for_k = for_k + s["kshift"]
    out.append(for_k)
    out.append(_values(s["v"][page, :, at], s["vscale"][page, :, at], c["format"]))
    return [torch.where(there[:, :, None, None], x, torch.zeros_like(x)).to(_type(c)).permute(0, 2, 1, 3).contiguous() for x in out]


def _by_sequence(s):
    """The query rows in 32 bits as [S, Hkv, T * G, d], and which of the T are there."""
    c = s["c"]
    start = s["row_start"].long()
    row = start[:-1, None] + torch.arange(c["rows"], device=start.device)
    there = row < start[1:, None]
    q = s["q"].float()[row.clamp(max=s["R"] - 1)]                                   # [S, T, Hq, d]
    q = q.view(c["S"], c["rows"], c["Hkv"], -1, c["d"]).permute(0, 2, 1, 3, 4)
    return q.reshape(c["S"], c["Hkv"], -1, c["d"]), there


def _plain_choose(s):
    c = s["c"]
    q, there = _by_sequence(s)
    mean = s["kmean"][s["table"].long()].permute(0, 2, 1, 3)                        # [S, Hkv, W, d]
    score = mean.double() @ q.double().transpose(2, 3).contiguous()                 # in 64 bits: the order of near ones
    there = there.repeat_interleave(c["Hq"] // c["Hkv"], 1)[:, None, None, :]
    score = torch.where(there, score, torch.full_like(score, -math.inf)).amax(3)
    pages = (s["length"].long() + c["page"] - 1) // c["page"]
    p = torch.arange(score.shape[2], device=score.device)
    always = (p < 1) | (p >= pages[:, None, None] - _tail(c))
    score = torch.where(always, torch.full_like(score, math.inf), score)
    score = torch.where(p < pages[:, None, None], score, torch.full_like(score, -math.inf))
    order = torch.sort(score, dim=2, descending=True, stable=True)[1][:, :, :c["count"]]
    beyond = score.shape[2]
    order = torch.where(order < pages[:, None, None], order, torch.full_like(order, beyond)).sort(2)[0]
    out = torch.full((c["S"], c["Hkv"], c["count"]), -1, dtype=torch.int32, device=score.device)
    out[:, :, :order.shape[2]] = torch.where(order < beyond, order, torch.full_like(order, -1)).to(torch.int32)
    return out


def _plain_attend(s, blocks):
    c = s["c"]
    q, _ = _by_sequence(s)
    dev, G = q.device, c["Hq"] // c["Hkv"]
    heads = torch.arange(c["Hkv"], device=dev)[None, :, None]
    if blocks is None:
        place = torch.arange(_width(c), device=dev).expand(c["S"], c["Hkv"], -1)
    else:
        place = blocks.long()
    page = s["table"].long()[torch.arange(c["S"], device=dev)[:, None, None], place.clamp(min=0)]
    pos = place[..., None] * c["page"] + torch.arange(c["page"], device=dev)
    length, start = s["length"].long(), s["row_start"].long()
    n = start[1:] - start[:-1]
    there = ((place[..., None] >= 0) & (pos < length[:, None, None, None])).flatten(2)
    t = torch.arange(c["rows"], device=dev)
    new = (pos.flatten(2) - (length - n)[:, None, None])[..., None]                 # number among the new tokens, [S, Hkv, keys, 1]
    if c["tree"]:
        mask = s["tree"][(start[:-1, None] + t).clamp(max=s["R"] - 1)][:, None, None, :]
        sees = (new < 0) | ((mask >> new.clamp(0, 63)) & 1).bool()
    else:
        sees = new <= t
    sees = (sees & there[..., None]).repeat_interleave(G, 3)                        # [S, Hkv, keys, T * G]
    k = _values(s["k"][page, heads], s["kscale"][page, heads], c["format"]).flatten(2, 3)
    score = (k @ q.transpose(2, 3).contiguous()) * s["scale"]
    score = torch.where(sees, score, torch.full_like(score, -math.inf))
    top = score.amax(2, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    v = _values(s["v"][page, heads], s["vscale"][page, heads], c["format"]).flatten(2, 3)
    out = (p.transpose(2, 3) @ v) / p.sum(2)[..., None].clamp(min=1e-30)            # [S, Hkv, T * G, d]
    out = out.view(c["S"], c["Hkv"], c["rows"], G, c["d"]).permute(0, 2, 1, 3, 4).reshape(c["S"], c["rows"], c["Hq"], c["d"])
    b, t, _ = _rows(s)
    return out[b, t].to(_type(c))


# ---- inputs ----

def _inputs(c, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(1000003 * int(seed) + 29)
    S, Hq, Hkv, d, page, W = c["S"], c["Hq"], c["Hkv"], c["d"], c["page"], _width(c)
    lengths, new = _lengths(c)
    R, pages = sum(new), S * W + 3

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    def whole(x, dtype=torch.int32):
        return torch.tensor(x, device=dev, dtype=dtype)

    s = {"c": c, "R": R, "length": whole(lengths), "row_start": whole([0] + new).cumsum(0).to(torch.int32),
         "first": whole([n - m for n, m in zip(lengths, new)]), "scale": float(torch.tensor(d ** -0.5, dtype=torch.float32)),
         "table": torch.randperm(pages, generator=g, device=dev)[:S * W].view(S, W).to(torch.int32)}
    # keys have a bias of their own in every channel, four channels a large one; the cache may take it off
    bias = normal(Hkv, d)
    bias[:, torch.randperm(d, generator=g, device=dev)[:4]] += 60.0
    s["kshift"] = bias
    k, v = normal(pages, Hkv, page, d), normal(pages, Hkv, page, d)
    s["k"], s["kscale"] = _codes(k if c["shift"] else k + 0.1 * bias[:, None], c["format"])
    s["v"], s["vscale"] = _codes(v, c["format"])
    if c["work"] in ("append", "choose", "turn"):
        mean = _values(s["k"], s["kscale"], c["format"]).mean(2)
        s["kmean"] = mean * math.sqrt(page) * 0.25 if c["work"] != "append" else mean
    s["q"] = (2.0 * normal(R, Hq, d)).to(_type(c))
    if c["work"] in ("append", "turn"):
        # the new keys and values as a projection of queries, keys and values leaves them: slices of one tensor
        s["qkv"] = torch.cat([s["q"], (normal(R, Hkv, d) + bias).to(_type(c)), normal(R, Hkv, d).to(_type(c))], 1)
        s["q"], s["k_new"], s["v_new"] = s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + Hkv], s["qkv"][:, Hq + Hkv:]
    if c["tree"]:
        # every drafted token has a parent among those before it, and sees its ancestors
        b, t, _ = _rows(s)
        parent = (torch.rand(R, generator=g, device=dev) * t).long()
        base = s["row_start"].long()[b]
        see = torch.ones(R, dtype=torch.int64, device=dev) << t
        for depth in range(6):                                  # ancestors up to 64 steps away, doubling
            see = torch.where(t > 0, see | see[base + parent], see)
            parent = parent[base + parent]
        s["tree"] = see
    if c["work"] == "attend" and c["count"]:
        place = torch.rand((S, Hkv, W), generator=g, device=dev)
        there = (s["length"].long() + page - 1) // page
        w = torch.arange(W, device=dev)
        place = torch.where(w == there[:, None, None] - 1, torch.full_like(place, 2.0), place)
        place = torch.where(w < there[:, None, None], place, torch.full_like(place, -1.0))
        value, at = place.topk(min(W, c["count"]), 2)
        at = torch.where(value >= 0, at, torch.full_like(at, W)).sort(2)[0]
        s["blocks"] = torch.full((S, Hkv, c["count"]), -1, dtype=torch.int32, device=dev)
        s["blocks"][:, :, :at.shape[2]] = torch.where(at < W, at, torch.full_like(at, -1)).to(torch.int32)
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    dev = s["q"].device
    # what a program keeps from step to step: where results go, the cache's description, workspaces
    if c["work"] in ("append", "read"):
        s["k_out"] = torch.empty((c["S"], c["Hkv"], c["rows"], c["d"]), dtype=_type(c), device=dev)
        s["v_out"] = torch.empty_like(s["k_out"])
    if c["work"] in ("choose", "turn"):
        s["blocks"] = torch.empty((c["S"], c["Hkv"], c["count"]), dtype=torch.int32, device=dev)
    if c["work"] in ("attend", "turn"):
        s["o"] = torch.empty((s["R"], c["Hq"], c["d"]), dtype=_type(c), device=dev)
    if own:
        import paper_2503_01873_amd as P
        s["cache"] = P.pasa_cache(s["k"], s["v"], s["kscale"], s["vscale"], s["table"], s["length"], S=c["S"], Hkv=c["Hkv"], d=c["d"],
                                  page=c["page"], pages=s["k"].shape[0], table_width=_width(c),
                                  format=P.CACHE_I8 if c["format"] == "i8" else P.CACHE_E4M3, kmean=s.get("kmean"),
                                  kshift=s["kshift"] if c["shift"] else None)
        s["io"] = P.IO_F16 if c["dtype"] == "f16" else P.IO_BF16
        for name, size in (("choose", P.pasa_cache_choose_workspace(s["cache"])),
                           ("attn", P.pasa_attn_cache_workspace(s["cache"], s["R"], c["Hq"]))):
            s[name + "_bytes"], s[name + "_ws"] = size, torch.empty(max(size, 1), dtype=torch.uint8, device=dev)
    return s


def run(s):
    c = s["c"]
    work = c["work"]
    if own:
        import paper_2503_01873_amd as P
        stream, cache = torch.cuda.current_stream(), s["cache"]
        if work in ("append", "turn"):
            P.pasa_cache_write(cache, s["k_new"], s["v_new"], s["R"], s["k_new"].stride(0), s["row_start"], stream, io_dtype=s["io"])
        if work in ("append", "read"):
            P.pasa_cache_read(cache, s["k_out"], s["v_out"], s["first"], c["rows"], stream, io_dtype=s["io"])
            return [s["k_out"], s["v_out"]] + ([s["kmean"]] if work == "append" else [])
        if work in ("choose", "turn"):
            P.pasa_cache_choose(cache, s["q"], s["R"], s["q"].stride(0), s["row_start"], c["Hq"], s["blocks"], c["count"], 1, _tail(c),
                                s["choose_ws"], s["choose_bytes"], stream, io_dtype=s["io"])
            if work == "choose":
                return s["blocks"]
        P.pasa_attn_cache(cache, s["q"], s["o"], s["R"], s["q"].stride(0), s["row_start"], c["Hq"], s["scale"], s["attn_ws"],
                          s["attn_bytes"], stream, tree=s.get("tree"), blocks=s.get("blocks"), count=c["count"], io_dtype=s["io"])
        return s["o"] if work == "attend" else [s["o"], s["blocks"], s["kmean"]]
    if work in ("append", "turn"):
        _plain_write(s)
    if work in ("append", "read"):
        return _plain_read(s) + ([s["kmean"]] if work == "append" else [])
    if work == "choose":
        return _plain_choose(s)
    if work == "attend":
        return _plain_attend(s, s.get("blocks"))
    blocks = _plain_choose(s)
    return [_plain_attend(s, blocks), blocks, s["kmean"]]


# ---- what a pass cannot do without ----

def _keys(c):
    """Keys that a pass of attention reads, of one KV head."""
    lengths, _ = _lengths(c)
    most = c["count"] * c["page"] if c["count"] else c["L"]
    return [min(n, most) for n in lengths]


def work_flops(c):
    lengths, new = _lengths(c)
    flops = 0.0
    if c["work"] in ("attend", "turn"):
        flops += sum(4.0 * c["d"] * c["Hq"] * m * n for m, n in zip(new, _keys(c)))
    if c["work"] in ("choose", "turn"):
        flops += sum(2.0 * c["d"] * c["Hq"] * m * ((n + c["page"] - 1) // c["page"]) for m, n in zip(new, lengths))
    return flops


def work(c):
    lengths, new = _lengths(c)
    Hkv, Hq, d, page, R = c["Hkv"], c["Hq"], c["d"], c["page"], sum(new)
    token = Hkv * (2 * d + 8)                                   # codes and scales of a token's key and value
    moved = 0
    if c["work"] in ("append", "turn"):
        older = sum((n - m) % page for n, m in zip(lengths, new))
        touched = sum((n - 1) // page - (n - m) // page + 1 for n, m in zip(lengths, new))
        moved += R * (4 * Hkv * d + token) + older * Hkv * (d + 4) + touched * Hkv * 4 * d
    if c["work"] == "append":
        moved += 4 * c["S"] * c["rows"] * Hkv * d               # back in 16 bits
    if c["work"] == "read":
        moved += R * token + 4 * c["S"] * c["rows"] * Hkv * d
    if c["work"] in ("choose", "turn"):
        moved += 2 * R * Hq * d + sum((n + page - 1) // page for n in lengths) * Hkv * 4 * d + 4 * c["S"] * Hkv * c["count"]
    if c["work"] in ("attend", "turn"):
        moved += 4 * R * Hq * d + sum(_keys(c)) * token
    return {"bytes": moved, "flops": work_flops(c)}


# ---- the same in 64 bits, from the definitions ----

def _exact_codes(x, format):
    """The values that x [n, d] is held as, and their scales."""
    top = x.abs().max(1, keepdim=True)[0]
    scale = (top / (127 if format == "i8" else 448)).float().double()
    scale[top < 2.0 ** -100] = 1.0
    if format == "i8":
        return torch.round(x / scale), scale
    size = (x / scale).abs()
    grid = torch.tensor([m * 2.0 ** (e - 3) for e in range(-6, 9) for m in (range(0, 16) if e == -6 else range(8, 16)) if m * 2.0 ** (e - 3) <= 448],
                        dtype=torch.float64, device=x.device)                          # e4m3's values that are not negative
    up = torch.searchsorted(grid, size).clamp(max=grid.numel() - 1)
    low, high = grid[(up - 1).clamp(min=0)], grid[up]
    middle = (low + high) / 2
    take = (size > middle) | ((size == middle) & (up % 2 == 0))                        # a tie goes to the even one
    return torch.where(take, high, low) * torch.sign(x), scale


def _exact_old(s, which, b, h, format):
    """What sequence b, head h of the cache holds, [tokens, d]."""
    page = s["table"][b].long()
    codes = s[which][page, h].reshape(-1, s["c"]["d"])
    x = codes.double() - 128 if format == "i8" else codes.view(torch.float8_e4m3fn).double()
    return x * s[which + "scale"][page, h].reshape(-1, 1).double()


def exact(c, seed):
    s = _inputs(c, seed)
    dev = s["q"].device
    lengths, new = _lengths(c)
    S, Hq, Hkv, d, page, fmt, G = c["S"], c["Hq"], c["Hkv"], c["d"], c["page"], c["format"], c["Hq"] // c["Hkv"]
    wide = {"dtype": torch.float64, "device": dev}
    o = torch.zeros((s["R"], Hq, d), **wide)
    back = torch.zeros((2, S, Hkv, c["rows"], d), **wide)
    kmean = s["kmean"].double() if "kmean" in s else None
    blocks = torch.full((S, Hkv, c["count"]), -1, dtype=torch.int64, device=dev)
    r0 = 0
    for b in range(S):
        n, m = lengths[b], new[b]
        pages = (n + page - 1) // page
        ids = s["table"][b].long()
        for h in range(Hkv):
            if c["work"] != "choose":
                k, v = _exact_old(s, "k", b, h, fmt), _exact_old(s, "v", b, h, fmt)
            if c["work"] in ("append", "turn"):
                x = s["k_new"][r0:r0 + m, h].double() - (s["kshift"][h].double() if c["shift"] else 0.0)
                x = x.float().double()                          # the difference is held in 32 bits
                for held, fresh in ((k, x), (v, s["v_new"][r0:r0 + m, h].double())):
                    code, scale = _exact_codes(fresh, fmt)
                    held[n - m:n] = code * scale
                for p in range((n - m) // page, pages):
                    kmean[ids[p], h] = k[p * page:min(n, (p + 1) * page)].mean(0)
            if c["work"] in ("append", "read"):
                back[0, b, h, :m] = k[n - m:n] + (s["kshift"][h].double() if c["shift"] else 0.0)
                back[1, b, h, :m] = v[n - m:n]
            rows = s["q"][r0:r0 + m, h * G:(h + 1) * G].double()                # [m, G, d]
            if c["work"] in ("choose", "turn"):
                score = (rows.reshape(-1, d) @ kmean[ids[:pages], h].t().contiguous()).max(0)[0]
                score[0] = math.inf
                score[max(0, pages - _tail(c)):] = math.inf
                at = torch.sort(score, descending=True, stable=True)[1][:c["count"]].sort()[0]
                blocks[b, h, :at.numel()] = at
            if c["work"] in ("attend", "turn"):
                see = torch.arange(n, device=dev)[None, :] <= torch.arange(n - m, n, device=dev)[:, None]
                if c["tree"]:
                    bits = s["tree"][r0:r0 + m, None] >> torch.arange(m, device=dev)[None, :]
                    see[:, n - m:] = (bits & 1).bool()
                if c["count"]:
                    at = (blocks if c["work"] == "turn" else s["blocks"].long())[b, h]
                    only = torch.zeros(pages, dtype=torch.bool, device=dev)
                    only[at[at >= 0]] = True
                    keep = see & only.repeat_interleave(page)[:n]
                else:
                    keep = see
                score = (rows.reshape(-1, d) @ k[:n].t().contiguous()).view(m, G, n) * s["scale"]
                score.masked_fill_(~keep[:, None], -math.inf)
                score = torch.softmax(score, 2)
                o[r0:r0 + m, h * G:(h + 1) * G] = (score.view(-1, n) @ v[:n]).view(m, G, d)
        r0 += m
    if c["work"] in ("append", "read"):
        return [back[0], back[1]] + ([kmean] if c["work"] == "append" else [])
    return blocks if c["work"] == "choose" else o if c["work"] == "attend" else [o, blocks, kmean]
