"""Rotary positions on the GPU against the oracle."""
import numpy as np
import pytest

import paper_2503_01873_amd as P
from oracle import rotary_oracle as ro
from tests import cache_harness as ch
from tests.test_rotary import SCALING

pytestmark = pytest.mark.gpu


def _bound(y, wide, dtype):
    """Elements: cos and sin are rounded to fp32, a product and a multiply-add round once each (2^-24 of the products, twice, and of the sum), the type once.  Angles in
    64 bits are off by 3 2^-53 of the phase: 2^-20 for positions of 31 bits, 2^-33 up to 2^18, which 2^-25 of the products covers."""
    return 3.5 * 2.0 ** -24 * wide + (ch.HALF_STEP[dtype] + 2.0 ** -24) * np.abs(y) + ch.TINY[dtype] + 2.0 ** -130


def _rotary(layout, rot, base=1e4, magnitude=1.0, **kw):
    r = P.pasa_rotary()
    scaling = kw.pop("scaling", "plain")
    P.pasa_rotary_set(r, P.ROTARY_PAIRS if layout else P.ROTARY_HALVES, rot, base, scaling=SCALING[scaling], magnitude=magnitude, **kw)
    return r, ro.frequencies(rot, base, scaling, **kw)


def _type(dtype):
    import torch
    return torch.float16 if dtype == "f16" else torch.bfloat16


def _flat(n, dtype):
    import torch
    return torch.full((n,), float("nan"), dtype=_type(dtype), device="cuda:0")


def _check(got, ref, dtype):
    y, wide = ref
    off = np.abs(got - y) - _bound(y, wide, dtype)
    assert not (off > 0).any() and np.isfinite(got).all(), float(off.max())


SIZES = [(64, 64), (128, 128), (128, 64), (64, 16), (128, 32), (64, 2), (128, 6), (128, 126), (64, 40), (128, 96), (64, 24)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("d,rot", SIZES)
def test_sequences(d, rot, layout, dtype):
    """Every size of what is turned, out of a joint projection and in plain layouts, forward and back, into another tensor and in place."""
    import torch
    g = np.random.default_rng([d, rot, layout])
    B, H, N, extra = 2, 3, 37, 2
    r, f = _rotary(layout, rot, magnitude=1.25)
    x = ch.rounded(2 * g.standard_normal((B, N, H + extra, d)), dtype)
    t = torch.from_numpy(x).to("cuda:0").to(_type(dtype))
    xs = (N * (H + extra) * d, d, (H + extra) * d)
    for row0, back in ((0, False), (262144 - N, False), (5, True), (-11, False)):
        want = ro.rotate(x[:, :, :H].astype(np.float64), np.broadcast_to(row0 + np.arange(N), (B, N)), f, layout, 1.25, back)
        want = [w.transpose(0, 2, 1, 3) for w in want]
        flat = _flat(B * H * N * d + 256, dtype)
        P.pasa_rotate(r, t, flat, B, H, N, d, torch.cuda.current_stream(), x_strides=xs, row0=row0, transposed=back, io_dtype=ch.IO[dtype])
        torch.cuda.synchronize()
        assert bool(torch.isnan(flat[B * H * N * d:]).all())
        _check(flat[:B * H * N * d].view(B, H, N, d).double().cpu().numpy(), want, dtype)
        # in place: of the other heads, and of the channels from rot on, nothing changes
        u = t.clone()
        P.pasa_rotate(r, u, u, B, H, N, d, torch.cuda.current_stream(), x_strides=xs, y_strides=xs, row0=row0, transposed=back, io_dtype=ch.IO[dtype])
        torch.cuda.synchronize()
        assert torch.equal(u[:, :, H:], t[:, :, H:]) and torch.equal(u[:, :, :H, rot:], t[:, :, :H, rot:])
        assert torch.equal(u[:, :, :H].transpose(1, 2).contiguous().view(-1), flat[:B * H * N * d])


@pytest.mark.parametrize("scaling", SCALING)
def test_scaled_frequencies(scaling):
    import torch
    g = np.random.default_rng(3)
    kw = {} if scaling == "plain" else dict(scaling=scaling, factor=8.0, original=4096.0, slow=1.0, fast=4.0)
    r, f = _rotary(0, 128, base=500000.0, **kw)
    x = ch.rounded(g.standard_normal((1, 2, 500, 128)), "bf16")
    t = torch.from_numpy(x).to("cuda:0").bfloat16()
    y = torch.empty_like(t)
    P.pasa_rotate(r, t, y, 1, 2, 500, 128, torch.cuda.current_stream(), row0=30000, io_dtype=P.IO_BF16)
    want = ro.rotate(x.transpose(0, 2, 1, 3).astype(np.float64), 30000 + np.arange(500)[None], f, 0)
    _check(y.double().cpu().numpy(), [w.transpose(0, 2, 1, 3) for w in want], "bf16")


@pytest.mark.parametrize("B,H,N,d,rot,layout", [(1, 1, 1, 64, 64, 0), (1, 40, 1, 128, 128, 1), (3, 1, 1000, 64, 20, 0), (1, 36, 1500, 128, 128, 0), (2, 7, 1301, 128, 64, 1),
                                                (1, 500, 9, 64, 64, 0), (700, 2, 3, 64, 18, 1),
                                                (2, 9, 1100, 128, 126, 0)])
def test_numbers_of_tokens_and_heads(B, H, N, d, rot, layout):
    """One token a workgroup and four, heads shared out over several, positions of its own for every token, strides with gaps."""
    import torch
    g = np.random.default_rng([B, H, N])
    r, f = _rotary(layout, rot)
    position = g.integers(-(1 << 20), 1 << 20, (B, N)).astype(np.int32)
    x = ch.rounded(g.standard_normal((B, H, N, d)), "f16")
    t = torch.from_numpy(x).to("cuda:0").half()
    ys = (H * (N + 2) * (d + 8), (N + 2) * (d + 8), d + 8)
    flat = _flat(B * ys[0], "f16")
    P.pasa_rotate(r, t, flat, B, H, N, d, torch.cuda.current_stream(), y_strides=ys, positions=torch.from_numpy(position).to("cuda:0"))
    torch.cuda.synchronize()
    got = flat.view(B, H, N + 2, d + 8)
    assert bool(torch.isnan(got[:, :, N:]).all()) and bool(torch.isnan(got[..., d:]).all())
    want = ro.rotate(x.transpose(0, 2, 1, 3).astype(np.float64), position, f, layout)
    _check(got[:, :, :N, :d].double().cpu().numpy(), [w.transpose(0, 2, 1, 3) for w in want], "f16")


def test_rows_shared_by_batch_entries_and_what_is_not_finite():
    """A batch stride of 0 reads the same rows at other positions; infinities and NaN stay with their pairs."""
    import torch
    g = np.random.default_rng(5)
    r, f = _rotary(0, 64)
    x = ch.rounded(g.standard_normal((1, 2, 4, 64)), "f16")
    x[0, 0, 1, 3], x[0, 1, 2, 40] = np.inf, np.nan
    t = torch.from_numpy(x).to("cuda:0").half()
    y = torch.empty((3, 2, 4, 64), dtype=torch.float16, device="cuda:0")
    position = torch.tensor([[0, 1, 2, 3], [7, 7, 7, 7], [1000, 0, 5, -5]], dtype=torch.int32, device="cuda:0")
    P.pasa_rotate(r, t, y, 3, 2, 4, 64, torch.cuda.current_stream(), x_strides=(0, 4 * 64, 64), positions=position)
    with np.errstate(invalid="ignore"):
        want = ro.rotate(np.broadcast_to(x, (3, 2, 4, 64)).transpose(0, 2, 1, 3).astype(np.float64), position.cpu().numpy(), f, 0)[0].transpose(0, 2, 1, 3)
    got = y.double().cpu().numpy()
    # inf times a cos or sin is inf or, at position 0, NaN
    assert np.array_equal(np.isfinite(got), np.isfinite(want)) and not np.isfinite(got[:, 0, 1, [3, 35]]).any() and not np.isfinite(got[:, 1, 2, [8, 40]]).any()
    there = np.isfinite(want)
    assert (np.abs(got[there] - want[there]) <= 2.0 ** -10 * 8).all()


@pytest.mark.parametrize("far", [2 ** 31 - 1, -2 ** 31, 123456789])
def test_positions_of_any_size(far):
    """The phase of a position of 31 bits is off by 3 2^-53 of itself: 2^-20 turns and less."""
    import torch
    g = np.random.default_rng(6)
    r, f = _rotary(1, 128)
    x = ch.rounded(g.standard_normal((1, 1, 3, 128)), "f16")
    t = torch.from_numpy(x).to("cuda:0").half()
    y = torch.empty_like(t)
    position = np.array([[far, far // 3, 0]], np.int32)
    P.pasa_rotate(r, t, y, 1, 1, 3, 128, torch.cuda.current_stream(), positions=torch.from_numpy(position).to("cuda:0"))
    want, wide = ro.rotate(x.transpose(0, 2, 1, 3).astype(np.float64), position, f, 1)
    got = y.double().cpu().numpy().transpose(0, 2, 1, 3)
    assert (np.abs(got - want) <= _bound(want, wide, "f16") + 2.0 ** -18 * wide).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lengths,rows,behind", [
    ([9000, 3, 0, 77, 64], [1, 1, 0, 1, 1], 0),
    ([500, 64, 9, 5, 100], [48, 64, 0, 9, 70], 3),                      # more rows than tokens; more rows than a tree has bits
    ([5], [5], 1),
    (list(range(1, 65)), [1] * 64, 0), (list(range(1, 71)), [b % 3 for b in range(70)], 2), ([40] * 5000, [1] * 5000, 0),
])
@pytest.mark.parametrize("tree", [False, True])
def test_rows_of_a_step(lengths, rows, behind, tree, dtype):
    import torch
    g = np.random.default_rng([len(lengths), tree])
    heads, d, page, width = 5, 64, 16, 1000
    R = sum(rows) + behind
    r, f = _rotary(0, 32)
    x = ch.rounded(g.standard_normal((R, heads + 1, d)), dtype)
    bits = None
    if tree:
        bits = np.zeros(R, np.uint64)
        for r0, m in zip(ch.starts(rows), rows):
            for t in range(min(m, 64)):
                bits[r0 + t] = np.uint64(1 << t) | (bits[r0 + int(g.integers(0, t))] if t and g.random() < 0.8 else np.uint64(0))
        bits[0] = np.uint64(2 ** 64 - 1)                                # bits of rows that are not there, or of all
    dev = "cuda:0"
    length = ch.ints(lengths)
    any_ = torch.zeros(64, dtype=torch.uint8, device=dev)
    other = torch.zeros(64, dtype=torch.uint8, device=dev)
    cache = P.pasa_cache(any_, other, any_, other, ch.ints([[0] * 1]), length, S=len(lengths), Hkv=1, d=d, page=page, pages=1, table_width=width)
    t = torch.from_numpy(x).to(dev).to(_type(dtype)).view(R, -1)
    y = torch.full((R, (heads + 2) * d), float("nan"), dtype=t.dtype, device=dev)
    tt = None if tree is False else torch.from_numpy(bits.view(np.int64)).to(dev)
    start = ch.starts(rows)
    P.pasa_cache_rotate(cache, r, t, y, heads, R, t.stride(0), y.stride(0), ch.ints(start), torch.cuda.current_stream(), tree=tt, io_dtype=ch.IO[dtype])
    torch.cuda.synchronize()
    position = ro.positions(np.array(lengths), start, R, page * width, bits)
    there = np.array([p is not None for p in position])
    got = y.view(R, heads + 2, d).double().cpu().numpy()
    assert np.isnan(got[:, heads:]).all() and np.isnan(got[~there]).all()
    want = ro.rotate(x[there, :heads].astype(np.float64), np.array([p for p in position if p is not None]), f, 0)
    _check(got[there, :heads], want, dtype)
    # in place, as a step does it
    u = t.clone()
    P.pasa_cache_rotate(cache, r, u, u, heads, R, t.stride(0), t.stride(0), ch.ints(start), torch.cuda.current_stream(), tree=tt, io_dtype=ch.IO[dtype])
    v, at = u.view(R, heads + 1, d), torch.from_numpy(there).to(dev)
    assert torch.equal(v[at][:, :heads], y.view(R, heads + 2, d)[at][:, :heads])
    assert torch.equal(v[:, heads:], t.view(R, heads + 1, d)[:, heads:]) and torch.equal(v[~at], t.view(R, heads + 1, d)[~at])


def test_row_numbers_beyond_their_range():
    """row_start that does not begin at 0 or goes beyond the rows; lengths beyond the table."""
    import torch
    g = np.random.default_rng(9)
    d, R = 64, 20
    r, f = _rotary(1, 64)
    x = ch.rounded(g.standard_normal((R, 1, d)), "f16")
    any_, other = (torch.zeros(64, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    lengths = [1000, -5, 30]
    cache = P.pasa_cache(any_, other, any_, other, ch.ints([0]), ch.ints(lengths), S=3, Hkv=1, d=d, page=16, pages=1, table_width=10)
    for start in ([3, 9, 9, 500], [-4, 2, 5, 12], [20, 20, 20, 20], [0, 0, 0, 0]):
        t = torch.from_numpy(x).to("cuda:0").half().view(R, d)
        y = torch.full_like(t, float("nan"))
        P.pasa_cache_rotate(cache, r, t, y, 1, R, d, d, ch.ints(start), torch.cuda.current_stream())
        position = ro.positions(np.array(lengths), np.array(start), R, 160)
        there = np.array([p is not None for p in position])
        got = y.view(R, 1, d).double().cpu().numpy()
        assert np.isnan(got[~there]).all()
        if there.any():
            _check(got[there], ro.rotate(x[there].astype(np.float64), np.array([p for p in position if p is not None]), f, 1), "f16")


def test_tensors_beyond_4_GiB_and_a_captured_call_on_another_stream():
    """Offsets of more than 2^32 bytes, and 2^31 elements; the same call out of a graph, replayed with other positions."""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    H, N, d = 64, 300001, 128
    r, f = _rotary(0, 128)
    x = torch.zeros((N, H, d), dtype=torch.float16, device="cuda:0")
    g = np.random.default_rng(11)
    rows = [0, 1, 131071, 262145, N - 1]
    some = ch.rounded(g.standard_normal((len(rows), H, d)), "f16")
    x[rows] = torch.from_numpy(some).to("cuda:0").half()
    y = torch.full((H, N, d), float("nan"), dtype=torch.float16, device="cuda:0")
    positions = torch.arange(N, dtype=torch.int32, device="cuda:0")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    call = lambda st: P.pasa_rotate(r, x, y, 1, H, N, d, st, x_strides=(0, d, H * d), positions=positions)
    with torch.cuda.stream(stream):
        call(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(torch.cuda.current_stream())
    for shift in (0, -5, 77):
        if shift:
            positions.add_(shift)
            y.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
        got = y[:, rows].double().cpu().numpy().transpose(1, 0, 2)
        _check(got, ro.rotate(some.astype(np.float64), positions[rows].cpu().numpy(), f, 0), "f16")
        assert bool(torch.isfinite(y[:, -1]).all()) and bool(torch.isfinite(y[-1]).all())


def test_gradients_agree_with_differences():
    """Through autograd: the function's value against differences in 64 bits."""
    import torch
    B, H, N, d = 1, 2, 5, 64
    r, f = _rotary(0, 32, magnitude=1.1)

    class Rotate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            y = torch.empty_like(x)
            P.pasa_rotate(r, x, y, B, H, N, d, torch.cuda.current_stream(), row0=100)
            return y

        @staticmethod
        def backward(ctx, dy):
            dx = torch.empty_like(dy)
            P.pasa_rotate(r, dy.contiguous(), dx, B, H, N, d, torch.cuda.current_stream(), row0=100, transposed=True)
            return dx

    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.randn((B, H, N, d), generator=g, device="cuda:0").half().requires_grad_()
    w = torch.randn((B, H, N, d), generator=g, device="cuda:0").half()
    (Rotate.apply(x).float() * w.float()).sum().backward()
    at = lambda z: (ro.rotate(z.transpose(0, 2, 1, 3), 100 + np.arange(N)[None], f, 0, 1.1)[0].transpose(0, 2, 1, 3) * w.double().cpu().numpy()).sum()
    z = x.detach().double().cpu().numpy()
    rng = np.random.default_rng(0)
    for _ in range(40):
        i = tuple(int(rng.integers(0, n)) for n in z.shape)
        e = np.zeros_like(z)
        e[i] = 1e-3
        difference = (at(z + e) - at(z - e)) / 2e-3                      # the map is linear: exact but for 64 bits
        # the weights' gradient comes in fp16 once, and goes out once: half a step of a sum of two products
        assert abs(float(x.grad[i]) - difference) <= 2.0 ** -11 * abs(difference) + 2.0 ** -21 * 16 + 2.0 ** -25
