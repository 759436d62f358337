"""Rotary positions against the formula in 64 bits."""
import math
from decimal import Decimal, getcontext

import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import DTYPES, check, half_step

pytestmark = pytest.mark.gpu

# Of a turned channel, relative to amplitude (|u| + |v|): the turn's fraction (at most 1/2) is rounded to 32 bits, 2 pi 2^-26 radians; CUDA's sine and cosine of it are good
# to 2 units of 2^-24; amplitude, products and sum are rounded once each: 2^-23.3 + 2^-23 + 3 2^-24 < 2^-21.
TURN_ERR = 2.0 ** -21


def tensor(B, H, N, D, dtype, layout, gen, scale=1.0):
    """[B,H,N,D] in the order of the layout; NaN in everything of the buffer that is not the tensor."""
    unit = 16 // torch.empty((), dtype=dtype).element_size()
    wide = -(-D // unit) * unit
    if layout == "heads":
        t = torch.full((B, H, N + 1, wide), float("nan"), dtype=dtype, device="cuda")[:, :, :N, :D]
    elif layout == "rows":
        t = torch.full((B, N, H, wide), float("nan"), dtype=dtype, device="cuda")[..., :D].transpose(1, 2)
    else:                                # the first heads of a fused output
        t = torch.full((B, N, H + 2, wide), float("nan"), dtype=dtype, device="cuda")[:, :, :H, :D].transpose(1, 2)
    return t.copy_(torch.randn((B, H, N, D), device="cuda", generator=gen) * scale)


def angles(B, N, pairs, freq, n_text, grid, positions, offset):
    """([B or 1, N, pairs] in 64 bits, [N] which tokens turn)"""
    freq = freq.cuda()
    if positions is not None:
        pos = torch.zeros((*positions.shape[:2], 3), dtype=torch.float64, device="cuda")
        pos[..., :positions.shape[2]] = positions.double()
        on = torch.ones(N, dtype=torch.bool, device="cuda")
    else:
        T, h, w = grid
        n = torch.arange(N, device="cuda") - n_text
        pos = torch.stack((n // (h * w), n // w % h, n % w), -1).double()[None]
        on = n >= 0
    pos = pos + torch.tensor([float(o) for o in offset], dtype=torch.float64, device="cuda")
    axis = torch.tensor([a for a in range(3) for _ in range(pairs[a])], device="cuda")
    return pos[..., axis] * freq, on


def ref(x, angle, on, half, amplitude, inverse):
    x = x.double()
    P = angle.shape[-1]
    a = angle[:, None] * (-1 if inverse else 1)
    m = float(torch.tensor(amplitude, dtype=torch.float32))
    iu = torch.arange(P, device="cuda") * (1 if half else 2)
    iv = iu + (P if half else 1)
    u, v = x[..., iu], x[..., iv]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., iu], y[..., iv] = m * (u * a.cos() - v * a.sin()), m * (u * a.sin() + v * a.cos())
    size[..., iu] = size[..., iv] = m * (u.abs() + v.abs())
    keep = ~on[None, None, :, None]
    return torch.where(keep, x, y), torch.where(keep, 0.0, size), iu, iv


def run(B, H, N, D, pairs, dtype="bf16", layout="rows", half=False, inverse=False, n_text=0, grid=None, positions=None, offset=(0, 0, 0), amplitude=1.0, in_place=False,
        freq=None, out="heads", seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = tensor(B, H, N, D, DTYPES[dtype], layout, gen)
    pairs = tuple(pairs) + (0,) * (3 - len(pairs))
    if freq is None:
        freq, _ = cn.rope_frequencies(pairs)
    grid = grid or (N - n_text, 1, 1)
    angle, on = angles(B, N, pairs, freq, n_text, grid, positions, offset)
    want, size, *_ = ref(x, angle, on, half, amplitude, inverse)
    y = x if in_place else tensor(B, H, N, D, DTYPES[dtype], out, gen)
    base = y._base if y._base is not None else y
    before = base.clone()
    s = cn.make_rope_shape(x, y, pairs, n_text=n_text, grid=grid, positions=positions, offset=offset, layout=cn.ROPE_HALF if half else cn.ROPE_INTERLEAVED,
                           amplitude=amplitude, inverse=inverse)
    got = cn.rope(x, freq.cuda(), s, positions=positions, Y=y)
    check(got, want, TURN_ERR * size + half_step(y.dtype) * want.abs() + 2.0 ** -149, "y")
    outside = before.isnan()             # what is not the tensor is as it was
    assert torch.equal(base.isnan(), outside)
    P = sum(pairs)
    assert torch.equal(y[:, :, ~on].double(), want[:, :, ~on]) and torch.equal(y[..., 2 * P:].double(), want[..., 2 * P:])
    return got


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,pairs", [(2, 1), (6, 3), (8, 4), (16, 5), (33, 16), (64, 32), (64, 24), (72, 36), (80, 40), (96, 48), (128, 64), (128, 33), (130, 2), (256, 128), (255, 1)])
def test_every_head(D, pairs, half, dtype):
    run(2, 3, 37, D, (pairs,), dtype, half=half, seed=D + pairs)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("layout,out", [("rows", "rows"), ("heads", "heads"), ("fused", "rows"), ("fused", "heads"), ("heads", "fused")])
@pytest.mark.parametrize("B,H,N,n_text,grid", [(1, 1, 1, 0, (1, 1, 1)), (2, 5, 31, 0, (31, 1, 1)), (1, 24, 13 + 3 * 7 * 5, 13, (3, 7, 5)), (2, 3, 60, 60, (0, 4, 4)),
                                               (1, 80, 2 * 9 * 16, 0, (2, 9, 16)), (3, 2, 1 + 1 * 1 * 400, 1, (1, 1, 400))])
def test_grids_layouts_and_text(half, layout, out, B, H, N, n_text, grid):
    for inverse in (False, True):
        run(B, H, N, 64, (12, 10, 10), "bf16", layout, half, inverse, n_text, grid, offset=(5, 0, -3), out=out, seed=N)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(half, dtype):
    run(2, 4, 6 + 30, 96, (10, 12, 14), dtype, "fused", half, False, 6, (2, 3, 5), in_place=True)


@pytest.mark.parametrize("axes,pairs", [(1, (20,)), (2, (8, 12)), (3, (4, 8, 8))])
@pytest.mark.parametrize("shared", [False, True])
def test_positions_as_a_tensor(axes, pairs, shared):
    gen = torch.Generator(device="cuda").manual_seed(axes)
    B, N = 3, 45
    p = torch.randint(-(1 << 31), (1 << 31) - 1, (1 if shared else B, N + 2, axes), device="cuda", generator=gen, dtype=torch.int64).int()[:, 2:]
    p[:, 0] = 0
    run(B, 2, N, 64, pairs, "f32", "heads", True, positions=p)
    run(B, 2, N, 64, pairs, "bf16", "rows", False, True, positions=p, offset=(1 << 30, 0, 0) if axes == 1 else (0, 0, 0))
    if shared:                           # the same seen by every entry
        run(B, 2, N, 64, pairs, "f32", "heads", True, positions=p.expand(B, N, axes))


def test_far_positions_keep_their_angle():
    """2^31 - 1 positions out, frequency 1 radian: 64 bits have the angle to 2^-22 radians, 32 bits nothing of it.  Two neighbours there differ by one turn of the
    pair, which is what the plain formula gives at position 1."""
    x = torch.zeros((1, 1, 2, 4), device="cuda")[..., :2]          # rows on 16-byte boundaries
    x[..., 0] = 1
    p = torch.tensor([[[(1 << 31) - 2], [(1 << 31) - 1]]], dtype=torch.int32, device="cuda")
    y = cn.rope(x, torch.ones(1, dtype=torch.float64, device="cuda"), cn.make_rope_shape(x, None, 1, positions=p), positions=p)[0, 0].double()
    turn = torch.atan2(y[1, 1], y[1, 0]) - torch.atan2(y[0, 1], y[0, 0])
    assert abs(math.remainder(float(turn) - 1.0, 2 * math.pi)) < 2.0 ** -20       # two angles, each to 2^-21


def test_scaled_frequencies():
    for mode, kw in ((cn.ROPE_SCALE_LINEAR, dict(factor=4.0)), (cn.ROPE_SCALE_BASE, dict(factor=(2.0, 1.0, 1.5))), (cn.ROPE_SCALE_RAMP, dict(factor=8.0, original=(21, 30, 52), low=0.5, high=4.0))):
        freq, m = cn.rope_frequencies((22, 21, 21), scaling=mode, **kw)
        run(1, 4, 9 + 2 * 5 * 6, 128, (22, 21, 21), "f32", n_text=9, grid=(2, 5, 6), freq=freq, amplitude=m)


def test_what_does_not_turn_keeps_its_bits():
    """Text tokens and the channels behind the pairs: copied, infinities and NaN among them."""
    for half in (False, True):
        for dtype in (torch.bfloat16, torch.float32):
            x = torch.randn((1, 2, 5 + 12, 32), device="cuda").to(dtype)
            x[:, :, :5, ::3], x[:, :, 2, 1::3] = float("inf"), float("nan")
            x[..., 21:24], x[..., 25] = float("-inf"), float("nan")
            for y in (torch.empty_like(x), x.clone()):
                src = x if y.data_ptr() != x.data_ptr() else y
                s = cn.make_rope_shape(src, y, (4, 3, 3), n_text=5, grid=(3, 2, 2), layout=int(half))
                cn.rope(src, cn.rope_frequencies((4, 3, 3), device="cuda")[0], s, Y=y)
                kind = torch.int16 if dtype == torch.bfloat16 else torch.int32
                assert torch.equal(y[:, :, :5].contiguous().view(kind), x[:, :, :5].contiguous().view(kind))
                assert torch.equal(y[..., 20:].contiguous().view(kind), x[..., 20:].contiguous().view(kind))
                assert torch.isfinite(y[:, :, 5:, :20]).all()


def test_broadcast_input_and_wide_batches():
    gen = torch.Generator(device="cuda").manual_seed(3)
    one = torch.randn((2, 1, 50, 64), device="cuda", generator=gen).bfloat16()
    x = one.expand(2, 7, 50, 64)
    freq, _ = cn.rope_frequencies(32)
    y = cn.rope(x, freq.cuda(), cn.make_rope_shape(x, None, 32))
    z = cn.rope(one, freq.cuda(), cn.make_rope_shape(one, None, 32))
    assert torch.equal(y, z.expand_as(y))
    many = torch.randn((65535, 1, 1, 8), device="cuda", generator=gen)
    assert torch.equal(cn.rope(many, torch.ones(4, dtype=torch.float64, device="cuda"), cn.make_rope_shape(many, None, 4)), many)      # position 0


@pytest.mark.parametrize("half", [False, True])
def test_gradient(half):
    """The inverse call is the transposed map: against differences of sum(dy rope(x)) (the map is linear: they are exact but for rounding), and the product with its own
    inverse is the amplitude squared."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, H, N, D, pairs, m = 2, 3, 4 + 24, 48, (8, 6, 6), 1.25
    x, dy = (torch.randn((B, H, N, D), device="cuda", generator=gen) for _ in range(2))
    freq = cn.rope_frequencies(pairs, device="cuda")[0]
    how = dict(n_text=4, grid=(2, 3, 4), layout=int(half), amplitude=m)
    f, b = cn.make_rope_shape(x, None, pairs, **how), cn.make_rope_shape(x, None, pairs, inverse=True, **how)
    dx = cn.rope(dy, freq, b).double()
    for _ in range(20):
        e = torch.randn((B, H, N, D), device="cuda", generator=gen)
        up, down = (cn.rope(x + sign * e, freq, f).double() for sign in (1, -1))
        difference = (dy.double() * (up - down)).sum() / 2
        size = (dy.double().abs() * (x.abs() + e.abs()).double()).sum()
        assert abs(difference - (dx * e.double()).sum()) <= 8 * m * TURN_ERR * size
    back = cn.rope(cn.rope(x, freq, f), freq, b).double()
    P = sum(pairs)
    want = x.double().clone()
    want[:, :, 4:, :2 * P] *= m * m
    assert (back - want).abs().max() <= 8 * TURN_ERR * m * m * x.abs().max()


def test_offsets_that_pass_32_bits():
    """2.4e9 elements, the last token's heads far behind 2^31: in place, against the same tokens on their own."""
    N, H, D, tail = 300_000, 64, 128, 40
    x = torch.zeros((1, N, H, D), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    gen = torch.Generator(device="cuda").manual_seed(5)
    last = torch.randn((1, H, tail, D), device="cuda", generator=gen).bfloat16()
    x[:, :, -tail:] = last
    freq = cn.rope_frequencies(64, device="cuda")[0]
    cn.rope(x, freq, cn.make_rope_shape(x, x, 64), Y=x)
    want = cn.rope(last, freq, cn.make_rope_shape(last, None, 64, offset=(N - tail, 0, 0)))
    assert torch.equal(x[:, :, -tail:], want) and not x[:, :, :-tail].any()


def test_on_a_side_stream_and_replayed():
    x = torch.randn((1, 4, 64, 128), device="cuda").bfloat16()
    freq = cn.rope_frequencies(64, device="cuda")[0]
    s = cn.make_rope_shape(x, None, 64)
    want = cn.rope(x, freq, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(x)
    s = cn.make_rope_shape(x, y, 64)
    cn.rope(x, freq, s, Y=y, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cn.rope(x, freq, s, Y=y)
    for k in range(3):
        x.copy_(torch.randn((1, 4, 64, 128), device="cuda"))
        graph.replay()
        assert torch.equal(y, cn.rope(x, freq, s, Y=torch.empty_like(x)))


TWO_PI = Decimal("6.28318530717958647692528676655900576839433879875021")


@pytest.mark.parametrize("half", [False, True])
def test_sine_and_cosine_at_any_position(half):
    """fp32, against angles of 50 digits, out to positions of 2^32 with the offset.  CUDA's sine and cosine are good to a unit of 2^-24, and the rest of the angle is added with one
    rounding, 2^-25: less than 2^-23."""
    getcontext().prec = 50
    freq = torch.cat((cn.rope_frequencies(6)[0], torch.tensor([0.7312345678901234, 3.0], dtype=torch.float64)))
    pos = [0, 1, -1, 7, 100, 4097, 75599, 10 ** 6 + 3, -(10 ** 7) - 1, (1 << 27) + 1, (1 << 30) + 12345, -(1 << 30) - 999, (1 << 31) - 1, -(1 << 31)]
    x = torch.zeros((1, 1, len(pos), 16), device="cuda")
    x[..., slice(0, 8) if half else slice(0, 16, 2)] = 1
    p = torch.tensor(pos, dtype=torch.int64).int().cuda()[None, :, None]
    for offset in (0, (1 << 31) - 1, -(1 << 31)):
        y = cn.rope(x, freq.cuda(), cn.make_rope_shape(x, None, 8, positions=p, offset=(offset, 0, 0), layout=int(half)), positions=p)[0, 0].double().cpu()
        for n, at in enumerate(pos):
            for i, f in enumerate(freq.tolist()):
                angle = float((Decimal(at) + offset) * Decimal(f) % TWO_PI)
                u, v = (y[n, i], y[n, i + 8]) if half else (y[n, 2 * i], y[n, 2 * i + 1])
                assert abs(u - math.cos(angle)) <= 2.0 ** -23 and abs(v - math.sin(angle)) <= 2.0 ** -23, (at, offset, f)
