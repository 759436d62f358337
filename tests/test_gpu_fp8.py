"""8-bit operands and their matrix product against the definitions: the values exactly, the product in 64 bits."""
import math

import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import ACT_ERR, DTYPES, SLOPE_MOST, U32, act64, canvas, check, half_step, padded, untouched

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
ACTS = [cn.ACT_NONE, cn.ACT_GELU_TANH, cn.ACT_GELU, cn.ACT_SILU]


def quantize_ref(x, tile):
    """(values of q in 64 bits, scale in 64 bits) of a [B,N,K] without infinities and NaN, by the definition."""
    B, N, K = x.shape
    nb, kb = -(-N // tile), -(-K // 128)
    full = torch.zeros((B, nb * tile, kb * 128), dtype=torch.float64, device=x.device)
    full[:, :N, :K] = x.double()
    amax = full.abs().view(B, nb, tile, kb, 128).amax((2, 4)).clamp(min=2.0 ** -100)
    m, e = torch.frexp(amax)                       # amax = m 2^e, 1/2 <= m < 1; 448 = 0.875 x 2^9
    scale = torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875).int())
    v = full / scale.repeat_interleave(tile, 1).repeat_interleave(128, 2)
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), e.clamp(min=-5) - 4)        # four significant bits, 2^-9 below 2^-6
    return (torch.round(v / step) * step)[:, :N, :K], scale


def values(q, scale, tile=1):
    return q.double() * scale.double().repeat_interleave(tile, 1).repeat_interleave(128, 2)[:, :q.shape[1], :q.shape[2]]


def spread(shape, dtype, gen, extra=1):
    """Rows and blocks of very different size."""
    x = padded(shape, dtype, gen, extra=extra)
    return x.mul_(torch.exp2(torch.randint(-20, 20, (*shape[:2], 1), device="cuda", generator=gen).float()).to(dtype))


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,K", [(1, 1, 1), (1, 1, 128), (2, 3, 37), (1, 130, 129), (3, 257, 520), (1, 1000, 1541), (1, 128, 4096), (1, 5, 16000), (2, 33, 640)])
def test_quantize(B, N, K, dtype, tile):
    gen = torch.Generator(device="cuda").manual_seed(N + K)
    x = spread((B, N, K), DTYPES[dtype], gen)
    q64, s64 = quantize_ref(x, tile)
    buf = torch.full((B, N + 1, -(-K // 16) * 16 + 16), 77, dtype=torch.uint8, device="cuda")
    q = buf.view(E4M3)[:, :N, :K]
    for how in ("own", "rows", "blocks"):
        nb, kb = s64.shape[1:]
        scale = None if how == "own" else torch.full((B, nb + 1, kb + 1), 77.0, device="cuda")[:, :nb, :kb] if how == "rows" else \
            torch.full((B, kb + 1, nb + 3), 77.0, device="cuda")[:, :kb, :nb].transpose(1, 2)
        s = cn.make_quantize_shape(x, q, scale, block_rows=tile)
        got, scale = cn.quantize_fp8(x, s, Q=q, scale=scale)
        assert torch.equal(scale.double(), s64) and torch.equal(got.double(), q64)
        if how != "own":
            assert int((scale._base != 77.0).sum()) <= scale.numel()
    buf[:, :N, :K] = 77
    assert (buf == 77).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_borders(dtype):
    """Blocks whose largest magnitude is at, just below and just above 448 times a power of two; every midpoint between neighbouring values; the smallest steps; zeros;
    magnitudes at both ends of the type."""
    t = DTYPES[dtype]
    rows = []
    for top in (448.0, 447.0 if dtype == "f32" else 446.0, 450.0, 256.0, 255.0, 1.0, 2.0 ** -90, 2.0 ** -120, 2.0 ** 100, 0.0):
        fine = torch.arange(0, 127, device="cuda").float() / 126 * 512 - 256       # at multiples of 1/16 of a step and more
        mids = torch.cat([torch.arange(16, 32, device="cuda").float() * 2.0 ** e + 2.0 ** (e - 1) for e in range(-14, -7)])[:126]
        tiny = torch.arange(-63, 63, device="cuda").float() * 2.0 ** -11
        for body in (fine, mids, tiny):
            r = torch.zeros(128, device="cuda")
            r[1:1 + len(body)] = body * (top / 512 if body is fine else 1.0)
            r[0] = top
            rows.append(r)
    x = torch.stack(rows).to(t)[None]
    q64, s64 = quantize_ref(x, 1)
    q, s = cn.quantize_fp8(x, cn.make_quantize_shape(x, None, None))
    assert torch.equal(s.double(), s64) and torch.equal(q.double(), q64)
    assert (q.double().abs() <= 448).all()


@pytest.mark.parametrize("tile", [1, 128])
def test_quantize_infinities_and_nan(tile):
    x = torch.randn((1, 256, 304), device="cuda").bfloat16()
    x[0, 3, 5], x[0, 4, 140], x[0, 200, 299] = float("nan"), float("-inf"), float("inf")
    q, s = cn.quantize_fp8(x, cn.make_quantize_shape(x, None, None, block_rows=tile))
    bad = torch.zeros_like(s, dtype=torch.bool)
    for r, c in ((3, 0), (4, 1), (200, 2)):
        bad[0, r // tile, c] = True
    assert torch.equal(s.isnan(), bad)
    wide = bad.repeat_interleave(tile, 1).repeat_interleave(128, 2)[:, :, :304]
    assert torch.equal(q.float().isnan(), wide)
    y = torch.where(wide, torch.zeros_like(x), x)
    q2, s2 = cn.quantize_fp8(y, cn.make_quantize_shape(y, None, None, block_rows=tile))
    assert torch.equal(torch.where(wide, 0.0, q.float()), torch.where(wide, 0.0, q2.float())) and torch.equal(s[~bad], s2[~bad])


# ---- the product -----------------------------------------------------------------------------------------
def eight(shape, gen, extra=0):
    """e4m3 values of every size in rows on 16-byte boundaries, NaN behind them."""
    wide = -(-shape[-1] // 16) * 16 + 16
    buf = torch.full((*shape[:-2], shape[-2] + extra, wide), 0x7F, dtype=torch.uint8, device="cuda")
    view = buf.view(E4M3)[..., :shape[-2], :shape[-1]]
    view.copy_(torch.randn(shape, device="cuda", generator=gen) * 40)
    return view


def make(B, N, K, M, x="bf16", y="bf16", p="bf16", bias=True, gate=True, residual=True, seed=0, extra=1, powers=False):
    """powers: every scale is a power of two, as quantize_fp8 makes them (and the tensor cores apply them); else any number (and the epilogue does)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kb = -(-K // 128)

    def size(*n):
        return torch.exp2(torch.randint(-2, 3, n, device="cuda", generator=gen).float()) if powers else torch.exp(0.5 * torch.randn(n, device="cuda", generator=gen))
    t = dict(x_scale=None, y=y)
    if x == "e4m3":
        t["x"] = eight((B, N, K), gen, extra)
        t["x_scale"] = torch.full((B, kb, N + 5 + extra), float("nan"), device="cuda")[:, :, :N].transpose(1, 2).copy_(size(B, N, kb) / (32 if powers else 40))
    else:
        t["x"] = padded((B, N, K), DTYPES[x], gen, extra=extra).mul_(size(B, N, 1).to(DTYPES[x]))
    t["w"] = eight((M, K), gen)
    t["w_scale"] = torch.full((-(-M // 128), kb + 2), float("nan"), device="cuda")[:, :kb].copy_(size(-(-M // 128), kb) * (2.0 ** round(math.log2(1 / K ** 0.5)) / 32 if powers else 1.5 / 40 / K ** 0.5))
    vec = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
    t["bias"] = vec(M).to(DTYPES[p]) if bias else None
    t["gate"] = vec(B, 6, M)[:, 2].to(DTYPES[p]) if gate else None
    t["residual"] = padded((B, N, M), DTYPES[y], gen, extra=extra) if residual else None
    return t


def call(t, act, extra=1, Y=None):
    B, N, _ = t["x"].shape
    M = t["w"].shape[0]
    buf, y = canvas((B, N, M), DTYPES[t["y"]], extra=extra)
    s = cn.make_linear_fp8_shape(t["x"], t["w"], t["w_scale"], y, x_scale=t["x_scale"], residual=t["residual"], bias=t["bias"], gate=t["gate"], activation=act)
    ws = torch.full((cn.linear_fp8_workspace_bytes(s) + 256,), 255, dtype=torch.uint8, device="cuda")
    cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, x_scale=t["x_scale"], bias=t["bias"], gate=t["gate"], residual=t["residual"], Y=y, ws=ws[:-256])
    assert cn.query_status(ws) == cn.OK, cn.last_cuda_error()
    assert untouched(buf, y) and (ws[-256:] == 255).all()
    return y


def product_ref(t, act):
    """(y, allowed error before its rounding): the tensor cores lose at most a step of 2^-23 of a sum's magnitude for each product of 32 k they add to it (as layer_util's
    sum_error has it for 16 k of bf16), within a block or, with exponents, within a run; a block's own 4 products as much again, the scales' product is rounded once, and
    the sums over blocks, runs, warps and pairs add a rounding each: (K / 32 + 16) 2^-23 covers either way with (K / 128 + 40) 2^-24 beside it."""
    q, s = (t["x"].double(), t["x_scale"]) if t["x_scale"] is not None else quantize_ref(t["x"], 1)
    x, w = values(q, s), values(t["w"][None], t["w_scale"][None], 128)[0]
    z, mag = x @ w.T, x.abs() @ w.abs().T
    if t["bias"] is not None:
        z, mag = z + t["bias"].double(), mag + t["bias"].double().abs()
    ez = ((t["x"].shape[-1] / 32 + 16) * 2 + t["x"].shape[-1] / 128 + 40) * U32 * mag
    y = act64(z, act)
    ey = (SLOPE_MOST if act else 1.0) * ez + (ACT_ERR * (z.abs() + 1) if act else 0)
    if t["gate"] is not None:
        g = t["gate"].double()[:, None]
        y, ey = y * g, ey * g.abs() + U32 * (y * g).abs()
    if t["residual"] is not None:
        y = y + t["residual"].double()
        ey = ey + U32 * y.abs()
    return y, ey


def check_call(t, act, **kw):
    y = call(t, act, **kw)
    ry, ey = product_ref(t, act)
    check(y, ry, ey + half_step(y.dtype) * (ry.abs() + ey), "y")
    return y


# rows, in, out: single rows, both sides of the few-row kernel's limit, tile and block borders, odd everything, few tiles (shared k), many tiles (persistent)
SIZES = [(1, 1, 1), (1, 1536, 1536), (2, 37, 19), (7, 1541, 333), (8, 4096, 16), (9, 64, 130), (16, 5120, 40), (16, 200, 9000), (17, 5120, 40), (33, 65, 257),
         (64, 8, 8), (127, 1000, 129), (128, 128, 128), (129, 127, 300), (256, 256, 256), (257, 1541, 513), (300, 4099, 96), (513, 512, 1536), (700, 9000, 333),
         (1100, 200, 5000), (5003, 100, 2100), (64, 13000, 1536), (3000, 1536, 1536)]


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("x", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("N,K,M", SIZES)
def test_every_size(N, K, M, x, powers):
    check_call(make(1, N, K, M, x=x, seed=N + K + M, powers=powers), cn.ACT_GELU_TANH)


@pytest.mark.parametrize("x", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("B,N,K,M", [(1, 5, 300, 2500), (2, 4, 1541, 9001), (1, 11, 130, 4777), (1, 3, 1541, 10007), (2, 8, 520, 18001), (1, 1, 130, 19009), (1, 13, 700, 30001)])
def test_few_rows_into_many(B, N, K, M, x):
    """Tiles of W that share x: 1, 2 and 4 of them, up to 8 and up to 16 rows, the last ones in part."""
    check_call(make(B, N, K, M, x=x, seed=M), cn.ACT_SILU)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("B,N", [(3, 1), (2, 6), (2, 150), (3, 301)])
@pytest.mark.parametrize("x,y,p", [("bf16", "bf16", "f32"), ("e4m3", "f32", "bf16"), ("f32", "f32", "f32")])
@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("powers", [True, False])
def test_activations_types_and_entries(act, B, N, x, y, p, extra, powers):
    """extra = 1: a padded batch, whose entries do not follow each other evenly."""
    check_call(make(B, N, 200, 264, x, y, p, seed=N, extra=extra, powers=powers), act, extra=extra)


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("N,K,M", [(40, 30000, 64), (20, 70000, 40), (600, 20000, 700), (300, 5121, 2240), (9000, 3000, 1000)])
def test_long_sums(N, K, M, y, powers):
    """Runs of 5120 for fp32 outputs and of 65536 for bf16 ones, in one pair's hands or in several."""
    check_call(make(1, N, K, M, x="e4m3", y=y, powers=powers), cn.ACT_NONE)


def test_one_scale_that_is_no_power_of_two():
    """Anywhere, the last of all among them: the same result to within the roundings, by the other way."""
    base = make(1, 300, 1100, 500, x="e4m3", powers=True)
    want = check_call(base, cn.ACT_NONE)
    for name, at in (("w_scale", (3, 8)), ("w_scale", (0, 0)), ("x_scale", (0, 299, 8)), ("x_scale", (0, 0, 0))):
        for value in (3.0, 0.0, -0.25, 1.5 * 2.0 ** -127, 2.0 ** -127):
            t = {**base, name: base[name].clone()}
            t[name][at] = value
            check_call(t, cn.ACT_NONE)
    assert torch.equal(check_call(base, cn.ACT_NONE), want)


def test_scales_at_both_ends():
    """Exponents of every size whose products stay in range."""
    t = make(1, 150, 400, 300, x="e4m3", y="f32", bias=False, gate=False, residual=False)
    e = torch.arange(-120, 121, 60, device="cuda").float()
    t["x_scale"].copy_(torch.exp2(e[torch.arange(150, device="cuda") % 5])[None, :, None].expand(1, 150, 4))
    for shift in (0.0, 60.0, -60.0):
        t["w_scale"].fill_(2.0 ** -shift)
        keep = (e[torch.arange(150, device="cuda") % 5] - shift).abs() <= 100
        y, (ry, ey) = call(t, cn.ACT_NONE), product_ref(t, cn.ACT_NONE)
        check(y[:, keep], ry[:, keep], (ey + half_step(y.dtype) * (ry.abs() + ey))[:, keep], "y")


@pytest.mark.parametrize("bias,gate,residual", [(False, False, False), (True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("N", [3, 200])
def test_parts_that_are_left_out(bias, gate, residual, N):
    t = make(2, N, 130, 96, bias=bias, gate=gate, residual=residual)
    for act in (cn.ACT_NONE, cn.ACT_SILU):
        check_call(t, act)


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("N", [4, 40, 500])
def test_sums_are_taken_in_32_bits(N, powers):
    """fp32 outputs: blocks of different scale, positive terms only.  A sum of 5120 terms in the tensor cores is cut off at each of its 160 products, by half a step of 2^-23 of what it
    has reached on average, which is half of the result on average: 80 times 2^-24; sums of blocks in the epilogue lose less."""
    t = make(1, N, 5120, 300, x="e4m3", y="f32", bias=False, gate=False, residual=False, powers=powers)
    t["x"].copy_(t["x"].float().abs())
    t["w"].copy_(t["w"].float().abs())
    y = check_call(t, cn.ACT_NONE)
    ry, _ = product_ref(t, cn.ACT_NONE)
    assert (y.double() - ry).norm() <= 80 * U32 * ry.norm()


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("N", [5, 300])
def test_a_nan_stays_in_its_row_or_column(N, powers):
    t = make(1, N, 300, 400, bias=False, gate=False, residual=False, powers=powers)
    clean = call(t, cn.ACT_NONE)
    t["x"][0, 2, 140], t["w_scale"][1, 2] = float("inf"), float("nan")
    y = call(t, cn.ACT_NONE)
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[0, 2], bad[0, :, 128:256] = True, True
    assert torch.equal(y.isnan(), bad) and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("N", [3, 130, 2000])
def test_residual_in_place_and_the_same_bits_every_time(N, powers):
    t = make(2, N, 700, 520, y="f32", powers=powers)
    want = call(t, cn.ACT_SILU)
    for _ in range(3):
        y = t["residual"].clone()
        s = cn.make_linear_fp8_shape(t["x"], t["w"], t["w_scale"], y, residual=y, bias=t["bias"], gate=t["gate"], activation=cn.ACT_SILU)
        cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, bias=t["bias"], gate=t["gate"], residual=y, Y=y)
        assert torch.equal(y, want)


@pytest.mark.parametrize("powers", [True, False])
@pytest.mark.parametrize("N", [9, 17, 777])
def test_quantized_by_the_call_or_before_it(N, powers):
    """The same bits either way."""
    t = make(2, N, 645, 390, powers=powers)
    y = call(t, cn.ACT_GELU)
    q, s = cn.quantize_fp8(t["x"], cn.make_quantize_shape(t["x"], None, None))
    assert torch.equal(y, call({**t, "x": q, "x_scale": s}, cn.ACT_GELU))
    assert torch.equal(y, call({**t, "x": q, "x_scale": s.contiguous()}, cn.ACT_GELU))


def test_captured_and_on_two_streams():
    """Two graphs with a workspace each, replayed together on two streams, over inputs that change."""
    ts = [make(1, n, 1536, 768, seed=n, powers=n == 300) for n in (300, 12, 200)]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in ts]
    for t in ts:
        y = torch.empty((1, t["x"].shape[1], 768), dtype=torch.bfloat16, device="cuda")
        s = cn.make_linear_fp8_shape(t["x"], t["w"], t["w_scale"], y, residual=t["residual"], bias=t["bias"], gate=t["gate"])
        ws = torch.empty(cn.linear_fp8_workspace_bytes(s), dtype=torch.uint8, device="cuda")
        cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, bias=t["bias"], gate=t["gate"], residual=t["residual"], Y=y, ws=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, bias=t["bias"], gate=t["gate"], residual=t["residual"], Y=y, ws=ws)
        graphs.append((g, ws))
        outs.append(y)
    for k in range(4):
        for t in ts:
            t["x"].copy_(torch.randn(t["x"].shape, device="cuda") * (k + 1))
        torch.cuda.synchronize()
        for (g, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for t, y, (_, ws) in zip(ts, outs, graphs):
            assert cn.query_status(ws) == cn.OK
            assert torch.equal(y, call(t, cn.ACT_NONE))


def test_captured_with_scales_that_change():
    """A graph whose scales are powers of two in some replays and any numbers in others: each replay looks at its own."""
    t = make(2, 150, 700, 300, x="e4m3", powers=True)
    other = make(2, 150, 700, 300, x="e4m3", powers=False, seed=1)
    _, y = canvas((2, 150, 300), torch.bfloat16)
    s = cn.make_linear_fp8_shape(t["x"], t["w"], t["w_scale"], y, x_scale=t["x_scale"], residual=t["residual"], bias=t["bias"], gate=t["gate"])
    ws = torch.empty(cn.linear_fp8_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    kw = dict(x_scale=t["x_scale"], bias=t["bias"], gate=t["gate"], residual=t["residual"], Y=y, ws=ws)
    cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, **kw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, **kw)
    powers = {k: t[k].clone() for k in ("x_scale", "w_scale")}
    for xs, wsc in ((powers, powers), (other, powers), (powers, other), (powers, powers), (other, other), (powers, powers)):
        t["x_scale"].copy_(xs["x_scale"])
        t["w_scale"].copy_(wsc["w_scale"])
        g.replay()
        torch.cuda.synchronize()
        assert cn.query_status(ws) == cn.OK
        ry, ey = product_ref(t, cn.ACT_NONE)
        check(y, ry, ey + half_step(y.dtype) * (ry.abs() + ey), "y")


@pytest.mark.parametrize("at", [None, (0, 0, 0), (1299, 16, 1)])
def test_many_padded_entries(at):
    """Entries that do not follow each other evenly, more of them than a pass over the scales has CTAs; one scale, the first or the last, that is no power of two."""
    t = make(1300, 17, 200, 72, x="e4m3", powers=True)
    if at:
        t["x_scale"][at] *= 1.5
    check_call(t, cn.ACT_NONE)


def test_offsets_that_pass_32_bits():
    """600000 rows of 4096, 2.4e9 bytes: the last rows against the same rows on their own."""
    rows, wide, tail = 600_000, 4096, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros((1, rows, wide), dtype=torch.bfloat16, device="cuda")
    x[:, -tail:] = torch.randn((tail, wide), device="cuda", generator=gen)
    last = x[:, -tail:].clone()
    q, s = cn.quantize_fp8(x, cn.make_quantize_shape(x, None, None))
    q1, s1 = cn.quantize_fp8(last, cn.make_quantize_shape(last, None, None))
    assert torch.equal(q[:, -tail:].float(), q1.float()) and torch.equal(s[:, -tail:], s1)
    w = eight((64, wide), gen)
    ws = torch.full((1, 32), 2.0 ** -6, device="cuda")
    t = dict(x=x, w=w, w_scale=ws, x_scale=None, y="bf16", bias=None, gate=None, residual=None)
    y = call(t, cn.ACT_NONE)
    assert torch.equal(y, call({**t, "x": q, "x_scale": s}, cn.ACT_NONE)) and not y[:, :-tail].any()
    ry, ey = product_ref({**t, "x": last}, cn.ACT_NONE)
    check(y[:, -tail:], ry, ey + half_step(y.dtype) * (ry.abs() + ey), "y")
    # into that width
    up = eight((wide, 64), gen)
    small = torch.zeros((1, rows, 64), device="cuda")
    small[:, -tail:] = torch.randn((tail, 64), device="cuda", generator=gen)
    t = dict(x=small, w=up, w_scale=torch.full((32, 1), 2.0 ** -4, device="cuda"), x_scale=None, y="bf16", bias=None, gate=None, residual=None)
    s = cn.make_linear_fp8_shape(small, up, t["w_scale"], x)
    _, wk = cn.linear_fp8(small, up, t["w_scale"], s, Y=x)
    assert cn.query_status(wk) == cn.OK
    ry, ey = product_ref({**t, "x": small[:, -tail:]}, cn.ACT_NONE)
    check(x[:, -tail:], ry, ey + half_step(x.dtype) * (ry.abs() + ey), "y")
    assert not x[:, :-tail].any()


@pytest.mark.parametrize("powers,most", [(True, 32), (False, 16)])
@pytest.mark.parametrize("N,K,M", [(4, 5120, 300), (40, 5120, 300), (500, 5120, 300), (300, 10240, 300), (4, 10240, 300), (2000, 5120, 2240), (2000, 10240, 2240)])
def test_sums_of_blocks_and_of_runs(N, K, M, powers, most):
    """fp32 outputs, positive terms only.  Any scales: the tensor cores sum up one block, four products of 32 k, each of which cuts off at most 2^-23 of what the block has reached, 5/8 of
    it on average: 5 times 2^-24; the scales' product is rounded once: 1; K / 128 sums are rounded to nearest, half a step of what each has reached, half of the result on average, up or
    down: 0.58 sqrt(K / 384) 2^-24, 3 at K = 10240, three times that allowed: 16 in all.  Powers of two: runs of 2560 at most, 80 products, each of which cuts off half a step on average;
    a step is 2^-24 to 2^-23 of what the run has reached, 1.44 2^-24 on average, and the run has reached half of its sum on average: 80 x 0.72 / 2 = 29, and 3 for joining: 32."""
    t = make(1, N, K, M, x="e4m3", y="f32", bias=False, gate=False, residual=False, powers=powers)
    t["x"].copy_(t["x"].float().abs())
    t["w"].copy_(t["w"].float().abs())
    y = call(t, cn.ACT_NONE)
    ry, _ = product_ref(t, cn.ACT_NONE)
    assert (y.double() - ry).norm() <= most * U32 * ry.norm()


@pytest.mark.parametrize("x", ["bf16", "e4m3"])
def test_a_record_with_a_residual_used_without(x):
    """A padded residual keeps the record's entries apart; the call without it takes them as one run, in the workspace that the record asks for."""
    t = make(5, 60, 700, 264, x=x, extra=0, powers=True)
    if x == "e4m3":
        t["x_scale"] = t["x_scale"].contiguous()
    apart = padded((5, 60, 264), torch.bfloat16, torch.Generator(device="cuda").manual_seed(1), extra=3)
    _, y = canvas((5, 60, 264), torch.bfloat16)
    s = cn.make_linear_fp8_shape(t["x"], t["w"], t["w_scale"], y, x_scale=t["x_scale"], residual=apart, bias=t["bias"], gate=t["gate"])
    for residual in (apart, None):
        need = cn.linear_fp8_workspace_bytes(s)
        ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
        cn.linear_fp8(t["x"], t["w"], t["w_scale"], s, x_scale=t["x_scale"], bias=t["bias"], gate=t["gate"], residual=residual, Y=y, ws=ws[:need])
        assert cn.query_status(ws) == cn.OK and (ws[need:] == 255).all()
        ry, ey = product_ref({**t, "residual": residual}, cn.ACT_NONE)
        check(y, ry, ey + half_step(y.dtype) * (ry.abs() + ey), "y")


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_many_padded_entries_quantised_by_the_call(x):
    """CTAs of every entry's rows, and behind them those of the weight's scales."""
    for w_scale in (1.0, 1.5):
        t = make(1300, 17, 200, 72, x=x, powers=True)
        t["w_scale"] *= w_scale
        check_call(t, cn.ACT_NONE)
