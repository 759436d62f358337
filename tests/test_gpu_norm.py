"""Layer norm and its gradients against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import DTYPES, U32, canvas, check, depth, half_step, norm_ref, padded, untouched, xh_error

pytestmark = pytest.mark.gpu

EPS = 1e-6


def make(B, H, N, C, x, y, p, affine, mod, seed=0, heads=False, scale=1.0, offset=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = {}
    if heads:           # the first of three parts of a fused projection's output, [B,N,3,H,C]
        t["x"] = (torch.randn((B, N, 3, H, C), device="cuda", generator=gen) * scale + offset).to(DTYPES[x])[:, :, 0].permute(0, 2, 1, 3)
    else:
        t["x"] = padded((B, H, N, C), DTYPES[x], gen, scale, extra=1)
        t["x"] += offset
    t["dy"] = padded((B, H, N, C), DTYPES[y], gen)
    vec = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
    t["weight"] = (1 + 0.3 * vec(C)).to(DTYPES[p]) if affine else None
    t["bias"] = (0.3 * vec(C)).to(DTYPES[p]) if affine else None
    six = 0.4 * vec(B, 6, C)
    t["shift"], t["scale"] = (six[:, 1], six[:, 4]) if mod else (None, None)
    return t


def forward(t, y_dtype, eps=EPS):
    x = t["x"]
    buf, y = canvas(x.shape, y_dtype, extra=1)
    s = cn.make_norm_shape(x, y, t["weight"], t["scale"], shift=t["shift"], eps=eps)
    mean, rstd = (torch.full(x.shape[:3], float("nan"), device="cuda") for _ in range(2))
    out = cn.layer_norm(x, s, weight=t["weight"], bias=t["bias"], shift=t["shift"], scale=t["scale"], Y=y, mean=mean, rstd=rstd)
    assert out.data_ptr() == y.data_ptr()
    assert untouched(buf, y)
    return y, mean, rstd


def check_forward(t, y, mean, rstd, eps=EPS):
    ref, m, r, xh, a, c = norm_ref(t["x"], t["weight"], t["bias"], t["shift"], t["scale"], eps)
    e = xh_error(t["x"], m, r, xh)
    check(mean, m, 44 * U32 * t["x"].double().abs().amax(-1), "mean")
    check(rstd, r, r * (70 * U32 + 2 * 44 * U32 * t["x"].double().abs().amax(-1) * r), "rstd")
    check(y, ref, e * a.abs() + 4 * U32 * ((xh * a).abs() + c.abs()) + half_step(y.dtype) * ref.abs(), "y")


def check_backward(t, g, mean, rstd):
    x, dy = t["x"].double(), t["dy"].double()
    _, _, _, _, a, _ = norm_ref(t["x"], t["weight"], t["bias"], t["shift"], t["scale"], EPS)
    r = rstd.double()[..., None]
    xh = (x - mean.double()[..., None]) * r             # the call is given the statistics
    e_xh = 3 * U32 * (xh.abs() + (x.abs() + mean.double()[..., None].abs()) * r)
    C = x.shape[-1]
    gg = dy * a
    m1, m2 = gg.mean(-1, keepdim=True), (gg * xh).mean(-1, keepdim=True)
    ref = r * (gg - m1 - xh * m2)
    # sums over a row are 44 additions deep at most (see xh_error)
    e1 = 48 * U32 * gg.abs().mean(-1, keepdim=True)
    e2 = 48 * U32 * (gg * xh).abs().mean(-1, keepdim=True) + (gg.abs() * e_xh).mean(-1, keepdim=True)
    tol = r * (4 * U32 * (gg.abs() + m1.abs() + (xh * m2).abs()) + e1 + xh.abs() * e2 + e_xh * m2.abs())
    check(g.dX, ref, tol + half_step(g.dX.dtype) * ref.abs(), "dX")
    rows = x.shape[1] * x.shape[2]
    P, Pa, S, Sa = (dy * xh).sum((1, 2)), ((dy * xh).abs() * (depth(rows) * U32) + dy.abs() * e_xh).sum((1, 2)), dy.sum((1, 2)), dy.abs().sum((1, 2)) * depth(rows) * U32
    k = 1 + t["scale"].double() if t["scale"] is not None else torch.ones((x.shape[0], 1), dtype=torch.float64, device="cuda")
    B = x.shape[0]
    if t["weight"] is not None:
        check(g.dweight, (k * P).sum(0), (k.abs() * Pa).sum(0) + (B + 4) * U32 * (k * P).abs().sum(0), "dweight")
        check(g.dbias, (k * S).sum(0), (k.abs() * Sa).sum(0) + (B + 4) * U32 * (k * S).abs().sum(0), "dbias")
    else:
        assert g.dweight is None and g.dbias is None
    if t["scale"] is not None:
        w = t["weight"].double() if t["weight"] is not None else torch.ones(C, dtype=torch.float64, device="cuda")
        b = t["bias"].double() if t["bias"] is not None else torch.zeros(C, dtype=torch.float64, device="cuda")
        check(g.dshift, S, Sa + U32 * S.abs(), "dshift")
        check(g.dscale, w * P + b * S, w.abs() * Pa + b.abs() * Sa + 3 * U32 * ((w * P).abs() + (b * S).abs()), "dscale")
    else:
        assert g.dshift is None and g.dscale is None


def backward(t, mean, rstd):
    buf, dx = canvas(t["x"].shape, t["x"].dtype, extra=1)
    s = cn.make_norm_shape(t["x"], t["dy"], t["weight"], t["scale"], shift=t["shift"], dX=dx, eps=EPS)
    ws = torch.full((cn.layer_norm_backward_workspace_bytes(s),), 255, dtype=torch.uint8, device="cuda")
    g = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, weight=t["weight"], bias=t["bias"], scale=t["scale"], dX=dx, ws=ws)
    assert untouched(buf, dx)
    return g


WIDTHS = [1, 5, 8, 63, 64, 65, 128, 130, 256, 257, 511, 512, 513, 1000, 1536, 2047, 2049, 5120, 8192, 8193, 16384]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_every_width_and_type(C, x, y):
    t = make(2, 1, 37, C, x, y, "f32" if C % 2 else "bf16", affine=True, mod=True, seed=C)
    out, mean, rstd = forward(t, DTYPES[y])
    check_forward(t, out, mean, rstd)
    check_backward(t, backward(t, mean, rstd), mean, rstd)


@pytest.mark.parametrize("B,H,N", [(1, 1, 1), (3, 1, 1), (1, 1, 5003), (2, 3, 700), (5, 1, 149), (300, 1, 2)])
@pytest.mark.parametrize("C", [64, 1536])
@pytest.mark.parametrize("affine,mod", [(True, False), (False, True), (False, False)])
def test_rows_entries_and_what_there_is(B, H, N, C, affine, mod):
    t = make(B, H, N, C, "bf16", "bf16", "bf16", affine, mod, seed=N)
    out, mean, rstd = forward(t, torch.bfloat16)
    check_forward(t, out, mean, rstd)
    check_backward(t, backward(t, mean, rstd), mean, rstd)


@pytest.mark.parametrize("C", [64, 128, 96])
def test_heads_of_a_fused_projection_in_place(C):
    """Q of [B,N,3,H,C]: normalised where it lies, K and V beside it stay as they are."""
    B, H, N = 2, 5, 333
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn((B, N, 3, H, C), device="cuda", generator=gen).bfloat16()
    t = make(B, H, N, C, "bf16", "bf16", "f32", True, False)
    t["x"] = qkv[:, :, 0].permute(0, 2, 1, 3)
    before, rest = t["x"].clone(), qkv[:, :, 1:].clone()
    s = cn.make_norm_shape(t["x"], t["x"], t["weight"], eps=EPS)
    cn.layer_norm(t["x"], s, weight=t["weight"], bias=t["bias"], Y=t["x"])
    y = t["x"].clone()
    assert torch.equal(qkv[:, :, 1:], rest)
    t["x"] = before
    ref, m, r, xh, a, c = norm_ref(before, t["weight"], t["bias"], None, None, EPS)
    check(y, ref, xh_error(before, m, r, xh) * a.abs() + 4 * U32 * ((xh * a).abs() + c.abs()) + half_step(y.dtype) * ref.abs(), "y")


@pytest.mark.parametrize("C", [128, 1000, 5120])
@pytest.mark.parametrize("scale,offset", [(1.0, 1000.0), (1e-3, 3.0), (1e4, -1e4), (0.0, 2.5), (0.0, 0.0), (1e-12, 0.0)])
def test_large_means_and_constant_rows(C, scale, offset):
    t = make(1, 1, 33, C, "f32", "f32", "f32", True, False, seed=3, scale=scale, offset=offset)
    out, mean, rstd = forward(t, torch.float32)
    check_forward(t, out, mean, rstd)
    check_backward(t, backward(t, mean, rstd), mean, rstd)


def test_a_row_that_is_not_finite_keeps_to_itself():
    t = make(1, 1, 40, 1536, "f32", "bf16", "f32", True, False)
    clean = forward(t, torch.bfloat16)[0].clone()
    t["x"][0, 0, 7, 100] = float("inf")
    t["x"][0, 0, 9, 3] = float("nan")
    y = forward(t, torch.bfloat16)[0]
    keep = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(y[:, :, keep], clean[:, :, keep])
    assert not torch.isfinite(y[0, 0, 7]).any() and torch.isnan(y[0, 0, 9]).all()


def test_shared_modulation_and_broadcast_input():
    """One shift and scale for all entries (batch stride 0); an input that all entries share."""
    t = make(1, 1, 50, 640, "bf16", "bf16", "bf16", True, True, seed=5)
    t["x"] = t["x"].expand(4, 1, 50, 640)
    t["dy"] = padded((4, 1, 50, 640), torch.bfloat16, torch.Generator(device="cuda").manual_seed(2))
    t["shift"], t["scale"] = t["shift"].expand(4, 640), t["scale"].expand(4, 640)
    out, mean, rstd = forward(t, torch.bfloat16)
    check_forward(t, out, mean, rstd)
    check_backward(t, backward(t, mean, rstd), mean, rstd)


def test_vectors_that_are_aligned_to_their_type_only():
    t = make(2, 1, 20, 640, "bf16", "bf16", "f32", True, True)
    raw = torch.randn(4000, device="cuda")
    t["weight"], t["bias"] = raw[1:641], raw[643:1283]
    t["scale"], t["shift"] = raw[5:2 * 641 + 5].view(2, 641)[:, :640], raw[1290:2 * 643 + 1290].view(2, 643)[:, 2:642]
    out, mean, rstd = forward(t, torch.bfloat16)
    check_forward(t, out, mean, rstd)
    check_backward(t, backward(t, mean, rstd), mean, rstd)


def test_gradients_overwrite_their_inputs():
    t = make(1, 1, 300, 1536, "bf16", "bf16", "bf16", True, False)
    _, mean, rstd = forward(t, torch.bfloat16)
    ref = backward(t, mean, rstd)
    for name in ("dy", "x"):
        u = {k: v.clone() if torch.is_tensor(v) else v for k, v in t.items()}
        s = cn.make_norm_shape(u["x"], u["dy"], u["weight"], dX=u[name], eps=EPS)
        g = cn.layer_norm_backward(u["dy"], u["x"], mean, rstd, s, weight=u["weight"], bias=u["bias"], dX=u[name])
        assert torch.equal(g.dX, ref.dX) and torch.equal(g.dweight, ref.dweight) and torch.equal(g.dbias, ref.dbias)


def test_only_what_is_wanted():
    t = make(2, 1, 100, 200, "bf16", "bf16", "bf16", True, True)
    _, mean, rstd = forward(t, torch.bfloat16)
    s = cn.make_norm_shape(t["x"], t["dy"], t["weight"], t["scale"], eps=EPS, dX=t["x"].clone())
    full = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, weight=t["weight"], bias=t["bias"], scale=t["scale"])
    for name, field in dict(weight="dweight", bias="dbias", shift="dshift", scale="dscale").items():
        g = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, weight=t["weight"], bias=t["bias"], scale=t["scale"], want=(name,))
        assert torch.equal(getattr(g, field), getattr(full, field)) and torch.equal(g.dX, full.dX)
        assert all(v is None for f, v in g._asdict().items() if f not in ("dX", field))
    g = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, weight=t["weight"], bias=t["bias"], scale=t["scale"], want=())
    assert torch.equal(g.dX, full.dX)


@pytest.mark.parametrize("C", [96, 700])
def test_gradients_against_differences(C):
    """The loss <dy, y> moves by <gradient, direction> h to first order: central differences of the forward call, fp32 throughout."""
    t = make(2, 1, 24, C, "f32", "f32", "f32", True, True, seed=C)
    _, mean, rstd = forward(t, torch.float32)
    g = backward(t, mean, rstd)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for name, grad in (("x", g.dX), ("weight", g.dweight), ("bias", g.dbias), ("shift", g.dshift), ("scale", g.dscale)):
        v = torch.randn(t[name].shape, device="cuda", generator=gen)
        h, loss = 2.0 ** -7, []
        for sign in (1, -1):
            u = dict(t)
            u[name] = t[name] + sign * h * v
            y = forward(u, torch.float32)[0]
            loss.append((y.double() * t["dy"].double()).sum())
        slope = (loss[0] - loss[1]) / (2 * h)
        ref = (grad.double() * v.double()).sum()
        # y's rounding errors (64 U32 of values about 1, independent) against h, and the third-order term, h^2 |v|^3 sums, of x alone
        noise = 64 * U32 * t["dy"].double().norm() / h
        third = h * h * (t["dy"].double().abs() * (1 + v.double().abs() ** 3)).sum() * 4 if name == "x" else 0
        assert abs(slope - ref) <= noise + third + 1e-5 * abs(ref), name


def test_same_bits_again_streams_and_graphs():
    t = make(2, 1, 700, 1536, "f32", "bf16", "f32", True, True)
    y0, mean, rstd = forward(t, torch.bfloat16)
    g0 = backward(t, mean, rstd)
    s = cn.make_norm_shape(t["x"], y0, t["weight"], t["scale"], shift=t["shift"], eps=EPS)
    sb = cn.make_norm_shape(t["x"], t["dy"], t["weight"], t["scale"], shift=t["shift"], dX=t["x"], eps=EPS)
    run = lambda: (cn.layer_norm(t["x"], s, weight=t["weight"], bias=t["bias"], shift=t["shift"], scale=t["scale"], Y=y),  # noqa: E731
                   cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, sb, weight=t["weight"], bias=t["bias"], scale=t["scale"], dX=dx))
    y, dx = canvas(y0.shape, torch.bfloat16, extra=1)[1], torch.empty_strided(t["x"].shape, t["x"].stride(), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _, g = run()
    side.synchronize()
    assert torch.equal(y, y0) and all(torch.equal(a, b) for a, b in zip(g, g0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, g = run()
    for _ in range(2):
        y.zero_(), dx.zero_(), g.dweight.zero_(), g.dscale.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y0) and all(torch.equal(a, b) for a, b in zip(g, g0))


def test_gradients_of_a_norm_that_is_shifted_only():
    t = make(2, 1, 90, 264, "bf16", "f32", "f32", True, True, seed=6)
    t["scale"] = None
    out, mean, rstd = forward(t, torch.float32)
    check_forward(t, out, mean, rstd)
    s = cn.make_norm_shape(t["x"], t["dy"], t["weight"], shift=t["shift"], dX=t["x"].clone(), eps=EPS)
    g = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, weight=t["weight"], bias=t["bias"], modulated=True)
    one = dict(t, scale=torch.zeros((2, 264), device="cuda"))             # a scale of zero is no scale
    s = cn.make_norm_shape(t["x"], t["dy"], t["weight"], one["scale"], shift=t["shift"], dX=t["x"].clone(), eps=EPS)
    ref = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, weight=t["weight"], bias=t["bias"], scale=one["scale"])
    assert all(torch.equal(a, b) for a, b in zip(g, ref))


@pytest.mark.parametrize("C", [96, 1000, 1024, 1032, 1536, 5120, 16384])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_statistics_of_rows_that_are_not_finite(C, x):
    """By the formula: a NaN or an infinity makes the variance NaN, and so rstd and every channel of y, while the mean is what the channels sum up to.  On both
    sides of 1024 channels, from which on several warps share a row; in the first warp's channels and in later ones."""
    t = make(1, 1, 40, C, x, "f32", "f32", True, True)
    clean = [v.clone() for v in forward(t, torch.float32)]
    inf, nan = float("inf"), float("nan")
    bad = {3: (0, nan), 7: (C - 1, nan), 11: (0, inf), 12: (C - 1, inf), 20: (C // 2, -inf), 21: (C * 3 // 4, nan), 30: (0, inf)}
    for row, (c, v) in bad.items():
        t["x"][0, 0, row, c] = v
    t["x"][0, 0, 30, C - 1] = -inf
    y, mean, rstd = forward(t, torch.float32)
    keep = [i for i in range(40) if i not in bad]
    for got, was in zip((y, mean, rstd), clean):
        assert torch.equal(got[:, :, keep], was[:, :, keep])
    want = t["x"].double().mean(-1)
    for row in bad:
        assert torch.isnan(y[0, 0, row]).all() and torch.isnan(rstd[0, 0, row]), row
        assert torch.equal(mean[0, 0, row].double().nan_to_num(nan=7.0), want[0, 0, row].nan_to_num(nan=7.0)), row


@pytest.mark.parametrize("p", ["bf16", "f32"])
@pytest.mark.parametrize("C", [128, 1541])
def test_a_norm_with_a_bias_only(p, C):
    """As with a weight of ones: the same bits, the bias's gradient and the scale's, which reads the bias, among them."""
    t = make(2, 1, 90, C, "bf16", "bf16", p, True, True)
    ones = dict(t, weight=torch.ones_like(t["weight"]))
    y, mean, rstd = forward(ones, torch.bfloat16)
    ref = backward(ones, mean, rstd)
    s = cn.make_norm_shape(t["x"], y, None, t["scale"], shift=t["shift"], eps=EPS, bias=t["bias"])
    out = cn.layer_norm(t["x"], s, bias=t["bias"], shift=t["shift"], scale=t["scale"], Y=torch.empty_strided(y.shape, y.stride(), dtype=y.dtype, device="cuda"))
    assert torch.equal(out, y)
    s = cn.make_norm_shape(t["x"], t["dy"], None, t["scale"], shift=t["shift"], eps=EPS, bias=t["bias"])
    g = cn.layer_norm_backward(t["dy"], t["x"], mean, rstd, s, bias=t["bias"], scale=t["scale"])
    assert g.dweight is None and all(torch.equal(getattr(g, n), getattr(ref, n)) for n in ("dX", "dbias", "dshift", "dscale"))
