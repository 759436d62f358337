"""Norm, gate, residual stream and norm in one pass, and the gradients, against the formulas in 64 bits."""
import itertools

import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import DTYPES, U32, canvas, check, depth, half_step, padded, untouched, xh_error

pytestmark = pytest.mark.gpu

EPS1, EPS2 = 1e-5, 3e-6
NONE, LAYER, RMS = cn.NORM_NONE, cn.NORM_LAYER, cn.NORM_RMS
VECTORS = ("post_weight", "post_bias", "gate", "weight", "bias", "shift", "scale")


def make(B, N, C, r="f32", x="bf16", y="bf16", p="bf16", m="f32", have=VECTORS, post=RMS, pre=LAYER, alpha=1.0, seed=0, extra=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = dict(post=post, pre=pre, alpha=alpha, extra=extra, y_dtype=DTYPES[y])
    t["r"] = padded((B, N, C), DTYPES[r], gen, 2.0, extra=extra)
    t["r"] += torch.randn(C, device="cuda", generator=gen).to(DTYPES[r])          # channels of their own offset
    t["x"] = padded((B, N, C), DTYPES[x], gen, extra=extra)
    t["dy"], t["ds"] = padded((B, N, C), DTYPES[y], gen, extra=extra), padded((B, N, C), DTYPES[r], gen, extra=extra)
    vec = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
    of = dict(post_weight=1 + 0.3 * vec(C), post_bias=0.5 * vec(C), weight=1 + 0.3 * vec(C), bias=0.5 * vec(C))
    six = 0.5 * vec(B, 6, C)
    of.update(gate=six[:, 2], shift=six[:, 3], scale=six[:, 4])
    for k in VECTORS:
        t[k] = of[k].to(DTYPES[m if k in ("gate", "shift", "scale") else p]) if k in have else None
    return t


def record(t, S, Y, **kw):
    return cn.make_block_norm_shape(t["r"], t["x"], S, Y, **{k: t[k] for k in VECTORS}, post=t["post"], pre=t["pre"], post_eps=EPS1, eps=EPS2, residual_scale=t["alpha"], **kw)


def forward(t, keep=True, in_place=False):
    B, N, C = t["x"].shape
    sbuf, S = canvas((B, N, C), t["r"].dtype, extra=t["extra"])
    ybuf, Y = canvas((B, N, C), t["y_dtype"], extra=t["extra"])
    R = t["r"]
    if in_place:
        R = S.copy_(R)
    stats = torch.full((4, B, N), 77.0, device="cuda") if keep else None
    s = record({**t, "r": R}, S, Y)
    got = cn.block_norm(R, t["x"], s, **{k: t[k] for k in VECTORS}, S=S, Y=Y, stats=stats)
    assert got[0] is S and got[1] is Y and untouched(sbuf, S) and untouched(ybuf, Y)
    return S, Y, stats


def norm64(x, kind, eps, err=None):
    """(xh, mean, rstd, error of xh): that of layer_util.xh_error; an RMS norm has no mean to be off; `err`: what x itself is off by."""
    x = x.double()
    zero = torch.zeros_like(x[..., 0])
    if kind == NONE:
        return x, zero, zero + 1, torch.zeros_like(x) if err is None else err
    mean = x.mean(-1) if kind == LAYER else zero
    rstd = (((x - mean[..., None]) ** 2).mean(-1) + eps) ** -0.5
    xh = (x - mean[..., None]) * rstd[..., None]
    e = xh_error(x, mean, rstd, xh) if kind == LAYER else xh.abs() * (70 * U32)
    if err is not None:                  # through the mean, and through the deviation
        e = e + rstd[..., None] * (err + (err.mean(-1, keepdim=True) if kind == LAYER else 0)) + xh.abs() * (rstd[..., None] * (xh.abs() * err).mean(-1, keepdim=True))
    return xh, mean, rstd, e


def vec64(t, name, other):
    v = t[name]
    if v is None:
        return torch.full((), other, dtype=torch.float64, device="cuda")
    return v.double()[:, None] if v.dim() == 2 else v.double()


def check_forward(t, S, Y, stats):
    w1, b1, gate, w2, b2 = (vec64(t, *a) for a in (("post_weight", 1), ("post_bias", 0), ("gate", 1), ("weight", 1), ("bias", 0)))
    k, shift = 1 + vec64(t, "scale", 0), vec64(t, "shift", 0)
    xh, m1, r1, e1 = norm64(t["x"], t["post"], EPS1)
    p = (xh * w1 + b1) * gate
    r = t["r"].double() * float(torch.tensor(t["alpha"], dtype=torch.float32))
    s = r + p
    es = e1 * (w1 * gate).abs() + 4 * U32 * ((xh * w1 * gate).abs() + (b1 * gate).abs()) + U32 * (r.abs() + s.abs())
    check(S, s, es + half_step(S.dtype) * (s.abs() + es), "S")
    sh, m2, r2, e2 = norm64(s, t["pre"], EPS2, es)
    y = (sh * w2 + b2) * k + shift
    ey = e2 * (w2 * k).abs() + 4 * U32 * ((sh * w2 * k).abs() + (b2 * k).abs() + shift.abs())
    check(Y, y, ey + half_step(Y.dtype) * (y.abs() + ey), "Y")
    if stats is not None:
        big, em = t["x"].double().abs().amax(-1), es.mean(-1)
        check(stats[0], m1, 44 * U32 * big * (t["post"] == LAYER), "post mean")
        check(stats[2], m2, (44 * U32 * s.abs().amax(-1) + em) * (t["pre"] == LAYER), "pre mean")
        # relative: half of the squares' error, the mean's against the deviation, the input's, rsqrt
        check(stats[1], r1, r1 * (0 if t["post"] == NONE else 70 * U32 + 44 * U32 * big * r1), "post rstd")
        check(stats[3], r2, r2 * (70 * U32 + 44 * U32 * s.abs().amax(-1) * r2 + r2 * (sh.abs() * es).mean(-1) + r2 * em), "pre rstd")


def backward(t, S, stats, want=VECTORS, ds=True):
    B, N, C = t["x"].shape
    rbuf, dR = canvas((B, N, C), t["r"].dtype, extra=t["extra"])
    xbuf, dX = canvas((B, N, C), t["x"].dtype, extra=t["extra"])
    s = record(t, S, t["dy"], dS=t["ds"], dR=dR, dX=dX)
    ws = torch.full((cn.block_norm_backward_workspace_bytes(s) + 256,), 255, dtype=torch.uint8, device="cuda")
    g = cn.block_norm_backward(t["dy"], S, t["x"], stats, s, dS=t["ds"] if ds else None, **{k: t[k] for k in VECTORS if k != "shift"}, dR=dR, dX=dX, want=want,
                               modulated=t["scale"] is not None or t["shift"] is not None, ws=ws[:-256])
    assert untouched(rbuf, dR) and untouched(xbuf, dX) and (ws[-256:] == 255).all()
    return g


def gradients64(t, S, stats, ds=True):
    """name -> (gradient, allowed error before its own rounding): every value is a few roundings (U32 of it each) from its operands; a mean over the channels is a sum at most 48
    additions deep (16 in a lane, 5 across it, 16 over the warps, and room), one over the rows depth(N)."""
    w1, b1, gate, w2, b2 = (vec64(t, *a) for a in (("post_weight", 1), ("post_bias", 0), ("gate", 1), ("weight", 1), ("bias", 0)))
    k = 1 + vec64(t, "scale", 0)
    m1, r1, m2, r2 = stats.double()[..., None]
    if t["post"] != LAYER:
        m1 = m1 * 0
    if t["post"] == NONE:
        r1 = r1 * 0 + 1
    if t["pre"] != LAYER:
        m2 = m2 * 0
    bar = lambda v: v.mean(-1, keepdim=True)  # noqa: E731
    dy, sh, xh = t["dy"].double(), (S.double() - m2) * r2, (t["x"].double() - m1) * r1
    d = t["ds"].double() if ds else torch.zeros_like(sh)
    v = dy * w2 * k
    G = d + r2 * (v - (bar(v) if t["pre"] == LAYER else 0) - sh * bar(v * sh))
    eG = r2 * (8 * U32 * v.abs() + 60 * U32 * bar(v.abs()) + 70 * U32 * sh.abs() * bar((v * sh).abs())) + 3 * U32 * (d.abs() + G.abs())
    q = G * gate * w1
    eq = eG * (gate * w1).abs() + 4 * U32 * q.abs()
    dX, eX = q, eq
    if t["post"] != NONE:
        dX = r1 * (q - (bar(q) if t["post"] == LAYER else 0) - xh * bar(q * xh))
        eX = r1 * (eq + bar(eq) + 60 * U32 * bar(q.abs()) + xh.abs() * (bar(eq * xh.abs()) + 70 * U32 * bar((q * xh).abs()))) + \
            6 * U32 * r1 * (q.abs() + bar(q.abs()) + xh.abs() * bar((q * xh).abs()))
    alpha = float(torch.tensor(t["alpha"], dtype=torch.float32))
    out = dict(dR=(alpha * G, abs(alpha) * (eG + U32 * G.abs())), dX=(dX, eX))
    n = depth(dy.shape[1])
    rows = {}
    for name, a, ea, b in (("P1", G, eG, xh), ("S1", G, eG, None), ("P2", dy, 0 * dy, sh), ("S2", dy, 0 * dy, None)):
        f = a if b is None else a * b
        e = ea if b is None else ea * b.abs() + 5 * U32 * f.abs()
        rows[name] = (f.sum(1), e.sum(1) + n * U32 * f.abs().sum(1))

    def mix(*pairs):                     # sum of factor x row sum
        val = sum(f * rows[s][0] for f, s in pairs)
        return val, sum(f.abs() * rows[s][1] + 4 * U32 * (f * rows[s][0]).abs() for f, s in pairs)
    flat = lambda f: f[:, 0] if f.dim() == 3 else f  # noqa: E731
    one = torch.ones((dy.shape[0], 1), dtype=torch.float64, device="cuda")
    g, kk = flat(gate) * one, flat(k) * one
    for name, f, s in (("dpost_weight", g, "P1"), ("dpost_bias", g, "S1"), ("dweight", kk, "P2"), ("dbias", kk, "S2")):
        val, e = mix((f, s))
        out[name] = (val.sum(0), e.sum(0) + dy.shape[0] * U32 * val.abs().sum(0))
    out["dgate"], out["dscale"], out["dshift"] = mix((w1, "P1"), (b1, "S1")), mix((w2, "P2"), (b2, "S2")), rows["S2"]
    return out


def check_backward(t, S, stats, g, ds=True):
    ref = gradients64(t, S, stats, ds)
    for name in g._fields:
        got = getattr(g, name)
        if got is not None:
            r, e = ref[name]
            check(got, r, e + half_step(got.dtype) * (r.abs() + e), name)


# channels: single ones, both sides of every change of the rows' forms (256, 512, 1024, 2048, 4096, 8192), odd ones
WIDTHS = [1, 7, 8, 64, 255, 256, 257, 511, 512, 513, 776, 1000, 1024, 1025, 1536, 1541, 2048, 2049, 3333, 4096, 4104, 5120, 6001, 8191, 8192]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("post,pre", [(RMS, LAYER), (LAYER, RMS)])
def test_every_width(C, post, pre):
    for N, types in ((1, ("f32", "bf16", "bf16", "bf16")), (37, ("f32", "f32", "f32", "f32")), (133, ("bf16", "bf16", "f32", "f32"))):
        t = make(2, N, C, *types, post=post, pre=pre, seed=C + N)
        S, Y, stats = forward(t)
        check_forward(t, S, Y, stats)
        check_backward(t, S, stats, backward(t, S, stats))


@pytest.mark.parametrize("r,x,y", list(itertools.product(["f32", "bf16"], repeat=3)))
@pytest.mark.parametrize("post", [NONE, LAYER, RMS])
@pytest.mark.parametrize("pre", [LAYER, RMS])
def test_types_and_kinds(r, x, y, post, pre):
    for p, m, C, extra in (("f32", "bf16", 520, 1), ("bf16", "f32", 1301, 0)):
        t = make(3, 50, C, r, x, y, p, m, post=post, pre=pre, alpha=0.75, extra=extra, seed=C)
        S, Y, stats = forward(t)
        check_forward(t, S, Y, stats)
        check_backward(t, S, stats, backward(t, S, stats))


@pytest.mark.parametrize("have", [(), ("gate",), ("post_weight",), ("post_bias",), ("weight",), ("bias",), ("shift",), ("scale",), ("gate", "shift", "scale"), ("post_bias", "bias", "gate"),
                                  ("post_weight", "weight")])
def test_parts_that_are_left_out(have):
    for post, pre, alpha in ((NONE, LAYER, 1.0), (LAYER, RMS, -2.0), (RMS, RMS, 0.0)):
        t = make(2, 20, 392, have=have, post=post, pre=pre, alpha=alpha)
        S, Y, stats = forward(t, in_place=True)
        check_forward(t, S, Y, stats)
        check_backward(t, S, stats, backward(t, S, stats, ds=False), ds=False)
        S2, Y2, _ = forward(t, keep=False)
        assert torch.equal(S, S2) and torch.equal(Y, Y2)


def test_only_what_is_wanted():
    t = make(2, 90, 640)
    S, _, stats = forward(t)
    full = backward(t, S, stats)
    for want in ((), ("gate",), ("weight", "post_bias"), ("shift", "scale", "post_weight")):
        g = backward(t, S, stats, want)
        for name in full._fields:
            got = getattr(g, name)
            if name in ("dR", "dX") or name[1:] in want:
                assert torch.equal(got, getattr(full, name)), name
            else:
                assert got is None


@pytest.mark.parametrize("N,C", [(3000, 1536), (700, 5120), (20000, 72)])
def test_many_rows_and_the_same_bits_every_time(N, C):
    t = make(2, N, C, seed=1)
    S, Y, stats = forward(t)
    check_forward(t, S, Y, stats)
    g = backward(t, S, stats)
    check_backward(t, S, stats, g)
    S2, Y2, stats2 = forward(t)
    assert torch.equal(S, S2) and torch.equal(Y, Y2) and torch.equal(stats, stats2)
    for a, b in zip(g, backward(t, S, stats)):
        assert torch.equal(a, b)


def test_gradients_in_place():
    """dR over dS and dX over X."""
    t = make(2, 77, 776, x="f32")
    S, _, stats = forward(t)
    want = backward(t, S, stats)
    ds, x = t["ds"].clone(), t["x"].clone()
    s = cn.make_block_norm_shape(None, x, S, t["dy"], **{k: t[k] for k in VECTORS}, dS=ds, dR=ds, dX=x, post=t["post"], pre=t["pre"], post_eps=EPS1, eps=EPS2)
    g = cn.block_norm_backward(t["dy"], S, x, stats, s, dS=ds, **{k: t[k] for k in VECTORS if k != "shift"}, dR=ds, dX=x)
    for a, b in zip(g, want):
        assert torch.equal(a, b)


def test_broadcast_input():
    """One row of x for every token and entry, one gate row for every entry: inputs with strides of 0."""
    t = make(3, 40, 264, extra=0)
    row = t["x"][:1, :1].clone()
    t["x"] = row.expand(3, 40, 264)
    t["gate"] = t["gate"][:1].expand(3, 264)
    S, Y, stats = forward(t)
    check_forward(t, S, Y, stats)
    _, dX = canvas((3, 40, 264), row.dtype)
    s = record(t, S, t["dy"], dS=t["ds"], dX=dX)
    g = cn.block_norm_backward(t["dy"], S, t["x"], stats, s, dS=t["ds"], **{k: t[k] for k in VECTORS if k != "shift"}, dX=dX)
    check_backward(t, S, stats, g)       # the broadcast inputs' gradients are the sums of these


@pytest.mark.parametrize("C", [100, 1536, 5120])
def test_rows_that_are_not_finite_stay_to_themselves(C):
    t = make(1, 30, C, x="f32", y="f32")
    clean = forward(t)
    t["x"][0, 3, C // 2], t["x"][0, 7, 5], t["r"][0, 11, C - 1], t["r"][0, 12, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    S, Y, stats = forward(t)
    keep = torch.ones(30, dtype=torch.bool, device="cuda")
    keep[[3, 7, 11, 12]] = False
    assert torch.equal(S[0, keep], clean[0][0, keep]) and torch.equal(Y[0, keep], clean[1][0, keep]) and torch.equal(stats[:, 0, keep], clean[2][:, 0, keep])
    assert Y[0, ~keep].isnan().all()


@pytest.mark.parametrize("post,pre", [(LAYER, LAYER), (RMS, RMS), (NONE, LAYER), (LAYER, RMS)])
def test_gradients_against_differentiation_and_differences(post, pre):
    """fp32 throughout: against torch's differentiation of the formula in 64 bits, and along random directions against central differences of it (step 1e-4 in 64 bits: off by
    1e-8 of the third derivative, and 1e-12 of the sum by rounding).  What the kernels' own gradients may be off by is gradients64's."""
    t = make(2, 9, 200, "f32", "f32", "f32", "f32", "f32", post=post, pre=pre, alpha=0.5, extra=0)
    S, _, stats = forward(t)
    names = ("r", "x", *VECTORS)
    leaf = {k: t[k].double().clone().requires_grad_() for k in names}

    def norm(v, kind, eps):
        if kind == NONE:
            return v
        mean = v.mean(-1, keepdim=True) if kind == LAYER else 0
        return (v - mean) / (((v - mean) ** 2).mean(-1, keepdim=True) + eps).sqrt()

    def loss(f):
        s = 0.5 * f["r"] + f["gate"][:, None] * (norm(f["x"], post, EPS1) * f["post_weight"] + f["post_bias"])
        y = (norm(s, pre, EPS2) * f["weight"] + f["bias"]) * (1 + f["scale"][:, None]) + f["shift"][:, None]
        return (t["dy"].double() * y).sum() + (t["ds"].double() * s).sum()
    loss(leaf).backward()
    g = backward(t, S, stats)
    got = dict(r=g.dR, x=g.dX, **{k: getattr(g, "d" + k) for k in VECTORS})
    ref = gradients64(t, S, stats)
    for k in names:
        # the saved S and statistics are rounded to 32 bits: as much again as gradients64 allows, 64 times over for what their errors pass through
        r, e = ref["d" + {"r": "R", "x": "X"}.get(k, k)]
        check(got[k], leaf[k].grad, 64 * (e + U32 * r.abs()), k)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(5):
        e = {k: torch.randn(t[k].shape, device="cuda", dtype=torch.float64, generator=gen) for k in names}
        with torch.no_grad():
            up, down = (loss({k: leaf[k] + h * e[k] for k in names}) for h in (1e-4, -1e-4))
        along = sum((got[k].double() * e[k]).sum() for k in names)
        size = sum((got[k].double().abs() * e[k].abs()).sum() for k in names)
        assert abs((up - down) / 2e-4 - along) <= 1e-5 * size


def test_captured_beside_an_eager_call():
    t = make(1, 64, 1024, extra=0)
    S, Y, stats = (v.clone() for v in forward(t))
    s = record(t, S, Y, dS=t["ds"])
    ws = torch.empty(cn.block_norm_backward_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    dR, dX = torch.empty_like(S), torch.empty_like(t["x"])
    s = record(t, S, Y, dS=t["ds"], dR=dR, dX=dX)
    vec = {k: t[k] for k in VECTORS}
    back = {k: t[k] for k in VECTORS if k != "shift"}

    def both():
        cn.block_norm(t["r"], t["x"], s, **vec, S=S, Y=Y, stats=stats)
        return cn.block_norm_backward(Y, S, t["x"], stats, s, dS=t["ds"], **back, dR=dR, dX=dX, ws=ws)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = both()
    for k in range(3):
        t["r"].copy_(torch.randn(t["r"].shape, device="cuda"))
        graph.replay()
        want = [v.clone() for v in g]
        e = both()
        for a, b in zip(e, want):
            assert torch.equal(a, b)


def test_offsets_that_pass_32_bits():
    rows, wide, tail = 600_000, 4096, 200
    gen = torch.Generator(device="cuda").manual_seed(1)
    r = torch.zeros((1, rows, wide), dtype=torch.bfloat16, device="cuda")
    x = torch.zeros_like(r)
    for v in (r, x):
        v[:, -tail:] = torch.randn((tail, wide), device="cuda", generator=gen)
    small = [v[:, -tail:].clone() for v in (r, x)]
    how = dict(post=LAYER, pre=RMS)
    stats, st = torch.empty((4, 1, rows), device="cuda"), torch.empty((4, 1, tail), device="cuda")
    s, y = cn.block_norm(r, x, cn.make_block_norm_shape(r, x, r, r, **how), S=r, stats=stats)
    s1, y1 = cn.block_norm(*small, cn.make_block_norm_shape(*small, small[0], small[0], **how), stats=st)
    assert torch.equal(s[:, -tail:], s1) and torch.equal(y[:, -tail:], y1) and not y[:, :-tail].any()
    g = cn.block_norm_backward(y, s, x, stats, cn.make_block_norm_shape(None, x, s, y, **how), dS=s, dX=x, dR=s, want=())
    g1 = cn.block_norm_backward(y1, s1, small[1], st, cn.make_block_norm_shape(None, small[1], s1, y1, **how), dS=s1, want=())
    assert torch.equal(g.dR[:, -tail:], g1.dR) and torch.equal(g.dX[:, -tail:], g1.dX)


@pytest.mark.parametrize("C", [5, 100, 1536, 5120])
@pytest.mark.parametrize("post", [NONE, LAYER, RMS])
@pytest.mark.parametrize("pre", [LAYER, RMS])
def test_rows_that_are_not_finite_with_every_norm(C, post, pre):
    """A NaN or an infinity, or finite values whose squares fp32 cannot sum up: NaN all along what is normed, and as its reciprocal deviation; the gradients likewise."""
    t = make(1, 30, C, x="f32", y="f32", post=post, pre=pre)
    clean = forward(t)
    grads = backward(t, clean[0], clean[2])
    in_x, in_r = dict(zip((3, 7, 21), ("nan", "inf", "1e25"))), dict(zip((11, 12, 20), ("-inf", "nan", "-1e25")))
    for row, v in in_x.items():
        t["x"][0, row, C // 2] = float(v)
    for row, v in in_r.items():
        t["r"][0, row, C - 1] = float(v)
    S, Y, stats = forward(t)
    bad = torch.zeros(30, dtype=torch.bool, device="cuda")
    bad[[*in_x, *in_r]] = True
    bad_x = torch.zeros_like(bad)
    bad_x[[*in_x]] = True
    assert torch.equal(S[0, ~bad], clean[0][0, ~bad]) and torch.equal(Y[0, ~bad], clean[1][0, ~bad]) and torch.equal(stats[:, 0, ~bad], clean[2][:, 0, ~bad])
    assert Y[0, bad].isnan().all() and stats[3, 0, bad].isnan().all()
    if post == NONE:
        assert (stats[1] == 1).all()
        at = S.clone()
        for rows, c in ((in_x, C // 2), (in_r, C - 1)):
            for row in rows:
                at[0, row, c] = 0
        assert at.isfinite().all()       # an infinity or a NaN reaches the stream in its own channel only
    else:
        assert torch.equal(stats[1, 0].isnan(), bad_x) and S[0, bad_x].isnan().all()
    g = backward(t, S, stats)
    for got, want in ((g.dR, grads.dR), (g.dX, grads.dX)):
        assert torch.equal(got[0, ~bad], want[0, ~bad]) and got[0, bad].isnan().all()
