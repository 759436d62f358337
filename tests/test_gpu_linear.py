"""Matrix product with bias, activation, gate and residual, and its gradients, against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import (A, ACT_ERR, Bc, DTYPES, SLOPE_MOST, U16, U32, act64, canvas, check, half_step, linear_grad_ref, linear_ref, padded, untouched)

pytestmark = pytest.mark.gpu

ACTS = [cn.ACT_NONE, cn.ACT_GELU_TANH, cn.ACT_GELU, cn.ACT_SILU]


def make(B, N, K, M, y="bf16", p="bf16", bias=True, gate=True, residual=True, seed=0, extra=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = dict(x=padded((B, N, K), torch.bfloat16, gen, extra=extra), w=padded((M, K), torch.bfloat16, gen, 1.5 / K ** 0.5),
             dy=padded((B, N, M), DTYPES[y], gen, extra=extra))
    vec = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
    t["bias"] = vec(M).to(DTYPES[p]) if bias else None
    t["gate"] = vec(B, 6, M)[:, 2].to(DTYPES[p]) if gate else None
    t["residual"] = padded((B, N, M), DTYPES[y], gen, extra=extra) if residual else None
    return t


def forward(t, act, keep=True, extra=1):
    B, N, _ = t["x"].shape
    M = t["w"].shape[0]
    buf, y = canvas((B, N, M), t["dy"].dtype, extra=extra)
    zbuf, z = canvas((B, N, M), torch.bfloat16, extra=extra)
    s = cn.make_linear_shape(t["x"], t["w"], y, residual=t["residual"], Z=z, bias=t["bias"], gate=t["gate"], activation=act)
    ws = torch.full((cn.linear_workspace_bytes(s),), 255, dtype=torch.uint8, device="cuda")
    out, _ = cn.linear(t["x"], t["w"], s, bias=t["bias"], gate=t["gate"], residual=t["residual"], Y=y, Z=z if keep else None, ws=ws)
    assert cn.query_status(ws) == cn.OK, cn.last_cuda_error()
    assert untouched(buf, y) and (untouched(zbuf, z) if keep else bool((zbuf == 77.0).all()))
    return out, z


def check_forward(t, act, y, z=None):
    ry, rz, ez, ey = linear_ref(t["x"], t["w"], t["bias"], t["gate"], t["residual"], act)
    if z is not None:
        check(z, rz, ez + U16 * rz.abs(), "z")
    check(y, ry, ey + half_step(y.dtype) * (ry.abs() + ey), "y")


def backward(t, z, act, need=("x", "w"), want=("bias", "gate"), extra=1):
    bx, dx = canvas(t["x"].shape, torch.bfloat16, extra=extra)
    bw, dw = canvas(t["w"].shape, torch.bfloat16)
    s = cn.make_linear_shape(t["x"], t["w"], t["dy"], Z=z, gate=t["gate"], dX=dx, dW=dw, activation=act)
    ws = torch.full((cn.linear_backward_workspace_bytes(s),), 255, dtype=torch.uint8, device="cuda")
    g = cn.linear_backward(t["dy"], t["x"], t["w"], s, Z=z, gate=t["gate"], dX=dx if "x" in need else None, dW=dw if "w" in need else None, want=want, ws=ws)
    assert cn.query_status(ws) == cn.OK, cn.last_cuda_error()
    assert untouched(bx, dx) if "x" in need else bool((bx == 77.0).all())
    assert untouched(bw, dw) if "w" in need else bool((bw == 77.0).all())
    return g


def check_backward(t, z, act, g):
    ref = linear_grad_ref(t["dy"], t["x"], t["w"], z, t["gate"], act)
    for name in ("dbias", "dgate", "dX", "dW"):
        got = getattr(g, name)
        if got is not None:
            r, e = ref[name]
            check(got, r, e + half_step(got.dtype) * (r.abs() + e), name)


# rows, in, out: single rows, both sides of the few-row kernel's limit, tile borders (128, 256), odd everything, a long k with few tiles (split), many tiles (persistent)
SIZES = [(1, 1, 1), (1, 1536, 1536), (2, 37, 19), (7, 1541, 333), (8, 4096, 16), (9, 64, 130), (16, 5120, 40), (17, 5120, 40), (33, 65, 257),
         (64, 8, 8), (127, 1000, 129), (128, 128, 128), (129, 63, 300), (256, 256, 256), (257, 1541, 513), (300, 4099, 96), (513, 512, 1536), (700, 9000, 333),
         (1100, 200, 5000), (5003, 100, 2100)]


@pytest.mark.parametrize("N,K,M", SIZES)
def test_every_size(N, K, M):
    t = make(1, N, K, M, seed=N + K + M)
    y, z = forward(t, cn.ACT_GELU_TANH)
    check_forward(t, cn.ACT_GELU_TANH, y, z)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("B,N", [(3, 1), (2, 6), (2, 150), (3, 301)])
@pytest.mark.parametrize("y,p", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("extra", [0, 1])
def test_activations_types_and_entries(act, B, N, y, p, extra):
    """extra = 1: a padded batch, whose entries do not follow each other evenly."""
    t = make(B, N, 200, 264, y, p, seed=N, extra=extra)
    out, z = forward(t, act, extra=extra)
    check_forward(t, act, out, z)
    g = backward(t, z, act, extra=extra)
    check_backward(t, z, act, g)


@pytest.mark.parametrize("bias,gate,residual", [(False, False, False), (True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("N", [3, 200])
def test_parts_that_are_left_out(bias, gate, residual, N):
    t = make(2, N, 130, 96, bias=bias, gate=gate, residual=residual)
    for act in (cn.ACT_NONE, cn.ACT_SILU):
        y, _ = forward(t, act, keep=False)
        check_forward(t, act, y)


GRAD_SIZES = [(1, 1, 1), (1, 300, 200), (2, 37, 19), (17, 1541, 333), (64, 64, 64), (129, 65, 257), (300, 96, 4099), (333, 1000, 1541), (700, 513, 129),
              (2500, 200, 264), (9001, 64, 130), (6000, 1500, 2100)]


@pytest.mark.parametrize("N,K,M", GRAD_SIZES)
@pytest.mark.parametrize("act,gate,dy", [(cn.ACT_GELU, True, "f32"), (cn.ACT_NONE, False, "bf16"), (cn.ACT_GELU_TANH, False, "bf16")])
def test_gradients_of_every_size(N, K, M, act, gate, dy):
    t = make(1, N, K, M, dy, gate=gate, seed=N)
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = padded((1, N, M), torch.bfloat16, gen, 1.5, extra=1)
    g = backward(t, z, act)
    check_backward(t, z, act, g)


def test_only_what_is_wanted():
    t = make(2, 150, 96, 200)
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = padded((2, 150, 200), torch.bfloat16, gen, extra=1)
    full = backward(t, z, cn.ACT_SILU)
    for need, want in ((("x",), ()), (("w",), ("bias",)), ((), ("gate",)), ((), ("bias", "gate")), (("x", "w"), ())):
        g = backward(t, z, cn.ACT_SILU, need, want)
        for name, on in (("dX", "x" in need), ("dW", "w" in need), ("dbias", "bias" in want), ("dgate", "gate" in want)):
            got = getattr(g, name)
            assert (got is not None) == on and (not on or torch.equal(got, getattr(full, name)))
    plain = {**t, "gate": None}
    g = backward(plain, None, cn.ACT_NONE)        # no pre-activation is needed
    check_backward(plain, None, cn.ACT_NONE, g)


@pytest.mark.parametrize("N", [7, 200])
def test_strides_of_axes_of_one_entry_do_not_matter(N):
    t = make(1, N, 128, 72)
    ref, z = forward(t, cn.ACT_SILU)
    u = {k: torch.as_strided(v, v.shape, (12345, *v.stride()[1:])) if k in ("x", "dy", "residual") else v for k, v in t.items()}
    y, _ = forward(u, cn.ACT_SILU)
    assert torch.equal(y, ref)
    for a, b in zip(backward(t, z, cn.ACT_SILU), backward(u, z, cn.ACT_SILU)):
        assert torch.equal(a, b)
    one = make(1, N, 128, 1)                 # a weight of one row
    one["w"] = torch.as_strided(one["w"], (1, 128), (13, 1))
    y, z = forward(one, cn.ACT_NONE)
    check_forward(one, cn.ACT_NONE, y, z)


@pytest.mark.parametrize("N", [5, 300])
@pytest.mark.parametrize("y", ["bf16", "f32"])
def test_residual_stream_in_place(N, y):
    t = make(1, N, 256, 384, y)
    ref, _ = forward(t, cn.ACT_NONE)
    stream = t["residual"]
    s = cn.make_linear_shape(t["x"], t["w"], stream, residual=stream, bias=t["bias"], gate=t["gate"])
    cn.linear(t["x"], t["w"], s, bias=t["bias"], gate=t["gate"], residual=stream, Y=stream)
    assert torch.equal(stream, ref)


@pytest.mark.parametrize("N", [4, 200])
def test_far_arguments_and_values_that_are_not_finite(N):
    """The activations at +-1e4 (their limits), and rows that are not finite keep to themselves."""
    t = make(1, N, 64, 128, "f32", bias=False, gate=False, residual=False)
    t["x"] *= 1e4
    for act in ACTS:
        y, z = forward(t, act)
        check_forward(t, act, y, z)
        z = z.clone()
        g = backward(t, z, act)
        check_backward(t, z, act, g)
    clean = forward(t, cn.ACT_NONE)[0].clone()
    t["x"][0, 1, 5] = float("nan")
    y = forward(t, cn.ACT_NONE)[0]
    keep = [i for i in range(N) if i != 1]
    assert torch.equal(y[:, keep], clean[:, keep]) and torch.isnan(y[0, 1]).all()


@pytest.mark.parametrize("N,K,M", [(300, 8192, 512), (3000, 8192, 2048), (3000, 5200, 1000)])
def test_fp32_output_of_a_long_sum(N, K, M):
    """At most 2560 products are summed up in one accumulator: 160 additions of 16 products, each of which cuts off half a step (2^-24) of the running sum
    on average; a sum of random terms grows with the square root, so that is 2/3 x 160 x 2^-24 of it, and of what several runs sum up to."""
    t = make(1, N, K, M, "f32", bias=False, gate=False, residual=False)
    y, _ = forward(t, cn.ACT_NONE, keep=False)
    ref = t["x"].double() @ t["w"].double().T
    assert (y.double() - ref).norm() <= 160 * 2 / 3 * 2.0 ** -24 * ref.norm()


def test_activation_over_its_range():
    """z = bias exactly (x = 0): the epilogue's activation alone, fp32 out, against 64 bits."""
    M = 4096
    x, w = torch.zeros((1, 40, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, 64), dtype=torch.bfloat16, device="cuda")
    bias = torch.linspace(-30, 30, M, device="cuda")
    y = torch.empty((1, 40, M), device="cuda")
    for act in ACTS:
        s = cn.make_linear_shape(x, w, y, bias=bias, activation=act)
        cn.linear(x, w, s, bias=bias, Y=y)
        ref = act64(bias.double(), act).expand(1, 40, M)
        check(y, ref, (ACT_ERR * (bias.double().abs() + 1) if act else 0) + U32 * ref.abs(), f"activation {act}")


def test_gradients_against_differences():
    """<dy, y> against <gradient, direction>, central differences of the forward call with fp32 output.  x and w lie on a grid of 2^-6 and
    move by one step of it, which bf16 holds exactly below 4."""
    B, N, K, M, act, h = 2, 40, 72, 88, cn.ACT_GELU_TANH, 2.0 ** -6
    t = make(B, N, K, M, "f32", "f32", residual=False, seed=4, extra=0)
    for k in ("x", "w"):
        t[k].copy_((t[k].float() / h).round().clamp(-64, 64) * h)
    _, z = forward(t, act, extra=0)
    g = backward(t, z, act, extra=0)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for name, grad in (("x", g.dX), ("w", g.dW), ("bias", g.dbias), ("gate", g.dgate)):
        v = torch.randint(0, 2, t[name].shape, device="cuda", generator=gen) * 2.0 - 1
        loss = []
        for sign in (1, -1):
            u = dict(t)
            u[name] = (t[name].float() + sign * h * v).to(t[name].dtype)
            loss.append((forward(u, act, extra=0)[0].double() * t["dy"].double()).sum())
        slope, ref = (loss[0] - loss[1]) / (2 * h), (grad.double() * v.double()).sum()
        # The backward call sees z rounded to bf16 (independent errors of at most U16 |z|) and rounds dz and the bf16 gradients: sums of independent
        # terms, taken as six times their 2-norm.  `along` is how z moves along the direction; for the gate it is act(z) that is read.
        dy, zz, gate, vd = t["dy"].double(), z.double(), t["gate"].double()[:, None], v.double()
        along = {"x": lambda: vd @ t["w"].double().T, "w": lambda: t["x"].double() @ vd.T, "bias": lambda: vd.expand_as(zz), "gate": lambda: vd[:, None].expand_as(zz)}[name]()
        if name == "gate":               # the loss is linear in the gate: no higher terms; the first slope is at most 1.13
            noise, third = 6 * U16 * SLOPE_MOST * (dy * zz * along).norm(), 0
        else:                            # second derivative at most 1.2, third at most 2
            noise = 6 * U16 * (1.2 * (dy * gate * zz * along).norm() + SLOPE_MOST * (dy * gate * along).norm() + (grad.double().norm() if grad.dtype == torch.bfloat16 else 0))
            third = h * h / 6 * 2 * ((dy * gate).abs() * along.abs() ** 3).sum()
        _, _, _, ey = linear_ref(t["x"], t["w"], t["bias"], t["gate"], None, act)      # errors of the two forward calls
        noise = noise + 6 * (dy * ey).norm() / h
        assert abs(slope - ref) <= noise + third + 1e-5 * abs(ref), (name, float(slope), float(ref))


@pytest.mark.parametrize("N,K,M", [(2, 1536, 1536), (300, 4099, 96), (3000, 256, 1300)])
def test_same_bits_again_streams_graphs_and_two_calls_at_once(N, K, M):
    t = make(1, N, K, M, "f32")
    act = cn.ACT_GELU
    y0, z0 = forward(t, act)
    g0 = backward(t, z0, act)
    y1, z1 = forward(t, act)
    g1 = backward(t, z1, act)
    assert torch.equal(y0, y1) and torch.equal(z0, z1) and all(torch.equal(a, b) for a, b in zip(g0, g1))

    def plan():
        y, z, dx, dw = (canvas(a.shape, a.dtype)[1] for a in (t["dy"], z0, t["x"], t["w"]))
        fs = cn.make_linear_shape(t["x"], t["w"], y, residual=t["residual"], Z=z, bias=t["bias"], gate=t["gate"], activation=act)
        bs = cn.make_linear_shape(t["x"], t["w"], t["dy"], Z=z, gate=t["gate"], dX=dx, dW=dw, activation=act)
        ws = torch.empty(max(cn.linear_workspace_bytes(fs), cn.linear_backward_workspace_bytes(bs)), dtype=torch.uint8, device="cuda")

        def run():
            cn.linear(t["x"], t["w"], fs, bias=t["bias"], gate=t["gate"], residual=t["residual"], Y=y, Z=z, ws=ws)
            return (y, z, *cn.linear_backward(t["dy"], t["x"], t["w"], bs, Z=z, gate=t["gate"], dX=dx, dW=dw, ws=ws))
        return run

    want = (y0, z0, *g0)
    streams, plans = [torch.cuda.Stream() for _ in range(2)], [plan(), plan()]
    got = []
    for st, run in zip(streams, plans):
        st.wait_stream(torch.cuda.current_stream())
    for st, run in zip(streams, plans):
        with torch.cuda.stream(st):
            got.append(run())
    torch.cuda.synchronize()
    for out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    run = plan()
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(2):
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("N", [257, 5003])
@pytest.mark.parametrize("y,gate", [("bf16", False), ("bf16", True), ("f32", True)])
def test_warps_with_rows_behind_the_last(N, y, gate):
    """The last warp of the rows holds lanes without a row, which skip residual, activation and stores of every piece of a wide tile; the loads from tensor
    memory between those pieces want the whole warp."""
    t = make(1, N, 192, 1000, y, gate=gate, seed=N)
    for act in (cn.ACT_GELU_TANH, cn.ACT_NONE):
        out, z = forward(t, act)
        check_forward(t, act, out, z)
    assert torch.equal(forward(t, cn.ACT_NONE)[0], out)


@pytest.mark.parametrize("act", ACTS[1:])
def test_small_values_keep_their_bits(act):
    """Relative to the value itself, down to where fp32 ends: an exponential whose argument was rounded four times at most (U32 of it each), and 64 U32 for an
    approximate exponential and reciprocal (2^-22 each), a polynomial of degree 8 whose terms sum up to twice its value (9 roundings: 18 U32, and 2 U32 of its
    own), products."""
    M = 4096
    x, w = torch.zeros((1, 40, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, 64), dtype=torch.bfloat16, device="cuda")
    bias = torch.linspace(-12, 12, M, device="cuda")
    y = torch.empty((1, 40, M), device="cuda")
    cn.linear(x, w, cn.make_linear_shape(x, w, y, bias=bias, activation=act), bias=bias, Y=y)
    z = bias.double()
    ref = {cn.ACT_GELU_TANH: z * torch.sigmoid(2 * A * (z + Bc * z ** 3)), cn.ACT_GELU: act64(z, act), cn.ACT_SILU: z * torch.sigmoid(z)}[act]
    arg = {cn.ACT_GELU_TANH: 2 * A * (z.abs() + Bc * z.abs() ** 3), cn.ACT_GELU: z * z / 2, cn.ACT_SILU: z.abs()}[act]
    check(y, ref.expand(1, 40, M), (ref.abs() * (4 * arg + 64) * U32 + 2.0 ** -118).expand(1, 40, M), f"activation {act}")


@pytest.mark.parametrize("act", ACTS[1:])
def test_slopes_of_the_largest_values(act):
    """Up to the largest bf16 of either sign the slopes are 0 and 1 (and 1/2 at 0), as sums of three rows."""
    big = torch.finfo(torch.bfloat16).max
    z = torch.tensor([-big, -1e30, -1e20, -1e10, -1e4, 1e4, 1e10, 1e20, 1e30, big, 0.0, -0.0], device="cuda").bfloat16().repeat(4)
    M = z.numel()
    x, w = torch.randn((1, 3, 64), device="cuda").bfloat16(), torch.randn((M, 64), device="cuda").bfloat16()
    zz, dy, gate, dw = z.expand(1, 3, M).contiguous(), torch.ones((1, 3, M), device="cuda"), torch.ones((1, M), device="cuda"), torch.empty_like(w)
    g = cn.linear_backward(dy, x, w, cn.make_linear_shape(x, w, dy, Z=zz, dW=dw, gate=gate, activation=act), Z=zz, dW=dw, gate=gate)
    want = (z > 0).double() + 0.5 * (z == 0).double()
    check(g.dbias, 3 * want, 3 * ACT_ERR * torch.ones_like(want), "dbias")
    value = 3 * z.double().clamp(min=0)
    check(g.dgate[0, :9], value[:9], ACT_ERR * (value[:9].abs() + 3), "dgate")          # three times the largest is infinite
    check(dw, want[:, None] * x.double().sum(1), (ACT_ERR + 2 * U16) * x.double().abs().sum(1).expand(M, 64), "dW")


def check_long_sum(N, K, M):
    """As test_fp32_output_of_a_long_sum: runs of 2560 products at most, whoever shares them out."""
    t = make(1, N, K, M, "f32", bias=False, gate=False, residual=False)
    y, _ = forward(t, cn.ACT_NONE, keep=False)
    ref = t["x"].double() @ t["w"].double().T
    assert (y.double() - ref).norm() <= 160 * 2 / 3 * 2.0 ** -24 * ref.norm()


@pytest.mark.parametrize("N,K,M", [(1, 65536, 7200), (8, 300000, 64), (8, 40961, 7200), (3, 65000, 3000)])
def test_fp32_output_of_a_long_sum_of_few_rows(N, K, M):
    """Four, eight and sixteen warps share k, two sums each."""
    check_long_sum(N, K, M)


@pytest.mark.parametrize("N,K,M", [(64, 30720, 1536), (1000, 13824, 1536), (300, 120000, 600), (512, 8960, 2048), (40, 41000, 5000)])
def test_fp32_output_of_a_long_sum_whose_k_is_shared(N, K, M):
    """Two and four pairs share a tile's k, each more than 2560 of it."""
    check_long_sum(N, K, M)


@pytest.mark.parametrize("B,N,K,M", [(1, 1 << 22, 8, 8), (2, 1 << 21, 8, 8), (1, 1 << 20, 64, 200), (3, 100001, 136, 72), (1, 75600, 1536, 1536)])
def test_weight_gradients_of_very_many_rows(B, N, K, M):
    """Terms of one sign, where what an accumulator cuts off adds up: at most a step (2^-23 of a running sum that is half the final one on average) per
    addition, two additions per 16 terms counted, over runs of 65536: 2 x 4096 x 2^-24 = 2^-11 of the sum, the additions of the runs and their shares
    2^-18 at most, and the rounding to bf16."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, dy = (torch.rand((B, N, n), device="cuda", generator=gen).add_(0.5).bfloat16() for n in (K, M))
    w = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    dw = torch.empty_like(w)
    s = cn.make_linear_shape(x, w, dy, dW=dw)
    ws = torch.empty(cn.linear_backward_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    cn.linear_backward(dy, x, w, s, dW=dw, want=(), ws=ws)
    assert cn.query_status(ws) == cn.OK
    ref = sum(d.double().T @ a.double() for d, a in zip(dy.flatten(0, 1).split(1 << 18), x.flatten(0, 1).split(1 << 18)))
    check(dw, ref, ref * (U16 + 2.0 ** -11 + 2.0 ** -18), "dW")


@pytest.mark.parametrize("N,K,M", [(40, 1 << 21, 64), (600, 1 << 18, 256), (2500, 70000, 2000), (3, 1 << 20, 40)])
def test_bf16_outputs_of_very_long_sums(N, K, M):
    """y, and dX of the transposed weight: as test_weight_gradients_of_very_many_rows."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.rand((1, N, K), device="cuda", generator=gen).add_(0.5).bfloat16()
    w = torch.rand((M, K), device="cuda", generator=gen).add_(0.5).bfloat16()
    bias, residual = torch.randn(M, device="cuda", generator=gen), torch.randn((1, N, M), device="cuda", generator=gen).bfloat16()
    y, z, dx = (torch.empty((1, N, M), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    _, ws = cn.linear(x, w, cn.make_linear_shape(x, w, y, bias=bias, residual=residual, Z=z), bias=bias, residual=residual, Y=y, Z=z)
    assert cn.query_status(ws) == cn.OK
    ref = sum(a.double() @ b.double().T for a, b in zip(x[0].split(1 << 17, 1), w.split(1 << 17, 1)))[None]
    e = ref * (2.0 ** -11 + 2.0 ** -18)
    zz = ref + bias.double()
    check(z, zz, e + U16 * (zz.abs() + e), "z")
    yy = zz + residual.double()
    check(y, yy, e + U16 * (yy.abs() + e), "y")
    wt = w.T.contiguous()
    cn.linear_backward(x, y, wt, cn.make_linear_shape(y, wt, x, dX=dx), dX=dx, want=())
    check(dx, ref, e + U16 * (ref + e), "dX")


def test_gradients_of_one_operand_without_the_other():
    t = make(2, 150, 96, 200)
    z = padded((2, 150, 200), torch.bfloat16, torch.Generator(device="cuda").manual_seed(1), extra=1)
    full = backward(t, z, cn.ACT_SILU)
    dx, dw = torch.empty_like(t["x"]), torch.empty_like(t["w"])
    s = cn.make_linear_shape(t["x"], t["w"], t["dy"], Z=z, gate=t["gate"], dX=dx, dW=dw, activation=cn.ACT_SILU)
    assert torch.equal(cn.linear_backward(t["dy"], None, t["w"], s, Z=z, gate=t["gate"], dX=dx).dX, full.dX)
    assert torch.equal(cn.linear_backward(t["dy"], t["x"], None, s, Z=z, gate=t["gate"], dW=dw).dW, full.dW)
    g = cn.linear_backward(t["dy"], None, None, s, Z=z, gate=t["gate"])
    assert g.dX is None and g.dW is None and torch.equal(g.dbias, full.dbias) and torch.equal(g.dgate, full.dgate)


# B, rows, in, out, type of y: sums in runs in tiles of 256 columns and of fewer, of one pair and shared by two and four, for either type; sums that are shared but
# need no runs.  Odd widths leave columns behind the last whole sector.
RUNS = [(2, 2000, 2570, 2050, "f32"), (2, 1501, 5200, 1000, "f32"), (2, 1000, 5200, 1000, "f32"), (2, 700, 5200, 517, "f32"), (2, 40, 12000, 1000, "f32"),
        (2, 900, 70001, 1100, "bf16"), (2, 40, 280001, 72, "bf16"), (2, 300, 2600, 300, "f32"), (2, 300, 2600, 300, "bf16"), (3, 33, 9001, 517, "f32")]


@pytest.mark.parametrize("B,N,K,M,y", RUNS)
@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("act", [cn.ACT_NONE, cn.ACT_GELU_TANH, cn.ACT_SILU])
def test_long_sums_with_everything_behind_them(B, N, K, M, y, extra, act):
    """Bias, pre-activation, activation, the entry's gate and the residual behind sums that are taken up in runs or shared; padded batches and others.  The
    bounds of linear_ref count a long accumulation, so the 2-norm is compared too: an output in bf16 is off by its rounding, one in fp32 by test_fp32_output_of_a_long_sum's bound."""
    t = make(B, N, K, M, y, "f32", seed=K, extra=extra)
    out, z = forward(t, act, extra=extra)
    check_forward(t, act, out, z)
    ry, rz, _, _ = linear_ref(t["x"], t["w"], t["bias"], t["gate"], t["residual"], act)
    assert (z.double() - rz).norm() <= U16 * rz.norm()
    # gate and slope make no more of the sum's error than themselves; the activation's own errors are ACT_ERR of 1 + |z|
    g = t["gate"].double()[:, None]
    bound = U16 * ry.norm() if y == "bf16" else 160 * 2 / 3 * 2.0 ** -24 * SLOPE_MOST * (g * rz).norm() + 2 * U32 * ry.norm() + (ACT_ERR * (g * (1 + rz.abs())).norm() if act else 0)
    assert (out.double() - ry).norm() <= bound
    stream = t["residual"]                     # onto the residual itself
    s = cn.make_linear_shape(t["x"], t["w"], stream, residual=stream, bias=t["bias"], gate=t["gate"], activation=act)
    cn.linear(t["x"], t["w"], s, bias=t["bias"], gate=t["gate"], residual=stream, Y=stream)
    assert torch.equal(stream, out)


@pytest.mark.parametrize("N,K,M,y", [(2000, 5200, 1000, "f32"), (64, 30720, 1536, "f32"), (40, 280001, 72, "bf16")])
def test_long_sums_give_the_same_bits_again(N, K, M, y):
    t = make(1, N, K, M, y, seed=1)
    out, _ = forward(t, cn.ACT_GELU)
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again, _ = forward(t, cn.ACT_GELU)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(again, out)


@pytest.mark.parametrize("N", [8, 9, 16])
def test_fp32_output_of_a_long_sum_of_two_column_tiles(N):
    check_long_sum(N, 90001, 72)
