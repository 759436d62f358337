"""The calls as a layer runs them: norm, projection, norm of Q and K, mask, attention, gated projection onto the residual stream,
and the feed-forward half with its gradients.  Every stage is compared with 64 bits on the inputs that the library's own earlier
stages gave it; the result of the whole chain with the same layer in fp32 torch operations."""
import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import U16, U32, check, half_step, linear_grad_ref, linear_ref, norm_ref, xh_error

pytestmark = pytest.mark.gpu

EPS = 1e-6
B, H, D, T, Hg, Wg, n_text = 2, 2, 64, 3, 10, 9, 11
N, C = n_text + T * Hg * Wg, 128


def _weights(gen):
    r = lambda *n, s=1.0: torch.randn(n, device="cuda", generator=gen) * s  # noqa: E731
    return dict(qkv=r(3 * C, C, s=C ** -0.5).bfloat16(), qkv_b=r(3 * C, s=0.1).bfloat16(), qn=(1 + r(D, s=0.2)).bfloat16(), kn=(1 + r(D, s=0.2)).bfloat16(),
                out=r(C, C, s=C ** -0.5).bfloat16(), out_b=r(C, s=0.1).bfloat16(), up=r(4 * C, C, s=C ** -0.5).bfloat16(), up_b=r(4 * C, s=0.1).bfloat16(),
                down=r(C, 4 * C, s=(4 * C) ** -0.5).bfloat16(), down_b=r(C, s=0.1).bfloat16(), six=r(B, 6, C, s=0.5))


def _norm(x, weight, shift, scale, out_dtype):
    y = torch.empty(x.shape, dtype=out_dtype, device="cuda")
    mean, rstd = (torch.empty(x.shape[:3], device="cuda") for _ in range(2))
    s = cn.make_norm_shape(x, y, weight, scale, shift=shift, eps=EPS)
    cn.layer_norm(x, s, weight=weight, shift=shift, scale=scale, Y=y, mean=mean, rstd=rstd)
    ref, m, r, xh, a, c = norm_ref(x, weight, None, shift, scale, EPS)
    check(y, ref, xh_error(x, m, r, xh) * a.abs() + 4 * U32 * ((xh * a).abs() + c.abs()) + half_step(out_dtype) * ref.abs(), "norm")
    return y, mean, rstd


def _linear(x, w, b, act=cn.ACT_NONE, gate=None, residual=None):
    y = torch.empty((*x.shape[:2], w.shape[0]), dtype=torch.float32 if residual is not None else torch.bfloat16, device="cuda")
    z = torch.empty(y.shape, dtype=torch.bfloat16, device="cuda")
    s = cn.make_linear_shape(x, w, y, residual=residual, Z=z, bias=b, gate=gate, activation=act)
    _, ws = cn.linear(x, w, s, bias=b, gate=gate, residual=residual, Y=y, Z=z)
    assert cn.query_status(ws) == cn.OK
    ry, rz, ez, ey = linear_ref(x, w, b, gate, residual, act)
    check(y, ry, ey + half_step(y.dtype) * (ry.abs() + ey), "linear")
    check(z, rz, ez + U16 * rz.abs(), "z")
    return y, z


def test_a_layer():
    gen = torch.Generator(device="cuda").manual_seed(0)
    W = _weights(gen)
    six = W["six"]
    stream = torch.randn((B, N, C), device="cuda", generator=gen) * 2 + 0.5

    # attention half
    h, _, _ = _norm(stream[:, None], None, six[:, 0], six[:, 1], torch.bfloat16)
    qkv, _ = _linear(h[:, 0], W["qkv"], W["qkv_b"])
    q, k, v = qkv.view(B, N, 3, H, D).permute(2, 0, 3, 1, 4)
    for t, w in ((q, W["qn"]), (k, W["kn"])):                    # in place, per head
        cn.layer_norm(t, cn.make_norm_shape(t, t, w, eps=EPS), weight=w, Y=t)
    o = torch.empty((B, N, H, D), dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)       # heads beside each other, as the projection reads them
    shape = cn.make_shape(B, H, N, D, n_text, T, Hg, Wg, 64, 64, Q=q, K=k, V=v, O=o)
    mask, bws = cn.build_connectivity(q, k, shape, cn.BuildParams(cn.MODE_TOPK, 0.5, 0.9, 0, 1, 1))
    _, _, ws = cn.sparse_attn(q, k, v, mask, None, shape, O=o)
    assert cn.query_status(ws) == cn.OK and cn.query_status(bws) == cn.OK
    mid, _ = _linear(o.permute(0, 2, 1, 3).reshape(B, N, C), W["out"], W["out_b"], gate=six[:, 2], residual=stream)

    # feed-forward half, kept for its gradients
    h2, mean, rstd = _norm(mid[:, None], None, six[:, 3], six[:, 4], torch.bfloat16)
    up, zu = _linear(h2[:, 0], W["up"], W["up_b"], act=cn.ACT_GELU_TANH)
    end, zd = _linear(up, W["down"], W["down_b"], gate=six[:, 5], residual=mid)

    # the same layer in torch, fp32, from the mask that was built
    def norm(x):
        return torch.nn.functional.layer_norm(x, x.shape[-1:], eps=EPS)
    f = {n: t.float() for n, t in W.items()}
    s = six[:, :, None]
    a = norm(stream) * (1 + s[:, 1]) + s[:, 0]
    tq, tk, tv = (a @ f["qkv"].T + f["qkv_b"]).view(B, N, 3, H, D).permute(2, 0, 3, 1, 4)
    tq, tk = norm(tq) * f["qn"], norm(tk) * f["kn"]
    keep = mask.bool().repeat_interleave(64, 2)[:, :, :N].repeat_interleave(64, 3)[..., :N]
    p = (tq @ tk.mT * D ** -0.5).masked_fill(~keep, float("-inf")).softmax(-1)
    tm = stream + s[:, 2] * ((p @ tv).permute(0, 2, 1, 3).reshape(B, N, C) @ f["out"].T + f["out_b"])
    a = norm(tm) * (1 + s[:, 4]) + s[:, 3]
    te = tm + s[:, 5] * (torch.nn.functional.gelu(a @ f["up"].T + f["up_b"], approximate="tanh") @ f["down"].T + f["down_b"])
    # Five roundings to bf16 lie between the stream and its end on either branch (norm, qkv, q and k, attention's P, O; norm, up), each at most U16 of
    # values about 1 and averaged by the products: 2 U16 of the branches' size each, in the 2-norm.
    assert (end - te).norm() <= 10 * 2 * U16 * (te - stream).norm()

    # gradients of the feed-forward half, back to the stream behind the attention
    d_end = torch.randn((B, N, C), device="cuda", generator=gen)
    d_up = torch.empty_like(up)
    dws = {}

    def linear_backward(dy, x, w, z, gate, act, dx, name):
        dw = dws[name] = torch.empty_like(w)
        sh = cn.make_linear_shape(x, w, dy, Z=z, gate=gate, dX=dx, dW=dw, activation=act)
        g = cn.linear_backward(dy, x, w, sh, Z=z, gate=gate, dX=dx, dW=dw)
        for field, (r, e) in linear_grad_ref(dy, x, w, z, gate, act).items():
            got = getattr(g, field)
            check(got, r, e + half_step(got.dtype) * (r.abs() + e), f"{name} {field}")
        return g

    gd = linear_backward(d_end, up, W["down"], zd, six[:, 5], cn.ACT_NONE, d_up, "down")
    d_h2 = torch.empty_like(h2[:, 0])
    gu = linear_backward(d_up, h2[:, 0], W["up"], zu, None, cn.ACT_GELU_TANH, d_h2, "up")
    sh = cn.make_norm_shape(mid[:, None], d_h2[:, None], None, six[:, 4], shift=six[:, 3], eps=EPS)
    gn = cn.layer_norm_backward(d_h2[:, None], mid[:, None], mean, rstd, sh, scale=six[:, 4])
    d_mid = d_end + gn.dX[:, 0]

    # the same gradients by torch's differentiation in 64 bits
    leaf = {n: W[n].double().requires_grad_() for n in ("up", "up_b", "down", "down_b")}
    m, s6 = mid.double().requires_grad_(), six.double().requires_grad_()
    a = torch.nn.functional.layer_norm(m, (C,), eps=EPS) * (1 + s6[:, 4, None]) + s6[:, 3, None]
    e = m + s6[:, 5, None] * (torch.nn.functional.gelu(a @ leaf["up"].T + leaf["up_b"], approximate="tanh") @ leaf["down"].T + leaf["down_b"])
    e.backward(d_end.double())
    # seven roundings at most (h2, up, z, dz twice, d_up, d_h2, the gradient's own), U16 each, in the 2-norm
    for name, got, ref in (("mid", d_mid, m.grad), ("down", gd.dW, leaf["down"].grad), ("up", gu.dW, leaf["up"].grad), ("down_b", gd.dbias, leaf["down_b"].grad),
                           ("up_b", gu.dbias, leaf["up_b"].grad), ("gate", gd.dgate, s6.grad[:, 5]), ("shift", gn.dshift, s6.grad[:, 3]), ("scale", gn.dscale, s6.grad[:, 4])):
        assert (got.double() - ref).norm() <= 8 * U16 * ref.norm(), name


@pytest.mark.parametrize("rows,width", [(5, 256), (300, 384), (3000, 640)])
def test_calls_behind_one_another_wait_for_one_another(rows, width):
    """Kernels may be launched while the one ahead drains.  A long chain in which every call needs the one before it, library calls, torch
    operations and buffers used again mixed, gives the bits that the same chain gives with a wait after every call."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = [(torch.randn((width, width), device="cuda", generator=gen) * width ** -0.5).bfloat16() for _ in range(3)]
    x0 = torch.randn((1, rows, width), device="cuda", generator=gen)
    mod = torch.randn((1, 2, width), device="cuda", generator=gen) * 0.1

    def run(wait):
        def after():
            if wait:
                torch.cuda.synchronize()
        stream, h, z, dx, dw = x0.clone(), *(torch.empty((1, rows, width), dtype=torch.bfloat16, device="cuda") for _ in range(3)), torch.empty_like(w[0])
        up = torch.empty_like(h)
        mean, rstd = (torch.empty((1, 1, rows), device="cuda") for _ in range(2))
        ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        ns = cn.make_norm_shape(stream[:, None], h[:, None], None, mod[:, 1], shift=mod[:, 0], eps=EPS)
        us = cn.make_linear_shape(h, w[0], up, Z=z, dX=dx, dW=dw, activation=cn.ACT_GELU_TANH)
        ds = cn.make_linear_shape(up, w[1], stream, residual=stream)
        bs = cn.make_norm_shape(stream[:, None], dx[:, None], None, mod[:, 1], shift=mod[:, 0], dX=stream[:, None].clone(), eps=EPS)
        for i in range(12):
            cn.layer_norm(stream[:, None], ns, shift=mod[:, 0], scale=mod[:, 1], Y=h[:, None], mean=mean, rstd=rstd)
            after()
            cn.linear(h, w[i % 3], us, Y=up, Z=z, ws=ws)
            after()
            g = cn.linear_backward(up, h, w[i % 3], us, Z=z, dX=dx, dW=dw, ws=ws)
            after()
            n = cn.layer_norm_backward(dx[:, None], stream[:, None], mean, rstd, bs, scale=mod[:, 1], ws=ws[:cn.layer_norm_backward_workspace_bytes(bs)])
            after()
            up += g.dbias.bfloat16() * 1e-3
            after()
            cn.linear(up, w[1], ds, residual=stream, Y=stream, ws=ws)
            after()
            stream *= 0.5
            stream += 0.01 * n.dX[:, 0]
            after()
        torch.cuda.synchronize()
        return stream, h, z, dx, dw, n.dscale, g.dbias
    want = run(True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))
    assert torch.isfinite(want[0]).all()


def test_offsets_that_pass_32_bits():
    """600000 rows of 4096 channels, 2.4e9 elements: the last rows, whose offsets do not fit 32 bits, against the same rows on their own."""
    rows, wide, tail = 600_000, 4096, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros((1, 1, rows, wide), dtype=torch.bfloat16, device="cuda")
    x[:, :, -tail:] = torch.randn((tail, wide), device="cuda", generator=gen)
    last = x[:, :, -tail:].clone()
    y = torch.empty_like(x)
    cn.layer_norm(x, cn.make_norm_shape(x, y), Y=y)
    assert torch.equal(y[:, :, -tail:], cn.layer_norm(last, cn.make_norm_shape(last, last)))
    assert not y[:, :, :-tail].any()
    # into and out of that width
    w = (torch.randn((wide, 64), device="cuda", generator=gen) / 8).bfloat16()
    small = torch.zeros((1, rows, 64), dtype=torch.bfloat16, device="cuda")
    small[:, -tail:] = torch.randn((tail, 64), device="cuda", generator=gen)
    z, out = x[:, 0], y[:, 0]                                     # rows of zeros but for the last
    s = cn.make_linear_shape(small, w, out, activation=cn.ACT_GELU)
    _, ws = cn.linear(small, w, s, Y=out)
    assert cn.query_status(ws) == cn.OK
    ry, _, _, ey = linear_ref(small[:, -tail:], w, None, None, None, cn.ACT_GELU)
    check(out[:, -tail:], ry, ey + U16 * (ry.abs() + ey), "y")
    assert not out[:, :-tail].any()
    dx, dw = torch.empty_like(small), torch.empty_like(w)
    s = cn.make_linear_shape(small, w, out, Z=z, dX=dx, dW=dw, activation=cn.ACT_GELU)
    g = cn.linear_backward(out, small, w, s, Z=z, dX=dx, dW=dw)
    ref = linear_grad_ref(out[:, -tail:], small[:, -tail:], w, z[:, -tail:], None, cn.ACT_GELU)
    for name, got in (("dX", dx[:, -tail:]), ("dW", dw), ("dbias", g.dbias)):
        r, e = ref[name]
        check(got, r, e + half_step(got.dtype) * (r.abs() + e), name)
    assert not dx[:, :-tail].any()
