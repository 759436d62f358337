"""The calls as a served layer runs them: block norm, 8-bit projection, norm of Q and K, rotary positions, attention, 8-bit projection, block norm; and the gradients of
the parts that are trained.  Every stage is compared with 64 bits on the inputs that the library's own earlier stages gave it; the whole with the same layer in torch."""
import pytest
import torch

from paper_2609_32420_b200 import carnator as cn
from tests.layer_util import U16, check, half_step
from tests.test_gpu_block_norm import EPS1, EPS2, VECTORS, check_forward, gradients64
from tests.test_gpu_fp8 import product_ref, values
from tests.test_gpu_rope import TURN_ERR, angles, ref as rope_ref

pytestmark = pytest.mark.gpu

B, H, D, T, Hg, Wg, n_text = 2, 2, 64, 3, 10, 9, 11
N, C = n_text + T * Hg * Wg, 128
PAIRS = (12, 10, 10)


def _quantized_weight(gen, rows, cols):
    w = (torch.randn((1, rows, cols), device="cuda", generator=gen) * cols ** -0.5).bfloat16()
    q, s = cn.quantize_fp8(w, cn.make_quantize_shape(w, None, None, block_rows=128))
    return q[0], s[0]


def _linear(x, w, ws, bias, act=cn.ACT_NONE):
    y = torch.empty((*x.shape[:2], w.shape[0]), dtype=torch.bfloat16, device="cuda")
    s = cn.make_linear_fp8_shape(x, w, ws, y, bias=bias, activation=act)
    _, wk = cn.linear_fp8(x, w, ws, s, bias=bias, Y=y)
    assert cn.query_status(wk) == cn.OK
    ry, ey = product_ref(dict(x=x, w=w, w_scale=ws, x_scale=None, bias=bias, gate=None, residual=None), act)
    check(y, ry, ey + U16 * (ry.abs() + ey), "8-bit projection")
    return y


def _block(t):
    S, Y = torch.empty_like(t["r"]), torch.empty((B, N, C), dtype=torch.bfloat16, device="cuda")
    stats = torch.empty((4, B, N), device="cuda")
    s = cn.make_block_norm_shape(t["r"], t["x"], S, Y, **{k: t[k] for k in VECTORS}, post=t["post"], pre=t["pre"], post_eps=EPS1, eps=EPS2, residual_scale=t["alpha"])
    cn.block_norm(t["r"], t["x"], s, **{k: t[k] for k in VECTORS}, S=S, Y=Y, stats=stats)
    check_forward(t, S, Y, stats)
    return S, Y, stats


def test_a_served_layer():
    gen = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *n, s=1.0: torch.randn(n, device="cuda", generator=gen) * s  # noqa: E731
    six = r(B, 6, C, s=0.5)
    (wqkv, sqkv), (wout, sout), (wup, sup) = (_quantized_weight(gen, *n) for n in ((3 * C, C), (C, C), (4 * C, C)))
    bqkv, bout, bup = (r(n, s=0.1).bfloat16() for n in (3 * C, C, 4 * C))
    qn, kn, pw = ((1 + r(n, s=0.2)).bfloat16() for n in (D, D, C))
    none = dict.fromkeys(VECTORS)
    stream, before = r(B, N, C, s=2.0) + 0.5, r(B, N, C).bfloat16()

    # the block before ends, this one begins
    t1 = dict(none, r=stream, x=before, post_weight=pw, gate=six[:, 2], shift=six[:, 0], scale=six[:, 1], post=cn.NORM_RMS, pre=cn.NORM_LAYER, alpha=1.0)
    mid, h, stats1 = _block(t1)
    qkv = _linear(h, wqkv, sqkv, bqkv)
    q, k, v = qkv.view(B, N, 3, H, D).permute(2, 0, 3, 1, 4)
    for t, w in ((q, qn), (k, kn)):
        cn.layer_norm(t, cn.make_norm_shape(t, t, w, eps=1e-6), weight=w, Y=t)
    # Q and K are one tensor of 2 H heads; in place
    qk = qkv.view(B, N, 3 * H, D)[:, :, :2 * H].transpose(1, 2)
    plain_qk = qk.clone()
    freq, m = cn.rope_frequencies(PAIRS, scaling=cn.ROPE_SCALE_RAMP, factor=2.0, original=(2, 10, 9), low=0.1, high=1.0)
    how = dict(n_text=n_text, grid=(T, Hg, Wg), amplitude=m)
    cn.rope(qk, freq.cuda(), cn.make_rope_shape(qk, qk, PAIRS, **how), Y=qk)
    angle, on = angles(B, N, PAIRS, freq, n_text, (T, Hg, Wg), None, (0, 0, 0))
    want, size, *_ = rope_ref(plain_qk, angle, on, False, m, False)
    check(qk, want, TURN_ERR * size + U16 * want.abs(), "rope")
    o = torch.empty((B, N, H, D), dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)
    shape = cn.make_shape(B, H, N, D, n_text, T, Hg, Wg, 64, 64, Q=q, K=k, V=v, O=o)
    mask, bws = cn.build_connectivity(q, k, shape, cn.BuildParams(cn.MODE_TOPK, 0.5, 0.9, 0, 1, 1))
    _, _, ws = cn.sparse_attn(q, k, v, mask, None, shape, O=o)
    assert cn.query_status(ws) == cn.OK and cn.query_status(bws) == cn.OK
    out = _linear(o.permute(0, 2, 1, 3).reshape(B, N, C), wout, sout, bout)
    # the attention half ends, the feed-forward half begins
    t2 = dict(none, r=mid, x=out, post_weight=pw, gate=six[:, 5], shift=six[:, 3], scale=six[:, 4], post=cn.NORM_RMS, pre=cn.NORM_LAYER, alpha=1.0)
    end, h2, stats2 = _block(t2)
    up = _linear(h2, wup, sup, bup, cn.ACT_GELU_TANH)

    # the same layer in torch, 64 bits, from the mask that was built
    def norm(x, kind, eps=1e-6):
        mean = x.mean(-1, keepdim=True) if kind == cn.NORM_LAYER else 0
        return (x - mean) * (((x - mean) ** 2).mean(-1, keepdim=True) + eps) ** -0.5
    f = {n: values(w[None], s[None], 128)[0] for n, w, s in (("qkv", wqkv, sqkv), ("out", wout, sout), ("up", wup, sup))}
    s6 = six.double()[:, :, None]
    tm = stream.double() + s6[:, 2] * norm(before.double(), cn.NORM_RMS, EPS1) * pw.double()
    a = norm(tm, cn.NORM_LAYER, EPS2) * (1 + s6[:, 1]) + s6[:, 0]
    tq, tk, tv = (a @ f["qkv"].T + bqkv.double()).view(B, N, 3, H, D).permute(2, 0, 3, 1, 4)
    tq, tk = (rope_ref(norm(x, cn.NORM_LAYER) * w.double(), angle, on, False, m, False)[0] for x, w in ((tq, qn), (tk, kn)))
    keep = mask.bool().repeat_interleave(64, 2)[:, :, :N].repeat_interleave(64, 3)[..., :N]
    p = (tq @ tk.mT * D ** -0.5).masked_fill(~keep, float("-inf")).softmax(-1)
    to = (p @ tv).permute(0, 2, 1, 3).reshape(B, N, C) @ f["out"].T + bout.double()
    te = tm + s6[:, 5] * norm(to, cn.NORM_RMS, EPS1) * pw.double()
    tu = torch.nn.functional.gelu((norm(te, cn.NORM_LAYER, EPS2) * (1 + s6[:, 4]) + s6[:, 3]) @ f["up"].T + bup.double(), approximate="tanh")
    # Three operands are taken to 8 bits on the way (h, o, h2): each is off by at most 2^-4 of a value, and by at most 2^-4 / sqrt 3 in the 2-norm (uniform over a step);
    # what goes through 16 bits is a sixteenth of that.  Four of the 8-bit error, in the 2-norm, of what the branches add.
    e8 = 2.0 ** -4 / 3 ** 0.5
    assert (mid.double() - tm).norm() <= 2 * U16 * (tm - stream.double()).norm()
    assert (end.double() - te).norm() <= 4 * e8 * (te - tm).norm()
    assert (up.double() - tu).norm() <= 5 * e8 * tu.norm()

    # gradients through both block norms, as a training step has them: from the second's outputs to the stream and to what the blocks put out
    dh2, dend = r(B, N, C).bfloat16(), r(B, N, C)
    grads = []
    for t, S, stats, dy, ds in ((t2, end, stats2, dh2, dend), (t1, mid, stats1, r(B, N, C).bfloat16(), None)):
        ds = ds if ds is not None else grads[-1].dR
        s = cn.make_block_norm_shape(None, t["x"], S, dy, **{n: t[n] for n in VECTORS}, dS=ds, post=t["post"], pre=t["pre"], post_eps=EPS1, eps=EPS2)
        g = cn.block_norm_backward(dy, S, t["x"], stats, s, dS=ds, **{n: t[n] for n in VECTORS if n != "shift"})
        want = gradients64(dict(t, dy=dy, ds=ds, y_dtype=dy.dtype), S, stats)
        for name in g._fields:
            got = getattr(g, name)
            if got is not None:
                rr, e = want[name]
                check(got, rr, e + half_step(got.dtype) * (rr.abs() + e), name)
        grads.append(g)
    # and through the turn: the gradient of the scores' side goes back by the inverse call
    dqk = r(B, 2 * H, N, D).bfloat16()
    back = cn.rope(dqk, freq.cuda(), cn.make_rope_shape(dqk, None, PAIRS, inverse=True, **how))
    want, size, *_ = rope_ref(dqk, angle, on, False, m, True)
    check(back, want, TURN_ERR * size + U16 * want.abs(), "rope's gradient")


@pytest.mark.parametrize("rows,width", [(5, 256), (300, 384), (2500, 640)])
def test_calls_behind_one_another_wait_for_one_another(rows, width):
    """Kernels may be launched while the one ahead drains.  A long chain in which every call needs the one before it, with library calls of other kinds, torch operations and
    buffers used again between them, gives the bits that the same chain gives with a wait after every call."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = [torch.randn((1, width, width), device="cuda", generator=gen).bfloat16() * width ** -0.5 for _ in range(3)]
    x0 = torch.randn((1, rows, width), device="cuda", generator=gen)
    mod = torch.randn((1, 3, width), device="cuda", generator=gen) * 0.1
    pairs = (20, 6, 6)
    freq = cn.rope_frequencies(pairs, device="cuda")[0]

    def run(wait):
        def after():
            if wait:
                torch.cuda.synchronize()
        stream, ds = x0.clone(), x0.clone() * 0.1
        h, out, dx = (torch.empty((1, rows, width), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        out.copy_(x0)
        q, qs = torch.empty((1, rows, width), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((1, -(-width // 128), rows), device="cuda").transpose(1, 2)
        wq, wqs = torch.empty((1, width, width), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((1, -(-width // 128), -(-width // 128)), device="cuda")
        stats = torch.empty((4, 1, rows), device="cuda")
        how = dict(gate=mod[:, 2], scale=mod[:, 1], shift=mod[:, 0])
        bs = cn.make_block_norm_shape(stream, out, stream, h, dS=ds, dR=ds, dX=dx, post=cn.NORM_RMS, **how)
        fs, ws_shape = cn.make_quantize_shape(h, q, qs), cn.make_quantize_shape(w[0], wq, wqs, block_rows=128)
        ls = cn.make_linear_fp8_shape(q, wq[0], wqs[0], out, x_scale=qs)
        ms = cn.make_linear_fp8_shape(h, wq[0], wqs[0], out)
        heads = out.view(1, rows, -1, 64).transpose(1, 2)
        rs = cn.make_rope_shape(heads, heads, pairs)
        ws = torch.empty(max(cn.linear_fp8_workspace_bytes(ls), cn.linear_fp8_workspace_bytes(ms), cn.block_norm_backward_workspace_bytes(bs)), dtype=torch.uint8, device="cuda")
        for i in range(12):
            cn.block_norm(stream, out, bs, **how, S=stream, Y=h, stats=stats)
            after()
            cn.quantize_fp8(w[i % 3], ws_shape, Q=wq, scale=wqs)
            after()
            if i % 2:
                cn.quantize_fp8(h, fs, Q=q, scale=qs)
                after()
                cn.linear_fp8(q, wq[0], wqs[0], ls, x_scale=qs, Y=out, ws=ws)
            else:
                cn.linear_fp8(h, wq[0], wqs[0], ms, Y=out, ws=ws)
            after()
            cn.rope(heads, freq, rs, Y=heads)
            after()
            g = cn.block_norm_backward(h, stream, out, stats, bs, dS=ds, gate=mod[:, 2], scale=mod[:, 1], dR=ds, dX=dx, ws=ws)
            after()
            out += (dx.float() * 1e-3 + g.dgate * 1e-4).bfloat16()
            after()
            ds *= 0.5
            stream *= 0.9
            after()
        torch.cuda.synchronize()
        return stream, h, out, ds, dx, q.view(torch.uint8), qs, g.dscale, g.dshift
    want = run(True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))
    assert torch.isfinite(want[0]).all()
