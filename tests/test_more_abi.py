"""Rotary positions, 8-bit operands and their product: what the calls refuse, before anything is launched, and what they compute on the host (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from paper_2609_32420_b200 import build as cbuild
from paper_2609_32420_b200 import carnator as cn

P, BIG = 1 << 20, 1 << 40       # a 256-byte aligned address that is never read, a workspace size that suffices
BAD, NOT = cn.ERR_INVALID_ARG, cn.ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def _built():
    cbuild.build_library()


def changed(s, kw):
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(s, k)[v[0]] = v[1]
        else:
            setattr(s, k, v)
    return s


def expect(status, call):
    before = cn.kernel_launches()
    assert call() == status
    assert cn.kernel_launches() == before


# ---- rotary positions -------------------------------------------------------------------------------------
def rope_shape(positions=False, **kw):
    x = torch.empty((2, 3, 40, 64), dtype=torch.bfloat16)
    p = torch.empty((2, 40, 3), dtype=torch.int32) if positions else None
    return changed(cn.make_rope_shape(x, x, (12, 10, 10), n_text=4, grid=(4, 3, 3), positions=p), kw)


def call_rope(s, X=P, freq=P, pos=None, Y=P):
    return cn.lib().carnator_rope(X, freq, pos, ctypes.byref(s), Y, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), BAD), (dict(H=0), BAD), (dict(N=-1), BAD), (dict(D=0), BAD), (dict(x_dtype=2), BAD), (dict(layout=2), BAD), (dict(layout=-1), BAD),
    (dict(amplitude=float("nan")), BAD), (dict(amplitude=float("inf")), BAD), (dict(pairs=(0, 13)), BAD), (dict(pairs=(1, -1)), BAD), (dict(n_text=5), BAD), (dict(n_text=-1), BAD),
    (dict(T=5), BAD), (dict(Wg=0), BAD), (dict(Hg=1 << 30, Wg=1 << 30), BAD), (dict(B=65536), NOT), (dict(H=65536), NOT),
    (dict(x_stride=(2, 60)), BAD), (dict(x_stride=(0, -8)), BAD), (dict(x_stride=(1, 1 << 39)), BAD), (dict(y_stride=(2, 32)), BAD), (dict(y_stride=(1, 0)), BAD),
])
def test_rope_refuses_bad_records(kw, status):
    expect(status, lambda: call_rope(rope_shape(**kw)))


def test_rope_refuses_bad_pointers_and_positions():
    for kw in (dict(X=None), dict(Y=None), dict(freq=None), dict(X=P + 8), dict(Y=P + 2), dict(freq=P + 4)):
        expect(BAD, lambda: call_rope(rope_shape(), **kw))
    expect(BAD, lambda: call_rope(rope_shape(True), pos=P + 2))
    for kw in (dict(axes=0), dict(axes=4), dict(axes=2), dict(pos_stride=(0, -1)), dict(pos_stride=(1, -1)), dict(pos_stride=(1, 1 << 39))):
        expect(BAD, lambda: call_rope(rope_shape(True, **kw), pos=P))
    s = rope_shape()
    s.pairs[:] = [0, 0, 0]
    expect(BAD, lambda: call_rope(s))
    s = rope_shape(D=258)
    s.x_stride[:], s.y_stride[:] = [1 << 20, 1 << 16, 264], [1 << 20, 1 << 16, 264]
    expect(NOT, lambda: call_rope(s))


def test_rope_frequencies():
    def plain(pairs, theta=10000.0):
        return [theta ** (-i / n) for n in pairs for i in range(n)]

    f, m = cn.rope_frequencies((22, 21, 21), theta=500.0)
    assert m == 1.0 and f.dtype == torch.float64 and f.tolist() == pytest.approx(plain((22, 21, 21), 500.0), rel=1e-14)
    f, m = cn.rope_frequencies(8, scaling=cn.ROPE_SCALE_LINEAR, factor=4)
    assert m == 1.0 and f.tolist() == pytest.approx([v / 4 for v in plain((8,))], rel=1e-14)
    f, _ = cn.rope_frequencies((8, 1), scaling=cn.ROPE_SCALE_BASE, factor=(3.0, 7.0))
    assert f.tolist() == pytest.approx([(10000 * 3 ** (16 / 14)) ** (-i / 8) for i in range(8)] + [1.0], rel=1e-13)
    assert f[7] * 3 == pytest.approx(plain((8,))[7], rel=1e-13)       # the slowest pair is slowed down by the factor, the fastest not at all
    f, m = cn.rope_frequencies((16, 4), scaling=cn.ROPE_SCALE_RAMP, factor=(4.0, 2.0), original=(1000.0, 50.0), low=1.0, high=32.0)
    assert m == pytest.approx(0.1 * math.log(4.0) + 1, rel=1e-15)
    want = []
    for n, factor, length in ((16, 4.0, 1000.0), (4, 2.0, 50.0)):
        for i in range(n):
            w = 10000.0 ** (-i / n)
            g = min(max((length * w / (2 * math.pi) - 1) / 31, 0.0), 1.0)
            want.append(w * (g + (1 - g) / factor))
    assert f.tolist() == pytest.approx(want, rel=1e-13)
    assert f[0] == 1.0 and f[15] == pytest.approx(plain((16,))[15] / 4, rel=1e-13)


def test_rope_frequencies_refuse():
    ramp = dict(scaling=cn.ROPE_SCALE_RAMP, factor=2.0, original=10.0)
    for kw in (dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(scaling=4), dict(scaling=-1), dict(pairs=-1), dict(pairs=(1 << 20) + 1),
               dict(scaling=cn.ROPE_SCALE_LINEAR, factor=0.5), dict(scaling=cn.ROPE_SCALE_BASE, factor=float("inf")), dict(scaling=cn.ROPE_SCALE_LINEAR, factor=float("nan")),
               {**ramp, "original": 0.0}, {**ramp, "low": 2.0, "high": 2.0}, {**ramp, "low": -1.0}, {**ramp, "high": float("inf")}):
        with pytest.raises(cn.CarnatorError):
            cn.rope_frequencies(**{"pairs": 4, **kw})
    L, s = cn.lib(), cn.RopeScaling()
    s.theta = 2.0
    assert L.carnator_rope_frequencies(None, (ctypes.c_double * 1)(), None) == BAD and L.carnator_rope_frequencies(ctypes.byref(s), None, None) == BAD
    assert L.carnator_rope_frequencies(ctypes.byref(s), (ctypes.c_double * 1)(), None) == cn.OK       # no pairs: nothing to fill
    with pytest.raises(ValueError):
        cn.rope_frequencies((1, 1, 1, 1))


# ---- block norms -------------------------------------------------------------------------------------------
def block_shape(**kw):
    x = torch.empty((2, 40, 128), dtype=torch.bfloat16)
    return changed(cn.make_block_norm_shape(x, x, x, x, post=cn.NORM_RMS), kw)


def call_block(s, R=P, X=P, w=P, gate=P, shift=P, S=P, Y=P, stats=P):
    return cn.lib().carnator_block_norm(R, X, w, P, gate, P, P, shift, P, ctypes.byref(s), S, Y, stats, None)


def call_block_backward(s, dY=P, dS=P, S=P, X=P, stats=P, w=P, gate=P, dR=P, dX=P, dw=P, dgate=P, ws=P, ws_bytes=BIG):
    return cn.lib().carnator_block_norm_backward(dY, dS, S, X, stats, w, P, gate, P, P, P, ctypes.byref(s), dR, dX, dw, P, dgate, P, P, P, P, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), BAD), (dict(N=0), BAD), (dict(C=-8), BAD), (dict(post=3), BAD), (dict(post=-1), BAD), (dict(pre=0), BAD), (dict(pre=3), BAD), (dict(stream_dtype=2), BAD),
    (dict(x_dtype=2), BAD), (dict(y_dtype=-1), BAD), (dict(weight_dtype=3), BAD), (dict(mod_dtype=2), BAD), (dict(eps=-1e-6), BAD), (dict(post_eps=float("nan")), BAD),
    (dict(eps=float("inf")), BAD), (dict(residual_scale=float("nan")), BAD), (dict(residual_scale=float("inf")), BAD), (dict(gate_stride=-1), BAD), (dict(shift_stride=-4), BAD),
    (dict(scale_stride=-4), BAD), (dict(C=8193), NOT), (dict(B=65536), NOT), (dict(B=1 << 15, N=1 << 16), NOT),
    (dict(x_stride=(1, 132)), BAD), (dict(x_stride=(0, -8)), BAD), (dict(s_stride=(0, 1 << 39)), BAD), (dict(y_stride=(1, 4)), BAD),
])
def test_block_norm_refuses_bad_records(kw, status):
    s = block_shape(**kw)
    expect(status, lambda: call_block(s))
    expect(status, lambda: call_block_backward(s))
    if not any(k.endswith("_stride") and isinstance(v, tuple) for k, v in kw.items()):
        assert cn.block_norm_backward_workspace_bytes(s) == 0


def test_block_norm_refuses_bad_pointers_and_overlapping_outputs():
    for kw in (dict(R=None), dict(X=None), dict(S=None), dict(Y=None), dict(R=P + 8), dict(X=P + 2), dict(S=P + 4), dict(Y=P + 8), dict(w=P + 1), dict(gate=P + 2), dict(shift=P + 1), dict(stats=P + 2)):
        expect(BAD, lambda: call_block(block_shape(), **kw))
    for kw in (dict(s_stride=(1, 0)), dict(s_stride=(0, 0)), dict(y_stride=(1, 64)), dict(r_stride=(1, 60))):
        expect(BAD, lambda: call_block(block_shape(**kw)))
    for kw in (dict(dY=None), dict(S=None), dict(X=None), dict(stats=None), dict(dR=None), dict(dX=None), dict(dS=P + 8), dict(dY=P + 2), dict(dR=P + 8), dict(dX=P + 8), dict(dw=P + 2), dict(dgate=P + 1)):
        expect(BAD, lambda: call_block_backward(block_shape(), **kw))
    for kw in (dict(dr_stride=(1, 0)), dict(dx_stride=(0, 128)), dict(ds_stride=(1, 4)), dict(s_stride=(1, -8))):
        expect(BAD, lambda: call_block_backward(block_shape(**kw)))
    need = cn.block_norm_backward_workspace_bytes(block_shape())
    assert need >= 4 * 128 * 4
    for kw in (dict(ws=None), dict(ws=P + 64), dict(ws_bytes=need - 1)):
        expect(cn.ERR_WORKSPACE, lambda: call_block_backward(block_shape(), **kw))


# ---- 8-bit operands ---------------------------------------------------------------------------------------
def quantize_shape(tile=1, **kw):
    x = torch.empty((2, 300, 200), dtype=torch.bfloat16)
    return changed(cn.make_quantize_shape(x, None, None, block_rows=tile), kw)


def call_quantize(s, X=P, Q=P, scale=P):
    return cn.lib().carnator_quantize_fp8(X, ctypes.byref(s), Q, scale, None)


@pytest.mark.parametrize("tile", [1, 128])
def test_quantize_refuses(tile):
    for kw, status in ((dict(B=0), BAD), (dict(N=0), BAD), (dict(K=-4), BAD), (dict(block_rows=64), BAD), (dict(block_rows=0), BAD), (dict(x_dtype=2), BAD), (dict(x_dtype=-1), BAD),
                       (dict(B=65536, N=1), NOT), (dict(N=1 << 27), NOT), (dict(K=(1 << 27) + 1), NOT),
                       (dict(x_stride=(1, 204)), BAD), (dict(x_stride=(0, -8)), BAD), (dict(q_stride=(1, 200)), BAD), (dict(q_stride=(1, 192)), BAD), (dict(q_stride=(0, 0)), BAD),
                       (dict(scale_stride=(1, 0)), BAD), (dict(scale_stride=(2, 0)), BAD), (dict(scale_stride=(0, -1)), BAD), (dict(scale_stride=(0, 1)), BAD), (dict(scale_stride=(2, 1 << 39)), BAD)):
        expect(status, lambda: call_quantize(quantize_shape(tile, **kw)))
    for kw in (dict(X=None), dict(Q=None), dict(scale=None), dict(X=P + 8), dict(Q=P + 8), dict(scale=P + 2)):
        expect(BAD, lambda: call_quantize(quantize_shape(tile), **kw))


def fp8_shape(x="bf16", **kw):
    X = torch.empty((2, 40, 208), dtype=torch.float8_e4m3fn if x == "e4m3" else torch.bfloat16)
    y = torch.empty((2, 40, 144), dtype=torch.bfloat16)
    s = cn.make_linear_fp8_shape(X, torch.empty((144, 208), dtype=torch.float8_e4m3fn), torch.empty((2, 2)), y, x_scale=torch.empty((2, 40, 2)) if x == "e4m3" else None, residual=y)
    return changed(s, kw)


def call_fp8(s, X=P, xs=None, W=P, w_scale=P, bias=P, gate=P, residual=P, Y=P, ws=P, ws_bytes=BIG):
    return cn.lib().carnator_linear_fp8(X, xs, W, w_scale, bias, gate, residual, ctypes.byref(s), Y, ws, ws_bytes, None)


def test_fp8_product_refuses():
    for kw, status in ((dict(B=0), BAD), (dict(N=-3), BAD), (dict(in_features=0), BAD), (dict(out_features=0), BAD), (dict(activation=4), BAD), (dict(activation=-1), BAD),
                       (dict(x_dtype=3), BAD), (dict(x_dtype=-1), BAD), (dict(y_dtype=2), BAD), (dict(bias_dtype=2), BAD), (dict(gate_dtype=3), BAD), (dict(gate_stride=-8), BAD),
                       (dict(B=1 << 15, N=1 << 16), NOT), (dict(B=70000, N=1), NOT), (dict(N=1 << 27), NOT), (dict(in_features=(1 << 27) + 1), NOT), (dict(out_features=(1 << 27) + 1), NOT)):
        s = fp8_shape(**kw)
        expect(status, lambda: call_fp8(s))
        assert cn.linear_fp8_workspace_bytes(s) == 0
    for kw in (dict(x_stride=(1, 204)), dict(x_stride=(1, 200)), dict(x_stride=(0, 0)), dict(w_stride=200), dict(w_stride=216), dict(w_stride=1 << 39), dict(y_stride=(1, 136)),
               dict(y_stride=(0, 64)), dict(residual_stride=(1, 0)), dict(w_scale_stride=(0, -1)), dict(w_scale_stride=(1, 1 << 39))):
        expect(BAD, lambda: call_fp8(fp8_shape(**kw)))
    for kw in (dict(x_stride=(1, 216)), dict(x_scale_stride=(0, -1)), dict(x_scale_stride=(2, 1 << 39))):
        expect(BAD, lambda: call_fp8(fp8_shape("e4m3", **kw), xs=P))
    for kw in (dict(X=None), dict(W=None), dict(w_scale=None), dict(Y=None), dict(X=P + 8), dict(W=P + 8), dict(w_scale=P + 2), dict(Y=P + 8), dict(residual=P + 8), dict(bias=P + 1), dict(gate=P + 2)):
        expect(BAD, lambda: call_fp8(fp8_shape(), **kw))
    expect(BAD, lambda: call_fp8(fp8_shape(), xs=P))               # scales of an X that has none,
    expect(BAD, lambda: call_fp8(fp8_shape("e4m3")))               # and none of one that has
    expect(BAD, lambda: call_fp8(fp8_shape("e4m3"), xs=P + 2))
    for s, xs in ((fp8_shape(), None), (fp8_shape("e4m3"), P)):
        need = cn.linear_fp8_workspace_bytes(s)
        assert need >= 256 + (80 * 256 if xs is None else 0)
        for kw in (dict(ws=None), dict(ws=P + 64), dict(ws_bytes=need - 1)):
            expect(cn.ERR_WORKSPACE, lambda: call_fp8(s, xs=xs, **kw))


def test_calls_without_a_gpu_fail_loudly():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for st in (call_rope(rope_shape()), call_block(block_shape()), call_block_backward(block_shape()), call_quantize(quantize_shape()), call_fp8(fp8_shape())):
        assert st in (cn.ERR_UNSUPPORTED, cn.ERR_CUDA)


def test_python_calls_check_tensors_against_the_record():
    bf, e4 = torch.bfloat16, torch.float8_e4m3fn
    x, freq, pos = torch.empty((1, 2, 6, 16), dtype=bf), torch.empty(8, dtype=torch.float64), torch.empty((1, 6, 1), dtype=torch.int32)
    rs, rp = cn.make_rope_shape(x, x, 8), cn.make_rope_shape(x, x, 8, positions=pos)
    bad = [lambda: cn.rope(x.float(), freq, rs, Y=x), lambda: cn.rope(x, freq.float(), rs, Y=x), lambda: cn.rope(x, freq[:7], rs, Y=x), lambda: cn.rope(x[:, :1], freq, rs, Y=x),
           lambda: cn.rope(x, freq, rs, Y=torch.empty((1, 6, 2, 16), dtype=bf).transpose(1, 2)), lambda: cn.rope(x, freq, rp, positions=pos.long(), Y=x),
           lambda: cn.rope(x, freq, rp, positions=pos[:, :5], Y=x), lambda: cn.make_rope_shape(x[0], None, 8), lambda: cn.make_rope_shape(x.half(), None, 8),
           lambda: cn.make_rope_shape(x.mT.contiguous().mT, None, 8), lambda: cn.make_rope_shape(x, None, 8, positions=pos[0]),
           lambda: cn.make_rope_shape(torch.empty((3, 1, 6, 16)), None, 8, positions=pos.expand(2, 6, 1))]
    t = torch.empty((1, 6, 64), dtype=bf)
    qs = cn.make_quantize_shape(t, None, None)
    bad += [lambda: cn.quantize_fp8(t.float(), qs), lambda: cn.quantize_fp8(t, qs, Q=torch.empty((1, 6, 64), dtype=torch.uint8)), lambda: cn.quantize_fp8(t, qs, scale=torch.empty((1, 6, 2))),
            lambda: cn.quantize_fp8(t[:, :5], qs), lambda: cn.make_quantize_shape(t[0], None, None), lambda: cn.make_quantize_shape(t.half(), None, None)]
    w, sc, y = torch.empty((32, 64), dtype=e4), torch.empty((1, 1)), torch.empty((1, 6, 32), dtype=bf)
    ls = cn.make_linear_fp8_shape(t, w, sc, y)
    bad += [lambda: cn.linear_fp8(t.float(), w, sc, ls, Y=y), lambda: cn.linear_fp8(t, w.view(torch.uint8), sc, ls, Y=y), lambda: cn.linear_fp8(t, w, sc.double(), ls, Y=y),
            lambda: cn.linear_fp8(t, w, torch.empty((1, 2)), ls, Y=y), lambda: cn.linear_fp8(t, w, sc, ls, Y=y.float()), lambda: cn.linear_fp8(t, w, sc, ls, Y=y, bias=torch.empty(31)),
            lambda: cn.linear_fp8(t, w, sc, ls, Y=y, ws=torch.empty(512, dtype=torch.uint8)[::2]), lambda: cn.make_linear_fp8_shape(t, w.to(bf), sc, y),
            lambda: cn.make_linear_fp8_shape(t.to(e4), w, sc, y), lambda: cn.make_linear_fp8_shape(t, w, sc, y, x_scale=torch.empty((1, 6, 1))), lambda: cn.make_linear_fp8_shape(t, w[:, :32], sc, y),
            lambda: cn.make_linear_fp8_shape(t, w, sc[0], y)]
    v, st = torch.empty(64), torch.empty((4, 1, 6))
    bs = cn.make_block_norm_shape(t, t, t, t, weight=v)
    bad += [lambda: cn.block_norm(t.float(), t, bs), lambda: cn.block_norm(t, t[:, :5], bs), lambda: cn.block_norm(t, t, bs, weight=v[:63]), lambda: cn.block_norm(t, t, bs, bias=v.to(bf)),
            lambda: cn.block_norm(t, t, bs, gate=torch.empty((2, 64))), lambda: cn.block_norm(t, t, bs, S=torch.empty((1, 6, 128), dtype=bf)[..., :64][:, ::2]),
            lambda: cn.block_norm(t, t, bs, stats=st[:3]), lambda: cn.block_norm_backward(t, t, t, st.double(), bs), lambda: cn.block_norm_backward(t, t, t, st, bs, dS=t.float()),
            lambda: cn.block_norm_backward(t, t, t, st, bs, ws=torch.empty(1 << 20, dtype=torch.uint8)[::2]), lambda: cn.make_block_norm_shape(t[0], t, t, t), lambda: cn.make_block_norm_shape(t, t.half(), t, t)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    if not torch.cuda.is_available():
        for call in (lambda: cn.rope(x, freq, rs, Y=x), lambda: cn.quantize_fp8(t, qs), lambda: cn.linear_fp8(t, w, sc, ls, Y=y)):
            with pytest.raises(cn.CarnatorError):
                call()


def test_rope_refuses_a_forgotten_positions_argument():
    """Without them the tokens would turn by their places in a plain line; given to a record that has none, they are refused, too."""
    for axes in (1, 2, 3, -1):
        expect(BAD, lambda: call_rope(rope_shape(axes=axes)))
    expect(BAD, lambda: call_rope(rope_shape(True)))
    expect(BAD, lambda: call_rope(rope_shape(), pos=P))
    x, freq = torch.empty((2, 2, 6, 16), dtype=torch.bfloat16), torch.empty(8, dtype=torch.float64)
    for entries, axes in ((1, 1), (2, 1), (2, 3)):
        pos = torch.empty((entries, 6, axes), dtype=torch.int32)
        for Y in (x, None):
            with pytest.raises(ValueError, match="positions"):
                cn.rope(x, freq, cn.make_rope_shape(x, x, 8, positions=pos), Y=Y)
            with pytest.raises(ValueError, match="positions"):
                cn.rope(x, freq, cn.make_rope_shape(x, x, 8), positions=pos, Y=Y)


@pytest.mark.parametrize("x", ["bf16", "e4m3"])
def test_fp8_workspace_is_no_larger_than_what_a_call_passes_on(x):
    """A word of exponents per row and 512 k (in tiles of 256 rows), one per column (tiles of 64 in 1 KB), a note per CTA, x in 8 bits where the call makes it; entries that follow each
    other evenly are one run of rows, padded ones fill tiles of their own."""
    for B, N, K, M, pad in ((65535, 1, 1536, 64, 0), (4096, 1, 5120, 512, 0), (64, 17, 5120, 5120, 0), (64, 17, 5120, 5120, 1), (3, 77, 4096, 1536, 0), (1, 75600, 5120, 5120, 0)):
        X = torch.empty((B, N + pad, K), dtype=torch.float8_e4m3fn if x == "e4m3" else torch.bfloat16, device="meta")[:, :N]
        Y, W = torch.empty((B, N + pad, M), dtype=torch.bfloat16, device="meta")[:, :N], torch.empty((M, K), dtype=torch.float8_e4m3fn, device="meta")
        ks = -(-K // 128)
        xs = torch.empty((B, N + pad, ks), device="meta")[:, :N] if x == "e4m3" else None
        s = cn.make_linear_fp8_shape(X, W, torch.empty((-(-M // 128), ks), device="meta"), Y, x_scale=xs)
        words, tiles = -(-K // 512), B * -(-N // 256) if pad else -(-B * N // 256)
        most = tiles * 256 * words * 4 + -(-M // 64) * words * 1024 + (512 + max(1184, B)) * 4 + (B * N * ks * 128 if x == "bf16" else 0) + 5 * 256
        assert cn.linear_fp8_workspace_bytes(s) <= most, (B, N, K, M, pad)
