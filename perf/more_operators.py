"""Operators between a layer's attention, its projections and the residual stream, as cases that can be timed and compared.

A case is one call on the tokens of a video diffusion transformer: widths, heads and grids are those of the package's workload
records (12 and 40 heads of 128, 21 x 30 x 52 and 21 x 45 x 80 tokens, 226 and 512 text tokens), the usual multiples of them, and
generic sizes between them.

    op            entry point                who calls it
    rope          rope                       on Q and K between their norm and the attention; inverse: its gradient
    block         block_norm                 at the end of a block: its output normed, gated, onto the stream, and the next block's norm
    block_grad    block_norm_backward        its gradients, those of all vectors included
    quantize      quantize_fp8               weights once per model, activations that several projections share
    linear_fp8    linear_fp8                 projections with 8-bit operands: bias, activation, gate per batch entry and residual in one pass

`own` chooses between the plain form (elementary torch operations in 32 bits, angles in 64) and the library's calls.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}

# The fields a case may leave out.
DEFAULTS = dict(
    B=1, H=1,                      # batch entries (2: both guidance branches in one call), heads
    x="bf16", y="bf16", r="f32",   # types of the input, of the output, of the residual stream
    p="bf16",                      # type of weights and biases (of the bias: linear_fp8)
    text=0, T=0, h=1, w=1,         # rope: text tokens in front, then the grid (T = 0: N tokens in a line)
    pt=0, ph=0, pw=0,              # rope: pairs of channels that turn with each axis
    layout="rows",                 # rope: "fused": the heads are Q and K of a fused projection's output
    half=False, inverse=False, given=False, scaled=False,      # rope: halves instead of neighbours; gradient; positions as a tensor; for a longer context
    post="rms", pre="layer",       # block: norms of the block's output and of the stream
    mod=True, gate=False, alpha=1.0, stats=False,
    tile=1,                        # quantize: rows that share a scale (1: activations, 128: weights)
    bias=True, act="none", residual=False,
)


def _full(case):
    return {**DEFAULTS, **case}


def listed():
    return [
        # the smallest: one token per guidance branch, its position in hand; latency
        dict(name="rope_token", op="rope", B=2, H=12, N=1, D=128, pt=64, half=True, given=True),
        # the largest: Q and K of a 14B-shaped layer at 720p, read beside V in the fused projection's output
        dict(name="rope_wan14b", op="rope", H=80, N=75600, D=128, T=21, h=45, w=80, pt=22, ph=21, pw=21, layout="fused"),
        # the gradient on text and video tokens, heads of 64 of which 48 channels turn, positions stretched to a longer clip
        dict(name="rope_grad_part", op="rope", B=2, H=24, N=17776, D=64, text=226, T=13, h=30, w=45, pt=8, ph=8, pw=8, half=True, inverse=True, scaled=True),
        # the smallest: one conditioning row per guidance branch
        dict(name="block_rows", op="block", B=2, N=1, C=1536, gate=True),
        # the largest: end of a block of a 14B-shaped layer in training, statistics kept for the backward pass
        dict(name="block_wan14b", op="block", N=75600, C=5120, gate=True, stats=True),
        # a short text sequence of odd width, stream in 16 bits
        dict(name="block_grad_text", op="block_grad", B=2, N=77, C=1541, r="bf16", p="f32", post="layer", gate=True, alpha=0.5),
        # an ordinary layer's tokens
        dict(name="block_grad_wan13b", op="block_grad", N=32760, C=1536, p="f32", gate=True),
        # the weights of a 14B-shaped layer's feed-forward half, once per model
        dict(name="quantize_weight", op="quantize", N=13824, K=5120, tile=128),
        # an ordinary layer's tokens in front of its projections
        dict(name="quantize_wan13b", op="quantize", N=32760, K=1536),
        # one timestep through the conditioning layer: a matrix against a single row
        dict(name="fp8_step", op="linear_fp8", N=1, K=1536, M=1536, act="silu"),
        # text tokens into the model's width
        dict(name="fp8_text", op="linear_fp8", N=512, K=4096, M=5120, act="gelu_tanh"),
        # output projection behind attention, gated, onto the 32-bit residual stream: 14B-shaped
        dict(name="fp8_out_wan14b", op="linear_fp8", N=75600, K=5120, M=5120, y="f32", gate=True, residual=True, p="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.3 else max(8, n // 8 * 8) if rng.random() < 0.5 else -(-n // 64) * 64


def _draw_rope(rng, c):
    c["D"], c["H"], c["x"] = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 256]), _log(rng, 1, 80), rng.choice(["bf16", "bf16", "f32"])
    pairs = c["D"] // 2 if rng.random() < 0.6 else rng.randint(3, c["D"] // 2)
    c["half"], c["inverse"], c["scaled"] = rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.4
    c["layout"] = rng.choice(["rows", "heads", "fused"])
    if rng.random() < 0.6:
        c["T"], c["h"], c["w"] = rng.randint(1, 24), rng.randint(1, 45), rng.randint(1, 80)
        c["text"] = rng.choice([0, 0, 226, 512, rng.randint(1, 600)])
        c["N"] = c["text"] + c["T"] * c["h"] * c["w"]
        c["ph"] = c["pw"] = pairs // 3
        c["pt"] = pairs - 2 * c["ph"]
    else:
        c["pt"], c["given"] = pairs, rng.random() < 0.5


def draw(rng):
    while True:
        op = rng.choice(["rope", "rope", "block", "block_grad", "quantize", "linear_fp8", "linear_fp8", "linear_fp8"])
        c = dict(op=op, B=rng.choice([1, 1, 2, 3]), N=_log(rng, 1, 75600))
        if op == "rope":
            _draw_rope(rng, c)
        elif op in ("block", "block_grad"):
            c["C"], c["post"], c["pre"] = _width(rng, 16, 8192), rng.choice(["none", "layer", "rms", "rms"]), rng.choice(["layer", "rms"])
            c["r"], c["x"], c["y"], c["p"] = (rng.choice(["f32", "bf16"]) for _ in range(4))
            c["mod"], c["gate"], c["alpha"] = rng.random() < 0.7, rng.random() < 0.7, rng.choice([1.0, 1.0, 0.5])
            if op == "block":
                c["stats"] = rng.random() < 0.5
        elif op == "quantize":
            c["K"], c["tile"], c["x"] = _width(rng, 16, 13824), rng.choice([1, 128]), rng.choice(["bf16", "bf16", "f32"])
            c["B"] = 1 if c["tile"] == 128 else c["B"]
        else:
            c["K"], c["M"] = _width(rng, 64, 8960), _width(rng, 64, 13824)
            c["act"], c["x"] = rng.choice(["none", "gelu_tanh", "gelu", "silu"]), rng.choice(["bf16", "bf16", "f32", "e4m3"])
            c["gate"], c["p"], c["bias"], c["residual"] = rng.random() < 0.4, rng.choice(["f32", "bf16"]), rng.random() < 0.8, rng.random() < 0.4
            c["y"] = rng.choice(["bf16", "f32"]) if c["residual"] else rng.choice(["bf16", "bf16", "f32"])
        w = work(c)
        if w["flops"] <= 3.9e12 and w["bytes"] <= 4.4e9:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _empty(shape, dtype):
    """Rows that start on 16-byte boundaries: [..., n] inside a buffer [..., n rounded up]."""
    unit = 16 // torch.empty((), dtype=dtype).element_size()
    return torch.empty((*shape[:-1], -(-shape[-1] // unit) * unit), dtype=dtype, device="cuda")[..., :shape[-1]]


def _rows(gen, shape, dtype, scale=1.0):
    return _empty(shape, dtype).copy_(torch.randn(shape, device="cuda", generator=gen).mul_(scale))


def _tokens(gen, shape, dtype):
    """Activations: channels of different size and offset, as residual streams have them."""
    spread = torch.exp(0.5 * torch.randn(shape[-1], device="cuda", generator=gen))
    offset = 0.5 * torch.randn(shape[-1], device="cuda", generator=gen)
    return _empty(shape, dtype).copy_(torch.randn(shape, device="cuda", generator=gen).mul_(spread).add_(offset))


def _vec(gen, shape, dtype, scale, around=0.0):
    return (around + scale * torch.randn(shape, device="cuda", generator=gen)).to(dtype)


def _frequencies(c):
    """Radians per position of every pair, and the amplitude: base 10000 per axis; stretched fourfold by wavelength where scaled: pairs that turn over 32
    times in the trained length stay, those that turn less than once are slowed down fourfold, those between by a ramp."""
    f, lengths = [], (c["T"] or c["N"], c["h"], c["w"])
    for pairs, length in zip((c["pt"], c["ph"], c["pw"]), lengths):
        for i in range(pairs):
            g = 10000.0 ** (-i / pairs)
            if c["scaled"]:
                keep = min(max((length * g / (2 * math.pi) - 1.0) / 31.0, 0.0), 1.0)
                g = g * (keep + (1 - keep) / 4.0)
            f.append(g)
    return f, 0.1 * math.log(4.0) + 1 if c["scaled"] else 1.0


def _prepare_rope(c, gen):
    B, H, N, D, dtype = c["B"], c["H"], c["N"], c["D"], _DTYPE[c["x"]]
    if c["layout"] == "heads":        # [B,H,N,D]
        x = torch.randn((B, H, N, D), device="cuda", generator=gen).to(dtype)
    elif c["layout"] == "rows":       # tokens first
        x = torch.randn((B, N, H, D), device="cuda", generator=gen).to(dtype).transpose(1, 2)
    else:                             # beside V, half as many heads
        x = torch.empty((B, N, H + (H + 1) // 2, D), dtype=dtype, device="cuda")[:, :, :H].transpose(1, 2)
        x.copy_(torch.randn((B, H, N, D), device="cuda", generator=gen))
    s = dict(op="rope", x=x, half=c["half"], inverse=c["inverse"], pairs=(c["pt"], c["ph"], c["pw"]), text=c["text"], grid=(c["T"] or N, c["h"], c["w"]), positions=None)
    if c["given"]:                    # each entry at a place of its own, far out
        s["positions"] = torch.randint(0, 1 << 20, (B, N, 1), device="cuda", generator=gen, dtype=torch.int32)
    f, s["amplitude"] = _frequencies(c)
    s["freq"] = torch.tensor(f, dtype=torch.float64, device="cuda")
    if own:
        from paper_2609_32420_b200 import carnator as cn
        scaling = dict(scaling=cn.ROPE_SCALE_RAMP, factor=(4.0, 4.0, 4.0), original=s["grid"], low=1.0, high=32.0) if c["scaled"] else {}
        s["freq"], amplitude = cn.rope_frequencies(s["pairs"], theta=10000.0, device="cuda", **scaling)
        s["y"] = torch.empty((B, N, H, D), dtype=dtype, device="cuda").transpose(1, 2) if c["layout"] != "heads" else torch.empty_like(x)
        s["shape"] = cn.make_rope_shape(x, s["y"], s["pairs"], n_text=s["text"], grid=s["grid"], positions=s["positions"],
                                        layout=cn.ROPE_HALF if c["half"] else cn.ROPE_INTERLEAVED, amplitude=amplitude, inverse=c["inverse"])
    return s


def _norm_stats(t, kind):
    t = t.double()
    mean = t.mean(-1) if kind == "layer" else torch.zeros(t.shape[:-1], dtype=torch.float64, device="cuda")
    rstd = ((t - mean[..., None]).square().mean(-1) + EPS).rsqrt() if kind != "none" else torch.ones_like(mean)
    return mean.float(), rstd.float()


def _prepare_block(c, gen):
    B, N, C, p = c["B"], c["N"], c["C"], _DTYPE[c["p"]]
    rt, xt, yt = _DTYPE[c["r"]], _DTYPE[c["x"]], _DTYPE[c["y"]]
    s = dict(op=c["op"], post=c["post"], pre=c["pre"], alpha=c["alpha"], r_dtype=rt, x_dtype=xt, y_dtype=yt, keep=c["stats"])
    s.update(pw=None, pb=None, gate=None, w=None, b=None, shift=None, scale=None)
    s["x"] = _rows(gen, (B, N, C), xt)
    if c["post"] != "none":
        s["pw"] = _vec(gen, C, p, 0.2, 1.0)
        s["pb"] = _vec(gen, C, p, 0.1) if c["post"] == "layer" else None
    if not c["mod"] or c["pre"] == "rms":
        s["w"] = _vec(gen, C, p, 0.2, 1.0)
        s["b"] = _vec(gen, C, p, 0.1) if c["pre"] == "layer" else None
    six = 0.3 * torch.randn((B, 6, -(-C // 4) * 4), device="cuda", generator=gen)       # the rows that a layer's modulation gives each batch entry
    if c["gate"]:
        s["gate"] = six[:, 2, :C]
    if c["mod"]:
        s["shift"], s["scale"] = six[:, 3, :C], six[:, 4, :C]
    if c["op"] == "block":
        s["r"] = _tokens(gen, (B, N, C), rt)
    else:
        s["s"], s["dy"], s["ds"] = _tokens(gen, (B, N, C), rt), _rows(gen, (B, N, C), yt), _rows(gen, (B, N, C), rt)
        s["stats"] = torch.stack([*_norm_stats(s["x"], c["post"]), *_norm_stats(s["s"], c["pre"])])
    if own:
        from paper_2609_32420_b200 import carnator as cn
        kind = dict(none=cn.NORM_NONE, layer=cn.NORM_LAYER, rms=cn.NORM_RMS)
        how = dict(post_weight=s["pw"], gate=s["gate"], weight=s["w"], scale=s["scale"], post=kind[c["post"]], pre=kind[c["pre"]], post_eps=EPS, eps=EPS, residual_scale=c["alpha"])
        if c["op"] == "block":
            s["s"], s["y"] = _empty((B, N, C), rt), _empty((B, N, C), yt)
            s["stats"] = torch.empty((4, B, N), device="cuda") if c["stats"] else None
            s["shape"] = cn.make_block_norm_shape(s["r"], s["x"], s["s"], s["y"], **how)
        else:
            s["dr"], s["dx"] = _empty((B, N, C), rt), _empty((B, N, C), xt)
            s["shape"] = cn.make_block_norm_shape(s["ds"], s["x"], s["s"], s["dy"], dS=s["ds"], dR=s["dr"], dX=s["dx"], **how)
            s["ws"] = torch.empty(cn.block_norm_backward_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    return s


def _scale_room(B, N, blocks):
    """[B,N,blocks] with the rows beside each other, as the products read them."""
    return torch.empty((B, blocks, N), device="cuda").transpose(1, 2)


def _prepare_quantize(c, gen):
    B, N, K = c["B"], c["N"], c["K"]
    s = dict(op="quantize", tile=c["tile"], x=_rows(gen, (B, N, K), _DTYPE[c["x"]], 1 / math.sqrt(K)) if c["tile"] > 1 else _tokens(gen, (B, N, K), _DTYPE[c["x"]]))
    if own:
        from paper_2609_32420_b200 import carnator as cn
        s["q"] = _empty((B, N, K), torch.float8_e4m3fn)
        s["s"] = _scale_room(B, N, -(-K // BLOCK)) if c["tile"] == 1 else torch.empty((B, -(-N // BLOCK), -(-K // BLOCK)), device="cuda")
        s["shape"] = cn.make_quantize_shape(s["x"], s["q"], s["s"], block_rows=c["tile"])
    return s


def _prepare_fp8(c, gen):
    B, N, K, M = c["B"], c["N"], c["K"], c["M"]
    y, p = _DTYPE[c["y"]], _DTYPE[c["p"]]
    s = dict(op="linear_fp8", act=c["act"], y_dtype=y, x_scale=None)
    s["x"] = _tokens(gen, (B, N, K), torch.bfloat16 if c["x"] == "e4m3" else _DTYPE[c["x"]])
    if c["x"] == "e4m3":              # in 8 bits already: another projection's input too
        q, scale = _quantized(s["x"], 1)
        s["x"], s["x_scale"] = _empty((B, N, K), q.dtype).copy_(q), _scale_room(B, N, scale.shape[-1]).copy_(scale)
    q, scale = _quantized(_rows(gen, (1, M, K), torch.bfloat16, 1 / math.sqrt(K)), BLOCK)
    s["w"], s["w_scale"] = _empty((M, K), q.dtype).copy_(q[0]), scale[0].contiguous()
    s["bias"] = _vec(gen, M, p, 0.1) if c["bias"] else None
    s["gate"] = _rows(gen, (B, 6, M), torch.float32, 0.3)[:, 2] if c["gate"] else None
    s["residual"] = _rows(gen, (B, N, M), y) if c["residual"] else None
    if own:
        from paper_2609_32420_b200 import carnator as cn
        act = {"none": cn.ACT_NONE, "gelu_tanh": cn.ACT_GELU_TANH, "gelu": cn.ACT_GELU, "silu": cn.ACT_SILU}[c["act"]]
        s["y"] = _empty((B, N, M), y)
        s["shape"] = cn.make_linear_fp8_shape(s["x"], s["w"], s["w_scale"], s["y"], x_scale=s["x_scale"], residual=s["residual"], bias=s["bias"], gate=s["gate"], activation=act)
        s["ws"] = torch.empty(cn.linear_fp8_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    return s


_PREPARE = dict(rope=_prepare_rope, block=_prepare_block, block_grad=_prepare_block, quantize=_prepare_quantize, linear_fp8=_prepare_fp8)


def prepare(case, seed):
    c = _full(case)
    return _PREPARE[c["op"]](c, torch.Generator(device="cuda").manual_seed(int(seed)))


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _angles(s):
    """[B or 1, tokens that turn, pairs] in 64 bits."""
    if s["positions"] is not None:
        return s["positions"].double() * s["freq"]
    T, h, w = s["grid"]
    n = torch.arange(T * h * w, device="cuda")
    pos = torch.stack((n // (h * w), n // w % h, n % w), dim=-1).double()
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(s["pairs"], device="cuda"), output_size=sum(s["pairs"]))
    return (pos[:, axis] * s["freq"])[None]


def _turn(x, cos, sin, half):
    """The pairs of x's channels turned; cos and sin [B,1,N,pairs]."""
    pairs = cos.shape[-1]
    if half:
        u, v = x[..., :pairs], x[..., pairs:2 * pairs]
    else:
        u, v = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
    a, b = u * cos - v * sin, u * sin + v * cos
    turned = torch.cat((a, b), -1) if half else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((turned, x[..., 2 * pairs:]), -1)


def _plain_rope(s):
    angle = _angles(s)[:, None]
    if s["inverse"]:
        angle = -angle
    x = s["x"].float()
    y = _turn(x[:, :, s["text"]:], (s["amplitude"] * angle.cos()).float(), (s["amplitude"] * angle.sin()).float(), s["half"])
    return dict(y=torch.cat((x[:, :, :s["text"]], y), 2).to(s["x"].dtype))


def _plain_norm(t, kind):
    """(normalised, mean, reciprocal deviation)"""
    if kind == "none":
        return t, torch.zeros_like(t[..., 0]), torch.ones_like(t[..., 0])
    mean = t.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(t[..., :1])
    d = t - mean
    rstd = torch.rsqrt(d.square().mean(-1, keepdim=True) + EPS)
    return d * rstd, mean[..., 0], rstd[..., 0]


def _affine(t, w, b, shift=None, scale=None):
    t = t if w is None else t * w.float()
    t = t if b is None else t + b.float()
    return t if scale is None else t * (1 + scale[:, None]) + shift[:, None]


def _plain_block(s):
    xh, m1, r1 = _plain_norm(s["x"].float(), s["post"])
    p = _affine(xh, s["pw"], s["pb"])
    if s["gate"] is not None:
        p = p * s["gate"][:, None]
    total = s["alpha"] * s["r"].float() + p
    sh, m2, r2 = _plain_norm(total, s["pre"])
    out = dict(s=total.to(s["r_dtype"]), y=_affine(sh, s["w"], s["b"], s["shift"], s["scale"]).to(s["y_dtype"]))
    if s["keep"]:
        out["stats"] = torch.stack((m1, r1, m2, r2))
    return out


def _through_norm(g, xh, rstd, kind):
    if kind == "none":
        return g
    d = g - xh * (g * xh).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(-1, keepdim=True)
    return rstd * d


def _plain_block_grad(s):
    m1, r1, m2, r2 = s["stats"][..., None]
    one = torch.ones((), device="cuda")
    gate = one if s["gate"] is None else s["gate"]
    pw, w = (one if t is None else t.float() for t in (s["pw"], s["w"]))
    k = one if s["scale"] is None else 1 + s["scale"]
    dy, xh, sh = s["dy"].float(), (s["x"].float() - m1) * r1, (s["s"].float() - m2) * r2
    G = s["ds"].float() + _through_norm(dy * (w * k if s["scale"] is None else (w * k)[:, None]), sh, r2, s["pre"])
    dx = _through_norm(G * (gate * pw if s["gate"] is None else (gate * pw)[:, None]), xh, r1, s["post"])
    out = dict(dr=(s["alpha"] * G).to(s["r_dtype"]), dx=dx.to(s["x_dtype"]))
    P1, S1, P2, S2 = (G * xh).sum(1), G.sum(1), (dy * sh).sum(1), dy.sum(1)
    if s["pw"] is not None:
        out["dpost_weight"] = (gate * P1).sum(0)
    if s["pb"] is not None:
        out["dpost_bias"] = (gate * S1).sum(0)
    if s["gate"] is not None:
        out["dgate"] = pw * P1 + (0 if s["pb"] is None else s["pb"].float() * S1)
    if s["w"] is not None:
        out["dweight"] = (k * P2).sum(0)
    if s["b"] is not None:
        out["dbias"] = (k * S2).sum(0)
    if s["scale"] is not None:
        out["dshift"], out["dscale"] = S2, w * P2 + (0 if s["b"] is None else s["b"].float() * S2)
    return out


def _tiles(t, tile):
    """[B, row tiles, tile, channel blocks, 128], filled up with zeros."""
    B, N, K = t.shape
    t = torch.nn.functional.pad(t, (0, -K % BLOCK, 0, -N % tile))
    return t.view(B, -(-N // tile), tile, -(-K // BLOCK), BLOCK)


def _quantized(x, tile):
    """(e4m3 values, scales): a scale is the smallest power of two that brings the block's largest magnitude to 448 or less."""
    B, N, K = x.shape
    t = _tiles(x.float(), tile)
    bits = t.abs().amax((2, 4)).clamp(min=2.0 ** -100).view(torch.int32)
    power = (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()       # 448 = 1.75 x 2^8
    scale, inverse = (power << 23).view(torch.float32), (254 - power << 23).view(torch.float32)
    q = (t * inverse[:, :, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(B, -1, q.shape[3] * BLOCK)[:, :N, :K], scale


def _plain_quantize(s):
    q, scale = _quantized(s["x"], s["tile"])
    return dict(q=q, scale=scale)


def _values(q, scale, tile):
    B, N, K = q.shape
    t = _tiles(q.to(scale.dtype), tile) * scale[:, :, None, :, None]
    return t.view(B, t.shape[1] * tile, -1)[:, :N, :K]


_A, _B = math.sqrt(2 / math.pi), 0.044715


def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_A * (z + _B * z * z * z)))
    return z


def _plain_fp8(s):
    q, scale = (s["x"], s["x_scale"]) if s["x_scale"] is not None else _quantized(s["x"], 1)
    z = torch.matmul(_values(q, scale, 1), _values(s["w"][None], s["w_scale"][None], BLOCK)[0].t())
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, s["act"])
    if s["gate"] is not None:
        y = y * s["gate"][:, None]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(s["y_dtype"]))


_PLAIN = dict(rope=_plain_rope, block=_plain_block, block_grad=_plain_block_grad, quantize=_plain_quantize, linear_fp8=_plain_fp8)


# ---- one pass ----------------------------------------------------------------------------------------------------------
def _own_run(s):
    from paper_2609_32420_b200 import carnator as cn
    op = s["op"]
    if op == "rope":
        return dict(y=cn.rope(s["x"], s["freq"], s["shape"], positions=s["positions"], Y=s["y"]))
    if op == "block":
        S, Y = cn.block_norm(s["r"], s["x"], s["shape"], post_weight=s["pw"], post_bias=s["pb"], gate=s["gate"], weight=s["w"], bias=s["b"],
                             shift=s["shift"], scale=s["scale"], S=s["s"], Y=s["y"], stats=s["stats"])
        return dict(s=S, y=Y, stats=s["stats"])
    if op == "block_grad":
        g = cn.block_norm_backward(s["dy"], s["s"], s["x"], s["stats"], s["shape"], dS=s["ds"], post_weight=s["pw"], post_bias=s["pb"], gate=s["gate"],
                                   weight=s["w"], bias=s["b"], scale=s["scale"], dR=s["dr"], dX=s["dx"], ws=s["ws"])
        return dict(dr=g.dR, dx=g.dX, dpost_weight=g.dpost_weight, dpost_bias=g.dpost_bias, dgate=g.dgate, dweight=g.dweight, dbias=g.dbias,
                    dshift=g.dshift, dscale=g.dscale)
    if op == "quantize":
        q, scale = cn.quantize_fp8(s["x"], s["shape"], Q=s["q"], scale=s["s"])
        return dict(q=q, scale=scale)
    y, _ = cn.linear_fp8(s["x"], s["w"], s["w_scale"], s["shape"], x_scale=s["x_scale"], bias=s["bias"], gate=s["gate"], residual=s["residual"], Y=s["y"], ws=s["ws"])
    return dict(y=y)


def run(s):
    return _own_run(s) if own else _PLAIN[s["op"]](s)


# ---- the definitions in 64 bits, gradients by torch's own differentiation -------------------------------------------------
_ACT64 = dict(none=lambda z: z, silu=torch.nn.functional.silu, gelu=torch.nn.functional.gelu,
              gelu_tanh=lambda z: torch.nn.functional.gelu(z, approximate="tanh"))


def _exact_rope(s):
    """Pairs as complex numbers, times m exp(i angle)."""
    pairs, text = sum(s["pairs"]), s["text"]
    x = s["x"].double()
    head, rest = x[:, :, text:, :2 * pairs], x[:, :, text:, 2 * pairs:]
    B, H, N, _ = head.shape
    z = head.reshape(B, H, N, 2, pairs).transpose(-1, -2) if s["half"] else head.reshape(B, H, N, pairs, 2)
    z = torch.view_as_complex(z.contiguous())
    if s["positions"] is not None:
        angle = torch.einsum("bna,p->bnp", s["positions"].double(), s["freq"])[:, None]
    else:
        axes = torch.cartesian_prod(*(torch.arange(n, device="cuda", dtype=torch.float64) for n in s["grid"]))
        angle = torch.cat([torch.outer(axes[:, a], f) for a, f in enumerate(torch.split(s["freq"], list(s["pairs"])))], -1)
    z = z * torch.polar(torch.full_like(angle, s["amplitude"]), -angle if s["inverse"] else angle)
    z = torch.view_as_real(z)
    z = z.transpose(-1, -2).reshape(B, H, N, 2 * pairs) if s["half"] else z.reshape(B, H, N, 2 * pairs)
    return dict(y=torch.cat((x[:, :, :text], torch.cat((z, rest), -1)), 2))


def _leaf(t):
    return None if t is None else t.double().requires_grad_()


def _norm64(t, kind, w, b):
    C = t.shape[-1:]
    if kind == "layer":
        return torch.nn.functional.layer_norm(t, C, w, b, EPS)
    return t if kind == "none" else torch.nn.functional.rms_norm(t, C, w, EPS)


def _modulated(y, t):
    return y if t["scale"] is None else torch.addcmul(t["shift"][:, None], y, 1 + t["scale"][:, None])


def _gated(p, t):
    return p if t["gate"] is None else torch.einsum("bnc,bc->bnc", p, t["gate"])


def _stats64(t, kind):
    mean = t.mean(-1) if kind == "layer" else 0 * t[..., 0]
    return mean, ((t.square().mean(-1) - mean ** 2 + EPS) ** -0.5 if kind != "none" else 1 + 0 * mean)


def _exact_block(s):
    t = {k: None if s[k] is None else s[k].double() for k in ("r", "x", "pw", "pb", "gate", "w", "b", "shift", "scale")}
    total = torch.add(_gated(_norm64(t["x"], s["post"], t["pw"], t["pb"]), t), t["r"], alpha=s["alpha"])
    out = dict(s=total, y=_modulated(_norm64(total, s["pre"], t["w"], t["b"]), t))
    if s["keep"]:
        out["stats"] = torch.stack([*_stats64(t["x"], s["post"]), *_stats64(total, s["pre"])])
    return out


def _exact_block_grad(s):
    t = {k: _leaf(s[k]) for k in ("s", "x", "pw", "pb", "gate", "w", "b", "shift", "scale")}
    _modulated(_norm64(t["s"], s["pre"], t["w"], t["b"]), t).backward(s["dy"].double())
    G = t["s"].grad + s["ds"].double()
    _gated(_norm64(t["x"], s["post"], t["pw"], t["pb"]), t).backward(G)
    names = dict(dx="x", dpost_weight="pw", dpost_bias="pb", dgate="gate", dweight="w", dbias="b", dshift="shift", dscale="scale")
    return dict(dr=s["alpha"] * G, **{n: t[k].grad for n, k in names.items() if t[k] is not None})


def _quantized64(x, tile):
    """The nearest value with four significant bits (a step of 2^-9 below 2^-6), ties to even, of the block's values over the scale."""
    B, N, K = x.shape
    rows, cols = torch.arange(N, device="cuda") // tile, torch.arange(K, device="cuda") // BLOCK
    a = x.double()
    most = torch.zeros((B, int(rows[-1]) + 1, K), dtype=torch.float64, device="cuda").index_reduce_(1, rows, a.abs(), "amax")
    most = torch.zeros((B, most.shape[1], int(cols[-1]) + 1), dtype=torch.float64, device="cuda").index_reduce_(2, cols, most, "amax")
    most = most.clamp(min=2.0 ** -100)
    scale = torch.exp2(torch.floor(torch.log2(most)) - 8)
    scale = torch.where(448 * scale < most, 2 * scale, scale)
    v = a / scale[:, rows][:, :, cols]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step, scale


def _exact_quantize(s):
    q, scale = _quantized64(s["x"], s["tile"])
    return dict(q=q, scale=scale)


def _exact_fp8(s):
    rows, cols = (torch.arange(n, device="cuda") // BLOCK for n in s["w"].shape)
    w = s["w"].double() * s["w_scale"].double()[rows][:, cols]
    q, scale = (s["x"].double(), s["x_scale"].double()) if s["x_scale"] is not None else _quantized64(s["x"], 1)
    y = _ACT64[s["act"]](torch.nn.functional.linear(q.mul_(scale[:, :, cols]), w, None if s["bias"] is None else s["bias"].double()))
    y = y if s["gate"] is None else torch.einsum("bnm,bm->bnm", y, s["gate"].double())
    return dict(y=y if s["residual"] is None else y + s["residual"])


_EXACT = dict(rope=_exact_rope, block=_exact_block, block_grad=_exact_block_grad, quantize=_exact_quantize, linear_fp8=_exact_fp8)


def exact(case, seed):
    s = prepare(case, seed)
    with torch.enable_grad():
        return _EXACT[s["op"]](s)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    """Each input read once, each output written once; the products of the matrix cores count as flops, the few operations per
    element of the others do not bound anything."""
    c = _full(case)
    size = {"f32": 4.0, "bf16": 2.0, "e4m3": 1.0}
    B, N, op = c["B"], c["N"], c["op"]
    if op == "rope":
        values = float(B * N * c["H"] * c["D"])
        return {"bytes": 2 * size[c["x"]] * values + (4.0 * B * N if c["given"] else 0) + 8.0 * (c["pt"] + c["ph"] + c["pw"]), "flops": 3.0 * values}
    if op in ("block", "block_grad"):
        C, rows = c["C"], B * N
        vectors = size[c["p"]] * C * (dict(none=0, rms=1, layer=2)[c["post"]] + (1 if c["pre"] == "rms" else 0 if c["mod"] else 2))
        vectors += 4.0 * B * C * ((1 if c["gate"] else 0) + (2 if c["mod"] else 0))
        if op == "block":
            return {"bytes": rows * C * (2 * size[c["r"]] + size[c["x"]] + size[c["y"]]) + vectors + (16.0 * rows if c["stats"] else 0), "flops": 14.0 * rows * C}
        return {"bytes": rows * C * (3 * size[c["r"]] + 2 * size[c["x"]] + size[c["y"]]) + 2 * vectors + 16.0 * rows, "flops": 30.0 * rows * C}
    K = c["K"]
    if op == "quantize":
        return {"bytes": B * N * K * (size[c["x"]] + 1.0) + 4.0 * B * -(-N // c["tile"]) * -(-K // BLOCK), "flops": 2.0 * B * N * K}
    M, rows, y = c["M"], B * N, size[c["y"]]
    scales = 4.0 * -(-M // BLOCK) * -(-K // BLOCK) + (4.0 * rows * -(-K // BLOCK) if c["x"] == "e4m3" else 0)
    return {"bytes": size[c["x"]] * rows * K + 1.0 * M * K + scales + y * rows * M * (2 if c["residual"] else 1)
            + (size[c["p"]] * M if c["bias"] else 0) + (4.0 * B * M if c["gate"] else 0), "flops": 2.0 * rows * K * M}
