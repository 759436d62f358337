"""The operators around a layer's attention, as cases that can be timed and compared.

A case is one call on the tokens of a video diffusion transformer: the widths and token counts are those of the package's
workload records (12 and 40 heads of 128, 32760 and 75600 tokens, 226 and 512 text tokens), the usual multiples of them (six
modulation rows, the widths of feed-forward layers), and generic sizes between them.

    op           entry point             who calls it
    norm         layer_norm              in front of every projection (modulated per request), and on Q and K per head (affine)
    norm_grad    layer_norm_backward     its gradients, those of weight, bias, shift and scale included
    linear       linear                  projections: bias, activation, gate per batch entry and residual in one pass
    linear_grad  linear_backward         its gradients from the saved pre-activation

`own` chooses between the plain form (elementary torch operations in 32 bits) and the library's calls.
"""
import math

import torch

own = False

EPS = 1e-6
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}

# The fields a case may leave out.
DEFAULTS = dict(
    B=1, H=1,            # batch entries (2: both guidance branches in one call), heads (1: whole token rows)
    layout="rows",       # "heads": the rows are heads of one third of a fused projection's output
    x="bf16", y="bf16",  # types of the input and of the output (linear: of output and residual)
    p="bf16",            # type of weight and bias (norm), of the bias (linear)
    affine=True,         # norm: weight and bias
    mod=False,           # norm: shift and scale, one row per batch entry
    stats=False,         # norm: a training pass keeps mean and reciprocal deviation
    bias=True, act="none", gate=False, residual=False,
    keep=False,          # linear: a training pass keeps the pre-activation
    need_x=True,         # linear_grad: False where the input takes no gradient (the first layer)
)


def _full(case):
    return {**DEFAULTS, **case}


def listed():
    return [
        # the smallest call: one conditioning row per guidance branch, modulated; latency
        dict(name="norm_rows", op="norm", B=2, N=1, C=1536, x="f32", affine=False, mod=True),
        # Q in front of attention, 12 heads of 128, read from and written beside the fused projection's output
        dict(name="norm_heads", op="norm", H=12, N=32760, C=128, layout="heads"),
        # the largest: residual stream of a 14B-shaped layer in 32 bits, modulated, statistics kept for the backward pass
        dict(name="norm_wan14b", op="norm", N=75600, C=5120, x="f32", affine=False, mod=True, stats=True),
        # a short text sequence of odd width, rows padded to 16 bytes, two entries
        dict(name="norm_grad_text", op="norm_grad", B=2, N=77, C=1541, p="f32"),
        # an ordinary layer's tokens, modulated and affine, residual stream in 32 bits
        dict(name="norm_grad_wan13b", op="norm_grad", N=32760, C=1536, x="f32", p="f32", mod=True),
        # one timestep through the conditioning layer: a matrix against a single row
        dict(name="linear_step", op="linear", N=1, K=1536, M=1536, act="silu"),
        # the modulation of both guidance branches: six rows of width 5120 from one, the weights are all of the traffic
        dict(name="linear_modulation", op="linear", B=2, N=1, K=5120, M=30720, y="f32"),
        # text tokens into the model's width
        dict(name="linear_text", op="linear", N=512, K=4096, M=5120, act="gelu_tanh"),
        # feed-forward, upper half, of a 1.3B-shaped layer in training: the pre-activation is kept
        dict(name="linear_ffn_wan13b", op="linear", N=32760, K=1536, M=8960, act="gelu_tanh", keep=True),
        # output projection behind attention, gated, onto the 32-bit residual stream: 14B-shaped
        dict(name="linear_out_wan14b", op="linear", N=75600, K=5120, M=5120, y="f32", gate=True, residual=True, p="f32"),
        # gradients on a short sequence of odd widths, arriving from a 32-bit residual stream
        dict(name="linear_grad_odd", op="linear_grad", B=2, N=333, K=1000, M=1541, act="gelu", gate=True, y="f32"),
        # gradients of the feed-forward's upper half
        dict(name="linear_grad_wan13b", op="linear_grad", N=32760, K=1536, M=8960, act="gelu_tanh"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.3 else max(8, n // 8 * 8) if rng.random() < 0.5 else -(-n // 64) * 64


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm_grad", "linear", "linear", "linear_grad"])
        c = dict(op=op, B=rng.choice([1, 1, 2, 3]), N=_log(rng, 1, 75600))
        if op in ("norm", "norm_grad"):
            c["x"], c["p"] = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
            if rng.random() < 0.3:
                c["H"], c["C"], c["layout"], c["x"] = _log(rng, 2, 48), rng.choice([64, 128]), "heads", "bf16"
            else:
                c["C"], c["mod"] = _width(rng, 16, 8192), rng.random() < 0.5
            c["affine"] = rng.random() < 0.6 or not c.get("mod")
            c["y"] = rng.choice(["bf16", "bf16", "f32"])
            if op == "norm":
                c["stats"] = rng.random() < 0.5
        else:
            c["K"], c["M"] = _width(rng, 64, 8960), _width(rng, 64, 13824)
            c["act"] = rng.choice(["none", "gelu_tanh", "gelu", "silu"])
            c["gate"], c["p"] = rng.random() < 0.4, rng.choice(["f32", "bf16"])
            if op == "linear":
                c["bias"], c["residual"] = rng.random() < 0.8, rng.random() < 0.4
                c["keep"] = rng.random() < 0.4
                c["y"] = "f32" if c["residual"] and rng.random() < 0.5 else "bf16"
            else:
                c["need_x"] = rng.random() < 0.85
                c["y"] = rng.choice(["bf16", "bf16", "f32"])
        w = work(c)
        if w["flops"] <= 3.9e12 and w["bytes"] <= 2.3e9:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _rows(gen, shape, dtype, scale=1.0):
    """Normal values in rows that start on 16-byte boundaries: [..., n] inside a buffer [..., n rounded up]."""
    unit = 16 // torch.empty((), dtype=dtype).element_size()
    buf = torch.randn((*shape[:-1], -(-shape[-1] // unit) * unit), device="cuda", generator=gen).mul_(scale).to(dtype)
    return buf[..., :shape[-1]]


def _empty(shape, dtype):
    unit = 16 // torch.empty((), dtype=dtype).element_size()
    return torch.empty((*shape[:-1], -(-shape[-1] // unit) * unit), dtype=dtype, device="cuda")[..., :shape[-1]]


def _tokens(c, gen, dtype):
    """[B,H,N,C] activations: channels of different size and offset, as residual streams have them."""
    B, H, N, C = c["B"], c["H"], c["N"], c["C"]
    if c["layout"] == "heads":
        x = torch.randn((B, N, 3, H, C), device="cuda", generator=gen)[:, :, 0].permute(0, 2, 1, 3)
    else:
        x = _rows(gen, (B, H, N, C), torch.float32)
    spread = torch.exp(0.5 * torch.randn(C, device="cuda", generator=gen))
    offset = 0.5 * torch.randn(C, device="cuda", generator=gen)
    x.mul_(spread).add_(offset)
    if dtype is torch.float32:
        return x
    if c["layout"] == "heads":
        out = torch.empty((B, N, 3, H, C), dtype=dtype, device="cuda")[:, :, 0].permute(0, 2, 1, 3)
    else:
        out = _empty((B, H, N, C), dtype)
    return out.copy_(x)


def _prepare_norm(c, gen):
    B, H, N, C = c["B"], c["H"], c["N"], c["C"]
    p = _DTYPE[c["p"]]
    s = dict(op=c["op"], stats=c["stats"], x=_tokens(c, gen, _DTYPE[c["x"]]), y_dtype=_DTYPE[c["y"]], weight=None, bias=None, shift=None, scale=None)
    if c["affine"]:
        s["weight"] = (1 + 0.2 * torch.randn(C, device="cuda", generator=gen)).to(p)
        s["bias"] = (0.1 * torch.randn(C, device="cuda", generator=gen)).to(p)
    if c["mod"]:      # two of the six rows that a layer's modulation gives each batch entry
        six = 0.3 * torch.randn((B, 6, -(-C // 4) * 4), device="cuda", generator=gen)
        s["shift"], s["scale"] = six[:, 0, :C], six[:, 1, :C]
    if c["op"] == "norm_grad":
        s["dy"] = _rows(gen, (B, H, N, C), s["y_dtype"])
        var, mean = torch.var_mean(s["x"].double(), dim=-1, correction=0)
        s["mean"], s["rstd"] = mean.float(), (var + EPS).rsqrt().float()
    if own:
        from paper_2609_32420_b200 import carnator as cn
        if c["op"] == "norm":
            s["y"] = _empty((B, H, N, C), s["y_dtype"])
            s["shape"] = cn.make_norm_shape(s["x"], s["y"], s["weight"], s["scale"], eps=EPS)
            s["mean"], s["rstd"] = (torch.empty((B, H, N), device="cuda") if c["stats"] else None for _ in range(2))
        else:
            s["dx"] = _empty((B, H, N, C), s["x"].dtype)
            s["shape"] = cn.make_norm_shape(s["x"], s["dy"], s["weight"], s["scale"], dX=s["dx"], eps=EPS)
            s["ws"] = torch.empty(cn.layer_norm_backward_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_linear(c, gen):
    B, N, K, M = c["B"], c["N"], c["K"], c["M"]
    y, p = _DTYPE[c["y"]], _DTYPE[c["p"]]
    s = dict(op=c["op"], act=c["act"], keep=c["keep"], y_dtype=y, bias=None, gate=None, residual=None, z=None, need_x=c["need_x"])
    s["x"] = _rows(gen, (B, N, K), torch.bfloat16)
    s["w"] = _rows(gen, (M, K), torch.bfloat16, 1 / math.sqrt(K))
    bias = (0.1 * torch.randn(M, device="cuda", generator=gen)).to(p)
    if c["gate"]:
        s["gate"] = _rows(gen, (B, 6, M), torch.float32, 0.3)[:, 2]
    if c["op"] == "linear":
        s["bias"] = bias if c["bias"] else None
        s["residual"] = _rows(gen, (B, N, M), y) if c["residual"] else None
    else:
        s["z"] = _empty((B, N, M), torch.bfloat16).copy_(torch.matmul(s["x"], s["w"].t()).add_(bias))
        s["dy"] = _rows(gen, (B, N, M), y)
    if own:
        from paper_2609_32420_b200 import carnator as cn
        act = {"none": cn.ACT_NONE, "gelu_tanh": cn.ACT_GELU_TANH, "gelu": cn.ACT_GELU, "silu": cn.ACT_SILU}[c["act"]]
        if c["op"] == "linear":
            s["y"] = _empty((B, N, M), y)
            s["z"] = _empty((B, N, M), torch.bfloat16) if c["keep"] else None
            s["shape"] = cn.make_linear_shape(s["x"], s["w"], s["y"], residual=s["residual"], Z=s["z"], bias=s["bias"], gate=s["gate"], activation=act)
            s["ws"] = torch.empty(cn.linear_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
        else:
            s["dx"] = _empty((B, N, K), torch.bfloat16) if c["need_x"] else None
            s["dw"] = _empty((M, K), torch.bfloat16)
            s["shape"] = cn.make_linear_shape(s["x"], s["w"], s["dy"], Z=s["z"], gate=s["gate"], dX=s["dx"], dW=s["dw"], activation=act)
            s["ws"] = torch.empty(cn.linear_backward_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    c = _full(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return (_prepare_norm if c["op"].startswith("norm") else _prepare_linear)(c, gen)


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt(d.square().mean(-1, keepdim=True) + EPS)
    y = d * rstd
    if s["weight"] is not None:
        y = y * s["weight"].float() + s["bias"].float()
    if s["scale"] is not None:
        y = y * (1 + s["scale"][:, None, None]) + s["shift"][:, None, None]
    out = dict(y=y.to(s["y_dtype"]))
    if s["stats"]:
        out.update(mean=mean[..., 0], rstd=rstd[..., 0])
    return out


def _plain_norm_grad(s):
    dy, rstd = s["dy"].float(), s["rstd"][..., None]
    xh = (s["x"].float() - s["mean"][..., None]) * rstd
    a = torch.ones((), device="cuda")
    if s["weight"] is not None:
        a = s["weight"].float()
    if s["scale"] is not None:
        a = a * (1 + s["scale"])[:, None, None]
    g = dy * a
    out = dict(dx=(rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))).to(s["x"].dtype))
    P, S = (dy * xh).sum((1, 2)), dy.sum((1, 2))          # per batch entry and channel
    if s["weight"] is not None:
        k = 1 + s["scale"] if s["scale"] is not None else torch.ones((), device="cuda")
        out.update(dweight=(k * P).sum(0), dbias=(k * S).sum(0))
    if s["scale"] is not None:
        out.update(dshift=S, dscale=P if s["weight"] is None else P * s["weight"].float() + S * s["bias"].float())
    return out


_A, _B = math.sqrt(2 / math.pi), 0.044715


def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_A * (z + _B * z * z * z)))
    return z


def _slope(z, act):
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(_A * (z + _B * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _A * (1 + 3 * _B * z * z)
    return torch.ones_like(z)


def _plain_linear(s):
    z = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, s["act"])
    if s["gate"] is not None:
        y = y * s["gate"][:, None]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(y=y.to(s["y_dtype"]))
    if s["keep"]:
        out["z"] = z.to(torch.bfloat16)
    return out


def _plain_linear_grad(s):
    dy, z, out = s["dy"].float(), s["z"].float(), {}
    if s["gate"] is not None:
        out["dgate"] = (dy * _act(z, s["act"])).sum(1)
        dy = dy * s["gate"][:, None]
    dz = dy * _slope(z, s["act"])
    out["dbias"] = dz.sum((0, 1))
    if s["need_x"]:
        out["dx"] = torch.matmul(dz, s["w"].float()).to(torch.bfloat16)
    out["dw"] = torch.matmul(dz.flatten(0, 1).t(), s["x"].float().flatten(0, 1)).to(torch.bfloat16)
    return out


_PLAIN = dict(norm=_plain_norm, norm_grad=_plain_norm_grad, linear=_plain_linear, linear_grad=_plain_linear_grad)


# ---- one pass ----------------------------------------------------------------------------------------------------------
def _own_run(s):
    from paper_2609_32420_b200 import carnator as cn
    op = s["op"]
    if op == "norm":
        y = cn.layer_norm(s["x"], s["shape"], weight=s["weight"], bias=s["bias"], shift=s["shift"], scale=s["scale"], Y=s["y"], mean=s["mean"], rstd=s["rstd"])
        return dict(y=y, mean=s["mean"], rstd=s["rstd"])
    if op == "norm_grad":
        g = cn.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["shape"], weight=s["weight"], bias=s["bias"], scale=s["scale"],
                                   dX=s["dx"], ws=s["ws"], want=("weight", "bias", "shift", "scale"))
        return dict(dx=g.dX, dweight=g.dweight, dbias=g.dbias, dshift=g.dshift, dscale=g.dscale)
    if op == "linear":
        y, _ = cn.linear(s["x"], s["w"], s["shape"], bias=s["bias"], gate=s["gate"], residual=s["residual"], Y=s["y"], Z=s["z"], ws=s["ws"])
        return dict(y=y, z=s["z"])
    g = cn.linear_backward(s["dy"], s["x"], s["w"], s["shape"], Z=s["z"], gate=s["gate"], dX=s["dx"], dW=s["dw"], ws=s["ws"], want=("bias", "gate"))
    return dict(dgate=g.dgate, dbias=g.dbias, dx=g.dX, dw=g.dW)


def run(s):
    return _own_run(s) if own else _PLAIN[s["op"]](s)


# ---- the definitions in 64 bits, gradients by torch's own differentiation -------------------------------------------------
_ACT64 = dict(none=lambda z: z, silu=torch.nn.functional.silu, gelu=torch.nn.functional.gelu,
              gelu_tanh=lambda z: torch.nn.functional.gelu(z, approximate="tanh"))


def _leaf(t):
    return None if t is None else t.double().requires_grad_()


def _exact_norm(s, grads):
    t = {k: _leaf(s[k]) if grads else None if s[k] is None else s[k].double() for k in ("x", "weight", "bias", "shift", "scale")}
    y = torch.nn.functional.layer_norm(t["x"], t["x"].shape[-1:], t["weight"], t["bias"], EPS)
    if t["scale"] is not None:
        y = torch.addcmul(t["shift"][:, None, None], y, 1 + t["scale"][:, None, None])
    if not grads:
        out = dict(y=y)
        if s["stats"]:
            var, mean = torch.var_mean(t["x"], dim=-1, correction=0)
            out.update(mean=mean, rstd=(var + EPS) ** -0.5)
        return out
    y.backward(s["dy"].double())
    return {n: t[k].grad for n, k in dict(dx="x", dweight="weight", dbias="bias", dshift="shift", dscale="scale").items() if t[k] is not None}


def _exact_linear(s):
    z = torch.nn.functional.linear(s["x"].double(), s["w"].double(), None if s["bias"] is None else s["bias"].double())
    y = _ACT64[s["act"]](z)
    if s["gate"] is not None:
        y = torch.einsum("bnm,bm->bnm", y, s["gate"].double())
    out = dict(y=y if s["residual"] is None else s["residual"].double() + y)
    if s["keep"]:
        out["z"] = z
    return out


def _exact_linear_grad(s):
    z, gate = _leaf(s["z"]), _leaf(s["gate"])
    y = _ACT64[s["act"]](z)
    y = y if gate is None else torch.einsum("bnm,bm->bnm", y, gate)
    y.backward(s["dy"].double())
    out = {} if gate is None else dict(dgate=gate.grad)
    out["dbias"] = z.grad.flatten(0, 1).sum(0)
    if s["need_x"]:
        out["dx"] = torch.einsum("bnm,mk->bnk", z.grad, s["w"].double())
    out["dw"] = torch.einsum("bnm,bnk->mk", z.grad, s["x"].double())
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.enable_grad():
        if s["op"].startswith("norm"):
            return _exact_norm(s, s["op"] == "norm_grad")
        return _exact_linear(s) if s["op"] == "linear" else _exact_linear_grad(s)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    """Each input read once, each output written once; the products of the matrix cores count as flops, the few operations per
    element of the norms do not bound anything."""
    c = _full(case)
    size = {"f32": 4.0, "bf16": 2.0}
    B, N = c["B"], c["N"]
    if c["op"].startswith("norm"):
        rows, C = B * c["H"] * N, c["C"]
        vectors = (2 * size[c["p"]] * C if c["affine"] else 0) + (8.0 * B * C if c["mod"] else 0)
        if c["op"] == "norm":
            return {"bytes": rows * C * (size[c["x"]] + size[c["y"]]) + vectors + (8.0 * rows if c["stats"] else 0), "flops": 8.0 * rows * C}
        return {"bytes": rows * C * (2 * size[c["x"]] + size[c["y"]]) + 2 * vectors + 8.0 * rows, "flops": 14.0 * rows * C}
    K, M, rows, y = c["K"], c["M"], B * N, size[c["y"]]
    gate = 4.0 * B * M if c["gate"] else 0
    if c["op"] == "linear":
        return {"bytes": 2.0 * (rows * K + M * K) + y * rows * M * (2 if c["residual"] else 1) + (2.0 * rows * M if c["keep"] else 0)
                + (size[c["p"]] * M if c["bias"] else 0) + gate, "flops": 2.0 * rows * K * M}
    products = 2 if c["need_x"] else 1
    return {"bytes": 2.0 * (rows * K + M * K) * products + (2.0 + y) * rows * M + 4.0 * M + 2 * gate, "flops": 2.0 * products * rows * K * M}
