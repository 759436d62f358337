"""64-bit plain forms of layer norm, matrix product and their gradients, with the error that 32-bit sums and one rounding allow.

U32 = 2^-24 is half a step of fp32, U16 = 2^-8 half a step of bf16 (relative).
"""
import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half_step(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def padded(shape, dtype, gen, scale=1.0, extra=0):
    """Normal values in rows on 16-byte boundaries, NaN behind the last column (and in ``extra`` more rows of the second to last axis)."""
    unit = 16 // torch.empty((), dtype=dtype).element_size()
    wide = -(-shape[-1] // unit) * unit + unit
    buf = torch.full((*shape[:-2], shape[-2] + extra, wide), float("nan"), dtype=dtype, device="cuda")
    view = buf[..., :shape[-2], :shape[-1]]
    view.copy_(torch.randn(shape, device="cuda", generator=gen) * scale)
    return view


def canvas(shape, dtype, extra=0):
    """(buffer of a sentinel, view of `shape` inside it): what a call writes outside its rows shows."""
    unit = 16 // torch.empty((), dtype=dtype).element_size()
    buf = torch.full((*shape[:-2], shape[-2] + extra, -(-shape[-1] // unit) * unit + unit), 77.0, dtype=dtype, device="cuda")
    return buf, buf[..., :shape[-2], :shape[-1]]


def untouched(buf, view):
    """Whether everything of the buffer outside the view still holds the sentinel."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask[..., :view.shape[-2], :view.shape[-1]] = False
    return bool((buf[mask] == 77.0).all())


def check(got, ref, tol, what):
    assert got.shape == ref.shape, what
    g = got.double()
    assert torch.isfinite(g).all(), f"{what}: not finite"
    over = (g - ref).abs() - tol
    worst = over.argmax()
    assert over.max() <= 0, f"{what}: {g.flatten()[worst]} for {ref.flatten()[worst]}, allowed {tol.expand_as(ref).flatten()[worst]}"


# ---- layer norm ----------------------------------------------------------------------------------------
def norm_ref(x, weight, bias, shift, scale, eps):
    """(y, mean, rstd, xh, a, ranges) in 64 bits; a [B,1,1,C] or scalar: the factor of xh."""
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    var = ((x - mean) ** 2).mean(-1, keepdim=True)
    rstd = (var + eps) ** -0.5
    xh = (x - mean) * rstd
    a = torch.ones((x.shape[0], 1, 1, x.shape[-1]), dtype=torch.float64, device=x.device)
    c = torch.zeros_like(a)
    if weight is not None:
        a = a * weight.double()
    if bias is not None:
        c = c + bias.double()
    if scale is not None:
        k = 1 + scale.double()[:, None, None]
        a, c = a * k, c * k
    if shift is not None:
        c = c + shift.double()[:, None, None]
    return xh * a + c, mean[..., 0], rstd[..., 0], xh, a, c


def xh_error(x, mean, rstd, xh):
    """Of the normalised value: the mean is a 32-bit sum of C values (at most 40 additions deep: 8 V in a lane, 5 + 5 across lanes; V <= 4),
    so it is off by at most 42 U32 max|x|; the difference from it is rounded once; the variance is a sum of the same depth of squares of
    such differences, so rstd is off by at most half of (2 x 42 + 44) U32 of itself plus a shift by the mean's error (second order, and
    counted with the first), plus the four steps of rsqrt and products."""
    big = x.double().abs().amax(-1, keepdim=True)
    off_mean = 44 * U32 * big
    r = rstd[..., None]
    # the mean's error moves every squared difference by 2 |d| e: relative to the variance at most 2 e rstd
    return off_mean * r * (1 + xh.abs() * 1.0) + xh.abs() * (70 * U32)


# ---- activations -----------------------------------------------------------------------------------------
A, Bc = math.sqrt(2 / math.pi), 0.044715


def act64(z, act):
    if act == 3:
        return z / (1 + torch.exp(-z))
    if act == 2:
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if act == 1:
        return 0.5 * z * (1 + torch.tanh(A * (z + Bc * z ** 3)))
    return z


def slope64(z, act):
    if act == 3:
        s = 1 / (1 + torch.exp(-z))
        return s + z * s * (1 - s)
    if act == 2:
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == 1:
        t = torch.tanh(A * (z + Bc * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * A * (1 + 3 * Bc * z * z)
    return torch.ones_like(z)


# Value and slope are computed from z in 32 bits with an exponential and a division good to 2^-21 of a sigmoid between 0 and 1 (its argument, up to
# |2 A z (1 + B z^2)| < 90 before the sigmoid vanishes, is rounded to U32 of itself: 90 U32 = 2^-17.5 of s (1 - s) |u| < 0.3): 2^-19 of |z| + 1.
ACT_ERR = 2.0 ** -19
SLOPE_MOST = 1.13               # largest slope of the three


def sum_error(terms, magnitude):
    """Of a tensor-core sum of `terms` products in fp32 whose absolute values sum to `magnitude`: at most one step (2^-23, the sums are cut off, not
    rounded) per addition, two additions per 16 terms counted, and 16 for joining partial sums."""
    return (terms / 8 + 16) * 2.0 ** -23 * magnitude


def linear_ref(x, w, bias, gate, residual, act):
    """(y, z, allowed error of z before rounding, of y before rounding) in 64 bits."""
    xd, wd = x.double(), w.double()
    z = xd @ wd.T
    mag = xd.abs() @ wd.abs().T
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    ez = sum_error(x.shape[-1], mag)
    y = act64(z, act)
    ey = (SLOPE_MOST if act else 1.0) * ez + (ACT_ERR * (z.abs() + 1) if act else 0)
    if gate is not None:
        g = gate.double()[:, None]
        y, ey = y * g, ey * g.abs() + U32 * (y * g).abs()
    if residual is not None:
        y = y + residual.double()
        ey = ey + U32 * y.abs()
    return y, z, ez, ey


def linear_grad_ref(dy, x, w, z, gate, act):
    """dict name -> (gradient, allowed error before its own rounding) in 64 bits."""
    d, zz = dy.double(), None if z is None else z.double()
    out = {}
    B, N, M = dy.shape
    if gate is not None:
        u = act64(zz, act)
        t = d * u
        out["dgate"] = (t.sum(1), d.abs().mul(ACT_ERR * (zz.abs() + 1) if act else 0).sum(1) + depth(N) * U32 * t.abs().sum(1))
        d = d * gate.double()[:, None]
    s = slope64(zz, act) if act else torch.ones_like(d)
    dz = d * s
    e = d.abs() * (ACT_ERR * (zz.abs() + 1)) + 3 * U32 * dz.abs() if act else 2 * U32 * dz.abs()
    flat = lambda t: t.flatten(0, 1)  # noqa: E731
    out["dbias"] = (flat(dz).sum(0), flat(e).sum(0) + depth(B * N) * U32 * flat(dz).abs().sum(0))
    rounded = dz.abs() * U16 + e              # dz is rounded to bf16 as an operand (where it is dy itself, it is not: less)
    if w is not None:
        wa = w.double().abs()
        out["dX"] = (dz @ w.double(), rounded @ wa + sum_error(M, dz.abs() @ wa))
    if x is not None:
        xa = flat(x.double()).abs()
        out["dW"] = (flat(dz).T @ flat(x.double()), flat(rounded).T @ xa + sum_error(B * N, flat(dz).abs().T @ xa))
    return out


def depth(n):
    """Additions that a term of a sum over n rows passes at most: one by one within a thread and over the partial rows."""
    return n + 64
