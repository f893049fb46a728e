"""The dense operators in 64 bits, with an elementwise bound on what the library may be off.

Every bound counts roundings.  u is half a step of the stored type (bf16 2^-8, fp32 2^-24) for each
rounding to it, and sums of n terms held in 32 bits are off by at most (n + 8) 2^-23 of the sum of
their terms' sizes, whatever their order (2^-23: products and sums may be rounded toward zero).
Activations are evaluated to within ACT of their size: a fast exponential of w is off by about
(|w| + 2) 2^-23, below 2^-17 for |w| < 32, and where |w| is more the sigmoid or its complement
is below 2^-46.
"""
from __future__ import annotations

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
ACT = {torch.bfloat16: 2.0 ** -17, torch.float32: 2.0 ** -19}
LIP = 1.13   # the largest |act'| of silu (1.0998) and gelu (1.1289)
CURVE = 1.2  # and above the largest |act''| (silu 0.5, gelu below 1.13)


def act(z, name):
    """act(z), act'(z)."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    c, k = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(c * (z + k * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * k * z * z)


def summed(n):
    return (n + 8) * 2.0 ** -23


def product(a, b):
    """(a b^T, the sum of the terms' sizes) in 64 bits."""
    return a @ b.t(), a.abs() @ b.abs().t()


def linear(x, w, bias=None, residual=None, name="none", alpha=1.0):
    """y and its bound, z and its bound."""
    u, dt = U[x.dtype], x.dtype
    z, size = product(x.double(), w.double())
    if bias is not None:
        z = z + bias.double()
        size = size + bias.double().abs()
    ez = summed(x.shape[1]) * size
    a, _ = act(z, name)
    ea = LIP * ez + (ACT[dt] * z.abs() if name != "none" else 0)
    y = alpha * a + (residual.double() if residual is not None else 0)
    ey = abs(alpha) * ea + 2.0 ** -22 * (abs(alpha) * a.abs() + y.abs())
    return y, ey + u * (y.abs() + ey), z, ez


def linear_grads(x, w, dy, z=None, ez=None, name="none", alpha=1.0):
    """{"dx": (value, bound), "dw": ..., "db": ...}; ez: how far the kept z may be off."""
    u, dt = U[x.dtype], x.dtype
    dz, e = alpha * dy.double(), torch.zeros_like(dy, dtype=torch.float64)
    if name != "none":
        _, da = act(z, name)
        dz = dz * da
        e = (CURVE * ez + 4 * ACT[dt] * (1 + z.abs().clamp(max=32))) * (alpha * dy.double()).abs()
    out = {"db": (dz.sum(0), e.sum(0) + summed(dy.shape[0]) * dz.abs().sum(0))}
    if name != "none":
        e = e + u * (dz.abs() + e)  # dz enters the products in the stored type
    out.update(_from_dz([(dz, e)], x, [w]))
    return {k: (v, b + 2.0 ** -22 * v.abs() + u * (v.abs() + b)) for k, (v, b) in out.items()}


def _from_dz(parts, x, ws):
    dx = ex = size = 0
    out = {}
    for i, ((dz, e), w) in enumerate(zip(parts, ws)):
        v, s = product(dz, w.double().t())
        dx, size = dx + v, size + s
        ex = ex + e @ w.double().abs()
        v, s = product(dz.t(), x.double().t())
        out["dw" if len(ws) == 1 else ("dw_gate", "dw_up")[i]] = (v, e.t() @ x.double().abs() + summed(x.shape[0]) * s)
    out["dx"] = (dx, ex + summed(len(ws) * ws[0].shape[0]) * size)
    return out


def gated(x, wg, wu, name="silu"):
    """h and its bound, and (g, eg, u, eu)."""
    u_, dt = U[x.dtype], x.dtype
    (g, sg), (u, su) = product(x.double(), wg.double()), product(x.double(), wu.double())
    eg, eu = summed(x.shape[1]) * sg, summed(x.shape[1]) * su
    a, _ = act(g, name)
    ea = LIP * eg + ACT[dt] * g.abs()
    h = a * u
    e = ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -22 * h.abs()
    return h, e + u_ * (h.abs() + e), (g, eg, u, eu)


def gated_grads(x, wg, wu, dh, kept, name="silu"):
    u_, dt = U[x.dtype], x.dtype
    g, eg, u, eu = kept
    a, da = act(g, name)
    d = dh.double()
    dg, du = d * u * da, d * a
    ea = LIP * eg + ACT[dt] * g.abs()
    eda = CURVE * eg + 4 * ACT[dt] * (1 + g.abs().clamp(max=32))
    edg = d.abs() * (eu * (da.abs() + eda) + u.abs() * eda) + 2.0 ** -22 * dg.abs()
    edu = d.abs() * ea + 2.0 ** -22 * du.abs()
    edg, edu = edg + u_ * (dg.abs() + edg), edu + u_ * (du.abs() + edu)
    out = _from_dz([(dg, edg), (du, edu)], x, [wg, wu])
    return {k: (v, b + u_ * (v.abs() + b)) for k, (v, b) in out.items()}


def turn(v, positions, inv_freq, sign=1):
    """v [T, heads, dh] rotated; positions [T], inv_freq [R/2] (None: as it is)."""
    if positions is None:
        return v
    a = sign * positions.double()[:, None, None] * inv_freq.double()
    half = inv_freq.numel()
    x, y = v[..., :half], v[..., half:2 * half]
    return torch.cat((x * a.cos() - y * a.sin(), y * a.cos() + x * a.sin(), v[..., 2 * half:]), -1)


def _pair_sizes(v, inv_freq):
    """What a rotation may be made of: for each column the sizes of its pair."""
    if inv_freq is None:
        return v.abs()
    half = inv_freq.numel()
    x, y = v[..., :half].abs(), v[..., half:2 * half].abs()
    return torch.cat((x + y, x + y, v[..., 2 * half:].abs()), -1)


# Relative error of a normed value before its rounding: the sum of squares (its terms are of one
# sign, so (dh + 8) 2^-23 of it, halved by the root), the root, the quotient and two products; of
# a rotated one: the sine and cosine of an angle rounded to 2^-24 of a turn, products, a sum.
def _norm_err(dh):
    return (dh / 2 + 12) * 2.0 ** -23


TURN_ERR = (2 * math.pi + 8) * 2.0 ** -23


def qk(v, gamma, eps, positions, inv_freq):
    u_, dh = U[v.dtype], v.shape[-1]
    d = v.double()
    n = d if gamma is None else gamma.double() * d / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    out = turn(n, positions, inv_freq)
    e = (TURN_ERR + (0 if gamma is None else _norm_err(dh))) * _pair_sizes(n, inv_freq)
    return out, e + u_ * (out.abs() + e)


def qk_grads(v, gamma, eps, positions, inv_freq, dout):
    """{"d": (value, bound)} and, with a norm, {"dgamma": ...}."""
    u_, dh = U[v.dtype], v.shape[-1]
    d = v.double()
    dn = turn(dout.double(), positions, inv_freq, -1)
    en = TURN_ERR * _pair_sizes(dout.double(), inv_freq)
    if gamma is None:
        return {"d": (dn, en + u_ * (dn.abs() + en))}
    inv = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    hat, rel = d * inv, _norm_err(dh)
    terms = dn * hat
    dgamma = terms.sum((0, 1))
    eg = ((en + 2.0 ** -22 * dn.abs()) * hat.abs() + (rel + summed(v.shape[0] * v.shape[1])) * terms.abs()).sum((0, 1))
    dhat = dn * gamma.double()
    ehat = en * gamma.double().abs() + 2.0 ** -23 * dhat.abs()
    mean, size = (dhat * hat).mean(-1, keepdim=True), (dhat * hat).abs().mean(-1, keepdim=True)
    emean = (ehat * hat.abs()).mean(-1, keepdim=True) + (rel + summed(dh)) * size
    dv = inv * (dhat - hat * mean)
    e = inv * (ehat + hat.abs() * emean + (2 * rel + 4 * 2.0 ** -23) * (dhat.abs() + (hat * mean).abs()))
    return {"d": (dv, e + u_ * (dv.abs() + e)), "dgamma": (dgamma, eg + u_ * (dgamma.abs() + eg))}


def check(got, value, bound, what):
    """Every element within its bound; non-finite ones alike."""
    got = got.double()
    fine = torch.isfinite(value) & torch.isfinite(bound)
    assert torch.equal(torch.isnan(got), torch.isnan(value)), f"{what}: NaN in other places"
    off = (got - value).abs()
    bad = fine & ~(off <= bound + 1e-37)
    if bad.any():
        i = (off / (bound + 1e-37)).masked_fill(~fine, 0).argmax().item()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside their bounds; worst at {i}: got "
                             f"{got.flatten()[i].item()}, expected {value.flatten()[i].item()} +- {bound.flatten()[i].item()}")
