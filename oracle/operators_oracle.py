"""64-bit statements of the operators of gated pre-norm blocks (RMS norm with the residual's addition, rotary positions, gated
feed-forward layer) and of how far a right implementation may be from them.

Every function takes torch tensors of any type on any device, works in float64 and shares no code with the library.  The
`*_bound` values are elementwise: `half` is the result type's half step (relative), E = 2^-24 the half step of fp32.
"""
from __future__ import annotations

import math

import torch

E = 2.0 ** -24


def half(dtype) -> float:
    """The largest rounding error of a type, relative to the value: half a step."""
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ RMS norm
def rmsnorm(x, delta, gamma, eps):
    """(s, y)."""
    s = x.double() if delta is None else x.double() + delta.double()
    return s, s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * gamma.double()


def rmsnorm_bwd(s, dy, gamma, eps, d_sum):
    """(dx, dgamma, bound of dx before its rounding, bound of dgamma)."""
    s, dy, g = s.double(), dy.double(), gamma.double() * dy.double()
    r = 1.0 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    h = s * r
    mean = (g * h).mean(-1, keepdim=True)
    dx = r * (g - h * mean)
    # sums of D terms in trees of at most 16 + 6 + 16 additions; r, h and the products a few more half steps each
    size = r * (g.abs() + h.abs() * (g * h).abs().mean(-1, keepdim=True))
    bound = 64 * E * size
    if d_sum is not None:
        dx = dx + d_sum.double()
        bound = bound + 2 * E * d_sum.double().abs()
    dgamma = (dy * h).sum(0)
    rows = s.shape[0]
    # a work-group adds up to ceil(rows / 768) rows one by one, then at most 768 partial sums follow
    serial = math.ceil(rows / 768) + 64 + min(rows, 768) / 8
    return dx, dgamma, bound, (32 + serial) * E * (dy * h).abs().sum(0)


# ------------------------------------------------------------------ rotary positions
def rotary(x, positions, freq, heads, layout, amplitude, backwards=False):
    """(rotated heads [tokens, heads, dh], bound before their rounding)."""
    rot, axes, period = 2 * freq.numel(), positions.shape[0], positions.shape[1]
    n = rot // 2
    out = x[:, :heads].double().clone()
    bound = torch.zeros_like(out)
    t = torch.arange(x.shape[0], device=x.device) % period
    for j in range(n):
        i, k = (j, j + n) if layout == "half" else (2 * j, 2 * j + 1)
        angle = (positions[0 if j < n / axes else 1].double()[t] * freq[j].double())[:, None]
        c, s = amplitude * torch.cos(angle), (-amplitude if backwards else amplitude) * torch.sin(angle)
        a, b = x[:, :heads, i].double(), x[:, :heads, k].double()
        out[..., i], out[..., k] = a * c - b * s, a * s + b * c
        # the fraction of a turn rounded (2 pi 2^-25), sine and cosine to four half steps, amplitude, products and sum one each
        bound[..., i] = bound[..., k] = 12 * E * abs(amplitude) * (a.abs() + b.abs())
    return out, bound


# ------------------------------------------------------------------ gated feed-forward layer
def act(v, gate):
    return v / (1.0 + torch.exp(-v)) if gate == "silu" else 0.5 * v * (1.0 + torch.erf(v / math.sqrt(2.0)))


def act_slope(v, gate):
    if gate == "silu":
        p = 1.0 / (1.0 + torch.exp(-v))
        return p + v * p * (1.0 - p)
    return 0.5 * (1.0 + torch.erf(v / math.sqrt(2.0))) + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)


# act and act' of the bf16 path: stated to 2e-6 of max(1, |v|); of the fp32 path: a few half steps
FAST = {torch.float32: 1e-6, torch.bfloat16: 4e-6}


def product_bound(size, K):
    """Rounding of K products added in fp32: matrix instructions add at least 2 of them at a time."""
    return (K / 2 + 16) * E * size


def gated_mlp(x, w, gate, act_dtype, x_scale=None):
    """dict of gu, h, y and their bounds (gu_bound, ...), which count every rounding to act_dtype on the way."""
    u = half(act_dtype)
    x8, w_in = x.double(), w["w_in"].double()
    if x_scale is not None:
        x8, w_in = x8 * x_scale.double()[:, None], w_in * w["in_scale"].double()[:, None]
    R, D = w_in.shape[0] // 2, x.shape[1]
    gu, gu_err = x8 @ w_in.t(), product_bound(x8.abs() @ w_in.abs().t(), D)
    if x_scale is not None:
        gu_err = gu_err + 4 * E * gu.abs()
    if w.get("b_in") is not None:
        gu = gu + w["b_in"].double()
        gu_err = gu_err + 2 * E * gu.abs()
    g, up = gu[:, :R], gu[:, R:]
    h = act(g, gate) * up
    # |act'| <= 1.13; act itself to FAST
    h_err = 1.13 * gu_err[:, :R] * up.abs() + act(g, gate).abs() * gu_err[:, R:] + FAST[act_dtype] * g.abs().clamp(min=1.0) * up.abs()
    h_held = h_err * (1 + u) + u * h.abs()
    wo = w["w_out"].double()
    y = h @ wo.t()
    y_err = h_held @ wo.abs().t() + product_bound(h.abs() @ wo.abs().t(), R)
    if w.get("b_out") is not None:
        y = y + w["b_out"].double()
        y_err = y_err + 2 * E * y.abs()
    return {"gu": gu, "gu_bound": gu_err * (1 + u) + u * gu.abs(), "h": h, "h_bound": h_held, "y": y, "y_bound": y_err * (1 + u) + u * y.abs()}


def gated_mlp_bwd(x, gu, h, dy, w, gate, act_dtype, grad_dtype):
    """dict of dx, w_in, w_out, b_in, b_out and their bounds; gu and h as the forward kept them."""
    u, v = half(act_dtype), half(grad_dtype)
    x8, dy8, h8, wi, wo = x.double(), dy.double(), h.double(), w["w_in"].double(), w["w_out"].double()
    M, R, D = x.shape[0], h.shape[1], x.shape[1]
    g, up = gu[:, :R].double(), gu[:, R:].double()
    dh, dh_err = dy8 @ wo, product_bound(dy8.abs() @ wo.abs(), D)
    d_gu = torch.cat([dh * up * act_slope(g, gate), dh * act(g, gate)], 1)
    fast = FAST[act_dtype] * g.abs().clamp(min=1.0)
    err = torch.cat([1.13 * dh_err * up.abs() + fast * (dh * up).abs(), dh_err * act(g, gate).abs() + fast * dh.abs()], 1) + 4 * E * d_gu.abs()
    held = err * (1 + u) + u * d_gu.abs()                     # [dg | du] as the products read it
    out = {"dx": d_gu @ wi, "w_in": d_gu.t() @ x8, "w_out": dy8.t() @ h8, "b_in": d_gu.sum(0), "b_out": dy8.sum(0)}
    size = d_gu.abs()
    errs = {"dx": held @ wi.abs() + product_bound(size @ wi.abs(), 2 * R), "w_in": held.t() @ x8.abs() + product_bound(size.t() @ x8.abs(), M),
            "w_out": product_bound(dy8.abs().t() @ h8.abs(), M), "b_in": held.sum(0) + product_bound(size.sum(0), M), "b_out": product_bound(dy8.abs().sum(0), M)}
    for n, e in errs.items():
        r = u if n == "dx" else v
        out[n + "_bound"] = e * (1 + r) + r * out[n].abs()
    return out


# ------------------------------------------------------------------ comparison
def worst(got, want, bound):
    """The largest |got - want| / bound; a NaN or infinity has to be where the oracle has the same one."""
    got = got.double()
    fine = torch.isfinite(want)
    if not torch.equal(fine, torch.isfinite(got)) or not torch.equal(torch.isnan(want), torch.isnan(got)) or not torch.equal(want[~fine & ~torch.isnan(want)], got[~fine & ~torch.isnan(got)]):
        return math.inf
    d, b = (got - want).abs()[fine], bound.expand_as(want)[fine]
    if not d.numel():
        return 0.0
    return float((d / b.clamp(min=1e-300)).max())


def rel2(got, want):
    n = torch.linalg.vector_norm(want)
    return float(torch.linalg.vector_norm(got.double() - want) / n) if n > 0 else float(torch.linalg.vector_norm(got.double()))
