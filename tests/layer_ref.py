"""Dense linear layer and layer norm in 64 bits, from their formulas, and bounds on what a
kernel that sums in fp32 and rounds once may be off: test infrastructure only."""
import math

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu", "tanh")
U = 2.0 ** -24  # half a step of fp32, relative


def half(dt):
    """Half a step of a type, relative to the value."""
    return torch.finfo(DT[dt]).eps / 2


def floor_of(dt):
    """Half the spacing of the type's smallest values (what rounding to a subnormal may cost)."""
    return {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}[dt]


def act_err(dt):
    """An activation or slope evaluated in fp32, relative to |z| (1 + |z| for a slope): library
    functions to a few steps in fp32; approximations far below the output's half step (2^-11,
    2^-8) in the 16-bit types."""
    return 2.0 ** -21 if dt == "f32" else 2.0 ** -18


def act(z, a):
    if a == "relu":
        return torch.clamp(z, min=0.0)
    if a == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    if a == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if a == "silu":
        return z * torch.sigmoid(z)
    if a == "tanh":
        return torch.tanh(z)
    return z


def slope(z, a):
    if a == "relu":
        return (z > 0).double()
    if a == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if a == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    if a == "silu":
        p = torch.sigmoid(z)
        return p * (1.0 + z * (1.0 - p))
    if a == "tanh":
        return 1.0 - torch.tanh(z) ** 2
    return torch.ones_like(z)


def f64(t):
    return None if t is None else t.detach().cpu().double()


def dense_fwd(X, W, bias, res, a, dt):
    """{name: (value, bound)} of Y and Z."""
    X, W, bias, res = map(f64, (X, W, bias, res))
    z = X @ W.t()
    size = X.abs() @ W.abs().t()
    if bias is not None:
        z = z + bias
        size = size + bias.abs()
    # a sum of n terms in fp32, whatever its order: n steps of the sum of their sizes at most
    ez = 2 * (X.shape[1] + 2) * U * size
    y = act(z, a)
    ey = 1.13 * ez + act_err(dt) * z.abs()  # 1.13: the largest slope of the activations
    if res is not None:
        y = y + res
        ey = ey + 2 * U * y.abs()
    return {"Y": (y, half(dt) * (y.abs() + ey) + ey + floor_of(dt)),
            "Z": (z, half(dt) * (z.abs() + ez) + ez + floor_of(dt))}


def dense_bwd(dY, Z, X, W, a, dt):
    """{name: (value, bound)} of dX, dW and dbias (X or W may be None)."""
    dY, Z, X, W = map(f64, (dY, Z, X, W))
    N, C = dY.shape
    if a == "none":
        g, eg, er = dY, torch.zeros_like(dY), torch.zeros_like(dY)
    else:
        g = dY * slope(Z, a)
        eg = (act_err(dt) * (1 + Z.abs()) + 2 * U) * dY.abs()
        er = eg + half(dt) * (g.abs() + eg) + floor_of(dt)  # rounded for the products
    out = {}
    if W is not None:
        v, s = g @ W, g.abs() @ W.abs()
        e = er @ W.abs() + 2 * (C + 2) * U * (s + er @ W.abs())
        out["dX"] = (v, half(dt) * (v.abs() + e) + e + floor_of(dt))
    if X is not None:
        v, s = g.t() @ X, g.t().abs() @ X.abs()
        e = er.t() @ X.abs() + 2 * (N + 2) * U * (s + er.t() @ X.abs())
        out["dW"] = (v, half(dt) * (v.abs() + e) + e + floor_of(dt))
    v = g.sum(0)
    e = eg.sum(0) + 2 * (N + 2) * U * (g.abs() + eg).sum(0)
    out["dbias"] = (v, half(dt) * (v.abs() + e) + e + floor_of(dt))
    return out


# fp32 row sums are trees: a lane's own elements in turn (32 at most, or 1/1024 of a long row),
# six exchanges, a few waves
def depth(D):
    return 48 + D // 1024


def norm_fwd(X, gamma, beta, eps, dt):
    X, gamma, beta = map(f64, (X, gamma, beta))
    D = X.shape[1]
    mean = X.mean(1, keepdim=True)
    d = X - mean
    var = (d * d).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    em = depth(D) * U * X.abs().mean(1, keepdim=True) + U * mean.abs()
    ed = em + U * (d.abs() + em)
    # the variance: the error of each difference, then the sum's; rstd half of that, relative
    ev = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + (depth(D) + 4) * U * (d.abs() + ed).square().mean(1, keepdim=True)
    er = rstd * (0.5 * ev * rstd * rstd + 4 * U)
    h = d * rstd
    y, eh = h, ed * (rstd + er) + d.abs() * er + 2 * U * h.abs()
    if gamma is not None:
        y, eh = h * gamma, eh * gamma.abs() + U * (h * gamma).abs()
    if beta is not None:
        y = y + beta
        eh = eh + U * y.abs()
    return {"Y": (y, half(dt) * (y.abs() + eh) + eh + floor_of(dt)), "mean": (mean[:, 0], em[:, 0] + 1e-45),
            "rstd": (rstd[:, 0], er[:, 0])}


def norm_bwd(dY, X, gamma, mean, rstd, past, dt):
    dY, X, gamma, mean, rstd, past = map(f64, (dY, X, gamma, mean, rstd, past))
    N, D = X.shape
    m, r = mean[:, None], rstd[:, None]
    h = (X - m) * r
    eh = 3 * U * h.abs()
    g = dY * gamma if gamma is not None else dY
    avg = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    c1, c2 = avg(g), avg(g * h)
    e1 = (depth(D) + 2) * U * avg(g.abs())
    e2 = (depth(D) + 6) * U * avg((g * h).abs())
    v = r * (g - c1 - h * c2)
    e = r * (e1 + e2 * h.abs() + eh * c2.abs() + 6 * U * (g.abs() + c1.abs() + (h * c2).abs()))
    if past is not None:
        v = v + past
        e = e + U * v.abs()
    out = {"dX": (v, half(dt) * (v.abs() + e) + e + floor_of(dt))}
    for name, t in (("dgamma", dY * h), ("dbeta", dY)):
        s, e = t.sum(0), (N + 6) * U * t.abs().sum(0)
        out[name] = (s, half(dt) * (s.abs() + e) + e + floor_of(dt))
    return out


def check(name, got, want):
    v, tol = want
    g = f64(got)
    assert g.shape == v.shape, (name, g.shape, v.shape)
    bad = ~((g - v).abs() <= tol)
    if bad.any():
        i = tuple(int(k[0]) for k in torch.nonzero(bad, as_tuple=True))
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds, first at {i}: got {g[i].item()!r}, "
                             f"want {v[i].item()!r} +- {tol[i].item()!r}")
