"""Plain 64-bit forms (CPU) of the operators around the recurrence, and the bounds that the kernels' results are held to.

Unit roundoffs: one rounding to a type of p significant bits is off by at most 2^-p of the value.  fp32 sums of n terms are off by at most
n 2^-24 of the sum of the terms' magnitudes, in whatever order they are formed."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
U32 = 2.0 ** -24
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}   # spacing of the subnormal numbers
# activation and slope kernels: hardware exponential and reciprocal, 7.1.26's 1.5e-7; the exponent's argument, rounded to fp32, moves the
# exponential by at most its own size times 2^-24, and what is left of that after the exponential's decay is below 2^-22
ACT = 4e-6


def d(x):
    return None if x is None else x.detach().cpu().double()


def within(name, got, ref, tol):
    got, ref = d(got), ref.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    bad = ~((got - ref).abs() <= tol)
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        tol = tol.expand_as(ref) if isinstance(tol, torch.Tensor) else torch.full_like(ref, tol)
        raise AssertionError("%s: %d of %d off, first at %s: %r, not %r (bound %.3g)" % (
            name, int(bad.sum()), bad.numel(), at, float(got[at]), float(ref[at]), float(tol[at])))


# ---- layer normalisation
def norm_fwd(x, weight, bias, eps):
    x, w, b = d(x), d(weight), d(bias)
    mean = x.mean(-1)
    rstd = ((x - mean.unsqueeze(-1)) ** 2).mean(-1).add(eps).rsqrt()
    y = (x - mean.unsqueeze(-1)) * rstd.unsqueeze(-1)
    y = y * w if w is not None else y
    return (y + b if b is not None else y), mean, rstd


def norm_bwd(dy, x, mean, rstd, weight):
    dy, x, w, r = d(dy), d(x), d(weight), d(rstd).unsqueeze(-1)
    h = (x - d(mean).unsqueeze(-1)) * r
    g = dy * w if w is not None else dy
    dx = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    width = x.shape[-1]
    return dx, (dy * h).reshape(-1, width).sum(0), dy.reshape(-1, width).sum(0)


# ---- linear layer
def act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.where(z == z, torch.zeros_like(z), z))
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def linear_fwd(x, w, bias, residual, name):
    """(y, bound, z, bound)"""
    dt = x.dtype
    x, w, bias, residual = d(x), d(w), d(bias), d(residual)
    z, mag = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        z, mag = z + bias, mag + bias.abs()
    ez = (x.shape[-1] + 8) * U32 * mag
    y = act(z, name)
    ey = 1.2 * ez + (ACT * (1 + z.abs()) * z.abs().clamp(max=8.0) if name in ("gelu", "silu") else 0)
    if residual is not None:
        y = y + residual
        ey = ey + U32 * y.abs()
    return y, ey + U[dt] * (y.abs() + ey) + TINY[dt], z, ez + U[dt] * (z.abs() + ez) + TINY[dt]


def linear_bwd(dy, x, w, pre, name):
    """dx, bound, dw, bound, d_bias, bound"""
    dt = x.dtype
    dy, x, w = d(dy), d(x), d(w)
    dz, edz = dy, torch.zeros_like(dy)
    if name != "none":
        z = d(pre)
        dz = dy * slope(z, name)
        edz = dy.abs() * (ACT * (1 + z.abs()).clamp(max=8.0) if name != "relu" else 0.0) + U32 * dz.abs()
    eb = (dz.shape[0] + 8) * U32 * (dz.abs() + edz).sum(0) + edz.sum(0)
    if name != "none":
        edz = edz + U[dt] * (dz.abs() + edz) + TINY[dt]
    dx, dw = dz @ w, dz.T @ x
    ex = (dz.shape[1] + 8) * U32 * ((dz.abs() + edz) @ w.abs()) + edz @ w.abs()
    ew = (dz.shape[0] + 8) * U32 * ((dz.abs() + edz).T @ x.abs()) + edz.T @ x.abs()
    return (dx, ex + U[dt] * (dx.abs() + ex) + TINY[dt], dw, ew + U[dt] * (dw.abs() + ew) + TINY[dt], dz.sum(0), eb)


# ---- beam selection, candidate by candidate
def select(logits, scores, finished, eos):
    """(scores, parent, token, finished) as lists, and the smallest distance between neighbours of different beams among the best."""
    x, scores = d(logits), d(scores)
    batch, beams, vocab = x.shape
    out = []
    closest = math.inf
    for b in range(batch):
        cand = []
        for i in range(beams):
            s = float(scores[b, i])
            if not s > -math.inf:
                continue
            if finished is not None and bool(finished[b, i]):
                cand.append((s, i * vocab + eos))
                continue
            row = x[b, i]
            row = torch.where(torch.isnan(row), torch.tensor(-math.inf, dtype=torch.float64), row).clamp(max=torch.finfo(torch.float32).max)
            top = float(row.max())
            if top == -math.inf:
                continue
            lp = s + ((row - top) - torch.log(torch.exp(row - top).sum()))
            keep = torch.argsort(lp, descending=True, stable=True)[:beams + 1].tolist()
            cand += [(float(lp[t]), i * vocab + t) for t in keep if float(lp[t]) > -math.inf]
        cand.sort(key=lambda c: (-c[0], c[1]))
        near = cand[:beams + 1]
        for u, v in zip(near, near[1:]):
            if u[1] // vocab != v[1] // vocab:
                closest = min(closest, u[0] - v[0])
        row = []
        for j in range(beams):
            if j < len(cand):
                s, place = cand[j]
                i, t = divmod(place, vocab)
                row.append((s, i, t, t == eos or (finished is not None and bool(finished[b, i]))))
            else:
                row.append((-math.inf, j, max(eos, 0), True))
        out.append(row)
    return out, closest
