"""Float64 definitions of the dense operators, with error bounds for kernels that accumulate in
float32 and round each result once.

HALF[t] is half a step of type t relative to the value; F = 2^-24 is float32's. A float32 sum of n
products x y is off by at most (n + 1) F sum |x y| whatever its order; products of bfloat16 values
are exact in float32 (the bound keeps the 1). Every function returns (values, bounds).
"""
import math

import torch

F = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: F}
F64 = torch.float64


def check(name, got, ref, bound):
    """|got - ref| <= bound everywhere; values that are not finite must be equal."""
    got = got.detach().to("cpu", F64)
    ref, bound = ref.cpu(), bound.cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fin = torch.isfinite(ref)
    assert torch.equal(got[~fin], ref[~fin]), name
    err = (got - ref).abs()[fin]
    if err.numel():
        over = (err - bound[fin]).max().item()
        assert torch.isfinite(got[fin]).all() and over <= 0, \
            f"{name}: off by {err.max().item():.3e}, {over:.3e} more than its bound"


# ---- layer norm ----

def layernorm(x, gain, bias, eps, dy=None):
    """A lane adds up to 64 values and 10 steps join the lanes: 80 F covers a sum, relative to the sum
    of magnitudes; the statistics enter every value, hence the factors below."""
    h = HALF[x.dtype]
    x, gain = x.to(F64), gain.to(F64)
    bias = torch.zeros_like(gain) if bias is None else bias.to(F64)
    n = x.shape[1]
    mean = x.mean(1, keepdim=True)
    c = x - mean
    var = (c ** 2).mean(1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    u = c * rstd
    e_mean = 80 * F * x.abs().mean(1, keepdim=True) + F * mean.abs()
    # a shift of every deviation by e_mean moves the variance by e_mean^2 at most (their sum is 0)
    r_rstd = 0.5 * (100 * F + (e_mean ** 2 + 4 * F * e_mean * c.abs().amax(1, keepdim=True)) / (var + eps)) + 4 * F
    e_u = u.abs() * (r_rstd + 4 * F) + rstd * (e_mean + F * x.abs())
    y = u * gain + bias
    out = {"y": (y, h * y.abs() + e_u * gain.abs() + 4 * F * (u * gain).abs() + 2 * F * y.abs()),
           "mean": (mean[:, 0], e_mean[:, 0]), "rstd": (rstd[:, 0], (r_rstd * rstd)[:, 0])}
    if dy is None:
        return out
    dy = dy.to(F64)
    g = dy * gain
    m0, m1 = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
    dx = rstd * (g - m0 - u * m1)
    e_g = F * g.abs()
    e_m0 = 90 * F * g.abs().mean(1, keepdim=True)
    e_m1 = 90 * F * (g * u).abs().mean(1, keepdim=True) + (g.abs() * e_u).mean(1, keepdim=True)
    e = e_g + e_m0 + e_u * m1.abs() + u.abs() * e_m1 + 6 * F * (g.abs() + m0.abs() + (u * m1).abs())
    rows = x.shape[0] + 20
    out["dx"] = dx, h * dx.abs() + rstd * e + (r_rstd + 4 * F) * dx.abs()
    out["dgain"] = (dy * u).sum(0), (dy.abs() * e_u).sum(0) + rows * F * (dy * u).abs().sum(0)
    out["dbias"] = dy.sum(0), rows * F * dy.abs().sum(0)
    return out


# ---- affine map ----

def act(z, kind):
    if kind == "relu":
        return z.clamp(min=0), (z > 0).to(F64)
    if kind == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def linear(x, w, bias, res, kind, dy=None):
    """Slopes of the activations are at most 1.13 and change by at most 1.1 per unit of z (gelu'' <= 0.8,
    silu'' <= 0.5); an activation itself is evaluated to 16 F of its value and of z."""
    h = HALF[x.dtype]
    x, w = x.to(F64), w.to(F64)
    k = x.shape[1]
    z = x @ w.t()
    e_z = (k + 2) * F * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.to(F64)
        e_z = e_z + F * z.abs()
    a, slope = act(z, kind)
    y = a if res is None else a + res.to(F64)
    out = {"y": (y, h * y.abs() + 1.13 * e_z + (16 * F * (a.abs() + z.abs()) if kind in ("gelu", "silu") else 0)
                 + 2 * F * (a.abs() + y.abs()))}
    if dy is None:
        return out
    dy = dy.to(F64)
    dz = dy * slope
    e_dz = torch.zeros_like(dz)
    if kind != "none":
        off = h * z.abs() + e_z          # z as it was saved
        if kind == "relu":               # its sign can only differ where the sum's can
            e_slope = (z.abs() <= e_z).to(F64)
        else:
            e_slope = 1.1 * off + 16 * F * (1 + z.abs())
        e_dz = dy.abs() * e_slope + F * dz.abs()
    m, n = dz.shape
    e_in = e_dz + (h * (dz.abs() + e_dz) if kind != "none" else 0)    # as it enters the products
    dx, dw, db = dz @ w, dz.t() @ x, dz.sum(0)
    out["dx"] = dx, h * dx.abs() + e_in @ w.abs() + (n + 2) * F * (dz.abs() @ w.abs())
    out["dw"] = dw, h * dw.abs() + e_in.t() @ x.abs() + (m + 70) * F * (dz.abs().t() @ x.abs())
    out["db"] = db, h * db.abs() + e_dz.sum(0) + (m + 70) * F * dz.abs().sum(0)
    return out


# ---- packed attention ----

def attention(q, k, v, cu_q, cu_k, used_k=None, causal=False, scale=None, d_o=None):
    """Per head of each sequence. A score is off by (d + 2) F scale sum |q k|; its exponential by that
    and by the float32 rounding of exponent (its own size and the reference's, 2^8 at most above it)
    and result. Probabilities and dS enter their products in the tensors' type."""
    h_ = HALF[q.dtype]
    hp = h_ if q.dtype == torch.bfloat16 else 0.0
    q, k, v = (t.detach().cpu().to(F64) for t in (q, k, v))
    d = q.shape[2]
    scale = scale or 1 / math.sqrt(d)
    heads, kv = q.shape[1], k.shape[1]
    grp = heads // kv
    cq, ck = cu_q.tolist(), cu_k.tolist()
    zeros = torch.zeros_like
    o, eo, dq, edq = zeros(q), zeros(q), zeros(q), zeros(q)
    dk, edk, dv, edv = zeros(k), zeros(k), zeros(v), zeros(v)
    lse = torch.full((heads, q.shape[0]), -math.inf, dtype=F64)
    elz = torch.zeros_like(lse)
    if d_o is not None:
        d_o = d_o.detach().cpu().to(F64)
    for s in range(len(cq) - 1):
        n = ck[s + 1] - ck[s] if used_k is None else int(used_k[s])
        rows, cols = slice(cq[s], cq[s + 1]), slice(ck[s], ck[s] + n)
        m = cq[s + 1] - cq[s]
        if m == 0 or n == 0:
            continue
        see = torch.ones(m, n, dtype=torch.bool)
        if causal:
            see = torch.arange(n)[None] <= torch.arange(m)[:, None] + n - m
        some = see.any(1)
        for hd in range(heads):
            a, b, c = q[rows, hd], k[cols, hd // grp], v[cols, hd // grp]
            x = scale * (a @ b.t())
            e_x = (d + 2) * F * scale * (a.abs() @ b.abs().t())
            x = torch.where(see, x, -math.inf)
            z = torch.logsumexp(x, 1)
            z0 = torch.where(some, z, 0.0)
            p = torch.where(some[:, None], torch.exp(x - z0[:, None]), 0.0)
            xs = torch.where(see, x, 0.0)
            big = xs.abs().amax(1)
            # relative error of exp(x - reference): scores, exponent rounding, the exponential
            rp = torch.where(see, e_x + 4 * F * (xs.abs() + big[:, None] + 12) + 8 * F, 0.0)
            rl = (p * rp).sum(1) + (n + 80) * F          # of the sum
            ov = p @ c
            o[rows, hd] = ov
            eo[rows, hd] = ((p * (rp + hp)) @ c.abs()) + (rl + (n + 80) * F)[:, None] * (p @ c.abs()) \
                + (h_ + 2 * F) * ov.abs()
            lse[hd, rows] = z
            elz[hd, rows] = torch.where(some, rl + 4 * F * (z0.abs() + 2), 0.0)
            if d_o is None:
                continue
            g = d_o[rows, hd]
            dp = g @ c.t()
            delta = (g * ov).sum(1, keepdim=True)
            # o enters delta rounded and with its own error
            e_delta = (g.abs() * eo[rows, hd]).sum(1, keepdim=True) + (d + 2) * F * (g * ov).abs().sum(1, keepdim=True)
            e_dp = (d + 2) * F * (g.abs() @ c.abs().t())
            rq = rp + elz[hd, rows][:, None] + 4 * F * (z0.abs()[:, None] + 2)
            ds = p * (dp - delta)
            e_ds = p * (e_dp + e_delta + F * (dp - delta).abs()) + ds.abs() * rq
            e_ds = e_ds + hp * (ds.abs() + e_ds)
            e_p = p * (rq + hp)
            acc = (n + m * grp + 80) * F
            dq[rows, hd] = scale * (ds @ b)
            edq[rows, hd] = scale * (e_ds @ b.abs() + acc * (ds.abs() @ b.abs()))
            dk[cols, hd // grp] += scale * (ds.t() @ a)
            edk[cols, hd // grp] += scale * (e_ds.t() @ a.abs() + acc * (ds.abs().t() @ a.abs()))
            dv[cols, hd // grp] += p.t() @ g
            edv[cols, hd // grp] += e_p.t() @ g.abs() + acc * (p.t() @ g.abs())
    out = {"o": (o, eo), "lse": (lse, elz)}
    if d_o is not None:
        out["dq"] = dq, edq + (h_ + 2 * F) * dq.abs()
        out["dk"] = dk, edk + (h_ + 2 * F) * dk.abs()
        out["dv"] = dv, edv + (h_ + 2 * F) * dv.abs()
    return out
