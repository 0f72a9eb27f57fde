"""Float64 definitions of rotary positions with head norms, the gated map and the 8-bit cache, with error
bounds for kernels that accumulate in float32 and round each result once (F and HALF as in dense_ref)."""
import math

import torch

from dense_ref import F, F64, HALF, act


# ---- rotary positions ----

def _turned(x, c, s, rot, interleaved):
    """The pairs (a, b) -> (a c - b s, a s + b c); the rest as it is."""
    out = x.clone()
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    return out


def rotary(x, pos, freq, gain, eps, interleaved, mag, dy=None):
    """x [rows, heads, d]. A cosine is off by 2 F (its argument, at most pi / 4 after the reduction, is rounded to
    float32: 0.8 F; the polynomial's last steps: 1.1 F at most), its product with mag by F more; the angle in 64
    bits by 2^-50 of itself. A head's sum of squares takes at most 32 additions in a lane and 6 joining
    lanes, all positive: 40 F, half of that in the root."""
    h = HALF[x.dtype]
    x, pos, freq = x.to(F64), pos.to(F64), freq.to(F64)
    rows, _, d = x.shape
    rot = 2 * freq.numel()
    pos = pos.reshape(rows, -1)
    t = pos.repeat_interleave(rot // 2 // pos.shape[1], 1) * freq
    c, s = mag * t.cos()[:, None], mag * t.sin()[:, None]
    e_c = (mag * (3 * F + 2.0 ** -50 * t.abs()))[:, None]
    rstd = u = None
    if gain is None:
        n, e_n = x, torch.zeros_like(x)
    else:
        gain = gain.to(F64)
        rstd = 1 / ((x * x).mean(2, keepdim=True) + eps).sqrt()
        u = x * rstd
        n = u * gain
        e_n = 28 * F * n.abs()

    def e_turn(v, e_v):
        """Error of turned values v with errors e_v."""
        big = _turned_abs(v.abs(), c.abs(), s.abs(), rot, interleaved)
        off = _turned_abs(e_v, c.abs(), s.abs(), rot, interleaved)
        both = _turned_abs(v.abs(), e_c, e_c, rot, interleaved, rest=0.0)
        return off + both + 3 * F * big

    y = _turned(n, c, s, rot, interleaved)
    e_y = e_turn(n, e_n)
    out = {"y": (y, h * (y.abs() + e_y) + e_y)}
    if dy is None:
        return out
    dy = dy.to(F64)
    dn = _turned(dy, c, -s, rot, interleaved)
    e_dn = e_turn(dy, torch.zeros_like(dy))
    if gain is None:
        out["dx"] = dn, h * (dn.abs() + e_dn) + e_dn
        return out
    g = dn * gain
    e_g = gain.abs() * e_dn + F * g.abs()
    m = (g * u).mean(2, keepdim=True)
    e_m = 80 * F * (g * u).abs().mean(2, keepdim=True) + (e_g * u.abs()).mean(2, keepdim=True)
    dx = rstd * (g - u * m)
    e = rstd * (e_g + u.abs() * e_m + 30 * F * (u * m).abs() + 3 * F * g.abs()) + 28 * F * dx.abs()
    out["dx"] = dx, h * (dx.abs() + e) + e
    terms = (dn * u).reshape(-1, d)
    out["dgain"] = terms.sum(0), ((terms.shape[0] + 50) * F * terms.abs() + (e_dn * u.abs()).reshape(-1, d)).sum(0)
    return out


def _turned_abs(v, c, s, rot, interleaved, rest=1.0):
    out = rest * v
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = v[..., ia], v[..., ib]
    out[..., ia], out[..., ib] = a * c + b * s, a * s + b * c
    return out


# ---- gated map ----

def gated(x, w, bias, kind, dy=None):
    """As dense_ref.linear: sums of k products are off by (k + 2) F of the sum of magnitudes, activations have
    slopes of at most 1.13 that change by 1.1 per unit, and are evaluated to 16 F of their value and of z."""
    h = HALF[x.dtype]
    x, w = x.to(F64), w.to(F64)
    k, n = x.shape[1], w.shape[0] // 2
    z = x @ w.t()
    e_z = (k + 2) * F * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.to(F64)
        e_z = e_z + F * z.abs()
    g, u, e_gate, e_u = z[:, :n], z[:, n:], e_z[:, :n], e_z[:, n:]
    a, slope = act(g, kind)
    own = 16 * F * (a.abs() + g.abs()) if kind in ("gelu", "silu") else 0
    e_a = 1.13 * e_gate + own
    y = a * u
    e_y = e_a * u.abs() + a.abs() * e_u + e_a * e_u + 2 * F * y.abs()
    out = {"y": (y, h * (y.abs() + e_y) + e_y)}
    if dy is None:
        return out
    dy = dy.to(F64)
    off_g, off_u = h * g.abs() + e_gate, h * u.abs() + e_u       # as they were saved
    if kind == "none":
        e_slope = torch.zeros_like(g)
    elif kind == "relu":                                        # its sign can only differ where the sum's can
        e_slope = (g.abs() <= e_gate).to(F64)
    else:
        e_slope = 1.1 * off_g + 16 * F * (1 + g.abs())
    dg, du = dy * u * slope, dy * a
    e_dg = dy.abs() * (off_u * slope.abs() + (u.abs() + off_u) * e_slope) + 3 * F * dg.abs()
    e_du = dy.abs() * (1.13 * off_g + own) + 2 * F * du.abs()
    dz, e_dz = torch.cat((dg, du), 1), torch.cat((e_dg, e_du), 1)
    m = dz.shape[0]
    e_in = e_dz + h * (dz.abs() + e_dz)                         # as it enters the products
    dx, dw, db = dz @ w, dz.t() @ x, dz.sum(0)
    e_dx = e_in @ w.abs() + (2 * n + 2) * F * ((dz.abs() + e_in) @ w.abs())
    e_dw = e_in.t() @ x.abs() + (m + 70) * F * ((dz.abs() + e_in).t() @ x.abs())
    e_db = e_dz.sum(0) + (m + 70) * F * (dz.abs() + e_dz).sum(0)
    for name, v, e in (("dx", dx, e_dx), ("dw", dw, e_dw), ("db", db, e_db)):
        out[name] = v, h * (v.abs() + e) + e
    return out


# ---- 8-bit cache ----

def quantise(x):
    """Rows of heads x [rows, heads, d] -> (values the bytes stand for [rows, heads, d] float64, codes
    [heads, rows]). By the definition: a search over the exponents, and the e4m3 numbers written out."""
    x = x.detach().cpu().to(F64)
    fin = torch.isfinite(x)
    top = torch.where(fin, x.abs(), 0.0).amax(2)
    e = torch.full(top.shape, 63)
    for cand in range(62, -65, -1):
        e = torch.where(top <= 448.0 * 2.0 ** cand, cand, e)
    scale = torch.tensor([2.0 ** i for i in range(-64, 64)], dtype=F64)[e + 64][..., None]
    y = (torch.where(fin, x, 0.0) / scale).clamp(-448, 448)
    grid = torch.tensor(sorted({m * 2.0 ** k for m in range(8, 16) for k in range(-9, 6)} | {m * 2.0 ** -9 for m in range(8)}),
                        dtype=F64)
    grid = grid[grid <= 448]
    hi = torch.searchsorted(grid, y.abs().contiguous()).clamp(max=len(grid) - 1)      # first grid value >= |y|
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - y.abs(), y.abs() - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)) | (hi == 0), hi, lo)   # nearest, ties to even
    q = torch.where(fin, grid[pick] * torch.sign(y) * scale, math.nan)
    return q, (e + 127).to(torch.uint8).t().contiguous()
