"""Dense operators beside the ball sparse attention layer: measured calls and their plain forms.

Around the sparse layer a model has dense parts: layer norms, affine maps with an activation or a
residual (the embedding before the blocks, the MLPs inside, the head behind them), and full
attention over whole clouds or prompts of different lengths, packed one behind another, which is
also what the sparse layer is compared with. The cases are those calls, from single tokens read
against a cache to training steps.

``own`` false: the operators in elementary torch operations, in 32 bits, rounded once at the end.
``own`` true: the calls of ``paper_2506_12541_amd.dense``.
"""
import math
import random

import torch

own = False

F32, F64 = torch.float32, torch.float64
EPS = 1e-5


# ---- cases ----

def _norm(name, rows, cols, dtype, train):
    return dict(name=name, op="layernorm", rows=rows, cols=cols, dtype=dtype, train=train)


def _linear(name, m, k, n, dtype, act, train, bias=True, residual=False):
    return dict(name=name, op="linear", m=m, k=k, n=n, dtype=dtype, act=act, train=train, bias=bias,
                residual=residual)


def _attention(name, seqs, q_lo, q_hi, heads, kv_heads, head_dim, dtype, causal, train, k_lo=0, k_hi=0, mix=1):
    """q_lo..q_hi: query rows of a sequence; k_hi > 0: keys of their own, k_lo..k_hi rows of a cache with
    k_hi rows for each sequence; else the keys are the sequence's own rows. mix: which lengths in the range."""
    return dict(name=name, op="attention", seqs=seqs, q_lo=q_lo, q_hi=q_hi, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, causal=causal, train=train, k_lo=k_lo, k_hi=k_hi, mix=mix)


def listed():
    return [
        # The norm of one step of a small batch of streams: latency.
        _norm("norm_step", 32, 512, "bf16", False),
        # Training on the block's residual stream: 65536 points of 8 heads of 64, float32.
        _norm("norm_train_65536", 65536, 512, "f32", True),
        # Training with wide bf16 rows.
        _norm("norm_train_wide", 16384, 4096, "bf16", True),
        # Two airflow clouds of 3586 points with an odd channel count.
        _norm("norm_train_odd", 7172, 333, "bf16", True),
        # A map of a few tokens: the weight is streamed once.
        _linear("linear_step", 4, 4096, 8192, "bf16", "gelu", False),
        # The MLP's first map over 65536 points, training.
        _linear("linear_train_65536", 65536, 512, 2048, "bf16", "gelu", True),
        # An output projection onto the residual stream, wide channels, inference.
        _linear("linear_residual", 8192, 4096, 4096, "bf16", "none", False, residual=True),
        # An embedding of one airflow cloud with odd widths, float32, training.
        _linear("linear_train_odd_f32", 3586, 515, 1029, "f32", "silu", True),
        # One new token for each of 32 streams, caches of up to 8192 rows, four query heads to a key head.
        _attention("attend_step", 32, 1, 1, 32, 8, 128, "bf16", True, False, k_lo=64, k_hi=8192),
        # Eight prompts of different lengths, causal, grouped heads.
        _attention("attend_prompt", 8, 200, 4096, 32, 8, 128, "bf16", True, False),
        # Training of full attention on 16 clouds of up to 3586 points, 8 heads of 64.
        _attention("attend_train_clouds", 16, 1500, 3586, 8, 8, 64, "bf16", False, True),
        # Float32 training on short ragged sequences.
        _attention("attend_train_f32", 5, 1, 700, 4, 2, 32, "f32", True, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["layernorm", "linear", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "layernorm":
        cols = _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        c = _norm(None, _log_int(rng, 1, min(1 << 17, (1 << 26) // cols)), cols, dtype, rng.random() < 0.6)
    elif op == "linear":
        k, n = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            k, n = max(64, k // 64 * 64), max(64, n // 64 * 64)
        train = rng.random() < 0.5
        cost = (1 << 37) if dtype == "bf16" else (1 << 34)
        m = _log_int(rng, 1, max(2, min(65536, cost // (k * n * (3 if train else 1)))))
        c = _linear(None, m, k, n, dtype, rng.choice(["none", "relu", "gelu", "silu"]), train,
                    bias=rng.random() < 0.7, residual=rng.random() < 0.3)
    else:
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        hd = rng.choice([32, 64, 64, 128])
        what = rng.choice(["step", "chunk", "whole", "whole"])
        if what == "whole":
            train = rng.random() < 0.6
            hi = _log_int(rng, 16, 4096 if dtype == "bf16" else 1024)
            seqs = min(rng.choice([1, 2, 3, 6, 16]), max(1, (1 << 29) // (heads * hi * hi)))
            c = _attention(None, seqs, max(1, hi // rng.choice([1, 3, 64])), hi, heads, kv, hd, dtype,
                           rng.random() < 0.5, train)
        else:
            hi = _log_int(rng, 32, 16384)
            q = 1 if what == "step" else _log_int(rng, 2, 256)
            seqs = min(_log_int(rng, 1, 64), max(1, (1 << 22) // (heads * hi)))
            c = _attention(None, seqs, max(1, q // 2), q, heads, kv, hd, dtype, rng.random() < 0.8, False,
                           k_lo=max(1, hi // 8), k_hi=hi)
        c["mix"] = rng.randrange(1 << 16)
    del c["name"]
    return c


def _lengths(case):
    """(query rows, key rows) of each sequence: part of the case, not of its seed."""
    r = random.Random(case["mix"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    k = [r.randint(case["k_lo"], case["k_hi"]) for _ in q] if case["k_hi"] else list(q)
    return q, k


def _pairs(lq, lk, causal):
    """Visible (query, key) pairs of one sequence; the last query sees the last key."""
    if not causal:
        return lq * lk
    first = max(0, lq - lk)                # rows before it see nothing
    n = lq - first
    return n * (lk - lq + first + 1) + n * (n - 1) // 2


# ---- inputs ----

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else F32


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape, scale=1.0, dtype=dt, shift=0.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case=case)
    if case["op"] == "layernorm":
        rows, cols = case["rows"], case["cols"]
        s.update(x=normal(rows, cols, scale=1.5, shift=0.3), gain=normal(cols, scale=0.1, dtype=F32, shift=1.0),
                 bias=normal(cols, scale=0.1, dtype=F32))
        if case["train"]:
            s["dy"] = normal(rows, cols)
    elif case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        s.update(x=normal(m, k), w=normal(n, k, scale=1.0 / math.sqrt(k)),
                 bias=normal(n, scale=0.1) if case["bias"] else None,
                 residual=normal(m, n) if case["residual"] else None)
        if case["train"]:
            s["dy"] = normal(m, n)
    else:
        lq, lk = _lengths(case)
        h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
        tq = sum(lq)
        cap = case["k_hi"]
        cu = lambda lens: torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        s.update(cu_q=cu(lq), max_q=max(lq), max_k=max(lk), used_k=None)
        if cap:
            s["cu_k"] = cu([cap] * len(lq))
            s["used_k"] = torch.tensor(lk, dtype=torch.int32, device="cuda")
        else:
            s["cu_k"] = s["cu_q"]
        tk = cap * len(lq) if cap else tq
        s.update(q=normal(tq, h, d, scale=1.4), k=normal(tk, hk, d, scale=1.4), v=normal(tk, hk, d))
        if case["train"]:
            s["d_o"] = normal(tq, h, d)
    return s


# ---- one pass ----

def run(state):
    return {"layernorm": _run_layernorm, "linear": _run_linear, "attention": _run_attention}[state["case"]["op"]](state)


def _run_layernorm(s):
    x, gain, bias, train = s["x"], s["gain"], s["bias"], s["case"]["train"]
    if own:
        from paper_2506_12541_amd import dense
        y, mean, rstd = dense.layernorm_forward(x, gain, bias, eps=EPS)
        if not train:
            return y, mean, rstd
        g = dense.layernorm_backward(x, gain, mean, rstd, s["dy"])
        return y, g["dx"], g["dgain"], g["dbias"]
    xf = x.to(F32)
    mean = xf.mean(1, keepdim=True)
    c = xf - mean
    rstd = (c.square().mean(1, keepdim=True) + EPS).rsqrt()
    xhat = c * rstd
    y = (xhat * gain + bias).to(x.dtype)
    if not train:
        return y, mean[:, 0], rstd[:, 0]
    dy = s["dy"].to(F32)
    g = dy * gain
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return y, dx.to(x.dtype), (dy * xhat).sum(0), dy.sum(0)


def _act(z, act):
    """The activation and its derivative."""
    if act == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        sg = 1 / (1 + torch.exp(-z))
        return z * sg, sg * (1 + z * (1 - sg))
    return z, None


def _run_linear(s):
    x, w, bias, residual, case = s["x"], s["w"], s["bias"], s["residual"], s["case"]
    act, train = case["act"], case["train"]
    if own:
        from paper_2506_12541_amd import dense
        y, pre = dense.linear_forward(x, w, bias, residual, act=act, save_pre=train)
        if not train:
            return y
        g = dense.linear_backward(x, w, s["dy"], pre, act=act, bias=bias is not None)
        return (y, g["dx"], g["dw"]) + ((g["db"],) if bias is not None else ())
    xf, wf = x.to(F32), w.to(F32)
    z = xf @ wf.t()
    if bias is not None:
        z = z + bias.to(F32)
    y, slope = _act(z, act)
    if residual is not None:
        y = y + residual.to(F32)
    y = y.to(x.dtype)
    if not train:
        return y
    dz = s["dy"].to(F32)
    if slope is not None:
        dz = dz * slope
    out = (y, (dz @ wf).to(x.dtype), (dz.t() @ xf).to(w.dtype))
    return out + ((dz.sum(0).to(bias.dtype),) if bias is not None else ())


def _spread(cu, used, most, total):
    """[sequences, most] rows of each sequence in the packed tensor, and whether each is one."""
    at = torch.arange(most, device=cu.device)
    length = cu[1:] - cu[:-1] if used is None else used
    return (cu[:-1, None] + at).clamp_(max=max(total - 1, 0)).long(), at < length[:, None], length


def _run_attention(s):
    q, k, v, case = s["q"], s["k"], s["v"], s["case"]
    causal, train = case["causal"], case["train"]
    if own:
        from paper_2506_12541_amd import dense
        o, lse = dense.attention_forward(q, k, v, s["cu_q"], s["cu_k"], s["used_k"], causal=causal)
        if not train:
            return o, lse
        g = dense.attention_backward(q, k, v, o, lse, s["d_o"], s["cu_q"], s["cu_k"], s["used_k"], causal=causal)
        return o, g["dq"], g["dk"], g["dv"]
    n, hk, d = case["seqs"], case["kv_heads"], case["head_dim"]
    grp = case["heads"] // hk
    scale = 1 / math.sqrt(d)
    rq, okq, lq = _spread(s["cu_q"], None, s["max_q"], q.shape[0])
    rk, okk, lk = _spread(s["cu_k"], s["used_k"], s["max_k"], k.shape[0])
    mq, mk = s["max_q"], s["max_k"]
    # padded: queries [n, key heads, group * rows, d], keys and values [n, key heads, rows, d]
    queries = lambda t: t[rq].to(F32).view(n, mq, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(n, hk, grp * mq, d)
    keys = lambda t: t[rk].to(F32).permute(0, 2, 1, 3).contiguous()
    qf, kf, vf = queries(q), keys(k), keys(v)
    vf = vf * okk[:, None, :, None]
    see = okq[:, :, None] & okk[:, None, :]
    if causal:
        see = see & (torch.arange(mk, device=q.device) <= (torch.arange(mq, device=q.device)[:, None]
                                                             + (lk - lq)[:, None, None]))
    see = see[:, None, None].expand(n, 1, grp, mq, mk).reshape(n, 1, grp * mq, mk)
    sc = (qf @ kf.transpose(2, 3)).mul_(scale).masked_fill_(~see, -math.inf)
    top = sc.amax(3, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = sc.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    of = p @ vf
    # back to packed rows
    pack = lambda t: t.view(n, hk, grp, mq, -1).permute(0, 3, 1, 2, 4).reshape(n, mq, hk * grp, -1)[okq]
    o = pack(of).to(q.dtype)
    if not train:
        return o, pack(total.log() + top)[..., 0].t().contiguous()
    do = queries(s["d_o"]) * okq[:, None, None, :, None].expand(n, 1, grp, mq, 1).reshape(n, 1, grp * mq, 1)
    dv = p.transpose(2, 3) @ do
    ds = p * (do @ vf.transpose(2, 3) - (do * of).sum(3, keepdim=True)) * scale
    dq, dk = ds @ kf, ds.transpose(2, 3) @ qf
    unpad = lambda t: t.permute(0, 2, 1, 3)[okk].to(k.dtype)
    return o, pack(dq).to(q.dtype), unpad(dk), unpad(dv)


# ---- floors ----

def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "layernorm":
        x, c = case["rows"] * case["cols"], case["cols"]
        if case["train"]:     # x and dy in, y and dx out, gain and bias in and their gradients out
            return {"bytes": 4 * x * esz + 16 * c, "flops": 16 * x}
        return {"bytes": 2 * x * esz + 8 * c + 8 * case["rows"], "flops": 7 * x}
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        b, r = n if case["bias"] else 0, m * n if case["residual"] else 0
        if case["train"]:     # x, w, bias, residual, dy in; y, dx, dw, db out
            return {"bytes": esz * (2 * m * k + 2 * n * k + 2 * m * n + 2 * b + r), "flops": 6 * m * n * k}
        return {"bytes": esz * (m * k + n * k + m * n + b + r), "flops": 2 * m * n * k}
    lq, lk = _lengths(case)
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(lq, lk))
    q, kv = sum(lq) * h * d, sum(lk) * hk * d
    if case["train"]:         # q, k, v, dO in; o, dq, dk, dv out
        return {"bytes": esz * (4 * q + 4 * kv), "flops": 14 * pairs * h * d}
    return {"bytes": esz * (2 * q + 2 * kv) + 4 * sum(lq) * h, "flops": 4 * pairs * h * d}


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"layernorm": _exact_layernorm, "linear": _exact_linear, "attention": _exact_attention}[case["op"]](s)


def _exact_layernorm(s):
    x, gain, bias = s["x"].to(F64), s["gain"].to(F64), s["bias"].to(F64)
    c = x.shape[1]
    mean = x.sum(1) / c
    var = ((x - mean[:, None]) ** 2).sum(1) / c
    std = (var + EPS).sqrt()
    y = gain * ((x - mean[:, None]) / std[:, None]) + bias
    if not s["case"]["train"]:
        return y, mean, 1 / std
    dy = s["dy"].to(F64)
    unit = (x - mean[:, None]) / std[:, None]
    du = dy * gain
    # d unit_j / d x_i = (delta_ij - 1/c - unit_i unit_j / c) / std
    dx = (du - du.sum(1, keepdim=True) / c - unit * ((du * unit).sum(1, keepdim=True) / c)) / std[:, None]
    return y, dx, (dy * unit).sum(0), dy.sum(0)


def _exact_linear(s):
    case = s["case"]
    x, w = s["x"].to(F64), s["w"].to(F64)
    z = torch.mm(x, w.t())
    if s["bias"] is not None:
        z += s["bias"].to(F64)
    act = case["act"]
    if act == "none":
        y, slope = z, torch.ones_like(z)
    elif act == "relu":
        y, slope = torch.where(z > 0, z, 0 * z), torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
    elif act == "gelu":
        upto = torch.special.erfc(-z / math.sqrt(2.0)) / 2     # normal distribution function
        y, slope = z * upto, upto + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    else:
        sg = torch.sigmoid(z)
        y, slope = z * sg, sg + z * sg * torch.sigmoid(-z)
    if s["residual"] is not None:
        y = y + s["residual"].to(F64)
    if not case["train"]:
        return y
    dz = s["dy"].to(F64) * slope
    out = (y, torch.mm(dz, w), torch.mm(dz.t(), x))
    return out + ((dz.sum(0),) if s["bias"] is not None else ())


def _exact_attention(s):
    case = s["case"]
    lq, lk = _lengths(case)
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    grp = h // hk
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    train = case["train"]
    o, dq = (torch.zeros(s["q"].shape, dtype=F64, device="cuda") for _ in range(2))
    dk, dv = (torch.zeros(s["k"].shape, dtype=F64, device="cuda") for _ in range(2))
    lse = torch.full((h, s["q"].shape[0]), -math.inf, dtype=F64, device="cuda")
    for i in range(case["seqs"]):
        a, b = lq[i], lk[i]
        if a == 0 or b == 0:
            continue
        rows, cols = slice(cq[i], cq[i] + a), slice(ck[i], ck[i] + b)
        hidden = None
        if case["causal"]:
            at = torch.arange(b - a, b, device="cuda")     # the last key that each query sees
            hidden = torch.arange(b, device="cuda")[None, :] > at[:, None]
        for j in range(h):
            q, k, v = s["q"][rows, j].to(F64), s["k"][cols, j // grp].to(F64), s["v"][cols, j // grp].to(F64)
            sc = torch.mm(q, k.t()) / math.sqrt(d)
            if hidden is not None:
                sc = torch.where(hidden, -math.inf, sc)
            z = torch.logsumexp(sc, 1)
            p = torch.where(torch.isfinite(z)[:, None], torch.exp(sc - z[:, None]), 0.0)
            lse[j, rows] = z
            o[rows, j] = torch.mm(p, v)
            if train:
                g = s["d_o"][rows, j].to(F64)
                dp = torch.mm(g, v.t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                dq[rows, j] = torch.mm(ds, k)
                dk[cols, j // grp] += torch.mm(ds.t(), q)
                dv[cols, j // grp] += torch.mm(p.t(), g)
    return (o, dq, dk, dv) if train else (o, lse)
