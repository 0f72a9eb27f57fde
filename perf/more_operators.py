"""Operators of the block around packed attention: measured calls and their plain forms.

Between a fused projection and the attention lie the norms of each head's queries and keys and the
rotation by their positions (a token's index, or a point's coordinates); in serving the keys and
values go into a cache of 8 bits that the attention reads; behind the attention comes the gated
feed-forward map. The cases are those calls, from single tokens to training steps.

``own`` false: the operators in elementary torch operations, in 32 bits, rounded once at the end
(angles of positions in 64). ``own`` true: the calls of ``paper_2506_12541_amd.dense``.
"""
import math
import random

import torch

own = False

F32, F64 = torch.float32, torch.float64
EPS = 1e-6
LOW, HIGH = -64, 63            # exponents of a cache row's scale
MOST = 448.0                   # the largest e4m3 value


# ---- cases ----

def _rotary(name, rows, heads, kv_heads, head_dim, rot, dtype, norm, interleaved, train, axes=1, reach=8192, factor=1.0,
            fused=False):
    """axes = 1: positions are integers below reach; more: coordinates in [0, reach). factor: the frequencies are
    scaled for a context that many times longer. fused: queries and keys are views of one projection."""
    return dict(name=name, op="rotary", rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot=rot, dtype=dtype,
                norm=norm, interleaved=interleaved, train=train, axes=axes, reach=reach, factor=factor, fused=fused)


def _cache(name, seqs, q_lo, q_hi, k_hi, kv_heads, head_dim, dtype, whole, mix=1):
    """q_lo..q_hi new rows of each sequence, written behind what its cache of k_hi rows holds; read back: those
    rows, or (whole) all that the cache holds."""
    return dict(name=name, op="cache", seqs=seqs, q_lo=q_lo, q_hi=q_hi, k_lo=q_hi, k_hi=k_hi, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, whole=whole, mix=mix)


def _attend(name, seqs, q_lo, q_hi, k_lo, k_hi, heads, kv_heads, head_dim, dtype, causal, mix=1):
    return dict(name=name, op="attend", seqs=seqs, q_lo=q_lo, q_hi=q_hi, k_lo=k_lo, k_hi=k_hi, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, causal=causal, mix=mix)


def _gated(name, m, k, n, dtype, act, train, bias=False):
    return dict(name=name, op="gated", m=m, k=k, n=n, dtype=dtype, act=act, train=train, bias=bias)


def listed():
    return [
        # One new token for each of 32 streams, grouped heads, normed, far positions of a context made 4 times longer: latency.
        _rotary("rotary_step", 32, 32, 8, 128, 128, "bf16", True, False, False, reach=131072, factor=4.0),
        # A batch of prompts, 16384 tokens, straight from the fused projection; neighbouring dimensions rotate.
        _rotary("rotary_prompt", 16384, 32, 8, 128, 128, "bf16", False, True, False, fused=True),
        # Training on 65536 points of 8 heads of 64: the three coordinates turn 8 pairs each, the rest of the head passes.
        _rotary("rotary_train_65536", 65536, 8, 8, 64, 48, "bf16", True, False, True, axes=3, reach=64),
        # Float32 training on one airflow cloud of 3586 points, odd head counts and sizes.
        _rotary("rotary_train_odd_f32", 3586, 6, 3, 80, 20, "f32", True, True, True, axes=2, reach=100),
        # The cache's share of one step of 32 streams: latency.
        _cache("cache_step", 32, 1, 1, 8192, 8, 128, "bf16", False),
        # Eight prompts of different lengths go into their caches and are read back whole.
        _cache("cache_prompt", 8, 200, 4096, 4096, 8, 128, "bf16", True),
        # One new token for each of 32 streams against caches of up to 8192 rows, four query heads to a key head.
        _attend("attend8_step", 32, 1, 1, 64, 8192, 32, 8, 128, "bf16", True),
        # Two streams far into a long context.
        _attend("attend8_long", 2, 1, 1, 65536, 131072, 32, 8, 128, "bf16", True),
        # Chunks of four prompts against what their caches hold.
        _attend("attend8_chunk", 4, 200, 1024, 1024, 8192, 32, 8, 128, "bf16", True),
        # A map of a few tokens: the weight is streamed once.
        _gated("gated_step", 4, 4096, 8192, "bf16", "silu", False),
        # The feed-forward of 65536 points, training.
        _gated("gated_train_65536", 65536, 512, 2048, "bf16", "silu", True),
        # Odd widths on one airflow cloud, float32, training.
        _gated("gated_train_odd_f32", 3586, 515, 1029, "f32", "gelu", True, bias=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "cache", "attend", "gated"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    if op == "rotary":
        hd = rng.choice([32, 64, 64, 128, 128, 2 * rng.randint(8, 128)])
        rot = rng.choice([hd, hd, hd // 4 * 2, 2 * rng.randint(1, hd // 2)])
        axes = rng.choice([a for a in (1, 1, 2, 3) if rot // 2 % a == 0])
        rows = _log_int(rng, 1, min(65536, (1 << (26 if dtype == "bf16" else 25)) // ((heads + kv) * hd)))
        c = _rotary(None, rows, heads, kv, hd, rot, dtype, rng.random() < 0.6, rng.random() < 0.5, rng.random() < 0.5, axes=axes,
                    reach=_log_int(rng, 16, 1 << 18) if axes == 1 else _log_int(rng, 2, 1024),
                    factor=rng.choice([1.0, 1.0, 2.0, 8.0]), fused=rng.random() < 0.5)
    elif op == "gated":
        k, n = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            k, n = max(64, k // 64 * 64), max(64, n // 64 * 64)
        train = rng.random() < 0.5
        cost = (1 << 36) if dtype == "bf16" else (1 << 33)
        m = _log_int(rng, 1, max(2, min(65536, cost // (k * n * (3 if train else 1)))))
        c = _gated(None, m, k, n, dtype, rng.choice(["none", "relu", "gelu", "silu", "silu"]), train, bias=rng.random() < 0.4)
    else:
        hd = rng.choice([32, 64, 128, 128])
        hi = _log_int(rng, 32, 32768)
        q = rng.choice([1, 1, _log_int(rng, 2, 512)])
        q = min(q, hi)
        if op == "cache":
            seqs = min(_log_int(rng, 1, 64), max(1, (1 << 25) // (hi * kv * hd)))
            c = _cache(None, seqs, max(1, q // 2), q, hi, kv, hd, dtype, rng.random() < 0.5)
        else:
            seqs = min(_log_int(rng, 1, 64), max(1, (1 << 22) // (heads * hi)), max(1, (1 << 29) // (heads * hi * q)))
            c = _attend(None, seqs, max(1, q // 2), q, max(1, hi // 8), hi, heads, kv, hd, dtype, rng.random() < 0.8)
        c["mix"] = rng.randrange(1 << 16)
    del c["name"]
    return c


def _lengths(case):
    """(new rows, cache rows in use with them) of each sequence: part of the case, not of its seed."""
    r = random.Random(case["mix"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    k = [r.randint(case["k_lo"], case["k_hi"]) for _ in q]
    if case["op"] == "cache" and case["whole"] and case["k_lo"] == case["k_hi"]:    # prompts: nothing before them
        k = list(q)
    return q, k


def _read(case):
    """Rows of each sequence that a cache case reads back."""
    q, k = _lengths(case)
    return k if case["whole"] else q


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


def _frequencies(case):
    """Angles a unit of position, and the factor on the rotated values, of a context that is longer by a factor: pairs
    that turn less than once in the 4096 positions of training are slowed by it, those that turn more than 32 times
    are kept, in between a line; coordinates: geometric from 1 on each axis."""
    pairs = case["rot"] // 2 // case["axes"]
    f = 10000.0 ** (-torch.arange(pairs, dtype=F64) / pairs)
    s = case["factor"]
    if s > 1:
        keep = ((f * (4096 / (2 * math.pi)) - 1) / 31).clamp_(0, 1)
        f = f * keep + f / s * (1 - keep)
    return f.repeat(case["axes"]).cuda(), 0.1 * math.log(s) + 1


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape, scale=1.0, dtype=dt, shift=0.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case=case)
    if case["op"] == "rotary":
        rows, h, hk, d = case["rows"], case["heads"], case["kv_heads"], case["head_dim"]
        if case["fused"]:
            qkv = normal(rows, h + 2 * hk, d, scale=1.3)
            q, k = qkv[:, :h], qkv[:, h:h + hk]
        else:
            q, k = normal(rows, h, d, scale=1.3), normal(rows, hk, d, scale=1.3)
        if case["axes"] == 1:
            at = torch.randint(0, case["reach"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        else:
            at = torch.rand((rows, case["axes"]), generator=gen, device="cuda").mul_(case["reach"])
        freq, mag = _frequencies(case)
        s.update(q=q, k=k, at=at, freq=freq, mag=mag, gain_q=None, gain_k=None)
        if case["norm"]:
            s.update(gain_q=normal(d, scale=0.1, dtype=F32, shift=1.0), gain_k=normal(d, scale=0.1, dtype=F32, shift=1.0))
        if case["train"]:
            s.update(dq=normal(rows, h, d), dk=normal(rows, hk, d))
        return s
    if case["op"] == "gated":
        m, k, n = case["m"], case["k"], case["n"]
        s.update(x=normal(m, k), w=normal(2 * n, k, scale=1.0 / math.sqrt(k)),
                 bias=normal(2 * n, scale=0.1) if case["bias"] else None)
        if case["train"]:
            s["dy"] = normal(m, n)
        return s
    lq, lk = _lengths(case)
    hk, d, cap = case["kv_heads"], case["head_dim"], case["k_hi"]
    cu = lambda lens: torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    s.update(cu_q=cu(lq), cu_k=cu([cap] * len(lq)), used=torch.tensor(lk, dtype=torch.int32, device="cuda"), max_k=max(lk))
    rows = cap * len(lq)
    # what the caches hold: rows quantised as they were written, a few heads with larger values than the rest
    loud = torch.exp2(torch.randint(-2, 3, (1, hk, 1), generator=gen, device="cuda").to(F32))
    for name in ("k", "v"):
        held = normal(rows, hk, d, scale=1.4 if name == "k" else 1.0, dtype=F32) * (1 if name == "k" else loud)
        byte, code = _quantise(held)
        s["cache_" + name], s["exp_" + name] = byte, code.t().contiguous()
        del held
    if case["op"] == "cache":
        n = sum(lq)
        lr = _read(case)
        s.update(k=normal(n, hk, d, scale=1.4), v=normal(n, hk, d) * loud.to(dt), cu_r=cu(lr), n_r=sum(lr))
    else:
        s.update(q=normal(sum(lq), case["heads"], d, scale=1.4), max_q=max(lq))
    return s


# ---- one pass ----

def run(state):
    return {"rotary": _run_rotary, "cache": _run_cache, "attend": _run_attend, "gated": _run_gated}[state["case"]["op"]](state)


def _pairs_of(x, rot, interleaved):
    """First and second values of the rotating pairs."""
    r = x[..., :rot]
    return (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])


def _joined(a, b, rest, interleaved):
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _run_rotary(s):
    case = s["case"]
    rot, inter, train = case["rot"], case["interleaved"], case["train"]
    if own:
        from paper_2506_12541_amd import dense
        how = dict(gain_q=s["gain_q"], gain_k=s["gain_k"], eps=EPS, interleaved=inter, magnitude=s["mag"])
        q, k = dense.rotary_forward(s["q"], s["k"], s["at"], s["freq"], **how)
        if not train:
            return q, k
        g = dense.rotary_backward(s["dq"], s["dk"], s["at"], s["freq"], q=s["q"], k=s["k"], **how)
        return (q, k, g["dq"], g["dk"]) + ((g["dgain_q"], g["dgain_k"]) if case["norm"] else ())
    at = s["at"].to(F64)
    at = at[:, None] if at.dim() == 1 else at.repeat_interleave(rot // 2 // case["axes"], dim=1)
    angle = at * s["freq"]
    cos, sin = ((t(angle) * s["mag"]).to(F32)[:, None] for t in (torch.cos, torch.sin))

    def forward(x, gain):
        n = x.to(F32)
        if gain is not None:
            n = n * (n.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain
        a, b = _pairs_of(n, rot, inter)
        return _joined(a * cos - b * sin, a * sin + b * cos, n[..., rot:], inter).to(x.dtype)

    def backward(x, gain, dy):
        g = dy.to(F32)
        a, b = _pairs_of(g, rot, inter)
        dn = _joined(a * cos + b * sin, b * cos - a * sin, g[..., rot:], inter)
        if gain is None:
            return dn.to(x.dtype), None
        xf = x.to(F32)
        rstd = (xf.square().mean(-1, keepdim=True) + EPS).rsqrt()
        xhat = xf * rstd
        g = dn * gain
        return (rstd * (g - xhat * (g * xhat).mean(-1, keepdim=True))).to(x.dtype), (dn * xhat).sum((0, 1))

    out = (forward(s["q"], s["gain_q"]), forward(s["k"], s["gain_k"]))
    if not train:
        return out
    dq, gq = backward(s["q"], s["gain_q"], s["dq"])
    dk, gk = backward(s["k"], s["gain_k"], s["dk"])
    return out + (dq, dk) + ((gq, gk) if case["norm"] else ())


def _two_to(e):
    """2^e of whole numbers, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(F32)


def _quantise(x):
    """e4m3 values of rows of a head and the codes (exponent + 127) of their scales."""
    xf = x.to(F32)
    part, e = torch.frexp(xf.abs().amax(-1))
    e = (e - 9 + (part > 0.875)).clamp_(LOW, HIGH)       # 448 = 0.875 2^9
    return (xf * _two_to(-e)[..., None]).clamp_(-MOST, MOST).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _rows_of(cu_q, cu_k, used, n, total):
    """The cache rows of n packed rows: the last of each sequence's that are in use."""
    at = torch.arange(n, device=cu_q.device)
    seq = torch.searchsorted(cu_q[1:].contiguous(), at, right=True, out_int32=True).long()
    return (cu_k[seq] + used[seq] - cu_q[seq + 1]).long() + at


def _run_cache(s):
    case, k, v = s["case"], s["k"], s["v"]
    if own:
        from paper_2506_12541_amd import dense
        cache = dense.Cache(s["cache_k"], s["cache_v"], s["exp_k"], s["exp_v"])
        dense.cache_write(cache, k, v, s["cu_q"], s["cu_k"], s["used"])
        kr, vr = dense.cache_read(cache, s["n_r"], s["cu_r"], s["cu_k"], s["used"], dtype=k.dtype)
        return kr, vr, s["exp_k"], s["exp_v"]
    to = _rows_of(s["cu_q"], s["cu_k"], s["used"], k.shape[0], s["exp_k"].shape[1])
    at = _rows_of(s["cu_r"], s["cu_k"], s["used"], s["n_r"], s["exp_k"].shape[1])

    def through(x, held, codes):
        byte, code = _quantise(x)
        held.view(torch.uint8)[to] = byte.view(torch.uint8)
        codes[:, to] = code.t()
        back = held.view(torch.uint8)[at].view(torch.float8_e4m3fn).to(F32)
        return (back * _two_to(codes[:, at].t().to(torch.int32) - 127)[..., None]).to(x.dtype)

    return through(k, s["cache_k"], s["exp_k"]), through(v, s["cache_v"], s["exp_v"]), s["exp_k"], s["exp_v"]


def _spread(first, length, most, total):
    """[sequences, most] rows of each sequence in a tensor of total rows, and whether each is one."""
    at = torch.arange(most, device=first.device)
    return (first[:, None] + at).clamp_(max=max(total - 1, 0)).long(), at < length[:, None]


def _run_attend(s):
    q, case = s["q"], s["case"]
    if own:
        from paper_2506_12541_amd import dense
        cache = dense.Cache(s["cache_k"], s["cache_v"], s["exp_k"], s["exp_v"])
        return dense.cache_attention_forward(q, cache, s["cu_q"], s["cu_k"], s["used"], causal=case["causal"])
    n, hk, d = case["seqs"], case["kv_heads"], case["head_dim"]
    grp = case["heads"] // hk
    cu_q, lk, mq, mk = s["cu_q"], s["used"], s["max_q"], s["max_k"]
    lq = cu_q[1:] - cu_q[:-1]
    rq, okq = _spread(cu_q[:-1], lq, mq, q.shape[0])
    rk, okk = _spread(s["cu_k"][:-1], lk, mk, s["cache_k"].shape[0])

    def held(byte, code):      # padded [n, key heads, rows, d] values of the caches
        x = byte.view(torch.uint8)[rk].view(torch.float8_e4m3fn).to(F32)
        x.mul_(_two_to(code.t()[rk].to(torch.int32) - 127)[..., None])
        return x.permute(0, 2, 1, 3).contiguous()

    # padded queries [n, key heads, group * rows, d]
    qf = q[rq].to(F32).view(n, mq, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(n, hk, grp * mq, d)
    kf = held(s["cache_k"], s["exp_k"])
    see = okq[:, :, None] & okk[:, None, :]
    if case["causal"]:
        see = see & (torch.arange(mk, device=q.device) <= (torch.arange(mq, device=q.device)[:, None] + (lk - lq)[:, None, None]))
    see = see[:, None, None].expand(n, 1, grp, mq, mk).reshape(n, 1, grp * mq, mk)
    sc = (qf @ kf.transpose(2, 3)).mul_(1 / math.sqrt(d)).masked_fill_(~see, -math.inf)
    del kf
    top = sc.amax(3, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = sc.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    of = (p @ held(s["cache_v"], s["exp_v"])) / torch.where(total > 0, total, torch.ones_like(total))
    pack = lambda t: t.view(n, hk, grp, mq, -1).permute(0, 3, 1, 2, 4).reshape(n, mq, hk * grp, -1)[okq]
    return pack(of).to(q.dtype), pack(total.log() + top)[..., 0].t().contiguous()


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
    return z, torch.ones_like(z)


def _run_gated(s):
    x, w, bias, case = s["x"], s["w"], s["bias"], s["case"]
    act, train, n = case["act"], case["train"], case["n"]
    if own:
        from paper_2506_12541_amd import dense
        y, pre = dense.gated_forward(x, w, bias, act=act, save_pre=train)
        if not train:
            return y
        g = dense.gated_backward(x, w, s["dy"], pre, act=act, bias=bias is not None)
        return (y, g["dx"], g["dw"]) + ((g["db"],) if bias is not None else ())
    xf, wf = x.to(F32), w.to(F32)
    z = xf @ wf.t()
    if bias is not None:
        z = z + bias.to(F32)
    a, slope = _act(z[:, :n], act)
    u = z[:, n:]
    y = (a * u).to(x.dtype)
    if not train:
        return y
    dy = s["dy"].to(F32)
    dz = torch.cat((dy * u * slope, dy * a), 1)
    out = (y, (dz @ wf).to(x.dtype), (dz.t() @ xf).to(w.dtype))
    return out + ((dz.sum(0).to(bias.dtype),) if bias is not None else ())


# ---- floors ----

def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rotary":
        x = case["rows"] * (case["heads"] + case["kv_heads"]) * case["head_dim"]
        small = 4 * case["rows"] * case["axes"] + 4 * case["rot"]
        if case["train"]:     # x and dy in, y and dx out
            return {"bytes": 4 * x * esz + small, "flops": 24 * x}
        return {"bytes": 2 * x * esz + small, "flops": 8 * x}
    if case["op"] == "gated":
        m, k, n = case["m"], case["k"], case["n"]
        b = 2 * n if case["bias"] else 0
        if case["train"]:     # x, w, bias, dy in; y, dx, dw, db out
            return {"bytes": esz * (2 * m * k + 4 * n * k + 2 * m * n + 2 * b), "flops": 12 * m * n * k}
        return {"bytes": esz * (m * k + 2 * n * k + m * n + b), "flops": 4 * m * n * k}
    lq, lk = _lengths(case)
    hk, d = case["kv_heads"], case["head_dim"]
    if case["op"] == "cache":   # new rows in, their bytes out; bytes read back in, values out (new bytes are read where they lie)
        new, back = 2 * sum(lq) * hk, 2 * sum(_read(case)) * hk
        return {"bytes": new * (d * esz + d + 1) + (back - new) * (d + 1) + back * d * esz, "flops": 4 * new * d + back * d}
    h = case["heads"]
    pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(lq, lk))
    return {"bytes": 2 * esz * sum(lq) * h * d + 2 * sum(lk) * hk * (d + 1) + 4 * sum(lq) * h, "flops": 4 * pairs * h * d}


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"rotary": _exact_rotary, "cache": _exact_cache, "attend": _exact_attend, "gated": _exact_gated}[case["op"]](s)


def _exact_rotary(s):
    case = s["case"]
    rot, rows, half = case["rot"], case["rows"], case["rot"] // 2
    at = s["at"].to(F64).reshape(rows, case["axes"])
    axis = torch.arange(half, device="cuda") // (half // case["axes"])
    turn = torch.polar(torch.full((rows, half), s["mag"], dtype=F64, device="cuda"), at[:, axis] * s["freq"][None, :])[:, None]

    def turned(x, by):       # the rotating part as complex numbers
        r, out = x[..., :rot], x.clone()
        if case["interleaved"]:
            z = torch.view_as_complex(r.reshape(*r.shape[:-1], half, 2).contiguous()) * by
            out[..., :rot] = torch.view_as_real(z).reshape(r.shape)
        else:
            z = torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous()) * by
            out[..., :half], out[..., half:rot] = z.real, z.imag
        return out

    out, grads, gains = [], [], []
    for name in ("q", "k"):
        x, gain = s[name].to(F64), s["gain_" + name]
        if gain is not None:
            root = ((x * x).sum(-1, keepdim=True) / case["head_dim"] + EPS).sqrt()
            unit, gain = x / root, gain.to(F64)
        out.append(turned(x if gain is None else unit * gain, turn))
        if case["train"]:
            dn = turned(s["d" + name].to(F64), turn.conj())
            if gain is None:
                grads.append(dn)
            else:             # d unit_j / d x_i = (delta_ij - unit_i unit_j / d) / root
                du = dn * gain
                grads.append((du - unit * ((du * unit).sum(-1, keepdim=True) / case["head_dim"])) / root)
                gains.append((dn * unit).reshape(-1, case["head_dim"]).sum(0))
    return tuple(out + grads + gains)


def _scale(e):
    """2^e of whole numbers in 64 bits (a power function may be off by a rounding, which decides ties)."""
    return ((e.to(torch.int64) + 1023) << 52).view(F64)


def _exact_cache(s):
    case = s["case"]
    lq, lk = _lengths(case)
    lr, cap, dev = _read(case), case["k_hi"], "cuda"
    to = torch.cat([torch.arange(i * cap + b - a, i * cap + b, device=dev) for i, (a, b) in enumerate(zip(lq, lk))])
    back = torch.cat([torch.arange(i * cap + b - a, i * cap + b, device=dev) for i, (a, b) in enumerate(zip(lr, lk))])
    out, codes = [], []
    for name in ("k", "v"):
        x = s[name].to(F64)
        top = x.abs().amax(2)
        e = torch.where(top > 0, torch.ceil(torch.log2(top / MOST)), torch.full_like(top, LOW))
        e = torch.where(top > MOST * _scale(e), e + 1, torch.where(top <= MOST * _scale(e - 1), e - 1, e)).clamp(LOW, HIGH)
        scale = _scale(e)[:, :, None]
        y = (x / scale).clamp(-MOST, MOST)
        step = _scale(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
        code = s["exp_" + name].clone()
        code[:, to] = (e.t() + 127).to(torch.uint8)
        held = s["cache_" + name].to(F64) * _scale(s["exp_" + name].t().to(torch.int64) - 127)[:, :, None]
        held[to] = torch.round(y / step) * step * scale
        out.append(held[back])
        codes.append(code)
    return (*out, *codes)


def _exact_attend(s):
    case = s["case"]
    lq, lk = _lengths(case)
    h, hk, d, cap = case["heads"], case["kv_heads"], case["head_dim"], case["k_hi"]
    grp = h // hk
    cq = s["cu_q"].tolist()
    o = torch.zeros(s["q"].shape, dtype=F64, device="cuda")
    lse = torch.full((h, s["q"].shape[0]), -math.inf, dtype=F64, device="cuda")
    for i in range(case["seqs"]):
        a, b = lq[i], lk[i]
        rows, cols = slice(cq[i], cq[i] + a), slice(i * cap, i * cap + b)
        hidden = None
        if case["causal"]:
            last = torch.arange(b - a, b, device="cuda")     # the last key that each query sees
            hidden = torch.arange(b, device="cuda")[None, :] > last[:, None]
        for j in range(hk):
            k, v = (s["cache_" + t][cols, j].to(F64) * _scale(s["exp_" + t][j, cols].to(torch.int64) - 127)[:, None] for t in ("k", "v"))
            for g in range(j * grp, (j + 1) * grp):
                sc = torch.mm(s["q"][rows, g].to(F64), k.t()) / math.sqrt(d)
                if hidden is not None:
                    sc = torch.where(hidden, -math.inf, sc)
                z = torch.logsumexp(sc, 1)
                p = torch.where(torch.isfinite(z)[:, None], torch.exp(sc - z[:, None]), 0.0)
                lse[g, rows] = z
                o[rows, g] = torch.mm(p, v)
    return o, lse


def _exact_gated(s):
    case = s["case"]
    n, act = case["n"], case["act"]
    x, w = s["x"].to(F64), s["w"].to(F64)
    bias = s["bias"].to(F64) if s["bias"] is not None else torch.zeros(2 * n, dtype=F64, device="cuda")
    z, u = torch.mm(x, w[:n].t()) + bias[:n], torch.mm(x, w[n:].t()) + bias[n:]
    if act == "none":
        a, slope = z, torch.ones_like(z)
    elif act == "relu":
        a, slope = torch.where(z > 0, z, 0 * z), torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
    elif act == "gelu":
        upto = torch.special.erfc(-z / math.sqrt(2.0)) / 2     # normal distribution function
        a, slope = z * upto, upto + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    else:
        sg = torch.sigmoid(z)
        a, slope = z * sg, sg + z * sg * torch.sigmoid(-z)
    if not case["train"]:
        return a * u
    dy = s["dy"].to(F64)
    dg, du = dy * u * slope, dy * a
    out = (a * u, torch.mm(dg, w[:n]) + torch.mm(du, w[n:]), torch.cat((torch.mm(dg.t(), x), torch.mm(du.t(), x))))
    return out + ((torch.cat((dg.sum(0), du.sum(0))),) if case["bias"] else ())
