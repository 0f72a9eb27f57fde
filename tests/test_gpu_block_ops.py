"""Rotary positions with head norms, the gated map, and the 8-bit cache with the attention that reads it, on the GPU
against their float64 definitions, within bounds derived from the types (tests/block_ref.py)."""
import ctypes as C
import math

import pytest
import torch

import block_ref as ref
import dense_ref
from dense_ref import check
from paper_2506_12541_amd import _lib, dense

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF, "f32": F32}


def gen(seed):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype).cuda()


def cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- rotary positions ----

def positions(g, rows, axes, reach, whole):
    if whole:
        t = torch.randint(0, reach, (rows, axes), generator=g, dtype=torch.int32)
    else:
        t = (torch.rand(rows, axes, generator=g) - 0.5) * reach
    return (t[:, 0].contiguous() if axes == 1 else t).cuda()


def check_rotary(g, dtype, rows, heads, kv, d, rot, norm, inter, axes=1, reach=5000, whole=True, mag=1.0, train=True):
    dt = DT[dtype]
    q, k = normal(g, rows, heads, d, dtype=dt, scale=1.3), normal(g, rows, kv, d, dtype=dt, scale=0.7)
    gq, gk = (normal(g, d, scale=0.2, shift=1.0) for _ in range(2)) if norm else (None, None)
    dq, dk = normal(g, rows, heads, d, dtype=dt), normal(g, rows, kv, d, dtype=dt)
    at = positions(g, rows, axes, reach, whole)
    freq, _ = dense.rotary_frequencies(rot, axes=axes)
    how = dict(gain_q=gq, gain_k=gk, eps=1e-5, interleaved=inter, magnitude=mag)
    yq, yk = dense.rotary_forward(q, k, at, freq, **how)
    got = dense.rotary_backward(dq, dk, at, freq, q=q, k=k, **how) if train else None
    for x, gain, dy, y, dx, dg in ((q, gq, dq, yq, "dq", "dgain_q"), (k, gk, dk, yk, "dk", "dgain_k")):
        want = ref.rotary(x.cpu(), at.cpu(), freq.cpu(), None if gain is None else gain.cpu(), 1e-5, inter, mag,
                          dy.cpu() if train else None)
        check("y", y, *want["y"])
        if train:
            check(dx, got[dx], *want["dx"])
            if gain is None:
                assert got[dg] is None
            else:
                check(dg, got[dg], *want["dgain"])


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,kv,d,rot", [(1, 1, 1, 2, 2), (3, 2, 1, 32, 32), (5, 4, 2, 64, 64), (33, 32, 8, 128, 128),
                                                 (7, 3, 3, 80, 20), (70, 8, 8, 64, 48), (9, 5, 1, 33, 6), (2, 1, 1, 256, 256),
                                                 (130, 2, 2, 34, 34), (4, 7, 1, 256, 2), (11, 3, 2, 96, 94), (6, 2, 1, 255, 130)])
def test_rotary(dtype, inter, norm, rows, heads, kv, d, rot):
    check_rotary(gen(rows + d + rot), dtype, rows, heads, kv, d, rot, norm, inter)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_axes_magnitude_and_far_positions(dtype):
    check_rotary(gen(1), dtype, 50, 4, 2, 64, 48, True, False, axes=3, reach=30, whole=False, mag=1.3)
    check_rotary(gen(2), dtype, 50, 4, 2, 64, 40, True, True, axes=4, reach=30, whole=True)
    check_rotary(gen(3), dtype, 50, 2, 2, 32, 32, False, True, axes=2, reach=1000, whole=False, mag=0.5)
    check_rotary(gen(4), dtype, 300, 2, 1, 64, 64, True, False, reach=(1 << 31) - 1)
    check_rotary(gen(5), dtype, 300, 2, 1, 64, 64, False, True, reach=1 << 24, whole=False)


def test_rotary_many_rows():
    check_rotary(gen(6), "bf16", 20000, 4, 4, 32, 32, True, False)
    check_rotary(gen(7), "f32", 6000, 3, 1, 40, 20, True, True)
    check_rotary(gen(8), "bf16", 9000, 40, 8, 128, 128, False, False, train=False)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rows,kv,d,dtype", [(4096, 46508, 2, "bf16"), (131072, 1025, 2, "f32"), (66000, 2200, 4, "bf16")])
def test_rotary_many_more_key_heads_than_query_heads(rows, kv, d, dtype, inter):
    """Keys beside one query head, against the same keys as queries: rows are shared out otherwise, each head's numbers
    are the same."""
    g, dt = torch.Generator("cuda").manual_seed(rows), DT[dtype]
    q, k = (torch.randn(rows, h, d, generator=g, device="cuda", dtype=dt) for h in (1, kv))
    at = torch.randint(0, 1 << 20, (rows,), generator=g, device="cuda", dtype=torch.int32)
    freq, _ = dense.rotary_frequencies(d)
    gain = torch.linspace(0.5, 1.5, d, device="cuda")
    how = dict(eps=1e-5, interleaved=inter)
    yq, yk = dense.rotary_forward(q, k, at, freq, gain_q=gain, gain_k=gain, **how)
    assert torch.equal(yk, dense.rotary_forward(k, None, at, freq, gain_q=gain, **how)[0])
    assert torch.equal(yq, dense.rotary_forward(q, None, at, freq, gain_q=gain, **how)[0])
    # some heads against the definition
    some = torch.tensor([0, 1, kv // 2, kv - 1])
    last = torch.arange(rows - 300, rows)
    check("y", yk[last][:, some], *ref.rotary(k[last][:, some].cpu(), at[last].cpu(), freq.cpu(), gain.cpu(), 1e-5, inter, 1.0)["y"])
    got = dense.rotary_backward(yq, yk, at, freq, q=q, k=k, gain_q=gain, gain_k=gain, **how)
    assert torch.equal(got["dk"], dense.rotary_backward(yk, None, at, freq, q=k, gain_q=gain, **how)["dq"])


# ---- gated map ----

def check_gated(g, dtype, m, k, n, act, bias, train=True):
    dt = DT[dtype]
    x, w = normal(g, m, k, dtype=dt), normal(g, 2 * n, k, dtype=dt, scale=1 / math.sqrt(k))
    b = normal(g, 2 * n, dtype=dt) if bias else None
    dy = normal(g, m, n, dtype=dt) if train else None
    want = ref.gated(x.cpu(), w.cpu(), None if b is None else b.cpu(), act, None if dy is None else dy.cpu())
    y, pre = dense.gated_forward(x, w, b, act=act, save_pre=train)
    got = dict(y=y)
    if train:
        got.update(dense.gated_backward(x, w, dy, pre, act=act, bias=True))
    for name, (value, bound) in want.items():
        check(name, got[name], value, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("bias", [False, True])
def test_gated_activations(dtype, act, bias):
    check_gated(gen(2), dtype, 70, 96, 132, act, bias)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 64, 64), (2, 512, 40), (5, 33, 17), (16, 1024, 256), (17, 72, 200),
                                   (48, 2048, 512), (64, 64, 64), (65, 31, 129), (100, 515, 1029), (128, 128, 128),
                                   (130, 200, 264), (256, 256, 256), (300, 513, 257), (515, 40, 1000), (1000, 1, 3),
                                   (2000, 256, 72), (2048, 320, 520), (33, 1000, 15), (40, 4100, 100)])
def test_gated_shapes(dtype, m, k, n):
    check_gated(gen(m + k + n), dtype, m, k, n, "gelu" if m % 2 else "silu", n % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gated_large_tiles(dtype):
    check_gated(gen(3), dtype, 4100, 192, 1160, "silu", True)
    check_gated(gen(4), dtype, 4096, 256, 2048, "gelu", False, train=False)


@pytest.mark.parametrize("m,k,n", [(700, 1101, 5505), (5001, 1500, 301)])
def test_gated_float32_tiles_of_long_contractions(m, k, n):
    """128 x 128 tiles, which very long and narrow products take as well, and 128 x 64 tiles, none by planes."""
    check_gated(gen(m), "f32", m, k, n, "silu", True)


# ---- 8-bit cache ----

def check_cache(g, dtype, lens, cap, used, kv, d, tail=0, k=None, v=None):
    dt = DT[dtype]
    rows, total = sum(lens) + tail, sum(cap) + tail
    k = normal(g, rows, kv, d, dtype=dt, scale=2.0) if k is None else k
    v = normal(g, rows, kv, d, dtype=dt, scale=0.1) if v is None else v
    cache = dense.cache_alloc(total, kv, d)
    g8 = torch.randint(0, 255, (4, total, kv, d), generator=g, dtype=torch.uint8).cuda()
    cache.k.view(torch.uint8).copy_(g8[0]), cache.v.view(torch.uint8).copy_(g8[1])
    cache.k_exp.copy_(g8[2, :, :, 0].t()), cache.v_exp.copy_(g8[3, :, :, 0].t())
    before = [t.view(torch.uint8).cpu().clone() for t in cache]
    cu_q, cu_k, used_k = cu(lens), cu(cap), ints(used)
    dense.cache_write(cache, k, v, cu_q, cu_k, used_k)
    kr, vr = dense.cache_read(cache, rows, cu_q, cu_k, used_k, dtype=dt)
    assert kr.dtype == dt
    after = [t.view(torch.uint8).cpu() for t in cache]
    for x, back, byte, code, was_byte, was_code in ((k, kr, after[0], after[2], before[0], before[2]),
                                                    (v, vr, after[1], after[3], before[1], before[3])):
        want, codes = ref.quantise(x)
        kept = torch.ones(total, dtype=torch.bool)
        src, cq, ck = torch.full((rows,), -1), cu_q.tolist(), cu_k.tolist()
        for s, n in enumerate(lens):
            for i in range(n):
                at = used[s] - n + i
                if at >= 0:
                    src[cq[s] + i] = ck[s] + at
                    kept[ck[s] + at] = False
        on = src >= 0
        assert torch.equal(code[:, src[on]], codes[:, on])
        assert torch.equal(byte[kept], was_byte[kept]) and torch.equal(code[:, kept], was_code[:, kept])
        want[~on] = 0
        back = back.cpu().double()
        assert torch.equal(back.isnan(), want.isnan())
        assert torch.equal(back[~want.isnan()], want[~want.isnan()])
        stored = byte[src[on]].view(torch.float8_e4m3fn).double() * 2.0 ** (codes[:, on].t().double() - 127)[..., None]
        assert torch.equal(stored.isnan(), want[on].isnan())
        assert torch.equal(stored[~stored.isnan()], want[on][~stored.isnan()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,d", [(1, 32), (8, 128), (3, 64), (5, 128)])
def test_cache_write_and_read(dtype, kv, d):
    check_cache(gen(kv + d), dtype, [1, 0, 7, 64, 3, 5], [4, 9, 7, 100, 8, 3], [1, 5, 7, 80, 2, 3], kv, d, tail=3)
    check_cache(gen(kv), dtype, [1] * 90, [5] * 90, [1 + i % 5 for i in range(90)], kv, d)
    check_cache(gen(kv), dtype, [1000, 600], [1500, 600], [1400, 600], kv, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_rounding(dtype):
    """Every bf16 magnitude: ties, subnormals, the borders of the scale, values past its range, not finite ones."""
    bits = torch.arange(1 << 15, dtype=torch.int32)
    x = (bits << 16).view(F32)                           # all positive bf16 numbers, infinity and NaN
    g = gen(3)
    sign = torch.where(torch.rand(x.shape, generator=g) < 0.5, -1.0, 1.0)
    # each beside one value that sets the scale (none, its binade, far above), in heads of 32
    d, groups = 32, []
    for top in (0.0, 1.0, 1.75, 448.0, 449.0, 2.0 ** -60, 2.0 ** 70):
        t = (x * sign)[torch.randperm(x.numel(), generator=g)].view(-1, d - 1 + 1).clone()
        if top:
            t[:, 0] = top
            t = torch.where(t.abs() <= top, t, t.sign())  # the rest below it
        groups.append(t)
    for i in (0, 1, 2):
        one = torch.zeros(x.numel(), d)                   # one value alone
        one[:, i] = x * sign
        groups.append(one[:: 1 + i])
    t = torch.cat(groups).view(-1, 1, d)
    t = torch.cat((t, torch.zeros(1, 1, d), torch.full((1, 1, d), math.nan))).to(DT[dtype]).cuda()
    n = t.shape[0]
    check_cache(g, dtype, [n], [n], [n], 1, d, k=t, v=-t)


def check_cache_attention(g, dtype, lq, cap, used, heads, kv, d, causal, tail=0, scale=0.0, amp=1.3):
    dt = DT[dtype]
    cu_q, cu_k, used_k = cu(lq), cu(cap), None if used is None else ints(used)
    tq, tk = sum(lq) + tail, sum(cap) + tail
    q = normal(g, tq, heads, d, dtype=dt, scale=amp)
    k, v = normal(g, tk, kv, d, scale=amp), normal(g, tk, kv, d) * torch.exp2(normal(g, 1, kv, 1).round())
    cache = dense.cache_alloc(tk, kv, d)
    one = cu([tk])
    dense.cache_write(cache, k, v, one, one, ints([tk]))
    kd, vd = dense.cache_read(cache, tk, one, one, ints([tk]), dtype=F32)
    assert torch.equal(kd.cpu().double(), ref.quantise(k)[0]) and torch.equal(vd.cpu().double(), ref.quantise(v)[0])
    for s, c in enumerate(cap):        # rows that are not in use hold NaN
        if used is not None:
            rows = slice(int(cu_k[s]) + used[s], int(cu_k[s]) + c)
            for t in (cache.k, cache.v):
                t.view(torch.uint8)[rows] = 0x7f
    want = dense_ref.attention(q, kd, vd, cu_q, cu_k, used, causal, scale or None)
    o, lse = dense.cache_attention_forward(q, cache, cu_q, cu_k, used_k, causal=causal, softmax_scale=scale)
    # float32 queries and probabilities enter as three parts, which triples the terms of each sum
    more = 3 if dtype == "f32" else 1
    check("o", o, want["o"][0], more * want["o"][1])
    check("lse", lse, want["lse"][0], more * want["lse"][1])


@pytest.mark.parametrize("heads,kv,d", [(8, 2, 128), (4, 4, 64), (5, 1, 32), (32, 8, 128)])
def test_cache_attention_steps_round_once(heads, kv, d):
    """bf16 outputs of few rows: rounded once. Probabilities enter their product as two bf16 parts, within 2^-16 of
    themselves, which doubles the terms of each sum; nothing else is off by more than float32 sums are."""
    g = gen(14)
    for lq, cap, used in (([1] * 6, [1024] * 6, [1, 1024, 0, 700, 257, 64]), ([2, 17], [5000, 3000], [4999, 2049]), ([1], [9000], [8999])):
        q, total = normal(g, sum(lq), heads, d, dtype=BF), sum(cap)
        k, v = normal(g, total, kv, d), normal(g, total, kv, d) * torch.exp2(normal(g, total, kv, 1).round())
        cache, one, cu_q, cu_k = dense.cache_alloc(total, kv, d), cu([total]), cu(lq), cu(cap)
        dense.cache_write(cache, k, v, one, one)
        kd, vd = dense.cache_read(cache, total, one, one, dtype=F32)
        o, _ = dense.cache_attention_forward(q, cache, cu_q, cu_k, ints(used), causal=True)
        want, e = dense_ref.attention(q.float(), kd, vd, cu_q, cu_k, used, True)["o"]
        whole = dense_ref.attention(q.float(), kd, vd.abs(), cu_q, cu_k, used, True)["o"][0]      # sum of p |v|
        e = 2 * e + 2.0 ** -16 * whole
        check("o", o, want, e + dense_ref.HALF[BF] * (want.abs() + e))


LENS = [1, 0, 7, 64, 65, 130, 33, 200]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 32), (4, 4, 64), (2, 2, 128), (8, 2, 64), (6, 2, 32), (8, 1, 128)])
def test_cache_attention_packed(dtype, causal, heads, kv, d):
    check_cache_attention(gen(heads + d), dtype, LENS, LENS, None, heads, kv, d, causal, tail=5)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_attention_other_key_lengths(dtype, causal):
    """Fewer keys than queries (causal: rows that see nothing), none, and more."""
    check_cache_attention(gen(6), dtype, [5, 70, 3, 64, 1, 0], [3, 20, 0, 300, 1, 9], None, 4, 2, 64, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 64), (5, 1, 32), (32, 1, 64)])
def test_cache_attention_steps(dtype, heads, kv, d):
    """Single and few tokens against caches that are partly filled, empty, and long enough to be split."""
    cap, used = [1024] * 6, [1, 1024, 0, 700, 257, 64]
    check_cache_attention(gen(7), dtype, [1] * 6, cap, used, heads, kv, d, True)
    check_cache_attention(gen(8), dtype, [3, 1, 4, 0, 2, 9], cap, used, heads, kv, d, True)
    check_cache_attention(gen(9), dtype, [2, 17], [5000, 3000], [4999, 2049], heads, kv, d, True, tail=3)
    check_cache_attention(gen(9), dtype, [3], [900], [555], heads, kv, d, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_attention_many_sequences_and_long_ones(dtype):
    lens = [(i * 7) % 23 for i in range(300)]
    check_cache_attention(gen(11), dtype, lens, [24] * 300, [i % 25 for i in range(300)], 4, 2, 64, True, tail=70)
    check_cache_attention(gen(11), dtype, [1] * 300, [64] * 300, [i % 65 for i in range(300)], 2, 2, 32, True)
    check_cache_attention(gen(12), dtype, [700], [1500], [1300], 4, 1, 64, True)
    check_cache_attention(gen(13), dtype, [1], [9000], [8999], 2, 1, 128, True, scale=0.3)


# ---- rotary: calls that the documentation allows ----

def rotary_args(g, dt, rows, heads, kv, d, rot, norm=True):
    q, k = normal(g, rows, heads, d, dtype=dt), normal(g, rows, kv, d, dtype=dt)
    dq, dk = normal(g, rows, heads, d, dtype=dt), normal(g, rows, kv, d, dtype=dt)
    at = torch.randint(0, 3000, (rows,), generator=g, dtype=torch.int32).cuda()
    freq, _ = dense.rotary_frequencies(rot)
    how = dict(gain_q=normal(g, d, shift=1.0), gain_k=normal(g, d, shift=1.0)) if norm else {}
    return q, k, dq, dk, at, freq, how


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(64, 48), (30, 14)])
def test_rotary_views_in_place_and_given_outputs(dtype, inter, d, rot):
    """Views of a fused projection, outputs in views, and outputs on top of inputs give the packed tensors' bits."""
    g, dt = gen(d), DT[dtype]
    q, k, dq, dk, at, freq, how = rotary_args(g, dt, 37, 4, 2, d, rot)
    how["interleaved"] = inter
    yq, yk = dense.rotary_forward(q, k, at, freq, **how)
    a = dense.rotary_backward(dq, dk, at, freq, q=q, k=k, **how)
    fused, dfused = (torch.full((37, 9, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
    fused[:, :4], fused[:, 4:6] = q, k
    vq, vk = fused[:, :4], fused[:, 4:6]
    oq, ok = dense.rotary_forward(vq, vk, at, freq, y_q=dfused[:, :4], y_k=dfused[:, 4:6], **how)
    assert torch.equal(oq, yq) and torch.equal(ok, yk) and (dfused[:, 6:] == 7).all()
    b = dense.rotary_backward(dq, dk, at, freq, q=vq, k=vk, dq=dfused[:, :4], dk=dfused[:, 4:6], **how)
    assert torch.equal(b["dq"], a["dq"]) and torch.equal(b["dk"], a["dk"]) and (dfused[:, 6:] == 7).all()
    assert torch.equal(b["dgain_q"], a["dgain_q"]) and torch.equal(b["dgain_k"], a["dgain_k"])
    eq, ek = dq.clone(), dk.clone()                    # gradients on top of the given ones
    c = dense.rotary_backward(eq, ek, at, freq, q=q, k=k, dq=eq, dk=ek, **how)
    assert torch.equal(eq, a["dq"]) and torch.equal(ek, a["dk"]) and torch.equal(c["dgain_q"], a["dgain_q"])
    dense.rotary_forward(vq, vk, at, freq, y_q=vq, y_k=vk, **how)       # in place, in views
    assert torch.equal(vq, yq) and torch.equal(vk, yk) and (fused[:, 6:] == 7).all()
    only, none = dense.rotary_forward(q, None, at, freq, gain_q=how["gain_q"], interleaved=inter)
    assert torch.equal(only, yq) and none is None
    one = dense.rotary_backward(dq, None, at, freq, q=q, gain_q=how["gain_q"], interleaved=inter)
    assert torch.equal(one["dq"], a["dq"]) and one["dk"] is None and one["dgain_k"] is None


def test_rotary_broadcast_and_head_major_inputs():
    g = gen(3)
    q, k, dq, dk, at, freq, how = rotary_args(g, BF, 21, 4, 2, 64, 64)
    for x in (q[:, :1].expand(21, 4, 64), q[:1].expand(21, 4, 64), q.transpose(0, 1).contiguous().transpose(0, 1)):
        y, _ = dense.rotary_forward(x, k, at, freq, **how)
        z, _ = dense.rotary_forward(x.contiguous(), k, at, freq, **how)
        assert torch.equal(y, z)
        a = dense.rotary_backward(x, dk, at, freq, q=q, k=k, **how)      # as the gradient too
        b = dense.rotary_backward(x.contiguous(), dk, at, freq, q=q, k=k, **how)
        assert torch.equal(a["dq"], b["dq"]) and torch.equal(a["dgain_q"], b["dgain_q"])


def test_rotary_turned_back_is_where_it_was():
    """Without a norm the backward turns back: a length times magnitude squared."""
    g = gen(4)
    q, k, _, _, at, freq, _ = rotary_args(g, F32, 50, 2, 1, 64, 32, norm=False)
    y, yk = dense.rotary_forward(q, k, at, freq, magnitude=2.0)
    back = dense.rotary_backward(y, yk, at, freq, magnitude=2.0)
    assert torch.allclose(back["dq"][..., :32], 4 * q[..., :32], atol=1e-5) and torch.equal(back["dq"][..., 32:], q[..., 32:])
    at64 = at.to(torch.int32)
    neg, _ = dense.rotary_forward(y, None, -at64, freq, magnitude=0.5)
    assert torch.allclose(neg[..., :32], q[..., :32], atol=1e-5)


def test_rotary_no_rows_and_values_that_are_not_finite():
    g = gen(5)
    q, k, dq, dk, at, freq, how = rotary_args(g, F32, 6, 2, 1, 64, 32)
    e = dense.rotary_forward(q[:0], k[:0], at[:0], freq, **how)
    b = dense.rotary_backward(dq[:0], dk[:0], at[:0], freq, q=q[:0], k=k[:0], **how)
    assert e[0].shape == (0, 2, 64) and b["dq"].shape == (0, 2, 64) and not b["dgain_q"].any() and not b["dgain_k"].any()
    want, _ = dense.rotary_forward(q, k, at, freq, **how)
    x = q.clone()
    x[1, 0, 5], x[3, 1, 40] = math.nan, math.inf
    y, _ = dense.rotary_forward(x, k, at, freq, **how)
    assert y[1, 0].isnan().all() and y[3, 1].isnan().any()         # their own heads, and no others
    keep = torch.ones(6, 2, dtype=torch.bool, device="cuda")
    keep[1, 0] = keep[3, 1] = False
    assert torch.equal(y[keep], want[keep])
    pos = at.float()
    pos[2], pos[4] = math.inf, math.nan
    y, _ = dense.rotary_forward(q, k, pos, freq, **how)
    assert y[[2, 4]][..., :32].isnan().all() and torch.equal(y[[2, 4]][..., 32:], want[[2, 4]][..., 32:])
    assert torch.equal(y[[0, 1, 3, 5]], want[[0, 1, 3, 5]])
    zero = torch.zeros_like(q)
    y, _ = dense.rotary_forward(zero, k, at, freq, **how)
    z = dense.rotary_backward(dq, dk, at, freq, q=zero, k=k, **how)
    assert not y.any() and z["dq"].isfinite().all() and not z["dgain_q"].any()


def test_rotary_long_tensors():
    """Offsets past 32 bits: the last rows of a tensor of more than 2^32 elements, in place."""
    rows, heads, d = (1 << 32) // (32 * 128) + 3, 32, 128
    x = torch.zeros(rows, heads, d, dtype=BF, device="cuda")
    g = gen(6)
    last = normal(g, 5, heads, d, dtype=BF)
    x[-5:] = last
    at = torch.arange(rows, dtype=torch.int32, device="cuda")
    freq, _ = dense.rotary_frequencies(128)
    want, _ = dense.rotary_forward(last, None, at[-5:].contiguous(), freq)
    dense.rotary_forward(x, None, at, freq, y_q=x)
    assert torch.equal(x[-5:], want) and not x[:-5:1000].any()


# ---- gated map: calls that the documentation allows ----

@pytest.mark.parametrize("m,k,n", [(800, 300, 700), (3586, 515, 1029), (1000, 2100, 600), (2001, 257, 1500)])
def test_gated_float32_planes(m, k, n):
    """Sizes at which float32 products run on operands split before."""
    check_gated(gen(m), "f32", m, k, n, "silu", True)


@pytest.mark.parametrize("m,k,n", [(1, 1024, 4096), (4, 1027, 4099), (5, 70001, 61), (8, 2052, 2050), (9, 4097, 1031),
                                   (16, 1100, 4000), (1, 1024, 8192), (3, 4099, 2051), (8, 70001, 121), (6, 1501, 6001)])
def test_gated_float32_few_rows(m, k, n):
    """Sizes at which float32 gradients of few rows read the weight, and write its gradient, once."""
    check_gated(gen(m), "f32", m, k, n, "silu" if m % 2 else "gelu", True)


def test_gated_float32_few_rows_strides_parts_and_values_that_are_not_finite():
    g, (m, k, n) = gen(6), (7, 1030, 8200)
    x, w, dy = normal(g, m, k), normal(g, 2 * n, k, scale=0.1), normal(g, m, n)
    x[1, k - 1], w[n, 3] = math.inf, 0.0
    dy[3, 5], dy[4, 7] = math.nan, math.inf
    _, pre = dense.gated_forward(x, w, act="none", save_pre=True)
    a = dense.gated_backward(x, w, dy, pre, act="none", bias=True)
    assert a["dx"][3].isnan().all() and not a["dx"][4].isfinite().any() and not a["dx"][1].isfinite().any()
    rest = [0, 2, 5, 6]
    some = dense.gated_backward(x[rest], w, dy[rest], pre[rest], act="none")["dx"]
    assert some.isfinite().all() and torch.equal(a["dx"][rest], some)
    assert not a["dw"].isfinite().any()      # every pre of row 1 is infinite, so its part of each dw is not finite
    rest = [0, 2, 3, 4, 5, 6]
    bad = ~dense.gated_backward(x[rest], w, dy[rest], pre[rest], act="none")["dw"].isfinite()
    assert bad[[5, 7, n + 5, n + 7]].all() and not bad.index_fill(0, torch.tensor([5, 7, n + 5, n + 7], device="cuda"), False).any()
    wide_x, wide_w, wide_dy = (torch.full((t.shape[0], t.shape[1] + 3), math.nan, device="cuda") for t in (x, w, dy))
    for wide, t in ((wide_x, x), (wide_w, w), (wide_dy, dy)):
        wide[:, :t.shape[1]] = t
    b = dense.gated_backward(wide_x[:, :k], wide_w[:, :k], wide_dy[:, :n], pre, act="none", bias=True)
    for name in a:
        assert torch.allclose(a[name], b[name], rtol=0, atol=0, equal_nan=True)
    for kw in (dict(need_dx=False), dict(need_dw=False), dict(need_dx=False, need_dw=False, bias=True)):
        part = dense.gated_backward(x, w, dy, pre, act="none", **kw)
        for name in ("dx", "dw", "db"):
            assert part[name] is None or torch.allclose(part[name], a[name], rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(200, 136, 132), (900, 264, 520)])
def test_gated_strides_and_parts(dtype, m, k, n):
    """Operands whose rows lie apart, aligned to 16 bytes and not; gradients that are not asked for."""
    g, dt = gen(5), DT[dtype]
    x, w, dy = normal(g, m, k, dtype=dt), normal(g, 2 * n, k, dtype=dt, scale=0.1), normal(g, m, n, dtype=dt)
    y, pre = dense.gated_forward(x, w, act="gelu", save_pre=True)
    a = dense.gated_backward(x, w, dy, pre, act="gelu", bias=True)

    def apart(t, more):
        buf = torch.full((t.shape[0], t.shape[1] + more), float("nan"), dtype=dt, device="cuda")
        buf[:, :t.shape[1]] = t
        return buf[:, :t.shape[1]]
    for more in (8, 3):
        ys, ps = dense.gated_forward(apart(x, more), apart(w, more), act="gelu", save_pre=True)
        b = dense.gated_backward(apart(x, more), apart(w, more), apart(dy, more), ps, act="gelu", bias=True)
        for u, v in ((y, ys), (pre, ps), *((a[name], b[name]) for name in a)):
            assert torch.allclose(u.float(), v.float(), rtol=2 * dense_ref.HALF[dt], atol=2e-3)
    plain, none = dense.gated_forward(x, w, act="gelu")
    assert torch.equal(plain, y) and none is None
    y3, p3 = dense.gated_forward(x.view(4, m // 4, k), w, act="gelu", save_pre=True)
    assert torch.equal(y3.view(m, n), y) and p3.shape == (4, m // 4, 2 * n)
    for kw in (dict(need_dx=False), dict(need_dw=False), dict(need_dx=False, need_dw=False, bias=True), dict(bias=True, need_dw=False)):
        some = dense.gated_backward(x, w, dy, pre, act="gelu", **kw)
        assert (some["dx"] is None) == (not kw.get("need_dx", True)) and (some["dw"] is None) == (not kw.get("need_dw", True))
        for name in ("dx", "dw", "db"):
            assert some[name] is None or torch.equal(some[name], a[name])


@pytest.mark.parametrize("m,k,n", [(3, 515, 40), (16, 1025, 33), (1, 4097, 70), (30, 1001, 129), (64, 257, 100), (7, 129, 9)])
def test_odd_contractions_of_few_rows(m, k, n):
    """Rows of an odd length, that begin inside 4-byte words in turn; operands that begin inside one."""
    check_gated(gen(m), "bf16", m, k, n, "silu", True)
    g = gen(m + 1)
    x, w = normal(g, m, k + 2, dtype=BF), normal(g, 2 * n, k + 2, dtype=BF, scale=0.1)
    for a, b in ((0, 0), (0, 1), (1, 0), (1, 1), (2, 1)):
        xs, ws = x[:, a:a + k], w[:, b:b + k]
        y, pre = dense.gated_forward(xs, ws, save_pre=True)
        want, want_pre = dense.gated_forward(xs.contiguous(), ws.contiguous(), save_pre=True)
        assert torch.equal(y, want) and torch.equal(pre, want_pre)
        want = dense_ref.linear(xs.cpu(), ws.cpu(), None, None, "none")["y"]
        check("affine", dense.linear_forward(xs, ws)[0], *want)
        check("affine, whole rows", dense.linear_forward(xs.contiguous(), ws.contiguous())[0], *want)


@pytest.mark.parametrize("m,k,n", [(3000, 1031, 1100), (1100, 4100, 801), (20001, 67, 2501)])
def test_gated_rows_that_are_copied(m, k, n):
    """bf16 products of rows that do not begin on 16 bytes and are long enough to be copied, and of other strides."""
    check_gated(gen(m), "bf16", m, k, n, "silu", True)
    g = gen(9)
    x, w, dy = normal(g, m, k, dtype=BF), normal(g, 2 * n, k, dtype=BF, scale=0.1), normal(g, m, n, dtype=BF)
    y, pre = dense.gated_forward(x, w, act="gelu", save_pre=True)
    a = dense.gated_backward(x, w, dy, pre, act="gelu", bias=True)

    def apart(t, ld):
        buf = torch.full((t.shape[0], ld), float("nan"), dtype=BF, device="cuda")
        buf[:, :t.shape[1]] = t
        return buf[:, :t.shape[1]]
    for lx, lw in ((k + 13, k + 13), ((k + 15) // 8 * 8, (k + 15) // 8 * 8), (k + 1, (k + 15) // 8 * 8), ((k + 15) // 8 * 8, k + 3)):
        xs, ws = apart(x, lx), apart(w, lw)
        ys, ps = dense.gated_forward(xs, ws, act="gelu", save_pre=True)
        b = dense.gated_backward(xs, ws, apart(dy, n + 3), ps, act="gelu", bias=True)
        for u, v in ((y, ys), (pre, ps), *((a[name], b[name]) for name in a)):
            assert torch.allclose(u.float(), v.float(), rtol=2 * dense_ref.HALF[BF], atol=2e-3)
        for kw in (dict(need_dx=False), dict(need_dw=False)):
            some = dense.gated_backward(xs, ws, dy, ps, act="gelu", **kw)
            for name in ("dx", "dw"):
                assert some[name] is None or torch.equal(some[name], b[name])


@pytest.mark.parametrize("dtype,m,k,n", [("bf16", 3000, 1031, 1100), ("bf16", 1100, 4100, 801), ("bf16", 900, 264, 520), ("bf16", 3, 515, 40),
                                         ("bf16", 1, 64, 64), ("f32", 800, 300, 700), ("f32", 4, 1027, 4099), ("f32", 12, 1500, 6000),
                                         ("f32", 300, 136, 132), ("f32", 30, 70, 9)])
def test_gated_gradients_without_the_other_operand(dtype, m, k, n):
    """The C entry with NULL for what a gradient that is not formed would read: copied rows, tiles, planes, few rows."""
    lib, g, dt = _lib.load(), gen(m), DT[dtype]
    x, w = normal(g, m, k, dtype=dt), normal(g, 2 * n, k, dtype=dt, scale=1 / math.sqrt(k))
    dy = normal(g, m, n, dtype=dt)
    _, pre = dense.gated_forward(x, w, save_pre=True)
    want = dense.gated_backward(x, w, dy, pre, bias=True)
    p = _lib.bsa_gated_t(m=m, k=k, n=n, dtype=_lib.BSA_BF16 if dtype == "bf16" else _lib.BSA_F32, act=dense.ACTIVATIONS["silu"])
    need = C.c_size_t()
    assert lib.bsa_gated_sizes(C.byref(p), None, C.byref(need)) == 0
    for formed in (("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db")):
        ws = torch.full((need.value,), 255, dtype=torch.uint8, device="cuda")       # NaN in both types
        got = {name: torch.full_like(want[name], float("nan")) for name in formed}
        out = [got[name].data_ptr() if name in got else None for name in ("dx", "dw", "db")]
        assert lib.bsa_gated_backward(C.byref(p), x.data_ptr() if "dw" in got else None, w.data_ptr() if "dx" in got else None,
                                      pre.data_ptr(), dy.data_ptr(), *out, ws.data_ptr(), need.value,
                                      torch.cuda.current_stream().cuda_stream) == 0
        for name in got:
            assert torch.equal(got[name], want[name]), (formed, name)


def test_gated_refusals_after_calls_that_passed():
    """A call like one that was checked before is checked where anything differs; records keep nothing of the values."""
    x, w, b = (torch.randn(s, device="cuda") for s in ((6, 40), (2 * 24, 40), (2 * 24,)))
    for scale in (1.0, 2.0):                 # the same shapes again
        y, pre = dense.gated_forward(scale * x, w, b, save_pre=True)
        dy = torch.ones_like(y)
        want = ref.gated((scale * x).cpu(), w.cpu(), b.cpu(), "silu", dy.cpu())
        got = dict(y=y, **dense.gated_backward(scale * x, w, dy, pre, bias=True))
        for name, (value, bound) in want.items():
            check(name, got[name], value, bound)
    for kw in (dict(act="tanh"), dict(act=["silu"]), dict(bias=b[1:]), dict(bias=b.to(BF)), dict(bias=b.cpu()), dict(w=w[1:]),
               dict(w=w.t()), dict(x=x.to(BF)), dict(x=x[:, 1:]), dict(x=x.cpu()), dict(x=None)):
        with pytest.raises(ValueError):
            dense.gated_forward(**{**dict(x=x, w=w, bias=b), **kw})
    for kw in (dict(pre=None), dict(pre=pre[1:]), dict(pre=pre.t().contiguous().t()), dict(dy=dy[:, 1:]), dict(dy=dy.to(BF)),
               dict(dy=None), dict(act="tanh")):
        with pytest.raises(ValueError):
            dense.gated_backward(**{**dict(x=x, w=w, dy=dy, pre=pre), **kw})


def test_gated_no_rows_and_values_that_are_not_finite():
    w = torch.ones(80, 24, device="cuda", dtype=BF)
    e = torch.zeros(0, 24, device="cuda", dtype=BF)
    y, pre = dense.gated_forward(e, w, save_pre=True)
    got = dense.gated_backward(e, w, y, pre, bias=True)
    assert y.shape == (0, 40) and got["dx"].shape == (0, 24) and not got["dw"].any() and not got["db"].any()
    for dt in (BF, F32):
        for m, k, n in ((3, 24, 40), (200, 72, 40), (300, 100, 40), (900, 300, 600)):
            x = torch.ones(m, k, device="cuda", dtype=dt)
            x[1, k - 1], x[2, 0] = math.inf, math.nan
            w = torch.full((2 * n, k), 1 / 16, device="cuda", dtype=dt)
            y, pre = dense.gated_forward(x, w, act="none", save_pre=True)
            assert (y[0] == (k / 16) ** 2).all() if k < 256 or dt == F32 else True
            assert (y[1] == math.inf).all() and y[2].isnan().all() and torch.equal(y[3:], y[:1].expand(m - 3, n))
            assert (pre[1] == math.inf).all() and pre[2].isnan().all()
            g = dense.gated_backward(x, w, torch.ones_like(y), pre, act="none")
            assert g["dx"][3:].isfinite().all() and (g["dx"][1] == math.inf).all() and g["dx"][2].isnan().all()


def test_gated_float32_values_that_do_not_split():
    """The largest float32 values and small ones through operands split before."""
    big, (m, k, n) = torch.finfo(F32).max, (900, 300, 600)
    g = gen(8)
    x, w = normal(g, m, k), normal(g, 2 * n, k, scale=0.1)
    x[2] = 0
    x[2, 5] = big
    w[:, 5] = 0.5
    x[3] = 2.0 ** -120                       # its parts reach into the denormal numbers
    _, pre = dense.gated_forward(x, w, act="none", save_pre=True)
    want = x.double().cpu() @ w.double().cpu().t()
    assert (pre[2] == big / 2).all()
    size = x[3:].double().cpu().abs() @ w.double().cpu().abs().t()
    check("pre", pre[3:], want[3:], (k + 2) * dense_ref.F * size + 2.0 ** -140)
    x[4, 7] = -math.inf
    _, pre = dense.gated_forward(x, w, act="none", save_pre=True)
    assert torch.equal(pre[4], -torch.sign(w[:, 7]) * math.inf) and (pre[2] == big / 2).all()
    check("pre beside an infinity", pre[5:], want[5:], (k + 2) * dense_ref.F * size[2:] + 2.0 ** -140)


# ---- 8-bit cache: calls that the documentation allows ----

def filled(g, rows, kv, d, layout="rows", amp=1.3):
    cache = dense.cache_alloc(rows, kv, d)
    if layout == "heads":                    # a head's rows one behind another
        cache = dense.Cache(*(torch.zeros(kv, rows, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).transpose(0, 1)
                              for _ in range(2)), cache.k_exp, cache.v_exp)
    elif layout == "fused":                  # keys and values side by side, as one of several layers
        both = torch.zeros(3, rows, 2 * kv, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        cache = dense.Cache(both[1, :, :kv], both[1, :, kv:], cache.k_exp, cache.v_exp)
    k, v = normal(g, rows, kv, d, scale=amp), normal(g, rows, kv, d)
    one = cu([rows])
    dense.cache_write(cache, k, v, one, one)
    return cache, k, v


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("lq", [[1, 1, 1], [300, 40, 200]])
def test_cache_layouts(d, lq):
    """Head-major and fused caches, and views of a fused projection, give the packed tensors' bits."""
    cap, used = cu([500, 64, 900]), ints([400, 64, 333])
    n, outs = sum(lq), []
    for layout in ("rows", "heads", "fused"):
        g = gen(d)
        cache, _, _ = filled(g, 1464, 4, d, layout)
        qkv = normal(g, n, 16, d, dtype=BF)
        if layout == "rows":
            q, k, v = (t.contiguous() for t in (qkv[:, :8], qkv[:, 8:12], qkv[:, 12:]))
        else:
            q, k, v = qkv[:, :8], qkv[:, 8:12], qkv[:, 12:]
        cu_q = cu(lq)
        dense.cache_write(cache, k, v, cu_q, cap, used)
        o, lse = dense.cache_attention_forward(q, cache, cu_q, cap, used, causal=True)
        kr, vr = dense.cache_read(cache, 797, cu([400, 64, 333]), cap, used, dtype=F32)
        outs.append((o, lse, kr, vr, cache.k_exp, cache.v_exp))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))
    oo = torch.full((n, 16, d), 3.0, dtype=BF, device="cuda")[:, 3:11]
    ll = torch.zeros(8, n, device="cuda")
    o, lse = dense.cache_attention_forward(q, cache, cu_q, cap, used, causal=True, o=oo, lse=ll)
    assert o is oo and lse is ll and torch.equal(o, outs[0][0]) and torch.equal(lse, outs[0][1])


def test_cache_attention_is_packed_attention_of_what_the_cache_holds():
    g = gen(12)
    lens = [700, 0, 130, 1, 64]
    cache, _, _ = filled(g, sum(lens), 2, 64)
    q = normal(g, sum(lens), 8, 64, dtype=BF)
    c = cu(lens)
    k, v = dense.cache_read(cache, sum(lens), c, c)
    for causal in (False, True):
        o, lse = dense.cache_attention_forward(q, cache, c, c, causal=causal)
        p, want = dense.attention_forward(q, k, v, c, causal=causal)
        assert torch.allclose(lse, want, rtol=1e-5, atol=1e-5) and torch.allclose(o.float(), p.float(), rtol=2 ** -6, atol=2 ** -7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lq,lk", [(5, 200), (150, 180), (1, 70), (300, 300)])
def test_cache_attention_nan_behind_the_mask(dtype, lq, lk):
    """NaN in a key or value reaches the queries that see it, and no others."""
    g = gen(lq)
    cache, _, _ = filled(g, lk, 2, 64)
    q = normal(g, lq, 4, 64, dtype=DT[dtype])
    cq, ck = cu([lq]), cu([lk])
    want, wl = dense.cache_attention_forward(q, cache, cq, ck, causal=True)
    for which in ("k", "v"):
        for row in {lk - 1, lk - 2 if lq > 1 else lk - 1, lk - 1 - lq // 2}:
            for col in (0, 37):
                byte = getattr(cache, which).view(torch.uint8)
                keep = byte[row, 1, col].clone()
                byte[row, 1, col] = 0xff
                o, lse = dense.cache_attention_forward(q, cache, cq, ck, causal=True)
                byte[row, 1, col] = keep
                first = max(row - (lk - lq), 0)               # the first query that sees the row
                assert torch.equal(o[:first], want[:first]) and torch.equal(o[:, :2], want[:, :2])
                assert o[first:, 2:, col].isnan().all()
                assert torch.equal(lse[:2], wl[:2]) and torch.equal(lse[2:, :first], wl[2:, :first])


def test_cache_attention_rows_in_no_sequence_and_sharp_rows():
    g = gen(14)
    cache, _, _ = filled(g, 300, 1, 64, amp=8.0)             # scores with a wide range
    q = normal(g, 40, 2, 64, dtype=BF, scale=4.0)
    cq, ck, used = cu([3, 0, 20]), cu([100, 50, 140]), ints([77, 50, 140])
    o, lse = dense.cache_attention_forward(q, cache, cq, ck, used, causal=True)
    assert not o[23:].any() and (lse[:, 23:] == -math.inf).all() and o[:23].isfinite().all()
    oo, ll = torch.full_like(o, 5.0), torch.full_like(lse, 5.0)
    dense.cache_attention_forward(q, cache, cq, ck, used, causal=True, o=oo, lse=ll)
    assert (oo[23:] == 5).all() and (ll[:, 23:] == 5).all() and torch.equal(oo[:23], o[:23]) and torch.equal(ll[:, :23], lse[:, :23])
    k, v = dense.cache_read(cache, 300, cu([300]), cu([300]), dtype=F32)
    want = dense_ref.attention(q, k, v, cq, ck, [77, 50, 140], True)
    check("o", o, *want["o"])
    check("lse", lse, *want["lse"])


def test_cache_offsets_past_32_bits():
    rows, kv, d = 4400000, 8, 128                            # 4.5 GB of keys
    g = gen(15)
    cache = dense.cache_alloc(rows, kv, d)
    k, v, q = normal(g, 300, kv, d, dtype=BF), normal(g, 300, kv, d, dtype=BF), normal(g, 2, 8, d, dtype=BF)
    cq, ck, used = cu([0, 300]), ints([0, rows - 400, rows]), ints([0, 350])
    dense.cache_write(cache, k, v, cq, ck, used)
    small = dense.cache_alloc(400, kv, d)
    one, last = ints([0, 400]), ints([350])
    dense.cache_write(small, k, v, cu([300]), one, last)
    assert torch.equal(cache.k[-400:].view(torch.uint8), small.k.view(torch.uint8))
    assert torch.equal(cache.v_exp[:, -400:], small.v_exp) and not cache.k_exp[:, :-400].any()
    kr, vr = dense.cache_read(cache, 300, cq, ck, used)
    ks, vs = dense.cache_read(small, 300, cu([300]), one, last)
    assert torch.equal(kr, ks) and torch.equal(vr, vs) and ks.any()
    o, lse = dense.cache_attention_forward(q, cache, cu([0, 2]), ck, used, causal=True)
    p, want = dense.cache_attention_forward(q, small, cu([2]), one, last, causal=True)
    assert torch.allclose(lse, want, rtol=1e-5, atol=1e-5) and torch.allclose(o.float(), p.float(), rtol=2 ** -6, atol=2 ** -7)


# ---- streams, graphs, together ----

def test_calls_on_a_stream_with_work_queued_on_it():
    """A call on a given stream waits for what is queued there, and leaves the current stream alone."""
    g = gen(20)
    q, k, dq, dk, at, freq, how = rotary_args(g, BF, 64, 8, 2, 64, 64)
    w, x = normal(g, 256, 512, dtype=BF, scale=0.05), normal(g, 64, 512, dtype=BF)
    cache, _, _ = filled(g, 512, 2, 64)
    cq, ck, used = cu([32, 32]), cu([256, 256]), ints([200, 256])

    def run(q, k, x, stream=None):
        a, b = dense.rotary_forward(q, k, at, freq, stream=stream, **how)
        r = dense.rotary_backward(dq, dk, at, freq, q=q, k=k, stream=stream, **how)
        dense.cache_write(cache, b, k, cq, ck, used, stream=stream)
        o, lse = dense.cache_attention_forward(a, cache, cq, ck, used, causal=True, stream=stream)
        kr, vr = dense.cache_read(cache, 64, cq, ck, used, stream=stream)
        y, pre = dense.gated_forward(x, w, save_pre=True, stream=stream)
        d = dense.gated_backward(x, w, y, pre, stream=stream)
        return [a, b, r["dq"], r["dgain_k"], o, lse, kr, vr, y, d["dx"], d["dw"]]
    want = [t.clone() for t in run(q, k, x)]
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    late = [torch.zeros_like(t) for t in (q, k, x)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(10):
            big = big @ big
            big = big / big.abs().amax()
        for t, u in zip(late, (q, k, x)):
            t.copy_(u)
    got = run(*late, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_serving_step_in_a_graph():
    """A captured step (norms and rotation, cache, attention, gated map) whose lengths grow on the device, replayed several
    times with eager work between, against the same steps run eagerly."""
    g = gen(21)
    seqs, heads, kv, d, cap = 5, 8, 2, 64, 96
    c = heads * d
    wqkv = normal(g, (heads + 2 * kv) * d, c, dtype=BF, scale=c ** -0.5)
    wo, wg, wd = (normal(g, *s, dtype=BF, scale=c ** -0.5) for s in ((c, c), (2 * 256, c), (c, 256)))
    gq, gk = normal(g, d, scale=0.1, shift=1.0), normal(g, d, scale=0.1, shift=1.0)
    freq, mag = dense.rotary_frequencies(d, scaling="ramp", factor=2.0, trained=64)
    x0, start = normal(g, seqs, c, dtype=BF), ints([1, 17, 60, 64, 30])
    cq, ck = cu([1] * seqs), cu([cap] * seqs)

    def step(x, used, at, cache):
        qkv = dense.linear_forward(x, wqkv)[0].view(seqs, heads + 2 * kv, d)
        q, k = dense.rotary_forward(qkv[:, :heads], qkv[:, heads:heads + kv], at, freq, gain_q=gq, gain_k=gk, magnitude=mag)
        dense.cache_write(cache, k, qkv[:, heads + kv:], cq, ck, used)
        o, lse = dense.cache_attention_forward(q, cache, cq, ck, used, causal=True)
        h, _ = dense.linear_forward(o.view(seqs, c), wo, residual=x)
        a, _ = dense.gated_forward(h, wg)
        y, _ = dense.linear_forward(a, wd, residual=h)
        return y, lse

    def fresh():
        cache, _, _ = filled(gen(22), cap * seqs, kv, d)
        return x0.clone(), start.clone(), start - 1, cache
    x, used, at, cache = fresh()
    eager = []
    for _ in range(6):
        y, lse = step(x, used, at, cache)
        eager.append((y.clone(), lse.clone(), [t.view(torch.uint8).clone() for t in cache]))
        x.copy_(y), used.add_(1), at.add_(1)
    x, used, at, cache = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, used, at, dense.Cache(*(t.clone() for t in cache)))      # warm up on a copy
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, lse = step(x, used, at, cache)
    for want_y, want_lse, want_cache in eager:
        graph.replay()
        torch.randn(1000, device="cuda").sum()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(lse, want_lse)
        assert all(torch.equal(t.view(torch.uint8), u) for t, u in zip(cache, want_cache))
        x.copy_(y), used.add_(1), at.add_(1)


def test_training_step_in_a_graph():
    """The backward calls captured beside the forward ones, two graphs on workspaces of their own, replayed in turn."""
    g = gen(23)
    graphs = []
    for rows in (70, 300):
        q, k, dq, dk, at, freq, how = rotary_args(g, BF, rows, 4, 2, 64, 32)
        x, w, dy = normal(g, rows, 128, dtype=F32), normal(g, 400, 128, scale=0.1), normal(g, rows, 200)

        def step():
            yq, yk = dense.rotary_forward(q, k, at, freq, **how)
            r = dense.rotary_backward(dq, dk, at, freq, q=q, k=k, **how)
            y, pre = dense.gated_forward(x, w, save_pre=True)
            d = dense.gated_backward(x, w, dy, pre, bias=True)
            return [yq, yk, r["dq"], r["dk"], r["dgain_q"], r["dgain_k"], y, d["dx"], d["dw"], d["db"]]
        want = [t.clone() for t in step()]
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = step()
        graphs.append((graph, got, want, (q, k, dq, dk, at, freq, how, x, w, dy)))     # a graph reads its inputs where they lie
    for _ in range(3):
        for graph, got, want, _ in graphs:
            for t in got:
                t.fill_(float("nan"))
            graph.replay()
        for graph, got, want, _ in graphs:
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_block_forward_and_backward_together():
    """One float32 block around packed attention, its gradients against autograd in 64 bits and against differences."""
    g = gen(24)
    lens, heads, kv, d, f = [40, 1, 23], 4, 2, 32, 96
    n, c = sum(lens), heads * d
    cq = cu(lens)
    at = torch.cat([torch.arange(v) for v in lens]).to(torch.int32).cuda()
    freq, _ = dense.rotary_frequencies(24)
    P = {name: normal(g, *s, scale=s[-1] ** -0.5) for name, s in (("wqkv", ((heads + 2 * kv) * d, c)), ("wo", (c, c)),
                                                               ("wg", (2 * f, c)), ("wd", (c, f)))}
    P.update(x=normal(g, n, c), gq=normal(g, d, scale=0.1, shift=1.0), gk=normal(g, d, scale=0.1, shift=1.0))
    dy = normal(g, n, c)
    sp = (heads, heads + kv)
    qkv, _ = dense.linear_forward(P["x"], P["wqkv"])
    t = qkv.view(n, -1, d)
    q, k = dense.rotary_forward(t[:, :sp[0]], t[:, sp[0]:sp[1]], at, freq, gain_q=P["gq"], gain_k=P["gk"])
    v = t[:, sp[1]:]
    o, lse = dense.attention_forward(q, k, v, cq, causal=True)
    h, _ = dense.linear_forward(o.view(n, c), P["wo"], residual=P["x"])
    a, pre = dense.gated_forward(h, P["wg"], save_pre=True)
    y, _ = dense.linear_forward(a, P["wd"], residual=h)
    b4 = dense.linear_backward(a, P["wd"], dy)
    b3 = dense.gated_backward(h, P["wg"], b4["dx"], pre)
    dh = dy + b3["dx"]
    b2 = dense.linear_backward(o.view(n, c), P["wo"], dh)
    b1 = dense.attention_backward(q, k, v, o, lse, b2["dx"].view(n, heads, d), cq, causal=True)
    dqkv = torch.empty_like(t)
    br = dense.rotary_backward(b1["dq"], b1["dk"], at, freq, q=t[:, :sp[0]], k=t[:, sp[0]:sp[1]], gain_q=P["gq"], gain_k=P["gk"],
                               dq=dqkv[:, :sp[0]], dk=dqkv[:, sp[0]:sp[1]])
    dqkv[:, sp[1]:] = b1["dv"]
    b0 = dense.linear_backward(P["x"], P["wqkv"], dqkv.view(n, -1))
    got = dict(wqkv=b0["dw"], wo=b2["dw"], wg=b3["dw"], wd=b4["dw"], x=dh + b0["dx"], gq=br["dgain_q"], gk=br["dgain_k"])

    def block(p):
        """In 64 bits on the CPU."""
        t = (p["x"] @ p["wqkv"].t()).view(n, -1, d)
        ang = at.cpu().double()[:, None] * freq.cpu()
        co, si = ang.cos()[:, None], ang.sin()[:, None]

        def turn(z, gain):
            z = z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain
            u, w = z[..., :12], z[..., 12:24]
            return torch.cat((u * co - w * si, u * si + w * co, z[..., 24:]), -1)
        q, k, v = turn(t[:, :sp[0]], p["gq"]), turn(t[:, sp[0]:sp[1]], p["gk"]), t[:, sp[1]:]
        outs, first = [], 0
        for m in lens:
            r = slice(first, first + m)
            first += m
            mask = torch.full((m, m), -math.inf, dtype=torch.float64).triu(1)
            for j in range(heads):
                s = q[r, j] @ k[r, j // 2].t() / math.sqrt(d) + mask
                outs.append((r, j, s.softmax(-1) @ v[r, j // 2]))
        o = torch.cat([torch.cat([x for r, j, x in outs if r.start == s], 1) for s in sorted({r.start for r, _, _ in outs})])
        h = p["x"] + o @ p["wo"].t()
        z = h @ p["wg"].t()
        return h + (torch.nn.functional.silu(z[:, :f]) * z[:, f:]) @ p["wd"].t()
    p64 = {name: t.cpu().double().requires_grad_() for name, t in P.items()}
    out = block(p64)
    (out * dy.cpu().double()).sum().backward()
    # ten float32 steps in a row, each within some 10 roundings of sums of 100 terms: 1e-4 of a tensor's largest value
    assert (y.cpu().double() - out).abs().max() <= 1e-4 * out.abs().max()
    for name, t in p64.items():
        assert (got[name].cpu().double() - t.grad).abs().max() <= 1e-4 * t.grad.abs().max(), name
    with torch.no_grad():                     # differences along one direction of every tensor
        for name in P:
            step = torch.randn(P[name].shape, generator=g).double()
            e = 1e-5
            up, down = ({**p64, name: p64[name] + s * e * step} for s in (1, -1))
            slope = ((block(up) - block(down)) * dy.cpu().double()).sum() / (2 * e)
            have = (got[name].cpu().double() * step).sum()
            scale = (got[name].cpu().double() * step).abs().sum()
            assert (slope - have).abs() <= 1e-4 * scale, name


def test_numbers_given_as_tensors_are_read_at_each_call():
    """Calls remember checked arguments by shapes and numbers: a tensor that stands for a number counts by its value."""
    g = gen(30)
    q, k, _, _, at, freq, _ = rotary_args(g, F32, 5, 2, 1, 32, 32, norm=False)
    scale = torch.tensor(1.0)
    a, _ = dense.rotary_forward(q, k, at, freq, magnitude=scale)
    scale.fill_(2.0)
    b, _ = dense.rotary_forward(q, k, at, freq, magnitude=scale)
    assert torch.equal(b, 2 * a)
    cache, _, _ = filled(g, 64, 1, 32)
    rows, c = torch.tensor(64), cu([64])
    assert dense.cache_read(cache, rows, c, c)[0].shape[0] == 64
    rows.fill_(7)
    assert dense.cache_read(cache, rows, cu([7]), cu([64]), ints([7]))[0].shape[0] == 7


def test_cache_attention_more_sequences_than_rows():
    g = gen(31)
    check_cache_attention(g, "bf16", [1] * 6, [1, 0, 0, 2, 0, 0], None, 2, 1, 32, True)
    check_cache_attention(g, "bf16", [2] * 70, [0, 1] * 35, None, 2, 2, 32, True)
    check_cache_attention(g, "bf16", [3, 2], [0, 0], None, 2, 2, 64, False)
