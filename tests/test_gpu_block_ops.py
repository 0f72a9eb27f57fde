"""Rotary positions with head norms, the gated map, and the 8-bit cache with the attention that reads it, on the GPU
against their float64 definitions, within bounds derived from the types (tests/block_ref.py)."""
import math

import pytest
import torch

import block_ref as ref
import dense_ref
from dense_ref import check
from paper_2506_12541_amd import dense

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
