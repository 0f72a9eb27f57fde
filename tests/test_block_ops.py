"""Argument checks of the rotary, gated and cache operators (host only: nothing is launched), their ctypes structs, and
the table of rotary frequencies."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

import block_ref
from paper_2506_12541_amd import _lib, dense

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, SMALL = _lib.BSA_ERR_INVALID_ARGUMENT, _lib.BSA_ERR_UNSUPPORTED, _lib.BSA_ERR_WORKSPACE_TOO_SMALL
PTR = 1 << 12     # never dereferenced: the calls below stop before a launch
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2506_12541_amd.build import build
        build()
    return _lib.load()


def rot(**kw):
    return _lib.bsa_rotary_t(**dict(dict(rows=4, heads=4, kv_heads=2, head_dim=64, rot=48, axes=1, dtype=1, eps=1e-5,
                                         magnitude=1.0), **kw))


def gat(**kw):
    return _lib.bsa_gated_t(**dict(dict(m=4, k=64, n=32, dtype=1, act=3), **kw))


def cac(**kw):
    return _lib.bsa_cache_t(**dict(dict(seqs=2, kv_heads=2, head_dim=64, dtype=1, rows=8, total_k=64), **kw))


def att(**kw):
    return _lib.bsa_attention_t(**dict(dict(seqs=2, heads=4, kv_heads=2, head_dim=64, total_q=8, total_k=1 << 16, dtype=1), **kw))


def test_struct_layouts_match_the_header(tmp_path):
    names = ("bsa_rotary_t", "bsa_gated_t", "bsa_cache_t")
    src = tmp_path / "sz.c"
    src.write_text('#include "bsa.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu\\n", '
                   + ", ".join(f"sizeof({n})" for n in names) + '); return 0; }\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(getattr(_lib, n)) for n in names]


# ---- rotary positions ----

@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=-1), INVALID), (dict(heads=65536), UNSUPPORTED),
    (dict(head_dim=1, rot=2), INVALID), (dict(head_dim=257), UNSUPPORTED), (dict(rot=0), INVALID), (dict(rot=47), INVALID),
    (dict(rot=66), INVALID), (dict(axes=0), INVALID), (dict(axes=5), INVALID), (dict(rot=44, axes=3), INVALID),
    (dict(pos_type=2), INVALID), (dict(interleaved=2), INVALID), (dict(dtype=2), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(magnitude=0.0), INVALID),
    (dict(magnitude=math.inf), INVALID), (dict(magnitude=math.nan), INVALID), (dict(q_row=-1, q_head=64), INVALID),
    (dict(oq_row=256, oq_head=32), INVALID), (dict(ok_row=64, ok_head=64), INVALID), (dict(oq_row=0, oq_head=64), INVALID)])
def test_rotary_refusals(lib, kw, code):
    p = rot(**kw)
    assert lib.bsa_rotary_sizes(C.byref(p), None) == code and lib.bsa_last_error()
    assert lib.bsa_rotary_forward(C.byref(p), *[PTR] * 8, None) == code
    assert lib.bsa_rotary_backward(C.byref(p), *[PTR] * 12, PTR, BIG, None) == code


def test_rotary_pointers(lib):
    need = C.c_size_t()
    p = rot(rows=4096)
    assert lib.bsa_rotary_sizes(None, None) == INVALID
    assert lib.bsa_rotary_sizes(C.byref(p), C.byref(need)) == 0 and need.value > 0
    q, k, pos, freq, yq, yk, far = (i * PTR for i in range(1, 8))

    def fwd(p=p, q=q, k=k, pos=pos, freq=freq, yq=yq, yk=yk):
        return lib.bsa_rotary_forward(C.byref(p), q, k, pos, freq, None, None, yq, yk, None)
    assert fwd(q=None) == fwd(k=None) == fwd(pos=None) == fwd(freq=None) == fwd(yq=None) == fwd(yk=None) == INVALID
    assert fwd(yq=yk) == fwd(yq=k) == fwd(yk=q) == INVALID and "only be" in lib.bsa_last_error().decode()
    apart = rot(q_row=512, q_head=64)
    assert fwd(p=apart, yq=q) == INVALID and "strides" in lib.bsa_last_error().decode()
    assert lib.bsa_rotary_forward(C.byref(rot(rows=0)), *[None] * 9) == 0

    def back(p=p, q=q, k=k, gq=far, gk=far, dyq=8 * PTR, dyk=9 * PTR, dq=yq, dk=yk, dgq=10 * PTR, dgk=11 * PTR, n=need.value - 1):
        return lib.bsa_rotary_backward(C.byref(p), q, k, pos, freq, gq, gk, dyq, dyk, dq, dk, dgq, dgk, PTR, n, None)
    assert back() == SMALL
    assert back(q=None) == back(k=None) == back(dyq=None) == back(dyk=None) == back(dq=None) == back(dk=None) == INVALID
    assert back(gq=None, q=None, dgq=None) == SMALL        # without its gain q is not read
    assert back(gq=None) == INVALID and "gain" in lib.bsa_last_error().decode()
    assert back(dq=yk) == back(dq=k) == back(dq=9 * PTR) == back(dk=q) == back(dk=8 * PTR) == INVALID
    assert back(dq=q) == back(dq=8 * PTR) == back(dk=k) == back(dk=9 * PTR) == SMALL
    assert back(p=apart, dq=q) == INVALID and "strides" in lib.bsa_last_error().decode()
    assert back(p=rot(rows=4096, kv_heads=0), k=None, dyk=None, dk=None) == SMALL      # no keys


# ---- gated map ----

@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), INVALID), (dict(m=1 << 31), INVALID), (dict(k=0), INVALID), (dict(n=0), INVALID),
    (dict(k=(1 << 24) + 1), UNSUPPORTED), (dict(n=(1 << 23) + 1), UNSUPPORTED), (dict(m=(1 << 31) - 1), UNSUPPORTED),
    (dict(dtype=-1), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(ld_x=63), INVALID),
    (dict(ld_w=1), INVALID), (dict(ld_y=31), INVALID), (dict(ld_dy=31), INVALID)])
def test_gated_refusals(lib, kw, code):
    p = gat(**kw)
    assert lib.bsa_gated_sizes(C.byref(p), None, None) == code and lib.bsa_last_error()
    assert lib.bsa_gated_forward(C.byref(p), *[PTR] * 6, BIG, None) == code
    assert lib.bsa_gated_backward(C.byref(p), *[PTR] * 8, BIG, None) == code


def test_gated_pointers(lib):
    f, b = C.c_size_t(), C.c_size_t()
    assert lib.bsa_gated_sizes(None, None, None) == INVALID
    p = gat(m=100, k=8192)                             # a split contraction
    assert lib.bsa_gated_sizes(C.byref(p), C.byref(f), C.byref(b)) == 0 and f.value > 0 and b.value > 0
    x, w, bias, y, pre, dy, dx, dw, db = (i * PTR for i in range(1, 10))

    def fwd(x=x, w=w, y=y, pre=pre):
        return lib.bsa_gated_forward(C.byref(p), x, w, bias, y, pre, PTR, f.value - 1, None)
    assert fwd() == fwd(pre=None) == SMALL
    assert fwd(x=None) == fwd(w=None) == fwd(y=None) == INVALID
    for t in (x, w, bias):
        assert fwd(y=t) == fwd(pre=t) == INVALID and "alias" in lib.bsa_last_error().decode()
    assert fwd(y=pre) == INVALID

    def back(x=x, w=w, pre=pre, dy=dy, dx=dx, dw=dw, db=db):
        return lib.bsa_gated_backward(C.byref(p), x, w, pre, dy, dx, dw, db, PTR, b.value - 1, None)
    assert back() == back(dx=None) == back(dw=None) == back(db=None) == SMALL
    assert back(pre=None) == back(dy=None) == back(x=None) == back(w=None) == INVALID
    assert back(x=None, dw=None) == back(w=None, dx=None) == SMALL
    for t in (x, w, pre, dy):
        assert back(dx=t) == back(dw=t) == back(db=t) == INVALID and "alias" in lib.bsa_last_error().decode()
    assert back(dx=None, dw=None, db=None) == 0        # nothing asked for
    assert lib.bsa_gated_forward(C.byref(gat(m=0)), *[None] * 6, 0, None) == 0


def test_gated_workspaces_begin_on_16_bytes(lib):
    """Pieces of 16 bytes go from the workspace straight into LDS."""
    f, b = C.c_size_t(), C.c_size_t()
    for kw in (dict(m=100, k=8192), dict(m=2048, k=1024, n=1024, dtype=0), dict(m=3000, k=1031, n=1100)):
        p = gat(**kw)
        assert lib.bsa_gated_sizes(C.byref(p), C.byref(f), C.byref(b)) == 0 and f.value > 0 and b.value > 0
        x, w, bias, y, pre, dy, dx, dw, db = (i * PTR for i in range(1, 10))
        for ws in (16 * PTR + 2, 16 * PTR + 4, 16 * PTR + 8):
            assert lib.bsa_gated_forward(C.byref(p), x, w, bias, y, pre, ws, f.value, None) == INVALID
            assert "aligned" in lib.bsa_last_error().decode()
            assert lib.bsa_gated_backward(C.byref(p), x, w, pre, dy, dx, dw, db, ws, b.value, None) == INVALID
            assert "aligned" in lib.bsa_last_error().decode()


# ---- 8-bit cache ----

@pytest.mark.parametrize("kw,code", [
    (dict(seqs=0), INVALID), (dict(seqs=(1 << 24) + 1), UNSUPPORTED), (dict(kv_heads=0), INVALID), (dict(kv_heads=65536), UNSUPPORTED),
    (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(total_k=-1), INVALID),
    (dict(rows=(1 << 30) + 1), UNSUPPORTED), (dict(total_k=(1 << 30) + 1), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(k_row=132, k_head=64), INVALID), (dict(v_row=-8, v_head=64), INVALID), (dict(ck_row=136, ck_head=64), INVALID),
    (dict(cv_row=128, cv_head=32), INVALID), (dict(ck_row=0, ck_head=64), INVALID), (dict(cv_row=64, cv_head=0), INVALID)])
def test_cache_refusals(lib, kw, code):
    p = cac(**kw)
    assert lib.bsa_cache_write(C.byref(p), *[i * PTR for i in range(1, 10)], None) == code and lib.bsa_last_error()
    assert lib.bsa_cache_read(C.byref(p), *[i * PTR for i in range(1, 10)], None) == code


def test_cache_pointers(lib):
    k, v, cu, ck, cv, ek, ev = (i * PTR for i in range(1, 8))

    def write(p=cac(), k=k, v=v, cu_q=cu, cu_k=cu, ck=ck, cv=cv, ek=ek, ev=ev):
        return lib.bsa_cache_write(C.byref(p), k, v, cu_q, cu_k, None, ck, cv, ek, ev, None)

    def read(p=cac(), k=k, v=v, cu_q=cu, cu_k=cu, ck=ck, cv=cv, ek=ek, ev=ev):
        return lib.bsa_cache_read(C.byref(p), ck, cv, ek, ev, cu_q, cu_k, None, k, v, None)
    for f in (write, read):
        for name in ("k", "v", "cu_q", "cu_k", "ck", "cv", "ek", "ev"):
            assert f(**{name: None}) == INVALID, name
        for name in ("k", "v", "ck", "cv"):
            assert f(**{name: 8 * PTR + 8}) == INVALID and "aligned" in lib.bsa_last_error().decode()
        for kw in (dict(k=ck), dict(k=cv), dict(v=ck), dict(v=cv)):
            assert f(**kw) == INVALID and "alias" in lib.bsa_last_error().decode()
        assert f(p=cac(rows=0)) == 0
    assert write(ck=cv) == write(ek=ev) == read(k=v) == INVALID
    assert read(p=cac(k_row=64, k_head=64)) == INVALID and "overlap" in lib.bsa_last_error().decode()
    assert lib.bsa_cache_write(None, *[PTR] * 9, None) == INVALID and lib.bsa_cache_read(None, *[PTR] * 9, None) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(seqs=0), INVALID), (dict(heads=3), INVALID), (dict(head_dim=48), UNSUPPORTED), (dict(total_q=-1), INVALID),
    (dict(causal=2), INVALID), (dict(zero_rest=2), INVALID), (dict(dtype=2), INVALID), (dict(softmax_scale=-1.0), INVALID),
    (dict(k_row=128, k_head=8), INVALID), (dict(v_row=136, v_head=64), INVALID), (dict(q_row=260, q_head=64), INVALID)])
def test_cache_attention_refusals(lib, kw, code):
    p = att(**kw)
    assert lib.bsa_cache_attention_sizes(C.byref(p), None) == code and lib.bsa_last_error()
    assert lib.bsa_cache_attention_forward(C.byref(p), *[i * PTR for i in range(1, 12)], BIG, None) == code


def test_cache_attention_pointers(lib):
    need, p = C.c_size_t(), att()
    assert lib.bsa_cache_attention_sizes(None, None) == INVALID
    assert lib.bsa_cache_attention_sizes(C.byref(p), C.byref(need)) == 0 and need.value > 0
    q, ck, cv, ek, ev, cu, o, lse = (i * PTR for i in range(1, 9))

    def fwd(p=p, q=q, ck=ck, cv=cv, ek=ek, ev=ev, cu_q=cu, cu_k=cu, o=o, lse=lse):
        return lib.bsa_cache_attention_forward(C.byref(p), q, ck, cv, ek, ev, cu_q, cu_k, None, o, lse, PTR, need.value - 1, None)
    assert fwd() == SMALL
    for name in ("q", "ck", "cv", "ek", "ev", "cu_q", "cu_k", "o", "lse"):
        assert fwd(**{name: None}) == INVALID, name
    for name in ("q", "ck", "cv", "o"):
        assert fwd(**{name: 9 * PTR + 8}) == INVALID and "aligned" in lib.bsa_last_error().decode()
    assert fwd(o=q) == fwd(o=ck) == fwd(o=cv) == INVALID
    assert fwd(p=att(o_row=256, o_head=32)) == INVALID and "overlap" in lib.bsa_last_error().decode()
    # the cache's strides are bytes: packed, and the first of two heads' halves
    assert fwd(p=att(k_row=128, k_head=64)) == fwd(p=att(k_row=64, k_head=1 << 22)) == SMALL
    assert lib.bsa_cache_attention_forward(C.byref(att(total_q=0)), *[None] * 11, 0, None) == 0
    assert lib.bsa_cache_attention_forward(C.byref(att(seqs=1 << 24)), *[None] * 11, 0, None) == UNSUPPORTED


# ---- binding ----

def test_binding_refuses_what_is_not_on_a_gpu():
    q, at, cu = torch.zeros(4, 2, 32), torch.zeros(4, dtype=torch.int32), torch.tensor([0, 4], dtype=torch.int32)
    freq, _ = dense.rotary_frequencies(32, device="cpu")
    cache = dense.cache_alloc(8, 2, 32, device="cpu")
    for call in (lambda: dense.rotary_forward(q, q, at, freq), lambda: dense.rotary_backward(q, q, at, freq),
                 lambda: dense.gated_forward(q[0], torch.zeros(4, 32)), lambda: dense.cache_write(cache, q, q, cu, cu),
                 lambda: dense.cache_read(cache, 4, cu, cu), lambda: dense.cache_attention_forward(q, cache, cu, cu)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_refuses_shapes(monkeypatch):
    monkeypatch.setattr(dense, "_tensor", lambda *a, **kw: None)       # the tensors here are on the CPU
    q, k = torch.zeros(4, 4, 32), torch.zeros(4, 2, 32)
    at, cu = torch.zeros(4, dtype=torch.int32), torch.tensor([0, 4], dtype=torch.int32)
    freq, _ = dense.rotary_frequencies(32, device="cpu")
    for call, what in ((lambda: dense.rotary_forward(q[0], k, at, freq), "q must be"),
                       (lambda: dense.rotary_forward(q, k[:3], at, freq), "k must be"),
                       (lambda: dense.rotary_forward(q, k[:, :, :8], at, freq), "k must be"),
                       (lambda: dense.rotary_forward(q, None, at, freq, gain_k=torch.ones(32)), "gain_k needs k"),
                       (lambda: dense.rotary_forward(q, None, at, freq, y_k=k), "y_k needs k"),
                       (lambda: dense.rotary_forward(q, k, at[:3], freq), "positions"),
                       (lambda: dense.rotary_forward(q, k, at.long(), freq), "positions"),
                       (lambda: dense.rotary_forward(q, k, at, freq[::2]), "freq"),
                       (lambda: dense.rotary_forward(q, k, at, freq, gain_q=torch.ones(16)), "gain_q"),
                       (lambda: dense.rotary_forward(q[:1, :1].expand(4, 4, 32), k, at, freq), "broadcast"),
                       (lambda: dense.rotary_backward(q, k, at, freq, gain_q=torch.ones(32)), "q is needed"),
                       (lambda: dense.rotary_backward(q, k, at, freq, q=q[:2], gain_q=torch.ones(32)), "shape"),
                       (lambda: dense.gated_forward(q[0], torch.zeros(5, 32)), "2 n"),
                       (lambda: dense.gated_forward(q[0], torch.zeros(4, 32), act="tanh"), "act"),
                       (lambda: dense.gated_backward(q[0], torch.zeros(4, 32), torch.zeros(4, 2), None), "pre"),
                       (lambda: dense.cache_read(dense.cache_alloc(8, 2, 32, "cpu"), 4, cu, cu, dtype=torch.float16), "dtype"),
                       (lambda: dense.cache_read(dense.cache_alloc(8, 2, 32, "cpu"), -1, cu, cu), "rows"),
                       (lambda: dense.cache_write(dense.cache_alloc(8, 2, 64, "cpu"), k, k, cu, cu), "heads of"),
                       (lambda: dense.cache_attention_forward(q, dense.cache_alloc(8, 2, 64, "cpu"), cu, cu), "head_dim")):
        with pytest.raises(ValueError, match=what):
            call()


def test_rotary_frequencies():
    f, mag = dense.rotary_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and mag == 1.0
    assert torch.allclose(f, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32), rtol=1e-14)
    assert torch.equal(dense.rotary_frequencies(48, axes=3, device="cpu")[0], dense.rotary_frequencies(16, device="cpu")[0].repeat(3))
    assert torch.equal(dense.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu")[0], f / 4)
    b, _ = dense.rotary_frequencies(64, scaling="base", factor=4.0, device="cpu")
    assert b[0] == 1 and torch.isclose(b[-1], f[-1] / 4, rtol=1e-12) and (b <= f).all()
    r, mag = dense.rotary_frequencies(64, scaling="ramp", factor=4.0, trained=4096, device="cpu")
    turns = f * 4096 / (2 * math.pi)
    assert torch.equal(r[turns >= 32], f[turns >= 32]) and torch.allclose(r[turns <= 1], f[turns <= 1] / 4, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (r[mid] < f[mid]).all() and (r[mid] > f[mid] / 4).all() and mag == 0.1 * math.log(4.0) + 1
    assert torch.equal(dense.rotary_frequencies(64, scaling="ramp", factor=1.0, trained=4096, device="cpu")[0], f)
    for kw in (dict(rot=7), dict(rot=0), dict(rot=8, axes=3), dict(rot=8, base=0.0), dict(rot=8, factor=0.5),
               dict(rot=8, scaling="other"), dict(rot=8, scaling="ramp"), dict(rot=8, scaling="ramp", trained=10, low=3, high=2)):
        with pytest.raises(ValueError):
            dense.rotary_frequencies(device="cpu", **kw)


# ---- the tests' own definition of the cache's numbers ----

def test_quantise_agrees_with_the_library_conversion():
    """block_ref.quantise, by its list of numbers, against torch's conversion to e4m3 with the same scales."""
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(64, 3, 32, generator=g) * 10.0 ** e for e in (-30, -3, 0, 2, 30)]).to(torch.bfloat16)
    values, codes = block_ref.quantise(x)
    scale = 2.0 ** (codes.t().double() - 127)[..., None]
    want = (x.double() / scale).clamp(-448, 448).float().to(torch.float8_e4m3fn).double() * scale
    assert torch.equal(values, want)
    top = x.double().abs().amax(2, keepdim=True) / scale
    assert ((top <= 448) & ((top > 224) | (codes.t()[..., None] == 63)) | (codes.t()[..., None] == 190)).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_definitions_gradients_are_their_differences(interleaved):
    """The float64 gradients that the GPU tests compare with, against central differences of the float64 outputs."""
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    x, gain, dy = r(3, 2, 20), r(20), r(3, 2, 20)
    at, freq = torch.tensor([0, 7, 1000]), dense.rotary_frequencies(12, device="cpu")[0]
    # bounds go by the type: float32 stands for it, the values are float64
    block_ref.HALF[torch.float64] = block_ref.HALF[torch.float32]
    try:
        f = lambda x, gain: (block_ref.rotary(x, at, freq, gain, 1e-3, interleaved, 1.5)["y"][0] * dy).sum()
        got = block_ref.rotary(x, at, freq, gain, 1e-3, interleaved, 1.5, dy)
        dx, dgain = r(3, 2, 20), r(20)
        e = 1e-6
        assert abs((f(x + e * dx, gain) - f(x - e * dx, gain)) / (2 * e) - (got["dx"][0] * dx).sum()) < 1e-6
        assert abs((f(x, gain + e * dgain) - f(x, gain - e * dgain)) / (2 * e) - (got["dgain"][0] * dgain).sum()) < 1e-6
        x, w, b, dy2 = r(5, 7), r(12, 7), r(12), r(5, 6)
        for act in ("none", "gelu", "silu"):
            f = lambda x, w, b: (block_ref.gated(x, w, b, act)["y"][0] * dy2).sum()
            got = block_ref.gated(x, w, b, act, dy2)
            for name, t in (("dx", r(5, 7)), ("dw", r(12, 7)), ("db", r(12))):
                up, down = ([v + s * e * t if n == name else v for n, v in (("dx", x), ("dw", w), ("db", b))] for s in (1, -1))
                assert abs((f(*up) - f(*down)) / (2 * e) - (got[name][0] * t).sum()) < 1e-6, (act, name)
    finally:
        del block_ref.HALF[torch.float64]
