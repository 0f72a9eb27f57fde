"""Argument checks of the dense operators (host only: nothing is launched) and their ctypes structs."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2506_12541_amd import _lib, dense

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, SMALL = _lib.BSA_ERR_INVALID_ARGUMENT, _lib.BSA_ERR_UNSUPPORTED, _lib.BSA_ERR_WORKSPACE_TOO_SMALL
PTR = 1 << 12     # never dereferenced: the calls below stop before a launch


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2506_12541_amd.build import build
        build()
    return _lib.load()


def norm(**kw):
    return _lib.bsa_layernorm_t(**dict(dict(rows=4, cols=64, dtype=1, eps=1e-5), **kw))


def lin(**kw):
    return _lib.bsa_linear_t(**dict(dict(m=4, k=64, n=32, dtype=1, act=0), **kw))


def att(**kw):
    return _lib.bsa_attention_t(**dict(dict(seqs=2, heads=4, kv_heads=2, head_dim=64, total_q=8, total_k=8, dtype=1), **kw))


def test_struct_layouts_match_the_header(tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('#include "bsa.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu\\n", '
                   'sizeof(bsa_layernorm_t), sizeof(bsa_linear_t), sizeof(bsa_attention_t)); return 0; }\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(_lib.bsa_layernorm_t), C.sizeof(_lib.bsa_linear_t), C.sizeof(_lib.bsa_attention_t)]


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=32769), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(ld_x=63), INVALID), (dict(ld_y=-1), INVALID), (dict(ld_dy=1), INVALID), (dict(ld_dx=63), INVALID)])
def test_layernorm_refusals(lib, kw, code):
    p = norm(**kw)
    assert lib.bsa_layernorm_sizes(C.byref(p), None) == code and lib.bsa_last_error()
    assert lib.bsa_layernorm_forward(C.byref(p), *[PTR] * 6, None) == code


def test_layernorm_pointers(lib):
    p, need = norm(rows=4096), C.c_size_t()
    assert lib.bsa_layernorm_sizes(None, None) == INVALID
    assert lib.bsa_layernorm_sizes(C.byref(p), C.byref(need)) == 0 and need.value > 0
    assert lib.bsa_layernorm_forward(C.byref(p), PTR, None, None, 2 * PTR, PTR, PTR, None) == INVALID
    assert lib.bsa_layernorm_forward(C.byref(p), PTR, PTR, None, PTR, PTR, PTR, None) == INVALID      # y is x
    assert lib.bsa_layernorm_backward(C.byref(p), *[PTR] * 5, 2 * PTR, None, PTR, PTR, 1 << 40, None) == INVALID
    assert lib.bsa_layernorm_backward(C.byref(p), *[PTR] * 5, 2 * PTR, PTR, PTR, PTR, need.value - 1, None) == SMALL
    q = norm(ld_dx=70)
    assert lib.bsa_layernorm_backward(C.byref(q), *[PTR] * 5, PTR, PTR, PTR, PTR, 1 << 40, None) == INVALID  # dx is x
    assert lib.bsa_layernorm_forward(C.byref(norm(rows=0)), *[None] * 6, None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), INVALID), (dict(m=1 << 31), INVALID), (dict(k=0), INVALID), (dict(n=0), INVALID),
    (dict(k=(1 << 24) + 1), UNSUPPORTED), (dict(m=(1 << 31) - 1, n=1 << 24), UNSUPPORTED), (dict(dtype=-1), INVALID),
    (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(ld_x=63), INVALID), (dict(ld_w=1), INVALID),
    (dict(ld_y=31), INVALID), (dict(ld_res=31), INVALID), (dict(ld_dy=31), INVALID)])
def test_linear_refusals(lib, kw, code):
    p = lin(**kw)
    assert lib.bsa_linear_sizes(C.byref(p), None, None) == code and lib.bsa_last_error()
    assert lib.bsa_linear_forward(C.byref(p), *[PTR] * 7, 1 << 40, None) == code


def test_linear_pointers(lib):
    f, b = C.c_size_t(), C.c_size_t()
    p = lin(m=4096, act=2)
    assert lib.bsa_linear_sizes(C.byref(p), C.byref(f), C.byref(b)) == 0 and b.value > 0
    assert lib.bsa_linear_forward(C.byref(p), PTR, None, None, None, 2 * PTR, None, PTR, 1 << 40, None) == INVALID
    assert lib.bsa_linear_forward(C.byref(p), PTR, PTR, None, None, PTR, None, PTR, 1 << 40, None) == INVALID  # y is x
    back = lambda pre, dx, n: lib.bsa_linear_backward(C.byref(p), PTR, PTR, pre, PTR, dx, 3 * PTR, 4 * PTR, PTR, n, None)
    assert back(None, 2 * PTR, 1 << 40) == INVALID and "pre" in lib.bsa_last_error().decode()
    assert back(PTR, PTR, 1 << 40) == INVALID
    assert back(PTR, 2 * PTR, b.value - 1) == SMALL
    assert lib.bsa_linear_backward(C.byref(p), *[None] * 8, 0, None) == 0        # nothing asked for
    assert lib.bsa_linear_forward(C.byref(lin(m=0)), *[None] * 7, 0, None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(seqs=0), INVALID), (dict(heads=3), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(heads=65536), UNSUPPORTED), (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
    (dict(total_q=-1), INVALID), (dict(total_k=1 << 31), INVALID), (dict(total_q=1 << 30, heads=64), UNSUPPORTED),
    (dict(causal=2), INVALID), (dict(zero_rest=-1), INVALID), (dict(dtype=2), INVALID), (dict(softmax_scale=-1.0), INVALID),
    (dict(softmax_scale=float("nan")), INVALID), (dict(q_row=260, q_head=64), INVALID), (dict(k_row=128, k_head=-8), INVALID),
    (dict(do_row=256, do_head=68), INVALID), (dict(dtype=0, v_row=130, v_head=64), INVALID)])
def test_attention_refusals(lib, kw, code):
    p = att(**kw)
    assert lib.bsa_attention_sizes(C.byref(p), None, None) == code and lib.bsa_last_error()
    assert lib.bsa_attention_forward(C.byref(p), *[PTR] * 9, 1 << 40, None) == code


def test_attention_pointers(lib):
    f, b = C.c_size_t(), C.c_size_t()
    p = att(total_k=1 << 16)
    assert lib.bsa_attention_sizes(C.byref(p), C.byref(f), C.byref(b)) == 0 and f.value > 0 and b.value > 0
    fwd = lambda q=PTR, k=PTR, o=2 * PTR, cu=PTR, n=1 << 40: lib.bsa_attention_forward(
        C.byref(p), q, k, PTR, cu, cu, None, o, PTR, PTR, n, None)
    assert fwd(q=None) == fwd(k=None) == fwd(o=None) == fwd(cu=None) == INVALID
    assert fwd(q=PTR + 8) == fwd(k=PTR + 2) == fwd(o=PTR + 8) == INVALID and "aligned" in lib.bsa_last_error().decode()
    assert fwd(o=PTR) == INVALID
    assert fwd(n=f.value - 1) == SMALL
    p.o_row, p.o_head = 256, 32                     # heads of o on top of each other
    assert fwd() == INVALID and "overlap" in lib.bsa_last_error().decode()
    p.o_row, p.o_head = 64, 8 * 64                  # head-major is fine (the short workspace is found next)
    assert fwd(n=f.value - 1) == SMALL
    p.o_row = p.o_head = 0
    back = lambda dq=2 * PTR, dk=3 * PTR, n=1 << 40: lib.bsa_attention_backward(
        C.byref(p), *[PTR] * 8, None, dq, dk, 4 * PTR, PTR, n, None)
    assert back(dq=None) == back(dk=None) == back(dq=PTR) == back(dk=PTR + 4) == INVALID
    assert back(n=b.value - 1) == SMALL
    assert lib.bsa_attention_forward(C.byref(att(total_q=0)), *[None] * 9, 0, None) == 0


def test_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros(4, 8)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        dense.layernorm_forward(x, torch.ones(8))
    with pytest.raises(ValueError, match="CUDA"):
        dense.linear_forward(x, torch.zeros(3, 8))
    with pytest.raises(ValueError, match="CUDA"):
        dense.attention_forward(x.view(4, 1, 8), x.view(4, 1, 8), x.view(4, 1, 8), cu)
    with pytest.raises(ValueError, match="both"):
        dense.attention_forward(x.view(4, 1, 8), x.view(4, 1, 8), x.view(4, 1, 8), cu, o=x)


def test_binding_refuses_heads_that_are_broadcast_over_rows_and_heads(monkeypatch):
    """Strides of 0 and 0 are the C ABI's packed tensor: a [rows, heads, d] tensor over the storage of one row of d
    elements (the gradient of o.sum((0, 1))) would be read, and as an output written, behind its end."""
    monkeypatch.setattr(dense, "_tensor", lambda *a, **kw: None)       # the tensors here are on the CPU
    o = torch.zeros(5, 3, 64, requires_grad=True)
    grad, = torch.autograd.grad((o.sum((0, 1)) * torch.ones(64)).sum(), o)
    one = torch.zeros(64)
    for t in (grad, one.expand(5, 3, 64), torch.zeros(7, 1, 1, 64)[2].expand(2, 3, 64)):
        assert t.stride()[:2] == (0, 0)
        with pytest.raises(ValueError, match="broadcast"):
            dense._heads(t, "d_o")
    # over one of them the strides say what they are; a dimension of one entry is not broadcast
    assert dense._heads(torch.zeros(5, 1, 64).expand(5, 3, 64), "k") == (64, 0)
    assert dense._heads(torch.zeros(1, 3, 64).expand(5, 3, 64), "k") == (0, 64)
    assert dense._heads(one.expand(5, 1, 64), "k") == (0, 64)
    assert dense._heads(one.expand(1, 3, 64), "k") == (192, 0)


def test_attention_refuses_an_output_that_is_broadcast(lib):
    for row, head in ((0, 64), (64, 0)):
        p = att(o_row=row, o_head=head)
        assert lib.bsa_attention_forward(C.byref(p), *[PTR] * 6, 2 * PTR, PTR, PTR, 1 << 40, None) == INVALID
        assert "overlap" in lib.bsa_last_error().decode()


def test_linear_refuses_outputs_on_its_inputs(lib):
    """Gradients and the kept pre-activation are written while other workgroups still read the inputs."""
    p, big = lin(m=4096, act=2), 1 << 40
    x, w, pre, dy, dx, dw, db, ws = (i * PTR for i in range(1, 9))
    back = lambda dx=dx, dw=dw, db=db: lib.bsa_linear_backward(C.byref(p), x, w, pre, dy, dx, dw, db, ws, 0, None)
    for t in (x, w, pre, dy):
        for kw in (dict(dx=t), dict(dw=t), dict(db=t), dict(dx=None, db=None, dw=t), dict(dx=None, dw=None, db=t)):
            assert back(**kw) == INVALID and "alias" in lib.bsa_last_error().decode(), (t // PTR, kw)
    assert back() == SMALL and back(dx=None) == SMALL and back(dw=None, db=None) == SMALL
    q = lin(m=4096)                                     # without an activation pre is not read
    assert lib.bsa_linear_backward(C.byref(q), x, w, pre, dy, pre, dw, db, ws, 0, None) == SMALL
    assert lib.bsa_linear_backward(C.byref(q), x, w, None, dy, dx, dw, None, ws, 0, None) == SMALL
    assert lib.bsa_linear_backward(C.byref(q), x, w, None, dy, dx, dy, None, ws, 0, None) == INVALID
    r = lin(m=100, k=8192, act=1)                       # a split contraction: the workspace is found short at last
    bias, res, y = 4 * PTR, 5 * PTR, 6 * PTR
    fwd = lambda y, pre: lib.bsa_linear_forward(C.byref(r), x, w, bias, res, y, pre, ws, 0, None)
    for t in (x, w, bias):
        assert fwd(t, 7 * PTR) == INVALID and "alias" in lib.bsa_last_error().decode()
    for t in (x, w, bias, res, y):
        assert fwd(y, t) == INVALID and "alias" in lib.bsa_last_error().decode()
    assert fwd(y, 7 * PTR) == SMALL and fwd(res, 7 * PTR) == SMALL and fwd(y, None) == SMALL


def test_launches_past_their_limit_are_refused(lib):
    """A grid times its threads has to stay below 2^32."""
    for kw in (dict(m=(1 << 31) - 1, n=8, k=8), dict(m=(1 << 31) - 255, n=8, k=8), dict(m=1 << 26, n=64, k=1 << 13)):
        p = lin(**kw)
        assert lib.bsa_linear_sizes(C.byref(p), None, None) == UNSUPPORTED and "tiles" in lib.bsa_last_error().decode()
    for kw in (dict(m=(1 << 31) - 256, n=8, k=8), dict(m=0, n=1 << 16, k=1 << 16), dict(m=1 << 20, n=1 << 10, k=1 << 10)):
        assert lib.bsa_linear_sizes(C.byref(lin(**kw)), None, None) == 0
    # single tokens (16-row tiles), then usual tiles; the checks of pointers come behind that of the grid
    forward = lambda p: lib.bsa_attention_forward(C.byref(p), *[None] * 9, 0, None)
    backward = lambda p: lib.bsa_attention_backward(C.byref(p), *[None] * 13, 0, None)
    for kw in (dict(seqs=1 << 24), dict(seqs=1 << 23, heads=1, kv_heads=1, total_q=1 << 27, total_k=1 << 27)):
        p = att(**kw)
        assert forward(p) == UNSUPPORTED and "tiles" in lib.bsa_last_error().decode()
    p = att(seqs=1 << 24)
    assert backward(p) == UNSUPPORTED and "tiles" in lib.bsa_last_error().decode()
    p = att(heads=1, kv_heads=1, head_dim=128, seqs=1 << 10, total_q=1 << 30, total_k=1 << 10)
    assert forward(p) == INVALID and backward(p) == UNSUPPORTED
    p = att(heads=1, kv_heads=1, seqs=1 << 22, total_q=1 << 27, total_k=1 << 27)
    assert forward(p) == backward(p) == INVALID
