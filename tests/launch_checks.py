"""What the entry points of libbsa.so launch, on the CPU: tests/test_launches.py runs this file, one check to a process, with
launch_stub.c in the HIP runtime's place. Not for a process that has loaded torch, whose own runtime would come first."""
import ctypes as C
import importlib.util
import os
import random
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 1 << 12     # stands for device memory, never dereferenced
BIG = 1 << 60     # bytes of a workspace
REPORT = C.CFUNCTYPE(None, C.c_char_p, C.POINTER(C.c_uint32 * 3), C.POINTER(C.c_uint32 * 3), C.POINTER(C.c_void_p))


def binding():
    spec = importlib.util.spec_from_file_location("_lib", os.path.join(ROOT, "paper_2506_12541_amd", "_lib.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Launch:
    def __init__(self, kernel, grid, block, args):
        self.kernel, self.grid, self.block, self.args = kernel, grid, block, args

    def threads(self, axis=0):
        return self.grid[axis] * self.block[axis]


class Library:
    """The library and, of each call, its launches. take: {part of a kernel's name: the types of its first arguments}."""

    def __init__(self, stub):
        self.stub = C.CDLL(stub, mode=C.RTLD_GLOBAL)
        self.abi = binding()
        self.lib = self.abi.load()
        self.take, self.launches = {}, []
        self.report = REPORT(self.note)
        self.stub.launch_stub_report(self.report)

    def note(self, kernel, grid, block, args):
        kernel = kernel.decode()
        types = next((t for name, t in self.take.items() if name in kernel), ())
        values = [t.from_buffer_copy(C.string_at(args[i], C.sizeof(t))) for i, t in enumerate(types)]
        self.launches.append(Launch(kernel, list(grid.contents), list(block.contents), values))

    def call(self, name, *args):
        self.launches = []
        status = getattr(self.lib, name)(*args)
        assert status == 0, (name, status, self.lib.bsa_last_error())
        assert self.launches, name
        return self.launches


class PadJob(C.Structure):          # of pad_rows_kernel
    _fields_ = [("src", C.c_void_p), ("ld", C.c_int64), ("rows", C.c_int64), ("dst", C.c_void_p)]


def copied_rows(b):
    """The gated map's backward copies the rows of the operands of the gradients that are formed, and of no others: the
    others' pointers may be NULL."""
    b.take = {"pad_rows_kernel": (PadJob, PadJob)}
    x, w, pre, dy, dx, dw, db = (i * PTR for i in range(1, 8))
    bf16 = b.abi.BSA_BF16
    for m, k, n, ldx, ldw in ((3000, 1031, 1100, 0, 0), (8191, 1023, 2047, 0, 0), (4096, 1024, 1024, 1025, 0),
                              (4096, 1024, 1024, 0, 1025), (4096, 1024, 1024, 1025, 1025)):
        p = b.abi.bsa_gated_t(m=m, k=k, n=n, dtype=bf16, act=3, ld_x=ldx, ld_w=ldw)

        def copies(x=x, w=w, dx=dx, dw=dw):
            run = b.call("bsa_gated_backward", C.byref(p), x, w, pre, dy, dx, dw, db, PTR * 16, BIG, None)
            jobs = [(j.src, j.rows) for r in run if "pad_rows_kernel" in r.kernel for j in r.args[:r.grid[2]]]
            assert all(src and rows for src, rows in jobs if src or rows), jobs
            return {src: rows for src, rows in jobs if rows}
        of_x = {x: m} if (ldx or k) % 8 else {}
        of_w = {w: 2 * n} if (ldw or k) % 8 else {}
        assert copies() == {**of_x, **of_w}, (m, k, n)
        assert copies(w=None, dx=None) == copies(dx=None) == of_x, (m, k, n)
        assert copies(x=None, dw=None) == copies(dw=None) == of_w, (m, k, n)
        assert copies(x=None, w=None, dx=None, dw=None) == {}, (m, k, n)


class RotParts(C.Structure):        # of rotary_kernel
    _fields_ = [(n, C.c_void_p) for n in ("x", "dy", "out", "gain")] + [
        (n, C.c_int64) for n in ("x_row", "x_head", "dy_row", "dy_head", "out_row", "out_head")] + [("heads", C.c_int32), ("magic", C.c_uint32)]


class RotP(C.Structure):
    _fields_ = [("part", RotParts * 2), ("pos", C.c_void_p), ("freq", C.c_void_p), ("rows", C.c_int64)] + [
        (n, C.c_int32) for n in ("hd", "rot", "half", "axes", "per_axis", "R", "G", "lrot", "pitch")] + [
        ("pitch_magic", C.c_uint32), ("axis_magic", C.c_uint32)]


def rotary_steps(b):
    """The divisions of a wave's step (an item by the heads, an angle by the row's pitch and the axis's pairs) are exact for
    every number that they are given."""
    b.take = {"rotary_kernel": (RotP,)}

    def exact(top, d, magic):
        """floor(x / d) as the high half of a product for x < top: it grows with x, so the ends of its steps decide."""
        if d == 1:
            return True
        return all((x * magic >> 32) == x // d for q in range((top + d - 1) // d) for x in (q * d, min(q * d + d, top) - 1))
    many = 0
    for heads, kv in ((1, 1), (8, 2), (32, 8), (1, 255), (1, 2049), (1, 11000), (1, 16384), (1, 20000), (1, 32769), (1, 46508),
                      (1, 65535), (2, 65535), (3, 40000), (200, 65521), (65535, 1), (65535, 65535), (300, 7)):
        for hd, rot, axes in ((2, 2, 1), (6, 4, 2), (32, 32, 1), (64, 48, 3), (255, 130, 1), (256, 256, 4)):
            for rows in (1, 2047, 4096, 10000, 131072, 1 << 24):
                for dtype in (0, 1):
                    p = b.abi.bsa_rotary_t(rows=rows, heads=heads, kv_heads=kv, head_dim=hd, rot=rot, axes=axes, dtype=dtype, eps=1e-5,
                                           magnitude=1.0)
                    q, k, pos, freq, g, h, dq, dk, yq, yk, dg, dh, ws = (i * PTR for i in range(1, 14))
                    for run in (b.call("bsa_rotary_forward", C.byref(p), q, k, pos, freq, None, None, yq, yk, None),
                                b.call("bsa_rotary_backward", C.byref(p), q, k, pos, freq, g, h, dq, dk, yq, yk, dg, dh, ws, BIG, None)):
                        r = run[0].args[0]
                        # the kernel's record is the one that this file knows
                        assert (r.rows, r.hd, r.rot, r.half, r.axes, r.part[0].heads, r.part[1].heads) == (
                            rows, hd, rot, rot // 2, axes, heads, kv)
                        at = heads, kv, hd, rows, dtype, r.R
                        assert 1 <= r.R and r.R * r.pitch <= 256, at      # the angles' place
                        assert all(exact(r.R * t.heads, t.heads, t.magic) for t in r.part), at
                        assert exact(r.R * r.pitch, r.pitch, r.pitch_magic) and exact(r.half, r.per_axis, r.axis_magic), at
                        many += r.R > 1
    assert many > 100


def launches_fit(b):
    """Calls that are accepted, and whose tensors fit a card of 288 GB, launch fewer than 2^32 threads (x) and 2^16 workgroups
    (y, z)."""
    abi, rng, card = b.abi, random.Random(1), 288e9
    p8 = [i * PTR for i in range(1, 14)]
    seen = [0, 0]

    def call(name, *args):
        b.launches = []
        status = getattr(b.lib, name)(*args)
        seen[status != 0] += 1
        assert status in (0, abi.BSA_ERR_UNSUPPORTED), (name, status, b.lib.bsa_last_error())
        assert not (status and b.launches), name
        for r in b.launches:
            assert r.threads() < 1 << 32 and max(r.grid[1:]) < 1 << 16, (name, r.kernel, r.grid, r.block)

    def maps(m, k, n, dtype):
        size = 2 if dtype == abi.BSA_BF16 else 4
        p = abi.bsa_linear_t(m=m, k=k, n=n, dtype=dtype, act=2)
        if size * (m * k + m * n + n * k) < card:
            call("bsa_linear_forward", C.byref(p), *p8[:6], ws, BIG, None)
            call("bsa_linear_backward", C.byref(p), *p8[:7], ws, BIG, None)
        p = abi.bsa_gated_t(m=m, k=k, n=n, dtype=dtype, act=3)
        if size * (m * k + m * n + 2 * n * k) < card and n <= 1 << 23:
            call("bsa_gated_forward", C.byref(p), *p8[:5], ws, BIG, None)
            call("bsa_gated_backward", C.byref(p), *p8[:7], ws, BIG, None)
    ws = 1 << 50
    for dtype in (abi.BSA_F32, abi.BSA_BF16):
        for m in (1 << 29, (1 << 30) - 129, 1 << 30, (1 << 31) - 256):
            for k in (1, 3, 8):
                for n in (1, 16, 17, 32, 33, 34, 48, 63, 64, 65, 66, 100, 128):
                    maps(m, k, n, dtype)
                    if n <= 66:
                        maps(m, n, k, dtype)
        for n in (1 << 22, 1 << 23, 1 << 24):
            for k, m in ((1, 1), (1, 17), (1, 300), (65, 17), (300, 1), (2049, 2), (4097, 40), (1, 4097), (8, 1 << 13)):
                maps(m, k, n, dtype)
                maps(m, n, k, dtype)
        for _ in range(4000):
            maps(*(int(2 ** rng.uniform(0, top)) for top in (31, 24, 24)), dtype)
    assert seen[0] > 5000, seen

    for _ in range(3000):
        d, dtype = 2 ** rng.randint(5, 7), rng.choice((abi.BSA_F32, abi.BSA_BF16))
        kv, group, seqs = (int(2 ** rng.uniform(0, top)) for top in (16, 7, 24))
        tq, tk = (int(2 ** rng.uniform(0, 30)) for _ in range(2))
        heads = kv * group
        if heads < 1 << 16 and tq * group <= 1 << 30 and kv < 1 << 16 and 2 * d * (2 * tq * heads + tk * kv) < card:
            p = abi.bsa_attention_t(seqs=seqs, heads=heads, kv_heads=kv, head_dim=d, total_q=tq, total_k=tk, dtype=dtype, zero_rest=1)
            call("bsa_cache_attention_forward", C.byref(p), *p8[:10], ws, BIG, None)
            call("bsa_attention_forward", C.byref(p), *p8[:8], ws, BIG, None)
            call("bsa_attention_backward", C.byref(p), *p8[:12], ws, BIG, None)
            p = abi.bsa_cache_t(seqs=seqs, kv_heads=kv, head_dim=d, dtype=dtype, rows=tq, total_k=tk)
            call("bsa_cache_write", C.byref(p), *p8[:9], None)
            call("bsa_cache_read", C.byref(p), *p8[:9], None)
            p = abi.bsa_rotary_t(rows=tq << rng.randint(0, 10), heads=heads, kv_heads=kv, head_dim=d, rot=d, axes=1, dtype=dtype, eps=1e-5,
                                 magnitude=1.0)
            call("bsa_rotary_forward", C.byref(p), *p8[:8], None)
            call("bsa_rotary_backward", C.byref(p), *p8[:12], ws, BIG, None)
    assert seen[0] > 8000, seen


if __name__ == "__main__":
    globals()[sys.argv[2]](Library(sys.argv[1]))
    print("checked")
