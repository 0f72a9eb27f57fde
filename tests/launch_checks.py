"""What the entry points of libbsa.so launch, on the CPU: tests/test_launches.py runs this file, one check to a process, with
launch_stub.c in the HIP runtime's place. Not for a process that has loaded torch, whose own runtime would come first."""
import ctypes as C
import importlib.util
import os
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


if __name__ == "__main__":
    globals()[sys.argv[2]](Library(sys.argv[1]))
    print("checked")
