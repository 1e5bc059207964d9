"""A launch that CUDA refuses fails its own call and no other: CUDA keeps the last error until it is read, and the library's next call (or any other user of the
runtime on that thread) would take it for its own. On the CPU, in a process whose CUDA runtime is a fake that refuses the call it is told to."""
import os
import subprocess
import sys

FAKE = r"""
#include <stddef.h>
#include <string.h>
static int last, countdown;
static char status[256];
void fake_refuse(int nth) { countdown = nth; }   /* the nth launch, attribute or copy from now on; 0: none */
static int call(void) { if (countdown > 0 && --countdown == 0) last = 1; else return 0; return 1; }
int cudaLaunchKernelExC(const void* c, const void* f, void** a) { return call(); }
int __cudaGetKernel(void** k, const void* f) { *k = (void*)f; return 0; }
int __cudaLaunchKernel(void* k, ...) { return call(); }
int cudaFuncSetAttribute(const void* f, int a, int v) { return call(); }
int cudaMemsetAsync(void* p, int v, size_t n, void* s) { return call(); }
int cudaMemcpyAsync(void* d, const void* s, size_t n, int k, void* st) { return call(); }
int cudaStreamSynchronize(void* s) { return 0; }
int cudaGetLastError(void) { const int e = last; last = 0; return e; }
int cudaPeekAtLastError(void) { return last; }
const char* cudaGetErrorString(int e) { return "refused by the fake"; }
int cudaGetDevice(int* d) { *d = 0; return 0; }
int cudaFree(void* p) { return 0; }
int cudaDeviceGetAttribute(int* v, int a, int d) { *v = a == 16 ? 152 : a == 97 ? 232448 : 0; return 0; }
int cudaGetSymbolAddress(void** p, const void* s) { *p = status; return 0; }
static int context(void** c) { *c = status; return 0; }
static int encode(void* m) { return 0; }
int cudaGetDriverEntryPointByVersion(const char* name, void** f, unsigned v, unsigned long long flags, int* q) {
  *f = strcmp(name, "cuCtxGetCurrent") ? (void*)encode : (void*)context;
  *q = 0;
  return 0;
}
"""

A = 0x7000_0000_0000  # device addresses; nothing reads them


def calls(lib):
    """(name, call, the CUDA calls that it makes in turn)"""
    import struct
    out = struct.pack("=QqQQqi4x", A, 1 << 20, A, 0, 0, 0)
    rows = lambda cols: lib.aqd_quant_rows(400, cols, A, cols, 0, out, None)  # noqa: E731
    norm = struct.pack("=qiiQqQqQqQif", 400, 24576, 0, A, 24576, A, 24576, 0, 0, A, 0, 1e-6)
    gate = struct.pack("=qiiQqQqi4x", 4, 64, 1, A, 64, A, 64, 0)
    w = struct.pack("=QQii", A, A, 512, 1024)

    def linear(m, x=A, ws=0, n=0):
        return lib.aqd_linear_int8(struct.pack("=qQqQQQqi4x", m, x, 1024, A, 0, A, 512, 2), w, ws, n, None)

    def distill(vocab, lse=None):
        d = struct.pack("=qiiQqQQifQQq", 4, vocab, 0, A, vocab, A, A, 8, 1.0, 0, A, vocab)
        return lib.aqd_distill_topk(d, A, A, None) if lse is None else lib.aqd_distill_topk_backward(d, lse, None)

    code = (b"\0" * 4)
    return [("rows in registers", lambda: rows(64), 1), ("rows in shared memory", lambda: rows(12284), 2),
            ("rows in a cluster", lambda: lib.aqd_rms_norm_quant(norm, out, None), 2), ("rows read twice", lambda: rows(4001 * 41), 1),
            ("gated rows", lambda: lib.aqd_gated_act_quant(gate, out, None), 1),
            ("weights", lambda: lib.aqd_linear_prepare_weights(A, 1024, w, A, 1 << 30, None), 2),
            ("few tokens", lambda: linear(8), 1), ("tokens at odd addresses", lambda: linear(8, A + 1, A, 1 << 30), 2),
            ("no workspace", lambda: linear(40, A + 1), 1), ("many tokens", lambda: linear(4000, A, A, 1 << 40), 3),
            ("distillation", lambda: distill(500), 1), ("of a large vocabulary", lambda: distill(100000), 2), ("gradient", lambda: distill(500, A), 1),
            ("status", lambda: lib.aqd_device_status(None, code), 1)]


def child(fake, path):
    import ctypes
    cuda = ctypes.CDLL(fake, ctypes.RTLD_GLOBAL)  # before the library: its calls are bound to the first definition
    lib = ctypes.CDLL(path)
    p, q, i, z = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    for name, args in (("aqd_quant_rows", [q, i, p, q, i, p, p]), ("aqd_rms_norm_quant", [p, p, p]), ("aqd_gated_act_quant", [p, p, p]),
                       ("aqd_linear_prepare_weights", [p, q, p, p, z, p]), ("aqd_linear_int8", [p, p, p, z, p]),
                       ("aqd_distill_topk", [p, p, p, p]), ("aqd_distill_topk_backward", [p, p, p]), ("aqd_device_status", [p, p])):
        getattr(lib, name).argtypes = args
    bad = []
    for name, call, steps in calls(lib):
        if call() != 0:
            bad.append(f"{name}: refused although nothing was")
        for nth in range(1, steps + 1):
            cuda.fake_refuse(nth)
            st = call()
            if st != 3:
                bad.append(f"{name}: {st} with its CUDA call {nth} refused")
            if cuda.cudaPeekAtLastError() != 0:
                bad.append(f"{name}: the refusal of CUDA call {nth} is left to the next call")
            if call() != 0:
                bad.append(f"{name}: fails after a call whose CUDA call {nth} was refused")
            cuda.cudaGetLastError()
        cuda.fake_refuse(steps + 1)
        if call() != 0:
            bad.append(f"{name}: more than {steps} CUDA calls")
        cuda.fake_refuse(0)
        cuda.cudaGetLastError()
    print("\n".join(bad))
    sys.exit(1 if bad else 0)


def test_a_refused_launch_is_its_own_calls_error(tmp_path):
    from paper_2007_06919_gb300 import build
    source, fake = tmp_path / "fake.c", tmp_path / "fake_cuda.so"
    source.write_text(FAKE)
    subprocess.run(["gcc", "-shared", "-fPIC", "-w", "-o", str(fake), str(source)], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), str(fake), build.build()], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    child(*sys.argv[1:3])
