"""CPU checks of the language-model operators' C entry points: argument errors come back as AQD_ERR_INVALID before any
launch (the device addresses below are never read), sizes of the prepared weights and of calls without rows."""
import ctypes

import pytest
import torch

from paper_2007_06919_gb300 import aqd, build

A = 0x7000_0000_0000  # an address no call may read
F32, F16, BF16, I32 = range(4)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return aqd._calls()


def out(codes=A, ldc=64, scales=A, values=0, ldv=64, vd=0):
    return aqd._ROW_CODES.pack(codes, ldc, scales, values, ldv, vd)


def norm(rows=4, cols=64, dtype=BF16, x=A, ldx=64, r=0, ldr=64, s=0, lds=64, w=A, wd=BF16, eps=1e-6):
    return aqd._RMS_NORM.pack(rows, cols, dtype, x, ldx, r, ldr, s, lds, w, wd, eps)


def gated(rows=4, cols=64, dtype=F16, g=A, ldg=64, u=A, ldu=64, act=0):
    return aqd._GATED_ACT.pack(rows, cols, dtype, g, ldg, u, ldu, act)


def weights(data=A, scales=A, n=64, k=128):
    return aqd._LINEAR_W.pack(data, scales, n, k)


def linear(m=4, x=A, ldx=128, xs=A, bias=0, y=A, ldy=64, yd=BF16):
    return aqd._LINEAR.pack(m, x, ldx, xs, bias, y, ldy, yd)


def distill(tokens=4, vocab=100, dtype=F32, x=A, ldx=100, idx=A, t=A, top=8, tau=1.0, w=0, g=0, ldg=100):
    return aqd._DISTILL.pack(tokens, vocab, dtype, x, ldx, idx, t, top, tau, w, g, ldg)


def test_row_quantizers_refuse(lib):
    f = lib.aqd_quant_rows
    assert f(0, 64, 0, 64, F32, out(codes=0, scales=0), None) == 0
    for args in ((-1, 64, A, 64, F32, out()), (1 << 31, 64, A, 64, F32, out()), (4, 0, A, 64, F32, out()),
                 (4, 64, None, 64, F32, out()), (4, 64, A, -1, F32, out()), (4, 64, A, 64, I32, out()), (4, 64, A, 64, 9, out()),
                 (4, 64, A + 2, 64, F32, out()), (4, 64, A, 64, F32, None), (4, 64, A, 64, F32, out(codes=0)),
                 (4, 64, A, 64, F32, out(ldc=63)), (4, 64, A, 64, F32, out(scales=0)), (4, 64, A, 64, F32, out(scales=A + 1)),
                 (4, 64, A, 64, F32, out(values=A, ldv=63)), (4, 64, A, 64, F32, out(values=A, vd=I32)),
                 (4, 64, A, 64, F32, out(values=A + 1, vd=F16))):
        assert f(*args, None) == 1, args
    n = lib.aqd_rms_norm_quant
    assert n(norm(rows=0, x=0, w=0), out(), None) == 0
    for a in (None, norm(rows=-1), norm(dtype=I32), norm(x=0), norm(ldx=-1), norm(x=A + 1), norm(r=A, ldr=-5), norm(r=A + 1), norm(w=0),
              norm(wd=7), norm(w=A + 1), norm(s=A + 8, lds=63), norm(s=A + 1), norm(s=A, lds=128), norm(r=A + 64, s=A + 64, lds=128),
              norm(eps=-1e-6), norm(eps=float("nan")), norm(eps=float("inf"))):
        assert n(a, out(), None) == 1, a
    g = lib.aqd_gated_act_quant
    assert g(gated(rows=0), out(), None) == 0
    for a in (None, gated(cols=0), gated(g=0), gated(u=0), gated(u=A + 1), gated(ldu=-1), gated(act=2), gated(act=-1), gated(dtype=-1)):
        assert g(a, out(), None) == 1, a


def test_product_refuses(lib):
    f = lib.aqd_linear_int8
    assert f(linear(m=0, x=0, y=0, xs=0), weights(data=0, scales=0), None, 0, None) == 0
    for a, w in ((None, weights()), (linear(), None), (linear(m=-1), weights()), (linear(m=1 << 31), weights()),
                 (linear(), weights(n=0)), (linear(), weights(k=0)), (linear(), weights(k=131072)), (linear(), weights(data=A + 16)),
                 (linear(), weights(data=0)), (linear(), weights(scales=0)), (linear(), weights(scales=A + 2)), (linear(x=0), weights()),
                 (linear(y=0), weights()), (linear(y=A + 1), weights()), (linear(yd=4), weights()), (linear(ldx=-1), weights()),
                 (linear(ldy=63), weights()), (linear(xs=0), weights()), (linear(xs=A + 1), weights()), (linear(bias=A + 3), weights())):
        assert f(a, w, None, 0, None) == 1, (a, w)
    assert f(linear(), weights(), A + 8, 1 << 20, None) == 1  # a workspace that is not aligned
    p = lib.aqd_linear_prepare_weights
    size = lib.aqd_linear_weights_bytes(64, 128)
    for a in ((None, 128, weights(), A, size), (A, -1, weights(), A, size), (A, 128, weights(n=-4), A, size),
              (A, 128, weights(), A + 8, size), (A, 128, weights(), A, size - 1), (A, 128, weights(), None, size)):
        assert p(*a, None) == 1, a


def test_weight_sizes(lib):
    f = lib.aqd_linear_weights_bytes
    for n, k in ((1, 1), (64, 128), (100, 130), (1 << 20, 4096)):
        assert f(n, k) >= n * k and f(n, k) % 128 == 0
    for n, k in ((0, 1), (1, 0), (-1, 4), (4, 131072), ((1 << 31) - 1, 131071)):
        assert f(n, k) == 0
    assert lib.aqd_linear_workspace_bytes(-1, weights()) == 0 and lib.aqd_linear_workspace_bytes(1 << 31, weights()) == 0
    assert lib.aqd_linear_workspace_bytes(4, weights(k=0)) == 0


def test_distillation_refuses(lib):
    f, b = lib.aqd_distill_topk, lib.aqd_distill_topk_backward
    assert f(distill(tokens=0, x=0), None, None, None) == 0 and b(distill(tokens=0), None, None) == 0
    wrong = [None, distill(tokens=-1), distill(tokens=1 << 31), distill(vocab=0), distill(dtype=I32), distill(x=0), distill(x=A + 1),
             distill(ldx=-1), distill(idx=0), distill(idx=A + 4), distill(t=0), distill(t=A + 2), distill(top=0), distill(top=1025),
             distill(tau=0.0), distill(tau=float("nan")), distill(tau=1e-45), distill(w=A + 1), distill(g=A + 8, ldg=99), distill(g=A + 2),
             distill(g=A, ldg=128)]
    for a in wrong:
        assert f(a, A, A, None) == 1, a
        assert b(a, A, None) == 1, a
    assert f(distill(), None, None, None) == 1          # nothing wanted
    assert f(distill(), A + 2, None, None) == 1
    assert b(distill(), A, None) == 1                   # no gradient
    assert b(distill(g=A + 16), None, None) == 1        # no lse
    assert b(distill(g=A + 16), A + 1, None) == 1


def test_tensors_off_the_gpu_are_refused(lib):
    x = torch.zeros(4, 64)
    for call in (lambda: aqd.quant_rows(x), lambda: aqd.rms_norm_quant(x, x[0]), lambda: aqd.gated_act_quant(x, x),
                 lambda: aqd.LinearWeights(x.to(torch.int8), x[:, 0].contiguous()),
                 lambda: aqd.distill_topk(x, torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2))):
        with pytest.raises(ValueError):
            call()


def test_packed_structs_have_the_header_sizes():
    """The struct layouts of include/aqd.h on a 64-bit machine."""
    p, q, i, f = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    for packed, fields in ((aqd._ROW_CODES, [p, q, p, p, q, i]), (aqd._RMS_NORM, [q, i, i, p, q, p, q, p, q, p, i, f]),
                           (aqd._GATED_ACT, [q, i, i, p, q, p, q, i]), (aqd._LINEAR_W, [p, p, i, i]),
                           (aqd._LINEAR, [q, p, q, p, p, p, q, i]), (aqd._DISTILL, [q, i, i, p, q, p, p, i, f, p, p, q])):
        c = type("S", (ctypes.Structure,), {"_fields_": [(f"f{n}", t) for n, t in enumerate(fields)]})
        assert packed.size == ctypes.sizeof(c)
