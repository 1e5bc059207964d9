"""Thin ctypes binding of libaqd (include/aqd.h), with the same entry-point names.

Only argument marshalling happens here: every step of the integer convolution path runs
in libaqd's CUDA kernels. PyTorch supplies device memory and the current stream. There is
no CPU fallback: if the library or a GPU is missing the calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from dataclasses import dataclass
from typing import NamedTuple

import torch

from . import build as _build

W_TWOS = 0
W_ODD = 1

STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "CUDA error", 4: "device wait timed out",
          5: "device check failed"}


class AqdError(RuntimeError):
    def __init__(self, status: int, func: str, msg: str):
        super().__init__(f"{func}: {STATUS.get(status, status)}: {msg}")
        self.status = status


class _Tensor(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("h", ctypes.c_int32), ("w", ctypes.c_int32), ("c", ctypes.c_int32),
                ("bits", ctypes.c_int32), ("data", ctypes.c_void_p)]


class _Requant(ctypes.Structure):
    _fields_ = [("m0", ctypes.c_void_p), ("shift", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("levels", ctypes.c_int32)]


class _Skip(ctypes.Structure):
    _fields_ = [("c", ctypes.c_void_p), ("d", ctypes.c_void_p), ("upsample", ctypes.c_int32),
                ("scale_main", ctypes.c_int32)]


class _Weights(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("cout", ctypes.c_int32), ("kh", ctypes.c_int32),
                ("kw", ctypes.c_int32), ("cin", ctypes.c_int32), ("w_bits", ctypes.c_int32),
                ("w_format", ctypes.c_int32)]


class _Job(ctypes.Structure):
    _fields_ = [("x", _Tensor), ("y", _Tensor), ("skip", _Tensor), ("level", ctypes.c_int32)]


EXPORTS = ["aqd_row_bytes", "aqd_quantize_multiplier", "aqd_status_string", "aqd_last_error",
           "aqd_device_status", "aqd_set_conv_path", "aqd_last_conv_path", "aqd_pack_codes",
           "aqd_unpack_codes", "aqd_conv_weights_bytes", "aqd_conv_prepare_weights", "aqd_conv_int",
           "aqd_conv_int_grouped", "aqd_conv_workspace_bytes", "aqd_conv_expand_input",
           "aqd_conv_int_grouped_expanded", "aqd_conv_int_grouped_chain", "aqd_requant", "aqd_residual_add_int",
           "aqd_maxpool_codes", "aqd_maxpool_expand", "aqd_conv_int_static_workspace", "aqd_selftest_wait_timeout",
           "aqd_conv_tower_sync_bytes", "aqd_conv_int_grouped_tower", "aqd_fake_quant",
           "aqd_fake_quant_backward_workspace_bytes", "aqd_fake_quant_backward",
           "aqd_bn_level_stats_workspace_bytes", "aqd_bn_level_stats", "aqd_quant_rows", "aqd_rms_norm_quant",
           "aqd_gated_act_quant", "aqd_linear_weights_bytes", "aqd_linear_prepare_weights",
           "aqd_linear_workspace_bytes", "aqd_linear_int8", "aqd_distill_topk", "aqd_distill_topk_backward",
           "aqd_kv_cache_bytes", "aqd_qk_norm_rope", "aqd_cache_write", "aqd_cache_read", "aqd_cache_attention_workspace_bytes",
           "aqd_cache_attention", "aqd_prompt_attention"]

_lib = None
_hot = None  # the same library for the calls below that pass their structs as packed bytes

# The C structs of include/aqd.h as packed bytes, for the calls a serving loop makes. Building a
# ctypes structure per tensor and job took most of a call's host time: the head tower's 25 jobs 128 us
# a call, 48 us this way; a whole detector at batch 1 1080 us, 530 us. Nothing is kept from one call
# for the next: every call reads and checks its tensors again.
_TENSOR = struct.Struct("=5i4xQ")       # aqd_tensor
_REQUANT = struct.Struct("=QQQi4x")     # aqd_requant_params
_SKIP = struct.Struct("=QQii")          # aqd_skip_params
_NO_TENSOR = (0, 0, 0, 0, 0, 0)


@functools.lru_cache(maxsize=None)
def _job_struct(n: int) -> struct.Struct:
    return struct.Struct("=" + "5i4xQ5i4xQ5i4xQi4x" * n)  # aqd_conv_job[n]


@functools.lru_cache(maxsize=None)
def _row_bytes(c: int, bits: int) -> int:
    return int(load().aqd_row_bytes(c, bits))


def lib_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True):
    """Loads libaqd.so (building it in-tree first if it is missing)."""
    global _lib, _hot
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        if not build_if_missing:
            raise FileNotFoundError(f"{path} is not built")
        _build.build()
    L = ctypes.CDLL(path)
    c_int, i32, i64, vp = ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    L.aqd_row_bytes.restype = i64
    L.aqd_row_bytes.argtypes = [i32, i32]
    L.aqd_quantize_multiplier.argtypes = [ctypes.c_double, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_int8)]
    L.aqd_status_string.restype = ctypes.c_char_p
    L.aqd_status_string.argtypes = [c_int]
    L.aqd_last_error.restype = ctypes.c_char_p
    L.aqd_device_status.argtypes = [vp, ctypes.POINTER(i32)]
    L.aqd_set_conv_path.restype = i32
    L.aqd_set_conv_path.argtypes = [i32]
    L.aqd_last_conv_path.restype = i32
    L.aqd_pack_codes.argtypes = [vp, i64, i32, i32, vp, vp]
    L.aqd_unpack_codes.argtypes = [vp, i64, i32, i32, i32, vp, vp]
    L.aqd_conv_weights_bytes.restype = ctypes.c_size_t
    L.aqd_conv_weights_bytes.argtypes = [i32, i32, i32, i32]
    L.aqd_conv_prepare_weights.argtypes = [vp, ctypes.POINTER(_Weights), vp, ctypes.c_size_t, vp]
    L.aqd_conv_int.argtypes = [ctypes.POINTER(_Tensor), ctypes.POINTER(_Weights), i32, i32, i32,
                               ctypes.POINTER(_Requant), ctypes.POINTER(_Tensor), ctypes.POINTER(_Skip),
                               ctypes.POINTER(_Tensor), vp, ctypes.c_size_t, vp]
    L.aqd_conv_int_grouped.argtypes = [ctypes.POINTER(_Job), i32, ctypes.POINTER(_Weights), i32, i32,
                                       ctypes.POINTER(_Requant), ctypes.POINTER(_Skip), vp, ctypes.c_size_t, vp]
    L.aqd_conv_expand_input.argtypes = [ctypes.POINTER(_Job), i32, ctypes.POINTER(_Weights), i32, i32, vp,
                                        ctypes.c_size_t, vp]
    L.aqd_conv_int_grouped_expanded.argtypes = L.aqd_conv_int_grouped.argtypes
    L.aqd_conv_int_grouped_chain.argtypes = [ctypes.POINTER(_Job), i32, ctypes.POINTER(_Weights), i32, i32,
                                             ctypes.POINTER(_Requant), ctypes.POINTER(_Skip), vp, ctypes.c_size_t,
                                             i32, vp, ctypes.c_size_t, vp]
    L.aqd_conv_int_static_workspace.argtypes = [ctypes.POINTER(_Tensor), ctypes.POINTER(_Weights), i32, i32, i32,
                                                ctypes.POINTER(_Requant), ctypes.POINTER(_Tensor),
                                                ctypes.POINTER(_Skip), ctypes.POINTER(_Tensor), vp]
    L.aqd_conv_int_static_workspace.restype = c_int
    L.aqd_conv_tower_sync_bytes.restype = ctypes.c_size_t
    L.aqd_conv_tower_sync_bytes.argtypes = [ctypes.POINTER(_Job), i32, i32, i32]
    L.aqd_conv_int_grouped_tower.argtypes = [ctypes.POINTER(_Job), i32, i32, ctypes.POINTER(_Weights),
                                             ctypes.POINTER(_Requant), i32, vp, vp, ctypes.c_size_t, vp,
                                             ctypes.c_size_t, i32, vp]
    L.aqd_conv_int_grouped_tower.restype = c_int
    L.aqd_selftest_wait_timeout.argtypes = [vp, vp]
    L.aqd_selftest_wait_timeout.restype = c_int
    L.aqd_conv_workspace_bytes.restype = ctypes.c_size_t
    L.aqd_conv_workspace_bytes.argtypes = [ctypes.POINTER(_Job), i32, ctypes.POINTER(_Weights), i32, i32]
    L.aqd_requant.argtypes = [ctypes.POINTER(_Tensor), ctypes.POINTER(_Requant), i32, ctypes.POINTER(_Tensor), vp]
    L.aqd_residual_add_int.argtypes = [ctypes.POINTER(_Tensor), ctypes.POINTER(_Tensor), ctypes.POINTER(_Skip),
                                       ctypes.POINTER(_Requant), i32, ctypes.POINTER(_Tensor), vp]
    L.aqd_maxpool_codes.argtypes = [ctypes.POINTER(_Tensor), i32, i32, i32, ctypes.POINTER(_Tensor), vp]
    L.aqd_maxpool_expand.argtypes = [ctypes.POINTER(_Tensor), i32, i32, i32, ctypes.POINTER(_Tensor),
                                     ctypes.POINTER(_Weights), i32, i32, vp, ctypes.c_size_t, vp]
    f32, i64, sz = ctypes.c_float, ctypes.c_int64, ctypes.c_size_t
    L.aqd_fake_quant.argtypes = [vp, i64, f32, i32, i32, vp, vp, vp]
    L.aqd_fake_quant_backward_workspace_bytes.restype = sz
    L.aqd_fake_quant_backward_workspace_bytes.argtypes = []
    L.aqd_fake_quant_backward.argtypes = [vp, vp, i64, f32, i32, i32, vp, vp, vp, sz, vp]
    L.aqd_bn_level_stats_workspace_bytes.restype = sz
    L.aqd_bn_level_stats_workspace_bytes.argtypes = [i32, i32]
    L.aqd_bn_level_stats.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(i64), i32, i32, vp, vp, vp, sz, vp]
    for name in ("aqd_quantize_multiplier", "aqd_device_status", "aqd_pack_codes", "aqd_unpack_codes",
                 "aqd_conv_prepare_weights", "aqd_conv_int", "aqd_conv_int_grouped", "aqd_conv_expand_input",
                 "aqd_conv_int_grouped_expanded", "aqd_conv_int_grouped_chain", "aqd_requant",
                 "aqd_residual_add_int", "aqd_maxpool_codes", "aqd_maxpool_expand", "aqd_fake_quant",
                 "aqd_fake_quant_backward", "aqd_bn_level_stats"):
        getattr(L, name).restype = c_int
    hot = ctypes.CDLL(path)
    for name, args in (("aqd_conv_int", [vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]),
                       ("aqd_conv_int_grouped", [vp, i32, vp, i32, i32, vp, vp, vp, sz, vp]),
                       ("aqd_conv_int_grouped_expanded", [vp, i32, vp, i32, i32, vp, vp, vp, sz, vp]),
                       ("aqd_conv_int_grouped_chain", [vp, i32, vp, i32, i32, vp, vp, vp, sz, i32, vp, sz, vp]),
                       ("aqd_conv_int_grouped_tower", [vp, i32, i32, vp, vp, i32, vp, vp, sz, vp, sz, i32, vp]),
                       ("aqd_conv_expand_input", [vp, i32, vp, i32, i32, vp, sz, vp]),
                       ("aqd_conv_int_static_workspace", [vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]),
                       ("aqd_conv_workspace_bytes", [vp, i32, vp, i32, i32]),
                       ("aqd_conv_tower_sync_bytes", [vp, i32, i32, i32]),
                       ("aqd_requant", [vp, vp, i32, vp, vp]),
                       ("aqd_residual_add_int", [vp, vp, vp, vp, i32, vp, vp]),
                       ("aqd_maxpool_codes", [vp, i32, i32, i32, vp, vp]),
                       ("aqd_maxpool_expand", [vp, i32, i32, i32, vp, vp, i32, i32, vp, sz, vp]),
                       ("aqd_quant_rows", [i64, i32, vp, i64, i32, vp, vp]),
                       ("aqd_rms_norm_quant", [vp, vp, vp]),
                       ("aqd_gated_act_quant", [vp, vp, vp]),
                       ("aqd_linear_weights_bytes", [i32, i32]),
                       ("aqd_linear_prepare_weights", [vp, i64, vp, vp, sz, vp]),
                       ("aqd_linear_workspace_bytes", [i64, vp]),
                       ("aqd_linear_int8", [vp, vp, vp, sz, vp]),
                       ("aqd_distill_topk", [vp, vp, vp, vp]),
                       ("aqd_distill_topk_backward", [vp, vp, vp]),
                       ("aqd_kv_cache_bytes", [i64, i32, i32, i32]),
                       ("aqd_qk_norm_rope", [vp, vp, vp]),
                       ("aqd_cache_write", [vp, vp, vp]),
                       ("aqd_cache_read", [vp, vp, vp]),
                       ("aqd_cache_attention_workspace_bytes", [i64, i32, i32, vp]),
                       ("aqd_cache_attention", [vp, vp, vp, sz, vp]),
                       ("aqd_prompt_attention", [vp, vp])):
        fn = getattr(hot, name)
        fn.argtypes = args
        fn.restype = sz if name.endswith("_bytes") else c_int
    _hot = hot
    _lib = L
    return L


def _calls():
    if _hot is None:
        load()
    return _hot


def _check(st: int, func: str):
    if st != 0:
        msg = load().aqd_last_error().decode(errors="replace")
        raise AqdError(st, func, msg)


# the current stream's handle without a Stream object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None) -> int:
    if stream is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _ptr(t: torch.Tensor | None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


# ------------------------------------------------------------------ tensors


def row_bytes(c: int, bits: int) -> int:
    return _row_bytes(c, bits)


@dataclass
class DTensor:
    """A packed NHWC code tensor (or int32 tensor) in device memory."""
    data: torch.Tensor  # uint8 [n, h, w, row_bytes] (any contiguous byte buffer of that size)
    n: int
    h: int
    w: int
    c: int
    bits: int

    @classmethod
    def empty(cls, n, h, w, c, bits, device="cuda"):
        rb = row_bytes(c, bits)
        if rb < 0:
            raise ValueError(f"no packed layout for C={c} at {bits} bits")
        return cls(torch.empty((n, h, w, rb), dtype=torch.uint8, device=device), n, h, w, c, bits)

    @classmethod
    def from_codes(cls, codes: torch.Tensor, bits: int) -> "DTensor":
        """codes: int32 CUDA tensor [n, h, w, c]."""
        n, h, w, c = codes.shape
        if bits == 32:
            data = codes.to(torch.int32).contiguous().view(torch.uint8).reshape(n, h, w, 4 * c)
            return cls(data, n, h, w, c, 32)
        out = cls.empty(n, h, w, c, bits, device=codes.device)
        pack_codes(codes.reshape(-1, c), bits, out=out.data)
        return out

    def codes(self, signed: bool = False) -> torch.Tensor:
        if self.bits == 32:
            v = self.data.contiguous().view(torch.int32)
            shape = (self.n, self.h, self.w, self.c)
            return v if v.shape == shape else v.reshape(shape)
        return unpack_codes(self.data.reshape(-1, row_bytes(self.c, self.bits)), self.c, self.bits,
                            signed).reshape(self.n, self.h, self.w, self.c)

    def _fields(self):
        """The fields of aqd_tensor, checked."""
        n, h, w, c, bits, d = self.n, self.h, self.w, self.c, self.bits, self.data
        assert d.nbytes == n * h * w * _row_bytes(c, bits)
        assert d.is_cuda and d.is_contiguous(), "device tensors must be contiguous CUDA tensors"
        return n, h, w, c, bits, d.data_ptr()

    def ct(self) -> _Tensor:
        return _Tensor(*self._fields())

    def _packed(self) -> bytes:
        return _TENSOR.pack(*self._fields())


def pack_codes(codes: torch.Tensor, bits: int, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """codes: int32 CUDA [rows, c] -> packed uint8 [rows, row_bytes]."""
    codes = codes.to(torch.int32).contiguous()
    c = codes.shape[-1]
    rows = codes.numel() // c
    rb = row_bytes(c, bits)
    if out is None:
        out = torch.empty((rows, rb), dtype=torch.uint8, device=codes.device)
    _check(load().aqd_pack_codes(_ptr(codes), rows, c, bits, _ptr(out), _stream(stream)), "aqd_pack_codes")
    return out


def unpack_codes(packed: torch.Tensor, c: int, bits: int, signed: bool = False, stream=None) -> torch.Tensor:
    packed = packed.contiguous()
    rb = row_bytes(c, bits)
    rows = packed.numel() // rb
    out = torch.empty((rows, c), dtype=torch.int32, device=packed.device)
    _check(load().aqd_unpack_codes(_ptr(packed), rows, c, bits, int(signed), _ptr(out), _stream(stream)),
           "aqd_unpack_codes")
    return out


# ------------------------------------------------------------------ parameters


@dataclass
class RequantParams:
    m0: torch.Tensor | None      # int32 [levels, cout]
    shift: torch.Tensor | None   # int8  [levels, cout]
    bias: torch.Tensor | None    # int32 [levels, cout]
    levels: int

    @classmethod
    def from_numpy(cls, m0, shift, bias, device="cuda"):
        def t(a, dt):
            return None if a is None else torch.as_tensor(a).to(dt).contiguous().to(device)
        ref = m0 if m0 is not None else bias
        return cls(t(m0, torch.int32), t(shift, torch.int8), t(bias, torch.int32), int(ref.shape[0]))

    def c(self) -> _Requant:
        return _Requant(_ptr(self.m0), _ptr(self.shift), _ptr(self.bias), self.levels)

    def _packed(self) -> bytes:
        return _REQUANT.pack(_ptr(self.m0) or 0, _ptr(self.shift) or 0, _ptr(self.bias) or 0, self.levels)


@dataclass
class SkipParams:
    c: torch.Tensor     # int32 [levels, cout]
    d: torch.Tensor     # int8  [levels, cout]
    upsample: int = 1
    scale_main: int = 0

    @classmethod
    def from_numpy(cls, c, d, upsample=1, scale_main=0, device="cuda"):
        return cls(torch.as_tensor(c).to(torch.int32).contiguous().to(device),
                   torch.as_tensor(d).to(torch.int8).contiguous().to(device), upsample, scale_main)

    def cs(self) -> _Skip:
        return _Skip(_ptr(self.c), _ptr(self.d), self.upsample, self.scale_main)

    def _packed(self) -> bytes:
        return _SKIP.pack(_ptr(self.c) or 0, _ptr(self.d) or 0, self.upsample, self.scale_main)


def quantize_multiplier(real: float) -> tuple[int, int]:
    m0 = ctypes.c_int32()
    sh = ctypes.c_int8()
    _check(load().aqd_quantize_multiplier(float(real), ctypes.byref(m0), ctypes.byref(sh)), "aqd_quantize_multiplier")
    return int(m0.value), int(sh.value)


class ConvWeights:
    """Prepared weights of one conv layer ([cout, kh, kw, cin] signed integers)."""

    def __init__(self, w_codes: torch.Tensor, w_bits: int, w_format: int = W_TWOS, stream=None):
        cout, kh, kw, cin = w_codes.shape
        packed = pack_codes(w_codes.reshape(-1, cin), w_bits, stream=stream)
        self._prepare(packed, cout, kh, kw, cin, w_bits, w_format, stream)

    @classmethod
    def from_packed(cls, packed: torch.Tensor, cout: int, kh: int, kw: int, cin: int, w_bits: int,
                    w_format: int = W_TWOS, stream=None) -> "ConvWeights":
        """packed: uint8 CUDA rows [cout*kh*kw, row_bytes(cin, w_bits)]."""
        self = cls.__new__(cls)
        self._prepare(packed.contiguous(), cout, kh, kw, cin, w_bits, w_format, stream)
        return self

    def _prepare(self, packed, cout, kh, kw, cin, w_bits, w_format, stream):
        L = load()
        nbytes = int(L.aqd_conv_weights_bytes(cout, kh, kw, cin))
        if nbytes == 0:
            raise ValueError("unsupported weight shape")
        self.buf = torch.zeros(nbytes + 256, dtype=torch.uint8, device=packed.device)
        off = (-self.buf.data_ptr()) % 256
        self.prepared = self.buf[off:off + nbytes]
        self.desc = _Weights(_ptr(self.prepared), cout, kh, kw, cin, w_bits, w_format)
        _check(L.aqd_conv_prepare_weights(_ptr(packed), ctypes.byref(self.desc), _ptr(self.prepared), nbytes,
                                          _stream(stream)), "aqd_conv_prepare_weights")
        self._packed = packed  # kept alive until the stream has consumed it
        self.cout, self.kh, self.kw, self.cin = cout, kh, kw, cin


def conv_out_hw(h, w, kh, kw, stride, pad):
    return (h + 2 * pad - kh) // stride + 1, (w + 2 * pad - kw) // stride + 1


def _ws(workspace: torch.Tensor | None):
    if workspace is None:
        return None, 0
    return _ptr(workspace), workspace.nbytes


def _opt(p) -> bytes | None:
    return None if p is None else p._packed()


def conv_int(x: DTensor, w: ConvWeights, stride: int, pad: int, y: DTensor, *, level: int = 0,
             rq: RequantParams | None = None, skip: DTensor | None = None, sp: SkipParams | None = None,
             workspace: torch.Tensor | None = None, stream=None) -> DTensor:
    wsp, wsb = _ws(workspace)
    st = _calls().aqd_conv_int(x._packed(), ctypes.byref(w.desc), stride, pad, level, _opt(rq), _opt(skip), _opt(sp),
                               y._packed(), wsp, wsb, _stream(stream))
    _check(st, "aqd_conv_int")
    return y


def conv_int_static_workspace(x: DTensor, w: ConvWeights, stride: int, pad: int, y: DTensor, *, level: int = 0,
                              rq: RequantParams | None = None, skip: DTensor | None = None,
                              sp: SkipParams | None = None, stream=None) -> DTensor:
    """conv_int on the workspace path with the library's own fixed workspace (no allocation);
    calls that overlap in time share that workspace and must be ordered by the caller."""
    st = _calls().aqd_conv_int_static_workspace(x._packed(), ctypes.byref(w.desc), stride, pad, level, _opt(rq),
                                                _opt(skip), _opt(sp), y._packed(), _stream(stream))
    _check(st, "aqd_conv_int_static_workspace")
    return y


def _jobs(jobs) -> bytes:
    """aqd_conv_job[len(jobs)] (a tensor that several jobs of one call share is read once)."""
    if len(jobs) == 1:
        x, y, skip, level = jobs[0]
        return _job_struct(1).pack(*x._fields(), *(_NO_TENSOR if y is None else y._fields()),
                                   *(_NO_TENSOR if skip is None else skip._fields()), level)
    seen = {}
    vals = []
    for x, y, skip, level in jobs:
        for t in (x, y, skip):
            if t is None:
                vals += _NO_TENSOR
                continue
            f = seen.get(id(t))
            if f is None:
                f = seen[id(t)] = t._fields()
            vals += f
        vals.append(level)
    return _job_struct(len(jobs)).pack(*vals)


def conv_workspace_bytes(jobs, w: ConvWeights, stride: int, pad: int) -> int:
    """Bytes of the expanded-activation workspace for these jobs (0: path not applicable)."""
    return int(_calls().aqd_conv_workspace_bytes(_jobs(jobs), len(jobs), ctypes.byref(w.desc), stride, pad))


def workspace_for(jobs, w: ConvWeights, stride: int, pad: int, device="cuda") -> torch.Tensor | None:
    """A 256-byte aligned workspace of the right size, or None when the path does not apply."""
    n = conv_workspace_bytes(jobs, w, stride, pad)
    if n == 0:
        return None
    buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + n]


def conv_int_grouped(jobs, w: ConvWeights, stride: int, pad: int, *, rq: RequantParams | None = None,
                     sp: SkipParams | None = None, workspace: torch.Tensor | None = None, stream=None):
    """jobs: list of (x: DTensor, y: DTensor, skip: DTensor | None, level: int)."""
    wsp, wsb = _ws(workspace)
    st = _calls().aqd_conv_int_grouped(_jobs(jobs), len(jobs), ctypes.byref(w.desc), stride, pad, _opt(rq), _opt(sp),
                                       wsp, wsb, _stream(stream))
    _check(st, "aqd_conv_int_grouped")


def conv_expand_input(jobs, w: ConvWeights, stride: int, pad: int, workspace: torch.Tensor, stream=None):
    """Only the expansion step of the workspace path: writes the zero-padded byte image of the
    jobs' inputs into `workspace` (jobs as for conv_int_grouped; y and skip are ignored)."""
    wsp, wsb = _ws(workspace)
    st = _calls().aqd_conv_expand_input(_jobs(jobs), len(jobs), ctypes.byref(w.desc), stride, pad, wsp, wsb,
                                        _stream(stream))
    _check(st, "aqd_conv_expand_input")


def conv_int_grouped_expanded(jobs, w: ConvWeights, stride: int, pad: int, *, rq: RequantParams | None = None,
                              sp: SkipParams | None = None, workspace: torch.Tensor, stream=None):
    """conv_int_grouped fed from a workspace that already holds the expansion of these jobs'
    inputs (written by conv_expand_input); launches only the tensor-core convolution."""
    wsp, wsb = _ws(workspace)
    st = _calls().aqd_conv_int_grouped_expanded(_jobs(jobs), len(jobs), ctypes.byref(w.desc), stride, pad, _opt(rq),
                                                _opt(sp), wsp, wsb, _stream(stream))
    _check(st, "aqd_conv_int_grouped_expanded")


def conv_int_grouped_chain(jobs, w: ConvWeights, stride: int, pad: int, *, rq: RequantParams | None = None,
                           sp: SkipParams | None = None, workspace: torch.Tensor, next_pad: int,
                           next_workspace: torch.Tensor, stream=None):
    """conv_int_grouped_expanded that also writes the outputs, one byte per code, as the
    zero-padded byte image the next stride-1 conv (padding next_pad) reads from
    next_workspace (whose border must hold zeros)."""
    wsp, wsb = _ws(workspace)
    nwp, nwb = _ws(next_workspace)
    st = _calls().aqd_conv_int_grouped_chain(_jobs(jobs), len(jobs), ctypes.byref(w.desc), stride, pad, _opt(rq), _opt(sp),
                                             wsp, wsb, next_pad, nwp, nwb, _stream(stream))
    _check(st, "aqd_conv_int_grouped_chain")


def tower_sync_bytes(jobs, layers: int, pad: int) -> int:
    """Bytes of per-tile counters for conv_int_grouped_tower (jobs: layer 0's jobs)."""
    return int(_calls().aqd_conv_tower_sync_bytes(_jobs(jobs), len(jobs), layers, pad))


def conv_int_grouped_tower(layer_jobs, ws: list, rqs: list, pad: int, *, ws_a: torch.Tensor,
                           ws_b: torch.Tensor, sync: torch.Tensor | None, input_expanded: bool = False,
                           stream=None):
    """layer_jobs: one list of (x, y, None, level) per layer, layer i's x being layer i-1's y;
    ws: ConvWeights per layer; rqs: RequantParams per layer. See aqd_conv_int_grouped_tower."""
    nl, nj = len(layer_jobs), len(layer_jobs[0])
    jobs = _jobs([jb for jobs in layer_jobs for jb in jobs])
    if len(ws) > nl or len(rqs) > nl:
        raise IndexError("more weights or requant tables than layers")
    # (what is missing reads as zeros, which the library refuses)
    jobs = jobs.ljust(nl * nj * _job_struct(1).size, b"\0")
    wd = b"".join([bytes(w.desc) for w in ws]).ljust(nl * ctypes.sizeof(_Weights), b"\0")
    rqa = b"".join([r._packed() for r in rqs]).ljust(nl * _REQUANT.size, b"\0")
    wap, wab = _ws(ws_a)
    wbp, wbb = _ws(ws_b)
    assert wab == wbb, "ws_a and ws_b must have the same size"
    sp_, sb = _ws(sync) if sync is not None else (None, 0)
    st = _calls().aqd_conv_int_grouped_tower(jobs, nj, nl, wd, rqa, pad, wap, wbp, wab, sp_, sb, int(input_expanded),
                                             _stream(stream))
    _check(st, "aqd_conv_int_grouped_tower")


def requant(acc: DTensor, rq: RequantParams, y: DTensor, *, level: int = 0, stream=None) -> DTensor:
    _check(_calls().aqd_requant(acc._packed(), rq._packed(), level, y._packed(), _stream(stream)), "aqd_requant")
    return y


def residual_add_int(a: DTensor, b: DTensor, sp: SkipParams, y: DTensor, *, rq: RequantParams | None = None,
                     level: int = 0, stream=None) -> DTensor:
    st = _calls().aqd_residual_add_int(a._packed(), b._packed(), sp._packed(), _opt(rq), level, y._packed(),
                                       _stream(stream))
    _check(st, "aqd_residual_add_int")
    return y


def maxpool_codes(x: DTensor, k: int, stride: int, pad: int, y: DTensor, stream=None) -> DTensor:
    st = _calls().aqd_maxpool_codes(x._packed(), k, stride, pad, y._packed(), _stream(stream))
    _check(st, "aqd_maxpool_codes")
    return y


def maxpool_expand(x: DTensor, k: int, stride: int, pad: int, y: DTensor, w: ConvWeights, conv_stride: int,
                   conv_pad: int, workspace: torch.Tensor, stream=None) -> DTensor:
    """maxpool_codes(x) -> y fused with conv_expand_input([(y, ...)], w, conv_stride, conv_pad,
    workspace): one pass writes y and the byte image of y for that convolution."""
    wsp, wsb = _ws(workspace)
    st = _calls().aqd_maxpool_expand(x._packed(), k, stride, pad, y._packed(), ctypes.byref(w.desc), conv_stride,
                                     conv_pad, wsp, wsb, _stream(stream))
    _check(st, "aqd_maxpool_expand")
    return y


def _f32(t: torch.Tensor | None):
    if t is None:
        return None
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous float32 CUDA tensor")
    return t.data_ptr()


def fake_quant(x: torch.Tensor, nu: float, bits: int, *, weight: bool = False, y: torch.Tensor | None = None,
               codes: torch.Tensor | None = None, stream=None):
    """Eq. 2 (weight=False) / Eq. 3 (weight=True) on a float32 tensor: returns (y, codes), the
    fake-quantized values and the uint8 codes (allocated when not given)."""
    y = torch.empty_like(x) if y is None else y
    codes = torch.empty(x.shape, dtype=torch.uint8, device=x.device) if codes is None else codes
    _check(load().aqd_fake_quant(_f32(x), x.numel(), float(nu), bits, int(weight), _f32(y), codes.data_ptr(),
                                 _stream(stream)), "aqd_fake_quant")
    return y, codes


def fake_quant_backward(x: torch.Tensor, gy: torch.Tensor, nu: float, bits: int, *, weight: bool = False,
                        gx: torch.Tensor | None = None, stream=None):
    """The STE backward of fake_quant: returns (gx, gnu) with gnu a one-element float64 CUDA
    tensor (the interval's gradient)."""
    gx = torch.empty_like(x) if gx is None else gx
    gnu = torch.empty(1, dtype=torch.float64, device=x.device)
    ws = torch.empty(int(load().aqd_fake_quant_backward_workspace_bytes()), dtype=torch.uint8, device=x.device)
    _check(load().aqd_fake_quant_backward(_f32(x), _f32(gy), x.numel(), float(nu), bits, int(weight), _f32(gx),
                                          gnu.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)),
           "aqd_fake_quant_backward")
    return gx, gnu


def bn_level_stats(zs, stream=None):
    """Per-level batch mean and biased variance (float64 [levels, c]) of float32 CUDA tensors
    with channels last (Sec. 3.2.2's multi-level BN)."""
    c = zs[0].shape[-1]
    dev = zs[0].device
    nlev = len(zs)
    ptrs = (ctypes.c_void_p * nlev)(*[_f32(z) for z in zs])
    pix = (ctypes.c_int64 * nlev)(*[z.numel() // c for z in zs])
    mean = torch.empty((nlev, c), dtype=torch.float64, device=dev)
    var = torch.empty((nlev, c), dtype=torch.float64, device=dev)
    wsb = int(load().aqd_bn_level_stats_workspace_bytes(nlev, c))
    ws = torch.empty(max(wsb, 8), dtype=torch.uint8, device=dev)
    _check(load().aqd_bn_level_stats(ptrs, pix, nlev, c, mean.data_ptr(), var.data_ptr(), ws.data_ptr(), ws.numel(),
                                     _stream(stream)), "aqd_bn_level_stats")
    return mean, var


# ------------------------------------------------------------------ 8-bit language-model operators

_F32, _F16, _BF16, _I32 = range(4)
_DTYPE = {torch.float32: _F32, torch.float16: _F16, torch.bfloat16: _BF16}
_OUT_DTYPE = {**_DTYPE, torch.int32: _I32}
_ACT = {"silu": 0, "gelu_tanh": 1}

_ROW_CODES = struct.Struct("=QqQQqi4x")            # aqd_row_codes
_RMS_NORM = struct.Struct("=qiiQqQqQqQif")         # aqd_rms_norm_args
_GATED_ACT = struct.Struct("=qiiQqQqi4x")           # aqd_gated_act_args
_LINEAR_W = struct.Struct("=QQii")                 # aqd_linear_weights
_LINEAR = struct.Struct("=qQqQQQqi4x")             # aqd_linear_args
_DISTILL = struct.Struct("=qiiQqQQifQQq")          # aqd_distill_args
_KV_CACHE = struct.Struct("=Qqiii4x")              # aqd_kv_cache
_QK_ROPE = struct.Struct("=qiiiiQqqQqqQqqQqqQqqQQifQQiiQ")  # aqd_qk_rope_args
_CACHE_ROWS = struct.Struct("=qi4xQqqQqqQ")        # aqd_cache_rows
_CACHE_ATTENTION = struct.Struct("=qiiifQqqQqqQQQQqi4x")  # aqd_cache_attention_args
_PROMPT = struct.Struct("=qqiiiiiif4xQqqQqqQqqQqqQQQ")  # aqd_prompt_attention_args


class RowCodes(NamedTuple):
    """Rows of 8-bit codes: codes int8 [..., cols], scales float32 [...], values (code x scale, or None) and,
    from rms_norm_quant with a residual, the sum of x and the residual."""
    codes: torch.Tensor
    scales: torch.Tensor
    values: torch.Tensor | None = None
    summed: torch.Tensor | None = None


def _rows_of(t: torch.Tensor, name: str, device: int | None = None):
    """(rows, columns, row stride) of a CUDA tensor's last dimension, the others taken together; ValueError where
    its rows are not evenly strided or their elements not adjacent. device: the index of the call's device."""
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise ValueError(f"{name} must be a CUDA tensor on the call's device")
    shape, strides = t.shape, t.stride()
    if len(shape) == 2:
        m, c = shape
        ld, last = strides
    elif len(shape) == 1:
        m, c, ld, last = 1, shape[0], shape[0], strides[0]
    elif not shape:
        raise ValueError(f"{name} needs at least one dimension")
    else:
        c, n = shape[-1], shape[-2]
        m = t.numel() // max(c, 1)
        ld, last = strides[-2], strides[-1]
        for i in range(len(shape) - 3, -1, -1):
            if shape[i] > 1 and n > 1 and strides[i] != n * ld:
                raise ValueError(f"the rows of {name} are not evenly strided")
            if n <= 1 and shape[i] > 1:
                ld = strides[i]
            n *= shape[i]
    if c < 1:
        raise ValueError(f"{name} has no columns")
    if last != 1 and c > 1:
        raise ValueError(f"the elements of a row of {name} must be adjacent")
    return m, c, (ld if m > 1 else max(ld, c))


def _runs_on(device: int, stream):
    """ValueError unless kernels go where the call's tensors are: the current device, and the stream's."""
    here = _raw_device() if _raw_device is not None else torch.cuda.current_device()
    if device != here or (stream is not None and stream.device.index != here):
        raise ValueError(f"the call's tensors are on device {device}, the current device is {here}"
                         + ("" if stream is None else f", the stream's {stream.device}"))


def _float_dtype(t: torch.Tensor, name: str) -> int:
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    return d


def _vector(t: torch.Tensor, n: int, dtype, name: str, device: int) -> int:
    """The address of a contiguous CUDA vector of n values."""
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or not t.is_cuda or t.get_device() != device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} values on the call's device")
    return t.data_ptr()


_empty = torch.empty


def _new(shape, dtype, device, stream):
    """A new tensor that belongs to the call's stream: memory that another stream may still be using is not written."""
    if stream is None:
        return _empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return _empty(shape, dtype=dtype, device=device)


def _row_codes_out(like: torch.Tensor, cols: int, codes: bool, values, stream):
    """New outputs of a quantizer for rows shaped like `like`, and their aqd_row_codes."""
    dev, shape = like.device, like.shape
    s = _new(shape[:-1], torch.float32, dev, stream)
    c = v = None
    cp = vp = vd = 0
    if codes:
        c = _new(shape, torch.int8, dev, stream)
        cp = c.data_ptr()
    elif not values:
        raise ValueError("at least one of codes and values is wanted")
    if values is not False and values is not None:
        vt = like.dtype if values is True else values
        vd = _DTYPE.get(vt)
        if vd is None:
            raise ValueError(f"values must be a bool, float32, float16 or bfloat16, got {values}")
        v = _new(shape, vt, dev, stream)
        vp = v.data_ptr()
    return c, s, v, _ROW_CODES.pack(cp, cols, s.data_ptr(), vp, cols, vd)


def quant_rows(x: torch.Tensor, *, codes: bool = True, values=False, stream=None) -> RowCodes:
    """8-bit codes of x's rows (its last dimension), one scale per row (aqd_quant_rows). values: True, or a type,
    for the values that the codes stand for too."""
    m, c, ld = _rows_of(x, "x")
    d = _float_dtype(x, "x")
    _runs_on(x.get_device(), stream)
    q, s, v, out = _row_codes_out(x, c, codes, values, stream)
    _check(_calls().aqd_quant_rows(m, c, x.data_ptr(), ld, d, out, _stream(stream)), "aqd_quant_rows")
    return RowCodes(q, s, v)


def rms_norm_quant(x: torch.Tensor, weight: torch.Tensor, *, eps: float = 1e-6, residual: torch.Tensor | None = None,
                   summed: torch.Tensor | None = None, codes: bool = True, values=False, stream=None) -> RowCodes:
    """8-bit codes of rms_norm(x + residual) * weight (aqd_rms_norm_quant), one scale per row. With a residual the
    sum comes back too, in `summed` where that is given (x or residual itself: in place)."""
    m, c, ld = _rows_of(x, "x")
    d = _float_dtype(x, "x")
    dev = x.get_device()
    _runs_on(dev, stream)
    rp = rl = sp = sl = 0
    if residual is not None:
        if residual.shape != x.shape or residual.dtype is not x.dtype:
            raise ValueError("residual must have x's shape and type")
        rl = _rows_of(residual, "residual", dev)[2]
        rp = residual.data_ptr()
        if summed is None:
            summed = _new(x.shape, x.dtype, x.device, stream)
            sp, sl = summed.data_ptr(), c
    if summed is not None and not sp:
        if summed.shape != x.shape or summed.dtype is not x.dtype:
            raise ValueError("summed must have x's shape and type")
        sl = _rows_of(summed, "summed", dev)[2]
        sp = summed.data_ptr()
    wd = _float_dtype(weight, "weight")
    wp = _vector(weight, c, weight.dtype, "weight", dev)
    q, s, v, out = _row_codes_out(x, c, codes, values, stream)
    args = _RMS_NORM.pack(m, c, d, x.data_ptr(), ld, rp, rl, sp, sl, wp, wd, eps)
    _check(_calls().aqd_rms_norm_quant(args, out, _stream(stream)), "aqd_rms_norm_quant")
    return RowCodes(q, s, v, summed)


def gated_act_quant(gate: torch.Tensor, up: torch.Tensor, *, act: str = "silu", codes: bool = True, values=False,
                    stream=None) -> RowCodes:
    """8-bit codes of act(gate) * up (aqd_gated_act_quant), one scale per row; act: "silu" or "gelu_tanh"."""
    m, c, lg = _rows_of(gate, "gate")
    d = _float_dtype(gate, "gate")
    if up.shape != gate.shape or up.dtype is not gate.dtype:
        raise ValueError("up must have gate's shape and type")
    dev = gate.get_device()
    _runs_on(dev, stream)
    lu = _rows_of(up, "up", dev)[2]
    if act not in _ACT:
        raise ValueError(f"act must be one of {sorted(_ACT)}, got {act!r}")
    q, s, v, out = _row_codes_out(gate, c, codes, values, stream)
    args = _GATED_ACT.pack(m, c, d, gate.data_ptr(), lg, up.data_ptr(), lu, _ACT[act])
    _check(_calls().aqd_gated_act_quant(args, out, _stream(stream)), "aqd_gated_act_quant")
    return RowCodes(q, s, v)


class LinearWeights:
    """Prepared weights of an 8-bit layer: codes int8 [n, k] and a float32 scale per output channel (the scales are
    read by every call, so a program may train them in place)."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, stream=None):
        if codes.dim() != 2 or codes.dtype != torch.int8:
            raise ValueError("codes must be an int8 matrix [n, k]")
        n, k, ld = _rows_of(codes, "codes")
        _runs_on(codes.get_device(), stream)
        sp = _vector(scales, n, torch.float32, "scales", codes.get_device())
        nbytes = int(_calls().aqd_linear_weights_bytes(n, k))
        if nbytes == 0:
            raise ValueError(f"unsupported weight shape {n} x {k}")
        buf = _new(nbytes + 256, torch.uint8, codes.device, stream)
        off = (-buf.data_ptr()) % 256
        self.prepared = buf[off:off + nbytes]
        self.n, self.k, self.scales, self.device, self.index = n, k, scales, codes.device, codes.get_device()
        self.desc = _LINEAR_W.pack(self.prepared.data_ptr(), sp, n, k)
        _check(_calls().aqd_linear_prepare_weights(codes.data_ptr(), ld, self.desc, self.prepared.data_ptr(), nbytes,
                                                   _stream(stream)), "aqd_linear_prepare_weights")
        self._codes = codes if stream is not None else None  # kept alive until that stream has consumed it

    @classmethod
    def from_float(cls, w: torch.Tensor, stream=None) -> "LinearWeights":
        """Weights [n, k] in floating point, each output channel by its own largest magnitude."""
        q = quant_rows(w, stream=stream)
        return cls(q.codes, q.scales, stream=stream)


@functools.lru_cache(maxsize=4096)
def _linear_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(_calls().aqd_linear_workspace_bytes(m, _LINEAR_W.pack(0, 0, n, k)))


def linear_workspace(m: int, *w: LinearWeights, stream=None) -> torch.Tensor | None:
    """A workspace for linear_int8 with up to m tokens, for one layer or for several whose calls follow one another on one stream; None where
    they need none. It belongs to the stream: released after calls were made there, its memory goes to that stream's later work only."""
    n = max(_linear_workspace_bytes(m, v.n, v.k) for v in w)
    if n == 0:
        return None
    buf = _new(n + 256, torch.uint8, w[0].device, stream)
    off = -buf.data_ptr() % 256
    return buf[off:off + n] if off else buf


def linear_int8(x: torch.Tensor, x_scale: torch.Tensor | None, w: LinearWeights, *, bias: torch.Tensor | None = None,
                out: torch.Tensor | None = None, out_dtype=torch.bfloat16, workspace: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """x (int8 codes [..., k], one scale per row) times w's codes, scaled per token and channel (aqd_linear_int8).
    out_dtype torch.int32: the integer sums. workspace: linear_workspace(m, w), which calls that may overlap in time must
    not share."""
    if x.dtype is not torch.int8:
        raise ValueError("x must hold int8 codes")
    dev = w.index
    m, k, ld = _rows_of(x, "x", dev)
    _runs_on(dev, stream)
    n = w.n
    if k != w.k:
        raise ValueError(f"x has {k} columns, the weights {w.k}")
    yd = _OUT_DTYPE.get(out_dtype if out is None else out.dtype)
    if yd is None:
        raise ValueError("the output must be float32, float16, bfloat16 or int32")
    if out is None:
        out = _new((m, n) if x.dim() == 2 else (*x.shape[:-1], n), out_dtype, w.device, stream)
        ldy = n
    else:
        if out.shape != (*x.shape[:-1], n):
            raise ValueError("out must have x's shape but for the last dimension, n")
        ldy = _rows_of(out, "out", dev)[2]
    xs = bp = 0
    if yd != _I32:
        if x_scale is None:
            raise ValueError("x_scale is required")
        xs = _vector(x_scale, m, torch.float32, "x_scale", dev)
        if bias is not None:
            bp = _vector(bias, n, torch.float32, "bias", dev)
    wsp, wsb = None, 0
    if workspace is not None:
        if not workspace.is_cuda or workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA tensor on the call's device")
        wsp, wsb = workspace.data_ptr(), workspace.nbytes
    _check(_calls().aqd_linear_int8(_LINEAR.pack(m, x.data_ptr(), ld, xs, bp, out.data_ptr(), ldy, yd), w.desc, wsp, wsb,
                                    _stream(stream)), "aqd_linear_int8")
    return out


# ------------------------------------------------------------------ attention of an 8-bit decoder


def _heads(t: torch.Tensor, name: str, device: int | None = None):
    """(tokens, heads, head_dim, stride of a token, of a head) of a CUDA tensor [tokens, heads, head_dim]; ValueError where the
    values of a head are not adjacent. device: the index of the call's device."""
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise ValueError(f"{name} must be a CUDA tensor on the call's device")
    if len(t.shape) != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    n, h, d = t.shape
    ld, ldh, last = t.stride()
    if last != 1 and d > 1:
        raise ValueError(f"the values of a head of {name} must be adjacent")
    return n, h, d, ld, ldh


def _out_heads(out: torch.Tensor | None, like: torch.Tensor, name: str, stream):
    """The tensor for an output of like's shape and type (a new one where out is None), and its two strides."""
    if out is None:
        n, h, d = like.shape
        return _new((n, h, d), like.dtype, like.device, stream), h * d, d
    if out.shape != like.shape or out.dtype is not like.dtype:
        raise ValueError(f"{name} must have its input's shape and type")
    _, _, _, ld, ldh = _heads(out, name, like.get_device())
    return out, ld, ldh


class KVCache:
    """A 4-bit cache of keys and values (aqd_kv_cache): `pages` pages of page_size places (a power of two, 16..1024), each
    place a key and a value row of every head. Its memory belongs to the stream current at construction, or to `stream`: it has to outlive
    the calls on others."""

    def __init__(self, pages: int, page_size: int, kv_heads: int, head_dim: int, device="cuda", stream=None):
        nbytes = int(_calls().aqd_kv_cache_bytes(pages, page_size, kv_heads, head_dim))
        if nbytes == 0:
            raise ValueError(f"unsupported cache shape: {pages} pages of {page_size}, {kv_heads} heads of {head_dim}")
        buf = _new(nbytes + 256, torch.uint8, device, stream)
        off = -buf.data_ptr() % 256
        self.data = buf[off:off + nbytes]
        self.pages, self.page_size, self.kv_heads, self.head_dim = pages, page_size, kv_heads, head_dim
        self.device, self.index = buf.device, buf.get_device()
        self.desc = _KV_CACHE.pack(self.data.data_ptr(), pages, page_size, kv_heads, head_dim)


class Rotated(NamedTuple):
    q: torch.Tensor
    k: torch.Tensor | None


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None, inv_freq: torch.Tensor | None, *,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6,
                 interleaved: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None,
                 v: torch.Tensor | None = None, cache: KVCache | None = None, slots: torch.Tensor | None = None,
                 stream=None) -> Rotated:
    """Queries [tokens, heads, head_dim] and keys [tokens, kv_heads, head_dim] normed for each head (where a weight is given) and
    turned by their position (aqd_qk_norm_rope): positions int64 [tokens], inv_freq float32, one for each turned pair. q_out, k_out: q and
    k themselves, in place. With a cache, keys and values v go to its places slots (int64 [tokens]) in the same pass, and k comes back only
    where k_out is given."""
    n, h, d, lq, lqh = _heads(q, "q")
    dt = _float_dtype(q, "q")
    dev = q.get_device()
    _runs_on(dev, stream)
    nk, hk, dk, lk, lkh = _heads(k, "k", dev)
    if nk != n or dk != d or k.dtype is not q.dtype:
        raise ValueError("k must have q's tokens, head_dim and type")
    rot, pp, fp = 0, 0, 0
    if inv_freq is not None and inv_freq.numel() > 0:
        rot = 2 * inv_freq.numel()
        if positions is None:
            raise ValueError("positions are required")
        fp = _vector(inv_freq, rot // 2, torch.float32, "inv_freq", dev)
        pp = _vector(positions, n, torch.int64, "positions", dev)
    wd, wq, wk = 0, 0, 0
    if q_weight is not None:
        wd = _float_dtype(q_weight, "q_weight")
        wq = _vector(q_weight, d, q_weight.dtype, "q_weight", dev)
    if k_weight is not None:
        if q_weight is not None and k_weight.dtype is not q_weight.dtype:
            raise ValueError("the weights must have one type")
        wd = _float_dtype(k_weight, "k_weight")
        wk = _vector(k_weight, d, k_weight.dtype, "k_weight", dev)
    vp = lv = lvh = sp = 0
    desc = None
    if cache is not None:
        if v is None or slots is None:
            raise ValueError("v and slots are required with a cache")
        nv, hv, dv, lv, lvh = _heads(v, "v", dev)
        if (nv, hv, dv) != (n, hk, d) or v.dtype is not q.dtype:
            raise ValueError("v must have k's shape and type")
        if cache.index != dev:
            raise ValueError("the cache must be on the call's device")
        vp, sp, desc = v.data_ptr(), _vector(slots, n, torch.int64, "slots", dev), cache.desc
    qo, lqo, lqoh = _out_heads(q_out, q, "q_out", stream)
    kp = lko = lkoh = 0
    if k_out is not None or cache is None:
        k_out, lko, lkoh = _out_heads(k_out, k, "k_out", stream)
        kp = k_out.data_ptr()
    args = _QK_ROPE.pack(n, h, hk, d, dt, q.data_ptr(), lq, lqh, k.data_ptr(), lk, lkh, vp, lv, lvh, qo.data_ptr(), lqo, lqoh,
                         kp, lko, lkoh, wq, wk, wd, eps, pp, fp, rot, 1 if interleaved else 0, sp)
    _check(_calls().aqd_qk_norm_rope(args, desc, _stream(stream)), "aqd_qk_norm_rope")
    return Rotated(qo, k_out)


def cache_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *, stream=None) -> None:
    """Rows of keys and values [tokens, kv_heads, head_dim] in 4 bits to the cache's places slots, int64 [tokens]
    (aqd_cache_write); a token whose slot lies outside the cache is skipped."""
    n, h, d, lk, lkh = _heads(k, "k", cache.index)
    dt = _float_dtype(k, "k")
    _runs_on(cache.index, stream)
    _, _, _, lv, lvh = _heads(v, "v", cache.index)
    if v.shape != k.shape or v.dtype is not k.dtype:
        raise ValueError("v must have k's shape and type")
    if h != cache.kv_heads or d != cache.head_dim:
        raise ValueError("k and v must have the cache's heads")
    sp = _vector(slots, n, torch.int64, "slots", cache.index)
    _check(_calls().aqd_cache_write(_CACHE_ROWS.pack(n, dt, k.data_ptr(), lk, lkh, v.data_ptr(), lv, lvh, sp), cache.desc,
                                    _stream(stream)), "aqd_cache_write")


def cache_read(cache: KVCache, slots: torch.Tensor, *, dtype=torch.bfloat16, stream=None):
    """(keys, values), [tokens, kv_heads, head_dim] of dtype: what the cache's places slots hold (aqd_cache_read); zeros for
    a slot outside the cache. A prompt that goes on from cached places reads them so for prompt_attention."""
    d = _DTYPE.get(dtype)
    if d is None:
        raise ValueError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
    _runs_on(cache.index, stream)
    n, h, w = slots.numel(), cache.kv_heads, cache.head_dim
    sp = _vector(slots, n, torch.int64, "slots", cache.index)
    k, v = _new((n, h, w), dtype, cache.device, stream), _new((n, h, w), dtype, cache.device, stream)
    _check(_calls().aqd_cache_read(_CACHE_ROWS.pack(n, d, k.data_ptr(), h * w, w, v.data_ptr(), h * w, w, sp), cache.desc,
                                   _stream(stream)), "aqd_cache_read")
    return k, v


@functools.lru_cache(maxsize=4096)
def _cache_attention_bytes(tokens: int, seqs: int, heads: int, page_size: int, kv_heads: int, head_dim: int) -> int:
    return int(_calls().aqd_cache_attention_workspace_bytes(tokens, seqs, heads, _KV_CACHE.pack(0, 1, page_size, kv_heads, head_dim)))


def cache_attention_workspace(q: torch.Tensor, cache: KVCache, seqs: int, *, stream=None) -> torch.Tensor:
    """A workspace for cache_attention with queries of q's shape and that many sequences, for calls that follow one another on
    one stream."""
    n = _cache_attention_bytes(q.shape[0], seqs, q.shape[1], cache.page_size, cache.kv_heads, cache.head_dim)
    if n == 0:
        raise ValueError("heads must be a multiple of the cache's")
    buf = _new(n + 256, torch.uint8, cache.device, stream)
    off = -buf.data_ptr() % 256
    return buf[off:off + n] if off else buf


def cache_attention(q: torch.Tensor, cache: KVCache, page_table: torch.Tensor, lengths: torch.Tensor, *,
                    starts: torch.Tensor | None = None, scale: float | None = None, out: torch.Tensor | None = None,
                    lse: bool | torch.Tensor = False, workspace: torch.Tensor | None = None, stream=None):
    """Attention of each sequence's last tokens over the cache (aqd_cache_attention): q [tokens, heads, head_dim], page_table int32
    [seqs, columns] (expanded: one row for all), lengths int32 [seqs] (places of each sequence, its queries' own among them), starts int32 [seqs + 1] for several
    queries a sequence. scale: 1 / sqrt(head_dim) where not given. Returns the output, or (output, lse [tokens, heads]) where lse is wanted.
    workspace: cache_attention_workspace(q, cache, seqs), which calls that may overlap in time must not share."""
    dev = cache.index
    n, h, d, lq, lqh = _heads(q, "q", dev)
    dt = _float_dtype(q, "q")
    _runs_on(dev, stream)
    if d != cache.head_dim:
        raise ValueError("q must have the cache's head_dim")
    if page_table.dtype is not torch.int32 or page_table.dim() != 2 or not page_table.is_cuda or page_table.get_device() != dev:
        raise ValueError("page_table must be an int32 matrix on the call's device")
    seqs, cols = page_table.shape
    lt, last = page_table.stride()
    if last != 1 and cols > 1:
        raise ValueError("the entries of a row of page_table must be adjacent")
    if seqs < 2:
        lt = max(lt, cols)
    elif 0 < lt < cols:
        raise ValueError("rows of page_table must not overlap (but one row may be all sequences')")
    lp = _vector(lengths, seqs, torch.int32, "lengths", dev)
    stp = 0 if starts is None else _vector(starts, seqs + 1, torch.int32, "starts", dev)
    o, lo, loh = _out_heads(out, q, "out", stream)
    ep, e = 0, None
    if lse is not False:
        e = _new((n, h), torch.float32, cache.device, stream) if lse is True else lse
        ep = _vector(e, n * h, torch.float32, "lse", dev)
    if workspace is None:
        workspace = cache_attention_workspace(q, cache, seqs, stream=stream)
    elif not workspace.is_cuda or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor on the call's device")
    args = _CACHE_ATTENTION.pack(n, seqs, h, dt, d ** -0.5 if scale is None else scale, q.data_ptr(), lq, lqh, o.data_ptr(), lo, loh, ep,
                                 stp, lp, page_table.data_ptr(), lt, cols)
    _check(_calls().aqd_cache_attention(args, cache.desc, workspace.data_ptr(), workspace.nbytes, _stream(stream)),
           "aqd_cache_attention")
    return o if e is None else (o, e)


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, *,
                     kv_starts: torch.Tensor | None = None, causal: bool = True, scale: float | None = None,
                     out: torch.Tensor | None = None, lse: bool | torch.Tensor = False, stream=None):
    """Attention over whole sequences packed one after another (aqd_prompt_attention): q [tokens, heads, head_dim], k and v
    [kv_tokens, kv_heads, head_dim], starts int32 [seqs + 1], kv_starts where a sequence has other keys than queries (causal: its queries are
    then the last ones). scale: 1 / sqrt(head_dim) where not given. Returns the output, or (output, lse [tokens, heads]) where lse is wanted."""
    n, h, d, lq, lqh = _heads(q, "q")
    dt = _float_dtype(q, "q")
    dev = q.get_device()
    _runs_on(dev, stream)
    nk, hk, dk, lk, lkh = _heads(k, "k", dev)
    _, _, _, lv, lvh = _heads(v, "v", dev)
    if dk != d or v.shape != k.shape or k.dtype is not q.dtype or v.dtype is not q.dtype:
        raise ValueError("k and v must have one shape, and q's head_dim and type")
    seqs = starts.numel() - 1
    if seqs < 0:
        raise ValueError("starts must hold seqs + 1 numbers")
    stp = _vector(starts, seqs + 1, torch.int32, "starts", dev)
    ksp = 0
    if kv_starts is not None:
        ksp = _vector(kv_starts, seqs + 1, torch.int32, "kv_starts", dev)
    elif nk != n:
        raise ValueError("kv_starts is required where keys and queries differ in number")
    o, lo, loh = _out_heads(out, q, "out", stream)
    ep, e = 0, None
    if lse is not False:
        e = _new((n, h), torch.float32, q.device, stream) if lse is True else lse
        ep = _vector(e, n * h, torch.float32, "lse", dev)
    args = _PROMPT.pack(n, nk, seqs, h, hk, d, dt, 1 if causal else 0, d ** -0.5 if scale is None else scale, q.data_ptr(), lq, lqh,
                        k.data_ptr(), lk, lkh, v.data_ptr(), lv, lvh, o.data_ptr(), lo, loh, ep, stp, ksp)
    _check(_calls().aqd_prompt_attention(args, _stream(stream)), "aqd_prompt_attention")
    return o if e is None else (o, e)


class DistillLoss(NamedTuple):
    loss: torch.Tensor
    lse: torch.Tensor
    grad: torch.Tensor | None = None


def _distill_args(logits, index, teacher, row_weight, tau, grad, stream):
    m, v, ld = _rows_of(logits, "logits")
    d = _float_dtype(logits, "logits")
    dev = logits.get_device()
    _runs_on(dev, stream)
    top = teacher.shape[-1] if teacher.dim() else 0
    if index.shape != teacher.shape or index.shape[:-1] != logits.shape[:-1]:
        raise ValueError("index and teacher must have the logits' shape but for the last dimension")
    ip = _vector(index, m * top, torch.int64, "index", dev)
    tp = _vector(teacher, m * top, torch.float32, "teacher", dev)
    wp = 0 if row_weight is None else _vector(row_weight, m, torch.float32, "row_weight", dev)
    gp = lg = 0
    if grad is not None:
        if grad.shape != logits.shape or grad.dtype is not logits.dtype:
            raise ValueError("grad must have the logits' shape and type")
        lg = _rows_of(grad, "grad", dev)[2]
        gp = grad.data_ptr()
    return m, _DISTILL.pack(m, v, d, logits.data_ptr(), ld, ip, tp, top, tau, wp, gp, lg)


def distill_topk(logits: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, *, tau: float = 1.0,
                 row_weight: torch.Tensor | None = None, grad: bool | torch.Tensor = False, stream=None) -> DistillLoss:
    """The distillation loss of each token of logits [..., vocab] against a teacher's top logits (aqd_distill_topk):
    teacher float32 [..., top] at the vocabulary places index int64 [..., top]. grad: True, or a tensor (the logits
    themselves: in place), for the gradient of the losses' sum in the same pass."""
    g = _new(logits.shape, logits.dtype, logits.device, stream) if grad is True else None if grad is False else grad
    _, args = _distill_args(logits, index, teacher, row_weight, tau, g, stream)
    loss = _new(logits.shape[:-1], torch.float32, logits.device, stream)
    lse = _new(logits.shape[:-1], torch.float32, logits.device, stream)
    _check(_calls().aqd_distill_topk(args, loss.data_ptr(), lse.data_ptr(), _stream(stream)), "aqd_distill_topk")
    return DistillLoss(loss, lse, g)


def distill_topk_backward(logits: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, lse: torch.Tensor,
                          row_weight: torch.Tensor | None = None, *, tau: float = 1.0,
                          grad: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gradient of distill_topk's losses from the lse that it returned; row_weight: the factor of each token's
    gradient."""
    g = _new(logits.shape, logits.dtype, logits.device, stream) if grad is None else grad
    m, args = _distill_args(logits, index, teacher, row_weight, tau, g, stream)
    lp = _vector(lse, m, torch.float32, "lse", logits.get_device())
    _check(_calls().aqd_distill_topk_backward(args, lp, _stream(stream)), "aqd_distill_topk_backward")
    return g


def device_status(stream=None) -> int:
    code = ctypes.c_int32()
    _check(load().aqd_device_status(_stream(stream), ctypes.byref(code)), "aqd_device_status")
    return int(code.value)


def selftest_wait_timeout(out: torch.Tensor, stream=None) -> None:
    """Launches the bounded-wait self-test into ``out`` (5 int64 on the device); see
    aqd_selftest_wait_timeout."""
    assert out.dtype == torch.int64 and out.is_cuda and out.numel() >= 5
    _check(load().aqd_selftest_wait_timeout(_ptr(out), _stream(stream)), "aqd_selftest_wait_timeout")


def set_conv_path(path: int) -> int:
    return int(load().aqd_set_conv_path(path))


def last_conv_path() -> int:
    return int(load().aqd_last_conv_path())
