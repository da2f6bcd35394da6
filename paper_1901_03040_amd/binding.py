"""ctypes binding of libqesgd.so: the same entry points as include/qesgd.h.

Argument marshalling only.  Tensors are torch tensors on the GPU (torch is used
for device memory and streams, nothing else); every step of the path runs in
the library's kernels.  There is no fallback: if the library has not been built
the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from functools import lru_cache
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqesgd.so")

NORM_L2 = 0
NORM_MAX = 1

OK = 0
ERR_NULL, ERR_DIM, ERR_LEVELS, ERR_BUCKET, ERR_WORKERS = -1, -2, -3, -4, -5
ERR_NORM_KIND, ERR_ALIGN, ERR_STRIDE, ERR_WORKSPACE, ERR_HIP = -6, -7, -8, -9, -10
ERR_BITS, ERR_DELTA, ERR_ROUNDS, ERR_SCRATCH = -11, -12, -13, -14
ERR_DTYPE, ERR_MODE, ERR_STEPS, ERR_COEFF, ERR_EXPERTS = -15, -16, -17, -18, -19
NOALLOC_SCRATCH_BYTES = 4 << 20
MX4_NEAREST, MX4_STOCHASTIC = 0, 1
MAX_STEPS = 32
MAX_EXPERTS, MAX_CHOICES = 1024, 16
GATE_ALL, GATE_CHOSEN = 0, 1
ROWS_F32 = 0x100
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class QesgdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


class _Layout(C.Structure):
    _fields_ = [("n_buckets", C.c_uint64), ("level_bits", C.c_uint32), ("reserved", C.c_uint32),
                ("sign_words", C.c_uint64), ("level_words", C.c_uint64),
                ("norms_off", C.c_uint64), ("signs_off", C.c_uint64), ("levels_off", C.c_uint64),
                ("bytes_per_worker", C.c_uint64), ("payload_bytes", C.c_uint64)]


@dataclass(frozen=True)
class Layout:
    n_buckets: int
    level_bits: int
    sign_words: int
    level_words: int
    norms_off: int
    signs_off: int
    levels_off: int
    bytes_per_worker: int
    payload_bytes: int


class _Mx4Layout(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("rows", "cols", "row_codes", "row_scales", "codes_off", "scales_off", "bytes",
                                          "payload_bytes")]


@dataclass(frozen=True)
class Mx4Layout:
    rows: int
    cols: int
    row_codes: int
    row_scales: int
    codes_off: int
    scales_off: int
    bytes: int
    payload_bytes: int


_lib = None


def lib():
    """Loads libqesgd.so once; raises if it is missing (there is no other path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: build it with "
                               "`python -m paper_1901_03040_amd.build` (hipcc, gfx950)")
        L = C.CDLL(LIB_PATH)
        u32, u64, vp, sz = C.c_uint32, C.c_uint64, C.c_void_p, C.c_size_t
        L.qesgd_layout_query.argtypes = [u64, u32, u64, C.POINTER(_Layout)]
        L.qesgd_layout_query.restype = C.c_int
        L.qesgd_workspace_bytes.argtypes = [u64, u32, u64, u32]
        L.qesgd_workspace_bytes.restype = sz
        L.qesgd_quantize_pack.argtypes = [vp, vp, u64, u32, u64, u32, u64, u32, u32, vp, vp, sz, vp]
        L.qesgd_quantize_pack.restype = C.c_int
        L.qesgd_quantize_pack_batched.argtypes = [vp, u64, vp, u64, u32, u64, u32, u64, u32, u32,
                                                  vp, u64, vp, sz, vp]
        L.qesgd_quantize_pack_batched.restype = C.c_int
        L.qesgd_quantize_pack_batched_noalloc.argtypes = [vp, u64, vp, u64, u32, u64, u32, u64, u32, u32,
                                                          vp, u64, vp]
        L.qesgd_quantize_pack_batched_noalloc.restype = C.c_int
        L.qesgd_unpack_aggregate.argtypes = [vp, u64, u32, u64, u32, u64, vp, vp]
        L.qesgd_unpack_aggregate.restype = C.c_int
        L.qesgd_apply_update.argtypes = [vp, vp, vp, vp, u64, vp]
        L.qesgd_apply_update.restype = C.c_int
        L.qesgd_unpack_aggregate_update.argtypes = [vp, u64, u32, u64, u32, u64, vp, vp, vp, vp, vp]
        L.qesgd_unpack_aggregate_update.restype = C.c_int
        L.qesgd_round.argtypes = [vp, u64, vp, u64, u32, u64, u32, u64, u32, u32, vp, u64, vp, sz, vp, vp, vp, vp, vp]
        L.qesgd_round.restype = C.c_int
        L.qesgd_gradient_round.argtypes = [vp, u64, u64, u32, u64, u32, u64, u32, u32, vp, u64, vp, sz, vp, vp, vp, vp, vp, vp]
        L.qesgd_gradient_round.restype = C.c_int
        L.qesgd_quantize_fixed.argtypes = [vp, vp, u64, C.c_float, u32, u64, u32, u32, vp, vp]
        L.qesgd_quantize_fixed.restype = C.c_int
        L.qesgd_dequantize_fixed_update.argtypes = [vp, u64, C.c_float, u32, vp, vp, vp, vp, vp]
        L.qesgd_dequantize_fixed_update.restype = C.c_int
        L.qesgd_epoch_commit.argtypes = [vp, vp, u32, u64, vp]
        L.qesgd_epoch_commit.restype = C.c_int
        f32 = C.c_float
        L.qesgd_mx4_layout_query.argtypes = [u64, u64, C.POINTER(_Mx4Layout)]
        L.qesgd_mx4_layout_query.restype = C.c_int
        L.qesgd_mx4_quantize_pack.argtypes = [vp, u32, u64, u64, u64, u64, u32, u32, u64, u32, u32, vp, u64, vp, u64, vp]
        L.qesgd_mx4_quantize_pack.restype = C.c_int
        L.qesgd_mx4_unpack_aggregate_update.argtypes = [vp, u64, u32, u64, u64, vp, vp, vp, vp, vp]
        L.qesgd_mx4_unpack_aggregate_update.restype = C.c_int
        L.qesgd_mx4_product_workspace_bytes.argtypes = [u64, u64, u64]
        L.qesgd_mx4_product_workspace_bytes.restype = sz
        L.qesgd_mx4_product.argtypes = [vp, vp, u64, u64, u64, vp, u32, u64, vp, sz, vp]
        L.qesgd_mx4_product.restype = C.c_int
        L.qesgd_orthogonalize_workspace_bytes.argtypes = [u64, u64, u32]
        L.qesgd_orthogonalize_workspace_bytes.restype = sz
        L.qesgd_orthogonalize.argtypes = [vp, u32, u64, u64, u32, vp, u32, f32, vp, vp, sz, vp]
        L.qesgd_orthogonalize.restype = C.c_int
        L.qesgd_orthogonal_update.argtypes = [vp, u64, u64, u32, vp, f32, u32, vp, u32, f32, f32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.qesgd_orthogonal_update.restype = C.c_int
        L.qesgd_route_workspace_bytes.argtypes = [u64, u32, u32]
        L.qesgd_route_workspace_bytes.restype = sz
        L.qesgd_route.argtypes = [vp, u32, u64, u64, u32, u32, u32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.qesgd_route.restype = C.c_int
        L.qesgd_route_backward.argtypes = [vp, u32, u64, u64, u32, u32, u32, vp, vp, vp, vp, u64, vp]
        L.qesgd_route_backward.restype = C.c_int
        L.qesgd_combine.argtypes = [vp, u32, u64, u64, vp, vp, u64, u32, u64, vp, u64, vp]
        L.qesgd_combine.restype = C.c_int
        L.qesgd_combine_backward.argtypes = [vp, u32, u64, vp, u64, u64, vp, vp, u64, u32, u64, vp, u64, vp, vp]
        L.qesgd_combine_backward.restype = C.c_int
        L.qesgd_mx4_grouped_columns.argtypes = [u64, u32]
        L.qesgd_mx4_grouped_columns.restype = u64
        L.qesgd_mx4_quantize_groups.argtypes = [vp, u32, u64, u64, vp, u32, vp, u32, u64, u64, u32, u64, u32, u32, vp, vp, vp]
        L.qesgd_mx4_quantize_groups.restype = C.c_int
        L.qesgd_mx4_grouped_product.argtypes = [vp, vp, u64, vp, u32, u64, u64, u64, vp, u32, u64, vp, sz, vp]
        L.qesgd_mx4_grouped_product.restype = C.c_int
        L.qesgd_mx4_grouped_gradient.argtypes = [vp, vp, vp, u32, u64, u64, u64, vp, u32, vp, sz, vp]
        L.qesgd_mx4_grouped_gradient.restype = C.c_int
        L.qesgd_mx4_vector_product.argtypes = [vp, u32, u64, u64, vp, u32, vp, u64, vp, u32, u64, u64, u64, vp, u64, vp, sz, vp]
        L.qesgd_mx4_vector_product.restype = C.c_int
        for name in ("grouped_product", "grouped_gradient", "vector_product"):
            f = getattr(L, f"qesgd_mx4_{name}_workspace_bytes")
            f.argtypes, f.restype = [u64, u64, u64, u32], sz
        L.qesgd_strerror.argtypes = [C.c_int]
        L.qesgd_strerror.restype = C.c_char_p
        L.qesgd_last_hip_error.argtypes = []
        L.qesgd_last_hip_error.restype = C.c_int
        L.qesgd_abi_version.argtypes = []
        L.qesgd_abi_version.restype = u32
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().qesgd_strerror(int(code)).decode()


# Both hand plain integers to ctypes (the argument types make the pointers), and the stream is asked for
# as a raw handle: building a torch.cuda.Stream object for it took 3.05 of the 9.7 us that a call took on
# the host, against 0.22 us (one call of qesgd_round at d = 256, now 5.6 us; the launch itself is about 3).
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    """torch stream, raw hipStream_t handle (int), or None = torch's current stream."""
    if stream is None:
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        stream = torch.cuda.current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(rc: int, where: str):
    if rc != OK:
        raise QesgdError(rc, where)


def qesgd_layout_query(d: int, s: int, bucket: int) -> Layout:
    out = _Layout()
    _check(lib().qesgd_layout_query(int(d), int(s), int(bucket), C.byref(out)), "qesgd_layout_query")
    return Layout(out.n_buckets, out.level_bits, out.sign_words, out.level_words, out.norms_off,
                  out.signs_off, out.levels_off, out.bytes_per_worker, out.payload_bytes)


def qesgd_workspace_bytes(d: int, s: int, bucket: int, K: int) -> int:
    return int(lib().qesgd_workspace_bytes(int(d), int(s), int(bucket), int(K)))


def qesgd_quantize_pack(x, center, d, s, bucket, norm_kind, seed, rnd, worker, packed,
                        workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().qesgd_quantize_pack(_ptr(x), _ptr(center), int(d), int(s), int(bucket), int(norm_kind),
                                     int(seed), int(rnd), int(worker), _ptr(packed), _ptr(workspace),
                                     ws_bytes, _stream(stream)), "qesgd_quantize_pack")


def qesgd_quantize_pack_batched(x_slab, x_stride, center, d, s, bucket, norm_kind, seed, rnd, K,
                                packed_slab, packed_stride, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().qesgd_quantize_pack_batched(_ptr(x_slab), int(x_stride), _ptr(center), int(d), int(s),
                                             int(bucket), int(norm_kind), int(seed), int(rnd), int(K),
                                             _ptr(packed_slab), int(packed_stride), _ptr(workspace),
                                             ws_bytes, _stream(stream)), "qesgd_quantize_pack_batched")


def qesgd_quantize_pack_batched_noalloc(x_slab, x_stride, center, d, s, bucket, norm_kind, seed, rnd, K,
                                        packed_slab, packed_stride, stream=None):
    _check(lib().qesgd_quantize_pack_batched_noalloc(_ptr(x_slab), int(x_stride), _ptr(center), int(d), int(s),
                                                     int(bucket), int(norm_kind), int(seed), int(rnd), int(K),
                                                     _ptr(packed_slab), int(packed_stride), _stream(stream)),
           "qesgd_quantize_pack_batched_noalloc")


def qesgd_unpack_aggregate(packed_slab, packed_stride, K, d, s, bucket, zbar, stream=None):
    _check(lib().qesgd_unpack_aggregate(_ptr(packed_slab), int(packed_stride), int(K), int(d), int(s),
                                        int(bucket), _ptr(zbar), _stream(stream)), "qesgd_unpack_aggregate")


def qesgd_apply_update(w_snap, zbar, u_out, zsum_inout, d, stream=None):
    _check(lib().qesgd_apply_update(_ptr(w_snap), _ptr(zbar), _ptr(u_out), _ptr(zsum_inout), int(d),
                                    _stream(stream)), "qesgd_apply_update")


def qesgd_unpack_aggregate_update(packed_slab, packed_stride, K, d, s, bucket, w_snap, zbar_out, u_out,
                                  zsum_inout, stream=None):
    _check(lib().qesgd_unpack_aggregate_update(_ptr(packed_slab), int(packed_stride), int(K), int(d),
                                               int(s), int(bucket), _ptr(w_snap), _ptr(zbar_out),
                                               _ptr(u_out), _ptr(zsum_inout), _stream(stream)),
           "qesgd_unpack_aggregate_update")


def qesgd_round(x_slab, x_stride, center, d, s, bucket, norm_kind, seed, rnd, K, packed_slab, packed_stride,
                w_snap, zbar_out, u_out, zsum_inout, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().qesgd_round(_ptr(x_slab), int(x_stride), _ptr(center), int(d), int(s), int(bucket), int(norm_kind),
                             int(seed), int(rnd), int(K), _ptr(packed_slab), int(packed_stride), _ptr(workspace),
                             ws_bytes, _ptr(w_snap), _ptr(zbar_out), _ptr(u_out), _ptr(zsum_inout), _stream(stream)),
           "qesgd_round")


def qesgd_gradient_round(x_slab, x_stride, d, s, bucket, norm_kind, seed, rnd, K, packed_slab, packed_stride,
                         w_snap, step_out, z_inout, u_out, zsum_inout, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().qesgd_gradient_round(_ptr(x_slab), int(x_stride), int(d), int(s), int(bucket), int(norm_kind), int(seed),
                                      int(rnd), int(K), _ptr(packed_slab), int(packed_stride), _ptr(workspace), ws_bytes,
                                      _ptr(w_snap), _ptr(step_out), _ptr(z_inout), _ptr(u_out), _ptr(zsum_inout),
                                      _stream(stream)), "qesgd_gradient_round")


def qesgd_quantize_fixed(x, center, d, delta, b, seed, rnd, worker, codes, stream=None):
    _check(lib().qesgd_quantize_fixed(_ptr(x), _ptr(center), int(d), float(delta), int(b), int(seed), int(rnd),
                                      int(worker), _ptr(codes), _stream(stream)), "qesgd_quantize_fixed")


def qesgd_dequantize_fixed_update(codes, d, delta, b, w_snap, z_out, u_out, zsum_inout, stream=None):
    _check(lib().qesgd_dequantize_fixed_update(_ptr(codes), int(d), float(delta), int(b), _ptr(w_snap), _ptr(z_out),
                                               _ptr(u_out), _ptr(zsum_inout), _stream(stream)),
           "qesgd_dequantize_fixed_update")


def qesgd_epoch_commit(w_inout, zsum_inout, rounds, d, stream=None):
    _check(lib().qesgd_epoch_commit(_ptr(w_inout), _ptr(zsum_inout), int(rounds), int(d), _stream(stream)),
           "qesgd_epoch_commit")


# ---- matrix parameters ------------------------------------------------------
#
# The kernels run on the current device and take addresses: a tensor of the host or of another device is refused here, and so are
# types that the call does not say (packed matrices are uint8), tensors that hold less than the call reads or writes, and views whose
# strides are not the call's: gaps, another order, a broadcast.  Small calls cost the host about 5 us, most of it in the launch, so the
# checks (0.5 us) stand in line and numbers (plain ints) go to ctypes as they are: with a loop over the tensors and int() around each number a
# call took 0.9 us more.

_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_U8 = torch.uint8


def _here(where: str, stream, t):
    """The current device, which t has to be on, and the handle of the stream."""
    device = t.get_device()
    if device < 0 or device != _current_device():
        _elsewhere(where, t)
    if stream is None:
        return device, _current_stream(device)
    return device, stream if isinstance(stream, int) else stream.cuda_stream


def _elsewhere(where: str, *tensors):
    raise ValueError(f"{where}: tensors on {sorted({str(t.device) for t in tensors if t is not None})}, not all on the current GPU")


def _dtype(t: torch.Tensor, where: str) -> int:
    code = DTYPES.get(t.dtype)
    if code is None:
        raise QesgdError(ERR_DTYPE, where)
    return code


def _view(where: str, t, *dims):
    """For a tensor that is not contiguous, or too short if it were: refuses it unless all that the call reads or writes, (count, stride) from
    the outermost dimension on, are elements of the view, in its order.  The call's dimensions are laid into the view's from the
    innermost on, as many into one as it has room for (a convolution's weights are a matrix whose columns are three of four dimensions)."""
    if t.is_contiguous():
        raise ValueError(f"{where}: a tensor of {t.numel()} elements, the call takes {1 + sum((n - 1) * step for n, step in dims if n > 1)}")
    own = []
    for size, stride in zip(t.shape, t.stride()):
        if own and own[-1][1] == size * stride:
            own[-1] = (own[-1][0] * size, stride)
        elif size != 1:
            own.append((size, stride))
    left = [d for d in dims if d[0] > 1]
    while left and own and 0 < own[-1][1] <= left[-1][1] and t.numel():
        size, stride = own.pop()
        at = 0
        while left and left[-1][1] % stride == 0 and at + (left[-1][0] - 1) * (left[-1][1] // stride) < size:
            n, step = left.pop()
            at += (n - 1) * (step // stride)
    if left or not t.numel():
        raise QesgdError(ERR_STRIDE, where)


@lru_cache(maxsize=256)
def _mx4_bytes(rows, cols):
    """Bytes of a packed matrix up to its last scale."""
    wide = (cols + 127) // 128 * 128
    return (rows * wide // 2 + 255) // 256 * 256 + rows * wide // 32


def _packed(where: str, device, t, rows, cols, K=1, stride=0):
    """Address of K packed matrices."""
    if t.get_device() != device:
        _elsewhere(where, t)
    if t.dtype is not _U8:
        raise QesgdError(ERR_DTYPE, where)
    if not t.is_contiguous() or t.numel() < (_mx4_bytes(rows, cols) if K == 1 else (K - 1) * stride + _mx4_bytes(rows, cols)):
        _view(where, t, (K, stride), (_mx4_bytes(rows, cols), 1))
    return t.data_ptr()


def _f32(where: str, device, count, *tensors):
    """Addresses of contiguous fp32 tensors of at least `count` elements, each of which may be None."""
    out = []
    for t in tensors:
        if t is None:
            out.append(None)
            continue
        if t.get_device() != device:
            _elsewhere(where, *tensors)
        if t.dtype is not torch.float32:
            raise QesgdError(ERR_DTYPE, where)
        if not t.is_contiguous():
            raise QesgdError(ERR_STRIDE, where)
        if t.numel() < count:
            _view(where, t, (count, 1))
        out.append(t.data_ptr())
    return out


def _ws(where: str, device, workspace):
    if workspace is None:
        return None, 0
    if workspace.get_device() != device:
        _elsewhere(where, workspace)
    if not workspace.is_contiguous():
        raise QesgdError(ERR_STRIDE, where)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def qesgd_mx4_layout_query(rows: int, cols: int) -> Mx4Layout:
    out = _Mx4Layout()
    _check(lib().qesgd_mx4_layout_query(int(rows), int(cols), C.byref(out)), "qesgd_mx4_layout_query")
    return Mx4Layout(*(getattr(out, n) for n, _ in _Mx4Layout._fields_))


def qesgd_mx4_quantize_pack(x, ld, x_stride, rows, cols, K, mode, seed, rnd, packed, packed_stride, packed_t=None,
                            packed_t_stride=0, worker=0, stream=None):
    where = "qesgd_mx4_quantize_pack"
    dtype = _dtype(x, where)
    device, stream = _here(where, stream, x)
    if not x.is_contiguous() or x.numel() < (K - 1) * x_stride + (rows - 1) * ld + cols:
        _view(where, x, (K, x_stride), (rows, ld), (cols, 1))
    p = None if packed is None else _packed(where, device, packed, rows, cols, K, packed_stride)
    pt = None if packed_t is None else _packed(where, device, packed_t, cols, rows, K, packed_t_stride)
    rc = (_lib or lib()).qesgd_mx4_quantize_pack(x.data_ptr(), dtype, ld, x_stride, rows, cols, K, mode, seed, rnd, worker, p,
                                                 packed_stride, pt, packed_t_stride, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_mx4_unpack_aggregate_update(packed_slab, packed_stride, K, rows, cols, w_snap, zbar_out, u_out, zsum_inout,
                                      stream=None):
    where = "qesgd_mx4_unpack_aggregate_update"
    device, stream = _here(where, stream, packed_slab)
    slab = _packed(where, device, packed_slab, rows, cols, K, packed_stride)
    rc = (_lib or lib()).qesgd_mx4_unpack_aggregate_update(slab, packed_stride, K, rows, cols, *_f32(where, device, rows * cols, w_snap,
                                                                                                    zbar_out, u_out, zsum_inout), stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_mx4_product_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().qesgd_mx4_product_workspace_bytes(int(M), int(N), int(K)))


def qesgd_mx4_product(a_packed, b_packed, M, N, K, c, ldc, workspace=None, stream=None):
    where = "qesgd_mx4_product"
    dtype = _dtype(c, where)
    device, stream = _here(where, stream, c)
    if not c.is_contiguous() or c.numel() < (M - 1) * ldc + N:
        _view(where, c, (M, ldc), (N, 1))
    ws, ws_bytes = (None, 0) if workspace is None else _ws(where, device, workspace)
    rc = (_lib or lib()).qesgd_mx4_product(_packed(where, device, a_packed, M, K), _packed(where, device, b_packed, N, K), M, N, K, c.data_ptr(),
                                           dtype, ldc, ws, ws_bytes, stream)
    if rc:
        raise QesgdError(rc, where)


@lru_cache(maxsize=64)
def _coeff_array(flat):
    return (C.c_float * len(flat))(*flat)


def _coeffs(coeffs):
    """(a, b, c) of every step as a C array, kept by its numbers."""
    if any(len(step) != 3 for step in coeffs):
        raise ValueError("coeffs: three numbers for each step")
    return _coeff_array(tuple([float(v) for step in coeffs for v in step]))


def qesgd_orthogonalize_workspace_bytes(rows: int, cols: int, n: int) -> int:
    return int(lib().qesgd_orthogonalize_workspace_bytes(int(rows), int(cols), int(n)))


def qesgd_orthogonalize(x, rows, cols, n, coeffs, eps, out, workspace, stream=None):
    where = "qesgd_orthogonalize"
    if out.dtype != x.dtype:
        raise QesgdError(ERR_DTYPE, where)
    dtype, steps = _dtype(x, where), _coeffs(coeffs)
    device, stream = _here(where, stream, x)
    if out.get_device() != device:
        _elsewhere(where, x, out)
    for t in (x, out):
        if not t.is_contiguous():
            raise QesgdError(ERR_STRIDE, where)
        if t.numel() < n * rows * cols:
            _view(where, t, (n * rows * cols, 1))
    ws, ws_bytes = _ws(where, device, workspace)
    _check(lib().qesgd_orthogonalize(x.data_ptr(), dtype, rows, cols, n, steps, len(coeffs), float(eps), out.data_ptr(), ws, ws_bytes,
                                     stream), where)


def qesgd_orthogonal_update(g, rows, cols, n, momentum_inout, mu, nesterov, coeffs, eps, alpha, step_out, z_inout, w_snap,
                            u_out, zsum_inout, workspace, stream=None):
    where = "qesgd_orthogonal_update"
    if g.dtype != torch.float32:
        raise QesgdError(ERR_DTYPE, where)
    steps = _coeffs(coeffs)
    device, stream = _here(where, stream, g)
    g, m, step, z, w, u, zsum = _f32(where, device, n * rows * cols, g, momentum_inout, step_out, z_inout, w_snap, u_out, zsum_inout)
    ws, ws_bytes = _ws(where, device, workspace)
    _check(lib().qesgd_orthogonal_update(g, rows, cols, n, m, float(mu), 1 if nesterov else 0, steps, len(coeffs), float(eps),
                                         float(alpha), step, z, w, u, zsum, ws, ws_bytes, stream), where)


# ---- layers of experts ------------------------------------------------------
#
# The same checks as above.  experts, offsets, order and slots are int32, gates and their gradients fp32, all contiguous.  These calls have five to eight tensors each: what is
# contiguous, of the right type and long enough, as nearly all are, is seen in line, and the functions below look at the rest (a function for each tensor: 0.1 us more for each).

_I32, _F32 = torch.int32, torch.float32


def _ints(where: str, device, t, count):
    """Address of a contiguous int32 tensor of at least `count` elements."""
    if t.get_device() != device:
        _elsewhere(where, t)
    if t.dtype is not _I32:
        raise QesgdError(ERR_DTYPE, where)
    if not t.is_contiguous():
        raise QesgdError(ERR_STRIDE, where)
    if t.numel() < count:
        _view(where, t, (count, 1))
    return t.data_ptr()


def _rows(where: str, device, t, kind, rows, ld, cols):
    """Address of `rows` rows of `cols` elements of that type, ld apart."""
    if t.get_device() != device:
        _elsewhere(where, t)
    if t.dtype is not kind:
        raise QesgdError(ERR_DTYPE, where)
    if not t.is_contiguous() or t.numel() < (rows - 1) * ld + cols:
        _view(where, t, (rows, ld), (cols, 1))
    return t.data_ptr()


def qesgd_route_workspace_bytes(T: int, E: int, k: int) -> int:
    return int(lib().qesgd_route_workspace_bytes(int(T), int(E), int(k)))


def qesgd_route(logits, ld, T, E, k, gate_kind, experts, gates, offsets, order, slots, workspace=None, stream=None):
    where, kind, pairs = "qesgd_route", logits.dtype, T * k
    dtype = _dtype(logits, where)
    device, stream = _here(where, stream, logits)
    x = logits.data_ptr() if logits.is_contiguous() and logits.numel() >= (T - 1) * ld + E else _rows(where, device, logits, kind, T, ld, E)
    e = experts.data_ptr() if experts.dtype is _I32 and experts.get_device() == device and experts.is_contiguous() and experts.numel() >= pairs \
        else _ints(where, device, experts, pairs)
    g = gates.data_ptr() if gates.dtype is _F32 and gates.get_device() == device and gates.is_contiguous() and gates.numel() >= pairs \
        else _f32(where, device, pairs, gates)[0]
    f = offsets.data_ptr() if offsets.dtype is _I32 and offsets.get_device() == device and offsets.is_contiguous() and offsets.numel() > E \
        else _ints(where, device, offsets, E + 1)
    o = order.data_ptr() if order.dtype is _I32 and order.get_device() == device and order.is_contiguous() and order.numel() >= pairs \
        else _ints(where, device, order, pairs)
    s = slots.data_ptr() if slots.dtype is _I32 and slots.get_device() == device and slots.is_contiguous() and slots.numel() >= pairs \
        else _ints(where, device, slots, pairs)
    ws, ws_bytes = (None, 0) if workspace is None else _ws(where, device, workspace)
    rc = (_lib or lib()).qesgd_route(x, dtype, ld, T, E, k, gate_kind, e, g, f, o, s, ws, ws_bytes, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_route_backward(logits, ld, T, E, k, gate_kind, experts, gates, dgates, dlogits, ld_d, stream=None):
    where, kind, pairs = "qesgd_route_backward", dlogits.dtype, T * k
    dtype = _dtype(dlogits, where)
    device, stream = _here(where, stream, dlogits)
    x = None if logits is None else _rows(where, device, logits, kind, T, ld, E)
    g, dg = _f32(where, device, pairs, gates, dgates)
    rc = (_lib or lib()).qesgd_route_backward(x, dtype, ld, T, E, k, gate_kind, _ints(where, device, experts, pairs), g, dg,
                                              _rows(where, device, dlogits, kind, T, ld_d, E), ld_d, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_combine(rows, ld, R, slots, gates, T, k, N, out, ld_out, stream=None):
    where, kind, pairs = "qesgd_combine", out.dtype, T * k
    dtype = _dtype(out, where)
    device, stream = _here(where, stream, out)
    own = kind                                                # the rows' type
    if rows.dtype is _F32 and kind is not _F32:
        dtype, own = dtype | ROWS_F32, _F32
    x = rows.data_ptr() if rows.dtype is own and rows.get_device() == device and rows.is_contiguous() and rows.numel() >= (R - 1) * ld + N \
        else _rows(where, device, rows, own, R, ld, N)
    y = out.data_ptr() if out.is_contiguous() and out.numel() >= (T - 1) * ld_out + N else _rows(where, device, out, kind, T, ld_out, N)
    s = None if slots is None else slots.data_ptr() if slots.dtype is _I32 and slots.get_device() == device and slots.is_contiguous() and \
        slots.numel() >= pairs else _ints(where, device, slots, pairs)
    g = None if gates is None else gates.data_ptr() if gates.dtype is _F32 and gates.get_device() == device and gates.is_contiguous() and \
        gates.numel() >= pairs else _f32(where, device, pairs, gates)[0]
    rc = (_lib or lib()).qesgd_combine(x, dtype, ld, R, s, g, T, k, N, y, ld_out, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_combine_backward(dy, ld_dy, rows, ld, R, slots, gates, T, k, N, drows, ld_d, dgates, stream=None):
    where, kind, pairs = "qesgd_combine_backward", dy.dtype, T * k
    dtype = _dtype(dy, where)
    device, stream = _here(where, stream, dy)
    d = dy.data_ptr() if dy.is_contiguous() and dy.numel() >= (T - 1) * ld_dy + N else _rows(where, device, dy, kind, T, ld_dy, N)
    own = kind                                                # the rows' type
    if rows is not None and rows.dtype is _F32 and kind is not _F32:
        dtype, own = dtype | ROWS_F32, _F32
    x = None if rows is None else _rows(where, device, rows, own, R, ld, N)
    dr = None if drows is None else _rows(where, device, drows, kind, R, ld_d, N)
    s = None if slots is None else slots.data_ptr() if slots.dtype is _I32 and slots.get_device() == device and slots.is_contiguous() and \
        slots.numel() >= pairs else _ints(where, device, slots, pairs)
    g, dg = _f32(where, device, pairs, gates, dgates)
    rc = (_lib or lib()).qesgd_combine_backward(d, dtype, ld_dy, x, ld, R, s, g, T, k, N, dr, ld_d, dg, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_mx4_grouped_columns(R: int, E: int) -> int:
    return int(lib().qesgd_mx4_grouped_columns(int(R), int(E)))


def qesgd_mx4_quantize_groups(x, ld, T, order, per, offsets, E, R, cols, mode, seed, rnd, packed, packed_t=None, worker=0, stream=None):
    where, kind = "qesgd_mx4_quantize_groups", x.dtype
    dtype = _dtype(x, where)
    device, stream = _here(where, stream, x)
    a = x.data_ptr() if x.is_contiguous() and x.numel() >= (T - 1) * ld + cols else _rows(where, device, x, kind, T, ld, cols)
    o = None if order is None else order.data_ptr() if order.dtype is _I32 and order.get_device() == device and order.is_contiguous() and \
        order.numel() >= R else _ints(where, device, order, R)
    f = offsets.data_ptr() if offsets.dtype is _I32 and offsets.get_device() == device and offsets.is_contiguous() and offsets.numel() > E \
        else _ints(where, device, offsets, E + 1)
    p = None if packed is None else _packed(where, device, packed, R, cols)
    pt = None if packed_t is None else _packed(where, device, packed_t, cols, (R + 127 * min(E, R)) // 128 * 128)
    rc = (_lib or lib()).qesgd_mx4_quantize_groups(a, dtype, ld, T, o, per, f, E, R, cols, mode, seed, rnd, worker, p, pt, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_mx4_grouped_product_workspace_bytes(R: int, N: int, K: int, E: int) -> int:
    return int(lib().qesgd_mx4_grouped_product_workspace_bytes(int(R), int(N), int(K), int(E)))


def qesgd_mx4_grouped_product(a_packed, b_slab, b_stride, offsets, E, R, N, K, c, ldc, workspace=None, stream=None):
    where, kind = "qesgd_mx4_grouped_product", c.dtype
    dtype = _dtype(c, where)
    device, stream = _here(where, stream, c)
    y = c.data_ptr() if c.is_contiguous() and c.numel() >= (R - 1) * ldc + N else _rows(where, device, c, kind, R, ldc, N)
    f = offsets.data_ptr() if offsets.dtype is _I32 and offsets.get_device() == device and offsets.is_contiguous() and offsets.numel() > E \
        else _ints(where, device, offsets, E + 1)
    ws, ws_bytes = (None, 0) if workspace is None else _ws(where, device, workspace)
    rc = (_lib or lib()).qesgd_mx4_grouped_product(_packed(where, device, a_packed, R, K), _packed(where, device, b_slab, N, K, E, b_stride), b_stride, f, E, R, N,
                                                   K, y, dtype, ldc, ws, ws_bytes, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_mx4_grouped_gradient_workspace_bytes(R: int, N: int, K: int, E: int) -> int:
    return int(lib().qesgd_mx4_grouped_gradient_workspace_bytes(int(R), int(N), int(K), int(E)))


def qesgd_mx4_grouped_gradient(a_packed_t, b_packed_t, offsets, E, R, N, K, d, workspace=None, stream=None):
    where, kind = "qesgd_mx4_grouped_gradient", d.dtype
    dtype = _dtype(d, where)
    device, stream = _here(where, stream, d)
    columns = (R + 127 * min(E, R)) // 128 * 128
    y = d.data_ptr() if d.is_contiguous() and d.numel() >= E * N * K else _rows(where, device, d, kind, E, N * K, N * K)
    ws, ws_bytes = (None, 0) if workspace is None else _ws(where, device, workspace)
    rc = (_lib or lib()).qesgd_mx4_grouped_gradient(_packed(where, device, a_packed_t, N, columns), _packed(where, device, b_packed_t, K, columns),
                                                    _ints(where, device, offsets, E + 1), E, R, N, K, y, dtype, ws, ws_bytes, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_mx4_vector_product_workspace_bytes(R: int, N: int, K: int, E: int) -> int:
    return int(lib().qesgd_mx4_vector_product_workspace_bytes(int(R), int(N), int(K), int(E)))


def qesgd_mx4_vector_product(x, ld, T, order, per, w_slab, w_stride, offsets, E, R, N, K, y, ldy, workspace=None, stream=None):
    where, kind = "qesgd_mx4_vector_product", x.dtype
    dtype = _dtype(x, where)
    device, stream = _here(where, stream, y)
    own = kind                                                # y's type
    if y.dtype is _F32 and kind is not _F32:
        dtype, own = dtype | ROWS_F32, _F32
    a = x.data_ptr() if x.get_device() == device and x.is_contiguous() and x.numel() >= (T - 1) * ld + K \
        else _rows(where, device, x, kind, T, ld, K)
    c = y.data_ptr() if y.dtype is own and y.is_contiguous() and y.numel() >= (R - 1) * ldy + N else _rows(where, device, y, own, R, ldy, N)
    o = None if order is None else order.data_ptr() if order.dtype is _I32 and order.get_device() == device and order.is_contiguous() and \
        order.numel() >= R else _ints(where, device, order, R)
    f = None if offsets is None else offsets.data_ptr() if offsets.dtype is _I32 and offsets.get_device() == device and offsets.is_contiguous() and \
        offsets.numel() > E else _ints(where, device, offsets, E + 1)
    ws, ws_bytes = (None, 0) if workspace is None else _ws(where, device, workspace)
    rc = (_lib or lib()).qesgd_mx4_vector_product(a, dtype, ld, T, o, per, _packed(where, device, w_slab, N, K, E, w_stride), w_stride, f, E, R, N, K, c, ldy, ws,
                                                  ws_bytes, stream)
    if rc:
        raise QesgdError(rc, where)


def qesgd_abi_version() -> int:
    return int(lib().qesgd_abi_version())


def qesgd_last_hip_error() -> int:
    return int(lib().qesgd_last_hip_error())


# ---- allocation helpers (torch is the allocator) ---------------------------

def alloc_packed(lay: Layout, K: int, device="cuda") -> torch.Tensor:
    """[K, bytes_per_worker] uint8, 256-byte aligned rows (torch's allocator aligns to 512)."""
    t = torch.empty((K, lay.bytes_per_worker), dtype=torch.uint8, device=device)
    assert t.data_ptr() % 256 == 0
    return t


def planes(packed_row: torch.Tensor, lay: Layout):
    """Views (norms f32[nb], signs i32[sign_words], levels i32[level_words]) of one packed block."""
    norms = packed_row[lay.norms_off: lay.norms_off + 4 * lay.n_buckets].view(torch.float32)
    signs = packed_row[lay.signs_off: lay.signs_off + 4 * lay.sign_words].view(torch.int32)
    levels = packed_row[lay.levels_off: lay.levels_off + 4 * lay.level_words].view(torch.int32)
    return norms, signs, levels


def alloc_mx4(lay: Mx4Layout, K: Optional[int] = None, device="cuda") -> torch.Tensor:
    """[bytes] or [K, bytes] uint8 for the packed 4-bit form, 256-byte aligned."""
    t = torch.empty((lay.bytes,) if K is None else (K, lay.bytes), dtype=torch.uint8, device=device)
    assert t.data_ptr() % 256 == 0
    return t


def alloc_workspace(n_bytes: int, device="cuda") -> Optional[torch.Tensor]:
    """Device scratch of that many bytes, None for none."""
    return torch.empty(n_bytes, dtype=torch.uint8, device=device) if n_bytes else None
