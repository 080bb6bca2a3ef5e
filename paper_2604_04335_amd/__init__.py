"""Python binding of the MI355X DiT denoising-step attention library.

Argument marshalling only: every step of the computation runs in the HIP
kernels behind the C ABI declared in include/dit_attn.h.  PyTorch is used by
callers for device memory and streams; this module itself only needs ctypes
and numpy, and accepts anything with `data_ptr()` (torch tensors) or a raw
integer device address.

There is no CPU fallback: if the shared library has not been built
(`python -m paper_2604_04335_amd.build`) importing the symbols raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct

import numpy as np

__all__ = [
    "DitAttnError",
    "lib_path",
    "load_library",
    "dit_attn_version",
    "dit_attn_create",
    "dit_attn_varlen_fwd",
    "dit_attn_varlen_fwd_noalloc",
    "dit_attn_varlen_fwd_lse",
    "dit_attn_cross_varlen_fwd",
    "dit_attn_merge",
    "dit_attn_sp_pack_heads",
    "dit_attn_sp_unpack_heads",
    "dit_attn_rope_table",
    "dit_attn_qk_norm_rope",
    "dit_attn_masked_varlen_fwd",
    "RopeSpec",
    "NormHeads",
    "AttnMask",
    "ROPE_PLAIN",
    "ROPE_LINEAR",
    "ROPE_BASE",
    "ROPE_BANDS",
    "ROPE_INTERLEAVED",
    "ROPE_HALF",
    "NORM_NONE",
    "NORM_RMS",
    "NORM_LAYER",
    "dit_sched_laxity",
    "dit_sched_plan_round",
    "SchedCandidate",
    "dit_attn_destroy",
    "dit_attn_last_error",
    "dit_attn_plan",
    "dit_attn_plan_cache_victim",
    "dit_attn_set_kernel",
    "dit_attn_set_split_kv",
    "dit_attn_last_launch_clock",
    "dit_attn_last_launch_kernel",
    "KERNEL_AUTO",
    "KERNEL_128",
    "KERNEL_PINGPONG",
    "DitAttention",
]

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB = None

ERROR_NAMES = {
    0: "DIT_ATTN_OK",
    -1: "DIT_ATTN_ERR_NULL",
    -2: "DIT_ATTN_ERR_HEAD_DIM",
    -3: "DIT_ATTN_ERR_CU_SEQLENS",
    -4: "DIT_ATTN_ERR_HIP",
    -5: "DIT_ATTN_ERR_SCALE",
    -6: "DIT_ATTN_ERR_N_HEADS",
    -7: "DIT_ATTN_ERR_ALIGN",
    -8: "DIT_ATTN_ERR_CAPACITY",
    -9: "DIT_ATTN_ERR_KERNEL",
    -10: "DIT_ATTN_ERR_PARTS",
    -11: "DIT_ATTN_ERR_LIMIT",
    -12: "DIT_ATTN_ERR_CAPTURE",
    -13: "DIT_ATTN_ERR_MASK",
    -14: "DIT_ATTN_ERR_ROPE",
    -15: "DIT_ATTN_ERR_NORM",
    -16: "DIT_ATTN_ERR_STRIDE",
}


class SchedCandidate(ctypes.Structure):
    """dit_sched_candidate of include/dit_sched.h."""
    _fields_ = [("gpus", ctypes.c_int32), ("gpu_mask", ctypes.c_uint32), ("laxity", ctypes.c_double),
                ("hold", ctypes.c_int32), ("reserved", ctypes.c_int32)]


ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BANDS = 0, 1, 2, 3
ROPE_INTERLEAVED, ROPE_HALF = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2


class RopeSpec(ctypes.Structure):
    """dit_attn_rope of include/dit_attn.h.  axis_dim: rotated elements of each axis; theta, factor and original_length: one
    value for all axes or one for each."""
    _fields_ = [("n_axes", ctypes.c_int32), ("scaling", ctypes.c_int32), ("axis_dim", ctypes.c_int32 * 4),
                ("theta", ctypes.c_double * 4), ("factor", ctypes.c_double * 4), ("original_length", ctypes.c_double * 4),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("magnitude", ctypes.c_double)]

    def __init__(self, axis_dim, theta=10000.0, scaling=ROPE_PLAIN, factor=1.0, original_length=0.0, low=1.0, high=32.0,
                 magnitude=1.0):
        dims = [int(d) for d in axis_dim]

        def each(name, x):
            vals = [float(v) for v in x] if hasattr(x, "__len__") else [float(x)] * len(dims)
            if len(vals) != len(dims):
                raise ValueError(f"{name}: one value, or one for each of the {len(dims)} axes")
            return (ctypes.c_double * 4)(*vals)

        if not 1 <= len(dims) <= 4:
            raise ValueError("1 to 4 axes")
        super().__init__(len(dims), int(scaling), (ctypes.c_int32 * 4)(*dims), each("theta", theta), each("factor", factor),
                         each("original_length", original_length), float(low), float(high), float(magnitude))

    @property
    def rot_dim(self) -> int:
        return sum(self.axis_dim[:self.n_axes])


class NormHeads(ctypes.Structure):
    """dit_attn_norm_heads of include/dit_attn.h: one side, queries or keys.  x and out: bf16 tensors [n_rows, n_heads, head_dim]
    whose heads are contiguous (rows may be strided), out = x replaces in place; or integer addresses with n_heads given.
    weight, bias: fp32 [head_dim] or None."""
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("out_row_stride", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("n_heads", ctypes.c_int32)]
    _needs = (None, None, None, None)  # of a structure whose fields were filled in one by one

    def __init__(self, x, out, weight=None, bias=None, n_heads=None, row_stride=None, out_row_stride=None):
        # What a call has to agree with: the shapes of tensors whose strides are their own, the elements of weight and bias, and the
        # device of all (of which -2 is none).
        x_shape = out_shape = device = n_weight = None
        if hasattr(x, "stride"):
            x_shape, device, self.x = x.shape, x.get_device(), x.data_ptr()
            if n_heads is None:
                n_heads = x_shape[1]
            if row_stride is None:
                row_stride = _row_stride(x, "x", x_shape)
            else:
                _check_kind(x, "x", _BF16)
                x_shape = None
        else:
            self.x = _ptr(x)
        if hasattr(out, "stride"):
            out_shape, where, self.out = out.shape, out.get_device(), out.data_ptr()
            if out_row_stride is None:
                out_row_stride = _row_stride(out, "out", out_shape)
                if out_shape == x_shape:
                    out_shape = None
            else:
                _check_kind(out, "out", _BF16)
                out_shape = None
            if where != device:
                device = where if device is None else -2
        else:
            self.out = _ptr(out)
        # (Fields are 0 to begin with.)
        if row_stride:
            self.row_stride = int(row_stride)
        if out_row_stride:
            self.out_row_stride = int(out_row_stride)
        self.n_heads = int(n_heads)
        if weight is not None:
            self.weight = _array(weight, "weight", _FP32)
            if hasattr(weight, "stride"):
                n_weight, where = weight.numel(), weight.get_device()
                if where != device:
                    device = where if device is None else -2
        if bias is not None:
            self.bias = _array(bias, "bias", _FP32)
            if hasattr(bias, "stride"):
                n, where = bias.numel(), bias.get_device()
                n_weight = n if n_weight is None or n < n_weight else n_weight
                if where != device:
                    device = where if device is None else -2
        self._held = (x, out, weight, bias)
        self._needs = (x_shape, out_shape, n_weight, device)

    def _check(self, n_rows: int, head_dim: int, on) -> None:
        x_shape, out_shape, n_weight, device = self._needs
        if x_shape is not None:
            _check_size("x", x_shape, n_rows, self.n_heads, head_dim)
        if out_shape is not None:
            _check_size("out", out_shape, n_rows, self.n_heads, head_dim)
        if n_weight is not None and n_weight < head_dim:
            raise ValueError(f"weight, bias: at least {head_dim} elements, not {n_weight}")
        if device != on and device is not None:
            _check_device("x, out, weight, bias", device, on)


class AttnMask(ctypes.Structure):
    """dit_attn_mask of include/dit_attn.h.  prefix: host integers, one a sequence; slopes: device fp32 [n_heads]; q_doc, k_doc:
    device int32 [Tq], [Tk]."""
    _fields_ = [("causal", ctypes.c_int32), ("softcap", ctypes.c_float), ("prefix", ctypes.POINTER(ctypes.c_int32)),
                ("slopes", ctypes.c_void_p), ("q_doc", ctypes.c_void_p), ("k_doc", ctypes.c_void_p)]
    n_prefix, _held = None, (None, None, None, None)  # of a structure whose fields were filled in one by one

    def __init__(self, causal=False, prefix=None, softcap=0.0, slopes=None, q_doc=None, k_doc=None):
        self.n_prefix = None
        if prefix is not None:
            prefix = [int(x) for x in prefix]
            self.n_prefix = len(prefix)
            prefix = (ctypes.c_int32 * max(len(prefix), 1))(*prefix)
        super().__init__(int(causal), float(softcap), prefix, _array(slopes, "slopes", _FP32), _array(q_doc, "q_doc", _INT32),
                         _array(k_doc, "k_doc", _INT32))
        self._held = (prefix, slopes, q_doc, k_doc)


class DitAttnError(RuntimeError):
    def __init__(self, code: int, message: str = ""):
        self.code = code
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {message}")


def lib_path() -> str:
    return os.path.join(_PKG_DIR, "libdit_attn.so")


def load_library() -> ctypes.CDLL:
    """Load libdit_attn.so (built in-tree).  Raises if it is missing: there is no fallback."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing; build it with `python -m paper_2604_04335_amd.build`")
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    i32p = ctypes.POINTER(ctypes.c_int32)
    lib.dit_attn_version.restype = ctypes.c_char_p
    lib.dit_attn_version.argtypes = []
    lib.dit_attn_create.restype = ctypes.c_int
    lib.dit_attn_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int]
    lib.dit_attn_varlen_fwd.restype = ctypes.c_int
    lib.dit_attn_varlen_fwd.argtypes = [vp, vp, vp, vp, i32p, i32, i32, i32, ctypes.c_float, vp, vp]
    lib.dit_attn_varlen_fwd_noalloc.restype = ctypes.c_int
    lib.dit_attn_varlen_fwd_noalloc.argtypes = [vp, vp, vp, vp, i32p, i32, i32, i32, ctypes.c_float, vp, vp]
    lib.dit_attn_destroy.restype = None
    lib.dit_attn_destroy.argtypes = [vp]
    lib.dit_attn_varlen_fwd_lse.restype = ctypes.c_int
    lib.dit_attn_varlen_fwd_lse.argtypes = [vp, vp, vp, vp, i32p, i32, i32, i32, ctypes.c_float, vp, vp, vp]
    lib.dit_attn_cross_varlen_fwd.restype = ctypes.c_int
    lib.dit_attn_cross_varlen_fwd.argtypes = [vp, vp, vp, vp, i32p, i32p, i32, i32, i32, ctypes.c_float, vp, vp, vp]
    for fn in (lib.dit_attn_sp_pack_heads, lib.dit_attn_sp_unpack_heads):
        fn.restype = ctypes.c_int
        fn.argtypes = [vp, vp, vp, i64, i32, i32, i32, vp]
    lib.dit_attn_rope_table.restype = ctypes.c_int
    lib.dit_attn_rope_table.argtypes = [vp, vp, i64, ctypes.POINTER(RopeSpec), vp, vp]
    lib.dit_attn_qk_norm_rope.restype = ctypes.c_int
    lib.dit_attn_qk_norm_rope.argtypes = [vp, ctypes.POINTER(NormHeads), ctypes.POINTER(NormHeads), i64, i32, i32, ctypes.c_float, vp,
                                          i32, i32, vp]
    lib.dit_attn_masked_varlen_fwd.restype = ctypes.c_int
    lib.dit_attn_masked_varlen_fwd.argtypes = [vp, vp, vp, vp, ctypes.POINTER(i64), vp, vp, i32, i32, i32, i32, ctypes.c_float,
                                               ctypes.POINTER(AttnMask), vp, vp, vp]
    lib.dit_sched_laxity.restype = ctypes.c_double
    lib.dit_sched_laxity.argtypes = [ctypes.c_double, ctypes.c_double, i32, ctypes.c_double]
    f64p = ctypes.POINTER(ctypes.c_double)
    lib.dit_sched_plan_round.restype = ctypes.c_int
    lib.dit_sched_plan_round.argtypes = [i32, ctypes.POINTER(SchedCandidate), i32p, i32, f64p, i32, ctypes.c_double, f64p, i32,
                                         i32p, i32p, i32p, i32p, i32p, i32p, f64p]
    lib.dit_attn_merge.restype = ctypes.c_int
    lib.dit_attn_merge.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), i32, i64, i32, i32, vp, vp, vp]
    lib.dit_attn_last_error.restype = ctypes.c_char_p
    lib.dit_attn_last_error.argtypes = [vp]
    lib.dit_attn_set_split_kv.restype = ctypes.c_int
    lib.dit_attn_set_split_kv.argtypes = [vp, ctypes.c_int]
    lib.dit_attn_set_kernel.restype = ctypes.c_int
    lib.dit_attn_set_kernel.argtypes = [vp, ctypes.c_int]
    lib.dit_attn_last_launch_kernel.restype = ctypes.c_int
    lib.dit_attn_last_launch_kernel.argtypes = [vp]
    lib.dit_attn_last_launch_clock.restype = ctypes.c_int
    lib.dit_attn_last_launch_clock.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.dit_attn_plan_cache_victim.restype = i32
    lib.dit_attn_plan_cache_victim.argtypes = [ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint8), i32]
    lib.dit_attn_plan.restype = i64
    lib.dit_attn_plan.argtypes = [i32p, i32, i32, i32, i32p, i64, i32p]
    _LIB = lib
    return lib


def _ptr(x) -> int:
    if type(x) is int:
        return x
    if x is None:
        return 0
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x)


_I64x3 = ctypes.c_int64 * 3

# What the rotation table, the norm and rotation and the masked attention ask of tensors, so that none is read as another kind, past
# its end or on another device than the context's.  Addresses are taken as they are.
_CTX_DEVICE: dict = {}  # device of every context


class _Kind(set):
    """Tensor types that an argument may have, as far as they have been met, and the names of all: this module does not import
    torch."""

    def __init__(self, what, *names):
        super().__init__()
        self.what, self.names = what, names

    def meet(self, dtype) -> bool:
        if str(dtype) not in self.names:
            return False
        self.add(dtype)
        return True


_BF16 = _Kind("bf16", "torch.bfloat16", "torch.int16", "torch.uint16")  # the integers: bit patterns
_FP32 = _Kind("fp32", "torch.float32")
_INT32 = _Kind("int32", "torch.int32", "torch.uint32")


def _check_kind(x, name: str, kind: _Kind) -> None:
    if x.dtype not in kind and not kind.meet(x.dtype):
        raise ValueError(f"{name}: a {kind.what} tensor, not {x.dtype}")


def _row_stride(x, name: str, shape) -> int:
    """Elements from row to row of a bf16 tensor [rows, heads, head_dim] with contiguous heads; 0: contiguous."""
    if x.dtype in _BF16 or _BF16.meet(x.dtype):
        if x.is_contiguous():
            return 0
        if len(shape) == 3:
            row, head, one = x.stride()
            if (one == 1 or shape[2] == 1) and (head == shape[2] or shape[1] == 1):
                if shape[0] == 1:
                    return 0
                if row > 0:  # 0, which an expanded tensor has, would stand for contiguous rows
                    return row
    raise ValueError(f"{name}: a bf16 tensor [rows, heads, head_dim] whose heads are contiguous")


def _check_size(name: str, shape, n_rows: int, heads: int, head_dim: int) -> None:
    """At least n_rows rows of heads * head_dim elements.  A contiguous tensor of other than three dimensions may hold them too."""
    if len(shape) == 3:
        rows, h, d = shape
        if rows >= n_rows and h == heads and d == head_dim:
            return
    elif len(shape) < 2 or shape[-1] == heads * head_dim or shape[-2:] == (heads, head_dim):
        if math.prod(shape) >= n_rows * heads * head_dim:
            return
    raise ValueError(f"{name}: {n_rows} rows of {heads} heads of {head_dim} elements, not {tuple(shape)}")


def _check_device(name: str, where: int, device) -> None:
    if where != device and device is not None:  # (the library refuses a call without a context)
        raise ValueError(f"{name}: on device {where} (-1: the host), the context on {device}")


def _operand(x, name: str, n_rows: int, heads, head_dim: int, device, own: bool):
    """(address, elements from row to row or 0) of queries, keys, values or an output; own: the tensor's strides count.  heads is
    None in a call that the library refuses."""
    if not hasattr(x, "stride"):
        return _ptr(x), 0
    row = 0
    if own:
        shape = x.shape
        row = _row_stride(x, name, shape)
        if heads is not None:
            _check_size(name, shape, n_rows, heads, head_dim)
    else:
        _check_kind(x, name, _BF16)
    where = x.get_device()
    if where != device:
        _check_device(name, where, device)
    return x.data_ptr(), row


def _array(x, name: str, kind: _Kind, size: int = 0, device=None) -> int:
    """Address of a contiguous device array of at least `size` elements; a tensor of another kind is refused."""
    if x is None:
        return 0
    try:
        dtype = x.dtype
    except AttributeError:
        return int(x)
    if (dtype not in kind and not kind.meet(dtype)) or not x.is_contiguous():
        raise ValueError(f"{name}: a contiguous {kind.what} tensor")
    if size and x.numel() < size:
        raise ValueError(f"{name}: at least {size} elements, not {x.numel()}")
    if device is not None:
        where = x.get_device()
        if where != device:
            _check_device(name, where, device)
    return x.data_ptr()


def _cu_array(cu_seqlens) -> np.ndarray:
    if hasattr(cu_seqlens, "detach"):  # torch tensor: must live on the host
        if cu_seqlens.device.type != "cpu":
            raise ValueError("cu_seqlens must be a host array")
        cu_seqlens = cu_seqlens.detach().numpy()
    return np.ascontiguousarray(cu_seqlens, dtype=np.int32)


def dit_attn_version() -> str:
    return load_library().dit_attn_version().decode()


def dit_attn_last_error(ctx) -> str:
    return load_library().dit_attn_last_error(ctypes.c_void_p(ctx or 0)).decode()


def dit_attn_create(device_id: int = 0) -> int:
    """Returns an opaque context handle (an integer address)."""
    lib = load_library()
    h = ctypes.c_void_p()
    rc = lib.dit_attn_create(ctypes.byref(h), int(device_id))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(None))
    _CTX_DEVICE[int(h.value)] = int(device_id)
    return int(h.value)


KERNEL_AUTO, KERNEL_128, KERNEL_PINGPONG = -1, 0, 1


def dit_attn_set_kernel(ctx, kernel: int) -> None:
    """Force one of the library's kernels for later calls on `ctx` (KERNEL_AUTO: chosen per pack)."""
    rc = load_library().dit_attn_set_kernel(ctypes.c_void_p(ctx), int(kernel))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_set_split_kv(ctx, max_splits: int) -> None:
    """Allow small packs to split every sequence's keys into up to max_splits chunks (1 = off); see include/dit_attn.h."""
    rc = load_library().dit_attn_set_split_kv(ctypes.c_void_p(ctx), int(max_splits))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_last_launch_clock(ctx):
    """(shader clock in MHz, milliseconds) sampled by the first workgroup of the last launch; synchronises the device."""
    mhz, ms = ctypes.c_double(0.0), ctypes.c_double(0.0)
    rc = load_library().dit_attn_last_launch_clock(ctypes.c_void_p(ctx), ctypes.byref(mhz), ctypes.byref(ms))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))
    return mhz.value, ms.value


def dit_attn_last_launch_kernel(ctx) -> int:
    """KERNEL_128 / KERNEL_PINGPONG: the kernel the last forward call launched; KERNEL_AUTO before any."""
    return int(load_library().dit_attn_last_launch_kernel(ctypes.c_void_p(ctx)))


def dit_attn_destroy(ctx) -> None:
    if ctx:
        _CTX_DEVICE.pop(ctx, None)
        load_library().dit_attn_destroy(ctypes.c_void_p(ctx))


def dit_attn_varlen_fwd(ctx, q, k, v, cu_seqlens, n_heads: int, head_dim: int, scale: float, out, stream=None,
                        n_seqs: int | None = None) -> None:
    """One denoising-step attention call; see include/dit_attn.h.

    q, k, v, out: device buffers (torch tensors or integer addresses), bf16 [T, n_heads, head_dim].
    cu_seqlens: host int32 sequence of n_seqs + 1 offsets.  stream: integer hipStream_t or None.
    Raises DitAttnError on a non-zero return code.
    """
    lib = load_library()
    cu = _cu_array(cu_seqlens)
    if n_seqs is None:
        n_seqs = len(cu) - 1
    rc = lib.dit_attn_varlen_fwd(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(q)), ctypes.c_void_p(_ptr(k)),
                                 ctypes.c_void_p(_ptr(v)), cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                 int(n_seqs), int(n_heads), int(head_dim), float(scale),
                                 ctypes.c_void_p(_ptr(out)), ctypes.c_void_p(_ptr(stream)))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_varlen_fwd_noalloc(ctx, q, k, v, cu_seqlens, n_heads: int, head_dim: int, scale: float, out, stream=None,
                                n_seqs: int | None = None) -> None:
    """dit_attn_varlen_fwd for callers that cannot allocate: same arguments and result, fixed limits; see include/dit_attn.h."""
    lib = load_library()
    cu = _cu_array(cu_seqlens)
    if n_seqs is None:
        n_seqs = len(cu) - 1
    rc = lib.dit_attn_varlen_fwd_noalloc(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(q)), ctypes.c_void_p(_ptr(k)),
                                         ctypes.c_void_p(_ptr(v)), cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                         int(n_seqs), int(n_heads), int(head_dim), float(scale),
                                         ctypes.c_void_p(_ptr(out)), ctypes.c_void_p(_ptr(stream)))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_varlen_fwd_lse(ctx, q, k, v, cu_seqlens, n_heads: int, head_dim: int, scale: float, out, lse, stream=None,
                            n_seqs: int | None = None) -> None:
    """dit_attn_varlen_fwd that also writes lse (device fp32 [T, n_heads], natural log); see include/dit_attn.h."""
    lib = load_library()
    cu = _cu_array(cu_seqlens)
    if n_seqs is None:
        n_seqs = len(cu) - 1
    rc = lib.dit_attn_varlen_fwd_lse(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(q)), ctypes.c_void_p(_ptr(k)),
                                     ctypes.c_void_p(_ptr(v)), cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                     int(n_seqs), int(n_heads), int(head_dim), float(scale),
                                     ctypes.c_void_p(_ptr(out)), ctypes.c_void_p(_ptr(lse)), ctypes.c_void_p(_ptr(stream)))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_cross_varlen_fwd(ctx, q, k, v, cu_seqlens_q, cu_seqlens_k, n_heads: int, head_dim: int, scale: float, out,
                              lse=None, stream=None, n_seqs: int | None = None) -> None:
    """Cross-attention with separate query and key boundaries; lse may be None.  See include/dit_attn.h."""
    lib = load_library()
    cq = _cu_array(cu_seqlens_q)
    ck = None if cu_seqlens_k is None else _cu_array(cu_seqlens_k)
    if n_seqs is None:
        n_seqs = len(cq) - 1
    i32p = ctypes.POINTER(ctypes.c_int32)
    rc = lib.dit_attn_cross_varlen_fwd(ctypes.c_void_p(ctx), ctypes.c_void_p(_ptr(q)), ctypes.c_void_p(_ptr(k)),
                                       ctypes.c_void_p(_ptr(v)), cq.ctypes.data_as(i32p),
                                       None if ck is None else ck.ctypes.data_as(i32p),
                                       int(n_seqs), int(n_heads), int(head_dim), float(scale),
                                       ctypes.c_void_p(_ptr(out)), ctypes.c_void_p(_ptr(lse)), ctypes.c_void_p(_ptr(stream)))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_merge(ctx, o_parts, lse_parts, total_rows: int, n_heads: int, head_dim: int, out, lse_out=None,
                   stream=None) -> None:
    """Merge partial results over disjoint key sets; o_parts / lse_parts: sequences of device buffers.  See the header."""
    lib = load_library()
    n = len(o_parts)
    vp = ctypes.c_void_p
    o_arr = (vp * max(n, 1))(*[vp(_ptr(x)) for x in o_parts])
    l_arr = (vp * max(n, 1))(*[vp(_ptr(x)) for x in lse_parts]) if len(lse_parts) == n else None
    if l_arr is None:
        raise ValueError("o_parts and lse_parts must have the same length")
    rc = lib.dit_attn_merge(vp(ctx), o_arr, l_arr, int(n), int(total_rows), int(n_heads), int(head_dim), vp(_ptr(out)),
                            vp(_ptr(lse_out)), vp(_ptr(stream)))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def _sp_layout(name, ctx, src, dst, n_rows, n_heads, head_dim, sp_degree, stream):
    vp = ctypes.c_void_p
    rc = getattr(load_library(), name)(vp(ctx), vp(_ptr(src)), vp(_ptr(dst)), int(n_rows), int(n_heads), int(head_dim),
                                       int(sp_degree), vp(_ptr(stream)))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_sp_pack_heads(ctx, src, dst, n_rows: int, n_heads: int, head_dim: int, sp_degree: int, stream=None) -> None:
    """[n_rows, H, D] -> [p, n_rows, H/p, D] (block g goes to rank g); see include/dit_attn.h."""
    _sp_layout("dit_attn_sp_pack_heads", ctx, src, dst, n_rows, n_heads, head_dim, sp_degree, stream)


def dit_attn_sp_unpack_heads(ctx, src, dst, n_rows: int, n_heads: int, head_dim: int, sp_degree: int, stream=None) -> None:
    """[p, n_rows, H/p, D] -> [n_rows, H, D] (block g came from rank g); see include/dit_attn.h."""
    _sp_layout("dit_attn_sp_unpack_heads", ctx, src, dst, n_rows, n_heads, head_dim, sp_degree, stream)


_MAX_ROWS = 2 ** 34  # more are refused by the library
_AXES = struct.Struct("6i").unpack_from  # n_axes, scaling and axis_dim of a RopeSpec


def dit_attn_rope_table(ctx, positions, n_rows: int, rope: RopeSpec, table, stream=None) -> None:
    """table[r, pair] = (cos, sin) of the row's positions; positions: device int32 [n_rows, n_axes]; see include/dit_attn.h."""
    n_positions = n_values = 0
    if isinstance(rope, RopeSpec) and n_rows <= _MAX_ROWS:
        axes, _, *dims = _AXES(rope)
        size = sum(dims[:axes])
        if 1 <= axes <= 4 and size <= 128:  # else the library refuses the call
            n_positions, n_values = n_rows * axes, n_rows * size
    device = _CTX_DEVICE.get(ctx)
    rc = load_library().dit_attn_rope_table(ctx, _array(positions, "positions", _INT32, n_positions, device), n_rows, rope,
                                            _array(table, "table", _FP32, n_values, device), _ptr(stream))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_qk_norm_rope(ctx, q, k, n_rows: int, head_dim: int, norm: int, eps: float, table=None, rot_dim: int = 0,
                          layout: int = ROPE_INTERLEAVED, stream=None) -> None:
    """Norm of queries and keys for each head and rotation; q, k: NormHeads, or None for one of them; see include/dit_attn.h."""
    device, n_values = _CTX_DEVICE.get(ctx), 0
    if n_rows <= _MAX_ROWS and (head_dim == 128 or head_dim == 64):  # else the library refuses the call
        if rot_dim <= head_dim:
            n_values = n_rows * rot_dim
        if isinstance(q, NormHeads):
            q._check(n_rows, head_dim, device)
        if isinstance(k, NormHeads):
            k._check(n_rows, head_dim, device)
    rc = load_library().dit_attn_qk_norm_rope(ctx, q, k, n_rows, head_dim, norm, eps, _array(table, "table", _FP32, n_values, device),
                                              rot_dim, layout, _ptr(stream))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_masked_varlen_fwd(ctx, q, k, v, cu_seqlens_q, cu_seqlens_k, n_heads: int, n_kv_heads: int, head_dim: int, scale: float,
                               mask: AttnMask | None, out, lse=None, stream=None, row_strides=None, n_seqs: int | None = None) -> None:
    """Attention with masks, capped scores and a distance bias; see include/dit_attn.h.

    q, k, v: bf16 tensors [rows, heads, head_dim] whose rows may be strided, or integer addresses (with row_strides, three
    numbers of elements, 0: contiguous).  cu_seqlens_k may be None (that of the queries); mask, lse may be None.  Tensors of
    another type, shape or device than the call reads, or too small for it, raise ValueError; with row_strides their type and
    device are looked at alone.
    """
    lib = load_library()
    cq = _cu_array(cu_seqlens_q)
    ck = None if cu_seqlens_k is None else _cu_array(cu_seqlens_k)
    if n_seqs is None:
        n_seqs = len(cq) - 1
    if (ck is not None and len(ck) <= n_seqs) or len(cq) <= n_seqs:
        raise ValueError("cu_seqlens_q and cu_seqlens_k need n_seqs + 1 entries")
    if mask is not None and mask.n_prefix is not None and mask.n_prefix < n_seqs:
        raise ValueError("mask.prefix needs an entry for every sequence")
    device, heads, kv_heads, rows, keys = _CTX_DEVICE.get(ctx), None, None, 0, 0
    if n_seqs >= 0 and (head_dim == 128 or head_dim == 64) and n_heads > 0 and n_kv_heads > 0 and n_heads % n_kv_heads == 0:
        heads, kv_heads = n_heads, n_kv_heads  # else the library refuses the call
        rows = cq.item(n_seqs)
        keys = rows if ck is None else ck.item(n_seqs)
    own = row_strides is None
    q_at, q_row = _operand(q, "q", rows, heads, head_dim, device, own)
    k_at, k_row = _operand(k, "k", keys, kv_heads, head_dim, device, own)
    v_at, v_row = _operand(v, "v", keys, kv_heads, head_dim, device, own)
    out_at, out_row = _operand(out, "out", rows, heads, head_dim, device, True)
    if out_row != 0:
        raise ValueError("out: contiguous rows")
    if not own:
        row_strides = _I64x3(*row_strides)
    elif q_row or k_row or v_row:
        row_strides = _I64x3(q_row, k_row, v_row)
    if mask is not None and heads is not None:
        _, slopes, q_doc, k_doc = mask._held
        if slopes is not None:
            _array(slopes, "slopes", _FP32, n_heads, device)
        if q_doc is not None:
            _array(q_doc, "q_doc", _INT32, rows, device)
        if k_doc is not None:
            _array(k_doc, "k_doc", _INT32, keys, device)
    # (The boundaries' bytes: an array's address takes longer.)
    rc = lib.dit_attn_masked_varlen_fwd(ctx, q_at, k_at, v_at, row_strides, cq.tobytes(),
                                        None if ck is None else ck.tobytes(), n_seqs, n_heads, n_kv_heads, head_dim, scale, mask, out_at,
                                        _array(lse, "lse", _FP32, rows * heads if heads else 0, device), _ptr(stream))
    if rc != 0:
        raise DitAttnError(rc, dit_attn_last_error(ctx))


def dit_attn_plan(cu_seqlens, n_heads: int, head_dim: int):
    """Host-only: the ordered work-list as an int32 array [n_items, 4] and the tile height block_m."""
    lib = load_library()
    cu = _cu_array(cu_seqlens)
    n_seqs = len(cu) - 1
    cu_p = cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    bm = ctypes.c_int32(0)
    n = lib.dit_attn_plan(cu_p, n_seqs, int(n_heads), int(head_dim), None, 0, ctypes.byref(bm))
    if n < 0:
        raise DitAttnError(int(n), "dit_attn_plan")
    items = np.zeros((max(int(n), 1), 4), dtype=np.int32)
    n2 = lib.dit_attn_plan(cu_p, n_seqs, int(n_heads), int(head_dim),
                           items.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), int(items.shape[0]), ctypes.byref(bm))
    if n2 < 0:
        raise DitAttnError(int(n2), "dit_attn_plan")
    return items[:int(n2)], int(bm.value)


def dit_attn_plan_cache_victim(last_use, pinned) -> int:
    """Host-only: which of the cached packs (use counters, pin flags) the plan cache evicts next; -1 if all are pinned."""
    lu = np.ascontiguousarray(last_use, dtype=np.uint64)
    pn = np.ascontiguousarray(pinned, dtype=np.uint8)
    assert lu.size == pn.size
    return int(load_library().dit_attn_plan_cache_victim(lu.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                                         pn.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)), int(lu.size)))


class DitAttention:
    """Owns one context; `forward` takes torch tensors and uses torch's current stream."""

    def __init__(self, device_id: int = 0):
        self.device_id = int(device_id)
        self.ctx = dit_attn_create(self.device_id)

    def forward(self, q, k, v, cu_seqlens, scale: float | None = None, out=None, stream=None):
        import torch  # device memory and streams only

        T, H, D = q.shape
        assert q.dtype == torch.bfloat16 and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        assert k.shape == q.shape and v.shape == q.shape
        if out is None:
            out = torch.empty_like(q)
        if scale is None:
            scale = float(D) ** -0.5
        if stream is None:
            stream = torch.cuda.current_stream(q.device).cuda_stream
        dit_attn_varlen_fwd(self.ctx, q, k, v, cu_seqlens, H, D, scale, out, stream)
        return out

    __call__ = forward

    def close(self):
        if self.ctx:
            dit_attn_destroy(self.ctx)
            self.ctx = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def dit_sched_laxity(deadline: float, t_now: float, steps_remaining: int, t_step: float) -> float:
    """Eq. 1 of the paper for a configuration; see include/dit_sched.h."""
    return float(load_library().dit_sched_laxity(float(deadline), float(t_now), int(steps_remaining), float(t_step)))


def dit_sched_plan_round(n_gpus: int, videos, image_deadlines, t_now: float, t_img):
    """One round of the paper's Algorithm 1 (include/dit_sched.h).  videos: per video a sequence of candidates, each a
    SchedCandidate or a tuple (gpus, gpu_mask, laxity, hold).  Returns a dict with choice, video_gpus, image_batch,
    image_gpu (one GPU id per image batch), recoverable, utility.  Raises DitAttnError on an error code."""
    lib = load_library()
    flat, offs = [], [0]
    for cands in videos:
        for c in cands:
            flat.append(c if isinstance(c, SchedCandidate) else SchedCandidate(int(c[0]), int(c[1]), float(c[2]), int(bool(c[3])), 0))
        offs.append(len(flat))
    arr = (SchedCandidate * max(len(flat), 1))(*flat)
    offs_a = np.asarray(offs, dtype=np.int32)
    dl = np.ascontiguousarray(image_deadlines, dtype=np.float64)
    timg = np.ascontiguousarray(t_img, dtype=np.float64)
    G, n_img = len(videos), int(dl.size)
    choice = np.zeros(max(G, 1), dtype=np.int32)
    batch = np.zeros(max(n_img, 1), dtype=np.int32)
    gpu = np.zeros(max(int(n_gpus), 1), dtype=np.int32)
    nb, vg, rec = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
    util = ctypes.c_double(0.0)
    i32p, f64p = ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_double)
    rc = lib.dit_sched_plan_round(int(n_gpus), arr, offs_a.ctypes.data_as(i32p), G,
                                  dl.ctypes.data_as(f64p) if n_img else None, n_img, float(t_now),
                                  timg.ctypes.data_as(f64p), int(timg.size), choice.ctypes.data_as(i32p),
                                  batch.ctypes.data_as(i32p), gpu.ctypes.data_as(i32p), ctypes.byref(nb), ctypes.byref(vg),
                                  ctypes.byref(rec), ctypes.byref(util))
    if rc != 0:
        raise DitAttnError(rc, "dit_sched_plan_round")
    return {"choice": choice[:G].tolist(), "video_gpus": int(vg.value), "image_batch": batch[:n_img].tolist(),
            "image_gpu": gpu[:int(nb.value)].tolist(), "n_batches": int(nb.value), "recoverable": int(rec.value),
            "utility": float(util.value)}
