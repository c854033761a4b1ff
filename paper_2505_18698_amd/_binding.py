"""ctypes binding of libmonarch_attn.so: argument marshalling only.

Every step of the forward pass runs in the library's HIP kernels.  There is
no fallback: if the library is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmonarch_attn.so")

MA_F32, MA_BF16, MA_F16 = 0, 1, 2
MA_OK, MA_EINVAL, MA_EUNSUPPORTED, MA_EHIP, MA_ENOMEM = 0, 1, 2, 3, 4
STATUS_NAMES = {0: "MA_OK", 1: "MA_EINVAL", 2: "MA_EUNSUPPORTED", 3: "MA_EHIP", 4: "MA_ENOMEM"}
KIND_NAMES = {0: "r_half_step", 1: "l_half_step", 2: "r_half_step_final", 3: "monarch_apply",
              4: "monarch_fused_head", 5: "objective_sum", 6: "exact_attention", 7: "l_bwd", 8: "r_bwd",
              9: "monarch_fused_group", 10: "seq_attention", 11: "seq_join", 12: "seq_stats", 13: "seq_bwd",
              14: "seq_bwd_join", 15: "paged_plan", 16: "paged_write"}
PATH_AUTO, PATH_HALF_STEPS, PATH_FUSED, PATH_GROUPED = 0, 1, 2, 3

# Every symbol declared in include/monarch_attn.h.
EXPORTS = (
    "monarch_attn_fwd",
    "monarch_attn_fwd_varlen",
    "monarch_attn_fwd_objective",
    "monarch_attn_exact_fwd",
    "monarch_attn_bwd",
    "monarch_attn_bwd_varlen",
    "monarch_attn_bwd_check",
    "monarch_attn_bwd_workspace_bytes",
    "monarch_attn_last_error",
    "monarch_attn_check",
    "monarch_attn_workspace_bytes",
    "monarch_attn_release_workspace",
    "monarch_attn_set_path",
    "monarch_attn_timing_enable",
    "monarch_attn_timing_read",
    "monarch_attn_build_id",
    "monarch_attn_fwd_noalloc",
    "monarch_attn_fwd_prepad",
    "monarch_attn_exact_packed_fwd",
    "monarch_attn_exact_packed_bwd",
    "monarch_attn_exact_paged_fwd",
    "monarch_attn_paged_plan",
    "monarch_attn_paged_write",
)


class MonarchAttnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -m paper_2505_18698_amd.build` "
            "(the HIP library is required, there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    i64, i32, vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
    lib.monarch_attn_fwd.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_fwd.restype = ctypes.c_int
    lib.monarch_attn_fwd_varlen.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_fwd_varlen.restype = ctypes.c_int
    lib.monarch_attn_fwd_objective.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_fwd_objective.restype = ctypes.c_int
    lib.monarch_attn_exact_fwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, vp]
    lib.monarch_attn_exact_fwd.restype = ctypes.c_int
    lib.monarch_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_bwd.restype = ctypes.c_int
    lib.monarch_attn_bwd_varlen.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_bwd_varlen.restype = ctypes.c_int
    lib.monarch_attn_bwd_check.argtypes = [i64, i64, i64, i64, i32, i32]
    lib.monarch_attn_bwd_check.restype = ctypes.c_int
    lib.monarch_attn_bwd_workspace_bytes.argtypes = [i64, i64, i64, i64, i64, i64, i32, i32]
    lib.monarch_attn_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.monarch_attn_last_error.argtypes = []
    lib.monarch_attn_last_error.restype = ctypes.c_char_p
    lib.monarch_attn_check.argtypes = [i64, i64, i64, i64, i32, i32]
    lib.monarch_attn_check.restype = ctypes.c_int
    lib.monarch_attn_workspace_bytes.argtypes = [i64, i64, i64, i64, i64, i64, i32, i32]
    lib.monarch_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.monarch_attn_release_workspace.argtypes = []
    lib.monarch_attn_release_workspace.restype = ctypes.c_int
    lib.monarch_attn_set_path.argtypes = [i32]
    lib.monarch_attn_set_path.restype = ctypes.c_int
    lib.monarch_attn_timing_enable.argtypes = [i32]
    lib.monarch_attn_timing_enable.restype = ctypes.c_int
    lib.monarch_attn_timing_read.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32), i32]
    lib.monarch_attn_timing_read.restype = ctypes.c_int32
    lib.monarch_attn_fwd_prepad.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_fwd_prepad.restype = ctypes.c_int
    lib.monarch_attn_fwd_noalloc.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i32, i32, vp]
    lib.monarch_attn_fwd_noalloc.restype = ctypes.c_int
    for name, argtypes in (
        ("monarch_attn_exact_packed_fwd", [vp] * 7 + [i64] * 8 + [i32, i32, i32, vp]),
        ("monarch_attn_exact_packed_bwd", [vp] * 11 + [i64] * 8 + [i32, i32, i32, vp]),
        ("monarch_attn_exact_paged_fwd", [vp] * 8 + [i64] * 9 + [i32, i32, vp]),
        ("monarch_attn_paged_plan", [vp] * 10 + [i64] * 5 + [vp]),
        ("monarch_attn_paged_write", [vp] * 5 + [i64] * 7 + [i32, vp]),
    ):
        getattr(lib, name).argtypes = argtypes
        getattr(lib, name).restype = ctypes.c_int
    lib.monarch_attn_build_id.argtypes = []
    lib.monarch_attn_build_id.restype = ctypes.c_char_p
    _check_provenance(lib)
    return lib


def _source_hash() -> str:
    import importlib.util

    spec = importlib.util.spec_from_file_location("_ma_build_hash", os.path.join(_PKG, "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod.source_hash()


def _check_provenance(lib) -> None:
    """Refuse a library built from other sources than the ones beside it."""
    built = lib.monarch_attn_build_id().decode()
    here = _source_hash()
    if built != here:
        raise ImportError(
            f"{LIB_PATH} was built from sources {built}, but the sources here hash to {here}: "
            "rebuild it (`python -m paper_2505_18698_amd.build`)")


def monarch_attn_build_id() -> str:
    """The source hash compiled into the library."""
    return LIB.monarch_attn_build_id().decode()


LIB = _load()
MAX_T_16BIT = 4      # MONARCH_ATTN_MAX_T_16BIT
MAX_T_16BIT_BWD = 4  # MONARCH_ATTN_MAX_T_16BIT_BWD


def monarch_attn_last_error() -> str:
    return LIB.monarch_attn_last_error().decode()


def _check(rc: int) -> None:
    if rc != MA_OK:
        raise MonarchAttnError(rc, monarch_attn_last_error())


def monarch_attn_fwd_raw(q: int, k: int, v: int, out: int, B: int, H: int, N: int, d: int,
                         m: int, b: int, T: int, dtype: int, stream: int | None) -> int:
    """The C call with integer device addresses; returns the status code."""
    return LIB.monarch_attn_fwd(q, k, v, out, B, H, N, d, m, b, T, dtype, stream or None)


class _Torch:
    """What every call needs of torch, looked up once (the package itself
    imports without it).  A short call is bound by this module's own time as
    much as by the GPU's: one of 16 heads of 256 rows takes 7.1 us in all."""

    def __init__(self):
        import torch

        self.Tensor = torch.Tensor
        self.int32, self.int64, self.float32 = torch.int32, torch.int64, torch.float32
        self.codes = {torch.float32: MA_F32, torch.bfloat16: MA_BF16, torch.float16: MA_F16}
        self.device = torch.cuda.device
        self.current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.current_stream = raw or (lambda index: torch.cuda.current_stream(index).cuda_stream)


_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        _TORCH = _Torch()
    return _TORCH


def dtype_code(torch_dtype) -> int:
    codes = _torch().codes
    if torch_dtype not in codes:
        raise TypeError(f"unsupported dtype {torch_dtype}")
    return codes[torch_dtype]


def _check_tensors(q, *others):
    """q and the others (k, v, out, or k, v, dout, dq, dk, dv): contiguous
    [B, H, N, d] device tensors of one shape, dtype and device."""
    Tensor = _torch().Tensor
    ok = isinstance(q, Tensor) and q.is_cuda
    if ok:
        shape, dtype, device = q.shape, q.dtype, q.device
        ok = len(shape) == 4 and q.is_contiguous()
        for t in others:
            ok = ok and isinstance(t, Tensor) and t.device == device and t.dtype == dtype and t.shape == shape \
                and t.is_contiguous()
    if not ok:
        _refuse_tensors(q, others)


def _refuse_tensors(q, others):
    """Raise for the first tensor that _check_tensors does not accept."""
    names = ("q", "k", "v", "out") if len(others) == 3 else ("q", "k", "v", "dout", "dq", "dk", "dv")
    for name, t in zip(names, (q, *others)):
        if not isinstance(t, _torch().Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a device tensor")
        if t.dim() != 4 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous [B, H, N, d] tensor")
        if t.shape != q.shape or t.dtype != q.dtype or t.device != q.device:
            raise ValueError(f"{name} must match q in shape, dtype and device")


def _stream(q, stream):
    """The hipStream_t to launch on: `stream`, or torch's current stream of
    q's device (read through torch's raw-stream hook where it exists: a
    fraction of the cost of torch.cuda.current_stream)."""
    if stream is None:
        return _torch().current_stream(q.device.index)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _call(fn, q, *args):
    """fn(*args) with q's device current; raises on a failure status."""
    rt = _torch()
    index = q.device.index
    if rt.current_device() == index:
        rc = fn(*args)
    else:
        with rt.device(index):
            rc = fn(*args)
    if rc != MA_OK:
        raise MonarchAttnError(rc, monarch_attn_last_error())


def monarch_attn_fwd(q, k, v, out, m: int, b: int, T: int, stream=None):
    """O = MonarchAttention(q, k, v) into `out`; torch device tensors [B, H, N, d].

    `stream`: a torch.cuda.Stream, an integer hipStream_t, or None for torch's
    current stream.  Asynchronous on that stream.  Returns `out`.
    """
    _check_tensors(q, k, v, out)
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_fwd, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, N, d, m, b, T,
          dtype_code(q.dtype), _stream(q, stream) or None)
    return out


NOALLOC_SCRATCH_BYTES = 64 << 20  # MONARCH_ATTN_NOALLOC_SCRATCH_BYTES


def monarch_attn_fwd_noalloc(q, k, v, out, m: int, b: int, T: int, stream=None):
    """monarch_attn_fwd without any device allocation: the states go to the
    library's per-device scratch array (NOALLOC_SCRATCH_BYTES; larger calls
    raise MA_EUNSUPPORTED).  Calls that can overlap on one device race on that
    array.  Returns `out`."""
    _check_tensors(q, k, v, out)
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_fwd_noalloc, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, N, d, m,
          b, T, dtype_code(q.dtype), _stream(q, stream))
    return out


def _check_lens(q, lens):
    rt = _torch()
    if not isinstance(lens, rt.Tensor) or lens.device != q.device or lens.dtype != rt.int32 \
            or not lens.is_contiguous() or tuple(lens.shape) != (q.shape[0],):
        raise ValueError("lens must be a contiguous int32 tensor [B] on the device of q")


def monarch_attn_fwd_varlen(q, k, v, out, lens, m: int, b: int, T: int, stream=None):
    """monarch_attn_fwd over a batch of post-padded sequences: lens (int32 device
    tensor [B]) holds the real rows of each batch element; rows >= lens[beta]
    of q, k, v count as zero whatever they hold, and those of out are written
    as zero.  Returns `out`."""
    _check_tensors(q, k, v, out)
    _check_lens(q, lens)
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_fwd_varlen, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lens.data_ptr(),
          B, H, N, d, m, b, T, dtype_code(q.dtype), _stream(q, stream))
    return out


def monarch_attn_fwd_prepad(q, k, v, out, m: int, b: int, T: int, lens=None, stream=None):
    """monarch_attn_fwd over pre-padded sequences (the padding rows first).
    lens None: all N rows real, pre-padded to m*b.  lens (int32 device tensor
    [B]): batch element beta's real rows are its LAST lens[beta] rows; its
    other rows of q, k, v count as zero and are written as zero in `out`.
    Returns `out`."""
    _check_tensors(q, k, v, out)
    if lens is not None:
        _check_lens(q, lens)
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_fwd_prepad, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
          None if lens is None else lens.data_ptr(), B, H, N, d, m, b, T, dtype_code(q.dtype), _stream(q, stream))
    return out


def monarch_attn_fwd_objective(q, k, v, out, obj, m: int, b: int, T: int, stream=None):
    """monarch_attn_fwd, plus obj[B, H, T] (float32 device tensor): the variational
    objective f(M^(t); Q, K) after every step t.  Returns (out, obj)."""
    _check_tensors(q, k, v, out)
    rt = _torch()
    if not isinstance(obj, rt.Tensor) or obj.device != q.device or obj.dtype != rt.float32 \
            or not obj.is_contiguous() or tuple(obj.shape) != (q.shape[0], q.shape[1], T):
        raise ValueError("obj must be a contiguous float32 tensor [B, H, T] on the device of q")
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_fwd_objective, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
          obj.data_ptr(), B, H, N, d, m, b, T, dtype_code(q.dtype), _stream(q, stream))
    return out, obj


def monarch_attn_exact_fwd(q, k, v, out, lse=None, stream=None):
    """Exact softmax attention into `out`; with `lse` (float32 device tensor
    [B, H, N]) also every row's logsumexp.  Returns (out, lse)."""
    _check_tensors(q, k, v, out)
    B, H, N, d = q.shape
    rt = _torch()
    if lse is not None and (not isinstance(lse, rt.Tensor) or lse.device != q.device
                            or lse.dtype != rt.float32 or not lse.is_contiguous()
                            or tuple(lse.shape) != (B, H, N)):
        raise ValueError("lse must be a contiguous float32 tensor [B, H, N] on the device of q")
    _call(LIB.monarch_attn_exact_fwd, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
          None if lse is None else lse.data_ptr(), B, H, N, d, dtype_code(q.dtype), _stream(q, stream))
    return out, lse


def monarch_attn_bwd(q, k, v, dout, dq, dk, dv, m: int, b: int, T: int, stream=None):
    """dq, dk, dv = the gradient of <MonarchAttention(q, k, v), dout> into the
    given tensors (all [B, H, N, d], one dtype).  Asynchronous on `stream`
    (torch's current stream when None).  Returns (dq, dk, dv)."""
    _check_tensors(q, k, v, dout, dq, dk, dv)
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_bwd, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(), dq.data_ptr(),
          dk.data_ptr(), dv.data_ptr(), B, H, N, d, m, b, T, dtype_code(q.dtype), _stream(q, stream))
    return dq, dk, dv


def monarch_attn_bwd_varlen(q, k, v, dout, dq, dk, dv, lens, m: int, b: int, T: int, stream=None):
    """The gradient of monarch_attn_fwd_varlen (lens: int32 device tensor [B]);
    rows >= lens[beta] of dq, dk, dv are written as zero.  Returns (dq, dk, dv)."""
    _check_tensors(q, k, v, dout, dq, dk, dv)
    _check_lens(q, lens)
    B, H, N, d = q.shape
    _call(LIB.monarch_attn_bwd_varlen, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(), dq.data_ptr(),
          dk.data_ptr(), dv.data_ptr(), lens.data_ptr(), B, H, N, d, m, b, T, dtype_code(q.dtype),
          _stream(q, stream))
    return dq, dk, dv


def monarch_attn_bwd_check(N: int, d: int, m: int, b: int, T: int, dtype: int) -> int:
    return LIB.monarch_attn_bwd_check(N, d, m, b, T, dtype)


def monarch_attn_bwd_workspace_bytes(B, H, N, d, m, b, T, dtype) -> int:
    return int(LIB.monarch_attn_bwd_workspace_bytes(B, H, N, d, m, b, T, dtype))


def monarch_attention(q, k, v, m: int, b: int, T: int, stream=None):
    """Allocate `out` with torch and run monarch_attn_fwd."""
    import torch

    out = torch.empty_like(q)
    return monarch_attn_fwd(q, k, v, out, m, b, T, stream)


_AUTOGRAD_FN = None


def _autograd_function():
    """torch.autograd.Function whose forward is monarch_attn_fwd (or _varlen)
    and whose backward is monarch_attn_bwd (or _varlen), both on torch's
    current stream."""
    global _AUTOGRAD_FN
    if _AUTOGRAD_FN is None:
        import torch

        class MonarchAttentionFn(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, v, m, b, T, lens):
                q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
                ctx.save_for_backward(q, k, v, lens) if lens is not None else ctx.save_for_backward(q, k, v)
                ctx.shape = (m, b, T)
                out = torch.empty_like(q)
                if lens is None:
                    return monarch_attn_fwd(q, k, v, out, m, b, T)
                return monarch_attn_fwd_varlen(q, k, v, out, lens, m, b, T)

            @staticmethod
            def backward(ctx, dout):
                saved = ctx.saved_tensors
                q, k, v = saved[:3]
                m, b, T = ctx.shape
                dq, dk, dv = (torch.empty_like(q) for _ in range(3))
                if len(saved) == 3:
                    monarch_attn_bwd(q, k, v, dout.contiguous(), dq, dk, dv, m, b, T)
                else:
                    monarch_attn_bwd_varlen(q, k, v, dout.contiguous(), dq, dk, dv, saved[3], m, b, T)
                return dq, dk, dv, None, None, None, None

        _AUTOGRAD_FN = MonarchAttentionFn
    return _AUTOGRAD_FN


def monarch_attention_autograd(q, k, v, m: int, b: int, T: int, lens=None):
    """MonarchAttention as a differentiable torch op: the forward pass and, on
    backward, the gradient with respect to q, k and v.  With lens (int32
    device tensor [B]) the batch is padded per sequence, as in
    monarch_attn_fwd_varlen."""
    return _autograd_function().apply(q, k, v, m, b, T, lens)


# ---- exact attention over packed sequences and paged caches ----

PLAN_NO_PAGES, PLAN_TABLE_FULL, PLAN_BAD_LENGTH, PLAN_NO_SLOTS = 1, 2, 4, 8  # MA_PLAN_*: bits of the plan's status
PLAN_MAX_B = 8192  # MONARCH_ATTN_PLAN_MAX_B


_MAX_ROW = 1 << 20  # elements between two rows, at most (MA_EUNSUPPORTED beyond)


def _rows(t, dtype, device):
    """The row stride of t, [rows, heads, d] of that dtype on that device with
    the heads of a row adjacent, or -1 where it is nothing of the kind."""
    _, h, d = t.shape
    x, y, z = t.stride()
    if (z == 1 or d == 1) and (y == d or h == 1) and t.dtype == dtype and t.device == device:
        return x if t.shape[0] > 1 else h * d
    return -1


def _is(t, shape, dtype, device):
    """Whether t is a contiguous tensor of that shape, dtype and device."""
    return t.shape == shape and t.dtype == dtype and t.device == device and t.is_contiguous()


def _check_rows(name, t, like, like_name="q"):
    """Raise unless t is [rows, heads, d] on the device and of the dtype of `like`, the heads of a row adjacent."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dim() != 3 or _rows(t, t.dtype, t.device) < 0:
        raise ValueError(f"{name} must be a [rows, heads, d] tensor whose rows are contiguous")
    if t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name} must match {like_name} in dtype and device")


def _check_like(name, t, shape, like, dtype=None):
    """Raise unless t is a contiguous device tensor of `shape` on the device of `like` (and of its dtype, or `dtype`)."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    dtype = like.dtype if dtype is None else dtype
    if not _is(t, shape, dtype, like.device):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on the device of the others")


def _check_packed(q, k, v, cu_seqlens):
    """Sizes (B, total, Hq, Hkv, d) and row strides of packed q [total, Hq, d], k and v [total, Hkv, d]."""
    rt = _torch()
    try:
        # (one pass without names: a short call is bound by these checks as much as by the GPU)
        total, Hq, d = q.shape
        Hkv = k.shape[1]
        dtype, device = q.dtype, q.device
        ldq, ldk, ldv = _rows(q, dtype, device), _rows(k, dtype, device), _rows(v, dtype, device)
        if q.is_cuda and ldq >= 0 and ldk >= 0 and ldv >= 0 and k.shape == v.shape == (total, Hkv, d) \
                and cu_seqlens.dtype == rt.int32 and cu_seqlens.dim() == 1 and cu_seqlens.shape[0] > 0 \
                and cu_seqlens.device == device and cu_seqlens.is_contiguous():
            return (cu_seqlens.shape[0] - 1, total, Hq, Hkv, d), (ldq, ldk, ldv)
    except (AttributeError, ValueError, IndexError):  # no tensor, or not of three dimensions
        pass
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_rows(name, t, q)
    if k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError("k and v must be [total, Hkv, d] tensors with the rows and head dimension of q")
    if not isinstance(cu_seqlens, rt.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 1:
        raise ValueError("cu_seqlens must be an int32 tensor [B + 1]")
    _check_like("cu_seqlens", cu_seqlens, cu_seqlens.shape, q, rt.int32)
    raise ValueError("q, k and v must be device tensors")


def _check_each(like, *tensors):
    """Raise for the first of the (name, tensor, shape, dtype) that is no contiguous tensor of that kind on the device of `like`."""
    device = like.device
    for name, t, shape, dtype in tensors:
        try:
            if t.shape == shape and t.dtype == dtype and t.device == device and t.is_contiguous():
                continue
        except AttributeError:
            pass
        _check_like(name, t, shape, like, dtype)


def monarch_attn_exact_packed_fwd(q, k, v, out, cu_seqlens, causal: bool = True, lse=None, rest=None,
                                  clear: bool = False, stream=None):
    """Exact softmax attention over sequences that lie one after another:
    q [total, Hq, d], k and v [total, Hkv, d] (rows may be strided, as in parts
    of a joint projection), sequence i the rows cu_seqlens[i] to
    cu_seqlens[i + 1] (int32 device tensor [B + 1]).  Writes the rows of the
    sequences in out [total, Hq, d] and, with lse (float32 device tensor
    [Hq, total]), every row's logsumexp; with rest (like out, 16-bit types) also
    what rounding out leaves, for the gradient.  Rows of no sequence are left,
    or, with clear, zero in out.  Returns (out, lse)."""
    sizes, strides = _check_packed(q, k, v, cu_seqlens)
    _check_each(q, ("out", out, q.shape, q.dtype))
    if lse is not None:
        _check_each(q, ("lse", lse, (q.shape[1], q.shape[0]), _torch().float32))
    if rest is not None:
        _check_each(q, ("rest", rest, q.shape, q.dtype))
    _packed_fwd(q, k, v, out, cu_seqlens, causal, lse, rest, clear, stream, sizes + strides)
    return out, lse


def _packed_fwd(q, k, v, out, cu_seqlens, causal, lse, rest, clear, stream, dims):
    _call(LIB.monarch_attn_exact_packed_fwd, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
          None if lse is None else lse.data_ptr(), None if rest is None else rest.data_ptr(), cu_seqlens.data_ptr(),
          *dims, bool(causal), bool(clear), dtype_code(q.dtype), _stream(q, stream) or None)


def monarch_attn_exact_packed_bwd(q, k, v, out, lse, dout, dq, dk, dv, cu_seqlens, causal: bool = True, rest=None,
                                  clear: bool = False, stream=None):
    """The gradient of monarch_attn_exact_packed_fwd from its out, lse and rest
    (None: without) and dout = dL/dout, into dq [total, Hq, d], dk and dv [total, Hkv, d]
    (contiguous; rows of no sequence are left, or, with clear, zero).  Returns
    (dq, dk, dv)."""
    sizes, strides = _check_packed(q, k, v, cu_seqlens)
    rows, keys, dtype = q.shape, k.shape, q.dtype
    _check_each(q, ("out", out, rows, dtype), ("dout", dout, rows, dtype), ("dq", dq, rows, dtype), ("dk", dk, keys, dtype),
                ("dv", dv, keys, dtype), ("lse", lse, (rows[1], rows[0]), _torch().float32))
    if rest is not None:
        _check_each(q, ("rest", rest, rows, dtype))
    _packed_bwd(q, k, v, out, lse, dout, dq, dk, dv, cu_seqlens, causal, rest, clear, stream, sizes + strides)
    return dq, dk, dv


def _packed_bwd(q, k, v, out, lse, dout, dq, dk, dv, cu_seqlens, causal, rest, clear, stream, dims):
    _call(LIB.monarch_attn_exact_packed_bwd, q, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
          lse.data_ptr(), None if rest is None else rest.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(),
          dv.data_ptr(), cu_seqlens.data_ptr(), *dims, bool(causal), bool(clear), dtype_code(q.dtype),
          _stream(q, stream) or None)


_PACKED_FN = None


def _packed_function():
    """torch.autograd.Function of monarch_attn_exact_packed_fwd and _bwd."""
    global _PACKED_FN
    if _PACKED_FN is None:
        import torch

        def whole(t):  # contiguous and 16-byte aligned
            t = t.contiguous()
            return t if t.data_ptr() % 16 == 0 else t.clone()

        def rows(t):  # the kernels' layout: heads of a row adjacent, rows 16-byte aligned
            n = t.element_size()
            fits = t.dim() == 3 and t.stride(2) == 1 and t.stride(1) == t.shape[2] and t.stride(0) * n % 16 == 0 \
                and t.shape[1] * t.shape[2] <= t.stride(0) <= _MAX_ROW and t.data_ptr() % 16 == 0
            return t if fits else whole(t)

        class ExactAttentionPackedFn(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, v, cu_seqlens, causal):
                q, k, v = rows(q), rows(k), rows(v)
                sizes, strides = _check_packed(q, k, v, cu_seqlens)
                out = q.new_empty(q.shape)
                lse = q.new_empty((sizes[2], sizes[1]), dtype=torch.float32)
                # (the gradient reads no row of no sequence: rest stays as it is there)
                rest = q.new_empty(q.shape) if q.element_size() == 2 else None
                _packed_fwd(q, k, v, out, cu_seqlens, causal, lse, rest, True, None, sizes + strides)
                ctx.save_for_backward(q, k, v, out, lse, cu_seqlens, rest)
                ctx.call = causal, sizes + strides
                return out

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dout):
                # (what the forward pass checked or made itself is not checked again: small calls are bound by the host)
                q, k, v, out, lse, cu_seqlens, rest = ctx.saved_tensors
                dq, dk, dv = q.new_empty(q.shape), q.new_empty(k.shape), q.new_empty(k.shape)
                causal, dims = ctx.call
                _packed_bwd(q, k, v, out, lse, whole(dout), dq, dk, dv, cu_seqlens, causal, rest, True, None, dims)
                return dq, dk, dv, None, None

        _PACKED_FN = ExactAttentionPackedFn
    return _PACKED_FN


def exact_attention_packed(q, k, v, cu_seqlens, causal: bool = True):
    """Exact attention over packed sequences as a differentiable torch op (see
    monarch_attn_exact_packed_fwd; tensors in other layouts are copied).  Rows
    of no sequence get zero output and zero gradients.  Differentiable once.

    A backward pass can be captured into a HIP graph together with its forward
    pass, after one of the same size on the capture stream.  As with every torch
    op, no autograd graph of the same leaves from outside the capture may be alive then
    (drop its outputs, or capture with leaves of its own): torch would wait
    for the stream of that graph, which ends the capture and may end the process."""
    return _packed_function().apply(q, k, v, cu_seqlens, causal)


def _check_cache(k_pages, v_pages, heads, d, like, like_name):
    """Raise unless k_pages and v_pages are contiguous [pages, heads, page, d] of the dtype and on the device of
    `like` (heads None: any number); their shape."""
    try:
        shape = k_pages.shape
        if len(shape) == 4 and v_pages.shape == shape and shape[3] == d and (heads is None or shape[1] == heads) \
                and k_pages.dtype == v_pages.dtype == like.dtype and k_pages.device == v_pages.device == like.device \
                and k_pages.is_contiguous() and v_pages.is_contiguous():
            return shape
    except AttributeError:
        pass
    if not isinstance(k_pages, _torch().Tensor) or not k_pages.is_cuda:
        raise TypeError("k_pages must be a device tensor")
    if k_pages.dim() != 4 or not k_pages.is_contiguous():
        raise ValueError("k_pages must be a contiguous [pages, Hkv, page, d] tensor")
    if k_pages.shape[3] != d or heads is not None and k_pages.shape[1] != heads or k_pages.dtype != like.dtype \
            or k_pages.device != like.device:
        raise ValueError(f"k_pages must match {like_name} in heads, head dimension, dtype and device")
    _check_like("v_pages", v_pages, k_pages.shape, k_pages)
    return k_pages.shape


def monarch_attn_exact_paged_fwd(q, k_pages, v_pages, out, cu_seqlens, kv_lens, block_table, causal: bool = True,
                                 lse=None, stream=None):
    """Exact softmax attention of new tokens, q [total, Hq, d] packed by
    cu_seqlens (int32 [B + 1]), over the cached ones: token t of sequence i in
    row t % page of page block_table[i, t // page] (int32 [B, blocks]) of
    k_pages and v_pages [pages, Hkv, page, d].  kv_lens (int32 [B]): tokens in
    the cache, the new ones (its last) among them.  Writes out [total, Hq, d]
    and, if given, lse (float32 [Hq, total]).  Returns (out, lse)."""
    rt = _torch()
    try:
        ldq = _rows(q, q.dtype, q.device) if q.is_cuda else -1
    except (AttributeError, ValueError):
        ldq = -1
    if ldq < 0:
        _check_rows("q", q, q)
    total, Hq, d = q.shape
    pages, Hkv, page, _ = _check_cache(k_pages, v_pages, None, d, q, "q")
    if not isinstance(block_table, rt.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be an int32 tensor [B, blocks]")
    B, blocks = block_table.shape
    int32 = rt.int32
    _check_each(q, ("out", out, q.shape, q.dtype), ("block_table", block_table, (B, blocks), int32), ("kv_lens", kv_lens, (B,), int32),
                ("cu_seqlens", cu_seqlens, (B + 1,), int32))
    if lse is not None:
        _check_each(q, ("lse", lse, (Hq, total), rt.float32))
    _call(LIB.monarch_attn_exact_paged_fwd, q, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), out.data_ptr(),
          None if lse is None else lse.data_ptr(), cu_seqlens.data_ptr(), kv_lens.data_ptr(), block_table.data_ptr(),
          B, total, Hq, Hkv, d, ldq, pages, page, blocks, bool(causal), dtype_code(q.dtype), _stream(q, stream) or None)
    return out, lse


def monarch_attn_paged_plan(past, fresh, ring, free_in, block_table, cu_seqlens, kv_lens, slots, free_out, status,
                            page: int, stream=None):
    """The tables of a step on the GPU, from past[B] cached and fresh[B] new
    tokens of every request: pages from the ring of free ones (`ring`, and
    free_in = (first, count)) into block_table [B, blocks], row starts
    cu_seqlens [B + 1], kv_lens [B], the slot of every new token in slots
    (int64 [capacity], -1 behind the last), what stays free in free_out [2] and
    0 or PLAN_* bits in status [1].  All int32 device tensors but slots.

    With bits in status a request did not fit and was cut: attention over these tables is meaningless for it, and
    its kv_lens, which count tokens without a slot, are not the next step's past."""
    rt = _torch()
    int32 = rt.int32
    try:
        (B,), (F,), (capacity,), (_, blocks) = past.shape, ring.shape, slots.shape, block_table.shape
        ok = past.is_cuda
    except (AttributeError, ValueError):
        ok = False
    if not ok:
        for name, t in (("past", past), ("ring", ring), ("slots", slots), ("block_table", block_table)):
            if not isinstance(t, rt.Tensor) or not t.is_cuda:
                raise TypeError(f"{name} must be a device tensor")
            if t.dim() != (2 if name == "block_table" else 1):
                raise ValueError(f"{name} must have {2 if name == 'block_table' else 1} dimension(s)")
    _check_each(past, ("past", past, (B,), int32), ("fresh", fresh, (B,), int32), ("ring", ring, (F,), int32),
                ("free_in", free_in, (2,), int32), ("block_table", block_table, (B, blocks), int32),
                ("cu_seqlens", cu_seqlens, (B + 1,), int32), ("kv_lens", kv_lens, (B,), int32),
                ("slots", slots, (capacity,), rt.int64), ("free_out", free_out, (2,), int32), ("status", status, (1,), int32))
    _call(LIB.monarch_attn_paged_plan, past, past.data_ptr(), fresh.data_ptr(), ring.data_ptr(), free_in.data_ptr(),
          block_table.data_ptr(), cu_seqlens.data_ptr(), kv_lens.data_ptr(), slots.data_ptr(), free_out.data_ptr(),
          status.data_ptr(), B, F, blocks, page, capacity, _stream(past, stream) or None)
    return block_table, cu_seqlens, kv_lens, slots, free_out, status


def monarch_attn_paged_write(k, v, k_pages, v_pages, slots, stream=None):
    """Rows of k and v [rows, Hkv, d] (may be strided) into the slots (int64
    [rows], all different; -1: nowhere) of k_pages and v_pages
    [pages, Hkv, page, d].  Returns (k_pages, v_pages)."""
    try:
        ok = k.is_cuda and v.shape == k.shape
        ldk, ldv = _rows(k, k.dtype, k.device), _rows(v, k.dtype, k.device)
    except (AttributeError, ValueError):
        ok = False
    if not ok or ldk < 0 or ldv < 0:
        _check_rows("k", k, k, "k")
        _check_rows("v", v, k, "k")
        raise ValueError("v must match k in shape")
    rows, Hkv, d = k.shape
    pages, _, page, _ = _check_cache(k_pages, v_pages, Hkv, d, k, "k")
    _check_each(k, ("slots", slots, (rows,), _torch().int64))
    _call(LIB.monarch_attn_paged_write, k, k.data_ptr(), v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
          slots.data_ptr(), rows, Hkv, d, ldk, ldv, pages, page, dtype_code(k.dtype), _stream(k, stream) or None)
    return k_pages, v_pages


def monarch_attn_check(N: int, d: int, m: int, b: int, T: int, dtype: int) -> int:
    return LIB.monarch_attn_check(N, d, m, b, T, dtype)


def fused_applies(d: int, m: int, b: int, dtype: int) -> bool:
    """Whether the one-workgroup-per-head kernel covers this shape."""
    return dtype in (MA_BF16, MA_F16) and d <= 64 and m <= 16 and b <= 16


def grouped_applies(d: int, m: int, b: int, dtype: int) -> bool:
    """Whether the one-workgroup-per-(head, group of classes) kernel (PATH_GROUPED)
    covers this shape (without per-sequence lengths or the objective)."""
    return dtype in (MA_BF16, MA_F16) and d <= 64 and m <= 64 and b <= 32


def monarch_attn_workspace_bytes(B, H, N, d, m, b, T, dtype) -> int:
    return int(LIB.monarch_attn_workspace_bytes(B, H, N, d, m, b, T, dtype))


def monarch_attn_release_workspace() -> None:
    _check(LIB.monarch_attn_release_workspace())


def monarch_attn_set_path(path: int) -> int:
    """Select the execution path (PATH_AUTO, PATH_HALF_STEPS, PATH_FUSED); returns the previous one."""
    prev = LIB.monarch_attn_set_path(path)
    if prev < 0:
        raise MonarchAttnError(MA_EINVAL, monarch_attn_last_error())
    return prev


def monarch_attn_timing_enable(flag: bool) -> None:
    _check(LIB.monarch_attn_timing_enable(1 if flag else 0))


def monarch_attn_timing_read(cap: int = 256):
    """[(kind name, ms), ...] for the launches of the last timed call."""
    ms = (ctypes.c_float * cap)()
    kind = (ctypes.c_int32 * cap)()
    n = LIB.monarch_attn_timing_read(ms, kind, cap)
    if n < 0:
        raise MonarchAttnError(MA_EHIP, monarch_attn_last_error())
    return [(KIND_NAMES.get(kind[i], str(kind[i])), float(ms[i])) for i in range(min(n, cap))]
