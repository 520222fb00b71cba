"""ctypes binding of ``libcudallm_gemm.so``: one Python function per C entry
point, same names, argument marshalling only.

Device buffers are passed as integer addresses (``tensor.data_ptr()``) or as
torch tensors (their ``data_ptr()`` is taken); streams as integer handles
(``torch.cuda.current_stream().cuda_stream``).  Nothing here computes: if the
shared library is missing this module raises, it never falls back to the CPU.
"""
from __future__ import annotations

import ctypes
import os

F32, BF16, F16 = 0, 1, 2
VARIANT_AUTO = -1

OK = 0
ERR_INVALID_POINTER = -1
ERR_INVALID_DIM = -2
ERR_INVALID_LD = -3
ERR_INVALID_DTYPE = -4
ERR_INVALID_VARIANT = -5
ERR_UNSUPPORTED_SHAPE = -6
ERR_UNSUPPORTED_DEVICE = -7
ERR_CUDA = -8
ERR_DEVICE_TIMEOUT = -9
ERR_WORKSPACE = -10
ERR_MISALIGNED = -11
ERR_TOO_LARGE = -12
NOALLOC_SCRATCH_BYTES = 8 << 20

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcudallm_gemm.so")
_lib = None

_i64 = ctypes.c_int64
_vp = ctypes.c_void_p
_int = ctypes.c_int
_sz = ctypes.c_size_t

_f32 = ctypes.c_float


class CTensor(ctypes.Structure):
    """``cudallm_tensor`` of include/cudallm_layers.h."""
    _fields_ = [("data", _vp), ("out", _vp), ("n", _i64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class XattnShape(ctypes.Structure):
    """``cudallm_xattn_shape`` of include/cudallm_layers.h: sizes, strides and scale of a layer."""
    _fields_ = [(n, _i64) for n in ("batch", "q_rows", "kv_rows", "q_heads", "kv_heads", "head_dim")] + [
        (n, _i64 * 3) for n in ("q_stride", "k_stride", "v_stride", "o_stride")] + [
        ("dtype", ctypes.c_int32), ("scale", _f32)]

    @classmethod
    def of(cls, q, k, v, o, scale=None):
        """From tensors (batch, rows, heads, head_dim) of any strides with a contiguous last dimension;
        scale defaults to 1 / sqrt(head_dim)."""
        if not (q.shape == o.shape and k.shape == v.shape and q.dim() == k.dim() == 4
                and q.shape[0] == k.shape[0] and q.shape[3] == k.shape[3]):
            raise ValueError("q and o (batch, q_rows, q_heads, head_dim), k and v (batch, kv_rows, kv_heads, head_dim)")
        if not (q.dtype == k.dtype == v.dtype == o.dtype):
            raise TypeError("operands of one type are needed")
        code = {"torch.bfloat16": BF16, "torch.float16": F16}.get(str(q.dtype))
        if code is None:
            raise TypeError(f"bf16 or fp16 operands, not {q.dtype}")
        if any(t.shape[3] > 1 and t.stride(3) != 1 for t in (q, k, v, o)):
            raise ValueError("the last dimension must be contiguous")
        s = cls(batch=q.shape[0], q_rows=q.shape[1], kv_rows=k.shape[1], q_heads=q.shape[2], kv_heads=k.shape[2],
                head_dim=q.shape[3], dtype=code,
                scale=(q.shape[3] ** -0.5 if q.shape[3] else 1.0) if scale is None else scale)
        for field, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("o_stride", o)):
            setattr(s, field, (_i64 * 3)(*t.stride()[:3]))
        return s

    def layouts(self):
        """What tensors of q, k, v, o have to be, as the fields say: (strides, sizes, type, extent in elements) of each;
        then the number and type of kv_lens and of lse.  Worked out anew whenever a field has changed."""
        raw = bytes(self)
        kept = getattr(self, "_kept", None)
        if kept is None or kept[0] != raw:
            import torch
            dtype = {BF16: torch.bfloat16, F16: torch.float16}.get(self.dtype)
            out = []
            for rows, heads, st in ((self.q_rows, self.q_heads, self.q_stride), (self.kv_rows, self.kv_heads, self.k_stride),
                                    (self.kv_rows, self.kv_heads, self.v_stride), (self.q_rows, self.q_heads, self.o_stride)):
                size, strides = (self.batch, rows, heads, self.head_dim), (*st, 1)
                extent = 0 if 0 in size else 1 + sum((n - 1) * d for n, d in zip(size, strides))
                out.append((strides, torch.Size(size) if min(size) >= 0 else size, dtype, extent))
            out += [(self.batch, torch.int32), (self.batch * self.q_heads * self.q_rows, torch.float32)]
            kept = self._kept = (raw, out)
        return kept[1]


# name -> (restype, argtypes); mirrors include/cudallm_gemm.h, cudallm_tasks.h and cudallm_layers.h
SIGNATURES = {
    "cudallm_gemm_bf16": (_int, [_vp, _vp, _vp] + [_i64] * 6 + [_int, _vp]),
    "cudallm_gemm_f32": (_int, [_vp, _vp, _vp] + [_i64] * 6 + [_int, _vp]),
    "cudallm_gemm_tf32": (_int, [_vp, _vp, _vp] + [_i64] * 6 + [_vp]),
    "cudallm_mhsa_bf16": (_int, [_vp, _vp, _vp, _vp] + [_i64] * 7 + [_vp]),
    "cudallm_gemm_bf16_batched": (_int, [_vp, _vp, _vp] + [_i64] * 10 + [_int, _vp]),
    "cudallm_gemm_bf16_variant": (_int, [_int, _vp, _vp, _vp] + [_i64] * 10 + [_int, _vp]),
    "cudallm_gemm_bf16_host": (_int, [_vp, _vp, _vp] + [_i64] * 6 + [_int, _vp, _sz, _vp]),
    "cudallm_host_staging_bytes": (_sz, [_i64] * 6 + [_int]),
    "cudallm_gemm_bf16_splitk_noalloc": (_int, [_vp, _vp, _vp] + [_i64] * 6 + [_int, _int, _vp]),
    "cudallm_num_variants": (_int, []),
    "cudallm_dispatch_set": (_int, [_i64, _i64, _i64, _i64, _int, _int]),
    "cudallm_dispatch_get": (_int, [_i64, _i64, _i64, _i64, _int, ctypes.POINTER(ctypes.c_int)]),
    "cudallm_dispatch_set_class": (_int, [_i64, _i64, _i64, _i64, _int, _int, _int]),
    "cudallm_dispatch_get_class": (_int, [_i64, _i64, _i64, _i64, _int, _int, ctypes.POINTER(ctypes.c_int)]),
    "cudallm_dispatch_clear": (_int, []),
    "cudallm_dispatch_load_packaged": (_int, []),
    "cudallm_variant_code": (_int, [_int, _int, _int]),
    "cudallm_variant_name": (ctypes.c_char_p, [_int]),
    "cudallm_variant_supports": (_int, [_int] + [_i64] * 7 + [_int]),
    "cudallm_select_variant": (_int, [_i64] * 7 + [_int]),
    "cudallm_workspace_bytes": (_sz, [_i64] * 7 + [_int]),
    "cudallm_set_workspace": (_int, [_vp, _sz]),
    "cudallm_set_workspace_for_stream": (_int, [_vp, _vp, _sz]),
    "cudallm_reserve_workspace": (_int, [_sz]),
    "cudallm_shutdown": (_int, []),
    "cudallm_debug_set": (_int, [_int, ctypes.c_ulonglong]),
    "cudallm_device_status": (_int, [_vp, ctypes.POINTER(_int), ctypes.POINTER(_int)]),
    "cudallm_strerror": (ctypes.c_char_p, [_int]),
    "cudallm_version": (_int, []),
    "cudallm_transpose_f32": (_int, [_vp, _vp] + [_i64] * 4 + [_vp]),
    "cudallm_sum_f32": (_int, [_vp, _i64, _vp, _vp]),
    "cudallm_dot_f32": (_int, [_vp, _vp, _i64, _vp, _vp]),
    "cudallm_layernorm_f32": (_int, [_vp, _vp, _vp, _vp, _i64, _i64, ctypes.c_float, _vp]),
    "cudallm_layernorm_rows": (_int, [_vp] * 6 + [_i64] * 4 + [_int, _int, _f32, _vp]),
    "cudallm_layernorm_rows_bwd": (_int, [_vp] * 8 + [_i64] * 5 + [_int, _int, _vp, _sz, _vp]),
    "cudallm_layernorm_rows_bwd_scratch_bytes": (_sz, [_i64, _i64]),
    "cudallm_grad_norm": (_int, [ctypes.POINTER(CTensor), _i64, _vp, _vp, _sz, _vp]),
    "cudallm_grad_clip": (_int, [ctypes.POINTER(CTensor), _i64, _vp, _f32, _f32, _vp]),
    "cudallm_grad_clip_norm": (_int, [ctypes.POINTER(CTensor), _i64, _f32, _f32, _vp, _vp, _sz, _vp]),
    "cudallm_grad_norm_scratch_bytes": (_sz, [_i64]),
    "cudallm_xattn_fwd": (_int, [ctypes.POINTER(XattnShape)] + [_vp] * 7 + [_sz, _vp]),
    "cudallm_xattn_fwd_scratch_bytes": (_sz, [ctypes.POINTER(XattnShape)]),
    "cudallm_xattn_bwd": (_int, [ctypes.POINTER(XattnShape)] + [_vp] * 11 + [_sz, _vp]),
    "cudallm_xattn_bwd_scratch_bytes": (_sz, [ctypes.POINTER(XattnShape)]),
}


class CudallmError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status}: {strerror(status)}")


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2506_09092_b200.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _p(x):
    """Address of a device/host buffer: int, None, or anything with data_ptr()."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


_get_device = None


def _d(*xs):
    """Addresses of device buffers: ints, Nones, or CUDA tensors on the current device."""
    global _get_device
    if _get_device is None:
        import torch
        _get_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
    cur, out = -2, []
    for x in xs:
        if x is None or isinstance(x, int):
            out.append(x)
            continue
        dev = x.get_device()
        if dev != cur:
            if dev < 0:
                raise TypeError("a CUDA tensor is needed, not one in host memory")
            cur = _get_device()
            if dev != cur:
                raise ValueError(f"the tensor is on device {dev}, the current device is {cur}")
        out.append(x.data_ptr())
    return out


def _laid_out(operands, kv_lens, at_lens, lse, at_lse):
    """Refuses tensors that do not hold the attention operands as an XattnShape says.  `operands`: names, tensors
    and their entries of ``layouts``; addresses are taken as they are."""
    for name, t, at in operands:
        if t is not None and t.__class__ is not int and not (
                t.stride() == at[0] and t.shape == at[1] and t.dtype is at[2]):
            _check_layout(name, t, *at)
    for name, t, (n, dtype) in (("kv_lens", kv_lens, at_lens), ("lse", lse, at_lse)):
        if t is not None and t.__class__ is not int:
            if t.dtype is not dtype:
                raise TypeError(f"{name} has to be {dtype}, not {t.dtype}")
            if t.numel() < n or not t.is_contiguous():
                raise ValueError(f"{name}: {n} contiguous elements are needed")


def _check_layout(name, t, strides, size, dtype, extent):
    """Another type; a (batch, rows, heads, head_dim) tensor of other strides (those of sizes of one do not count);
    one of other sizes (a flat buffer, say) that ends before the operand does."""
    if isinstance(t, int) or dtype is None or extent == 0:         # (a type that the C call refuses; nothing there)
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} has to be {dtype}, as the shape says, not {t.dtype}")
    if t.shape == size:
        if any(n > 1 and a != b for n, a, b in zip(size, t.stride(), strides)):
            raise ValueError(f"{name} has strides {t.stride()}, the shape says {strides}")
    elif (1 + sum((n - 1) * d for n, d in zip(t.shape, t.stride())) if t.numel() else 0) < extent:
        raise ValueError(f"{name}: {tuple(t.shape)} ends before {tuple(size)} of strides {strides} does")


def _s(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _check(st: int, where: str, check: bool):
    if check and st != OK:
        raise CudallmError(st, where)
    return st


def gemm_bf16(A, B, C, M, N, K, lda, ldb, ldc, out_dtype, stream=None, check=True):
    st = lib().cudallm_gemm_bf16(_p(A), _p(B), _p(C), M, N, K, lda, ldb, ldc, out_dtype, _s(stream))
    return _check(st, "cudallm_gemm_bf16", check)


def gemm_f32(A, B, C, M, N, K, lda, ldb, ldc, variant=VARIANT_AUTO, stream=None, check=True):
    """fp32 operands and result (the paper's Task 2 as stated), computed on the
    bf16 tensor cores from three-piece splits of the operands."""
    st = lib().cudallm_gemm_f32(_p(A), _p(B), _p(C), M, N, K, lda, ldb, ldc, variant, _s(stream))
    return _check(st, "cudallm_gemm_f32", check)


def gemm_tf32(A, B, C, M, N, K, lda, ldb, ldc, stream=None, check=True):
    """fp32 operands and result with the tensor cores reading the operands as TF32."""
    st = lib().cudallm_gemm_tf32(_p(A), _p(B), _p(C), M, N, K, lda, ldb, ldc, _s(stream))
    return _check(st, "cudallm_gemm_tf32", check)


def mhsa_bf16(Q, K, V, O, N, d_model, h, ldq, ldk, ldv, ldo, stream=None, check=True):
    """Multi-head self-attention (Task 6): bf16 Q, K, V (N x d_model), fp32 O."""
    st = lib().cudallm_mhsa_bf16(_p(Q), _p(K), _p(V), _p(O), N, d_model, h, ldq, ldk, ldv, ldo, _s(stream))
    return _check(st, "cudallm_mhsa_bf16", check)


def transpose_f32(A, AT, rows, cols, lda, ldat, stream=None, check=True):
    """Task 8: AT (cols x rows, pitch ldat) = transpose of A (rows x cols, pitch lda), fp32."""
    st = lib().cudallm_transpose_f32(_p(A), _p(AT), rows, cols, lda, ldat, _s(stream))
    return _check(st, "cudallm_transpose_f32", check)


def sum_f32(x, n, result, stream=None, check=True):
    """Task 14: result[0] (device fp32) = sum of the n fp32 elements of x."""
    st = lib().cudallm_sum_f32(_p(x), n, _p(result), _s(stream))
    return _check(st, "cudallm_sum_f32", check)


def dot_f32(a, b, n, result, stream=None, check=True):
    """Task 15: result[0] (device fp32) = a . b over n fp32 elements."""
    st = lib().cudallm_dot_f32(_p(a), _p(b), n, _p(result), _s(stream))
    return _check(st, "cudallm_dot_f32", check)


def layernorm_f32(x, gamma, beta, y, batch, m, eps=1e-5, stream=None, check=True):
    """Task 4: LayerNorm of ``batch`` samples of ``m`` fp32 elements; gamma / beta may be None."""
    st = lib().cudallm_layernorm_f32(_p(x), _p(gamma), _p(beta), _p(y), batch, m, ctypes.c_float(eps), _s(stream))
    return _check(st, "cudallm_layernorm_f32", check)


def layernorm_rows(x, gamma, beta, y, mean, rstd, rows, n, ldx, ldy, dtype, param_dtype, eps=1e-5, stream=None,
                   check=True):
    """LayerNorm of every row of x (rows x n); gamma, beta, mean and rstd may be None."""
    st = lib().cudallm_layernorm_rows(*_d(x, gamma, beta, y, mean, rstd), rows, n, ldx, ldy, dtype,
                                      param_dtype, eps, _s(stream))
    return _check(st, "cudallm_layernorm_rows", check)


def layernorm_rows_bwd_scratch_bytes(rows, n) -> int:
    return int(lib().cudallm_layernorm_rows_bwd_scratch_bytes(rows, n))


def layernorm_rows_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, rows, n, lddy, ldx, lddx, dtype, param_dtype,
                       scratch, scratch_bytes, stream=None, check=True):
    """Gradient of ``layernorm_rows``; dx, dgamma and dbeta may each be None."""
    *ptrs, scr = _d(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, scratch)
    st = lib().cudallm_layernorm_rows_bwd(*ptrs, rows, n, lddy, ldx, lddx, dtype, param_dtype, scr, scratch_bytes,
                                          _s(stream))
    return _check(st, "cudallm_layernorm_rows_bwd", check)


class TensorTable:
    """The gradients of a model as the C calls take them: a host array of ``cudallm_tensor``.
    Built once for gradients that stay where they are; holds references to the tensors."""

    def __init__(self, tensors, outs=None):
        tensors = list(tensors)
        outs = tensors if outs is None else list(outs)
        if len(outs) != len(tensors):
            raise ValueError("as many outputs as tensors are needed")
        codes = {"torch.float32": F32, "torch.bfloat16": BF16, "torch.float16": F16}
        self.count = len(tensors)
        self.array = (CTensor * max(self.count, 1))()
        self._keep = (tensors, outs)
        spans, inputs = [], []
        for e, t, o in zip(self.array, tensors, outs):
            code = codes.get(str(t.dtype))
            if o is not t and (t.dtype != o.dtype or t.numel() != o.numel()):
                raise ValueError("an output has the size and type of its tensor")
            if code is None:
                raise TypeError(f"fp32, bf16 or fp16 gradients, not {t.dtype}")
            if not (t.is_contiguous() and (o is t or o.is_contiguous())):
                raise ValueError("contiguous tensors are needed")
            data, out = _d(t, o)
            n = t.numel()
            e.data, e.out, e.n, e.dtype = data, out, n, code
            if n:
                nbytes = n * t.element_size()
                spans.append((out, out + nbytes, data != out))
                inputs.append((data, data + nbytes, data != out))
        spans.sort()
        for (_, end, _a), (begin, _, _b) in zip(spans, spans[1:]):
            if begin < end:
                raise ValueError("two outputs overlap (a gradient that is scaled in place may be listed once)")
        # An output beside its tensor must not lie over any input, one in place not over the input of an
        # entry that is written elsewhere (inputs that are scaled in place are outputs, compared above).
        apart = [s for s in spans if s[2]]
        if apart and (_meet(apart, inputs) or _meet([s for s in spans if not s[2]], [s for s in inputs if s[2]])):
            raise ValueError("an output overlaps a gradient of the list")


def _meet(some, others):
    """Whether one of `some` address ranges (begin, end, ...) overlaps one of `others`."""
    if not some or not others:
        return False
    end = [0, 0]
    for begin, stop, kind in sorted([(s[0], s[1], 0) for s in some] + [(s[0], s[1], 1) for s in others]):
        if begin < end[1 - kind]:
            return True
        if stop > end[kind]:
            end[kind] = stop
    return False


def tensor_table(tensors, outs=None) -> TensorTable:
    """Table of contiguous CUDA tensors for the grad_* calls; ``outs`` where the scaled ones go
    (None: in place).  Outputs that overlap each other, or what another entry reads, are refused."""
    return TensorTable(tensors, outs)


def grad_norm_scratch_bytes(table) -> int:
    return int(lib().cudallm_grad_norm_scratch_bytes(table if isinstance(table, int) else table.count))


def grad_norm(table, norm, scratch, scratch_bytes, stream=None, check=True):
    """norm[0] (device fp32) = the norm of all tensors of the table together."""
    st = lib().cudallm_grad_norm(table.array, table.count, *_d(norm, scratch), scratch_bytes, _s(stream))
    return _check(st, "cudallm_grad_norm", check)


def grad_clip(table, norm, max_norm, eps=1e-6, stream=None, check=True):
    """Scale the table's tensors by min(1, max_norm / (norm[0] + eps))."""
    st = lib().cudallm_grad_clip(table.array, table.count, *_d(norm), max_norm, eps, _s(stream))
    return _check(st, "cudallm_grad_clip", check)


def grad_clip_norm(table, max_norm, eps, norm, scratch, scratch_bytes, stream=None, check=True):
    """``grad_norm`` and ``grad_clip`` together."""
    st = lib().cudallm_grad_clip_norm(table.array, table.count, max_norm, eps, *_d(norm, scratch), scratch_bytes,
                                      _s(stream))
    return _check(st, "cudallm_grad_clip_norm", check)


def xattn_fwd_scratch_bytes(shape) -> int:
    return int(lib().cudallm_xattn_fwd_scratch_bytes(shape))


def xattn_fwd(shape, q, k, v, kv_lens, o, lse, scratch, scratch_bytes, stream=None, check=True):
    """Cross attention: o = softmax(scale q k^T) v over the first kv_lens[b] states of each batch item
    (``shape``: an XattnShape); kv_lens, lse and scratch may be None.  Tensors must be laid out as the shape
    says, kv_lens int32 and lse contiguous fp32; addresses are not looked at."""
    if isinstance(shape, XattnShape):
        at_q, at_k, at_v, at_o, at_lens, at_lse = shape.layouts()
        _laid_out((("q", q, at_q), ("k", k, at_k), ("v", v, at_v), ("o", o, at_o)), kv_lens, at_lens, lse, at_lse)
    st = lib().cudallm_xattn_fwd(shape, *_d(q, k, v, kv_lens, o, lse, scratch), scratch_bytes, _s(stream))
    return _check(st, "cudallm_xattn_fwd", check)


def xattn_bwd_scratch_bytes(shape) -> int:
    return int(lib().cudallm_xattn_bwd_scratch_bytes(shape))


def xattn_bwd(shape, q, k, v, kv_lens, o, lse, d_o, dq, dk, dv, scratch, scratch_bytes, stream=None, check=True):
    """Gradients of ``xattn_fwd`` (d_o laid out like o, dq like q, dk like k, dv like v); dk and dv may
    both be None.  Tensors are checked as there: ``torch.empty_like(k)`` of a k that is a part of a larger tensor
    has other strides and is refused."""
    if isinstance(shape, XattnShape):
        at_q, at_k, at_v, at_o, at_lens, at_lse = shape.layouts()
        _laid_out((("q", q, at_q), ("k", k, at_k), ("v", v, at_v), ("o", o, at_o), ("d_o", d_o, at_o), ("dq", dq, at_q),
                   ("dk", dk, at_k), ("dv", dv, at_v)), kv_lens, at_lens, lse, at_lse)
    st = lib().cudallm_xattn_bwd(shape, *_d(q, k, v, kv_lens, o, lse, d_o, dq, dk, dv, scratch), scratch_bytes, _s(stream))
    return _check(st, "cudallm_xattn_bwd", check)


def gemm_bf16_batched(A, B, C, M, N, K, lda, ldb, ldc, strideA, strideB, strideC, batch,
                      out_dtype, stream=None, check=True):
    st = lib().cudallm_gemm_bf16_batched(_p(A), _p(B), _p(C), M, N, K, lda, ldb, ldc,
                                         strideA, strideB, strideC, batch, out_dtype, _s(stream))
    return _check(st, "cudallm_gemm_bf16_batched", check)


def gemm_bf16_variant(variant, A, B, C, M, N, K, lda, ldb, ldc, strideA, strideB, strideC, batch,
                      out_dtype, stream=None, check=True):
    st = lib().cudallm_gemm_bf16_variant(variant, _p(A), _p(B), _p(C), M, N, K, lda, ldb, ldc,
                                         strideA, strideB, strideC, batch, out_dtype, _s(stream))
    return _check(st, "cudallm_gemm_bf16_variant", check)


def gemm_bf16_host(A_host, B_host, C_host, M, N, K, lda, ldb, ldc, out_dtype, dev_buf, dev_bytes,
                   stream=None, check=True):
    st = lib().cudallm_gemm_bf16_host(_p(A_host), _p(B_host), _p(C_host), M, N, K, lda, ldb, ldc,
                                      out_dtype, _p(dev_buf), dev_bytes, _s(stream))
    return _check(st, "cudallm_gemm_bf16_host", check)


def gemm_bf16_splitk_noalloc(A, B, C, M, N, K, lda, ldb, ldc, out_dtype, split_k, stream=None,
                             check=True):
    """Split-K product whose scratch is an array built into the library: for
    callers that may not allocate device memory (see the header).  Synchronises
    ``stream``; the first call per device should come before any stream capture;
    calls that overlap on the GPU race on the shared scratch."""
    st = lib().cudallm_gemm_bf16_splitk_noalloc(_p(A), _p(B), _p(C), M, N, K, lda, ldb, ldc,
                                                out_dtype, split_k, _s(stream))
    return _check(st, "cudallm_gemm_bf16_splitk_noalloc", check)


def host_staging_bytes(M, N, K, lda, ldb, ldc, out_dtype) -> int:
    return int(lib().cudallm_host_staging_bytes(M, N, K, lda, ldb, ldc, out_dtype))


def dispatch_set(M, N, K, batch, out_dtype, variant, check=True) -> int:
    """Record ``variant`` as the kernel for products of this shape (-1 removes the entry):
    the library's automatic choice uses it before its cost model."""
    return _check(lib().cudallm_dispatch_set(M, N, K, batch, out_dtype, variant), "cudallm_dispatch_set", check)


def dispatch_get(M, N, K, batch, out_dtype) -> int:
    """The recorded variant for the shape, or -1."""
    v = ctypes.c_int(-1)
    _check(lib().cudallm_dispatch_get(M, N, K, batch, out_dtype, ctypes.byref(v)), "cudallm_dispatch_get", True)
    return int(v.value)


def dispatch_set_class(M, N, K, batch, out_dtype, tma_addressable, variant, check=True) -> int:
    """Record ``variant`` for the whole class of shapes that are tiled like this one."""
    return _check(lib().cudallm_dispatch_set_class(M, N, K, batch, out_dtype, int(bool(tma_addressable)), variant),
                  "cudallm_dispatch_set_class", check)


def dispatch_get_class(M, N, K, batch, out_dtype, tma_addressable) -> int:
    v = ctypes.c_int(-1)
    _check(lib().cudallm_dispatch_get_class(M, N, K, batch, out_dtype, int(bool(tma_addressable)), ctypes.byref(v)),
           "cudallm_dispatch_get_class", True)
    return int(v.value)


def dispatch_load_packaged() -> int:
    """Enter the packaged search results into the class table; returns how many."""
    return int(lib().cudallm_dispatch_load_packaged())


def variant_code(variant: int, group_rows: int = 0, tail_parts: int = 0, check=True) -> int:
    """Variant id plus the two knobs the search varies -> the code the entry points take."""
    code = int(lib().cudallm_variant_code(variant, group_rows, tail_parts))
    if check and code < 0:
        raise CudallmError(code, "cudallm_variant_code")
    return code


def describe_code(code: int) -> str:
    """Human-readable form of a variant code: name, and the knobs that are set."""
    name = variant_name(code)
    g, t = (code >> 8) & 0xF, (code >> 12) & 0x7
    return name + (f"+g{1 << (g - 1)}" if g else "") + (f"+t{t}" if t else "")


def dispatch_clear() -> int:
    """Empty the dispatch table; returns how many entries it held."""
    return int(lib().cudallm_dispatch_clear())


def num_variants() -> int:
    return int(lib().cudallm_num_variants())


def variant_name(variant: int):
    s = lib().cudallm_variant_name(variant)
    return None if s is None else s.decode()


def variant_supports(variant, M, N, K, lda, ldb, ldc, batch, out_dtype) -> int:
    return int(lib().cudallm_variant_supports(variant, M, N, K, lda, ldb, ldc, batch, out_dtype))


def select_variant(M, N, K, lda, ldb, ldc, batch, out_dtype) -> int:
    return int(lib().cudallm_select_variant(M, N, K, lda, ldb, ldc, batch, out_dtype))


def workspace_bytes(M, N, K, lda, ldb, ldc, batch, out_dtype) -> int:
    return int(lib().cudallm_workspace_bytes(M, N, K, lda, ldb, ldc, batch, out_dtype))


def set_workspace(dev_ptr, nbytes: int, check=True):
    return _check(lib().cudallm_set_workspace(_p(dev_ptr), nbytes), "cudallm_set_workspace", check)


def set_workspace_for_stream(stream, dev_ptr, nbytes: int, check=True):
    """Attach a caller-owned workspace to ``stream`` (``dev_ptr=None`` removes it)."""
    return _check(lib().cudallm_set_workspace_for_stream(_s(stream), _p(dev_ptr), nbytes),
                  "cudallm_set_workspace_for_stream", check)


def reserve_workspace(nbytes: int, check=True):
    """Size the library's own workspace of the current device now."""
    return _check(lib().cudallm_reserve_workspace(nbytes), "cudallm_reserve_workspace", check)


def shutdown(check=True):
    """Release the library's workspaces, streams and events on every device."""
    return _check(lib().cudallm_shutdown(), "cudallm_shutdown", check)


DEBUG_WAIT_LIMIT_NS, DEBUG_MISS_NEXT_SPLIT_FLAGS, DEBUG_LAYERNORM_PATH, DEBUG_SKIP_NEXT_XATTN_LOADS = 1, 2, 3, 4


def debug_set(what: int, value: int, check=True):
    """Test hooks of the kernels' bounded waits (see the header)."""
    return _check(lib().cudallm_debug_set(what, value), "cudallm_debug_set", check)


def device_status(stream=None):
    """(code, detail) after synchronising ``stream``."""
    code, detail = _int(0), _int(0)
    lib().cudallm_device_status(_s(stream), ctypes.byref(code), ctypes.byref(detail))
    return code.value, detail.value


def strerror(status: int) -> str:
    return lib().cudallm_strerror(status).decode()


def version() -> int:
    return int(lib().cudallm_version())
