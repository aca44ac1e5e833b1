"""HEAL compensated GEMM for MI355X: Python binding of ``libheal.so``.

Argument marshalling only: every step of the computation runs in the HIP
kernels behind the C ABI declared in ``include/heal.h``.  PyTorch supplies
device memory and the current stream; nothing here computes on the host.
If the library is not built (``python -m paper_2606_21023_amd.build``), every
call raises ``HealError``: there is no fallback path.

Functions (names follow the C ABI):
  heal_split_f32(x)                   -> (hi, lo) bf16 bit patterns, torch.uint16
  heal_gemm_f32(A, B, out=None)       -> C = A @ B, bf16x3 compensated, FP32
  heal_gemm_f32_strided_batched(A, B, alpha=1.0, trans_b=False, out=None)
  heal_gemm_f32_instance(instance, A, B, ...)  -- a forced kernel instance
  heal_split_f16(x)                   -> (hi, lo) binary16 bit patterns (HEAL-Full pair)
  heal_maxabs_f32(x)                  -> max|x| as a 1-element float32 CUDA tensor
  heal_f16_weight_exponent(maxabs)    -> int e (host)
  heal_pack_f16_weight(W, e)          -> packed FP16 weight (torch.uint16)
  heal_gemm_f16w(A, W16, N, e, products)  -> HEAL-Base (1) / HEAL-Full (2) GEMM, FP32
  heal_presplit_b(B, trans_b=False)   -> packed bf16 (hi, lo) operand
  heal_gemm_f32_presplit(A, Bp, N)    -> bitwise equal to heal_gemm_f32(A, B)
  heal_quantize_i16(x)                -> (codes int16, max|x| 1-element tensor)
  heal_scores_i16(Q, Kt, maxQ, maxK, alpha)  -> dual-FP16 scores of INT16 codes, FP32
  KVCache(...), KVCache.empty(...)    -> the arrays of a key/value cache (INT8 blocks)
  heal_kv_append(cache, k, v, table, lens, ...)  -> tokens enter the cache; rotated queries
  heal_kv_read(cache, tokens, table, lens, ...)  -> (k, v) rows of the cache as FP32
  heal_kv_select(cache, q, n_sel, table, lens, ...)  -> the blocks that each token should read
  heal_kv_attention(cache, q, table, lens, ...)  -> attention over the cache, FP32
  KVPool(refs, block), KVPool.empty(...)  -> who holds which blocks of a cache
  heal_kv_release(pool, table, lens)  -> sequences give blocks up
  heal_kv_fork(pool, table, lens, parents, children)  -> sequences that share their beginning
  heal_kv_reserve(pool, tokens, table, lens, cu)  -> blocks of their own for tokens to append
  heal_kv_compact(pool, table)        -> held blocks first; (src, dst, count) of the moves
  heal_kv_copy(cache, blocks, slots)  -> blocks and slots copied by lists
  heal_block_norm(h, x, post, gate, scale, pre, ...)  -> (h + scale gate N(x), its norm), FP32
  LoraBank(a, b, ranks, scales)       -> the adapters of a projection
  heal_lora_add(y, x, bank, ids, cu)  -> y + s B (A x), each token with its request's adapter
  lib()                               -> the raw ctypes library
  build_id(), check_build()           -> the library's source hash; refuse a stale binary
"""
import ctypes
import os

__all__ = ["HealError", "lib", "library_path", "build_id", "check_build", "heal_split_f32", "heal_gemm_f32",
           "heal_gemm_f32_strided_batched", "heal_gemm_f32_instance", "select_instance",
           "INSTANCE_AUTO", "INSTANCE_LARGE", "INSTANCE_MEDIUM", "INSTANCE_SKINNY", "STATUS",
           "heal_split_f16", "heal_packed_size", "heal_maxabs_f32", "heal_f16_weight_exponent",
           "heal_pack_f16_weight", "heal_gemm_f16w", "heal_presplit_b", "heal_gemm_f32_presplit",
           "heal_quantize_i16", "heal_scores_i16", "KVCache", "heal_kv_append", "heal_kv_read",
           "heal_kv_select", "heal_kv_attention", "KVPool", "heal_kv_release", "heal_kv_fork", "heal_kv_reserve",
           "heal_kv_compact", "heal_kv_copy", "heal_block_norm", "LoraBank", "heal_lora_add"]

_HERE = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_HERE, "libheal.so")

INSTANCE_AUTO, INSTANCE_LARGE, INSTANCE_MEDIUM, INSTANCE_SKINNY = 0, 1, 2, 3
STATUS = {0: "HEAL_OK", 1: "HEAL_ERR_INVALID_VALUE", 2: "HEAL_ERR_UNSUPPORTED_DEVICE",
          3: "HEAL_ERR_LAUNCH"}


class HealError(RuntimeError):
    """A libheal call failed, or the library is missing."""

    def __init__(self, msg, status=None):
        super().__init__(msg)
        self.status = status


_lib = None
_i64 = ctypes.c_int64
_vp = ctypes.c_void_p


def lib():
    """Load ``libheal.so`` (once) and declare its C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(library_path):
        raise HealError("libheal.so is not built (expected at %s); run "
                        "`python -m paper_2606_21023_amd.build`" % library_path)
    L = ctypes.CDLL(library_path)
    L.heal_status_string.argtypes = [ctypes.c_int]
    L.heal_status_string.restype = ctypes.c_char_p
    L.heal_version.argtypes = []
    L.heal_version.restype = ctypes.c_int
    L.heal_build_id.argtypes = []
    L.heal_build_id.restype = ctypes.c_char_p
    L.heal_split_f32.argtypes = [_vp, _vp, _vp, _i64, _vp]
    L.heal_split_f32.restype = ctypes.c_int
    L.heal_gemm_f32.argtypes = [_i64, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _i64, _vp]
    L.heal_gemm_f32.restype = ctypes.c_int
    L.heal_gemm_f32_strided_batched.argtypes = [_i64, _i64, _i64, ctypes.c_float,
                                                _vp, _i64, _i64, _vp, _i64, _i64, ctypes.c_int,
                                                _vp, _i64, _i64, _i64, _vp]
    L.heal_gemm_f32_strided_batched.restype = ctypes.c_int
    L.heal_gemm_f32_instance.argtypes = [ctypes.c_int] + L.heal_gemm_f32_strided_batched.argtypes
    L.heal_gemm_f32_instance.restype = ctypes.c_int
    L.heal_gemm_select_instance.argtypes = [_i64, _i64]
    L.heal_gemm_select_instance.restype = ctypes.c_int
    _c = ctypes.c_int
    L.heal_gemm_direct_tile.argtypes = [_c, _c, _i64, _i64, _i64, _i64]
    L.heal_gemm_direct_tile.restype = _c
    L.heal_split_f16.argtypes = [_vp, _vp, _vp, _i64, _vp]
    L.heal_split_f16.restype = _c
    L.heal_packed_size.argtypes = [_i64, _i64, _c]
    L.heal_packed_size.restype = _i64
    L.heal_maxabs_f32.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp]
    L.heal_maxabs_f32.restype = _c
    L.heal_f16_weight_exponent.argtypes = [ctypes.c_float, ctypes.POINTER(ctypes.c_int32)]
    L.heal_f16_weight_exponent.restype = _c
    L.heal_pack_f16_weight.argtypes = [_vp, _i64, _i64, _i64, ctypes.c_int32, _vp, _vp]
    L.heal_pack_f16_weight.restype = _c
    L.heal_gemm_f16w.argtypes = [_c, _i64, _i64, _i64, _vp, _i64, _vp, ctypes.c_int32, _vp, _i64,
                                 _vp]
    L.heal_gemm_f16w.restype = _c
    L.heal_gemm_f16w_instance.argtypes = [_c] + L.heal_gemm_f16w.argtypes
    L.heal_gemm_f16w_instance.restype = _c
    L.heal_presplit_b.argtypes = [_vp, _i64, _i64, _i64, _c, _vp, _vp]
    L.heal_presplit_b.restype = _c
    L.heal_gemm_f32_presplit.argtypes = [_i64, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _vp]
    L.heal_gemm_f32_presplit.restype = _c
    L.heal_gemm_f32_presplit_instance.argtypes = [_c] + L.heal_gemm_f32_presplit.argtypes
    L.heal_gemm_f32_presplit_instance.restype = _c
    L.heal_quantize_i16.argtypes = [_vp, _i64, _vp, _vp, _vp]
    L.heal_quantize_i16.restype = _c
    L.heal_scores_i16.argtypes = [_i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _vp,
                                  ctypes.c_float, _vp, _i64, _i64, _i64, _vp]
    L.heal_scores_i16.restype = _c
    L.heal_kv_append.argtypes = [_vp, _vp] + [_vp, _i64, _i64] * 2 + [_vp, _vp, _i64, _i64, _c] + [
        _vp, _i64, _i64, _i64, _vp, _i64, _i64, _vp]
    L.heal_kv_append.restype = _c
    L.heal_kv_read.argtypes = [_vp, _vp, _vp, _vp, _vp]
    L.heal_kv_read.restype = _c
    L.heal_kv_select.argtypes = [_vp, _vp, _vp] + [_i64] * 6 + [_vp, _vp]
    L.heal_kv_select.restype = _c
    L.heal_kv_attention.argtypes = [_vp, _vp, _vp, _i64, _i64, _i64, ctypes.c_float, _c, _i64, _vp, _i64,
                                    _vp, _i64, _i64, _vp, _i64, _vp, _i64, _vp]
    L.heal_kv_attention.restype = _c
    L.heal_kv_attention_workspace.argtypes = [_vp, _vp, _i64, _i64, _i64, _i64]
    L.heal_kv_attention_workspace.restype = _i64
    L.heal_kv_attention_tile.argtypes = L.heal_kv_attention_workspace.argtypes
    L.heal_kv_attention_tile.restype = _c
    L.heal_kv_release.argtypes = [_vp, _i64, _vp, _vp, _i64, _i64, _vp]
    L.heal_kv_release.restype = _c
    L.heal_kv_fork.argtypes = [_vp, _i64, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp]
    L.heal_kv_fork.restype = _c
    L.heal_kv_reserve.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp, _i64, _vp]
    L.heal_kv_reserve.restype = _c
    L.heal_kv_reserve_workspace.argtypes = [_vp, _vp]
    L.heal_kv_reserve_workspace.restype = _i64
    L.heal_kv_compact.argtypes = [_vp, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp]
    L.heal_kv_compact.restype = _c
    L.heal_kv_compact_workspace.argtypes = [_vp]
    L.heal_kv_compact_workspace.restype = _i64
    L.heal_kv_copy.argtypes = [_vp, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _vp]
    L.heal_kv_copy.restype = _c
    L.heal_block_norm.argtypes = [_i64] * 3 + [_vp, _i64, _i64] * 2 + [_vp, _vp, _i64, _i64, _i64, ctypes.c_float,
                                                                      _vp] + [_vp, _i64, _i64] * 2 + [_vp]
    L.heal_block_norm.restype = _c
    L.heal_lora_add.argtypes = [_vp, _i64, _i64, _vp, _vp] + [_vp, _i64] * 3 + [_vp, _i64, _vp]
    L.heal_lora_add.restype = _c
    L.heal_lora_workspace.argtypes = [_vp, _i64]
    L.heal_lora_workspace.restype = _i64
    _lib = L
    return L


def build_id():
    """The source hash the loaded ``libheal.so`` was built from."""
    return lib().heal_build_id().decode()


def check_build():
    """Raise ``HealError`` unless the loaded ``libheal.so`` was built from the
    sources beside it (a stale binary would test old code)."""
    from . import build as _build
    want, got = _build.source_hash(), build_id()
    if got != want:
        raise HealError("libheal.so was built from other sources (build id %s, sources %s); "
                        "rebuild with `python -m paper_2606_21023_amd.build`" % (got, want))
    return got


def _check(status, what):
    if status != 0:
        raise HealError("%s failed: %s" % (what, STATUS.get(status, status)), status)


class _Torch:
    """Stands for the module until a call needs it: the C library is built, and
    its host functions are called, without PyTorch."""

    def __getattr__(self, name):
        import importlib
        globals()["torch"] = module = importlib.import_module("torch")
        return getattr(module, name)


torch = _Torch()


def _stream():
    """The current device's current stream, as a raw pointer.  (The Stream object
    of torch.cuda.current_stream costs 3 us, a third of a small call; it stands in
    where torch lacks the raw accessors.)  The first call replaces itself."""
    global _stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    device = getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None:
        _stream = lambda: torch.cuda.current_stream().cuda_stream
    else:
        _stream = lambda: raw(device())
    return _stream()


def _tensor(t, name, dtype, ndim=None):
    """Check a CUDA tensor of a type and number of dimensions whose last one is
    contiguous; returns its shape and strides."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise HealError("%s must be a CUDA (HIP) tensor" % name)
    if t.dtype is not dtype:
        raise HealError("%s must be %s, got %s" % (name, str(dtype).replace("torch.", ""), t.dtype))
    shape, stride = t.shape, t.stride()
    if ndim is not None and len(shape) != ndim:
        raise HealError("%s must have %d dimensions, got %d" % (name, ndim, len(shape)))
    if stride[-1] != 1 and shape[-1] > 1 and t.numel():   # (0 dimensions: IndexError)
        # (a last dimension of one element has no stride to respect: torch
        # may report any, e.g. for the transpose of a one-row matrix)
        raise HealError("%s must be contiguous in its last dimension" % name)
    return shape, stride


def _ld(shape, stride):
    """Row stride of the last two dims, in elements."""
    return stride[-2] if shape[-2] > 1 else max(shape[-1], 1)


def _output(out, like, shape):
    """`out`, checked, or a new float32 tensor; and its strides."""
    if out is None:
        # (new_empty is 0.6 us faster, but follows a subclass)
        C = (like.new_empty(shape) if type(like) is torch.Tensor
             else torch.empty(shape, dtype=torch.float32, device=like.device))
        return C, C.stride()
    got, stride = _tensor(out, "out", torch.float32, len(shape))
    if tuple(got) != shape:
        raise HealError("out has shape %s, expected %s" % (tuple(got), shape))
    return out, stride


def heal_split_f32(x, hi=None, lo=None):
    """Split a contiguous float32 CUDA tensor into bf16 (hi, lo) bit patterns."""
    return _split("heal_split_f32", x, hi, lo)


def _split(what, x, hi, lo):
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype != torch.float32:
        raise HealError("x must be a float32 CUDA tensor")
    if not x.is_contiguous():
        raise HealError("x must be contiguous")
    if hi is None:
        hi = torch.empty(x.shape, dtype=torch.uint16, device=x.device)
    if lo is None:
        lo = torch.empty(x.shape, dtype=torch.uint16, device=x.device)
    _check(getattr(lib(), what)(x.data_ptr(), hi.data_ptr(), lo.data_ptr(), x.numel(), _stream()),
           what)
    return hi, lo


def heal_gemm_f32(A, B, out=None):
    """C = A @ B (A: M x K, B: K x N, row-major float32 CUDA tensors)."""
    shape_a, stride_a = _tensor(A, "A", torch.float32, 2)
    shape_b, stride_b = _tensor(B, "B", torch.float32, 2)
    M, K = shape_a
    N = shape_b[1]
    if shape_b[0] != K:
        raise HealError("inner dimensions differ: %s @ %s" % (tuple(A.shape), tuple(B.shape)))
    C, stride_c = _output(out, A, (M, N))
    _check((_lib or lib()).heal_gemm_f32(
        M, N, K, A.data_ptr(), B.data_ptr(), C.data_ptr(), _ld(shape_a, stride_a),
        _ld(shape_b, stride_b), _ld((M, N), stride_c), _stream()), "heal_gemm_f32")
    return C


def _batched(fn_args_prefix, A, B, alpha, trans_b, out, what):
    shape_a, stride_a = _tensor(A, "A", torch.float32, 3)
    shape_b, stride_b = _tensor(B, "B", torch.float32, 3)
    bat, M, K = shape_a
    N, Kb = (shape_b[1], shape_b[2]) if trans_b else (shape_b[2], shape_b[1])
    if Kb != K or shape_b[0] != bat:
        raise HealError("shapes do not match: A %s, B %s, trans_b=%s"
                        % (tuple(A.shape), tuple(B.shape), trans_b))
    C, stride_c = _output(out, A, (bat, M, N))
    many = bat > 1
    st = fn_args_prefix(M, N, K, ctypes.c_float(alpha), A.data_ptr(), _ld(shape_a, stride_a),
                        stride_a[0] if many else 0, B.data_ptr(), _ld(shape_b, stride_b),
                        stride_b[0] if many else 0, 1 if trans_b else 0, C.data_ptr(),
                        _ld((M, N), stride_c), stride_c[0] if many else 0, bat, _stream())
    _check(st, what)
    return C


def heal_gemm_f32_strided_batched(A, B, alpha=1.0, trans_b=False, out=None):
    """C[b] = alpha * A[b] @ op(B[b]) for 3-D tensors; op(B) = B^T if trans_b."""
    return _batched((_lib or lib()).heal_gemm_f32_strided_batched, A, B, alpha, trans_b, out,
                    "heal_gemm_f32_strided_batched")


def heal_gemm_f32_instance(instance, A, B, alpha=1.0, trans_b=False, out=None):
    """As heal_gemm_f32_strided_batched with a forced kernel instance (2-D or 3-D)."""
    squeeze = A.dim() == 2
    if squeeze:
        A, B = A.unsqueeze(0), B.unsqueeze(0)
        out = out.unsqueeze(0) if out is not None else None
    f = lib().heal_gemm_f32_instance
    C = _batched(lambda *a: f(int(instance), *a), A, B, alpha, trans_b, out,
                 "heal_gemm_f32_instance")
    return C[0] if squeeze else C


def select_instance(M, N):
    """The instance heal_gemm_f32 chooses for an M x N output by its size."""
    return lib().heal_gemm_select_instance(M, N)


# ---- FP16 forms, pre-split operand, INT16 scores ---------------------------

def heal_split_f16(x, hi=None, lo=None):
    """HEAL-Full pair of a contiguous float32 CUDA tensor, binary16 bit patterns."""
    return _split("heal_split_f16", x, hi, lo)


def heal_packed_size(K, N, planes):
    n = (_lib or lib()).heal_packed_size(K, N, planes)
    if n < 0:
        raise HealError("invalid packed size K=%d N=%d planes=%d" % (K, N, planes))
    return n


def heal_maxabs_f32(x, out=None):
    """max|x| of a 2-D (or contiguous) float32 CUDA tensor, as a 1-element tensor."""
    shape, stride = _tensor(x, "x", torch.float32)
    if len(shape) == 2:
        rows, cols, ld = shape[0], shape[1], _ld(shape, stride)
    else:
        if not x.is_contiguous():
            raise HealError("x must be 2-D or contiguous")
        rows, cols, ld = 1, x.numel(), max(x.numel(), 1)
    out = out if out is not None else torch.empty(1, dtype=torch.float32, device=x.device)
    _check(lib().heal_maxabs_f32(x.data_ptr(), rows, cols, ld, out.data_ptr(), _stream()),
           "heal_maxabs_f32")
    return out


def heal_f16_weight_exponent(maxabs):
    """Largest e with maxabs * 2^e <= 65504 (host)."""
    e = ctypes.c_int32()
    _check(lib().heal_f16_weight_exponent(ctypes.c_float(float(maxabs)), ctypes.byref(e)),
           "heal_f16_weight_exponent")
    return e.value


def heal_pack_f16_weight(W, e, out=None):
    """Packed RNE_f16(W * 2^e) of an N x K float32 weight (torch.uint16, 1-D)."""
    shape, stride = _tensor(W, "W", torch.float32, 2)
    N, K = shape
    size = heal_packed_size(K, N, 1)
    out = out if out is not None else torch.empty(size, dtype=torch.uint16, device=W.device)
    _check(lib().heal_pack_f16_weight(W.data_ptr(), N, K, _ld(shape, stride), int(e),
                                      out.data_ptr(), _stream()), "heal_pack_f16_weight")
    return out


def heal_gemm_f16w(A, W16, N, e, products, out=None, instance=INSTANCE_AUTO):
    """HEAL-Base (products=1) or HEAL-Full (products=2): A (M x K float32) times
    the packed FP16 weight of an N x K matrix, scaled back by 2^-e."""
    shape, stride = _tensor(A, "A", torch.float32, 2)
    M, K = shape
    C, stride_c = _output(out, A, (M, N))
    if W16.numel() < heal_packed_size(K, N, 1):
        raise HealError("W16 is smaller than the packed size")
    _check(_lib.heal_gemm_f16w_instance(int(instance), int(products), M, N, K, A.data_ptr(),
                                        _ld(shape, stride), W16.data_ptr(), int(e), C.data_ptr(),
                                        _ld((M, N), stride_c), _stream()), "heal_gemm_f16w")
    return C


def heal_presplit_b(B, trans_b=False, out=None):
    """Packed bf16 (hi, lo) of B (K x N, or N x K with trans_b)."""
    shape, stride = _tensor(B, "B", torch.float32, 2)
    K, N = (shape[1], shape[0]) if trans_b else (shape[0], shape[1])
    size = heal_packed_size(K, N, 2)
    out = out if out is not None else torch.empty(size, dtype=torch.uint16, device=B.device)
    _check(lib().heal_presplit_b(B.data_ptr(), K, N, _ld(shape, stride), 1 if trans_b else 0,
                                 out.data_ptr(), _stream()), "heal_presplit_b")
    return out


def heal_gemm_f32_presplit(A, Bp, N, out=None, instance=INSTANCE_AUTO):
    """C = A @ B from the pre-split packed B of an operand with N columns."""
    shape, stride = _tensor(A, "A", torch.float32, 2)
    M, K = shape
    C, stride_c = _output(out, A, (M, N))
    if Bp.numel() < heal_packed_size(K, N, 2):
        raise HealError("Bp is smaller than the packed size")
    _check(_lib.heal_gemm_f32_presplit_instance(int(instance), M, N, K, A.data_ptr(),
                                                _ld(shape, stride), Bp.data_ptr(), C.data_ptr(),
                                                _ld((M, N), stride_c), _stream()),
           "heal_gemm_f32_presplit")
    return C


def heal_quantize_i16(x, q=None, maxabs=None):
    """INT16 codes of a contiguous float32 CUDA tensor and its max|x| (device)."""
    _tensor(x, "x", torch.float32)
    if not x.is_contiguous():
        raise HealError("x must be contiguous")
    q = q if q is not None else torch.empty(x.shape, dtype=torch.int16, device=x.device)
    maxabs = maxabs if maxabs is not None else torch.empty(1, dtype=torch.float32, device=x.device)
    _check((_lib or lib()).heal_quantize_i16(x.data_ptr(), x.numel(), q.data_ptr(),
                                             maxabs.data_ptr(), _stream()), "heal_quantize_i16")
    return q, maxabs


def heal_scores_i16(Q, Kt, maxQ, maxK, alpha=1.0, out=None):
    """Scores of INT16 codes: Q (batch x M x d), Kt (batch x N x d) -> batch x M x N
    FP32 (2-D inputs give a 2-D result)."""
    squeeze = Q.dim() == 2
    if squeeze:
        Q, Kt = Q.unsqueeze(0), Kt.unsqueeze(0)
        out = out.unsqueeze(0) if out is not None else None
    shape_q, stride_q = _tensor(Q, "Q", torch.int16, 3)
    shape_k, stride_k = _tensor(Kt, "Kt", torch.int16, 3)
    bat, M, K = shape_q
    N = shape_k[1]
    if shape_k[0] != bat or shape_k[2] != K:
        raise HealError("shapes do not match: Q %s, Kt %s" % (tuple(Q.shape), tuple(Kt.shape)))
    S = out if out is not None else torch.empty((bat, M, N), dtype=torch.float32, device=Q.device)
    shape_s, stride_s = _tensor(S, "out", torch.float32, 3)
    many = bat > 1
    _check((_lib or lib()).heal_scores_i16(
        M, N, K, Q.data_ptr(), _ld(shape_q, stride_q), stride_q[0] if many else 0,
        maxQ.data_ptr(), Kt.data_ptr(), _ld(shape_k, stride_k), stride_k[0] if many else 0,
        maxK.data_ptr(), ctypes.c_float(alpha), S.data_ptr(), _ld(shape_s, stride_s), stride_s[0] if many else 0,
        bat, _stream()), "heal_scores_i16")
    return S[0] if squeeze else S


# ---- key/value cache ---------------------------------------------------------

class _CCache(ctypes.Structure):
    _fields_ = [(n, _i64) for n in ("blocks", "slots", "heads", "dim", "block")] + [
        (n, _vp) for n in ("k_codes", "v_codes", "scales", "k_mean", "k_recent", "v_recent")]


class _CBatch(ctypes.Structure):
    _fields_ = [("seqs", _i64), ("tokens", _i64), ("cu", _vp), ("lens", _vp), ("table", _vp),
                ("table_ld", _i64), ("table_cols", _i64), ("slots", _vp)]


class KVCache:
    """The arrays of a key/value cache (``include/heal.h`` has their layouts):

      k_codes  int8    (blocks, heads, block, dim)
      v_codes  int8    (blocks, heads, dim, block)
      scales   float32 (blocks, heads, 2)
      k_mean   float32 (blocks, heads, dim)
      k_recent float32 (slots, heads, 2 * block, dim)
      v_recent float32 (slots, heads, dim, 2 * block)

    dim is 64, 96 or 128, block 16, 32, 64 or 128 tokens.  The arrays are the
    caller's: contiguous CUDA tensors of one device, kept as attributes.  Their
    addresses are taken once, so the attributes cannot be set and a tensor must not get
    other memory (``set_``, ``resize_``, ``data``); other arrays are another KVCache.
    """

    def __init__(self, k_codes, v_codes, scales, k_mean, k_recent, v_recent):
        shape, _ = _tensor(k_codes, "k_codes", torch.int8, 4)
        blocks, heads, block, dim = shape
        _tensor(k_recent, "k_recent", torch.float32, 4)
        slots = k_recent.shape[0]
        arrays = {"k_codes": k_codes, "v_codes": v_codes, "scales": scales, "k_mean": k_mean,
                  "k_recent": k_recent, "v_recent": v_recent}
        shapes = {"k_codes": (blocks, heads, block, dim), "v_codes": (blocks, heads, dim, block),
                  "scales": (blocks, heads, 2), "k_mean": (blocks, heads, dim),
                  "k_recent": (slots, heads, 2 * block, dim), "v_recent": (slots, heads, dim, 2 * block)}
        for name, t in arrays.items():
            want = shapes[name]
            _tensor(t, name, torch.int8 if name.endswith("codes") else torch.float32, len(want))
            if tuple(t.shape) != want:
                raise HealError("%s has shape %s, expected %s" % (name, tuple(t.shape), want))
            if not t.is_contiguous() or t.data_ptr() % 16:
                raise HealError("%s must be contiguous and 16-byte aligned" % name)
            if t.device != k_codes.device:
                raise HealError("%s is on %s, k_codes on %s" % (name, t.device, k_codes.device))
        if dim not in (64, 96, 128) or block not in (16, 32, 64, 128) or not (blocks and slots and heads):
            raise HealError("no cache of %d blocks, %d slots, %d heads, dim %d, block %d"
                            % (blocks, slots, heads, dim, block))
        c = _CCache(blocks, slots, heads, dim, block, *(t.data_ptr() for t in arrays.values()))
        self.__dict__.update(arrays, blocks=blocks, slots=slots, heads=heads, dim=dim, block=block,
                             device=k_codes.device, _index=k_codes.get_device(), _f32=torch.float32,
                             _i32=torch.int32, _c=c, _ref=ctypes.byref(c))

    def __setattr__(self, name, value):
        raise HealError("a KVCache keeps the addresses of its arrays: make another one to change %s" % name)

    def __delattr__(self, name):
        raise HealError("a KVCache keeps the addresses of its arrays: %s stays" % name)

    @classmethod
    def empty(cls, blocks, slots, heads, dim, block=64, device="cuda"):
        """A cache of its own, not cleared (nothing of it is read before it is written)."""
        def f(*shape):
            return torch.empty(shape, dtype=torch.float32, device=device)

        def i(*shape):
            return torch.empty(shape, dtype=torch.int8, device=device)
        return cls(i(blocks, heads, block, dim), i(blocks, heads, dim, block), f(blocks, heads, 2),
                   f(blocks, heads, dim), f(slots, heads, 2 * block, dim), f(slots, heads, dim, 2 * block))


# The checks of a decode step's tensors cost as much of the host's time as its launches
# do, so what is right is recognised by its attributes first (0.3 us a tensor, 0.6 by the
# checks that tell what is wrong), and only the rest is asked what is wrong with it.

def _kv_on(cache, t, name):
    if t.get_device() != cache._index:
        raise HealError("%s is on %s, the cache on %s" % (name, t.device, cache.device))


def _kv_ints(cache, t, name, ndim, size=None):
    shape, stride = _tensor(t, name, torch.int32, ndim)
    _kv_on(cache, t, name)
    if size is not None and shape[0] != size:
        raise HealError("%s has %d entries, expected %d" % (name, shape[0], size))
    return shape, stride


def _kv_list(cache, t, name, size):
    """A dense int32 vector of that size on the cache's device; its address."""
    try:
        if (t.dtype is cache._i32 and t.get_device() == cache._index and t.shape == (size,)
                and (size <= 1 or t.stride(0) == 1)):
            return t.data_ptr()
    except AttributeError:
        pass
    _kv_ints(cache, t, name, 1, size)
    return t.data_ptr()


def _kv_rows(cache, t, name, tokens=None, heads=None):
    """A (tokens, heads, dim) float32 tensor; returns shape, token and head strides."""
    try:
        shape, stride = t.shape, t.stride()
        if (t.dtype is cache._f32 and t.get_device() == cache._index and len(shape) == 3
                and shape[2] == cache.dim and stride[2] == 1 and (tokens is None or shape[0] == tokens)
                and (heads is None or shape[1] == heads)):
            return shape, stride[0], stride[1]
    except AttributeError:
        pass
    shape, stride = _tensor(t, name, torch.float32, 3)
    _kv_on(cache, t, name)
    if shape[2] != cache.dim or (tokens is not None and shape[0] != tokens) or (
            heads is not None and shape[1] != heads):
        raise HealError("%s has shape %s, expected (%s, %s, %d)"
                        % (name, tuple(shape), "tokens" if tokens is None else tokens,
                           "heads" if heads is None else heads, cache.dim))
    return shape, stride[0], stride[1]


def _kv_batch(cache, tokens, table, lens, cu, slots):
    if not isinstance(cache, KVCache):
        raise HealError("cache must be a KVCache")
    if _device() != cache._index:
        raise HealError("the cache is on %s, the current device is another" % cache.device)
    try:
        shape, stride = table.shape, table.stride()
        if not (table.dtype is cache._i32 and table.get_device() == cache._index and len(shape) == 2
                and (stride[1] == 1 or shape[1] <= 1)):
            shape = None
    except AttributeError:
        shape = None
    if shape is None:
        shape, stride = _kv_ints(cache, table, "table", 2)
    seqs, cols = shape
    if cu is not None:
        cu = _kv_list(cache, cu, "cu", seqs + 1)
    elif tokens != seqs:
        raise HealError("%d tokens of %d sequences need cu" % (tokens, seqs))
    if slots is not None:
        slots = _kv_list(cache, slots, "slots", seqs)
    elif seqs > cache.slots:
        raise HealError("%d sequences, the cache has %d slots" % (seqs, cache.slots))
    return _CBatch(seqs, tokens, cu, _kv_list(cache, lens, "lens", seqs), table.data_ptr(),
                   stride[0] if seqs > 1 else cols or 1, cols, slots)


def _kv_new(cache, shape):
    """A new float32 tensor beside the cache."""
    like = cache.scales
    return (like.new_empty(shape) if type(like) is torch.Tensor
            else torch.empty(shape, dtype=torch.float32, device=cache.device))


def _device():
    """The current device's number.  (The first call replaces itself.)"""
    global _device
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _device()


def _kv_group(cache, heads_q):
    if heads_q < 1 or heads_q % cache.heads:
        raise HealError("%d query heads for %d key/value heads" % (heads_q, cache.heads))


def _kv_angles(cache, t, name, like):
    try:
        shape = t.shape
        if (t.dtype is cache._f32 and t.get_device() == cache._index and len(shape) == 2 and t.is_contiguous()
                and (like is None or shape == like)):
            return shape
    except AttributeError:
        pass
    _tensor(t, name, torch.float32, 2)
    _kv_on(cache, t, name)
    raise HealError("cos and sin must be contiguous and of one shape")


def heal_kv_append(cache, k, v, table, lens, cu=None, slots=None, cos=None, sin=None,
                   interleaved=False, q=None, q_out=None):
    """The tokens' keys (rotated by their places) and values enter the cache.

    k, v: (tokens, heads, dim) float32; table (sequences, columns), lens and slots
    (sequences), cu (sequences + 1): int32.  lens counts the new tokens.  cos, sin:
    (places, rot / 2) float32 or None.  With q (tokens, any heads, dim) the queries
    are rotated too, into q_out (which may be q) or a new tensor, and returned; rows of
    tokens of no sequence are not written.
    """
    if not isinstance(cache, KVCache):
        raise HealError("cache must be a KVCache")
    shape, k_token, k_head = _kv_rows(cache, k, "k", None, cache.heads)
    tokens = shape[0]
    _, v_token, v_head = _kv_rows(cache, v, "v", tokens, cache.heads)
    batch = _kv_batch(cache, tokens, table, lens, cu, slots)
    places = rot = 0
    if (cos is None) != (sin is None):
        raise HealError("cos and sin come together")
    if cos is not None:
        shape = _kv_angles(cache, cos, "cos", None)
        _kv_angles(cache, sin, "sin", shape)
        places, rot = shape[0], 2 * shape[1]
    heads_q = q_token = q_head = qo_token = qo_head = 0
    if q is not None:
        shape, q_token, q_head = _kv_rows(cache, q, "q", tokens)
        heads_q = shape[1]
        if q_out is None:
            q_out = _kv_new(cache, shape)
            qo_token, qo_head = heads_q * cache.dim, cache.dim
        else:
            _, qo_token, qo_head = _kv_rows(cache, q_out, "q_out", tokens, heads_q)
    elif q_out is not None:
        raise HealError("q_out without q")
    with_q = q is not None and q.numel() > 0
    _check((_lib or lib()).heal_kv_append(
        cache._ref, ctypes.byref(batch), k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head,
        cos.data_ptr() if rot else None, sin.data_ptr() if rot else None, places, rot,
        1 if interleaved else 0, q.data_ptr() if with_q else None, q_token, q_head, heads_q,
        q_out.data_ptr() if with_q else None, qo_token, qo_head, _stream()), "heal_kv_append")
    return q_out


def heal_kv_read(cache, tokens, table, lens, cu=None, slots=None):
    """(k, v), each (tokens, heads, dim) float32: what the cache holds of each
    sequence's last tokens (cu says how many).  Rows it does not hold are zeros;
    rows of no sequence are not written."""
    batch = _kv_batch(cache, tokens, table, lens, cu, slots)
    shape = (tokens, cache.heads, cache.dim)
    k, v = _kv_new(cache, shape), _kv_new(cache, shape)
    _check((_lib or lib()).heal_kv_read(cache._ref, ctypes.byref(batch), k.data_ptr(), v.data_ptr(),
                                        _stream()), "heal_kv_read")
    return k, v


def heal_kv_select(cache, q, n_sel, table, lens, cu=None, slots=None, keep_first=1, keep_last=1, out=None):
    """(tokens, heads, n_sel) int32: for each token and key/value head the first
    keep_first and last keep_last blocks and the others that score highest,
    ascending, -1 behind the last.  Rows of tokens of no sequence are not written.
    (slots is not needed; it is checked if given.)"""
    if not isinstance(cache, KVCache):
        raise HealError("cache must be a KVCache")
    shape, q_token, q_head = _kv_rows(cache, q, "q")
    tokens, heads_q = shape[0], shape[1]
    _kv_group(cache, heads_q)
    batch = _kv_batch(cache, tokens, table, lens, cu, slots)
    if n_sel < 1:
        raise HealError("n_sel must be positive, got %d" % n_sel)
    if out is None:
        out = torch.empty((tokens, cache.heads, n_sel), dtype=torch.int32, device=q.device)
    else:
        _kv_sel(cache, out, "out", tokens, n_sel)
    _check((_lib or lib()).heal_kv_select(cache._ref, ctypes.byref(batch), q.data_ptr(), q_token, q_head,
                                          heads_q, n_sel, keep_first, keep_last, out.data_ptr(), _stream()),
           "heal_kv_select")
    return out


def _kv_sel(cache, t, name, tokens, n_sel=None):
    shape, _ = _tensor(t, name, torch.int32, 3)
    _kv_on(cache, t, name)
    if shape[0] != tokens or shape[1] != cache.heads or shape[2] < 1 or (n_sel and shape[2] != n_sel):
        raise HealError("%s has shape %s, expected (%d, %d, %s)"
                        % (name, tuple(shape), tokens, cache.heads, n_sel or "n_sel"))
    if not t.is_contiguous():
        raise HealError("%s must be contiguous" % name)
    return shape[2]


def heal_kv_attention(cache, q, table, lens, cu=None, slots=None, scale=None, causal=True, window=0,
                      sel=None, out=None, lse=None, chunk=0):
    """Attention of q (tokens, heads_q, dim) float32 over the cache; returns out.

    scale: dim ** -0.5 by default; window: 0, or how many tokens back a token sees;
    sel: int32 (tokens, heads, n) of ``heal_kv_select``, or None for all blocks;
    lse: a contiguous float32 (tokens, heads_q) that is written too; chunk: 0, or
    tokens summed at a time (a multiple of 64), for bits that do not depend on the
    batch.  Rows of tokens of no sequence are not written, in out and in lse.
    """
    if not isinstance(cache, KVCache):
        raise HealError("cache must be a KVCache")
    shape, q_token, q_head = _kv_rows(cache, q, "q")
    tokens, heads_q = shape[0], shape[1]
    _kv_group(cache, heads_q)
    batch = _kv_batch(cache, tokens, table, lens, cu, slots)
    n_sel = _kv_sel(cache, sel, "sel", tokens) if sel is not None else 0
    if out is None:
        out = _kv_new(cache, shape)
        out_token, out_head = heads_q * cache.dim, cache.dim
    else:
        _, out_token, out_head = _kv_rows(cache, out, "out", tokens, heads_q)
    if lse is not None:
        _tensor(lse, "lse", torch.float32, 2)
        _kv_on(cache, lse, "lse")
        if lse.shape != (tokens, heads_q) or not lse.is_contiguous():
            raise HealError("lse must be a contiguous (%d, %d) tensor" % (tokens, heads_q))
    scale = cache.dim ** -0.5 if scale is None else float(scale)
    if tokens == 0:
        return out
    L, ref = _lib or lib(), ctypes.byref(batch)
    size = L.heal_kv_attention_workspace(cache._ref, ref, heads_q, window, n_sel, chunk)
    space = _kv_new(cache, size // 4) if size > 0 else None
    _check(L.heal_kv_attention(
        cache._ref, ref, q.data_ptr(), q_token, q_head, heads_q, scale, 1 if causal else 0,
        window, sel.data_ptr() if n_sel else None, n_sel, out.data_ptr(), out_token, out_head,
        lse.data_ptr() if lse is not None else None, chunk, space.data_ptr() if size > 0 else None,
        max(size, 0), _stream()), "heal_kv_attention")
    return out

# ---- pages of a cache ----------------------------------------------------------

class _CPool(ctypes.Structure):
    _fields_ = [("blocks", _i64), ("block", _i64), ("refs", _vp)]


class KVPool:
    """Who holds which block of a cache (or of one for each layer): refs, a contiguous
    int32 CUDA vector with the number of table entries that hold each block, 0 where
    it is free; block: tokens of a block.  Its address is taken once, as a KVCache takes
    those of its arrays."""

    def __init__(self, refs, block):
        (blocks,), _ = _tensor(refs, "refs", torch.int32, 1)
        if block not in (16, 32, 64, 128) or not 1 <= blocks <= 1 << 30:
            raise HealError("no pool of %d blocks of %s tokens" % (blocks, block))
        c = _CPool(blocks, block, refs.data_ptr())
        self.__dict__.update(refs=refs, blocks=blocks, block=block, device=refs.device, _index=refs.get_device(),
                             _i32=torch.int32, _c=c, _ref=ctypes.byref(c))

    def __setattr__(self, name, value):
        raise HealError("a KVPool keeps the address of its counts: make another one to change %s" % name)

    def __delattr__(self, name):
        raise HealError("a KVPool keeps the address of its counts: %s stays" % name)

    @classmethod
    def empty(cls, blocks, block=64, device="cuda"):
        """A pool of its own, all blocks free."""
        return cls(torch.zeros(blocks, dtype=torch.int32, device=device), block)


def _kv_pool(pool, table):
    """Checks pool and table; returns rows, row stride, columns."""
    if not isinstance(pool, KVPool):
        raise HealError("pool must be a KVPool")
    if _device() != pool._index:
        raise HealError("the pool is on %s, the current device is another" % pool.device)
    try:
        shape, stride = table.shape, table.stride()
        if not (table.dtype is pool._i32 and table.get_device() == pool._index and len(shape) == 2
                and (stride[1] == 1 or shape[1] <= 1)):
            shape = None
    except AttributeError:
        shape = None
    if shape is None:
        shape, stride = _kv_ints(pool, table, "table", 2)
    rows, cols = shape
    return rows, stride[0] if rows > 1 else cols or 1, cols


def _kv_ints_new(pool, n):
    like = pool.refs
    return like.new_empty(n) if type(like) is torch.Tensor else torch.empty(n, dtype=torch.int32, device=pool.device)


def _count(t, name):
    try:
        return len(t)
    except TypeError:
        raise HealError("%s must be an int32 CUDA vector" % name) from None


def _kv_scratch(pool, size):
    """size bytes of workspace beside the pool, or None."""
    return _kv_ints_new(pool, (size + 3) // 4) if size > 0 else None


def heal_kv_release(pool, table, lens):
    """Rows of table (rows, columns) int32 are cut back to lens (rows) int32 tokens: the
    entries behind give their blocks up and become -1 (0 frees a row)."""
    rows, ld, cols = _kv_pool(pool, table)
    _check((_lib or lib()).heal_kv_release(pool._ref, rows, _kv_list(pool, lens, "lens", rows), table.data_ptr(),
                                           ld, cols, _stream()), "heal_kv_release")


def heal_kv_fork(pool, table, lens, parents, children):
    """Rows children[j] of table become copies of rows parents[j], whose blocks (as many as
    lens says) are then held once more; what the children held is given up.  A pair
    whose child is a parent too, or the child of an earlier pair, is left out."""
    rows, ld, cols = _kv_pool(pool, table)
    at = _kv_list(pool, lens, "lens", rows)
    pairs = _count(parents, "parents")
    _check((_lib or lib()).heal_kv_fork(
        pool._ref, rows, at, table.data_ptr(), ld, cols, pairs, _kv_list(pool, parents, "parents", pairs),
        _kv_list(pool, children, "children", pairs), _stream()), "heal_kv_fork")


def heal_kv_reserve(pool, tokens, table, lens, cu=None, missing=None):
    """Before ``heal_kv_append`` of `tokens` tokens with the same table, lens and cu: every block
    that they touch becomes its sequence's own.  Returns missing, an int32 (1) on the device: the
    number of blocks that the pool lacked, in which case nothing is changed, or 0."""
    rows, ld, cols = _kv_pool(pool, table)
    if cu is not None:
        cu = _kv_list(pool, cu, "cu", rows + 1)
    elif tokens != rows:
        raise HealError("%d tokens of %d sequences need cu" % (tokens, rows))
    missing_at = None
    if missing is None:
        missing = _kv_ints_new(pool, 1)
        missing_at = missing.data_ptr()
    batch = _CBatch(rows, tokens, cu, _kv_list(pool, lens, "lens", rows), None, 1, 0, None)
    ref, L = ctypes.byref(batch), _lib or lib()
    size = L.heal_kv_reserve_workspace(pool._ref, ref)
    space = _kv_scratch(pool, size)
    _check(L.heal_kv_reserve(pool._ref, ref, table.data_ptr(), ld, cols, missing_at or _kv_list(pool, missing, "missing", 1),
                             space.data_ptr() if space is not None else None, max(size, 0), _stream()),
           "heal_kv_reserve")
    return missing


def heal_kv_compact(pool, table, src=None, dst=None, count=None):
    """The held blocks become the first ones of the pool; table (all of the program's
    rows) and refs follow.  Returns (src, dst, count) for ``heal_kv_copy``: int32 (blocks // 2),
    -1 behind the moves, and their number (1)."""
    rows, ld, cols = _kv_pool(pool, table)
    most = pool.blocks // 2

    def ints(t, name, n):
        if t is None:
            t = _kv_ints_new(pool, n)
            return t, t.data_ptr()
        return t, _kv_list(pool, t, name, n)
    src, at_src = ints(src, "src", most)
    dst, at_dst = ints(dst, "dst", most)
    count, at_count = ints(count, "count", 1)
    L = _lib or lib()
    size = L.heal_kv_compact_workspace(pool._ref)
    space = _kv_scratch(pool, size)
    _check(L.heal_kv_compact(pool._ref, rows, table.data_ptr(), ld, cols, at_src if most else None,
                             at_dst if most else None, at_count, space.data_ptr(), size, _stream()),
           "heal_kv_compact")
    return src, dst, count


def heal_kv_copy(cache, blocks=None, slots=None, count=None):
    """Copies blocks (codes, scales, means) and slots (FP32 rows) of a cache: blocks = (src,
    dst), slots = (src, dst), int32 vectors; count: None, or an int32 (1), how many of the
    pairs of blocks.  No destination twice, nor a source as destination."""
    if not isinstance(cache, KVCache):
        raise HealError("cache must be a KVCache")
    if _device() != cache._index:
        raise HealError("the cache is on %s, the current device is another" % cache.device)

    def pairs(lists, name):
        if lists is None:
            return 0, None, None
        if not isinstance(lists, (tuple, list)) or len(lists) != 2:
            raise HealError("%s must be a pair of int32 CUDA vectors" % name)
        src, dst = lists
        n = _count(src, name + "[0]")
        return n, _kv_list(cache, src, name + "[0]", n), _kv_list(cache, dst, name + "[1]", n)
    n_blocks, b_src, b_dst = pairs(blocks, "blocks")
    n_slots, s_src, s_dst = pairs(slots, "slots")
    if count is not None:
        if blocks is None:
            raise HealError("count without blocks")
        count = _kv_list(cache, count, "count", 1)
    _check((_lib or lib()).heal_kv_copy(cache._ref, n_blocks, b_src, b_dst, count, n_slots, s_src, s_dst, _stream()),
           "heal_kv_copy")


# ---- the residual stream, adapters ------------------------------------------------

class _CNorm(ctypes.Structure):
    _fields_ = [("weight", _vp), ("bias", _vp), ("eps", ctypes.c_float), ("centred", ctypes.c_int)]


class _CBank(ctypes.Structure):
    _fields_ = [("adapters", _i64), ("rank", _i64), ("K", _i64), ("N", _i64), ("type", ctypes.c_int), ("a", _vp),
                ("b", _vp), ("ranks", _vp), ("scales", _vp)]


def _norm_rows(t, name, shape, index):
    """A float32 tensor of that shape (2-D or 3-D); its address and two strides."""
    try:
        stride = t.stride()
        if (t.dtype is torch.float32 and t.shape == shape and t.get_device() == index and stride[-1] == 1):
            return t.data_ptr(), stride[0], stride[1] if len(shape) == 3 else 0
    except AttributeError:
        pass
    got, stride = _tensor(t, name, torch.float32, len(shape))
    if got != shape:
        raise HealError("%s has shape %s, expected %s" % (name, tuple(got), tuple(shape)))
    if t.get_device() != index:
        raise HealError("%s is on %s, h on another device" % (name, t.device))
    return t.data_ptr(), stride[0], stride[1] if len(shape) == 3 else 0


def _norm_vector(t, name, dim, index):
    if t is None:
        return None
    try:
        if t.dtype is torch.float32 and t.shape == (dim,) and t.get_device() == index and t.stride(0) == 1:
            return t.data_ptr()
    except AttributeError:
        pass
    (n,), _ = _tensor(t, name, torch.float32, 1)
    if n != dim or t.get_device() != index:
        raise HealError("%s must be a vector of %d beside h" % (name, dim))
    return t.data_ptr()


def _norm_spec(weight, bias, name, dim, index, eps, centred):
    if weight is None:
        if bias is not None:
            raise HealError("%s_bias without %s" % (name, name))
        return None
    return ctypes.byref(_CNorm(_norm_vector(weight, name, dim, index),
                               None if bias is None else _norm_vector(bias, name + "_bias", dim, index), eps,
                               1 if centred else 0))


def _like(t, shape):
    """A new float32 tensor beside t."""
    return t.new_empty(shape) if type(t) is torch.Tensor else torch.empty(shape, dtype=torch.float32, device=t.device)


def heal_block_norm(h, x=None, post=None, gate=None, scale=1.0, pre=None, eps=1e-6, centred=False, post_bias=None,
                    pre_bias=None, h_out=None, out=None):
    """(h', out): h' = h + scale * gate * N(x; post) and out = N(h'; pre), as
    ``include/heal.h`` writes them.

    h: float32 (tokens, dim) or (tokens, heads, dim); x the same, or None: then h' is h
    itself.  post, pre: weights (dim) of the norms, or None for no norm there (without
    pre, out is None).  gate: a float32 tensor of as many dimensions that broadcasts to h, its
    last dimension dense, or None.  centred: norms about the mean, with biases post_bias and pre_bias where they
    are given.  h_out (which may be h or x) and out (h or x likewise) are new tensors by default.
    """
    shape, stride = _tensor(h, "h", torch.float32)
    if len(shape) not in (2, 3) or shape[-1] < 1:
        raise HealError("h must be (tokens, dim) or (tokens, heads, dim), got %s" % (tuple(shape),))
    index, dim = h.get_device(), shape[-1]
    if _device() != index:
        raise HealError("h is on %s, the current device is another" % h.device)
    wide = len(shape) == 3
    if x is None and (post is not None or gate is not None or h_out is not None):
        raise HealError("post, gate and h_out need x")
    if x is None and pre is None:
        raise HealError("nothing to do: neither x nor pre")
    x_at = _norm_rows(x, "x", shape, index) if x is not None else (None, 0, 0)
    g = (None, 0, 0, 0)
    if gate is not None:
        got, gs = _tensor(gate, "gate", torch.float32, len(shape))
        if gate.get_device() != index or any(a != b and a != 1 for a, b in zip(got, shape)):
            raise HealError("gate %s does not broadcast to h %s" % (tuple(got), tuple(shape)))
        g = (gate.data_ptr(), gs[0] if got[0] > 1 else 0, gs[1] if wide and got[1] > 1 else 0, 1 if got[-1] > 1 else 0)
    spec_post = _norm_spec(post, post_bias, "post", dim, index, eps, centred)
    spec_pre = _norm_spec(pre, pre_bias, "pre", dim, index, eps, centred)
    ho_at = out_at = (None, 0, 0)
    if x is not None:
        if h_out is None:
            h_out = _like(h, shape)
            ho_at = (h_out.data_ptr(), *h_out.stride()[:2])
        else:
            ho_at = _norm_rows(h_out, "h_out", shape, index)
    if pre is not None:
        if out is None:
            out = _like(h, shape)
            out_at = (out.data_ptr(), *out.stride()[:2])
        else:
            out_at = _norm_rows(out, "out", shape, index)
    elif out is not None:
        raise HealError("out without pre")
    _check((_lib or lib()).heal_block_norm(
        shape[0], shape[1] if wide else 1, dim, h.data_ptr(), stride[0], stride[1] if wide else 0, *x_at, spec_post, *g,
        scale, spec_pre, *ho_at, *out_at, _stream()), "heal_block_norm")
    return (h if x is None else h_out), out


class LoraBank:
    """Low-rank adapters of one projection, for ``heal_lora_add``: a (adapters, rank, K)
    and b (adapters, N, rank), contiguous CUDA tensors of float32, bfloat16 or float16;
    ranks int32 (adapters) where some use fewer of the rows of a and columns of b; scales
    float32 (adapters), 1 by default.  Addresses are taken once, as in a KVCache."""

    def __init__(self, a, b, ranks=None, scales=None):
        types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        if not isinstance(a, torch.Tensor) or a.dtype not in types:
            raise HealError("a must be a float32, bfloat16 or float16 CUDA tensor")
        (many, rank, K), _ = _tensor(a, "a", a.dtype, 3)
        (many_b, N, rank_b), _ = _tensor(b, "b", a.dtype, 3)
        if many_b != many or rank_b != rank or not (many and rank and K and N):
            raise HealError("a %s and b %s are not (adapters, rank, K) and (adapters, N, rank)"
                            % (tuple(a.shape), tuple(b.shape)))
        for name, t, dtype in (("ranks", ranks, torch.int32), ("scales", scales, torch.float32)):
            if t is not None:
                (n,), _ = _tensor(t, name, dtype, 1)
                if n != many:
                    raise HealError("%s has %d entries for %d adapters" % (name, n, many))
        for name, t in (("a", a), ("b", b), ("ranks", ranks), ("scales", scales)):
            if t is None:
                continue
            if t.device != a.device:
                raise HealError("%s is on %s, a on %s" % (name, t.device, a.device))
            if not t.is_contiguous() or (name in "ab" and t.data_ptr() % 16):
                raise HealError("%s must be contiguous, a and b 16-byte aligned" % name)
        c = _CBank(many, rank, K, N, types[a.dtype], a.data_ptr(), b.data_ptr(),
                   ranks.data_ptr() if ranks is not None else None, scales.data_ptr() if scales is not None else None)
        self.__dict__.update(a=a, b=b, ranks=ranks, scales=scales, adapters=many, rank=rank, K=K, N=N, device=a.device,
                             _index=a.get_device(), _i32=torch.int32, _c=c, _ref=ctypes.byref(c))

    def __setattr__(self, name, value):
        raise HealError("a LoraBank keeps the addresses of its arrays: make another one to change %s" % name)

    def __delattr__(self, name):
        raise HealError("a LoraBank keeps the addresses of its arrays: %s stays" % name)


def _lora_rows(bank, t, name, cols):
    """A float32 (tokens, cols) tensor on the bank's device; its shape and row stride."""
    try:
        shape, stride = t.shape, t.stride()
        if (t.dtype is torch.float32 and t.get_device() == bank._index and len(shape) == 2 and shape[1] == cols
                and stride[1] == 1):
            return shape, stride[0] if shape[0] > 1 else cols
    except AttributeError:
        pass
    shape, stride = _tensor(t, name, torch.float32, 2)
    _kv_on(bank, t, name)
    if shape[1] != cols:
        raise HealError("%s has shape %s for adapters of %d by %d" % (name, tuple(shape), bank.K, bank.N))
    return shape, _ld(shape, stride)


def heal_lora_add(y, x, bank, ids, cu=None, out=None):
    """out = y + s B (A x) with the adapter of each token's sequence.

    y (tokens, N), x (tokens, K): float32; ids (sequences) int32, -1 for none (out is y
    there); cu (sequences + 1) int32, or None where every token is a sequence.  out may be
    y, a new tensor by default.  Rows of tokens of no sequence (before cu[0], behind
    cu[-1]) are not written: out keeps what it held, and in a new tensor they are
    undefined; with out=y they stay y's.
    """
    if not isinstance(bank, LoraBank):
        raise HealError("bank must be a LoraBank")
    if _device() != bank._index:
        raise HealError("the adapters are on %s, the current device is another" % bank.device)
    shape, x_ld = _lora_rows(bank, x, "x", bank.K)
    tokens = shape[0]
    y_shape, y_ld = _lora_rows(bank, y, "y", bank.N)
    if y_shape[0] != tokens:
        raise HealError("x %s and y %s for adapters of %d by %d" % (tuple(shape), tuple(y_shape), bank.K, bank.N))
    if out is None:
        out, o_ld = _like(y, y_shape), bank.N
    else:
        o_shape, o_ld = _lora_rows(bank, out, "out", bank.N)
        if o_shape[0] != tokens:
            raise HealError("out has shape %s, expected %s" % (tuple(o_shape), tuple(y_shape)))
    seqs = _count(ids, "ids")
    ids = _kv_list(bank, ids, "ids", seqs)
    if cu is not None:
        cu = _kv_list(bank, cu, "cu", seqs + 1)
    elif tokens != seqs:
        raise HealError("%d tokens of %d sequences need cu" % (tokens, seqs))
    if tokens == 0:
        return out
    L = _lib or lib()
    size = L.heal_lora_workspace(bank._ref, tokens)
    space = _like(y, (size + 3) // 4) if size > 0 else None
    _check(L.heal_lora_add(bank._ref, tokens, seqs, cu, ids, x.data_ptr(), x_ld, y.data_ptr(), y_ld, out.data_ptr(), o_ld,
                           space.data_ptr() if size > 0 else None, max(size, 0), _stream()), "heal_lora_add")
    return out
