"""Python binding of libisoquant.so (declared in include/isoquant.h).

Argument marshalling only: every step of the quantize/dequantize path runs in
the library's HIP kernels.  PyTorch provides device memory and streams; tensors
are passed as raw device pointers together with the current HIP stream.  The
functions carry the C names; device outputs are allocated here when the caller
does not pass them.  A missing library is an ImportError, never a fallback.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libisoquant.so")

ISOQ_FULL, ISOQ_FAST, ISOQ_PLANAR2D, ISOQ_BLOCK8 = 0, 1, 2, 3
ISOQ_F32, ISOQ_F16 = 0, 1
ISOQ_ROPE_PAIRS, ISOQ_ROPE_HALVES = 0, 1
LAYOUTS = {"pairs": ISOQ_ROPE_PAIRS, "halves": ISOQ_ROPE_HALVES}
VARIANTS = {"full": ISOQ_FULL, "fast": ISOQ_FAST, "2d": ISOQ_PLANAR2D, "8d": ISOQ_BLOCK8}

STATUS = {0: "ISOQ_OK", 1: "ISOQ_E_INVALID", 2: "ISOQ_E_UNSUPPORTED", 3: "ISOQ_E_NULL",
          4: "ISOQ_E_ALIGN", 5: "ISOQ_E_HIP", 6: "ISOQ_E_NOMEM", 7: "ISOQ_E_DEVICE"}


class IsoqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = lib.isoq_last_hip_error().decode() if status in (5, 6) else ""
        super().__init__(f"{where}: {STATUS.get(status, status)} ({isoq_status_string(status)})"
                         + (f" [{detail}]" if detail else ""))


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python paper_2603_28430_amd/build.py`")
    # PyTorch ships its own HIP runtime (same soname).  Loading torch first
    # makes the library bind to that runtime instead of a second copy, which
    # would not see the GPU that torch has already opened.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(LIB_PATH)
    vp, dp, fp, i64 = ctypes.c_void_p, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_float), ctypes.c_int64
    c_int = ctypes.c_int
    L.isoq_params_init.argtypes = [ctypes.POINTER(vp), c_int, c_int, c_int, c_int, dp, dp, ctypes.c_uint64]
    L.isoq_params_destroy.argtypes = [vp]
    L.isoq_params_export.argtypes = [vp, fp, fp, fp]
    L.isoq_params_info.argtypes = [vp] + [ctypes.POINTER(c_int)] * 4
    L.isoq_quantize.argtypes = [vp, c_int, vp, i64, i64, vp, vp, vp]
    L.isoq_dequantize.argtypes = [vp, c_int, vp, vp, i64, i64, vp, vp]
    L.isoq_roundtrip.argtypes = [vp, c_int, vp, i64, i64, vp, vp]
    L.isoq_kv_append.argtypes = [vp, vp, c_int, vp, vp, vp, i64, c_int, vp, vp, vp, vp, i64, c_int, vp]
    L.isoq_sketch_init.argtypes = [ctypes.POINTER(vp), vp, c_int, dp, ctypes.c_uint64]
    L.isoq_sketch_destroy.argtypes = [vp]
    L.isoq_sketch_export.argtypes = [vp, ctypes.POINTER(c_int), fp]
    L.isoq_quantize_qjl.argtypes = [vp, vp, c_int, vp, i64, i64, vp, vp, vp, vp, vp]
    L.isoq_kv_append_qjl.argtypes = [vp, vp, c_int, vp, vp, i64, c_int, vp, vp, vp, vp, i64, c_int, vp]
    L.isoq_kv_scores_qjl.argtypes = [vp, vp, c_int, vp, c_int, c_int, c_int, vp, vp, vp, vp, i64, c_int, vp, c_int,
                                     vp, ctypes.c_float, vp, i64, vp]
    L.isoq_kv_scores_filled.argtypes = L.isoq_kv_scores_qjl.argtypes
    L.isoq_kv_scores.argtypes = [vp, c_int, vp, c_int, c_int, c_int, vp, vp, i64, c_int, vp, c_int, vp,
                                 ctypes.c_float, vp, i64, vp]
    L.isoq_kv_attn.argtypes = [vp, vp, c_int, vp, vp, i64, c_int, c_int, c_int, c_int, vp, vp, vp, vp, i64, c_int, vp,
                               c_int, vp, i64, ctypes.c_float, vp, vp, vp, ctypes.c_size_t, vp]
    L.isoq_kv_attn_workspace.argtypes = [vp, vp, c_int, i64, c_int, c_int, c_int, c_int, c_int, c_int, i64]
    L.isoq_kv_attn_workspace.restype = ctypes.c_size_t
    L.isoq_kv_attn_cross.argtypes = L.isoq_kv_attn.argtypes
    L.isoq_kv_attn_prefix.argtypes = L.isoq_kv_attn.argtypes[:20] + [vp, c_int, vp, i64, vp, c_int, i64] + L.isoq_kv_attn.argtypes[20:]
    L.isoq_kv_attn_prefix_workspace.argtypes = L.isoq_kv_attn_workspace.argtypes + [c_int, i64, c_int, i64]
    L.isoq_kv_attn_prefix_workspace.restype = ctypes.c_size_t
    L.isoq_kv_copy_blocks.argtypes = [vp, vp, vp, i64, c_int, vp, vp, vp, vp, vp, vp, i64, c_int, vp]
    L.isoq_kv_compact.argtypes = [vp, vp, vp, c_int, c_int, vp, c_int, vp, c_int, c_int, vp, vp, vp, vp, vp, vp, i64,
                                  c_int, vp]
    L.isoq_kv_plan.argtypes = [vp, vp, c_int, vp, c_int, c_int, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp]
    L.isoq_rope_init.argtypes = [ctypes.POINTER(vp), c_int, c_int, c_int, dp, ctypes.c_double]
    L.isoq_rope_destroy.argtypes = [vp]
    L.isoq_rope_freqs.argtypes = [c_int] + [ctypes.c_double] * 5 + [dp]
    L.isoq_qk_norm_rope.argtypes = [vp, c_int, vp, i64, c_int, vp, i64, c_int, vp, i64, vp, vp, ctypes.c_float, vp, vp, vp]
    L.isoq_packed_bytes.argtypes = [c_int, c_int]
    L.isoq_packed_bytes.restype = ctypes.c_size_t
    L.isoq_record_bytes.argtypes = [c_int, c_int, c_int]
    L.isoq_record_bytes.restype = ctypes.c_size_t
    L.isoq_raw_params_per_set.argtypes = [c_int, c_int]
    L.isoq_raw_params_per_set.restype = ctypes.c_size_t
    L.isoq_export_params_per_set.argtypes = [c_int, c_int]
    L.isoq_export_params_per_set.restype = ctypes.c_size_t
    L.isoq_codebook_lloyd.argtypes = [c_int, c_int, c_int, dp]
    L.isoq_rotation_draws.argtypes = [c_int, c_int, c_int, ctypes.c_uint64, dp]
    L.isoq_status_string.argtypes = [c_int]
    L.isoq_status_string.restype = ctypes.c_char_p
    L.isoq_last_hip_error.argtypes = []
    L.isoq_last_hip_error.restype = ctypes.c_char_p
    for f in ("isoq_params_init", "isoq_params_destroy", "isoq_params_export", "isoq_params_info",
              "isoq_quantize", "isoq_dequantize", "isoq_roundtrip", "isoq_kv_append", "isoq_kv_scores", "isoq_sketch_init",
              "isoq_sketch_destroy", "isoq_sketch_export", "isoq_quantize_qjl", "isoq_kv_append_qjl",
              "isoq_kv_scores_qjl", "isoq_kv_scores_filled", "isoq_kv_attn", "isoq_kv_attn_cross",
              "isoq_kv_attn_prefix",
              "isoq_kv_copy_blocks", "isoq_kv_compact", "isoq_kv_plan", "isoq_rope_init", "isoq_rope_destroy",
              "isoq_rope_freqs", "isoq_qk_norm_rope", "isoq_codebook_lloyd",
              "isoq_rotation_draws"):
        getattr(L, f).restype = c_int
    return L


lib = _load()


def _check(st: int, where: str):
    if st != 0:
        raise IsoqError(st, where)


def _variant(v) -> int:
    return VARIANTS[v] if isinstance(v, str) else int(v)


def isoq_status_string(status: int) -> str:
    return lib.isoq_status_string(int(status)).decode()


def isoq_packed_bytes(d: int, bits: int) -> int:
    return int(lib.isoq_packed_bytes(int(d), int(bits)))


def isoq_record_bytes(variant, d: int, bits: int) -> int:
    return int(lib.isoq_record_bytes(_variant(variant), int(d), int(bits)))


def isoq_raw_params_per_set(variant, d: int) -> int:
    return int(lib.isoq_raw_params_per_set(_variant(variant), int(d)))


def isoq_export_params_per_set(variant, d: int) -> int:
    return int(lib.isoq_export_params_per_set(_variant(variant), int(d)))


def isoq_codebook_lloyd(bits: int, d: int, iters: int = 200) -> np.ndarray:
    out = np.zeros(1 << bits)
    _check(lib.isoq_codebook_lloyd(int(bits), int(d), int(iters),
                                   out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))),
           "isoq_codebook_lloyd")
    return out


def isoq_rotation_draws(variant, d: int, n_sets: int = 1, seed: int = 1) -> np.ndarray:
    v = _variant(variant)
    out = np.zeros(n_sets * isoq_raw_params_per_set(v, d))
    _check(lib.isoq_rotation_draws(v, int(d), int(n_sets), int(seed),
                                   out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))),
           "isoq_rotation_draws")
    return out


class Params:
    """Owner of an isoq_params handle (freed by close() or garbage collection)."""

    def __init__(self, handle: int, variant: int, d: int, bits: int, n_sets: int):
        self.handle = ctypes.c_void_p(handle)
        self.variant, self.d, self.bits, self.n_sets = variant, d, bits, n_sets
        self.record_bytes = isoq_record_bytes(variant, d, bits)

    def close(self):
        if self.handle:
            _check(lib.isoq_params_destroy(self.handle), "isoq_params_destroy")
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def isoq_params_init(variant, d: int, bits: int, n_sets: int = 1, rot=None, codebook=None,
                     seed: int = 1) -> Params:
    """Create a handle on the current device (see include/isoquant.h)."""
    v = _variant(variant)
    dp = ctypes.POINTER(ctypes.c_double)
    rot_a = None if rot is None else np.ascontiguousarray(rot, dtype=np.float64)
    cb_a = None if codebook is None else np.ascontiguousarray(codebook, dtype=np.float64)
    if rot_a is not None and rot_a.size != n_sets * isoq_raw_params_per_set(v, d):
        raise ValueError("rot has the wrong number of raw draws")
    if cb_a is not None and cb_a.size != (1 << bits):
        raise ValueError("codebook must have 2**bits levels")
    h = ctypes.c_void_p()
    _check(lib.isoq_params_init(ctypes.byref(h), v, int(d), int(bits), int(n_sets),
                                None if rot_a is None else rot_a.ctypes.data_as(dp),
                                None if cb_a is None else cb_a.ctypes.data_as(dp), int(seed)),
           "isoq_params_init")
    return Params(h.value, v, int(d), int(bits), int(n_sets))


def isoq_params_destroy(p: Params) -> None:
    p.close()


def isoq_params_export(p: Params):
    """(unit rotation parameters [n_sets * per_set], levels [2^b], thresholds [2^b - 1]), fp32."""
    rot = np.zeros(p.n_sets * isoq_export_params_per_set(p.variant, p.d), np.float32)
    lev = np.zeros(1 << p.bits, np.float32)
    thr = np.zeros((1 << p.bits) - 1, np.float32)
    fp = ctypes.POINTER(ctypes.c_float)
    _check(lib.isoq_params_export(p.handle, rot.ctypes.data_as(fp), lev.ctypes.data_as(fp),
                                  thr.ctypes.data_as(fp)), "isoq_params_export")
    return rot, lev, thr


def isoq_params_info(p: Params):
    vals = [ctypes.c_int() for _ in range(4)]
    _check(lib.isoq_params_info(p.handle, *[ctypes.byref(v) for v in vals]), "isoq_params_info")
    return tuple(v.value for v in vals)


# --- device calls ----------------------------------------------------------------
# A decode step's kernels run for about 5 us, so the calls below are written for
# few Python operations: pointers and sizes go to ctypes as plain integers (its
# argument types are declared above), shapes are compared as the tuples that
# they are, and a failed placement test is spelled out only after it failed.
try:
    import torch as _torch_module
except ImportError:
    _torch_module = None


def _torch():
    if _torch_module is None:
        raise ImportError("the device calls need torch")
    return _torch_module


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    c = _torch()._C
    return c._cuda_getCurrentRawStream(c._cuda_getDevice())   # of torch.cuda.current_stream()


def _dtype_code(t) -> int:
    torch = _torch()
    if t == torch.float16:
        return ISOQ_F16
    if t == torch.float32:
        return ISOQ_F32
    raise TypeError(f"rows must be float16 or float32, got {t}")


def _is_gpu(t) -> bool:
    return t.is_cuda


def _rows(x, d):
    _device_tensors(x, x=x)
    if x.dim() < 1 or x.shape[-1] != d:
        raise ValueError(f"x: last dimension must be d={d}")
    return x.numel() // d


def _like(name, t, dtypes, numel):
    """Type and size of a tensor argument: one of `dtypes`, `numel` elements."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if t.numel() != numel:
        raise ValueError(f"{name} must hold {numel} elements, got {t.numel()}")


def _device_tensors(ref, **ts):
    """Every tensor a kernel touches: on the GPU, contiguous, on ref's device
    (a pointer of the wrong kind or into the wrong memory would fault the GPU)."""
    for name, t in ts.items():
        if not _is_gpu(t):
            raise ValueError(f"{name} must be on the GPU")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.device != ref.device:
            raise ValueError(f"{name} must be on {ref.device}, got {t.device}")


def _placed(ref, ts):
    """_device_tensors for the decoding calls, the tensors named by their place."""
    dev = ref.get_device()
    for t in ts:
        if not (_is_gpu(t) and t.is_contiguous() and t.get_device() == dev):
            _device_tensors(ref, **{f"arg{i}": t for i, t in enumerate(ts)})


def _on_current(ref, ts, stream):
    """_placed, on the current device (where kernels are launched), which is the stream's too."""
    dev = ref.get_device()
    if dev < 0:
        _placed(ref, ts)
    for t in ts:   # (a device of 0 or more is a GPU)
        if t.get_device() != dev or not t.is_contiguous():
            _placed(ref, ts)
    if dev != _torch_module._C._cuda_getDevice():
        raise ValueError(f"tensors on {ref.device}, which is not the current device")
    if stream is not None and stream.device != ref.device:
        raise ValueError(f"tensors on {ref.device}, stream on {stream.device}")


def isoq_roundtrip(p: Params, x, rows_per_set: int = 1, x_hat=None, stream=None):
    """x_hat = stage-1 quantize->dequantize of x (same shape and dtype)."""
    n = _rows(x, p.d)
    _dtype_code(x.dtype)
    if x_hat is None:
        x_hat = _torch().empty_like(x)
    _like("x_hat", x_hat, (x.dtype,), n * p.d)
    _device_tensors(x, x_hat=x_hat)
    _check(lib.isoq_roundtrip(p.handle, _dtype_code(x.dtype), x.data_ptr(), n,
                              int(rows_per_set), x_hat.data_ptr(), _stream_ptr(stream)),
           "isoq_roundtrip")
    return x_hat


def isoq_quantize(p: Params, x, rows_per_set: int = 1, idx_packed=None, norms=None, stream=None):
    """(packed index records [n, isoq_record_bytes] uint8, norms [n] fp32)."""
    torch = _torch()
    n = _rows(x, p.d)
    if idx_packed is None:
        idx_packed = torch.empty((n, p.record_bytes), dtype=torch.uint8, device=x.device)
    if norms is None:
        norms = torch.empty((n,), dtype=torch.float32, device=x.device)
    _dtype_code(x.dtype)
    _like("idx_packed", idx_packed, (torch.uint8,), n * p.record_bytes)
    _like("norms", norms, (torch.float32,), n)
    _device_tensors(x, idx_packed=idx_packed, norms=norms)
    _check(lib.isoq_quantize(p.handle, _dtype_code(x.dtype), x.data_ptr(), n,
                             int(rows_per_set), idx_packed.data_ptr(),
                             norms.data_ptr(), _stream_ptr(stream)), "isoq_quantize")
    return idx_packed, norms


def isoq_dequantize(p: Params, idx_packed, norms, dtype=None, rows_per_set: int = 1, x_hat=None,
                    stream=None):
    """Rows [n, d] of `dtype` (default float16) from packed records and norms."""
    torch = _torch()
    _like("norms", norms, (torch.float32,), norms.numel() if isinstance(norms, torch.Tensor) else 0)
    n = norms.numel()
    _device_tensors(norms, norms=norms)
    if x_hat is None:
        x_hat = torch.empty((n, p.d), dtype=dtype or torch.float16, device=norms.device)
    _like("idx_packed", idx_packed, (torch.uint8,), n * p.record_bytes)
    _like("x_hat", x_hat, (torch.float16, torch.float32), n * p.d)
    if dtype is not None and x_hat.dtype != dtype:
        raise TypeError(f"x_hat is {x_hat.dtype}, dtype asks for {dtype}")
    _device_tensors(norms, idx_packed=idx_packed, x_hat=x_hat)
    _check(lib.isoq_dequantize(p.handle, _dtype_code(x_hat.dtype), idx_packed.data_ptr(),
                               norms.data_ptr(), n, int(rows_per_set),
                               x_hat.data_ptr(), _stream_ptr(stream)), "isoq_dequantize")
    return x_hat


def _ptr(t):
    return None if t is None else t.data_ptr()


def isoq_kv_append(pk: Params, k_new, slot_mapping, k_idx, k_rho, pv: Params = None, v_new=None,
                   v_idx=None, v_rho=None, stream=None):
    """Quantize new rows k_new (and v_new) [n_tokens, n_heads, d] into paged caches
    k_idx (v_idx) [n_blocks, n_heads, block_size, record_bytes] uint8 and k_rho
    (v_rho) [n_blocks, n_heads, block_size] fp32 at the slots slot_mapping
    [n_tokens] int64 (see include/isoquant.h).  The bytes of each
    [block_size, record_bytes] plane hold its records piece-major (pieces of
    P bytes, P = 16 or 8 when it divides record_bytes, else P = record_bytes:
    piece j of position s at byte (j block_size + s) P)."""
    torch = _torch()
    rows, cache = k_new.shape, k_idx.shape
    if len(rows) != 3 or len(cache) != 4 or k_rho.dim() != 3:
        raise ValueError("k_new [n_tokens, n_heads, d], k_idx [n_blocks, n_heads, block_size, R], "
                         "k_rho [n_blocks, n_heads, block_size]")
    n_tokens, n_heads, d = rows
    n_blocks, nh, block_size, rb = cache
    if d != pk.d or nh != n_heads or rb != pk.record_bytes or k_rho.shape != cache[:3]:
        raise ValueError("cache shapes do not match the rows and the handle")
    if slot_mapping.dtype != torch.int64 or slot_mapping.numel() != n_tokens:
        raise ValueError("slot_mapping must be int64 [n_tokens]")
    if k_idx.dtype != torch.uint8 or k_rho.dtype != torch.float32:
        raise TypeError("k_idx uint8, k_rho float32")
    dtype = k_new.dtype
    if v_new is None:
        _placed(k_new, (k_new, slot_mapping, k_idx, k_rho))
    else:
        if pv is None or v_idx is None or v_rho is None:
            raise ValueError("v_new needs pv, v_idx and v_rho")
        if v_new.shape != rows or v_idx.shape != cache or v_rho.shape != cache[:3] or v_new.dtype != dtype:
            raise ValueError("V tensors must have the shapes and dtype of the K tensors")
        _placed(k_new, (k_new, slot_mapping, k_idx, k_rho, v_new, v_idx, v_rho))
    st = lib.isoq_kv_append(pk.handle, None if pv is None else pv.handle, _dtype_code(dtype), k_new.data_ptr(),
                            _ptr(v_new), slot_mapping.data_ptr(), n_tokens, n_heads, k_idx.data_ptr(),
                            k_rho.data_ptr(), _ptr(v_idx), _ptr(v_rho), n_blocks, block_size, _stream_ptr(stream))
    if st:
        _check(st, "isoq_kv_append")


def isoq_kv_scores(pk: Params, q, k_idx, k_rho, block_table, seq_lens, scale: float = 1.0,
                   max_len=None, scores=None, stream=None, sketch=None, k_signs=None, k_gamma=None):
    """Attention logits scale * <q, k_hat> of queries q [n_seqs, n_q_heads, d]
    against the paged key cache k_idx [n_blocks, n_kv_heads, block_size, R] /
    k_rho [n_blocks, n_kv_heads, block_size], with block_table int32
    [n_seqs, max_blocks] and seq_lens int32 [n_seqs].  Returns fp32 scores
    [n_seqs, n_q_heads, max_len]; the kernel does not write positions at or
    past a sequence's length or behind an out-of-range block-table entry: a
    `scores` tensor allocated here holds -inf there, a caller's keeps its
    contents (see include/isoquant.h)."""
    torch = _torch()
    if q.dim() != 3 or k_idx.dim() != 4 or k_rho.dim() != 3 or block_table.dim() != 2:
        raise ValueError("q [n_seqs, n_q_heads, d], k_idx [n_blocks, n_kv_heads, block_size, R], "
                         "k_rho [n_blocks, n_kv_heads, block_size], block_table [n_seqs, max_blocks]")
    n_seqs, n_q_heads, d = q.shape
    cache = k_idx.shape
    n_blocks, n_kv_heads, block_size, rb = cache
    if d != pk.d or rb != pk.record_bytes or k_rho.shape != cache[:3]:
        raise ValueError("cache shapes do not match the queries and the handle")
    rows, max_blocks = block_table.shape
    if rows != n_seqs or seq_lens.numel() != n_seqs:
        raise ValueError("block_table and seq_lens need one row per sequence")
    if block_table.dtype != torch.int32 or seq_lens.dtype != torch.int32:
        raise TypeError("block_table and seq_lens must be int32")
    if max_len is None:
        max_len = max_blocks * block_size
    shape = (n_seqs, n_q_heads, max_len)
    # positions without a key (at or past a sequence's length, or behind an
    # invalid block-table entry) read as -inf in a tensor allocated here, so a
    # softmax over max_len ignores them: written by the same launch (which
    # takes max_len up to _FILL_MAX) instead of a pass of their own, unless there
    # is no key at all
    filled = scores is None and 0 < max_len <= _FILL_MAX and n_blocks > 0 and max_blocks > 0
    if filled:
        scores = torch.empty(shape, dtype=torch.float32, device=q.device)
    elif scores is None:
        scores = torch.full(shape, float("-inf"), dtype=torch.float32, device=q.device)
    elif scores.shape != shape or scores.dtype != torch.float32:
        raise ValueError("scores must be fp32 [n_seqs, n_q_heads, max_len]")
    if sketch is None:
        k_signs = k_gamma = None
        _placed(q, (q, k_idx, k_rho, block_table, seq_lens, scores))
    else:
        if k_signs is None or k_gamma is None:
            raise ValueError("a sketch needs k_signs and k_gamma")
        if (k_signs.shape != cache[:3] + (sketch.m // 8,) or k_signs.dtype != torch.uint8
                or k_gamma.shape != cache[:3] or k_gamma.dtype != torch.float32):
            raise ValueError("k_signs [n_blocks, n_kv_heads, block_size, m/8] uint8, k_gamma like k_rho")
        _placed(q, (q, k_idx, k_rho, block_table, seq_lens, scores, k_signs, k_gamma))
    head_args = (_dtype_code(q.dtype), q.data_ptr(), n_seqs, n_q_heads, n_kv_heads, k_idx.data_ptr(),
                 k_rho.data_ptr())
    cache_args = (n_blocks, block_size, block_table.data_ptr(), max_blocks, seq_lens.data_ptr(), float(scale),
                  scores.data_ptr(), int(max_len), _stream_ptr(stream))
    if filled:
        st = lib.isoq_kv_scores_filled(pk.handle, None if sketch is None else sketch.handle, *head_args,
                                       _ptr(k_signs), _ptr(k_gamma), *cache_args)
    elif sketch is None:
        st = lib.isoq_kv_scores(pk.handle, *head_args, *cache_args)
    else:
        st = lib.isoq_kv_scores_qjl(pk.handle, sketch.handle, *head_args, k_signs.data_ptr(), k_gamma.data_ptr(),
                                    *cache_args)
    if st:
        _check(st, "isoq_kv_scores" if sketch is None else "isoq_kv_scores_qjl")
    return scores


_FILL_MAX = 65535 * 1024   # the filled call's largest max_len


def isoq_kv_scores_qjl(pk: Params, sketch, q, k_idx, k_rho, k_signs, k_gamma, block_table, seq_lens,
                       scale: float = 1.0, max_len=None, scores=None, stream=None):
    """isoq_kv_scores with the stage-2 residual correction (see include/isoquant.h)."""
    return isoq_kv_scores(pk, q, k_idx, k_rho, block_table, seq_lens, scale, max_len, scores, stream,
                          sketch=sketch, k_signs=k_signs, k_gamma=k_gamma)


def isoq_kv_attn_workspace(pk: Params, pv: Params, dtype, n_tokens: int, max_q_len: int, n_seqs: int, n_q_heads: int,
                           n_kv_heads: int, block_size: int, max_blocks_per_seq: int, max_len: int) -> int:
    """Bytes of workspace that isoq_kv_attn takes for these sizes (see include/isoquant.h)."""
    return int(lib.isoq_kv_attn_workspace(pk.handle, pv.handle, _dtype_code(dtype), int(n_tokens), int(max_q_len),
                                          int(n_seqs), int(n_q_heads), int(n_kv_heads), int(block_size),
                                          int(max_blocks_per_seq), int(max_len)))


def _attn_buffers(q, k_idx, k_rho, out, lse, workspace, need):
    # (new_empty of a tensor of the type: 0.4 us less than torch.empty with one)
    if out is None:
        out = _torch_module.empty_like(q)
    if lse is None:
        lse = k_rho.new_empty(q.shape[0], q.shape[1])
    if workspace is None and need:
        workspace = k_idx.new_empty(need)
    return out, lse, workspace


def isoq_kv_attn(pk: Params, q, k_idx, k_rho, pv: Params, v_idx, v_rho, block_table, seq_lens, scale: float = 1.0,
                 q_start=None, max_q_len=None, max_len=None, out=None, lse=None, workspace=None, stream=None,
                 causal: bool = True, prefix=None):
    """Attention of new tokens' queries q [n_tokens, n_q_heads, d] over the paged
    caches k_idx, v_idx [n_blocks, n_kv_heads, block_size, R] / k_rho, v_rho
    [n_blocks, n_kv_heads, block_size] with block_table int32 [n_seqs,
    max_blocks] and seq_lens int32 [n_seqs].  One token a sequence, or with
    q_start int32 [n_seqs + 1] the tokens q_start[s] .. q_start[s + 1] - 1 of
    sequence s, at most max_q_len, which are its last positions (causal).
    max_q_len and max_len (the longest sequence's positions) are bounds that the
    call is planned by, by default n_tokens and what block_table holds: give both
    where they are known (64 single tokens at 2,000 positions, 8 x 4 heads, with
    q_start: 39 us with max_q_len=1, 191 without).
    Returns (out like q, lse fp32 [n_tokens, n_q_heads]); rows of no sequence
    are not written (see include/isoquant.h).  workspace: a uint8 tensor of at
    least isoq_kv_attn_workspace(...) bytes.  What is not passed (out, lse,
    workspace) is allocated from torch's pool for `stream`, by default the
    current one.  causal=False is isoq_kv_attn_cross; prefix is what
    isoq_kv_attn_prefix, to be called instead, makes of its arguments."""
    torch = _torch()
    if prefix is not None and not causal:
        raise ValueError("attention behind a prefix is causal")
    shape, cache, table = q.shape, k_idx.shape, block_table.shape
    if len(shape) != 3 or len(cache) != 4 or len(table) != 2:
        raise ValueError("q [n_tokens, n_q_heads, d], k_idx [n_blocks, n_kv_heads, block_size, R], "
                         "k_rho [n_blocks, n_kv_heads, block_size], block_table [n_seqs, max_blocks]")
    n_tokens, n_q_heads, d = shape
    n_blocks, n_kv_heads, block_size, rb = cache
    n_seqs, max_blocks = table
    norms = (n_blocks, n_kv_heads, block_size)
    if d != pk.d or rb != pk.record_bytes or v_idx.shape != cache or k_rho.shape != norms or v_rho.shape != norms:
        raise ValueError("cache shapes do not match the queries and the handle")
    if seq_lens.shape != (n_seqs,):
        raise ValueError("block_table and seq_lens need one row per sequence")
    byte, single, whole = torch.uint8, torch.float32, torch.int32
    if k_idx.dtype != byte or v_idx.dtype != byte or k_rho.dtype != single or v_rho.dtype != single:
        raise TypeError("k_idx and v_idx uint8, k_rho and v_rho float32")
    if block_table.dtype != whole or seq_lens.dtype != whole:
        raise TypeError("block_table and seq_lens must be int32")
    code = _dtype_code(q.dtype)
    if max_q_len is None:
        max_q_len = 1 if q_start is None else max(1, n_tokens)
    if q_start is None:
        if n_tokens != n_seqs or max_q_len != 1:
            raise ValueError("without q_start there is one token a sequence")
    elif q_start.shape != (n_seqs + 1,) or q_start.dtype != torch.int32:
        raise ValueError("q_start must be int32 [n_seqs + 1]")
    if out is not None and (out.shape != shape or out.dtype != q.dtype):
        raise ValueError("out must have q's shape and dtype")
    if lse is not None and (lse.shape != (n_tokens, n_q_heads) or lse.dtype != torch.float32):
        raise ValueError("lse must be fp32 [n_tokens, n_q_heads]")
    if max_len is None:
        max_len = max_blocks * block_size
    if prefix is None:
        need = lib.isoq_kv_attn_workspace(pk.handle, pv.handle, code, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads,
                                          block_size, max_blocks, max_len)
    else:
        need = lib.isoq_kv_attn_prefix_workspace(pk.handle, pv.handle, code, n_tokens, max_q_len, n_seqs, n_q_heads,
                                                 n_kv_heads, block_size, max_blocks, max_len, *prefix.sizes)
    if workspace is not None and (workspace.dtype != torch.uint8 or workspace.numel() < need):
        raise ValueError(f"workspace must be uint8 of at least {need} bytes")
    tensors = [q, k_idx, k_rho, v_idx, v_rho, block_table, seq_lens]
    for t in (q_start, out, lse, workspace):
        if t is not None:
            tensors.append(t)
    if prefix is not None:
        tensors += prefix.tensors
    _on_current(q, tensors, stream)
    if stream is None:
        out, lse, workspace = _attn_buffers(q, k_idx, k_rho, out, lse, workspace, need)
    else:
        with torch.cuda.stream(stream):
            out, lse, workspace = _attn_buffers(q, k_idx, k_rho, out, lse, workspace, need)
    if prefix is None:
        st = (lib.isoq_kv_attn if causal else lib.isoq_kv_attn_cross)(
            pk.handle, pv.handle, code, q.data_ptr(), _ptr(q_start), n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads,
            k_idx.data_ptr(), k_rho.data_ptr(), v_idx.data_ptr(), v_rho.data_ptr(), n_blocks, block_size,
            block_table.data_ptr(), max_blocks, seq_lens.data_ptr(), max_len, scale, out.data_ptr(), lse.data_ptr(),
            _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream))
    else:
        st = lib.isoq_kv_attn_prefix(
            pk.handle, pv.handle, code, q.data_ptr(), _ptr(q_start), n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads,
            k_idx.data_ptr(), k_rho.data_ptr(), v_idx.data_ptr(), v_rho.data_ptr(), n_blocks, block_size,
            block_table.data_ptr(), max_blocks, seq_lens.data_ptr(), max_len, *prefix.args, scale, out.data_ptr(),
            lse.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream))
    if st:
        _check(st, "isoq_kv_attn" if causal and prefix is None else "isoq_kv_attn_cross" if prefix is None else
               "isoq_kv_attn_prefix")
    return out, lse


def isoq_kv_attn_cross(pk: Params, q, k_idx, k_rho, pv: Params, v_idx, v_rho, block_table, seq_lens, scale: float = 1.0,
                       q_start=None, max_q_len=None, max_len=None, out=None, lse=None, workspace=None, stream=None):
    """isoq_kv_attn with every token of a sequence attending to all of its
    seq_lens positions: a decoder's attention to its encoder's states, which stand
    in the cache (see include/isoquant.h).  Arguments and results as isoq_kv_attn."""
    return isoq_kv_attn(pk, q, k_idx, k_rho, pv, v_idx, v_rho, block_table, seq_lens, scale, q_start, max_q_len, max_len,
                        out, lse, workspace, stream, False)


class _Prefix:
    """The arguments of isoq_kv_attn_prefix beyond those of isoq_kv_attn, checked."""
    __slots__ = ("tensors", "sizes", "args")

    def __init__(self, table, lens, start, max_tokens, max_len, n_tokens, block_size):
        whole = _torch_module.int32
        if table.dim() != 2 or lens.shape != (table.shape[0],) or table.dtype != whole or lens.dtype != whole:
            raise ValueError("prefix_table int32 [n_prefixes, max_prefix_blocks], prefix_lens int32 [n_prefixes]")
        n, blocks = table.shape
        self.tensors = [table, lens]
        if start is not None:
            if start.shape != (n + 1,) or start.dtype != whole:
                raise ValueError("prefix_start must be int32 [n_prefixes + 1]")
            self.tensors.append(start)
        elif n > 1:
            raise ValueError("several prefixes need prefix_start")
        max_tokens = n_tokens if max_tokens is None else max_tokens
        max_len = blocks * block_size if max_len is None else max_len
        self.sizes = (n, max_tokens, blocks, max_len)
        self.args = (table.data_ptr(), blocks, lens.data_ptr(), max_len, _ptr(start), n, max_tokens)


def isoq_kv_attn_prefix(pk: Params, q, k_idx, k_rho, pv: Params, v_idx, v_rho, block_table, seq_lens, prefix_table,
                        prefix_lens, prefix_start=None, scale: float = 1.0, q_start=None, max_q_len=None, max_len=None,
                        max_prefix_tokens=None, max_prefix_len=None, out=None, lse=None, workspace=None, stream=None):
    """isoq_kv_attn for sequences that share long beginnings: prefix_table int32
    [n_prefixes, max_prefix_blocks] and prefix_lens int32 [n_prefixes] are in the
    same cache once, and prefix p is what the sequences prefix_start[p] ..
    prefix_start[p + 1] - 1 (int32 [n_prefixes + 1]; None: one prefix, of all) begin
    with; block_table and seq_lens are the sequences' own positions after it.
    Rows are to be rotated by positions that count the prefix's (isoq_kv_plan's do not).
    max_prefix_tokens: tokens of one prefix's sequences at most (by default all
    there are); max_prefix_len: positions of the longest prefix at most.  Other
    arguments and results as isoq_kv_attn, workspace of at least
    isoq_kv_attn_prefix_workspace(...) bytes."""
    _torch()
    if q.dim() != 3 or k_idx.dim() != 4:
        raise ValueError("q [n_tokens, n_q_heads, d], k_idx [n_blocks, n_kv_heads, block_size, R]")
    prefix = _Prefix(prefix_table, prefix_lens, prefix_start, max_prefix_tokens, max_prefix_len, q.shape[0], k_idx.shape[2])
    return isoq_kv_attn(pk, q, k_idx, k_rho, pv, v_idx, v_rho, block_table, seq_lens, scale, q_start, max_q_len, max_len,
                        out, lse, workspace, stream, True, prefix)


def isoq_kv_attn_prefix_workspace(pk: Params, pv: Params, dtype, n_tokens: int, max_q_len: int, n_seqs: int,
                                  n_q_heads: int, n_kv_heads: int, block_size: int, max_blocks_per_seq: int, max_len: int,
                                  n_prefixes: int, max_prefix_tokens: int, max_prefix_blocks: int,
                                  max_prefix_len: int) -> int:
    """Bytes of workspace that isoq_kv_attn_prefix takes for these sizes (see include/isoquant.h)."""
    return int(lib.isoq_kv_attn_prefix_workspace(pk.handle, pv.handle, _dtype_code(dtype), int(n_tokens), int(max_q_len),
                                                 int(n_seqs), int(n_q_heads), int(n_kv_heads), int(block_size),
                                                 int(max_blocks_per_seq), int(max_len), int(n_prefixes),
                                                 int(max_prefix_tokens), int(max_prefix_blocks), int(max_prefix_len)))


class Sketch:
    """Owner of an isoq_sketch handle (stage-2 projection of a quantizer)."""

    def __init__(self, handle: int, p: Params, m: int):
        self.handle = ctypes.c_void_p(handle)
        self.params, self.m, self.d = p, int(m), p.d

    def close(self):
        if self.handle:
            _check(lib.isoq_sketch_destroy(self.handle), "isoq_sketch_destroy")
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def isoq_sketch_init(p: Params, m: int, S=None, seed: int = 7) -> Sketch:
    """Stage-2 sketch of quantizer p: projection S [m, d] (given, or drawn from seed)."""
    dp = ctypes.POINTER(ctypes.c_double)
    S_a = None if S is None else np.ascontiguousarray(S, dtype=np.float64)
    if S_a is not None and S_a.shape != (m, p.d):
        raise ValueError("S must be [m, d]")
    h = ctypes.c_void_p()
    _check(lib.isoq_sketch_init(ctypes.byref(h), p.handle, int(m),
                                None if S_a is None else S_a.ctypes.data_as(dp), int(seed)),
           "isoq_sketch_init")
    return Sketch(h.value, p, m)


def isoq_sketch_destroy(sk: Sketch) -> None:
    sk.close()


def isoq_sketch_export(sk: Sketch):
    """(m, S as used, float32 [m, d])."""
    m = ctypes.c_int()
    S = np.zeros((sk.m, sk.d), np.float32)
    _check(lib.isoq_sketch_export(sk.handle, ctypes.byref(m), S.ctypes.data_as(ctypes.POINTER(ctypes.c_float))),
           "isoq_sketch_export")
    return m.value, S


def isoq_quantize_qjl(p: Params, sk: Sketch, x, rows_per_set: int = 1, idx_packed=None, norms=None,
                      signs=None, gamma=None, stream=None):
    """(records [n, R] uint8, norms [n] fp32, sign sketch [n, m/8] uint8, gamma [n] fp32)."""
    torch = _torch()
    n = _rows(x, p.d)
    dev = x.device
    if idx_packed is None:
        idx_packed = torch.empty((n, p.record_bytes), dtype=torch.uint8, device=dev)
    if norms is None:
        norms = torch.empty((n,), dtype=torch.float32, device=dev)
    if signs is None:
        signs = torch.empty((n, sk.m // 8), dtype=torch.uint8, device=dev)
    if gamma is None:
        gamma = torch.empty((n,), dtype=torch.float32, device=dev)
    _dtype_code(x.dtype)
    _like("idx_packed", idx_packed, (torch.uint8,), n * p.record_bytes)
    _like("norms", norms, (torch.float32,), n)
    _like("signs", signs, (torch.uint8,), n * (sk.m // 8))
    _like("gamma", gamma, (torch.float32,), n)
    _device_tensors(x, idx_packed=idx_packed, norms=norms, signs=signs, gamma=gamma)
    _check(lib.isoq_quantize_qjl(p.handle, sk.handle, _dtype_code(x.dtype), _ptr(x), n, int(rows_per_set),
                                 _ptr(idx_packed), _ptr(norms), _ptr(signs), _ptr(gamma), _stream_ptr(stream)),
           "isoq_quantize_qjl")
    return idx_packed, norms, signs, gamma


def isoq_kv_append_qjl(pk: Params, sk: Sketch, k_new, slot_mapping, k_idx, k_rho, k_signs, k_gamma,
                       stream=None):
    """Quantize new key rows k_new [n_tokens, n_heads, d] with the stage-2
    sketch into the paged caches k_idx [n_blocks, n_heads, block_size, R],
    k_rho and k_gamma [n_blocks, n_heads, block_size] fp32 and k_signs
    [n_blocks, n_heads, block_size, m/8] uint8 at the slots slot_mapping
    [n_tokens] int64 (see include/isoquant.h)."""
    torch = _torch()
    if k_new.dim() != 3 or k_idx.dim() != 4 or k_rho.dim() != 3 or k_signs.dim() != 4 or k_gamma.dim() != 3:
        raise ValueError("k_new [n_tokens, n_heads, d], k_idx [n_blocks, n_heads, block_size, R], "
                         "k_signs [n_blocks, n_heads, block_size, m/8], k_rho and k_gamma [n_blocks, n_heads, "
                         "block_size]")
    n_tokens, n_heads, d = k_new.shape
    n_blocks, nh, block_size, rb = k_idx.shape
    cache = (n_blocks, nh, block_size)
    if (d != pk.d or nh != n_heads or rb != pk.record_bytes or k_rho.shape != cache
            or k_gamma.shape != cache or k_signs.shape != cache + (sk.m // 8,)):
        raise ValueError("cache shapes do not match the rows, the handle and the sketch")
    if slot_mapping.dtype != torch.int64 or slot_mapping.numel() != n_tokens:
        raise ValueError("slot_mapping must be int64 [n_tokens]")
    if (k_idx.dtype != torch.uint8 or k_signs.dtype != torch.uint8 or k_rho.dtype != torch.float32
            or k_gamma.dtype != torch.float32):
        raise TypeError("k_idx and k_signs uint8, k_rho and k_gamma float32")
    _placed(k_new, (k_new, slot_mapping, k_idx, k_rho, k_signs, k_gamma))
    st = lib.isoq_kv_append_qjl(pk.handle, sk.handle, _dtype_code(k_new.dtype), k_new.data_ptr(),
                                slot_mapping.data_ptr(), n_tokens, n_heads, k_idx.data_ptr(), k_rho.data_ptr(),
                                k_signs.data_ptr(), k_gamma.data_ptr(), n_blocks, block_size, _stream_ptr(stream))
    if st:
        _check(st, "isoq_kv_append_qjl")


def _cache_planes(pk: Params, k_idx, k_rho, v_idx, v_rho, sketch, k_signs, k_gamma):
    """Checks of the cache that a page call moves; the tensors that are there."""
    torch = _torch()
    cache = k_idx.shape
    if len(cache) != 4:
        raise ValueError("k_idx [n_blocks, n_heads, block_size, R], k_rho [n_blocks, n_heads, block_size]")
    norms = cache[:3]
    if cache[3] != pk.record_bytes or k_rho.shape != norms:
        raise ValueError("cache shapes do not match the handle")
    tensors = (k_idx, k_rho)
    if (v_idx is None) != (v_rho is None):
        raise ValueError("v_idx and v_rho come together")
    if v_idx is not None:
        if v_idx.shape != cache or v_rho.shape != norms:
            raise ValueError("V tensors must have the shapes of the K tensors")
        tensors = (k_idx, k_rho, v_idx, v_rho)
    if sketch is None:
        if k_signs is not None or k_gamma is not None:
            raise ValueError("k_signs and k_gamma need their sketch")
    else:
        if k_signs is None or k_gamma is None:
            raise ValueError("a sketch needs k_signs and k_gamma")
        if k_signs.shape != norms + (sketch.m // 8,) or k_gamma.shape != norms:
            raise ValueError("k_signs [n_blocks, n_heads, block_size, m/8], k_gamma like k_rho")
        tensors += (k_signs, k_gamma)
    byte, single = torch.uint8, torch.float32
    for i in range(0, len(tensors), 2):   # records (or signs) and norms in turn
        if tensors[i].dtype != byte or tensors[i + 1].dtype != single:
            raise TypeError("records and signs must be uint8, norms and gammas float32")
    return tensors


def isoq_kv_copy_blocks(pk: Params, block_pairs, k_idx, k_rho, v_idx=None, v_rho=None, sketch=None, k_signs=None,
                        k_gamma=None, stream=None):
    """Copy whole cache blocks: block_pairs int32 [n_pairs, 2], (source,
    destination) each, over all heads of the K (and V) records and norms and
    of the sketch's arrays (see include/isoquant.h)."""
    torch = _torch()
    tensors = _cache_planes(pk, k_idx, k_rho, v_idx, v_rho, sketch, k_signs, k_gamma)
    if block_pairs.dim() != 2 or block_pairs.shape[1] != 2 or block_pairs.dtype != torch.int32:
        raise ValueError("block_pairs must be int32 [n_pairs, 2]")
    _on_current(k_idx, tensors + (block_pairs,), stream)
    n_blocks, n_heads, block_size, _ = k_idx.shape
    st = lib.isoq_kv_copy_blocks(pk.handle, None if sketch is None else sketch.handle, block_pairs.data_ptr(),
                                 block_pairs.shape[0], n_heads, k_idx.data_ptr(), k_rho.data_ptr(), _ptr(v_idx),
                                 _ptr(v_rho), _ptr(k_signs), _ptr(k_gamma), n_blocks, block_size, _stream_ptr(stream))
    if st:
        _check(st, "isoq_kv_copy_blocks")


def isoq_kv_compact(pk: Params, keep, n_keep, block_table, k_idx, k_rho, v_idx=None, v_rho=None, sketch=None,
                    k_signs=None, k_gamma=None, stream=None):
    """Compact sequences in place to the positions that stay: keep int32
    [n_seqs, n_heads or 1, max_keep], strictly ascending, of which n_keep int32
    [n_seqs] count; block_table int32 [n_seqs, max_blocks].  Afterwards n_keep is
    the sequences' lengths (see include/isoquant.h)."""
    torch = _torch()
    tensors = _cache_planes(pk, k_idx, k_rho, v_idx, v_rho, sketch, k_signs, k_gamma)
    n_blocks, n_heads, block_size, _ = k_idx.shape
    if keep.dim() != 3 or keep.shape[1] not in (1, n_heads):
        raise ValueError("keep must be [n_seqs, n_heads or 1, max_keep]")
    n_seqs, keep_heads, max_keep = keep.shape
    if n_keep.shape != (n_seqs,) or block_table.dim() != 2 or block_table.shape[0] != n_seqs:
        raise ValueError("n_keep [n_seqs] and block_table [n_seqs, max_blocks] need one row per sequence")
    if keep.dtype != torch.int32 or n_keep.dtype != torch.int32 or block_table.dtype != torch.int32:
        raise TypeError("keep, n_keep and block_table must be int32")
    _on_current(k_idx, tensors + (keep, n_keep, block_table), stream)
    st = lib.isoq_kv_compact(pk.handle, None if sketch is None else sketch.handle, keep.data_ptr(), keep_heads,
                             max_keep, n_keep.data_ptr(), n_seqs, block_table.data_ptr(), block_table.shape[1],
                             n_heads, k_idx.data_ptr(), k_rho.data_ptr(), _ptr(v_idx), _ptr(v_rho), _ptr(k_signs),
                             _ptr(k_gamma), n_blocks, block_size, _stream_ptr(stream))
    if st:
        _check(st, "isoq_kv_compact")


def isoq_kv_plan(lens, new_lens, block_table, block_size: int, free_blocks, n_free, n_tokens=None, seq_lens=None,
                 q_start=None, slot_mapping=None, positions=None, n_free_out=None, stream=None):
    """Blocks and slots of a step's tokens from the sequences' lengths before and
    after it, lens and new_lens int32 [n_seqs]: block_table int32 [n_seqs,
    max_blocks] and free_blocks int32 [max_free], of which the first n_free (int32
    [1]) are free, are updated; n_tokens is the most new tokens that the step may
    have (by default as many as slot_mapping holds).  Returns (seq_lens int32
    [n_seqs], q_start int32 [n_seqs + 1], slot_mapping int64 [n_tokens], positions
    int32 [n_tokens], n_free_out int32 [1]): seq_lens may be lens, n_free_out
    n_free.  positions count from 0 in a sequence's own table: behind a prefix
    (isoq_kv_attn_prefix) add its length before isoq_qk_norm_rope.  See
    include/isoquant.h for sequences that are refused.  What is not passed is
    allocated from torch's pool for `stream`; where none of the int32 results is
    passed they are parts of one allocation, which any of them keeps."""
    torch = _torch()
    table = block_table.shape
    if len(table) != 2 or free_blocks.dim() != 1:
        raise ValueError("block_table [n_seqs, max_blocks], free_blocks [max_free]")
    n_seqs, max_blocks = table
    if lens.shape != (n_seqs,) or new_lens.shape != (n_seqs,) or n_free.shape != (1,):
        raise ValueError("lens and new_lens need one entry per row of block_table, n_free one")
    whole = torch.int32
    if (lens.dtype != whole or new_lens.dtype != whole or block_table.dtype != whole or free_blocks.dtype != whole
            or n_free.dtype != whole):
        raise TypeError("lens, new_lens, block_table, free_blocks and n_free must be int32")
    if n_tokens is None:
        if slot_mapping is None:
            raise ValueError("n_tokens, or a slot_mapping of that length")
        n_tokens = slot_mapping.numel()
    tensors = [lens, new_lens, block_table, free_blocks, n_free]
    for t, n in ((seq_lens, n_seqs), (q_start, n_seqs + 1), (slot_mapping, n_tokens), (positions, n_tokens), (n_free_out, 1)):
        if t is not None:
            if t.shape != (n,) or t.dtype != (torch.int64 if t is slot_mapping else whole):
                raise ValueError("seq_lens [n_seqs], q_start [n_seqs + 1], positions [n_tokens] and n_free_out [1] must be "
                                 "int32, slot_mapping [n_tokens] int64")
            tensors.append(t)
    _on_current(lens, tensors, stream)
    outs = seq_lens, q_start, slot_mapping, positions, n_free_out
    if stream is None:
        outs = _plan_buffers(lens, n_seqs, n_tokens, *outs)
    else:
        with torch.cuda.stream(stream):
            outs = _plan_buffers(lens, n_seqs, n_tokens, *outs)
    seq_lens, q_start, slot_mapping, positions, n_free_out = outs
    st = lib.isoq_kv_plan(lens.data_ptr(), new_lens.data_ptr(), n_seqs, block_table.data_ptr(), max_blocks, block_size,
                          free_blocks.data_ptr(), free_blocks.numel(), n_free.data_ptr(), seq_lens.data_ptr(),
                          q_start.data_ptr(), slot_mapping.data_ptr(), positions.data_ptr(), n_tokens,
                          n_free_out.data_ptr(), _stream_ptr(stream))
    if st:
        _check(st, "isoq_kv_plan")
    return outs


def _plan_buffers(lens, n_seqs, n_tokens, seq_lens, q_start, slot_mapping, positions, n_free_out):
    if slot_mapping is None:
        slot_mapping = lens.new_empty(n_tokens, dtype=_torch_module.int64)
    if seq_lens is None and q_start is None and positions is None and n_free_out is None:
        # (parts of one allocation, which takes half of the time of four)
        seq_lens, q_start, positions, n_free_out = _torch_module.split_with_sizes(
            lens.new_empty(2 * n_seqs + n_tokens + 2), (n_seqs, n_seqs + 1, n_tokens, 1))
        return seq_lens, q_start, slot_mapping, positions, n_free_out
    if seq_lens is None:
        seq_lens = lens.new_empty(n_seqs)
    if q_start is None:
        q_start = lens.new_empty(n_seqs + 1)
    if positions is None:
        positions = lens.new_empty(n_tokens)
    if n_free_out is None:
        n_free_out = lens.new_empty(1)
    return seq_lens, q_start, slot_mapping, positions, n_free_out


class Rope:
    """Owner of an isoq_rope handle (angles of rotary positions)."""

    def __init__(self, handle: int, d: int, rot_dim: int, layout: int):
        self.handle = ctypes.c_void_p(handle)
        self.d, self.rot_dim, self.layout = d, rot_dim, layout

    def close(self):
        if self.handle:
            _check(lib.isoq_rope_destroy(self.handle), "isoq_rope_destroy")
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def isoq_rope_freqs(rot_dim: int, base: float = 10000.0, factor: float = 1.0, original: float = 0.0, low: float = 1.0,
                    high: float = 32.0) -> np.ndarray:
    """Angles a position of the rot_dim / 2 pairs: base^(-2 i / rot_dim), slowed
    down by up to `factor` for contexts longer than `original` positions (see
    include/isoquant.h)."""
    out = np.zeros(max(0, int(rot_dim)) // 2)
    _check(lib.isoq_rope_freqs(int(rot_dim), float(base), float(factor), float(original), float(low), float(high),
                               out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))), "isoq_rope_freqs")
    return out


def isoq_rope_init(d: int, rot_dim=None, layout="halves", freqs=None, amplitude: float = 1.0) -> Rope:
    """Rotary positions of heads of width d on the current device: the first
    rot_dim coordinates (all by default) in pairs (2 i, 2 i + 1), layout "pairs", or
    (i, rot_dim / 2 + i), "halves"; freqs [rot_dim / 2] angles a position, by
    default isoq_rope_freqs(rot_dim)."""
    rot_dim = int(d) if rot_dim is None else int(rot_dim)
    if isinstance(layout, str):
        layout = LAYOUTS[layout]
    f = np.ascontiguousarray(isoq_rope_freqs(rot_dim) if freqs is None and rot_dim > 0 else [] if freqs is None else freqs,
                             dtype=np.float64)
    if f.shape != (max(0, rot_dim) // 2,):
        raise ValueError("freqs must hold rot_dim / 2 angles")
    h = ctypes.c_void_p()
    _check(lib.isoq_rope_init(ctypes.byref(h), int(d), rot_dim, int(layout),
                              f.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), float(amplitude)), "isoq_rope_init")
    return Rope(h.value, int(d), rot_dim, int(layout))


def isoq_rope_destroy(r: Rope) -> None:
    r.close()


def _token_stride(name, x):
    """Elements between the tokens of rows [n_tokens, heads, d], whose heads lie one after another."""
    n, heads, d = x.shape
    token, head, one = x.stride()
    if (d > 1 and one != 1) or (heads > 1 and head != d) or (n > 1 and token < heads * d):
        raise ValueError(f"{name}: a token's heads must be contiguous, tokens at least as far apart")
    return token if n > 1 else heads * d


def isoq_qk_norm_rope(rope: Rope, q, k, positions, q_weight=None, k_weight=None, eps: float = 1e-6, q_out=None,
                      k_out=None, stream=None):
    """Norms (where there is a weight, fp32 [d]) and rotary positions of new
    tokens' queries q [n_tokens, n_q_heads, d] and keys k [n_tokens, n_kv_heads, d]
    (or None): views into one projection's output may be passed, only a token's
    heads have to be contiguous.  positions int32 [n_tokens].  Returns (q_out,
    k_out), contiguous; they may be q and k themselves (see include/isoquant.h)."""
    torch = _torch()
    shape, d, dtype = q.shape, rope.d, q.dtype
    if len(shape) != 3 or shape[2] != d:
        raise ValueError(f"q must be [n_tokens, n_q_heads, {d}]")
    n_tokens, n_q_heads, _ = shape
    q_stride = n_q_heads * d if q.is_contiguous() else _token_stride("q", q)
    code = _dtype_code(dtype)
    if positions.shape != (n_tokens,) or positions.dtype != torch.int32:
        raise ValueError("positions must be int32 [n_tokens]")
    tensors = [positions]
    device = positions.get_device()
    if not _is_gpu(q) or q.get_device() != device:
        raise ValueError(f"q must be on {positions.device}, got {q.device}")
    k_stride = n_kv_heads = 0
    if k is not None:
        rows = k.shape
        if len(rows) != 3 or rows[0] != n_tokens or rows[2] != d or k.dtype != dtype:
            raise ValueError(f"k must be {dtype} [n_tokens, n_kv_heads, {d}]")
        n_kv_heads = rows[1]
        k_stride = n_kv_heads * d if k.is_contiguous() else _token_stride("k", k)
        if not _is_gpu(k) or k.get_device() != device:
            raise ValueError(f"k must be on {positions.device}, got {k.device}")
    elif k_out is not None or k_weight is not None:
        raise ValueError("k_out and k_weight need k")
    for w in (q_weight, k_weight):
        if w is not None:
            if w.shape != (d,) or w.dtype != torch.float32:
                raise ValueError("weights must be float32 [d]")
            tensors.append(w)
    for x, out in ((q, q_out), (k, k_out)):
        if out is not None:
            if out.shape != x.shape or out.dtype != dtype:
                raise ValueError("q_out and k_out must have the shapes and dtype of q and k")
            tensors.append(out)
    _on_current(positions, tensors, stream)
    if stream is None:
        q_out, k_out = _rope_buffers(q, k, q_out, k_out)
    else:
        with torch.cuda.stream(stream):
            q_out, k_out = _rope_buffers(q, k, q_out, k_out)
    st = lib.isoq_qk_norm_rope(rope.handle, code, q.data_ptr(), q_stride, n_q_heads, _ptr(k), k_stride, n_kv_heads,
                               positions.data_ptr(), n_tokens, _ptr(q_weight), _ptr(k_weight), eps, q_out.data_ptr(),
                               _ptr(k_out), _stream_ptr(stream))
    if st:
        _check(st, "isoq_qk_norm_rope")
    return q_out, k_out


def _rope_buffers(q, k, q_out, k_out):
    # (empty_like, which copies strides too: 0.6 us less than new_empty with a shape)
    if q_out is None:
        q_out = _torch_module.empty_like(q) if q.is_contiguous() else q.new_empty(q.shape)
    if k_out is None and k is not None:
        k_out = _torch_module.empty_like(k) if k.is_contiguous() else k.new_empty(k.shape)
    return q_out, k_out
