"""GB300 CDSL lookahead step: Python binding of the C ABI in include/cdsl.h.

Argument marshalling only: every step of the path runs in the CUDA library
``libcdsl_gb300.so`` (built in-tree by ``paper_2412_10418_gb300.build``). Importing this module
fails loudly when the library is missing; there is no CPU fallback.

Functions carry the C names (``cdsl_init``, ``cdsl_prefill``, ``cdsl_lookahead``,
``cdsl_verify``, ``cdsl_select``, ``cdsl_step`` ...) and take torch CUDA tensors where the C
call takes device pointers. ``Engine`` bundles a context with its workspace and outputs.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcdsl_gb300.so")

DTYPE_F32, DTYPE_BF16, DTYPE_F8E4M3, DTYPE_I4 = 0, 1, 2, 3   # (e4m3 and 4 bits: of a KvCache)
STATUS = {0: "CDSL_OK", 1: "CDSL_EINVAL", 2: "CDSL_ENOMEM", 3: "CDSL_ECUDA", 4: "CDSL_ETIMEOUT",
          5: "CDSL_ENONFINITE", 6: "CDSL_ESTATE", 7: "CDSL_ERANGE"}
(CDSL_OK, CDSL_EINVAL, CDSL_ENOMEM, CDSL_ECUDA, CDSL_ETIMEOUT, CDSL_ENONFINITE, CDSL_ESTATE,
 CDSL_ERANGE) = range(8)
S1, S2_S3, S4 = 1, 2, 4
TREE_MAX_NODES, TREE_MAX_BATCH, TREE_MAX_VOCAB = 128, 1024, 1 << 20


class CdslError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class ModelCfg(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("norm_eps", ctypes.c_float)]


class RunCfg(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("k", ctypes.c_int32), ("d", ctypes.c_int32),
                ("max_prompt", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("n_keywords", ctypes.c_int32), ("a_t", ctypes.c_float), ("r_t", ctypes.c_float),
                ("reward_head", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_chunk", ctypes.c_int32), ("acceptance", ctypes.c_int32),
                ("seed", ctypes.c_uint32), ("step1_budget", ctypes.c_int32)]


_P = ctypes.c_void_p
_I = ctypes.c_int32
EXPORTS = {
    "cdsl_num_weights": (_I, [ctypes.POINTER(ModelCfg)]),
    "cdsl_workspace_size": (_I, [ctypes.POINTER(ModelCfg), ctypes.POINTER(ModelCfg),
                                 ctypes.POINTER(RunCfg), ctypes.POINTER(ctypes.c_size_t)]),
    "cdsl_init": (_I, [ctypes.POINTER(ModelCfg), ctypes.POINTER(_P), ctypes.POINTER(ModelCfg),
                       ctypes.POINTER(_P), ctypes.POINTER(RunCfg), _P, _P, ctypes.c_size_t, _P,
                       ctypes.POINTER(_P)]),
    "cdsl_prefill": (_I, [_P, _P, ctypes.POINTER(ctypes.c_int32), _P]),
    "cdsl_lookahead": (_I, [_P, _P, _P, _P]),
    "cdsl_verify": (_I, [_P, _P, _P, _P, _P]),
    "cdsl_select": (_I, [_P, _P, _P, _P, _P, _P]),
    "cdsl_step": (_I, [_P, _P, _P, _P, _P, _P]),
    "cdsl_get_tokens": (_I, [_P, _P, _P]),
    "cdsl_get_counters": (_I, [_P, ctypes.POINTER(ctypes.c_int64)]),
    "cdsl_get_step1": (_I, [_P, _P, _P, _P]),
    "cdsl_get_status": (_I, [_P, ctypes.POINTER(ctypes.c_int32)]),
    "cdsl_profile": (_I, [_P, _I]),
    "cdsl_get_profile": (_I, [_P, _I, ctypes.POINTER(ctypes.c_double)]),
    "cdsl_get_profile_launches": (_I, [_P, ctypes.POINTER(ctypes.c_double), _I]),
    "cdsl_gemv_noalloc": (_I, [_P, _I, _I, _P, _I, _P, _P]),
    "cdsl_set_wait_limit": (_I, [_P, ctypes.c_uint64]),
    "cdsl_kv_write": (_I, [_P, _I, _P, _P, _I, _I, _P, _P, _P, _P, _P]),
    "cdsl_kv_read": (_I, [_P, _I, _I, _P, _P, _I, _I, _P, _P, _P, _P]),
    "cdsl_kv_commit": (_I, [_P, _P, _P, _P, _I, _P, _P, _P]),
    "cdsl_tree_mask": (_I, [_P, _I, _P, _P]),
    "cdsl_tree_attention_workspace": (_I, [_P, _I, _I, _P]),
    "cdsl_tree_attention": (_I, [_P, _I, _P, _I, _I, _I, _P, _P, _P, _P, ctypes.c_float, _I, _P, _P, _P,
                                 ctypes.c_size_t, _P, _P]),
    "cdsl_tree_verify": (_I, [_I, _I, _I, _P, _P, _I, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P,
                              _P, _P]),
    "cdsl_kv_pages_workspace": (_I, [_P, _I, _P]),
    "cdsl_kv_fork": (_I, [_P, _P, _P, _P, _I, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "cdsl_kv_resize": (_I, [_P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "cdsl_kv_compact": (_I, [_P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "cdsl_rope_turns": (_I, [_I, ctypes.c_double, ctypes.c_double, _I, ctypes.c_double, ctypes.c_double, _P]),
    "cdsl_rope": (_I, [_P, _I, _P, _P, _P, _P, _P, _P, _P, _P]),
    "cdsl_last_error": (ctypes.c_char_p, [_P]),
    "cdsl_destroy": (None, [_P]),
}


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(
            f"CUDA library {path} is missing: build it with "
            "`python -m paper_2412_10418_gb300.build` (there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    for name, (res, args) in EXPORTS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _check(code: int, ctx=None):
    if code:
        msg = lib().cdsl_last_error(ctx)
        raise CdslError(code, msg.decode() if msg else "")


def model_cfg(shape, dtype) -> ModelCfg:
    """ctypes config from any object with the decoder's shape attributes."""
    dt = dtype if isinstance(dtype, int) else (DTYPE_BF16 if dtype == "bf16" else DTYPE_F32)
    return ModelCfg(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads,
                    shape.head_dim, shape.d_ffn, shape.vocab, dt, shape.rope_theta,
                    shape.norm_eps)


ACCEPT_HARD, ACCEPT_SPECULATIVE = 0, 1


def run_cfg(batch, k, d, max_prompt, max_new, n_keywords, a_t, r_t, reward_head,
            page_size=0, max_chunk=0, acceptance=ACCEPT_HARD, seed=0, step1_budget=0) -> RunCfg:
    return RunCfg(batch, k, d, max_prompt, max_new, n_keywords, a_t, r_t, int(reward_head),
                  page_size, max_chunk, int(acceptance), int(seed) & 0xFFFFFFFF,
                  int(step1_budget))


# ------------------------------------------------------------------------------ C names

def cdsl_num_weights(cfg: ModelCfg) -> int:
    return lib().cdsl_num_weights(ctypes.byref(cfg))


def cdsl_workspace_size(tcfg: ModelCfg, dcfg: ModelCfg, run: RunCfg) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().cdsl_workspace_size(ctypes.byref(tcfg), ctypes.byref(dcfg), ctypes.byref(run),
                                     ctypes.byref(n)))
    return n.value


def cdsl_init(tcfg, t_weights: Sequence, dcfg, d_weights: Sequence, run, reward_head,
              workspace, stream) -> int:
    tw = (_P * len(t_weights))(*[w.data_ptr() for w in t_weights])
    dw = (_P * len(d_weights))(*[w.data_ptr() for w in d_weights])
    ctx = _P(0)
    _check(lib().cdsl_init(ctypes.byref(tcfg), tw, ctypes.byref(dcfg), dw, ctypes.byref(run),
                           _ptr(reward_head), workspace.data_ptr(), workspace.numel(),
                           stream, ctypes.byref(ctx)))
    return ctx.value


def cdsl_prefill(ctx, prompts, prompt_lens: Sequence[int], keywords):
    lens = (ctypes.c_int32 * len(prompt_lens))(*[int(x) for x in prompt_lens])
    _check(lib().cdsl_prefill(ctx, prompts.data_ptr(), lens, keywords.data_ptr()), ctx)


def cdsl_lookahead(ctx, roots=None, draft_tok=None, logq=None):
    _check(lib().cdsl_lookahead(ctx, _ptr(roots), _ptr(draft_tok), _ptr(logq)), ctx)


def cdsl_verify(ctx, logp=None, argmax=None, n_accept=None, logits=None):
    _check(lib().cdsl_verify(ctx, _ptr(logp), _ptr(argmax), _ptr(n_accept), _ptr(logits)), ctx)


def cdsl_select(ctx, beam=None, state=None, emitted=None, n_emitted=None, reward=None):
    _check(lib().cdsl_select(ctx, _ptr(beam), _ptr(state), _ptr(emitted), _ptr(n_emitted),
                             _ptr(reward)), ctx)


def cdsl_step(ctx, beam=None, state=None, emitted=None, n_emitted=None, reward=None):
    _check(lib().cdsl_step(ctx, _ptr(beam), _ptr(state), _ptr(emitted), _ptr(n_emitted),
                           _ptr(reward)), ctx)


def cdsl_get_tokens(ctx, tokens=None, lengths=None):
    _check(lib().cdsl_get_tokens(ctx, _ptr(tokens), _ptr(lengths)), ctx)


def cdsl_get_counters(ctx) -> List[int]:
    out = (ctypes.c_int64 * 8)()
    _check(lib().cdsl_get_counters(ctx, out), ctx)
    return list(out)


def cdsl_get_step1(ctx, need=None, tokens=None, reward=None):
    _check(lib().cdsl_get_step1(ctx, _ptr(need), _ptr(tokens), _ptr(reward)), ctx)


def cdsl_set_wait_limit(ctx, ns: int):
    """Limit (nanoseconds) of the tensor-core kernels' bounded waits; see include/cdsl.h."""
    _check(lib().cdsl_set_wait_limit(ctx, int(ns)), ctx)


def cdsl_get_status(ctx) -> int:
    v = ctypes.c_int32(0)
    _check(lib().cdsl_get_status(ctx, ctypes.byref(v)), ctx)
    return v.value


PROFILE_OFF, PROFILE_EVENTS, PROFILE_IN_GRAPH = 0, 1, 2


def cdsl_profile(ctx, mode):
    """mode 0 off, 1 CUDA events around direct launches, 2 in-graph stamps (see cdsl.h);
    True / False stand for 1 / 0."""
    _check(lib().cdsl_profile(ctx, int(mode)), ctx)


GEMM_IMPLS = {0: "gemm_simt", 1: "gemv_stream", 2: "gemm_tc"}
KERNEL_CLASSES = {0: "gemm_simt", 1: "gemv_stream", 2: "gemm_tc", 3: "attention", 4: "rmsnorm",
                  5: "row_stats", 6: "embed", 7: "step_logic"}
STAMPED_STEPS = 8   # cdsl_get_profile class of the stamped steps themselves (mode 2)


def cdsl_get_profile(ctx, impl: int):
    out = (ctypes.c_double * 4)()
    _check(lib().cdsl_get_profile(ctx, impl, out), ctx)
    return dict(launches=int(out[0]), ms=out[1], bytes=out[2], flops=out[3])


def cdsl_get_profile_launches(ctx, capacity: int = 8192):
    """Per-launch timing records [(class, ms, bytes, flops)] in launch order."""
    out = (ctypes.c_double * (4 * capacity))()
    n = lib().cdsl_get_profile_launches(ctx, out, capacity)
    if n < 0:
        raise CdslError(-n, cdsl_last_error(ctx))
    return [(int(out[4 * i]), out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]) for i in range(n)]


def cdsl_gemv_noalloc(w, x, y, stream=None):
    """y[R, N] = x[R, K] w^T in one weight-streaming kernel that needs no scratch in global
    memory (no device memory is allocated); see include/cdsl.h.

    The C ABI sees only pointers and sizes, so the shapes, dtypes, layouts and devices are
    checked here: w bfloat16 [N, K], x float32 [R, K], y float32 [R, N], all contiguous and on
    the current CUDA device. Anything else raises CdslError(CDSL_EINVAL) before the call."""
    import torch

    def bad(why):
        raise CdslError(CDSL_EINVAL, "cdsl_gemv_noalloc: " + why)

    ts = (w, x, y)
    if not all(isinstance(t, torch.Tensor) for t in ts):
        bad("w, x and y must be torch tensors")
    if w.dtype != torch.bfloat16 or x.dtype != torch.float32 or y.dtype != torch.float32:
        bad("w must be bfloat16, x and y float32")
    if w.dim() != 2 or x.dim() != 2 or y.dim() != 2:
        bad("w, x and y must be 2-D")
    N, K = w.shape
    R = x.shape[0]
    if tuple(x.shape) != (R, K) or tuple(y.shape) != (R, N):
        bad(f"shapes: w {tuple(w.shape)}, x {tuple(x.shape)}, y {tuple(y.shape)} "
            "(want [N, K], [R, K], [R, N])")
    if not all(t.is_contiguous() for t in ts):
        bad("w, x and y must be contiguous")
    dev = torch.cuda.current_device() if torch.cuda.is_available() else None
    if not all(t.is_cuda and t.device.index == dev for t in ts):
        bad("w, x and y must be on the current CUDA device")
    _check(lib().cdsl_gemv_noalloc(w.data_ptr(), N, K, x.data_ptr(), R, y.data_ptr(), stream))


def cdsl_last_error(ctx=None) -> str:
    m = lib().cdsl_last_error(ctx)
    return m.decode() if m else ""


def cdsl_destroy(ctx):
    lib().cdsl_destroy(ctx)


# ------------------------------------------------------------------------------ tree speculation
# The C ABI sees pointers, sizes and strides; types, shapes, layouts and devices are checked here, and
# anything the calls cannot take raises CdslError(CDSL_EINVAL) before a call, tensors of a device that is not the
# current one among it. `stream` is a cudaStream_t as an integer, None the current torch stream. Semantics:
# include/cdsl_tree.h.

class _KvCacheC(ctypes.Structure):
    _fields_ = [("d_pool", _P), ("d_scale", _P), ("d_page_table", _P), ("n_layers", _I), ("n_pages", _I),
                ("n_kv_heads", _I), ("page_size", _I), ("head_dim", _I), ("dtype", _I), ("batch", _I),
                ("max_pages", _I)]


class _Types:
    """torch and its types that the bindings compare with (torch is imported on first use)."""

    def __init__(self):
        import torch

        self.torch = torch
        self.i32, self.f32, self.bf16, self.u8 = torch.int32, torch.float32, torch.bfloat16, torch.uint8
        self.i64 = torch.int64
        self.values = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}
        self.devices = None                    # how many (asked at the first launch)
        self.caches = {torch.float8_e4m3fn: DTYPE_F8E4M3, torch.bfloat16: DTYPE_BF16, torch.uint8: DTYPE_I4}


_types: Optional[_Types] = None


def _torch() -> _Types:
    global _types
    if _types is None:
        _types = _Types()
    return _types


def _bad(fn: str, why: str):
    raise CdslError(CDSL_EINVAL, f"{fn}: {why}")


def _ints(fn: str, name: str, t, shape, device, dtype=None):
    """A contiguous int32 (or `dtype`) tensor of this shape on this device: its pointer."""
    if t.dtype is (dtype or _types.i32) and t.shape == shape and t.is_contiguous() and t.device == device:
        return t.data_ptr()
    _bad(fn, f"{name} must be a contiguous {dtype or _types.i32} tensor {tuple(shape)} on {device}, got "
             f"{t.dtype} {tuple(t.shape)} on {t.device}")


def _stream(fn: str, device, stream):
    """The stream of a launch (None: the current one). Launches go to the current device, which must be the tensors'.
    (Asking which it is takes 1 to 2 us a call; with one device there is no other.)"""
    cuda = _types.torch.cuda
    if _types.devices is None:
        _types.devices = cuda.device_count()
    if _types.devices > 1 and cuda.current_device() != device.index:
        _bad(fn, f"the tensors are on {device}, the current device is cuda:{cuda.current_device()}")
    return cuda.current_stream(device).cuda_stream if stream is None else stream


class KvCache:
    """A paged K/V cache in e4m3, bfloat16 or 4 bits: ``pool`` [layers, pages, 2, kv_heads, page_size, head_dim] of
    torch.float8_e4m3fn or torch.bfloat16, ``scale`` [layers, pages, 2, kv_heads, page_size] uint8 (a row's
    values are code * 2^(byte - 127)) and ``page_table`` [batch, max_pages] int32, all contiguous on one CUDA
    device. In 4 bits: ``pool`` [.., head_dim / 2] uint8 and ``scale`` [.., page_size, head_dim / 32] bfloat16. The tensors are the caller's; the object keeps them referenced. ``cache.at(page_table)`` is
    the same pool under another table (another set of sequences)."""

    def __init__(self, pool, scale, page_table):
        ty = _torch()
        if not pool.is_cuda:
            _bad("KvCache", "pool must be on a CUDA device")
        if pool.dim() != 6 or pool.shape[2] != 2 or not pool.is_contiguous() or pool.dtype not in ty.caches:
            _bad("KvCache", "pool must be a contiguous float8_e4m3fn or bfloat16 tensor [layers, pages, 2, "
                            "kv_heads, page_size, head_dim], or uint8 of head_dim / 2 bytes")
        L, N, _, H, P, D = pool.shape
        if pool.dtype is ty.u8:
            D *= 2
            _ints("KvCache", "scale", scale, pool.shape[:5] + (D // 32,), pool.device, ty.bf16)
        else:
            _ints("KvCache", "scale", scale, pool.shape[:5], pool.device, ty.u8)
        if page_table.dim() != 2:
            _bad("KvCache", "page_table must be [batch, max_pages]")
        _ints("KvCache", "page_table", page_table, page_table.shape, pool.device)
        self.pool, self.scale, self.page_table, self.device = pool, scale, page_table, pool.device
        self.batch, self.n_layers, self.n_kv_heads, self.head_dim = page_table.shape[0], L, H, D
        self.n_pages, self.max_pages = N, page_table.shape[1]
        self._c = _KvCacheC(pool.data_ptr(), scale.data_ptr(), page_table.data_ptr(), L, N, H, P, D,
                            ty.caches[pool.dtype], page_table.shape[0], page_table.shape[1])
        self._ref = ctypes.addressof(self._c)
        self._one, self._pages = ty.torch.Size((self.batch,)), ty.torch.Size((N,))

    @classmethod
    def empty(cls, n_layers, n_pages, n_kv_heads, page_size, head_dim, page_table, dtype=None):
        """A cache with memory of its own (dtype: torch.float8_e4m3fn, the default, torch.bfloat16, or torch.uint8 for 4
        bits)."""
        t = _torch().torch
        if dtype is t.uint8:
            shape = (n_layers, n_pages, 2, n_kv_heads, page_size)
            dev = page_table.device
            return cls(t.empty(shape + (head_dim // 2,), dtype=t.uint8, device=dev),
                       t.empty(shape + (head_dim // 32,), dtype=t.bfloat16, device=dev), page_table)
        pool = t.empty((n_layers, n_pages, 2, n_kv_heads, page_size, head_dim), dtype=dtype or t.float8_e4m3fn,
                       device=page_table.device)
        return cls(pool, t.empty(pool.shape[:5], dtype=t.uint8, device=page_table.device), page_table)

    def at(self, page_table):
        return KvCache(self.pool, self.scale, page_table)


def _rows(fn, cache, names, x, y, heads):
    """Two tensors [batch, T, heads, head_dim] of one type with a contiguous last dimension: (type code, T, both
    tensors' strides)."""
    code = _types.values.get(x.dtype)
    s = x.shape
    dev = cache.device
    if (code is None or len(s) != 4 or s[0] != cache.batch or s[2] != heads or s[3] != cache.head_dim
            or y.dtype is not x.dtype or y.shape != s or x.device != dev or y.device != dev):
        _bad(fn, f"{names} must be float32 or bfloat16 tensors [{cache.batch}, T, {heads}, {cache.head_dim}] of one type "
                 f"on {dev}, got {x.dtype} {tuple(s)} on {x.device} and {y.dtype} {tuple(y.shape)} on {y.device}")
    if x.is_contiguous() and y.is_contiguous():   # (by size: a decoding loop repeats a few)
        st = _contiguous.get(s)
        if st is None:
            if len(_contiguous) >= 256:
                _contiguous.clear()
            t = heads * cache.head_dim
            st = _contiguous[s] = _Strides6(*(s[1] * t, t, cache.head_dim) * 2)
        return code, s[1], st
    sx, sy = x.stride(), y.stride()
    if sx[3] != 1 or sy[3] != 1:
        _bad(fn, f"{names} must have a contiguous last dimension, got strides {tuple(sx)} and {tuple(sy)}")
    return code, s[1], _Strides6(*sx[:3], *sy[:3])


_Strides6 = ctypes.c_int64 * 6
_contiguous: dict = {}
_Strides4 = ctypes.c_int64 * 4


def cdsl_kv_write(cache: KvCache, layer: int, k, v, start, count=None, status=None, stream=None):
    """Rows k, v [batch, T, kv_heads, head_dim] (float32 or bfloat16, any strides but the last) into slots
    start[b] + i of the layer, i < count[b] (None: all)."""
    fn = "cdsl_kv_write"
    code, T, st = _rows(fn, cache, "k and v", k, v, cache.n_kv_heads)
    _check(lib().cdsl_kv_write(cache._ref, layer, k.data_ptr(), v.data_ptr(), code, T, st,
                               _ints(fn, "start", start, cache._one, cache.device),
                               None if count is None else _ints(fn, "count", count, cache._one, cache.device),
                               None if status is None else _ints(fn, "status", status, (1,), cache.device),
                               _stream(fn, cache.device, stream)))


def cdsl_kv_read(cache: KvCache, layer: int, start, k, v, count=None, status=None, stream=None):
    """Slots start[b] + i of layers layer .. layer + n - 1 back as values into k, v [n, batch, T, kv_heads,
    head_dim] (contiguous, float32 or bfloat16); rows i >= count[b] become zeros."""
    fn = "cdsl_kv_read"
    code = _types.values.get(k.dtype)
    s = k.shape
    if (code is None or len(s) != 5 or s[1] != cache.batch or s[3] != cache.n_kv_heads or s[4] != cache.head_dim
            or v.shape != s or v.dtype is not k.dtype or not k.is_contiguous() or not v.is_contiguous()
            or k.device != cache.device or v.device != cache.device):
        _bad(fn, f"k and v must be contiguous float32 or bfloat16 tensors [n_layers, {cache.batch}, T, "
                 f"{cache.n_kv_heads}, {cache.head_dim}] on {cache.device}")
    _check(lib().cdsl_kv_read(cache._ref, layer, s[0], k.data_ptr(), v.data_ptr(), code, s[2],
                              _ints(fn, "start", start, cache._one, cache.device),
                              None if count is None else _ints(fn, "count", count, cache._one, cache.device),
                              None if status is None else _ints(fn, "status", status, (1,), cache.device),
                              _stream(fn, cache.device, stream)))


def cdsl_kv_commit(cache: KvCache, lens, path, n_path, new_lens=None, status=None, stream=None):
    """The taken paths' rows of every layer to their places: slot lens[b] + path[b, i] to lens[b] + i; new_lens
    [batch] becomes lens + n_path."""
    fn = "cdsl_kv_commit"
    if path.dim() != 2:
        _bad(fn, "path must be [batch, T]")
    T = path.shape[1]
    _check(lib().cdsl_kv_commit(cache._ref, _ints(fn, "lens", lens, cache._one, cache.device),
                                _ints(fn, "path", path, (cache.batch, T), cache.device),
                                _ints(fn, "n_path", n_path, cache._one, cache.device), T,
                                None if new_lens is None else _ints(fn, "new_lens", new_lens, cache._one, cache.device),
                                None if status is None else _ints(fn, "status", status, (1,), cache.device),
                                _stream(fn, cache.device, stream)))


def cdsl_kv_pages_workspace(cache: KvCache, new_batch: Optional[int] = None) -> int:
    """Bytes of workspace that cdsl_kv_fork to new_batch sequences (None: as many as the cache has), cdsl_kv_resize and
    cdsl_kv_compact need."""
    n = ctypes.c_size_t(0)
    _check(lib().cdsl_kv_pages_workspace(cache._ref, cache.batch if new_batch is None else new_batch, ctypes.byref(n)))
    return n.value


def _workspace(fn, workspace, dev):
    if workspace.dtype is not _types.u8 or not workspace.is_contiguous() or workspace.device != dev:
        _bad(fn, f"workspace must be a contiguous uint8 tensor on {dev}")
    return workspace.data_ptr(), workspace.numel()


def cdsl_kv_fork(cache: KvCache, refs, src, lens, new_table, new_lens, new_refs, workspace, status=None, stream=None):
    """New sequence i goes on from the lens[src[i]] cached tokens of the cache's sequence src[i]: new_table [new_batch,
    max_pages], new_lens [new_batch] and the pages' numbers of holders new_refs [n_pages] from refs [n_pages]; partly filled last
    pages are copied for all successors of a sequence but the first. All int32. ``cache.at(new_table)`` is the cache after
    it."""
    fn = "cdsl_kv_fork"
    if src.dim() != 1:
        _bad(fn, "src must be [new_batch]")
    new, dev = src.shape[0], cache.device
    _check(lib().cdsl_kv_fork(
        cache._ref, _ints(fn, "refs", refs, cache._pages, dev), _ints(fn, "src", src, (new,), dev),
        _ints(fn, "lens", lens, cache._one, dev), new, _ints(fn, "new_table", new_table, (new, cache.max_pages), dev),
        _ints(fn, "new_lens", new_lens, (new,), dev), _ints(fn, "new_refs", new_refs, cache._pages, dev),
        *_workspace(fn, workspace, dev), None if status is None else _ints(fn, "status", status, (1,), dev),
        _stream(fn, dev, stream)))


def cdsl_kv_resize(cache: KvCache, refs, slots, new_table, new_refs, workspace, status=None, stream=None):
    """Sequence b has the pages of its first slots[b] slots afterwards: those behind are given back, missing ones dealt
    from the free ones (refs 0), lowest first. A page that the last slot lies in stays even if others hold it: to go back to
    a length inside a shared page, fork with that length. new_table and new_refs may be cache.page_table and refs."""
    fn = "cdsl_kv_resize"
    dev = cache.device
    _check(lib().cdsl_kv_resize(
        cache._ref, _ints(fn, "refs", refs, cache._pages, dev), _ints(fn, "slots", slots, cache._one, dev),
        _ints(fn, "new_table", new_table, cache.page_table.shape, dev), _ints(fn, "new_refs", new_refs, cache._pages, dev),
        *_workspace(fn, workspace, dev), None if status is None else _ints(fn, "status", status, (1,), dev),
        _stream(fn, dev, stream)))


def cdsl_kv_compact(cache: KvCache, refs, new_table, new_refs, page_map, n_live, workspace, status=None, stream=None):
    """The pages in use (refs > 0) move to the front of the pool, in every layer: n_live [1] how many there are, page_map
    [n_pages] each page's new place (-1: free). new_table and new_refs may be cache.page_table and refs."""
    fn = "cdsl_kv_compact"
    dev = cache.device
    _check(lib().cdsl_kv_compact(
        cache._ref, _ints(fn, "refs", refs, cache._pages, dev),
        _ints(fn, "new_table", new_table, cache.page_table.shape, dev), _ints(fn, "new_refs", new_refs, cache._pages, dev),
        _ints(fn, "page_map", page_map, cache._pages, dev), _ints(fn, "n_live", n_live, (1,), dev),
        *_workspace(fn, workspace, dev), None if status is None else _ints(fn, "status", status, (1,), dev),
        _stream(fn, dev, stream)))


class Rope:
    """Rotary positions of heads' first `rot` dimensions, for cdsl_rope. Pairs are i and i + rot / 2, or 2 i and 2 i + 1
    (`interleaved`). `factor` != 1 scales positions by parts for contexts longer than `original_len`: dimensions that turn
    fewer than `low` times over it go `factor` times slower, those that turn more than `high` times as before;
    `magnitude` multiplies what is turned."""

    def __init__(self, rot: int, *, theta: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
                 original_len: int = 0, low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, device="cuda"):
        t = _torch().torch
        turns = t.zeros(max(1, rot // 2), dtype=t.int64)
        _check(lib().cdsl_rope_turns(rot, theta, factor, original_len, low, high, turns.data_ptr()))
        if not 0.0 < magnitude < float("inf"):
            _bad("Rope", "magnitude must be positive and finite")
        self.rot, self.interleaved, self.magnitude = rot, int(bool(interleaved)), magnitude
        self.turns = turns.to(device)
        self.device = self.turns.device
        self._c = _RopeC(self.turns.data_ptr(), rot, self.interleaved, magnitude)
        self._ref = ctypes.addressof(self._c)


class _RopeC(ctypes.Structure):
    _fields_ = [("d_turns", _P), ("rot", _I), ("interleaved", _I), ("magnitude", ctypes.c_float)]


class _RopeRows(ctypes.Structure):
    _fields_ = [("dtype", _I), ("batch", _I), ("T", _I), ("head_dim", _I), ("n_heads", _I), ("n_kv_heads", _I),
                ("strides", ctypes.c_int64 * 12)]


_rope_rows: dict = {}


def cdsl_rope(rope: Rope, q, q_out, start, *, k=None, k_out=None, offset=None, inverse: bool = False, stream=None):
    """q (and k) [batch, T, heads, head_dim] turned by their positions start[b] + offset[b, t] (offset None: t) into q_out
    (and k_out), which may be the same tensors; any strides but the last. inverse: turned back, which takes gradients of the
    outputs to those of the inputs. (Outputs are written as memory: autograd records nothing, and a training program has
    both directions in a function of its own.)"""
    fn = "cdsl_rope"
    dt, s, dev = q.dtype, q.shape, rope.device
    code = _types.values.get(dt)
    ok = (code is not None and len(s) == 4 and q_out.dtype is dt and q_out.shape == s and q.device == dev
          and q_out.device == dev and (k is None) is (k_out is None))
    sk = None
    if ok and k is not None:
        sk = k.shape
        ok = (len(sk) == 4 and sk[0] == s[0] and sk[1] == s[1] and sk[3] == s[3] and k.dtype is dt and k_out.dtype is dt
              and k_out.shape == sk and k.device == dev and k_out.device == dev)
    if not ok:
        _bad(fn, f"q, k (with k_out, or neither) and their outputs must be float32 or bfloat16 tensors [batch, T, heads, "
                 f"head_dim] of one type on {dev}, got " +
                 ", ".join(f"{x.dtype} {tuple(x.shape)} on {x.device}" for x in (q, q_out, k, k_out) if x is not None))
    B, T, H, D = s
    if q.is_contiguous() and q_out.is_contiguous() and (k is None or k.is_contiguous() and k_out.is_contiguous()):
        key = (dt, s, sk)                      # (a decoding loop repeats a few)
        rows = _rope_rows.get(key)
        if rows is None:
            if len(_rope_rows) >= 256:
                _rope_rows.clear()
            K = 0 if k is None else sk[2]
            rows = _rope_rows[key] = _RopeRows(code, B, T, D, H, K, (ctypes.c_int64 * 12)(
                *(T * H * D, H * D, D) * 2, *(T * K * D, K * D, D) * 2))
    else:
        tensors = (q, q_out) if k is None else (q, q_out, k, k_out)
        strides = [x.stride() for x in tensors]
        if any(st[3] != 1 for st in strides):
            _bad(fn, f"q, k and their outputs must have a contiguous last dimension, got strides {strides}")
        rows = _RopeRows(code, B, T, D, H, 0 if k is None else sk[2],
                         (ctypes.c_int64 * 12)(*(n for st in strides for n in st[:3])))
    _check(lib().cdsl_rope(
        rope._ref, inverse, ctypes.addressof(rows), q.data_ptr(), q_out.data_ptr(), None if k is None else k.data_ptr(),
        None if k is None else k_out.data_ptr(), _ints(fn, "start", start, (B,), dev),
        None if offset is None else _ints(fn, "offset", offset, (B, T), dev), _stream(fn, dev, stream)))


def cdsl_tree_mask(parents: Sequence[int]):
    """(mask, depth) of a tree on the host: mask a CPU int32 tensor [T, (T + 31) // 32] of ancestor bits,
    depth [T] each node's number of ancestors. parents[i] < i; parents[0] is ignored."""
    t = _torch().torch
    T = len(parents)
    p = (ctypes.c_int32 * T)(*[int(x) for x in parents])
    mask = t.zeros((T, (T + 31) // 32), dtype=t.int32)
    depth = t.zeros(T, dtype=t.int32)
    _check(lib().cdsl_tree_mask(p, T, mask.data_ptr(), depth.data_ptr()))
    return mask, depth


def cdsl_tree_attention_workspace(cache: KvCache, T: int, n_heads: int) -> int:
    """Bytes of workspace that cdsl_tree_attention needs for trees of up to T nodes."""
    n = ctypes.c_size_t(0)
    _check(lib().cdsl_tree_attention_workspace(cache._ref, n_heads, T, ctypes.byref(n)))
    return n.value


def cdsl_tree_attention(cache: KvCache, layer: int, q, lens, mask, out, workspace, *, scale: float, max_len: int,
                        nodes=None, lse=None, status=None, stream=None):
    """Attention of each sequence's tree of T nodes, q and out [batch, T, n_heads, head_dim] (one type, any
    strides but the last), over its lens[b] cached slots and the tree's own after them, by the ancestor bits of
    mask [batch, T, (T + 31) // 32]."""
    fn = "cdsl_tree_attention"
    H = q.shape[2] if q.dim() == 4 else 0
    code, T, st = _rows(fn, cache, "q and out", q, out, H)
    dev = cache.device
    if workspace.dtype is not _types.u8 or not workspace.is_contiguous() or workspace.device != dev:
        _bad(fn, f"workspace must be a contiguous uint8 tensor on {dev}")
    _check(lib().cdsl_tree_attention(
        cache._ref, layer, q.data_ptr(), code, H, T, st, _ints(fn, "lens", lens, cache._one, dev),
        None if nodes is None else _ints(fn, "nodes", nodes, cache._one, dev),
        _ints(fn, "mask", mask, (cache.batch, T, (T + 31) // 32), dev), scale, max_len, out.data_ptr(),
        None if lse is None else _ints(fn, "lse", lse, (cache.batch, T, H), dev, _types.f32), workspace.data_ptr(), workspace.numel(),
        None if status is None else _ints(fn, "status", status, (1,), dev), _stream(fn, dev, stream)))


def cdsl_tree_verify(logits, tokens, parents, u, u_last, path, n_path, emitted, *, draft_logits=None,
                     temperature: float = 1.0, nodes=None, status=None, stream=None):
    """Which path of each sequence's tree the target takes, and the next token: logits (and draft_logits)
    [batch, T, vocab] float32 or bfloat16 with a contiguous last dimension; tokens, parents, path, emitted
    [batch, T] and n_path, nodes [batch] int32; u [batch, T] and u_last [batch] float32 in [0, 1)."""
    ty = _torch()
    fn = "cdsl_tree_verify"
    code = ty.values.get(logits.dtype)
    if code is None or logits.dim() != 3 or not logits.is_cuda or logits.stride(2) != 1:
        _bad(fn, "logits must be a CUDA float32 or bfloat16 tensor [batch, T, vocab] with a contiguous last dimension")
    B, T, V = logits.shape
    dev = logits.device
    st = logits.stride()
    sd = st
    if draft_logits is not None:
        sd = draft_logits.stride()
        if (draft_logits.dtype is not logits.dtype or draft_logits.shape != logits.shape or sd[2] != 1
                or draft_logits.device != dev):
            _bad(fn, "draft_logits must be like logits")
    one, all_ = (B,), (B, T)
    _check(lib().cdsl_tree_verify(
        B, T, V, logits.data_ptr(), _ptr(draft_logits), code, _Strides4(st[0], st[1], sd[0], sd[1]),
        _ints(fn, "tokens", tokens, all_, dev), _ints(fn, "parents", parents, all_, dev),
        None if nodes is None else _ints(fn, "nodes", nodes, one, dev), _ints(fn, "u", u, all_, dev, ty.f32),
        _ints(fn, "u_last", u_last, one, dev, ty.f32), temperature, _ints(fn, "path", path, all_, dev),
        _ints(fn, "n_path", n_path, one, dev), _ints(fn, "emitted", emitted, all_, dev),
        None if status is None else _ints(fn, "status", status, (1,), dev), _stream(fn, dev, stream)))


# ------------------------------------------------------------------------------ Engine

class Engine:
    """A context plus its workspace and per-step output tensors (all on one CUDA device).

    target_weights / draft_weights: torch tensors in the C ABI order (cdsl_num_weights of
    them), kept referenced for the engine's lifetime."""

    def __init__(self, target_shape, draft_shape, dtype, target_weights, draft_weights, *,
                 batch, k, d, max_prompt, max_new, n_keywords, a_t, r_t, reward_head=None,
                 page_size=0, max_chunk=0, acceptance=ACCEPT_HARD, seed=0, step1_budget=0,
                 stream=None, device="cuda"):
        import torch

        self.torch = torch
        self.tcfg = model_cfg(target_shape, dtype)
        self.dcfg = model_cfg(draft_shape, dtype)
        self.run = run_cfg(batch, k, d, max_prompt, max_new, n_keywords, a_t, r_t,
                           reward_head is not None, page_size, max_chunk, acceptance, seed,
                           step1_budget)
        self.B, self.k, self.d, self.V = batch, k, d, target_shape.vocab
        self.max_prompt, self.max_new = max_prompt, max_new
        self.tw, self.dw = list(target_weights), list(draft_weights)
        self.head = reward_head
        self.stream = stream if stream is not None else torch.cuda.Stream(device=device)
        nbytes = cdsl_workspace_size(self.tcfg, self.dcfg, self.run)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.ctx = cdsl_init(self.tcfg, self.tw, self.dcfg, self.dw, self.run, self.head, self.ws,
                             self.stream.cuda_stream)
        i32, f32 = torch.int32, torch.float32
        B, K, D = batch, k, d
        z = lambda *s, dt=i32: torch.zeros(s, dtype=dt, device=device)
        self.roots, self.draft_tok, self.logq = z(B, K), z(B, K, D), z(B, K, D, dt=f32)
        self.logp, self.argmax, self.n_accept = z(B, K, D, dt=f32), z(B, K, D + 1), z(B, K)
        self.beam, self.state, self.emitted = z(B), z(B), z(B, D + 1)
        self.n_emitted, self.reward = z(B), z(B, K, 2, dt=f32)

    def prefill(self, prompts, prompt_lens, keywords):
        with self.torch.cuda.stream(self.stream):
            self._prompts = prompts.to(self.ws.device, self.torch.int32).contiguous()
            self._kw = keywords.to(self.ws.device, self.torch.int32).contiguous()
        self.stream.synchronize()
        cdsl_prefill(self.ctx, self._prompts, prompt_lens, self._kw)

    def lookahead(self):
        cdsl_lookahead(self.ctx, self.roots, self.draft_tok, self.logq)

    def verify(self, logits=None):
        cdsl_verify(self.ctx, self.logp, self.argmax, self.n_accept, logits)

    def select(self):
        cdsl_select(self.ctx, self.beam, self.state, self.emitted, self.n_emitted, self.reward)

    def step(self):
        cdsl_step(self.ctx, self.beam, self.state, self.emitted, self.n_emitted, self.reward)

    def tokens(self):
        t = self.torch.empty((self.B, self.max_prompt + self.max_new), dtype=self.torch.int32,
                             device=self.ws.device)
        n = self.torch.empty(self.B, dtype=self.torch.int32, device=self.ws.device)
        cdsl_get_tokens(self.ctx, t, n)
        self.stream.synchronize()
        return t, n

    def step1(self):
        """Step-1 round 2 of the last select / step (budget 2): need [B], tokens [B, d+1]
        (x', lh_1..lh_d), reward [B]."""
        t = self.torch
        need = t.zeros(self.B, dtype=t.int32, device=self.ws.device)
        tok = t.zeros((self.B, self.d + 1), dtype=t.int32, device=self.ws.device)
        rew = t.zeros(self.B, dtype=t.float32, device=self.ws.device)
        cdsl_get_step1(self.ctx, need, tok, rew)
        self.stream.synchronize()
        return need, tok, rew

    def counters(self):
        return cdsl_get_counters(self.ctx)

    def status(self):
        return cdsl_get_status(self.ctx)

    def close(self):
        if getattr(self, "ctx", None):
            cdsl_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
