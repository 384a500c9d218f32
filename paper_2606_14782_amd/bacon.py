"""Thin Python binding of libbacon.so (include/bacon.h).

Argument marshalling only: every step of the pass runs in the HIP kernels of
the library.  torch tensors provide device memory and the current HIP stream.
Loading fails loudly when the library is missing; there is no other path.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbacon.so")

OK, ERR_INVALID, ERR_UNSUPPORTED, ERR_ORDER, ERR_WORKSPACE, ERR_HIP = range(6)
FP32, BF16 = 0, 1
TERM_E, TERM_L, TERM_T = 1, 2, 4

ENTRY_POINTS = [
    "bacon_default_params", "bacon_workspace_bytes", "bacon_init", "bacon_free",
    "bacon_begin_prompt", "bacon_score", "bacon_calibrate", "bacon_select_topk",
    "bacon_compact", "bacon_compress_layer", "bacon_compress_layer_lse", "bacon_compress_prompt",
    "bacon_window_lse", "bacon_window_lse_static", "bacon_debug_capture", "bacon_debug_device_errors",
    "bacon_allocate_heads", "bacon_alloc_output",
    "bacon_idx_count",
    "bacon_kept_rows",
    "bacon_profile_enable", "bacon_profile_read", "bacon_status_string", "bacon_last_error",
    "bacon_cache_layout", "bacon_cache_init", "bacon_cache_free", "bacon_cache_clear",
    "bacon_cache_tables", "bacon_cache_store", "bacon_cache_load", "bacon_cache_append",
    "bacon_cache_attend", "bacon_cache_work_bytes", "bacon_cache_step", "bacon_cache_advance",
    "bacon_cache_errors",
]


class Params(C.Structure):
    _fields_ = [("radius", C.c_int32), ("persist_m", C.c_int32), ("rho", C.c_double),
                ("gamma", C.c_float), ("eps", C.c_float), ("pool_kernel", C.c_int32),
                ("use_last_query", C.c_int32), ("terms", C.c_uint32), ("pool_mode", C.c_int32),
                ("head_alloc", C.c_int32), ("alloc_floor", C.c_float)]


# pooling of the score before the top-K (bacon_pool_mode)
POOL_MEAN_S, POOL_MAX_S, POOL_MEAN_B = 0, 1, 2
# head-wise budgets of the fused calls (bacon_head_alloc)
ALLOC_GIVEN, ALLOC_ADAPTIVE = 0, 1


class Shape(C.Structure):
    _fields_ = [("num_layers", C.c_int32), ("num_q_heads", C.c_int32),
                ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("window", C.c_int32),
                ("max_batch", C.c_int32), ("max_total_tokens", C.c_int64), ("dtype", C.c_int)]


class Batch(C.Structure):
    _fields_ = [("batch", C.c_int32), ("cu_seqlens", C.POINTER(C.c_int32)),
                ("budgets", C.POINTER(C.c_int32)), ("head_budgets", C.POINTER(C.c_int32))]


class KernelTime(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("launches", C.c_int64), ("total_ms", C.c_double)]


class CacheShape(C.Structure):
    _fields_ = [("num_layers", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("block_tokens", C.c_int32),
                ("max_batch", C.c_int32), ("max_blocks", C.c_int32), ("num_blocks", C.c_int64),
                ("dtype", C.c_int)]


class CacheOffsets(C.Structure):
    _fields_ = [("lens", C.c_size_t), ("starts", C.c_size_t), ("table", C.c_size_t),
                ("scales", C.c_size_t), ("codes", C.c_size_t), ("errors", C.c_size_t),
                ("total", C.c_size_t)]


# bits of a cache's error word
CACHE_NO_BLOCKS, CACHE_BAD_BLOCK, CACHE_BAD_INDEX = 1, 2, 4


class BaconError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"status {status}: {msg}")
        self.status = status


_lib = None


def lib() -> C.CDLL:
    """Load libbacon.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2606_14782_amd.build")
        L = C.CDLL(LIB_PATH)
        vp, sz = C.c_void_p, C.c_size_t
        ctxp = C.POINTER(C.c_void_p)
        L.bacon_default_params.argtypes = [C.POINTER(Params)]
        L.bacon_workspace_bytes.argtypes = [C.POINTER(Shape), C.POINTER(Params)]
        L.bacon_workspace_bytes.restype = sz
        L.bacon_init.argtypes = [ctxp, C.POINTER(Shape), C.POINTER(Params), vp, sz]
        L.bacon_free.argtypes = [vp]
        L.bacon_begin_prompt.argtypes = [vp, C.POINTER(Batch), vp]
        L.bacon_score.argtypes = [vp, C.c_int32, C.POINTER(Batch), vp, vp, vp, vp, vp, vp]
        L.bacon_calibrate.argtypes = [vp, C.c_int32, C.POINTER(Batch), vp, vp, vp, vp, vp, vp, vp]
        L.bacon_select_topk.argtypes = [vp, C.POINTER(Batch), vp, vp, vp]
        L.bacon_compact.argtypes = [vp, C.POINTER(Batch), vp, vp, vp, vp, vp, vp]
        L.bacon_compress_layer.argtypes = [vp, C.c_int32, C.POINTER(Batch), vp, vp, vp, vp, vp,
                                           vp, vp]
        L.bacon_compress_layer_lse.argtypes = [vp, C.c_int32, C.POINTER(Batch), vp, vp, vp, vp,
                                               vp, vp, vp, vp]
        L.bacon_window_lse.argtypes = [vp, C.POINTER(Batch), vp, vp, vp, vp]
        L.bacon_compress_prompt.argtypes = [vp, C.POINTER(Batch), C.c_int32, C.c_int32, vp, vp, vp,
                                            vp, vp, vp, vp, vp, vp]
        L.bacon_debug_capture.argtypes = [vp, vp, vp, vp]
        L.bacon_allocate_heads.argtypes = [vp, C.POINTER(Batch), vp, vp, vp]
        L.bacon_alloc_output.argtypes = [vp, vp]
        L.bacon_debug_device_errors.argtypes = [vp]
        L.bacon_debug_device_errors.restype = C.c_int32
        L.bacon_window_lse_static.argtypes = [C.POINTER(Shape), C.POINTER(Batch), vp, vp, vp, vp]
        L.bacon_idx_count.argtypes = [C.POINTER(Batch), C.c_int32]
        L.bacon_idx_count.restype = C.c_int64
        L.bacon_kept_rows.argtypes = [C.POINTER(Batch), C.c_int32, C.c_int32]
        L.bacon_kept_rows.restype = C.c_int64
        L.bacon_profile_enable.argtypes = [vp, C.c_int32]
        L.bacon_profile_read.argtypes = [vp, C.POINTER(KernelTime), C.c_int32]
        L.bacon_profile_read.restype = C.c_int32
        i32, i64, cap = C.c_int32, C.c_int64, C.POINTER(Batch)
        L.bacon_cache_layout.argtypes = [C.POINTER(CacheShape), C.POINTER(CacheOffsets)]
        L.bacon_cache_init.argtypes = [ctxp, C.POINTER(CacheShape), vp, sz]
        L.bacon_cache_free.argtypes = [vp]
        L.bacon_cache_clear.argtypes = [vp, i32, i32, vp]
        L.bacon_cache_tables.argtypes = [vp, cap, i32, vp, i32, i32, vp, i64, vp, vp]
        L.bacon_cache_store.argtypes = [vp, cap, i32, i32, i32, vp, vp, vp, i64, vp]
        L.bacon_cache_load.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
        L.bacon_cache_append.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, vp, i64, vp]
        L.bacon_cache_attend.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i32, vp, vp, vp, sz, vp]
        L.bacon_cache_work_bytes.argtypes = [vp, i32, i32, i32]
        L.bacon_cache_work_bytes.restype = sz
        L.bacon_cache_step.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, vp, i64, vp, i64, i32, vp, vp,
                                       vp, sz, vp]
        L.bacon_cache_advance.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp]
        L.bacon_cache_errors.argtypes = [vp]
        L.bacon_cache_errors.restype = i32
        for name in ("layout", "init", "free", "clear", "tables", "store", "load", "append", "attend",
                     "step", "advance"):
            getattr(L, "bacon_cache_" + name).restype = C.c_int
        L.bacon_status_string.argtypes = [C.c_int]
        L.bacon_status_string.restype = C.c_char_p
        L.bacon_last_error.restype = C.c_char_p
        for name in ("bacon_init", "bacon_free", "bacon_begin_prompt", "bacon_score",
                     "bacon_calibrate", "bacon_select_topk", "bacon_compact",
                     "bacon_compress_layer", "bacon_compress_layer_lse", "bacon_window_lse",
                     "bacon_compress_prompt", "bacon_debug_capture", "bacon_window_lse_static",
                     "bacon_allocate_heads", "bacon_alloc_output", "bacon_profile_enable"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != OK:
        raise BaconError(status, lib().bacon_last_error().decode())


def default_params(**overrides) -> Params:
    p = Params()
    lib().bacon_default_params(C.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


class BatchLayout:
    """Host copy of a packed batch: cu_seqlens, per-sequence budgets, and
    optionally a budget per (sequence, KV head) [batch, Hkv]."""

    def __init__(self, cu_seqlens, budgets, head_budgets=None):
        self.cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        self.budgets = np.ascontiguousarray(budgets, dtype=np.int32)
        self.head_budgets = (None if head_budgets is None else
                             np.ascontiguousarray(head_budgets, dtype=np.int32).reshape(len(self.budgets), -1))
        hb = (None if self.head_budgets is None else
              self.head_budgets.ctypes.data_as(C.POINTER(C.c_int32)))
        self.c = Batch(len(self.budgets), self.cu.ctypes.data_as(C.POINTER(C.c_int32)),
                       self.budgets.ctypes.data_as(C.POINTER(C.c_int32)), hb)

    @property
    def total(self) -> int:
        return int(self.cu[-1])

    def idx_count(self, num_kv_heads: int) -> int:
        return int(lib().bacon_idx_count(C.byref(self.c), num_kv_heads))

    def kept_rows(self, window: int, num_kv_heads: int = 1) -> int:
        return int(lib().bacon_kept_rows(C.byref(self.c), num_kv_heads, window))


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class Context:
    """A bacon_ctx with its workspace tensor on the current device."""

    def __init__(self, num_layers, num_q_heads, num_kv_heads, head_dim, window, max_batch,
                 max_total_tokens, dtype, params: Params | None = None, device="cuda"):
        import torch
        self.shape = Shape(num_layers, num_q_heads, num_kv_heads, head_dim, window, max_batch,
                           max_total_tokens, BF16 if dtype in ("bf16", BF16) else FP32)
        self.params = params or default_params()
        nbytes = lib().bacon_workspace_bytes(C.byref(self.shape), C.byref(self.params))
        if nbytes == 0:
            raise BaconError(ERR_INVALID, lib().bacon_last_error().decode())
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        base = self.workspace.data_ptr()
        aligned = (base + 255) & ~255
        self._h = C.c_void_p()
        _check(lib().bacon_init(C.byref(self._h), C.byref(self.shape), C.byref(self.params),
                                C.c_void_p(aligned), nbytes))
        self.device = device
        self.torch_dtype = torch.bfloat16 if self.shape.dtype == BF16 else torch.float32

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and h.value and _lib is not None:
            _lib.bacon_free(h)
            self._h = C.c_void_p()

    # ---- entry points (same names as the C ABI)
    def bacon_begin_prompt(self, batch: BatchLayout):
        _check(lib().bacon_begin_prompt(self._h, C.byref(batch.c), _stream()))

    def bacon_score(self, layer, batch: BatchLayout, q_win, k, want_lse=False):
        import torch
        Hkv, T = self.shape.num_kv_heads, batch.total
        B = torch.empty((Hkv, T), dtype=torch.float32, device=k.device)
        Q = torch.empty((Hkv, T), dtype=torch.float32, device=k.device)
        lse = (torch.empty((len(batch.budgets), self.shape.num_q_heads, self.shape.window),
                           dtype=torch.float32, device=k.device) if want_lse else None)
        _check(lib().bacon_score(self._h, layer, C.byref(batch.c), _ptr(q_win), _ptr(k),
                                 _ptr(lse), _ptr(B), _ptr(Q), _stream()))
        return B, Q, lse

    def bacon_calibrate(self, layer, batch: BatchLayout, B, Q, want_E=False, want_V=False):
        import torch
        Hkv, T = self.shape.num_kv_heads, batch.total
        S = torch.empty((Hkv, T), dtype=torch.float32, device=B.device)
        lam = torch.empty((len(batch.budgets), Hkv), dtype=torch.float32, device=B.device)
        E = torch.empty_like(S) if want_E else None
        V = torch.empty_like(S) if want_V else None
        _check(lib().bacon_calibrate(self._h, layer, C.byref(batch.c), _ptr(B), _ptr(Q), _ptr(S),
                                     _ptr(lam), _ptr(E), _ptr(V), _stream()))
        return {"S": S, "lambda": lam, "E": E, "V": V}

    def bacon_select_topk(self, batch: BatchLayout, S):
        import torch
        idx = torch.empty(batch.idx_count(self.shape.num_kv_heads), dtype=torch.int32,
                          device=S.device)
        _check(lib().bacon_select_topk(self._h, C.byref(batch.c), _ptr(S), _ptr(idx), _stream()))
        return idx

    def _kv_out(self, batch: BatchLayout, like):
        import torch
        rows = batch.kept_rows(self.shape.window, self.shape.num_kv_heads)
        shp = (rows, self.shape.num_kv_heads, self.shape.head_dim)
        return (torch.empty(shp, dtype=like.dtype, device=like.device),
                torch.empty(shp, dtype=like.dtype, device=like.device))

    def bacon_compact(self, batch: BatchLayout, k, v, idx):
        k_out, v_out = self._kv_out(batch, k)
        _check(lib().bacon_compact(self._h, C.byref(batch.c), _ptr(k), _ptr(v), _ptr(idx),
                                   _ptr(k_out), _ptr(v_out), _stream()))
        return k_out, v_out

    def bacon_compress_layer(self, layer, batch: BatchLayout, q_win, k, v, out=None):
        import torch
        if out is None:
            idx = torch.empty(batch.idx_count(self.shape.num_kv_heads), dtype=torch.int32,
                              device=k.device)
            k_out, v_out = self._kv_out(batch, k)
        else:
            idx, k_out, v_out = out
        _check(lib().bacon_compress_layer(self._h, layer, C.byref(batch.c), _ptr(q_win), _ptr(k),
                                          _ptr(v), _ptr(idx), _ptr(k_out), _ptr(v_out),
                                          _stream()))
        return idx, k_out, v_out

    def bacon_compress_layer_lse(self, layer, batch: BatchLayout, q_win, k, v, lse, out=None):
        """The fused pass with the window-row normalisers lse [B, Hq, W] (natural
        log) given, e.g. by the prefill attention."""
        import torch
        if out is None:
            idx = torch.empty(batch.idx_count(self.shape.num_kv_heads), dtype=torch.int32,
                              device=k.device)
            k_out, v_out = self._kv_out(batch, k)
        else:
            idx, k_out, v_out = out
        _check(lib().bacon_compress_layer_lse(self._h, layer, C.byref(batch.c), _ptr(q_win),
                                              _ptr(k), _ptr(v), _ptr(lse), _ptr(idx),
                                              _ptr(k_out), _ptr(v_out), _stream()))
        return idx, k_out, v_out

    def bacon_compress_prompt(self, first_layer, batch: BatchLayout, q_wins, ks, vs, lses=None,
                              outs=None, layer_batches=None):
        """The pass over layers first_layer .. first_layer + len(ks) - 1 in one
        call; returns [(idx, k_out, v_out)] per layer.  layer_batches: None, or
        one BatchLayout per layer (same sequences, the layer's own budgets)."""
        import torch
        n = len(ks)
        lb = layer_batches if layer_batches is not None else [batch] * n
        if outs is None:
            outs = []
            for k, b in zip(ks, lb):
                idx = torch.empty(b.idx_count(self.shape.num_kv_heads), dtype=torch.int32,
                                  device=k.device)
                outs.append((idx, *self._kv_out(b, k)))
        arr = lambda xs: (C.c_void_p * n)(*[x.data_ptr() for x in xs])
        lse_arr = arr(lses) if lses is not None else None
        lb_arr = None
        if layer_batches is not None:
            lb_arr = (C.c_void_p * n)(*[C.cast(C.byref(b.c), C.c_void_p).value for b in layer_batches])
        _check(lib().bacon_compress_prompt(
            self._h, C.byref(batch.c), first_layer, n, arr(q_wins), arr(ks), arr(vs), lse_arr,
            arr([o[0] for o in outs]), arr([o[1] for o in outs]), arr([o[2] for o in outs]),
            lb_arr, _stream()))
        return outs

    def bacon_debug_device_errors(self) -> int:
        """Test instrumentation: the device error word (synchronises)."""
        return int(lib().bacon_debug_device_errors(self._h))

    def bacon_allocate_heads(self, batch: BatchLayout, B, out=None):
        """AdaKV's head-wise budgets K_{b,h} [batch, Hkv] (int32 device tensor)
        from a window score B [Hkv, T]."""
        import torch
        bud = out if out is not None else torch.empty(
            (batch.c.batch, self.shape.num_kv_heads), dtype=torch.int32, device=B.device)
        _check(lib().bacon_allocate_heads(self._h, C.byref(batch.c), _ptr(B), _ptr(bud), _stream()))
        return bud

    def bacon_alloc_output(self, budgets=None):
        """Where the fused calls under the adaptive allocation write each
        layer's budgets: an int32 device tensor [num_layers, max_batch, Hkv],
        or None to stop."""
        _check(lib().bacon_alloc_output(self._h, _ptr(budgets)))

    def bacon_debug_capture(self, B=None, V=None, lam=None):
        """Test instrumentation: per-layer copies of B, V [L, Hkv, T] and lambda
        [L, B, Hkv] (float32 device tensors) from the fused calls; None turns it off."""
        _check(lib().bacon_debug_capture(self._h, _ptr(B), _ptr(V), _ptr(lam)))

    def bacon_window_lse(self, batch: BatchLayout, q_win, k, out=None):
        """The window-row normalisers lse [B, Hq, W] (natural log) alone, as
        bacon_compress_layer_lse takes them."""
        import torch
        s = self.shape
        lse = out if out is not None else torch.empty(
            (batch.c.batch, s.num_q_heads, s.window), dtype=torch.float32, device=k.device)
        _check(lib().bacon_window_lse(self._h, C.byref(batch.c), _ptr(q_win), _ptr(k), _ptr(lse),
                                      _stream()))
        return lse

    def bacon_profile_enable(self, enable=True):
        _check(lib().bacon_profile_enable(self._h, 1 if enable else 0))

    def bacon_profile_read(self) -> dict:
        arr = (KernelTime * 32)()
        n = lib().bacon_profile_read(self._h, arr, 32)
        return {arr[i].name.decode(): (int(arr[i].launches), float(arr[i].total_ms))
                for i in range(max(0, n))}


# Module-level functions with the C names, for callers that prefer them.
def bacon_begin_prompt(ctx: Context, batch):
    return ctx.bacon_begin_prompt(batch)


def bacon_score(ctx: Context, layer, batch, q_win, k, want_lse=False):
    return ctx.bacon_score(layer, batch, q_win, k, want_lse)


def bacon_calibrate(ctx: Context, layer, batch, B, Q, want_E=False, want_V=False):
    return ctx.bacon_calibrate(layer, batch, B, Q, want_E, want_V)


def bacon_select_topk(ctx: Context, batch, S):
    return ctx.bacon_select_topk(batch, S)


def bacon_compact(ctx: Context, batch, k, v, idx):
    return ctx.bacon_compact(batch, k, v, idx)


def bacon_compress_layer(ctx: Context, layer, batch, q_win, k, v, out=None):
    return ctx.bacon_compress_layer(layer, batch, q_win, k, v, out)


def bacon_compress_layer_lse(ctx: Context, layer, batch, q_win, k, v, lse, out=None):
    return ctx.bacon_compress_layer_lse(layer, batch, q_win, k, v, lse, out)


def bacon_compress_prompt(ctx: Context, first_layer, batch, q_wins, ks, vs, lses=None, outs=None,
                          layer_batches=None):
    return ctx.bacon_compress_prompt(first_layer, batch, q_wins, ks, vs, lses, outs, layer_batches)


def bacon_window_lse_static(shape: Shape, batch: BatchLayout, q_win, k, out=None):
    """bacon_window_lse without a context or workspace (static device scratch);
    returns lse [B, Hq, W] (out if given)."""
    import torch
    lse = out if out is not None else torch.empty(
        (batch.c.batch, shape.num_q_heads, shape.window), dtype=torch.float32, device=k.device)
    _check(lib().bacon_window_lse_static(C.byref(shape), C.byref(batch.c), _ptr(q_win), _ptr(k),
                                         _ptr(lse), _stream()))
    return lse


def bacon_debug_capture(ctx: Context, B=None, V=None, lam=None):
    return ctx.bacon_debug_capture(B, V, lam)


def bacon_window_lse(ctx: Context, batch, q_win, k, out=None):
    return ctx.bacon_window_lse(batch, q_win, k, out)


class Cache:
    """A bacon_cache: the kept rows of a model's layers in 8 bits, with its
    memory on `device`.

    lens, starts [num_layers, max_batch, Hkv] and table [.., max_blocks]
    (int32), scales [num_blocks, 2] (float32) and codes [num_blocks, 2,
    block_tokens * d] (uint8, e4m3) are views of that memory.  max_tokens: the
    longest a pair may become.  Tensors given to the calls are on the cache's
    device; every call runs on that device's current stream.  New tokens and
    queries may be views of one projection's output: only the heads of a token
    have to lie together, tokens evenly spaced.
    """

    def __init__(self, num_layers, num_q_heads, num_kv_heads, head_dim, window, block_tokens, max_batch,
                 max_tokens, num_blocks, dtype, device="cuda"):
        import torch
        if block_tokens < 1:
            raise BaconError(ERR_INVALID, "block_tokens must be >= 1")
        if dtype not in ("bf16", "fp32", BF16, FP32, torch.bfloat16, torch.float32):
            raise BaconError(ERR_UNSUPPORTED, f"dtype {dtype} is not supported (bf16 or fp32)")
        bf16 = dtype in ("bf16", BF16, torch.bfloat16)
        blocks = (max_tokens + block_tokens - 1) // block_tokens
        self.shape = CacheShape(num_layers, num_q_heads, num_kv_heads, head_dim, window, block_tokens,
                                max_batch, blocks, num_blocks, BF16 if bf16 else FP32)
        off = CacheOffsets()
        _check(lib().bacon_cache_layout(C.byref(self.shape), C.byref(off)))
        self._torch, self._L = torch, lib()
        self._raw_stream, self._current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        self._hq, self._hkv, self._d, self._work = num_q_heads, num_kv_heads, head_dim, {}
        dev = torch.device(device)
        if dev.type != "cuda":
            raise BaconError(ERR_INVALID, f"a cache lives on a GPU, not on {dev}")
        self.device = dev if dev.index is not None else torch.device(dev.type, torch.cuda.current_device())
        self.torch_dtype = torch.bfloat16 if self.shape.dtype == BF16 else torch.float32
        self.memory = torch.empty(off.total + 256, dtype=torch.uint8, device=self.device)
        skip = -self.memory.data_ptr() % 256
        self._h = C.c_void_p()
        _check(lib().bacon_cache_init(C.byref(self._h), C.byref(self.shape),
                                      C.c_void_p(self.memory.data_ptr() + skip), off.total))

        def part(at, dtype, *shape):
            n = int(np.prod(shape)) * dtype.itemsize
            return self.memory[skip + at:skip + at + n].view(dtype).view(shape)

        pairs = (num_layers, max_batch, num_kv_heads)
        self.lens = part(off.lens, torch.int32, *pairs)
        self.starts = part(off.starts, torch.int32, *pairs)
        self.table = part(off.table, torch.int32, *pairs, blocks)
        self.scales = part(off.scales, torch.float32, num_blocks, 2)
        self.codes = part(off.codes, torch.uint8, num_blocks, 2, block_tokens * head_dim)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h and h.value and _lib is not None:
            _lib.bacon_cache_free(h)
            self._h = C.c_void_p()

    # ---- checks and marshalling (short: a decode step's kernels take microseconds)
    def _call(self, fn, *args):
        """fn on the cache's device and that device's current stream."""
        at = self.device.index
        stream = self._raw_stream(at)
        if self._current() == at:
            status = fn(self._h, *args, stream)
        else:
            with self._torch.cuda.device(self.device):
                status = fn(self._h, *args, stream)
        if status:
            _check(status)

    def _whole(self, t, name, dtype, shape=None):
        """The pointer of a contiguous tensor of this dtype (and shape)."""
        if t is None:
            return None
        if t.dtype != dtype or not t.is_contiguous() or t.device != self.device:
            raise BaconError(ERR_INVALID, f"{name} must be a contiguous {dtype} tensor on {self.device}")
        if shape is not None and t.shape != shape:
            raise BaconError(ERR_INVALID, f"{name} has shape {tuple(t.shape)}, {tuple(shape)} expected")
        return t.data_ptr()

    def _tokens(self, t, name, heads):
        """Sequences, tokens, pointer and token distance of rows [num_seqs, tokens, heads, d]."""
        if t.dtype != self.torch_dtype or t.dim() != 4 or t.device != self.device:
            raise BaconError(ERR_INVALID, f"{name} must be a 4-d {self.torch_dtype} tensor on {self.device}")
        b, n, h, d = t.shape
        if h != heads or d != self._d or b < 1 or n < 1:
            raise BaconError(ERR_INVALID, f"{name} has shape {tuple(t.shape)}")
        sb, sn, sh, sd = t.stride()
        step = sn if n > 1 else sb if b > 1 else h * d
        if sd != 1 or h > 1 and sh != d or n > 1 and b > 1 and sb != n * sn:
            raise BaconError(ERR_INVALID, f"{name} has strides {t.stride()}: a token's heads lie together, "
                                          "tokens evenly spaced")
        return b, n, t.data_ptr(), step

    def _new_rows(self, k, v):
        """Sequences, tokens, and the pointers and distances of new tokens' K and V."""
        b, n, kp, ks = self._tokens(k, "k", self._hkv)
        bv, nv, vp, vs = self._tokens(v, "v", self._hkv)
        if bv != b or nv != n:
            raise BaconError(ERR_INVALID, f"k has {b} x {n} tokens, v {bv} x {nv}")
        return b, n, kp, ks, vp, vs

    def _counts(self, counts, b, name="counts"):
        return None if counts is None else self._whole(counts, name, self._torch.int32, (b,))

    # ---- entry points (same names as the C ABI)
    def bacon_cache_clear(self, first_seq=0, num_seqs=None):
        n = self.shape.max_batch - first_seq if num_seqs is None else num_seqs
        self._call(self._L.bacon_cache_clear, first_seq, n)

    def bacon_cache_tables(self, batch: BatchLayout, budgets=None, reserve=0, free=None, first_seq=0, used=None):
        """Lengths, tables and idx offsets of a prompt; budgets: None (the
        batch's) or int32 [num_layers, >= batch, Hkv] on the device; free: None
        or the int32 ids to take.  Returns the number of ids needed, int64 [1]
        on the device (more than given: some pairs found no blocks)."""
        s = self.shape
        if used is None:
            used = self._torch.empty(1, dtype=self._torch.int64, device=self.device)
        nb = 0
        if budgets is not None:
            if budgets.dim() != 3 or budgets.shape[0] != s.num_layers or budgets.shape[2] != s.num_kv_heads:
                raise BaconError(ERR_INVALID, f"budgets have shape {tuple(budgets.shape)}")
            nb = budgets.shape[1]
        ids = self._whole(free, "free", self._torch.int32)
        if free is not None and not ids:              # an empty tensor's address is NULL, which stands for every id
            ids = self.memory.data_ptr()
        self._call(self._L.bacon_cache_tables, C.byref(batch.c), first_seq,
                   self._whole(budgets, "budgets", self._torch.int32), nb, reserve,
                   ids, 0 if free is None else free.numel(),
                   self._whole(used, "used", self._torch.int64, (1,)))
        return used

    def _layers(self, xs, name, dtype, shape=None):
        """Number of layers, host array of their pointers and a layer's elements:
        a list of tensors, or one with the layers first."""
        if isinstance(xs, self._torch.Tensor):
            base, n = self._whole(xs, name, dtype), xs.shape[0]
            if n < 1 or shape is not None and xs.shape != (n, *shape):
                raise BaconError(ERR_INVALID, f"{name} has shape {tuple(xs.shape)}")
            size = xs.nbytes // n
            if not size:
                raise BaconError(ERR_INVALID, f"{name} is empty")
            return n, (C.c_uint64 * n)(*range(base, base + n * size, size)), xs.numel() // n
        n = len(xs)
        ptrs = [self._whole(x, name, dtype, shape) for x in xs]
        return n, (C.c_uint64 * n)(*ptrs), min((x.numel() for x in xs), default=0)

    def bacon_cache_store(self, batch: BatchLayout, ks, vs, idxs=None, first_seq=0, first_layer=0):
        """The kept rows of the layers first_layer, ..: ks, vs per-layer [T, Hkv,
        d] (lists, or stacked), idxs per-layer idx, or None (rows 0, 1, 2, ..)."""
        rows = (batch.total, self._hkv, self._d)
        n, k, _ = self._layers(ks, "k", self.torch_dtype, rows)
        nv, v, _ = self._layers(vs, "v", self.torch_dtype, rows)
        ni, idx, count = (n, None, 0) if idxs is None else self._layers(idxs, "idx", self._torch.int32)
        if nv != n or ni != n:
            raise BaconError(ERR_INVALID, f"{n} layers of K, {nv} of V" + ("" if idxs is None else f", {ni} of idx"))
        self._call(self._L.bacon_cache_store, C.byref(batch.c), first_seq, first_layer, n, k, v, idx, count)

    def bacon_cache_load(self, count, first_token=0, first_layer=0, num_layers=None, first_seq=0, num_seqs=None,
                         out=None):
        """The values held, rows first_token .. first_token + count - 1 of every
        pair (first_token < 0: from its end): K, V [layers, seqs, Hkv, count, d]."""
        s = self.shape
        nl = s.num_layers - first_layer if num_layers is None else num_layers
        ns = s.max_batch - first_seq if num_seqs is None else num_seqs
        shape = (nl, ns, s.num_kv_heads, count, s.head_dim)
        if out is None:
            if min(shape) < 1:
                raise BaconError(ERR_INVALID, f"a load of shape {shape}")
            both = self.scales.new_empty((2, *shape), dtype=self.torch_dtype)
            k, v = both.unbind(0)
            kp = both.data_ptr()
            vp = kp + both.nbytes // 2
        else:
            k, v = out
            kp, vp = (self._whole(k, "k_out", self.torch_dtype, shape), self._whole(v, "v_out", self.torch_dtype, shape))
        self._call(self._L.bacon_cache_load, first_layer, nl, first_seq, ns, first_token, count, kp, vp)
        return k, v

    def bacon_cache_append(self, layer, k, v, counts=None, first_seq=0):
        """Appends new tokens' rows k, v [num_seqs, tokens, Hkv, d]; counts
        (int32 [num_seqs], device): each sequence's own number of them."""
        b, n, *rows = self._new_rows(k, v)
        self._call(self._L.bacon_cache_append, layer, first_seq, b, n, self._counts(counts, b), *rows)

    def _attend_out(self, q, b, n, max_tokens, out, lse, want_lse, work):
        """Outputs and scratch of an attend, made where they are not given, and their pointers."""
        torch, shape = self._torch, (b, n, self._hq, self._d)
        if out is None:
            out = q.new_empty(shape)
            outp = out.data_ptr()
        else:
            outp = self._whole(out, "out", self.torch_dtype, shape)
        if lse is not None:
            lsep = self._whole(lse, "lse", torch.float32, shape[:3])
        elif want_lse:
            lse = q.new_empty(shape[:3], dtype=torch.float32)
            lsep = lse.data_ptr()
        else:
            lsep = None
        key = (b, n, max_tokens)
        need = self._work.get(key)
        if need is None:
            if len(self._work) > 1000:
                self._work.clear()
            need = self._work[key] = self._L.bacon_cache_work_bytes(self._h, b, n, max_tokens)
        if not need:
            return out, lse, outp, lsep, None, 0
        if work is None:
            work = q.new_empty(need, dtype=torch.uint8)
        return out, lse, outp, lsep, self._whole(work, "work", torch.uint8), work.numel()

    def bacon_cache_attend(self, layer, q, counts=None, max_tokens=None, first_seq=0, out=None, lse=None,
                           want_lse=False, work=None):
        """Attention of q [num_seqs, tokens, Hq, d] over the layer's cache:
        out, or (out, lse [num_seqs, tokens, Hq]) with want_lse or lse given.
        max_tokens: the longest length to expect (None: the table's)."""
        b, n, qp, qs = self._tokens(q, "q", self._hq)
        most = max_tokens or 0
        out, lse, *ptrs = self._attend_out(q, b, n, most, out, lse, want_lse, work)
        self._call(self._L.bacon_cache_attend, layer, first_seq, b, n, self._counts(counts, b), qp, qs, most, *ptrs)
        return out if lse is None else (out, lse)

    def bacon_cache_step(self, layer, q, k, v, counts=None, max_tokens=None, first_seq=0, out=None, lse=None,
                         want_lse=False, work=None):
        """bacon_cache_append(k, v), then bacon_cache_attend(q) over the grown cache."""
        b, n, qp, qs = self._tokens(q, "q", self._hq)
        bk, nk, *rows = self._new_rows(k, v)
        if bk != b or nk != n:
            raise BaconError(ERR_INVALID, f"q has {b} x {n} tokens, k {bk} x {nk}")
        most = max_tokens or 0
        out, lse, *ptrs = self._attend_out(q, b, n, most, out, lse, want_lse, work)
        self._call(self._L.bacon_cache_step, layer, first_seq, b, n, self._counts(counts, b), qp, qs, *rows, most,
                   *ptrs)
        return out if lse is None else (out, lse)

    def bacon_cache_advance(self, delta=0, counts=None, first_layer=0, num_layers=None, first_seq=0, num_seqs=None):
        """Moves the lengths by delta, or by counts (int32 [num_seqs], device; may be negative)."""
        nl = self.shape.num_layers - first_layer if num_layers is None else num_layers
        ns = self.shape.max_batch - first_seq if num_seqs is None else num_seqs
        self._call(self._L.bacon_cache_advance, first_layer, nl, first_seq, ns, delta, self._counts(counts, ns))

    def bacon_cache_errors(self) -> int:
        """The error word (CACHE_* bits); waits for the device."""
        with self._torch.cuda.device(self.device):
            return int(self._L.bacon_cache_errors(self._h))


def bacon_cache_clear(cache: Cache, first_seq=0, num_seqs=None):
    return cache.bacon_cache_clear(first_seq, num_seqs)


def bacon_cache_tables(cache: Cache, batch, budgets=None, reserve=0, free=None, first_seq=0, used=None):
    return cache.bacon_cache_tables(batch, budgets, reserve, free, first_seq, used)


def bacon_cache_store(cache: Cache, batch, ks, vs, idxs=None, first_seq=0, first_layer=0):
    return cache.bacon_cache_store(batch, ks, vs, idxs, first_seq, first_layer)


def bacon_cache_load(cache: Cache, count, first_token=0, first_layer=0, num_layers=None, first_seq=0, num_seqs=None,
                     out=None):
    return cache.bacon_cache_load(count, first_token, first_layer, num_layers, first_seq, num_seqs, out)


def bacon_cache_append(cache: Cache, layer, k, v, counts=None, first_seq=0):
    return cache.bacon_cache_append(layer, k, v, counts, first_seq)


def bacon_cache_attend(cache: Cache, layer, q, counts=None, max_tokens=None, first_seq=0, out=None, lse=None,
                       want_lse=False, work=None):
    return cache.bacon_cache_attend(layer, q, counts, max_tokens, first_seq, out, lse, want_lse, work)


def bacon_cache_step(cache: Cache, layer, q, k, v, counts=None, max_tokens=None, first_seq=0, out=None, lse=None,
                     want_lse=False, work=None):
    return cache.bacon_cache_step(layer, q, k, v, counts, max_tokens, first_seq, out, lse, want_lse, work)


def bacon_cache_advance(cache: Cache, delta=0, counts=None, first_layer=0, num_layers=None, first_seq=0,
                        num_seqs=None):
    return cache.bacon_cache_advance(delta, counts, first_layer, num_layers, first_seq, num_seqs)
