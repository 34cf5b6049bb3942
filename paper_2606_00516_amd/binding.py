"""ctypes binding of libeb.so (C ABI in include/eb_layer.h).

Argument marshalling only: torch tensors become device pointers, numpy
length arrays become host pointers, the current torch stream becomes the
hipStream_t.  Every computation runs in the library's HIP kernels.  Loading
raises if the library has not been built; nothing here falls back to another
implementation.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeb.so")

EB_OK = 0
STATUS = {0: "EB_OK", -1: "EB_ERR_NULL", -2: "EB_ERR_CONFIG", -3: "EB_ERR_BATCH", -4: "EB_ERR_MODE",
          -5: "EB_ERR_PAGES", -6: "EB_ERR_WORKSPACE", -7: "EB_ERR_LIMITS", -8: "EB_ERR_HIP"}
MODES = {"decode": 0, "prefill": 1, "mixed": 2}
EPILOGUES = {"store": 0, "residual": 1, "silu_mul": 2}

# every symbol include/eb_layer.h declares
SYMBOLS = ("eb_create", "eb_destroy", "eb_workspace_bytes", "eb_layer_step_decode", "eb_layer_step_prefill",
           "eb_layer_step_mixed", "eb_validate", "eb_status_str", "eb_last_error", "eb_op_rmsnorm",
           "eb_op_gemm_workspace_bytes", "eb_op_gemm", "eb_op_gemm_w8", "eb_op_moe_ffn_workspace_bytes", "eb_op_moe_ffn", "eb_op_rope_kv_append", "eb_op_attention",
           "eb_op_gather_kv", "eb_profile", "eb_profile_read", "eb_profile_stage_name", "eb_stack_workspace_bytes",
           "eb_stack_step", "eb_workspace_offset", "eb_noalloc_scratch_bytes", "eb_layer_step_mixed_noalloc",
           "eb_packed_weight_bytes", "eb_pack_weight", "eb_op_rotary_kv_append_workspace_bytes",
           "eb_op_rotary_kv_append", "eb_op_attention_mod_workspace_bytes", "eb_op_attention_mod",
           "eb_op_kv_evict_workspace_bytes", "eb_op_kv_evict")


class EbError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class LayerConfig(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32), ("expert_ffn", ctypes.c_int32),
                ("moe_renormalize", ctypes.c_int32), ("qk_norm", ctypes.c_int32)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")] + \
        [("w_dtype", ctypes.c_int32)] + [(n, ctypes.c_void_p) for n in ("s_qkv", "s_o", "s_gate_up", "s_down")] + \
        [(n, ctypes.c_void_p) for n in ("w_router", "w_experts_gate_up", "w_experts_down", "q_norm", "k_norm")] + \
        [(n, ctypes.c_void_p) for n in ("p_qkv", "p_o", "p_gate_up", "p_down")]


W_BF16, W_FP8_E4M3 = 0, 1


class KvCache(ctypes.Structure):
    _fields_ = [("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("num_pages", ctypes.c_int32),
                ("block_tables", ctypes.c_void_p), ("max_pages_per_seq", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


KV_BF16, KV_FP8_E4M3 = 0, 1
_CODE_DTYPES = (torch.uint8,) + ((torch.float8_e4m3fn,) if hasattr(torch, "float8_e4m3fn") else ())


class Batch(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_tokens", ctypes.c_int32),
                ("context_lens_host", ctypes.c_void_p), ("chunk_lens_host", ctypes.c_void_p)]


ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "wavelength": 3, "yarn": 4}


class Rotary(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("theta", ctypes.c_float), ("factor", ctypes.c_float), ("low", ctypes.c_float),
                ("high", ctypes.c_float), ("magnitude", ctypes.c_float), ("original_len", ctypes.c_int32),
                ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p)]


class ScoreMod(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("slopes", ctypes.c_void_p),
                ("window", ctypes.c_int32), ("prefix_lens_host", ctypes.c_void_p), ("first_key", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libeb.so (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run __graft_entry__.build() (hipcc, gfx950)")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, SZ, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_size_t, ctypes.c_void_p
    sig = {
        "eb_create": (I32, [P(LayerConfig), I32, I32, P(VP)]),
        "eb_destroy": (None, [VP]),
        "eb_workspace_bytes": (SZ, [VP, P(Batch), I32]),
        "eb_workspace_offset": (SZ, [VP, P(Batch), I32, I32]),
        "eb_noalloc_scratch_bytes": (SZ, []),
        "eb_layer_step_mixed_noalloc": (I32, [VP, P(LayerWeights), P(KvCache), P(Batch), VP, VP, VP]),
        "eb_validate": (I32, [P(LayerConfig), P(Batch), VP, I32, I32, I32]),
        "eb_status_str": (ctypes.c_char_p, [I32]),
        "eb_last_error": (ctypes.c_char_p, []),
        "eb_op_rmsnorm": (I32, [VP, VP, VP, VP, I32, VP]),
        "eb_op_gemm_workspace_bytes": (SZ, [I32, I32, I32]),
        "eb_op_gemm": (I32, [VP, VP, VP, VP, I32, I32, I32, I32, VP, SZ, VP]),
        "eb_op_gemm_w8": (I32, [VP, VP, VP, VP, VP, I32, I32, I32, I32, VP, SZ, VP]),
        "eb_packed_weight_bytes": (SZ, [ctypes.c_int, ctypes.c_int]),
        "eb_pack_weight": (I32, [VP, VP, ctypes.c_int, ctypes.c_int, VP]),
        "eb_op_moe_ffn_workspace_bytes": (SZ, [I32, I32, I32, I32, I32]),
        "eb_op_moe_ffn": (I32, [VP, VP, VP, VP, VP, I32, I32, I32, I32, I32, I32, VP, VP, VP, VP, SZ, VP]),
        "eb_op_rope_kv_append": (I32, [VP, VP, P(KvCache), P(Batch), VP, SZ, VP]),
        "eb_op_attention": (I32, [VP, VP, P(KvCache), P(Batch), VP, VP, SZ, I32, VP]),
        "eb_op_gather_kv": (I32, [VP, P(KvCache), P(Batch), VP, VP, VP, SZ, VP]),
        "eb_op_rotary_kv_append_workspace_bytes": (SZ, [VP, P(Batch)]),
        "eb_op_rotary_kv_append": (I32, [VP, P(Rotary), VP, P(KvCache), P(Batch), VP, VP, SZ, VP]),
        "eb_op_attention_mod_workspace_bytes": (SZ, [VP, P(Batch), P(ScoreMod), I32]),
        "eb_op_attention_mod": (I32, [VP, VP, P(KvCache), P(Batch), P(ScoreMod), VP, VP, VP, I32, VP, SZ, VP]),
        "eb_op_kv_evict_workspace_bytes": (SZ, [VP, I32, VP, VP]),
        "eb_op_kv_evict": (I32, [VP, P(KvCache), VP, I32, VP, VP, I32, I32, P(KvCache), VP, VP, I32, VP, SZ, VP]),
        "eb_profile": (I32, [VP, I32, ctypes.c_uint32]),
        "eb_profile_read": (I32, [VP, P(ctypes.c_float), I32]),
        "eb_profile_stage_name": (ctypes.c_char_p, [I32]),
        "eb_stack_workspace_bytes": (SZ, [VP, P(Batch), I32]),
        "eb_stack_step": (I32, [VP, I32, I32, P(LayerWeights), P(KvCache), P(Batch), VP, VP, VP, SZ, VP]),
    }
    for name in ("eb_layer_step_decode", "eb_layer_step_prefill", "eb_layer_step_mixed"):
        sig[name] = (I32, [VP, P(LayerWeights), P(KvCache), P(Batch), VP, VP, VP, SZ, VP])
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _check(status: int):
    if status != EB_OK:
        raise EbError(status, lib().eb_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def config_of(shape) -> LayerConfig:
    """LayerConfig from any object with the layer-shape attributes."""
    return LayerConfig(shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn,
                       getattr(shape, "page_size", 16), float(shape.rms_eps), float(shape.rope_theta),
                       getattr(shape, "n_experts", 0), getattr(shape, "top_k", 0), getattr(shape, "expert_ffn", 0),
                       1 if getattr(shape, "moe_renormalize", True) else 0, 1 if getattr(shape, "qk_norm", False) else 0)


class HostBatch:
    """Holds the host int32 length arrays alive for the duration of a call."""

    def __init__(self, context_lens, chunk_lens):
        self.ctx, self.chk = self._ints(context_lens), self._ints(chunk_lens)
        self.c = Batch(len(self.ctx), int(self.chk.sum()), self.ctx.ctypes.data, self.chk.ctypes.data)

    @staticmethod
    def _ints(a) -> np.ndarray:
        a = np.ascontiguousarray(a)
        if a.dtype == np.int32:
            return a
        b = a.astype(np.int32)
        if a.dtype.kind in "iu" and (a.tobytes() != b.astype(a.dtype).tobytes() or (a.dtype == np.uint32 and (b < 0).any())):
            raise ValueError("a request's length does not fit 32 bits")   # (numpy has cut it off)
        return b


def kv_struct(k_cache: torch.Tensor, v_cache: torch.Tensor, block_tables: torch.Tensor,
              kv_scales=None) -> KvCache:
    """bf16 caches, or 8-bit E4M3 code caches (uint8 / float8_e4m3fn) with
    kv_scales = (k_scale, v_scale).  The struct holds on to the tensors; its
    `sizes` are what its pointers do not carry: the tables' rows, the elements
    of a page (-1: not those of keys and values alike), the device (-2: not
    one)."""
    assert block_tables.dtype == torch.int32 and block_tables.dim() == 2
    assert k_cache.dtype == v_cache.dtype
    if k_cache.dtype in _CODE_DTYPES:
        if kv_scales is None:
            raise ValueError("an 8-bit cache needs kv_scales = (k_scale, v_scale)")
        kv = KvCache(_ptr(k_cache), _ptr(v_cache), int(k_cache.shape[0]), _ptr(block_tables),
                     int(block_tables.shape[1]), KV_FP8_E4M3, float(kv_scales[0]), float(kv_scales[1]))
    else:
        assert k_cache.dtype == torch.bfloat16
        kv = KvCache(_ptr(k_cache), _ptr(v_cache), int(k_cache.shape[0]), _ptr(block_tables),
                     int(block_tables.shape[1]), KV_BF16, 1.0, 1.0)
    page = k_cache.numel() // max(1, kv.num_pages)
    devices = {t.get_device() for t in (k_cache, v_cache, block_tables)}
    kv.sizes = (int(block_tables.shape[0]), page if v_cache.numel() >= kv.num_pages * page else -1,
                devices.pop() if len(devices) == 1 else -2)
    kv.held = (k_cache, v_cache, block_tables)
    return kv


def weights_struct(w: dict) -> LayerWeights:
    """Weights dict -> struct: bf16 projections, or uint8 / float8_e4m3fn
    codes with float32 row scales under s_qkv, s_o, s_gate_up, s_down;
    a mixture-of-experts layer brings w_router, w_experts_gate_up and
    w_experts_down instead of w_gate_up and w_down; a layer with q/k norms
    brings their gains under q_norm and k_norm; fragment-packed copies of
    the bf16 projections (eb_pack_weight) go under p_qkv, p_o, p_gate_up,
    p_down."""
    lw = LayerWeights(*[_ptr(w.get(k)) for k in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")])
    for k in ("w_router", "w_experts_gate_up", "w_experts_down", "q_norm", "k_norm", "p_qkv", "p_o", "p_gate_up",
              "p_down"):
        if k in w:
            setattr(lw, k, _ptr(w[k]))
    if w["w_qkv"].dtype in _CODE_DTYPES:
        lw.w_dtype = W_FP8_E4M3
        for k in ("s_qkv", "s_o", "s_gate_up", "s_down"):
            if w[k].dtype != torch.float32 or not w[k].is_contiguous():
                raise ValueError(f"{k} must be contiguous float32")
            setattr(lw, k, _ptr(w[k]))
    return lw


class Handle:
    """eb_create / eb_destroy."""

    def __init__(self, shape, max_seqs: int, max_tokens: int):
        self.shape = shape
        self.cfg = c = config_of(shape)
        self.n_q_heads, self.n_kv_heads, self.head_dim = c.n_q_heads, c.n_kv_heads, c.head_dim
        self.qkv_cols = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim
        self.page_keys = c.n_kv_heads * c.page_size   # keys of one page over the kv heads
        h = ctypes.c_void_p()
        _check(lib().eb_create(ctypes.byref(self.cfg), int(max_seqs), int(max_tokens), ctypes.byref(h)))
        self.h = h

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            lib().eb_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def eb_workspace_bytes(h: Handle, context_lens, chunk_lens, mode: str) -> int:
    hb = HostBatch(context_lens, chunk_lens)
    return int(lib().eb_workspace_bytes(h.h, ctypes.byref(hb.c), MODES[mode]))


WS_BUFFERS = {"qkv": 0, "attn": 1, "h1": 2, "mlp": 3, "norm": 4}


def eb_workspace_offset(h: Handle, context_lens, chunk_lens, mode: str, which: str) -> int:
    """Byte offset of an intermediate buffer inside a step's workspace (-1:
    none)."""
    hb = HostBatch(context_lens, chunk_lens)
    off = int(lib().eb_workspace_offset(h.h, ctypes.byref(hb.c), MODES[mode], WS_BUFFERS[which]))
    return -1 if off == (1 << 64) - 1 else off


def workspace_intermediates(h: Handle, ws: torch.Tensor, context_lens, chunk_lens, mode: str) -> dict:
    """Views of the intermediate buffers a layer step left in ``ws``: bf16
    qkv [T, (nq + 2 nkv) hd] (q normalised and rotated in place), attn
    [T, nq hd], h1 [T, d], mlp [T, ffn] (dense layers), norm [T, d]."""
    s = h.shape
    T = int(np.asarray(chunk_lens).sum())
    cols = {"qkv": (s.n_q_heads + 2 * s.n_kv_heads) * s.head_dim, "attn": s.n_q_heads * s.head_dim,
            "h1": s.hidden, "mlp": s.ffn, "norm": s.hidden}
    out = {}
    for name, c in cols.items():
        off = eb_workspace_offset(h, context_lens, chunk_lens, mode, name)
        if off < 0:
            continue
        out[name] = ws[off:off + T * c * 2].view(torch.bfloat16).view(T, c)
    return out


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    # torch's caching allocator returns 256-byte (or better) aligned blocks
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _own(stream, make, returned: bool = True):
    """Memory that a call makes itself, from the pool of the stream that will
    write it: another stream's may give out memory that kernels there are still
    to write.  What is returned is read and dropped on the current stream."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        t = make()
    if returned:
        t.record_stream(torch.cuda.current_stream())
    return t


def _own_ws(stream, nbytes: int, device="cuda") -> torch.Tensor:
    return _own(stream, lambda: alloc_workspace(nbytes, device), False)


def _step(name, h: Handle, weights: dict, k_cache, v_cache, block_tables, context_lens, chunk_lens,
          x: torch.Tensor, y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None,
          kv_scales=None):
    hb = HostBatch(context_lens, chunk_lens)
    mode = {"eb_layer_step_decode": "decode", "eb_layer_step_prefill": "prefill",
            "eb_layer_step_mixed": "mixed"}[name]
    if y is None:
        y = _own(stream, lambda: torch.empty_like(x))
    if ws is None:
        ws = _own_ws(stream, lib().eb_workspace_bytes(h.h, ctypes.byref(hb.c), MODES[mode]), x.device)
    kv = kv_struct(k_cache, v_cache, block_tables, kv_scales)
    w = weights_struct(weights)
    _check(getattr(lib(), name)(h.h, ctypes.byref(w), ctypes.byref(kv), ctypes.byref(hb.c), _ptr(x), _ptr(y),
                                _ptr(ws), ws.numel(), _stream(stream)))
    return y


def eb_layer_step_decode(h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x, y=None, ws=None,
                         stream=None, kv_scales=None):
    return _step("eb_layer_step_decode", h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x,
                 y, ws, stream, kv_scales)


def eb_layer_step_prefill(h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x, y=None, ws=None,
                          stream=None, kv_scales=None):
    return _step("eb_layer_step_prefill", h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x,
                 y, ws, stream, kv_scales)


def eb_layer_step_mixed(h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x, y=None, ws=None,
                        stream=None, kv_scales=None):
    return _step("eb_layer_step_mixed", h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x,
                 y, ws, stream, kv_scales)


def eb_noalloc_scratch_bytes() -> int:
    return int(lib().eb_noalloc_scratch_bytes())


def eb_layer_step_mixed_noalloc(h, weights, k_cache, v_cache, block_tables, context_lens, chunk_lens, x, y=None,
                                stream=None, kv_scales=None):
    """The mixed step on the library's fixed scratch (no workspace argument;
    y must be given by callers that cannot allocate)."""
    hb = HostBatch(context_lens, chunk_lens)
    if y is None:
        y = _own(stream, lambda: torch.empty_like(x))
    kv = kv_struct(k_cache, v_cache, block_tables, kv_scales)
    w = weights_struct(weights)
    _check(lib().eb_layer_step_mixed_noalloc(h.h, ctypes.byref(w), ctypes.byref(kv), ctypes.byref(hb.c), _ptr(x),
                                             _ptr(y), _stream(stream)))
    return y


def eb_stack_workspace_bytes(h: Handle, context_lens, chunk_lens, mode: str) -> int:
    hb = HostBatch(context_lens, chunk_lens)
    return int(lib().eb_stack_workspace_bytes(h.h, ctypes.byref(hb.c), MODES[mode]))


def eb_stack_step(h: Handle, mode: str, weights: list, caches: list, context_lens, chunk_lens, x: torch.Tensor,
                  y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """n = len(weights) layers; caches[l] = (k_cache, v_cache, block_tables)
    of layer l, plus (k_scale, v_scale) for an 8-bit cache (entries may
    repeat the same tensors)."""
    n = len(weights)
    if len(caches) != n:
        raise ValueError("one cache entry per layer")
    hb = HostBatch(context_lens, chunk_lens)
    if y is None:
        y = _own(stream, lambda: torch.empty_like(x))
    if ws is None:
        ws = _own_ws(stream, lib().eb_stack_workspace_bytes(h.h, ctypes.byref(hb.c), MODES[mode]), x.device)
    ws_arr = (LayerWeights * n)(*[weights_struct(w) for w in weights])
    kv_arr = (KvCache * n)(*[kv_struct(*c) for c in caches])
    _check(lib().eb_stack_step(h.h, MODES[mode], n, ws_arr, kv_arr, ctypes.byref(hb.c), _ptr(x), _ptr(y), _ptr(ws),
                               ws.numel(), _stream(stream)))
    return y


def eb_validate(shape, context_lens, chunk_lens, block_tables_host: np.ndarray, num_pages: int, mode: str) -> int:
    """Host-only validation; returns the status code (0 = EB_OK)."""
    cfg = config_of(shape)
    hb = HostBatch(context_lens, chunk_lens)
    bt = np.ascontiguousarray(block_tables_host, dtype=np.int32)
    mp = bt.shape[1] if bt.ndim == 2 else 0
    return int(lib().eb_validate(ctypes.byref(cfg), ctypes.byref(hb.c), bt.ctypes.data if bt.size else None,
                                 int(num_pages), int(mp), MODES.get(mode, mode) if isinstance(mode, str) else mode))


def eb_last_error() -> str:
    return lib().eb_last_error().decode()


def eb_status_str(status: int) -> str:
    return lib().eb_status_str(int(status)).decode()


def eb_op_rmsnorm(h: Handle, x: torch.Tensor, gamma: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None):
    out = _own(stream, lambda: torch.empty_like(x)) if out is None else out
    _check(lib().eb_op_rmsnorm(h.h, _ptr(x), _ptr(gamma), _ptr(out), int(x.shape[0]), _stream(stream)))
    return out


def eb_op_gemm(A: torch.Tensor, W: torch.Tensor, epilogue: str = "store", residual: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, stream=None):
    M, K = A.shape
    N = W.shape[0]
    ncol = N // 2 if epilogue == "silu_mul" else N
    if out is None:
        out = _own(stream, lambda: torch.empty(M, ncol, dtype=torch.bfloat16, device=A.device))
    nb = int(lib().eb_op_gemm_workspace_bytes(M, N, K))
    ws = _own_ws(stream, nb, A.device)
    _check(lib().eb_op_gemm(_ptr(A), _ptr(W), _ptr(out), _ptr(residual), M, N, K, EPILOGUES[epilogue], _ptr(ws),
                            ws.numel(), _stream(stream)))
    return out


def eb_packed_weight_bytes(rows: int, cols: int) -> int:
    return int(lib().eb_packed_weight_bytes(rows, cols))


def eb_pack_weight(W: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Fragment-packed copy of a bf16 [rows, cols] weight matrix (a flat
    bf16 tensor of rows * cols elements)."""
    if W.dtype != torch.bfloat16 or W.dim() != 2:
        raise ValueError("W must be a 2-D bf16 tensor")
    rows, cols = W.shape
    if out is None:
        out = _own(stream, lambda: torch.empty(rows * cols, dtype=torch.bfloat16, device=W.device))
    if out.numel() * 2 < eb_packed_weight_bytes(rows, cols):
        raise ValueError("out is smaller than the packed copy")
    _check(lib().eb_pack_weight(_ptr(W), _ptr(out), rows, cols, _stream(stream)))
    return out


def pack_layer_weights(w: dict, stream=None) -> dict:
    """The weights dict plus packed copies of its bf16 projections (those
    whose shape has a packed form)."""
    out = dict(w)
    if w.get("w_qkv") is None or w["w_qkv"].dtype != torch.bfloat16:
        return out
    for src, dst in (("w_qkv", "p_qkv"), ("w_o", "p_o"), ("w_gate_up", "p_gate_up"), ("w_down", "p_down")):
        t = w.get(src)
        if t is not None and eb_packed_weight_bytes(*t.shape) > 0:
            out[dst] = eb_pack_weight(t, stream=stream)
    return out


def eb_op_gemm_w8(A: torch.Tensor, W: torch.Tensor, w_scale: torch.Tensor, epilogue: str = "store",
                  residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None):
    """W: uint8 E4M3 codes [N, K]; w_scale: float32 [N], one scale per row."""
    if W.dtype not in _CODE_DTYPES or w_scale.dtype != torch.float32 or not w_scale.is_contiguous():
        raise TypeError("W must hold uint8 codes and w_scale contiguous float32 row scales")
    M, K = A.shape
    N = W.shape[0]
    if w_scale.numel() != N:
        raise ValueError("w_scale needs one scale per row of W")
    ncol = N // 2 if epilogue == "silu_mul" else N
    if out is None:
        out = _own(stream, lambda: torch.empty(M, ncol, dtype=torch.bfloat16, device=A.device))
    nb = int(lib().eb_op_gemm_workspace_bytes(M, N, K))
    ws = _own_ws(stream, nb, A.device)
    _check(lib().eb_op_gemm_w8(_ptr(A), _ptr(W), _ptr(w_scale), _ptr(out), _ptr(residual), M, N, K,
                               EPILOGUES[epilogue], _ptr(ws), ws.numel(), _stream(stream)))
    return out


def eb_op_moe_ffn(b: torch.Tensor, w_router: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor,
                  top_k: int, residual: Optional[torch.Tensor] = None, renormalize: bool = True,
                  out: Optional[torch.Tensor] = None, return_routing: bool = False,
                  ws: Optional[torch.Tensor] = None, stream=None):
    """MoE feed-forward block: b [T, d], w_router [E, d], w_gate_up [E, 2F, d],
    w_down [E, d, F], all bf16; returns out [T, d] (and the int32 expert ids
    and fp32 weights [T, top_k] with ``return_routing``)."""
    for t in (b, w_router, w_gate_up, w_down) + ((residual,) if residual is not None else ()):
        if t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise TypeError("MoE operands must be contiguous bf16")
    T, d = b.shape
    E = w_router.shape[0]
    F = w_gate_up.shape[1] // 2
    if w_router.shape != (E, d) or w_gate_up.shape != (E, 2 * F, d) or w_down.shape != (E, d, F):
        raise ValueError("MoE weight shapes do not match")
    make = lambda n, dtype: _own(stream, lambda: torch.empty(T, n, dtype=dtype, device=b.device))  # noqa: E731
    out = make(d, torch.bfloat16) if out is None else out
    ids = make(top_k, torch.int32) if return_routing else None
    wts = make(top_k, torch.float32) if return_routing else None
    if ws is None:
        ws = _own_ws(stream, int(lib().eb_op_moe_ffn_workspace_bytes(T, d, E, top_k, F)), b.device)
    _check(lib().eb_op_moe_ffn(_ptr(b), _ptr(residual), _ptr(w_router), _ptr(w_gate_up), _ptr(w_down), T, d, E,
                               int(top_k), F, 1 if renormalize else 0, _ptr(out), _ptr(ids), _ptr(wts), _ptr(ws),
                               ws.numel(), _stream(stream)))
    return (out, ids, wts) if return_routing else out


def _op_ws(h, hb, mode="mixed", device="cuda", stream=None):
    return _own_ws(stream, lib().eb_workspace_bytes(h.h, ctypes.byref(hb.c), MODES[mode]), device)


def eb_op_rope_kv_append(h: Handle, qkv: torch.Tensor, k_cache, v_cache, block_tables, context_lens, chunk_lens,
                         stream=None, kv_scales=None):
    hb = HostBatch(context_lens, chunk_lens)
    ws = _op_ws(h, hb, device=qkv.device, stream=stream)
    kv = kv_struct(k_cache, v_cache, block_tables, kv_scales)
    _check(lib().eb_op_rope_kv_append(h.h, _ptr(qkv), ctypes.byref(kv), ctypes.byref(hb.c), _ptr(ws), ws.numel(),
                                      _stream(stream)))
    return qkv


def eb_op_attention(h: Handle, qkv: torch.Tensor, k_cache, v_cache, block_tables, context_lens, chunk_lens,
                    mode: str = "mixed", out: Optional[torch.Tensor] = None, stream=None, kv_scales=None):
    hb = HostBatch(context_lens, chunk_lens)
    s = h.shape
    T = int(hb.chk.sum())
    if out is None:
        out = _own(stream, lambda: torch.empty(T, s.n_q_heads * s.head_dim, dtype=torch.bfloat16, device=qkv.device))
    ws = _op_ws(h, hb, mode if mode in MODES else "mixed", qkv.device, stream)
    kv = kv_struct(k_cache, v_cache, block_tables, kv_scales)
    _check(lib().eb_op_attention(h.h, _ptr(qkv), ctypes.byref(kv), ctypes.byref(hb.c), _ptr(out), _ptr(ws),
                                 ws.numel(), MODES[mode], _stream(stream)))
    return out


def eb_op_gather_kv(h: Handle, k_cache, v_cache, block_tables, context_lens, chunk_lens, stream=None,
                    kv_scales=None):
    """Dense copies of every cached position (raw elements: bf16, or the
    8-bit codes of an 8-bit cache)."""
    hb = HostBatch(context_lens, chunk_lens)
    s = h.shape
    total = int((hb.ctx.astype(np.int64) + hb.chk).sum())
    make = lambda: torch.empty(total, s.n_kv_heads, s.head_dim, dtype=k_cache.dtype, device=k_cache.device)  # noqa: E731
    ok, ov = _own(stream, make), _own(stream, make)
    ws = _op_ws(h, hb, device=k_cache.device, stream=stream)
    kv = kv_struct(k_cache, v_cache, block_tables, kv_scales if kv_scales is not None else (1.0, 1.0))
    _check(lib().eb_op_gather_kv(h.h, ctypes.byref(kv), ctypes.byref(hb.c), _ptr(ok), _ptr(ov), _ptr(ws), ws.numel(),
                                 _stream(stream)))
    return ok, ov


# ---------------------------------------------------------------------------
# operators on the paged cache: rotary append, modified attention, eviction.
# They take the structs that a program keeps between calls: kv_struct(..) of
# its cache and HostBatch(..) of the request lengths.  Structs made here hold
# on to the tensors they point to.
# ---------------------------------------------------------------------------

def _dev(t: torch.Tensor, dtype, name: str, numel: int = -1, dev: int = -1):
    """Device address of a contiguous GPU tensor of this dtype (and size), on
    device dev (-1: the current one)."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.get_device() != (dev if dev >= 0 else torch.cuda.current_device()):   # (a CPU tensor's is -1)
        raise ValueError(f"{name} must be on the current GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel >= 0 and t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements")
    return t.data_ptr()


def _raw_stream(stream, dev: int):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _i32(n, name: str) -> int:
    if not -2 ** 31 <= n < 2 ** 31:
        raise ValueError(f"{name} does not fit 32 bits")
    return int(n)


def _lens(a, name: str) -> np.ndarray:
    a = np.asarray(a)
    if a.dtype == np.int32 and a.flags.c_contiguous and a.ndim == 1:
        return a
    if a.ndim != 1 or (a.size and not np.issubdtype(a.dtype, np.integer)):
        raise TypeError(f"{name} must be a 1-D array of integers")
    if a.size and not (-2 ** 31 <= int(a.min()) and int(a.max()) < 2 ** 31):
        raise ValueError(f"{name} does not fit 32 bits")
    return np.ascontiguousarray(a, dtype=np.int32)


def _check_kv(h: Handle, kv: Optional[KvCache], num_seqs: int, dev: int):
    """Compares what kv_struct noted of a cache with the call that reads it."""
    sizes = getattr(kv, "sizes", None)   # (none in a struct filled by hand)
    if sizes is None:
        return
    rows, page, device = sizes
    if rows < num_seqs:
        raise ValueError("block_tables needs a row per request")
    if page != h.page_keys * h.head_dim:
        raise ValueError("the cache must be [pages, n_kv, 16, head_dim] of the handle's shape, keys and values alike")
    if device != dev:
        raise ValueError("the cache and its block_tables must be on the current GPU")


def _addr(a: np.ndarray) -> int:
    return a.__array_interface__["data"][0]


def _ws(ws: Optional[torch.Tensor], nbytes, stream, dev: int):
    """(tensor to keep alive, address, bytes) of a workspace; allocated when
    None."""
    if ws is None:
        ws = _own(stream, lambda: alloc_workspace(nbytes()), False)
    return ws, _dev(ws, torch.uint8, "ws", -1, dev), ws.numel()


def rotary(theta: float, rotary_dim: int = 0, layout: str = "half", scaling: str = "none", factor: float = 1.0,
           original_len: int = 0, low: float = 0.0, high: float = 0.0, magnitude: float = 0.0,
           q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None) -> Rotary:
    """The rotation of eb_op_rotary_kv_append (eb_rotary); zeros stand for
    the defaults the header gives."""
    r = Rotary(_i32(rotary_dim, "rotary_dim"), ROTARY_LAYOUTS[layout], ROTARY_SCALINGS[scaling], float(theta), float(factor),
               float(low), float(high), float(magnitude), _i32(original_len, "original_len"),
               None if q_norm is None else _dev(q_norm, torch.bfloat16, "q_norm"),
               None if k_norm is None else _dev(k_norm, torch.bfloat16, "k_norm"))
    r.held = (q_norm, k_norm)
    return r


def eb_op_rotary_kv_append_workspace_bytes(h: Handle, batch: HostBatch) -> int:
    return int(lib().eb_op_rotary_kv_append_workspace_bytes(h.h, ctypes.byref(batch.c)))


def eb_op_rotary_kv_append(h: Handle, rot: Rotary, qkv: torch.Tensor, kv: Optional[KvCache], batch: HostBatch,
                           positions: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Rotates the q heads of qkv in place and stores rotated k and v in the
    cache (kv None: rotates k in place too); returns qkv."""
    T, dev = batch.c.num_tokens, torch.cuda.current_device()
    p = _dev(qkv, torch.bfloat16, "qkv", T * h.qkv_cols, dev)
    pos = None if positions is None else _dev(positions, torch.int32, "positions", T, dev)
    _check_kv(h, kv, batch.c.num_seqs, dev)
    if h.cfg.qk_norm:
        for t, name in zip(getattr(rot, "held", ()), ("q_norm", "k_norm")):   # (a struct filled by hand holds none)
            if t is not None:
                _dev(t, torch.bfloat16, name, h.head_dim, dev)
    held, wp, wn = _ws(ws, lambda: eb_op_rotary_kv_append_workspace_bytes(h, batch), stream, dev)
    _check(_lib.eb_op_rotary_kv_append(h.h, rot, p, kv, batch.c, pos, wp, wn, _raw_stream(stream, dev)))
    return qkv


def score_mod(scale: float = 0.0, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, window: int = 0,
              first_key: Optional[torch.Tensor] = None, prefix_lens=None) -> ScoreMod:
    """Scores and masks of eb_op_attention_mod (eb_score_mod)."""
    pre = None if prefix_lens is None else _lens(prefix_lens, "prefix_lens")
    m = ScoreMod(float(scale), float(softcap), None if slopes is None else _dev(slopes, torch.float32, "slopes"),
                 _i32(window, "window"), None if pre is None else pre.ctypes.data,
                 None if first_key is None else _dev(first_key, torch.int32, "first_key"))
    m.held = (slopes, first_key, pre)
    return m


def _check_mod(h: Handle, batch: HostBatch, m: Optional[ScoreMod], dev: int = -1):
    if m is None:
        return None
    slopes, first, pre = getattr(m, "held", (None, None, None))   # (a struct filled by hand names its own addresses)
    if slopes is not None:   # one value per query head
        _dev(slopes, torch.float32, "slopes", h.n_q_heads, dev)
    if first is not None:    # one value per row
        _dev(first, torch.int32, "first_key", batch.c.num_tokens, dev)
    if pre is not None and len(pre) != batch.c.num_seqs:
        raise ValueError("prefix_lens needs one value per request")
    return m


def eb_op_attention_mod_workspace_bytes(h: Handle, batch: HostBatch, mod: Optional[ScoreMod] = None,
                                        want_weights: bool = False) -> int:
    return int(lib().eb_op_attention_mod_workspace_bytes(h.h, ctypes.byref(batch.c), _check_mod(h, batch, mod),
                                                         1 if want_weights else 0))


def eb_op_attention_mod(h: Handle, qkv: torch.Tensor, kv: KvCache, batch: HostBatch, mod: Optional[ScoreMod] = None,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        kv_weights: Optional[torch.Tensor] = None, weight_rows: int = 0,
                        ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention with modified scores and masks; out bf16 [T, n_q head_dim],
    lse fp32 [T, n_q] and kv_weights fp32 [pages, n_kv, 16] where wanted (then
    no two requests of the call may share a page)."""
    T, nq, dev = batch.c.num_tokens, h.n_q_heads, torch.cuda.current_device()
    p = _dev(qkv, torch.bfloat16, "qkv", T * h.qkv_cols, dev)
    if out is None:
        out = _own(stream, lambda: torch.empty(T, nq * h.head_dim, dtype=torch.bfloat16, device=qkv.device))
    o = _dev(out, torch.bfloat16, "out", T * nq * h.head_dim, dev)
    _check_kv(h, kv, batch.c.num_seqs, dev)
    z = None if lse is None else _dev(lse, torch.float32, "lse", T * nq, dev)
    w = None if kv_weights is None else _dev(kv_weights, torch.float32, "kv_weights", kv.num_pages * h.page_keys, dev)
    m = _check_mod(h, batch, mod, dev)
    held, wp, wn = _ws(ws, lambda: eb_op_attention_mod_workspace_bytes(h, batch, mod, w is not None), stream, dev)
    _check(_lib.eb_op_attention_mod(h.h, p, kv, batch.c, m, o, z, w, _i32(weight_rows, "weight_rows"), wp, wn,
                                    _raw_stream(stream, dev)))
    return out


def eb_op_kv_evict_workspace_bytes(h: Handle, lens, keep_lens) -> int:
    a, b = _lens(lens, "lens"), _lens(keep_lens, "keep_lens")
    if len(a) != len(b):
        raise ValueError("lens and keep_lens need one value per request each")
    return int(lib().eb_op_kv_evict_workspace_bytes(h.h, len(a), a.ctypes.data, b.ctypes.data))


def eb_op_kv_evict(h: Handle, src: KvCache, kv_weights: torch.Tensor, lens, keep_lens, dst: KvCache,
                   dst_weights: Optional[torch.Tensor] = None, sink: int = 0, recent: int = 0,
                   kept: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None) -> np.ndarray:
    """Copies the keys to keep from src's pages to dst's; returns the requests'
    new lengths.  kept: int32 [requests, n_kv, >= the largest of them]."""
    a, b = _lens(lens, "lens"), _lens(keep_lens, "keep_lens")
    if len(a) != len(b):
        raise ValueError("lens and keep_lens need one value per request each")
    dev = torch.cuda.current_device()
    _check_kv(h, src, len(a), dev)
    _check_kv(h, dst, len(a), dev)
    w = _dev(kv_weights, torch.float32, "kv_weights", src.num_pages * h.page_keys, dev)
    d = None if dst_weights is None else _dev(dst_weights, torch.float32, "dst_weights", dst.num_pages * h.page_keys, dev)
    k, stride = None, 0
    if kept is not None:
        if kept.dim() != 3 or kept.shape[0] != len(a) or kept.shape[1] != h.n_kv_heads:
            raise ValueError("kept must be [requests, n_kv, keys]")
        k, stride = _dev(kept, torch.int32, "kept", -1, dev), kept.shape[2]
    held, wp, wn = _ws(ws, lambda: eb_op_kv_evict_workspace_bytes(h, a, b), stream, dev)
    _check(_lib.eb_op_kv_evict(h.h, src, w, len(a), _addr(a), _addr(b), _i32(sink, "sink"), _i32(recent, "recent"), dst, d, k,
                               stride, wp, wn, _raw_stream(stream, dev)))
    return np.minimum(a, b)


def eb_profile(h: Handle, enable: bool = True, steps: int = 1, stages=None):
    """Record the stage events of the following steps (a ring of `steps`
    slots; `stages`: names of the stages to bracket, all if None), or stop
    recording."""
    mask = 0
    if stages is not None:
        names = [lib().eb_profile_stage_name(i).decode() for i in range(32) if lib().eb_profile_stage_name(i)]
        for n in stages:
            mask |= 1 << names.index(n)
    _check(lib().eb_profile(h.h, int(steps) if enable else 0, mask))


def eb_profile_read(h: Handle) -> dict:
    """Stage name -> ms, averaged over the recorded steps on this handle."""
    buf = (ctypes.c_float * 32)()
    n = lib().eb_profile_read(h.h, buf, 32)
    if n < 0:
        raise EbError(-8, "eb_profile_read failed")
    return {lib().eb_profile_stage_name(i).decode(): float(buf[i]) for i in range(n)}
