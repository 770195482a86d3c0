"""ctypes binding of libradixmlp.so: same names as the C ABI, argument marshalling only.

Every step of the path runs inside the library's HIP kernels.  PyTorch is used here for
device memory (tensors are passed as raw device pointers) and for the current HIP stream.
There is no fallback: if the shared library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Any, Mapping, Optional, Sequence, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libradixmlp.so")

RADIX_F32, RADIX_BF16, RADIX_F16 = 0, 1, 2
_DTYPES = {"f32": RADIX_F32, "bf16": RADIX_BF16, "f16": RADIX_F16}

EXPORTS = (
    "radix_model_create", "radix_model_destroy", "radix_model_hilo_layers", "radix_index_workspace_bytes", "radix_workspace_bytes",
    "radix_build_index", "radix_build_index_static", "radix_prefill_forward", "radix_prefill_forward_nodedup",
    "radix_dedup_decision",
    "radix_lm_head_workspace_bytes", "radix_lm_head",
    "radix_index_select_rows", "radix_device_status", "radix_status_string",
    "radix_cache_bytes", "radix_cache_workspace_bytes", "radix_cache_reset", "radix_cache_extend", "radix_cache_fork", "radix_cache_free",
    "radix_cache_compact", "radix_cache_copy_pages", "radix_cache_append", "radix_paged_attention_workspace_bytes", "radix_paged_attention",
    "radix_extend_workspace_bytes", "radix_extend_forward", "radix_token_logprobs_workspace_bytes", "radix_token_logprobs",
    "radix_score_tokens_workspace_bytes", "radix_score_tokens",
    "radix_timing_enable", "radix_timing_collect", "radix_debug_gemm_tile", "radix_debug_gemm_band", "radix_debug_gemm_plan", "radix_debug_gemm_plan_cus",
    "radix_debug_gemm_plan_us", "radix_debug_gemm_plan_folded",
    "radix_debug_index_first_round", "radix_debug_index_host_slots", "radix_debug_gemm_run", "radix_debug_gemm_run_folded",
)

TIMING_CATEGORIES = ("gemm_qkv", "gemm_o", "gemm_gateup", "gemm_down", "attention", "scatter", "gather", "rowops",
                     "gemm_hilo_layers")


class RadixError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = _lib().radix_status_string(code).decode() if _LIB is not None else "?"
        super().__init__(f"{where}: {msg} (status {code})")


class radix_model_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d", "n_q_heads", "n_kv_heads", "head_dim", "d_int", "vocab",
                                          "max_pos", "qk_norm", "dtype", "compute_dtype", "hilo_layers", "fold_norms", "lm_head")] + [("eps", C.c_float), ("rope_base", C.c_float)]


class radix_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("g1", "wq", "wk", "wv", "gq", "gk", "wo", "g2", "wg", "wu", "wd")]


class radix_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("gf", C.c_void_p), ("layers_host", C.POINTER(radix_layer_weights)),
                ("lm_head", C.c_void_p)]


class radix_fwd_opts(C.Structure):
    _fields_ = [("threshold", C.c_float), ("force_dedup", C.c_int32), ("attention_mode", C.c_int32),
                ("pad_compact_to", C.c_int32)]


class radix_cache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_kv_heads", "head_dim", "page_size", "n_pages", "dtype", "max_seqs",
                                          "max_pages")] + [(n, C.c_void_p) for n in ("pages", "page_refs", "page_table", "seq_lens")]


_LIB: Optional[C.CDLL] = None


def _lib() -> C.CDLL:
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it first (python -m paper_2601_15013_amd.build). "
                "There is no CPU or PyTorch fallback for this path.")
        lib = C.CDLL(LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        lib.radix_model_create.argtypes = [C.POINTER(radix_model_config), C.POINTER(radix_weights), C.POINTER(vp)]
        lib.radix_model_destroy.argtypes = [vp]
        lib.radix_model_hilo_layers.argtypes = [vp]
        lib.radix_index_workspace_bytes.argtypes = [i32, C.POINTER(sz)]
        lib.radix_workspace_bytes.argtypes = [vp, i32, i32, C.POINTER(sz)]
        lib.radix_build_index.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, C.POINTER(i32), vp, sz, vp]
        lib.radix_build_index_static.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, C.POINTER(i32), vp]
        lib.radix_prefill_forward.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32, C.POINTER(radix_fwd_opts),
                                              vp, vp, sz, vp]
        lib.radix_prefill_forward_nodedup.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, sz, vp]
        lib.radix_dedup_decision.argtypes = [C.POINTER(radix_model_config), i32, i32, i32, C.POINTER(radix_fwd_opts),
                                             C.POINTER(i32)]
        lib.radix_index_select_rows.argtypes = [vp, i32, vp, i32, sz, vp, vp, vp]
        lib.radix_lm_head_workspace_bytes.argtypes = [vp, i32, C.POINTER(sz)]
        lib.radix_lm_head.argtypes = [vp, vp, i32, vp, i32, vp, vp, sz, vp]
        lib.radix_device_status.argtypes = [vp, sz, vp]
        lib.radix_timing_enable.argtypes = [C.c_uint32, C.c_uint32]
        lib.radix_timing_collect.argtypes = [C.POINTER(C.c_float), C.POINTER(i32)]
        lib.radix_debug_gemm_tile.argtypes = [i32, i32, i32, i32, C.POINTER(i32), C.POINTER(i32)]
        lib.radix_debug_gemm_band.argtypes = [i32, i32, i32]
        lib.radix_debug_gemm_plan.argtypes = [i32] * 4 + [C.POINTER(i32)] * 7
        lib.radix_debug_gemm_plan_cus.argtypes = [i32] * 5 + [C.POINTER(i32)] * 7
        lib.radix_debug_gemm_run.argtypes = ([C.c_void_p] * 2 + [i32] * 5 + [C.c_void_p] + [i32] * 2 + [C.c_void_p] * 5 + [i32] * 3 +
                                             [C.c_void_p] + [i32] * 2 + [C.c_void_p] * 2)
        lib.radix_debug_gemm_run_folded.argtypes = ([vp] * 2 + [i32] * 4 + [vp] + [i32] * 2 + [vp] * 5 + [i32] * 2 + [vp, i32] +
                                                    [C.c_float] * 2 + [vp] * 4)
        lib.radix_debug_gemm_plan_us.argtypes = [i32] * 7 + [C.POINTER(C.c_double)]
        lib.radix_debug_index_first_round.argtypes = [i32] * 2
        cache, i64, szp = C.POINTER(radix_cache), C.c_int64, C.POINTER(sz)
        lib.radix_cache_bytes.argtypes = [cache, szp]
        lib.radix_cache_workspace_bytes.argtypes = [cache, i32, szp]
        lib.radix_cache_reset.argtypes = [cache, vp]
        lib.radix_cache_extend.argtypes = [cache, vp, vp, i32, vp, vp, sz, vp, vp]
        lib.radix_cache_fork.argtypes = [cache, vp, vp, i32, vp, sz, vp, vp]
        lib.radix_cache_free.argtypes = [cache, vp, vp, i32, vp, vp]
        lib.radix_cache_compact.argtypes = [cache, vp, vp, sz, vp, vp]
        lib.radix_cache_copy_pages.argtypes = [cache, vp, vp, i32, vp, sz, vp, vp]
        lib.radix_cache_append.argtypes = [cache, i32, vp, i64, vp, i64, vp, vp, vp, i32, i32, vp, vp]
        lib.radix_paged_attention_workspace_bytes.argtypes = [cache, i32, i32, i32, i32, i32, szp]
        lib.radix_paged_attention.argtypes = [cache, i32, vp, i64, i32, vp, vp, vp, i32, i32, i32, i32, vp, i64, vp, sz, vp, vp]
        lib.radix_extend_workspace_bytes.argtypes = [vp, cache, i32, i32, i32, szp]
        lib.radix_extend_forward.argtypes = [vp, cache, vp, vp, vp, i32, i32, i32, vp, vp, sz, vp]
        lib.radix_token_logprobs_workspace_bytes.argtypes = [i32, i32, i32, i32, szp]
        lib.radix_token_logprobs.argtypes = [vp, i32, i64, i32, i32, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp, vp]
        lib.radix_score_tokens_workspace_bytes.argtypes = [vp, i32, i32, i32, szp]
        lib.radix_score_tokens.argtypes = [vp, vp, i32, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        lib.radix_status_string.argtypes = [C.c_int]
        lib.radix_status_string.restype = C.c_char_p
        for n in EXPORTS:
            if n != "radix_status_string":
                getattr(lib, n).restype = C.c_int
        _LIB = lib
    return _LIB


def load_library() -> C.CDLL:
    """Load libradixmlp.so (raises if it has not been built)."""
    return _lib()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise RadixError(code, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _new_all(outputs: Sequence[Tuple[Tuple[int, ...], torch.dtype]], device: torch.device, stream: Optional[torch.cuda.Stream]) -> Tuple[torch.Tensor, ...]:
    """Outputs (shape, dtype) of a call on `stream`.  They are made there: what the current stream's freed tensors leave may still be written
    by kernels in its queue, for which `stream` does not wait.  And they are held, once freed, until the current stream has done what it was
    given by then.  (Entering a stream takes 6 us, so all are made at once.)"""
    current = None if stream is None else torch.cuda.current_stream(device)
    if stream == current:
        return tuple(torch.empty(shape, dtype=dtype, device=device) for shape, dtype in outputs)
    with torch.cuda.stream(stream):
        made = tuple(torch.empty(shape, dtype=dtype, device=device) for shape, dtype in outputs)
    for t in made:
        t.record_stream(current)
    return made


def _new(shape: Tuple[int, ...], dtype: torch.dtype, device: torch.device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    return _new_all([(shape, dtype)], device, stream)[0]


def _i32(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous int32 CUDA tensor")
    return t


class Model:
    """Owns a radix_model handle.  device: index of the device that its weights are on (None: not known)."""

    def __init__(self, handle: int, cfg: radix_model_config, device: Optional[int] = None):
        self.handle = handle
        self.cfg = cfg
        self.device = device

    @property
    def hilo_layers(self) -> int:
        """Leading layers with (hi, lo) GEMM inputs, as resolved by radix_model_create."""
        n = _lib().radix_model_hilo_layers(self.handle)
        _check(min(n, 0), "radix_model_hilo_layers")
        return n

    @property
    def compute_dtype(self) -> str:
        return {v: k for k, v in _DTYPES.items()}[self.cfg.compute_dtype]

    def close(self) -> None:
        if self.handle:
            _lib().radix_model_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def default_compute_dtype(weight_dtype: str) -> str:
    """Operand type the library is used with unless a caller says otherwise: fp32 weights multiply in fp32,
    bf16 weights as fp16 operands (see radixmlp.h, compute_dtype)."""
    return "f32" if weight_dtype == "f32" else "f16"


def make_config(cfg: Any, compute_dtype: Optional[str] = None, hilo_layers: int = 0,
                lm_head: int = 0, fold_norms: int = 0) -> radix_model_config:
    """cfg: any object with the shape attributes (n_layers, d, n_q_heads, ..., dtype).  The library-side
    settings are arguments of their own: compute_dtype ("f32" / "f16" / "bf16"; None = the default for the
    weight type), hilo_layers and lm_head as in radixmlp.h."""
    compute = compute_dtype or default_compute_dtype(cfg.dtype)
    return radix_model_config(cfg.n_layers, cfg.d, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.d_int, cfg.vocab,
                              cfg.max_pos, int(cfg.qk_norm), _DTYPES[cfg.dtype], _DTYPES[compute],
                              int(hilo_layers), int(fold_norms), int(lm_head), cfg.eps, cfg.rope_base)


def radix_model_create(cfg: Any, embed: torch.Tensor, gf: torch.Tensor,
                       layers: Sequence[Mapping[str, torch.Tensor]], lm_head: Optional[torch.Tensor] = None,
                       compute_dtype: Optional[str] = None, hilo_layers: int = 0, lm_head_mode: int = 0,
                       fold_norms: int = 0) -> Model:
    """embed/gf/layers/lm_head: CUDA tensors ([out, in] matrices in the config dtype, fp32 gains)."""
    c = make_config(cfg, compute_dtype, hilo_layers, lm_head_mode, fold_norms)
    arr = (radix_layer_weights * len(layers))()
    for l, lw in enumerate(layers):
        for name, _ in radix_layer_weights._fields_:
            t = lw.get(name)
            setattr(arr[l], name, None if t is None else t.data_ptr())
    w = radix_weights(embed.data_ptr(), gf.data_ptr(), arr, _ptr(lm_head))
    out = C.c_void_p()
    _check(_lib().radix_model_create(C.byref(c), C.byref(w), C.byref(out)), "radix_model_create")
    return Model(out.value, c, torch.cuda.current_device())          # (the library allocates on the current one)


def radix_index_workspace_bytes(max_B: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_index_workspace_bytes(max_B, C.byref(n)), "radix_index_workspace_bytes")
    return n.value


def radix_workspace_bytes(model: Model, max_N: int, max_B: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_workspace_bytes(model.handle, max_N, max_B, C.byref(n)), "radix_workspace_bytes")
    return n.value


def alloc_workspace(nbytes: int, device: str = "cuda") -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def radix_build_index(tok: torch.Tensor, pos: Optional[torch.Tensor], cu_seqlens: torch.Tensor, ws: torch.Tensor,
                      I_scatter: Optional[torch.Tensor] = None, I_gather: Optional[torch.Tensor] = None,
                      n_compact_dev: Optional[torch.Tensor] = None, sync: bool = True,
                      stream: Optional[torch.cuda.Stream] = None
                      ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, Optional[int]]:
    """Returns (I_scatter[N], I_gather[N] (first N' valid), n_compact_dev[1], N' or None if not sync)."""
    N, B = tok.numel(), cu_seqlens.numel() - 1
    dev = cu_seqlens.device
    if I_scatter is None:
        I_scatter = _new((N,), torch.int32, dev, stream)
    if I_gather is None:
        I_gather = _new((N,), torch.int32, dev, stream)
    if n_compact_dev is None:
        n_compact_dev = _new((1,), torch.int32, dev, stream)
    host = C.c_int32(-1)
    rc = _lib().radix_build_index(_ptr(_i32(tok, "tok")) if N else None, _ptr(pos), _ptr(_i32(cu_seqlens, "cu_seqlens")),
                                  B, N, _ptr(I_scatter), _ptr(I_gather), _ptr(n_compact_dev),
                                  C.byref(host) if sync else None, _ptr(ws), ws.numel(), _stream(stream))
    _check(rc, "radix_build_index")
    return I_scatter, I_gather, n_compact_dev, (host.value if sync else None)


def radix_build_index_static(tok: torch.Tensor, pos: Optional[torch.Tensor], cu_seqlens: torch.Tensor,
                             I_scatter: torch.Tensor, I_gather: torch.Tensor, n_compact_dev: torch.Tensor,
                             sync: bool = True, stream: Optional[torch.cuda.Stream] = None) -> Optional[int]:
    """radix_build_index without a workspace (the library's static scratch array); every buffer is the
    caller's, nothing is allocated here or in the library.  Returns N' (None if not sync)."""
    N, B = tok.numel(), cu_seqlens.numel() - 1
    host = C.c_int32(-1)
    rc = _lib().radix_build_index_static(_ptr(_i32(tok, "tok")) if N else None, _ptr(pos),
                                         _ptr(_i32(cu_seqlens, "cu_seqlens")), B, N, _ptr(I_scatter), _ptr(I_gather),
                                         _ptr(n_compact_dev), C.byref(host) if sync else None, _stream(stream))
    _check(rc, "radix_build_index_static")
    return host.value if sync else None


def radix_prefill_forward(model: Model, tok: torch.Tensor, pos: Optional[torch.Tensor], cu_seqlens: torch.Tensor,
                          max_seqlen: int, I_scatter: torch.Tensor, I_gather: torch.Tensor, n_compact: int,
                          ws: torch.Tensor, out: Optional[torch.Tensor] = None, threshold: Optional[float] = None,
                          force_dedup: bool = False, stream: Optional[torch.cuda.Stream] = None,
                          fused_attention: Optional[bool] = None, pad_compact_to: int = 0) -> torch.Tensor:
    """fused_attention: None = RADIX_ATTN_AUTO, False = RADIX_ATTN_THREE_KERNELS, True = RADIX_ATTN_FUSED;
    threshold: None = RADIX_THRESHOLD_AUTO."""
    N, B = tok.numel(), cu_seqlens.numel() - 1
    if out is None:
        out = _new((N, model.cfg.d), torch.float32, cu_seqlens.device, stream)
    mode = 0 if fused_attention is None else (2 if fused_attention else 1)
    opts = radix_fwd_opts(-1.0 if threshold is None else threshold, int(force_dedup), mode, int(pad_compact_to))
    rc = _lib().radix_prefill_forward(model.handle, _ptr(tok), _ptr(pos), _ptr(cu_seqlens), B, N, max_seqlen,
                                      _ptr(I_scatter), _ptr(I_gather), n_compact, C.byref(opts), _ptr(out),
                                      _ptr(ws), ws.numel(), _stream(stream))
    _check(rc, "radix_prefill_forward")
    return out


def radix_dedup_decision(config: radix_model_config, B: int, N: int, n_compact: int, threshold: Optional[float] = None,
                         force_dedup: bool = False, fused_attention: Optional[bool] = None) -> bool:
    """Would radix_prefill_forward deduplicate this batch?  Host arithmetic in the library, no GPU involved."""
    mode = 0 if fused_attention is None else (2 if fused_attention else 1)
    opts = radix_fwd_opts(-1.0 if threshold is None else threshold, int(force_dedup), mode, 0)
    out = C.c_int32(-1)
    _check(_lib().radix_dedup_decision(C.byref(config), B, N, n_compact, C.byref(opts), C.byref(out)),
           "radix_dedup_decision")
    return bool(out.value)


def radix_prefill_forward_nodedup(model: Model, tok: torch.Tensor, pos: Optional[torch.Tensor],
                                  cu_seqlens: torch.Tensor, max_seqlen: int, ws: torch.Tensor,
                                  out: Optional[torch.Tensor] = None,
                                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    N, B = tok.numel(), cu_seqlens.numel() - 1
    if out is None:
        out = _new((N, model.cfg.d), torch.float32, cu_seqlens.device, stream)
    rc = _lib().radix_prefill_forward_nodedup(model.handle, _ptr(tok), _ptr(pos), _ptr(cu_seqlens), B, N, max_seqlen,
                                              _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check(rc, "radix_prefill_forward_nodedup")
    return out


def radix_lm_head_workspace_bytes(model: Model, max_rows: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_lm_head_workspace_bytes(model.handle, max_rows, C.byref(n)), "radix_lm_head_workspace_bytes")
    return n.value


def radix_lm_head(model: Model, hidden: torch.Tensor, rows: Optional[torch.Tensor], ws: torch.Tensor,
                  out: Optional[torch.Tensor] = None, n_rows: Optional[int] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """logits[n_rows, vocab] (fp32) of hidden[rows] (or of the first n_rows rows when rows is None)."""
    if hidden.dtype != torch.float32 or not hidden.is_contiguous():
        raise TypeError("hidden must be a contiguous fp32 tensor")
    n_src = hidden.shape[0]
    n = rows.numel() if rows is not None else (n_src if n_rows is None else n_rows)
    if out is None:
        out = _new((n, model.cfg.vocab), torch.float32, hidden.device, stream)
    rc = _lib().radix_lm_head(model.handle, _ptr(hidden), n_src, None if rows is None else _ptr(_i32(rows, "rows")), n,
                              _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check(rc, "radix_lm_head")
    return out


def radix_index_select_rows(src: torch.Tensor, idx: torch.Tensor, out: Optional[torch.Tensor] = None,
                            status: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out[r] = src[idx[r]] over the leading axis (contiguous rows)."""
    assert src.is_contiguous()
    n_rows = idx.numel()
    row_bytes = (src.numel() // max(src.shape[0], 1)) * src.element_size()
    if out is None:
        out = _new((n_rows,) + tuple(src.shape[1:]), src.dtype, src.device, stream)
    rc = _lib().radix_index_select_rows(_ptr(src), src.shape[0], _ptr(_i32(idx, "idx")), n_rows, row_bytes, _ptr(out),
                                        _ptr(status), _stream(stream))
    _check(rc, "radix_index_select_rows")
    return out


# ---- paged key/value cache, attention over it, log-probabilities

_TORCH_DTYPES = {torch.float32: RADIX_F32, torch.bfloat16: RADIX_BF16, torch.float16: RADIX_F16}


def _launch(name: str, device: torch.device, stream: Optional[torch.cuda.Stream], *args: Any) -> None:
    """Calls the library with the stream as last argument, on `device` (the library launches on the current one).  The current stream's
    handle is asked for directly: torch.cuda.current_stream takes 2.6 us, a fifth of a small call."""
    fn, index = getattr(_lib(), name), device.index
    if torch.cuda.current_device() == index:
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream)
    _check(rc, name)


def _same_device(device: torch.device, **tensors: Optional[torch.Tensor]) -> None:
    index = device.index
    for name, t in tensors.items():
        if t is not None and t.get_device() != index:
            raise ValueError(f"{name} is on {t.device}, the call's other tensors on {device}")


def _model_there(model: Model, device: torch.device) -> None:
    if model.device is not None and model.device != device.index:
        raise ValueError(f"the model is on cuda:{model.device}, the call's tensors on {device}")


def _list(t: Optional[torch.Tensor], name: str, n: int) -> Optional[int]:
    """Pointer of an optional int32 list of n entries."""
    if t is None:
        return None
    if _i32(t, name).numel() != n:
        raise ValueError(f"{name} has {t.numel()} entries, not {n}")
    return _ptr(t)


def _out(t: Optional[torch.Tensor], name: str, shape: Tuple[int, ...], dtype: torch.dtype, device: torch.device,
         stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    if t is None:
        return _new(shape, dtype, device, stream)
    if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")
    return t


def _status(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else _ptr(_i32(t, "status"))


class Cache:
    """A radix_cache over the caller's tensors: pages [n_layers, n_pages, 2, n_kv_heads, page_size, head_dim] (fp32, bf16 or fp16),
    page_refs [n_pages], page_table [max_seqs, max_pages] and seq_lens [max_seqs] (int32), as described in radixmlp.h."""

    def __init__(self, pages: torch.Tensor, page_refs: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor):
        if pages.dim() != 6 or pages.shape[2] != 2 or pages.dtype not in _TORCH_DTYPES or not pages.is_cuda or not pages.is_contiguous():
            raise TypeError("pages must be a contiguous CUDA tensor [n_layers, n_pages, 2, n_kv_heads, page_size, head_dim] of fp32, bf16 or fp16")
        _same_device(pages.device, page_refs=page_refs, page_table=page_table, seq_lens=seq_lens)
        L, n_pages, _, kv, page_size, hd = pages.shape
        if _i32(page_refs, "page_refs").shape != (n_pages,):
            raise ValueError(f"page_refs must have shape ({n_pages},)")
        if _i32(page_table, "page_table").dim() != 2 or _i32(seq_lens, "seq_lens").shape != (page_table.shape[0],):
            raise ValueError("page_table must be [max_seqs, max_pages] and seq_lens [max_seqs]")
        self.pages, self.page_refs, self.page_table, self.seq_lens = pages, page_refs, page_table, seq_lens
        self.device, self.dtype = pages.device, pages.dtype
        self.n_kv_heads, self.head_dim = kv, hd
        self.struct = radix_cache(L, kv, hd, page_size, n_pages, _TORCH_DTYPES[pages.dtype], page_table.shape[0], page_table.shape[1],
                                  _ptr(pages), _ptr(page_refs), _ptr(page_table), _ptr(seq_lens))
        self.ref = C.byref(self.struct)
        n = C.c_size_t()
        _check(_lib().radix_cache_bytes(self.ref, C.byref(n)), "radix_cache_bytes")
        assert n.value == pages.numel() * pages.element_size()


def alloc_cache(n_layers: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, dtype: torch.dtype, max_seqs: int,
                max_pages: int, device: str = "cuda") -> Cache:
    """An empty cache in new tensors."""
    ints = dict(dtype=torch.int32, device=device)
    return Cache(torch.empty((n_layers, n_pages, 2, n_kv_heads, page_size, head_dim), dtype=dtype, device=device),
                 torch.zeros(n_pages, **ints), torch.full((max_seqs, max_pages), -1, **ints), torch.zeros(max_seqs, **ints))


def radix_cache_workspace_bytes(cache: Cache, max_n: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_cache_workspace_bytes(cache.ref, max_n, C.byref(n)), "radix_cache_workspace_bytes")
    return n.value


def radix_cache_reset(cache: Cache, stream: Optional[torch.cuda.Stream] = None) -> None:
    _launch("radix_cache_reset", cache.device, stream, cache.ref)


def radix_cache_extend(cache: Cache, cu_seqlens: torch.Tensor, ws: torch.Tensor, slots: Optional[torch.Tensor] = None,
                       past: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Room for the batch's new tokens; returns past[B], the lengths before (-1 everywhere if the call was refused)."""
    B = _i32(cu_seqlens, "cu_seqlens").numel() - 1
    _same_device(cache.device, cu_seqlens=cu_seqlens, ws=ws, slots=slots, past=past, status=status)
    past = _out(past, "past", (B,), torch.int32, cache.device, stream)
    _launch("radix_cache_extend", cache.device, stream, cache.ref, _list(slots, "slots", B), _ptr(cu_seqlens), B, _ptr(past),
            _ptr(ws), ws.numel(), _status(status))
    return past


def radix_cache_fork(cache: Cache, parents: torch.Tensor, children: torch.Tensor, ws: torch.Tensor,
                     status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    n = _i32(parents, "parents").numel()
    _same_device(cache.device, parents=parents, children=children, ws=ws, status=status)
    _launch("radix_cache_fork", cache.device, stream, cache.ref, _ptr(parents), _list(children, "children", n), n, _ptr(ws),
            ws.numel(), _status(status))


def radix_cache_free(cache: Cache, slots: torch.Tensor, keep_lens: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    n = _i32(slots, "slots").numel()
    _same_device(cache.device, slots=slots, keep_lens=keep_lens, status=status)
    _launch("radix_cache_free", cache.device, stream, cache.ref, _ptr(slots), _list(keep_lens, "keep_lens", n), n,
            _status(status))


def radix_cache_compact(cache: Cache, ws: torch.Tensor, n_used: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Returns n_used[1]: used pages, which are pages 0 .. n_used - 1 now."""
    _same_device(cache.device, ws=ws, n_used=n_used, status=status)
    n_used = _out(n_used, "n_used", (1,), torch.int32, cache.device, stream)
    _launch("radix_cache_compact", cache.device, stream, cache.ref, _ptr(n_used), _ptr(ws), ws.numel(), _status(status))
    return n_used


def radix_cache_copy_pages(cache: Cache, src: torch.Tensor, dst: torch.Tensor, ws: torch.Tensor, status: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
    n = _i32(src, "src").numel()
    _same_device(cache.device, src=src, dst=dst, ws=ws, status=status)
    _launch("radix_cache_copy_pages", cache.device, stream, cache.ref, _ptr(src), _list(dst, "dst", n), n, _ptr(ws), ws.numel(),
            _status(status))


def _token_rows(t: torch.Tensor, name: str, cache: Cache, heads: Optional[int] = None) -> int:
    """Checks a [N, heads, head_dim] tensor whose tokens are contiguous; returns the elements between tokens."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or t.dtype is not cache.dtype or shape[2] != cache.head_dim or (heads is not None and shape[1] != heads):
        raise TypeError(f"{name} must be a CUDA tensor [N, heads, {cache.head_dim}] of the cache's dtype {cache.dtype}")
    if (strides[2] != 1 and shape[2] > 1) or (strides[1] != shape[2] and shape[1] > 1):
        raise TypeError(f"{name}: the heads of a token must be contiguous")
    return strides[0] if shape[0] > 1 else shape[1] * shape[2]


def radix_cache_append(cache: Cache, layer: int, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor, past: torch.Tensor,
                       slots: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """k, v: [N, n_kv_heads, head_dim], may be views into fused q|k|v rows."""
    B, N = _i32(cu_seqlens, "cu_seqlens").numel() - 1, k.shape[0]
    if v.shape != k.shape:
        raise ValueError("k and v differ in shape")
    ks, vs = _token_rows(k, "k", cache, cache.n_kv_heads), _token_rows(v, "v", cache, cache.n_kv_heads)
    _same_device(cache.device, k=k, v=v, cu_seqlens=cu_seqlens, past=past, slots=slots, status=status)
    _launch("radix_cache_append", cache.device, stream, cache.ref, layer, _ptr(k), ks, _ptr(v), vs, _ptr(cu_seqlens),
            _list(past, "past", B), _list(slots, "slots", B), B, N, _status(status))


def radix_paged_attention_workspace_bytes(cache: Cache, n_q_heads: int, max_N: int, max_B: int, max_new: int,
                                          find_shared: bool = False) -> int:
    n = C.c_size_t()
    _check(_lib().radix_paged_attention_workspace_bytes(cache.ref, n_q_heads, max_N, max_B, max_new, int(find_shared),
                                                        C.byref(n)), "radix_paged_attention_workspace_bytes")
    return n.value


def radix_paged_attention(cache: Cache, layer: int, q: torch.Tensor, cu_seqlens: torch.Tensor, past: torch.Tensor, max_new: int,
                          ws: torch.Tensor, slots: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                          status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                          find_shared: bool = False) -> torch.Tensor:
    """q: [N, n_q_heads, head_dim], may be a view into fused rows; returns out of that shape.  find_shared: see radixmlp.h (pages that
    neighbours in the batch have in common are read once for several of them)."""
    B, N = _i32(cu_seqlens, "cu_seqlens").numel() - 1, q.shape[0]
    qs = _token_rows(q, "q", cache)
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    elif out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    os_ = _token_rows(out, "out", cache)
    _same_device(cache.device, q=q, cu_seqlens=cu_seqlens, past=past, ws=ws, slots=slots, out=out, status=status)
    _launch("radix_paged_attention", cache.device, stream, cache.ref, layer, _ptr(q), qs, q.shape[1], _ptr(cu_seqlens),
            _list(past, "past", B), _list(slots, "slots", B), B, N, max_new, int(find_shared), _ptr(out), os_, _ptr(ws), ws.numel(),
            _status(status))
    return out


def radix_extend_workspace_bytes(model: Model, cache: Cache, max_N: int, max_B: int, max_new: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_extend_workspace_bytes(model.handle, cache.ref, max_N, max_B, max_new, C.byref(n)),
           "radix_extend_workspace_bytes")
    return n.value


def radix_extend_forward(model: Model, cache: Cache, tok: torch.Tensor, cu_seqlens: torch.Tensor, max_new: int, ws: torch.Tensor,
                         slots: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Forward of the new tokens tok[N] behind what the cache holds of their slots; returns the hidden states [N, d]."""
    N, B = _i32(tok, "tok").numel(), _i32(cu_seqlens, "cu_seqlens").numel() - 1
    _model_there(model, cache.device)
    _same_device(cache.device, tok=tok, cu_seqlens=cu_seqlens, ws=ws, slots=slots, out=out)
    out = _out(out, "out", (N, model.cfg.d), torch.float32, cache.device, stream)
    _launch("radix_extend_forward", cache.device, stream, model.handle, cache.ref, _ptr(tok), _ptr(cu_seqlens), _list(slots,
            "slots", B), B, N, max_new, _ptr(out), _ptr(ws), ws.numel())
    return out


def radix_token_logprobs_workspace_bytes(max_rows: int, vocab: int, n_given: int, top_k: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_token_logprobs_workspace_bytes(max_rows, vocab, n_given, top_k, C.byref(n)), "radix_token_logprobs_workspace_bytes")
    return n.value


def _given(given: Optional[torch.Tensor], n: int) -> int:
    if given is None:
        return 0
    if _i32(given, "given").dim() != 2 or given.shape[0] != n:
        raise ValueError(f"given must be [{n}, n_given]")
    return given.shape[1]


def _answers(n: int, n_given: int, top_k: int, dev: torch.device, stream: Optional[torch.cuda.Stream]
             ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    return _new_all([((n, n_given), torch.float32), ((n,), torch.float32), ((n, top_k), torch.int32), ((n, top_k), torch.float32)], dev, stream)


def radix_token_logprobs(logits: torch.Tensor, given: Optional[torch.Tensor], ws: torch.Tensor, top_k: int = 0,
                         status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                         ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """logits [n, vocab] (rows may be strided), given [n, n_given] int32 or None.  Returns (logprobs [n, n_given], entropy [n],
    top_ids [n, top_k], top_logprobs [n, top_k])."""
    if logits.dim() != 2 or logits.dtype not in _TORCH_DTYPES or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError("logits must be a CUDA tensor [n, vocab] of fp32, bf16 or fp16 with contiguous rows")
    n, vocab = logits.shape
    g = _given(given, n)
    _same_device(logits.device, given=given, ws=ws, status=status)
    out = _answers(n, g, max(top_k, 0), logits.device, stream)
    _launch("radix_token_logprobs", logits.device, stream, _ptr(logits), _TORCH_DTYPES[logits.dtype], logits.stride(0) if n > 1 else vocab,
            n, vocab, _ptr(given), g, top_k, _ptr(out[0]), _ptr(out[1]), _ptr(out[2]), _ptr(out[3]), _ptr(ws), ws.numel(), _status(status))
    return out


def radix_score_tokens_workspace_bytes(model: Model, max_rows: int, n_given: int, top_k: int) -> int:
    n = C.c_size_t()
    _check(_lib().radix_score_tokens_workspace_bytes(model.handle, max_rows, n_given, top_k, C.byref(n)), "radix_score_tokens_workspace_bytes")
    return n.value


def radix_score_tokens(model: Model, hidden: torch.Tensor, rows: Optional[torch.Tensor], given: Optional[torch.Tensor], ws: torch.Tensor,
                       top_k: int = 0, n_rows: Optional[int] = None, stream: Optional[torch.cuda.Stream] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """radix_lm_head of hidden[rows] (or of the first n_rows rows) and radix_token_logprobs of its logits, which are not kept."""
    if hidden.dtype != torch.float32 or not hidden.is_cuda or not hidden.is_contiguous() or hidden.dim() != 2 or hidden.shape[1] != model.cfg.d:
        raise TypeError(f"hidden must be a contiguous fp32 CUDA tensor [n, {model.cfg.d}]")
    n_src = hidden.shape[0]
    n = rows.numel() if rows is not None else (n_src if n_rows is None else n_rows)
    g = _given(given, n)
    _model_there(model, hidden.device)
    _same_device(hidden.device, rows=rows, given=given, ws=ws)
    out = _answers(n, g, max(top_k, 0), hidden.device, stream)
    _launch("radix_score_tokens", hidden.device, stream, model.handle, _ptr(hidden), n_src, _list(rows, "rows", n), n, _ptr(given), g,
            top_k, _ptr(out[0]), _ptr(out[1]), _ptr(out[2]), _ptr(out[3]), _ptr(ws), ws.numel())
    return out


def radix_device_status(ws: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> int:
    return _lib().radix_device_status(_ptr(ws), ws.numel(), _stream(stream))


def radix_timing_enable(categories: Sequence[str], every_nth: int = 1) -> None:
    mask = 0
    for c in categories:
        mask |= 1 << TIMING_CATEGORIES.index(c)
    _check(_lib().radix_timing_enable(mask, every_nth), "radix_timing_enable")


def radix_timing_collect() -> dict:
    """{category: (total_ms, launches)} since the last collect."""
    n = len(TIMING_CATEGORIES)
    ms = (C.c_float * n)()
    cnt = (C.c_int32 * n)()
    _check(_lib().radix_timing_collect(ms, cnt), "radix_timing_collect")
    return {TIMING_CATEGORIES[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}


def radix_status_string(code: int) -> str:
    return _lib().radix_status_string(code).decode()
