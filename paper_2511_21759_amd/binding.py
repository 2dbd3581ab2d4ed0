"""ctypes binding of the C ABI in include/odb.h: argument marshalling only.

Every function has the name of the C entry point it calls.  Device buffers are
torch CUDA tensors (PyTorch-ROCm is the device allocator and stream provider);
all arithmetic happens inside libodb.so.  There is no fallback: if the library
has not been built, or a call fails, an exception is raised.

Three calls of 8-bit pages, whose latency counts, are packed and made by
_marshal (csrc/marshal.cpp), an extension of this Python and torch that is
loaded with the first of them; the others need libodb.so alone.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Dict, Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libodb.so")

#: every symbol include/odb.h declares
SYMBOLS = (
    "odb_model_create", "odb_model_destroy", "odb_model_init_random", "odb_model_set_tensor",
    "odb_model_get_tensor", "odb_cache_create", "odb_cache_destroy", "odb_cache_length", "odb_prefill",
    "odb_block_step", "odb_prefill_logits", "odb_block_step_logits", "odb_cache_read", "odb_strerror",
    "odb_last_error", "odb_profile_begin", "odb_profile_end", "odb_set_option", "odb_model_status",
    "odb_predict_length", "odb_accept_jump", "odb_block_step_shared", "odb_block_step_static",
    "odb_block_step_shared_rows", "odb_block_step_shared_logits", "odb_cache_truncate", "odb_generate",
    "odb_speculative_jump", "odb_page_tables", "odb_rope_table", "odb_qk_norm_rope", "odb_paged_attention",
    "odb_paged_attention_workspace", "odb_step_paged", "odb_qk_norm_rope_quant", "odb_paged_read_quant", "odb_paged_attention_quant",
    "odb_paged_attention_quant_workspace", "odb_step_paged_quant",
)

KERNEL_CLASSES = ("gemm_qkv", "attention", "gemm_o", "gemm_gate_up", "gemm_down", "gemm_lm_head", "rmsnorm")
OPT_KSPLIT_REDUCE = 0
STATIC_SCRATCH_BYTES = 32 << 20

T_EMBED, T_WQ, T_WK, T_WV, T_WO, T_WG, T_WU, T_WD, T_LM, T_G1, T_G2, T_GF = range(12)


class OdbError(RuntimeError):
    pass


class odb_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int), ("d_model", ctypes.c_int), ("n_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("d_ff", ctypes.c_int), ("vocab", ctypes.c_int),
                ("rope_base", ctypes.c_float), ("rms_eps", ctypes.c_float), ("mask_id", ctypes.c_int)]


_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
_FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class odb_allocator(ctypes.Structure):
    _fields_ = [("alloc", _ALLOC_FN), ("free", _FREE_FN), ("user", ctypes.c_void_p)]


class odb_generate_params(ctypes.Structure):
    _fields_ = [("block_len", ctypes.c_int), ("n_drafts", ctypes.c_int), ("tau", ctypes.c_float),
                ("eos_id", ctypes.c_int), ("truncate_thr", ctypes.c_float), ("share_from", ctypes.c_int),
                ("row_budget", ctypes.c_int)]


class odb_generate_event(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("length", ctypes.c_int), ("block_off", ctypes.c_int),
                ("block_len", ctypes.c_int), ("chosen", ctypes.c_int), ("n_masked", ctypes.c_int),
                ("cand_pos", ctypes.c_int * 4), ("cand_tok", ctypes.c_int * 4)]


class odb_generate_stats(ctypes.Structure):
    _fields_ = [("n_refresh", ctypes.c_int), ("n_step", ctypes.c_int), ("n_step_shared", ctypes.c_int),
                ("final_len", ctypes.c_int), ("n_events", ctypes.c_int), ("refresh_positions", ctypes.c_longlong),
                ("step_rows", ctypes.c_longlong), ("refresh_ms", ctypes.c_double), ("step_ms", ctypes.c_double),
                ("total_ms", ctypes.c_double)]


class odb_pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int),
                ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("dtype", ctypes.c_int),
                ("page_stride", ctypes.c_longlong), ("head_stride", ctypes.c_longlong), ("pos_stride", ctypes.c_longlong)]


class odb_rope(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("scaling", ctypes.c_int), ("factor", ctypes.c_double), ("original_len", ctypes.c_int),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double), ("magnitude", ctypes.c_double)]


class odb_qk_rows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("in_dtype", ctypes.c_int),
                ("rows", ctypes.c_int), ("n_heads", ctypes.c_int), ("q_row", ctypes.c_longlong), ("k_row", ctypes.c_longlong),
                ("v_row", ctypes.c_longlong), ("q_gain", ctypes.c_void_p), ("k_gain", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("table", ctypes.c_void_p), ("n_pos", ctypes.c_int), ("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("positions", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("q_out", ctypes.c_void_p), ("q_out_row", ctypes.c_longlong),
                ("row_end", ctypes.c_void_p)]


class odb_attention(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("q_row", ctypes.c_longlong), ("out_row", ctypes.c_longlong),
                ("cu_rows", ctypes.c_void_p), ("first_pos", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("tables", ctypes.c_void_p),
                ("columns", ctypes.c_int), ("n", ctypes.c_int), ("rows", ctypes.c_int), ("n_heads", ctypes.c_int),
                ("scale", ctypes.c_float), ("causal", ctypes.c_int), ("window", ctypes.c_int), ("sinks", ctypes.c_int),
                ("max_rows", ctypes.c_int), ("max_len", ctypes.c_int), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class odb_paged_rows(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("n", ctypes.c_int), ("b", ctypes.c_int), ("first_pos", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("tables", ctypes.c_void_p), ("columns", ctypes.c_int), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("table", ctypes.c_void_p), ("n_pos", ctypes.c_int), ("layer_stride", ctypes.c_longlong),
                ("skip", ctypes.c_int), ("max_len", ctypes.c_int), ("tau", ctypes.c_float), ("conf", ctypes.c_void_p),
                ("argmax", ctypes.c_void_p), ("unmask", ctypes.c_void_p), ("n_layers", ctypes.c_int)]


class odb_quant_pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("codes", ctypes.c_int), ("group", ctypes.c_int), ("dtype", ctypes.c_int), ("page_stride", ctypes.c_longlong),
                ("head_stride", ctypes.c_longlong), ("pos_stride", ctypes.c_longlong), ("scale_page_stride", ctypes.c_longlong),
                ("scale_head_stride", ctypes.c_longlong)]


class odb_quant_rows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("in_dtype", ctypes.c_int),
                ("rows", ctypes.c_int), ("n_heads", ctypes.c_int), ("q_row", ctypes.c_longlong), ("k_row", ctypes.c_longlong),
                ("v_row", ctypes.c_longlong), ("q_gain", ctypes.c_void_p), ("k_gain", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("table", ctypes.c_void_p), ("n_pos", ctypes.c_int), ("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("positions", ctypes.c_void_p), ("q_out", ctypes.c_void_p), ("q_out_row", ctypes.c_longlong), ("cu_rows", ctypes.c_void_p),
                ("first_pos", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("tables", ctypes.c_void_p), ("columns", ctypes.c_int),
                ("n", ctypes.c_int), ("odd", ctypes.c_void_p)]


EVENT_KINDS = ("refresh", "step", "shared")

_lib = None


def lib() -> ctypes.CDLL:
    """Loads libodb.so (built by `__graft_entry__.build()` / build.py) once."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise OdbError("%s is missing: build it with `python -m paper_2511_21759_amd.build` "
                       "(there is no fallback path)" % LIB_PATH)
    # PyTorch-ROCm ships its own HIP runtime; import it first so that the library
    # binds to the runtime torch uses (one runtime per process, shared streams).
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    L.odb_model_create.argtypes = [ctypes.POINTER(odb_config), ctypes.POINTER(odb_allocator), ctypes.POINTER(vp)]
    L.odb_model_destroy.argtypes = [vp]
    L.odb_model_destroy.restype = None
    L.odb_model_init_random.argtypes = [vp, ctypes.c_uint64, ctypes.c_double, vp]
    L.odb_model_set_tensor.argtypes = [vp, ci, ci, vp, ctypes.c_size_t]
    L.odb_model_get_tensor.argtypes = [vp, ci, ci, vp, ctypes.c_size_t]
    L.odb_cache_create.argtypes = [vp, ci, ci, ctypes.POINTER(vp)]
    L.odb_cache_destroy.argtypes = [vp]
    L.odb_cache_destroy.restype = None
    L.odb_cache_length.argtypes = [vp]
    L.odb_prefill.argtypes = [vp, vp, vp, ci, ci, vp, vp, vp]
    L.odb_block_step.argtypes = [vp, vp, vp, ci, ci, ci, cf, vp, vp, vp, vp]
    L.odb_prefill_logits.argtypes = [vp, vp, vp, ci, ci, vp, vp]
    L.odb_block_step_logits.argtypes = [vp, vp, vp, ci, ci, ci, vp, vp]
    L.odb_cache_read.argtypes = [vp, ci, ci, ci, ci, ci, vp]
    L.odb_profile_begin.argtypes = [vp, ci, ci]
    L.odb_profile_end.argtypes = [vp, ctypes.POINTER(ci), ctypes.POINTER(cf), ctypes.POINTER(cf)]
    L.odb_predict_length.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, cf, vp, vp]
    L.odb_cache_truncate.argtypes = [vp, ci]
    L.odb_generate.argtypes = [vp, vp, vp, ci, ci, vp, vp, vp, vp, ci, vp]
    L.odb_accept_jump.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, vp, vp, vp, vp, vp]
    L.odb_speculative_jump.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, vp, vp]
    L.odb_block_step_shared.argtypes = [vp, vp, vp, ci, ci, ci, ci, cf, vp, vp, vp, vp]
    L.odb_block_step_shared_rows.argtypes = [ci, ci, ci, ci]
    L.odb_block_step_shared_logits.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp, vp]
    L.odb_set_option.argtypes = [vp, ci, ci]
    L.odb_model_status.argtypes = [vp]
    L.odb_block_step_static.argtypes = [vp, vp, vp, ci, ci, ci, cf, vp, vp, vp, vp]
    L.odb_page_tables.argtypes = [vp, vp, ci, ci, vp, ci, vp, ci, vp, vp, vp, vp, vp, vp, vp, ci, vp, vp]
    L.odb_rope_table.argtypes = [vp, ci, ci, vp, vp]
    L.odb_qk_norm_rope.argtypes = [vp, vp, vp]
    L.odb_paged_attention.argtypes = [vp, vp, vp]
    L.odb_paged_attention_workspace.argtypes = [vp, vp]
    L.odb_paged_attention_workspace.restype = ctypes.c_longlong
    L.odb_step_paged.argtypes = [vp, vp, vp, vp]
    L.odb_qk_norm_rope_quant.argtypes = [vp, vp, vp]
    L.odb_paged_read_quant.argtypes = [vp, vp, ci, ci, vp, vp, ctypes.c_longlong, ctypes.c_longlong, vp]
    L.odb_paged_attention_quant.argtypes = [vp, vp, vp]
    L.odb_paged_attention_quant_workspace.argtypes = [vp, vp]
    L.odb_paged_attention_quant_workspace.restype = ctypes.c_longlong
    L.odb_step_paged_quant.argtypes = [vp, vp, vp, ctypes.c_longlong, vp]
    L.odb_strerror.argtypes = [ci]
    L.odb_strerror.restype = ctypes.c_char_p
    L.odb_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


_calls = None           # (library, _marshal, addresses of the library's store, read, attention and workspace)


def _entries():
    """Loads _marshal, which makes the calls of 8-bit pages whose tensors are as described (None from it: this file's own path goes through
    them again, and says what is wrong), and notes the entry points' addresses for it.  Published as a whole: other threads may look."""
    global _calls
    L = lib()
    try:
        from . import _marshal
    except ImportError as e:
        raise OdbError("_marshal.so cannot be loaded (%s): build it with `python -m paper_2511_21759_amd.build`" % e) from None
    _calls = (L, _marshal, *(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.odb_qk_norm_rope_quant, L.odb_paged_read_quant, L.odb_paged_attention_quant, L.odb_paged_attention_quant_workspace)))


def _here(index):
    """The current stream of device `index` if that is the current device, and _calls are those of the open library; else None."""
    if index < 0 or _torch.cuda.current_device() != index:
        return None
    if _calls is None or _calls[0] is not _lib:
        _entries()
    return _raw_stream(index) if _raw_stream is not None else _stream()


def _made(got):
    """What _marshal gave: results, or an error code."""
    if type(got) is int:
        _check(got)
    return got


def _check(rc: int) -> None:
    if rc != 0:
        L = lib()
        raise OdbError("%s: %s" % (L.odb_strerror(rc).decode(), L.odb_last_error().decode()))


def _stream() -> int:
    # the handle of torch.cuda.current_stream() without building the Stream object (a call of the jump controller is
    # bound by its host side: 15.3 us a call, of which the kernel takes 7); the function is not public, so the public way stays
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())


def _dev_i32(t):
    import torch
    if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
        raise OdbError("expected a contiguous int32 CUDA tensor")
    return t.data_ptr()


# ---- one function per C entry point ---------------------------------------------------------

class _TorchAllocator:
    """odb_allocator backed by torch.empty(dtype=uint8, device="cuda"): PyTorch stays the one owner of device
    memory (weights, caches, scratch and the working buffers of odb_generate all come from its caching allocator).
    The tensors are kept alive here, by address, until the library frees them."""

    def __init__(self):
        import torch
        self.live = {}

        def alloc(nbytes, _user):
            try:
                t = torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device="cuda")
            except RuntimeError:           # out of memory: the library reports ODB_E_NOMEM
                return None
            self.live[t.data_ptr()] = t    # (torch's blocks are aligned to 512 bytes)
            return t.data_ptr()

        def free(ptr, _user):
            self.live.pop(ptr, None)

        self._alloc, self._free = _ALLOC_FN(alloc), _FREE_FN(free)      # the callbacks must outlive the model
        self.struct = odb_allocator(self._alloc, self._free, None)


_allocators: Dict[int, _TorchAllocator] = {}


def odb_model_create(shape: Dict, torch_allocator: bool = True) -> int:
    """torch_allocator: hand the library an odb_allocator backed by torch (default); False = allocator NULL, the
    library then calls hipMalloc / hipFree itself."""
    cfg = odb_config(**{k: shape[k] for k, _ in odb_config._fields_})
    out = ctypes.c_void_p()
    al = _TorchAllocator() if torch_allocator else None
    _check(lib().odb_model_create(ctypes.byref(cfg), ctypes.byref(al.struct) if al else None, ctypes.byref(out)))
    if al:
        _allocators[out.value] = al
    return out.value


def odb_model_destroy(model: int) -> None:
    lib().odb_model_destroy(model)
    _allocators.pop(model, None)


def odb_model_init_random(model: int, seed: int, std: float) -> None:
    _check(lib().odb_model_init_random(model, seed, std, _stream()))


def odb_model_set_tensor(model: int, tensor_id: int, layer: int, bits: np.ndarray) -> None:
    bits = np.ascontiguousarray(bits, np.uint16)
    _check(lib().odb_model_set_tensor(model, tensor_id, layer, bits.ctypes.data, bits.size))


def odb_model_get_tensor(model: int, tensor_id: int, layer: int, n: int) -> np.ndarray:
    out = np.empty(n, np.uint16)
    _check(lib().odb_model_get_tensor(model, tensor_id, layer, out.ctypes.data, n))
    return out


def odb_cache_create(model: int, batch: int, max_len: int) -> int:
    out = ctypes.c_void_p()
    _check(lib().odb_cache_create(model, batch, max_len, ctypes.byref(out)))
    return out.value


def odb_cache_destroy(cache: int) -> None:
    lib().odb_cache_destroy(cache)


def odb_cache_length(cache: int) -> int:
    return lib().odb_cache_length(cache)


def odb_prefill(model: int, cache: int, tokens, resp_off: int, conf=None, argmax=None):
    """tokens: int32 CUDA tensor [B, L] -> (conf [B, L-resp_off] f32, argmax int32)."""
    import torch
    B, L = tokens.shape
    if conf is None:
        conf = torch.empty((B, L - resp_off), dtype=torch.float32, device=tokens.device)
    if argmax is None:
        argmax = torch.empty((B, L - resp_off), dtype=torch.int32, device=tokens.device)
    _check(lib().odb_prefill(model, cache, _dev_i32(tokens), L, resp_off, conf.data_ptr(), argmax.data_ptr(),
                             _stream()))
    return conf, argmax


def odb_predict_length(model: int, tokens, conf, argmax, resp_off: int, eos_id: int, truncate_thr: float, out=None):
    """tokens int32 [B, L], conf f32 / argmax int32 [B, L-resp_off] (CUDA tensors) -> new lengths int32 [B]."""
    import torch
    B, L = tokens.shape
    if conf.dtype != torch.float32 or argmax.dtype != torch.int32 or not conf.is_contiguous() or not argmax.is_contiguous():
        raise TypeError("conf must be contiguous float32 and argmax contiguous int32")
    if tuple(conf.shape) != (B, L - resp_off) or tuple(argmax.shape) != (B, L - resp_off):
        raise ValueError("conf / argmax must have shape [B, L - resp_off]")
    if out is None:
        out = torch.empty((B,), dtype=torch.int32, device=tokens.device)
    _check(lib().odb_predict_length(model, _dev_i32(tokens), conf.data_ptr(), argmax.data_ptr(), B, L, resp_off, eos_id,
                                    truncate_thr, out.data_ptr(), _stream()))
    return out


def odb_block_step_shared(model: int, cache: int, drafts, block_off: int, n_masked: int, tau: float,
                          conf=None, argmax=None, unmask=None):
    """drafts: int32 CUDA tensor [B, S, b] -> (conf f32, argmax int32, unmask uint8), each [B, S, b]."""
    import torch
    B, S, b = drafts.shape
    if conf is None:
        conf = torch.empty((B, S, b), dtype=torch.float32, device=drafts.device)
    if argmax is None:
        argmax = torch.empty((B, S, b), dtype=torch.int32, device=drafts.device)
    if unmask is None:
        unmask = torch.empty((B, S, b), dtype=torch.uint8, device=drafts.device)
    _check(lib().odb_block_step_shared(model, cache, _dev_i32(drafts), block_off, b, S, n_masked, tau, conf.data_ptr(),
                                       argmax.data_ptr(), unmask.data_ptr(), _stream()))
    return conf, argmax, unmask


def odb_block_step_shared_logits(model: int, cache: int, drafts, block_off: int, n_masked: int, vocab: int):
    """-> (logits f32 [rows, vocab], rowout int32 [rows]: index into [B, S, b] of every row, -1 for padding)."""
    import torch
    B, S, b = drafts.shape
    rows = lib().odb_block_step_shared_rows(B, b, S, n_masked)
    _check(min(rows, 0))
    logits = torch.empty((rows, vocab), dtype=torch.float32, device=drafts.device)
    rowout = torch.empty((rows,), dtype=torch.int32, device=drafts.device)
    _check(lib().odb_block_step_shared_logits(model, cache, _dev_i32(drafts), block_off, b, S, n_masked,
                                              logits.data_ptr(), rowout.data_ptr(), _stream()))
    return logits, rowout


def odb_cache_truncate(cache: int, new_len: int) -> None:
    _check(lib().odb_cache_truncate(cache, new_len))


def odb_generate(model: int, cache: int, tokens, prompt_len: int, block_len: int, n_drafts: int = 1, tau: float = 0.9,
                 eos_id: int = -1, truncate_thr: float = 0.9, share_from: int = -1, row_budget: int = 0,
                 max_events: int = 0, event_tokens: bool = False):
    """tokens: int32 CUDA tensor [prompt_len + resp_len] whose first prompt_len entries hold the prompt; decoded
    in place.  -> (stats dict, events list of dicts, event_tokens int32 CUDA tensor [n, L0] or None).
    An event's cand_pos / cand_tok hold the candidates in use: four with n_drafts = 8, else two."""
    import torch
    if tokens.dtype != torch.int32 or tokens.dim() != 1 or not tokens.is_contiguous() or not tokens.is_cuda:
        raise TypeError("tokens must be a contiguous 1-D int32 CUDA tensor")
    L0 = tokens.shape[0]
    gp = odb_generate_params(block_len, n_drafts, tau, eos_id, truncate_thr, share_from, row_budget)
    st = odb_generate_stats()
    ev = (odb_generate_event * max_events)() if max_events > 0 else None
    snap = torch.empty((max_events, L0), dtype=torch.int32, device=tokens.device) if event_tokens and max_events > 0 else None
    _check(lib().odb_generate(model, cache, tokens.data_ptr(), prompt_len, L0 - prompt_len, ctypes.byref(gp),
                              ctypes.byref(st), ctypes.cast(ev, ctypes.c_void_p) if ev is not None else None,
                              snap.data_ptr() if snap is not None else None, max_events, _stream()))
    stats = {name: getattr(st, name) for name, _ in odb_generate_stats._fields_}
    n = min(st.n_events, max_events)
    nc = 4 if n_drafts == 8 else 2
    events = [dict(kind=EVENT_KINDS[e.kind], L=e.length, block_off=e.block_off, block_len=e.block_len, chosen=e.chosen,
                   n_masked=e.n_masked, cand_pos=np.array(list(e.cand_pos)[:nc], np.int32),
                   cand_tok=np.array(list(e.cand_tok)[:nc], np.int32)) for e in (ev[i] for i in range(n))]
    return stats, events, (snap[:n] if snap is not None else None)


def odb_accept_jump(model: int, drafts, conf, argmax, unmask, cand_pos, cand_tok):
    """drafts/argmax int32, conf f32, unmask uint8: CUDA tensors [B, 4, b]; cand_pos/cand_tok int32 [B, 2]
    -> (chosen int32 [B], new_drafts int32 [B, 4, b], new_cand_pos int32 [B, 2], new_cand_tok int32 [B, 2])."""
    import torch
    B, S, b = drafts.shape
    if S != 4:
        raise ValueError("the accept-jump stage runs on four drafts")
    want = {"drafts": (drafts, torch.int32, (B, 4, b)), "conf": (conf, torch.float32, (B, 4, b)),
            "argmax": (argmax, torch.int32, (B, 4, b)), "unmask": (unmask, torch.uint8, (B, 4, b)),
            "cand_pos": (cand_pos, torch.int32, (B, 2)), "cand_tok": (cand_tok, torch.int32, (B, 2))}
    for name, (t, dt, shp) in want.items():
        if t.dtype != dt or tuple(t.shape) != shp or not t.is_contiguous() or not t.is_cuda:
            raise TypeError("%s must be a contiguous CUDA tensor of dtype %s and shape %s" % (name, dt, shp))
    chosen = torch.empty((B,), dtype=torch.int32, device=drafts.device)
    new_drafts = torch.empty_like(drafts)
    new_pos, new_tok = torch.empty_like(cand_pos), torch.empty_like(cand_tok)
    _check(lib().odb_accept_jump(model, drafts.data_ptr(), conf.data_ptr(), argmax.data_ptr(), unmask.data_ptr(),
                                 cand_pos.data_ptr(), cand_tok.data_ptr(), B, b, chosen.data_ptr(), new_drafts.data_ptr(),
                                 new_pos.data_ptr(), new_tok.data_ptr(), _stream()))
    return chosen, new_drafts, new_pos, new_tok


def odb_speculative_jump(model: int, drafts, conf, argmax, unmask, cand_pos, cand_tok, n_next: int):
    """drafts/argmax int32, conf f32, unmask uint8: CUDA tensors [B, S, b], S = 4 or 8; cand_pos/cand_tok int32 [B, 4]
    -> (chosen int32 [B], new_drafts int32 [B, n_next, b], new_cand_pos int32 [B, 4], new_cand_tok int32 [B, 4])."""
    import torch
    B, S, b = shape = drafts.shape
    i32 = torch.int32
    for name, t, dt, shp in (("drafts", drafts, i32, shape), ("conf", conf, torch.float32, shape), ("argmax", argmax, i32, shape),
                             ("unmask", unmask, torch.uint8, shape), ("cand_pos", cand_pos, i32, (B, 4)),
                             ("cand_tok", cand_tok, i32, (B, 4))):
        if t.dtype is not dt or t.shape != shp or not t.is_contiguous() or not t.is_cuda:
            raise TypeError("%s must be a contiguous CUDA tensor of dtype %s and shape %s" % (name, dt, tuple(shp)))
    chosen = drafts.new_empty((B,))
    new_drafts = drafts.new_empty((B, max(int(n_next), 1), b))
    new_pos, new_tok = torch.empty_like(cand_pos), torch.empty_like(cand_tok)
    _check(lib().odb_speculative_jump(model, drafts.data_ptr(), conf.data_ptr(), argmax.data_ptr(), unmask.data_ptr(),
                                      cand_pos.data_ptr(), cand_tok.data_ptr(), B, b, S, n_next, chosen.data_ptr(),
                                      new_drafts.data_ptr(), new_pos.data_ptr(), new_tok.data_ptr(), _stream()))
    return chosen, new_drafts, new_pos, new_tok


def odb_block_step(model: int, cache: int, drafts, block_off: int, tau: float, conf=None, argmax=None, unmask=None):
    """drafts: int32 CUDA tensor [B, S, b] -> (conf f32, argmax int32, unmask uint8), each [B, S, b]."""
    import torch
    B, S, b = drafts.shape
    if conf is None:
        conf = torch.empty((B, S, b), dtype=torch.float32, device=drafts.device)
    if argmax is None:
        argmax = torch.empty((B, S, b), dtype=torch.int32, device=drafts.device)
    if unmask is None:
        unmask = torch.empty((B, S, b), dtype=torch.uint8, device=drafts.device)
    _check(lib().odb_block_step(model, cache, _dev_i32(drafts), block_off, b, S, tau, conf.data_ptr(),
                                argmax.data_ptr(), unmask.data_ptr(), _stream()))
    return conf, argmax, unmask


def odb_block_step_static(model: int, cache: int, drafts, block_off: int, tau: float, conf, argmax, unmask):
    """odb_block_step in the library's fixed scratch area; the caller brings every output tensor (nothing is
    allocated on the way, here or in the library)."""
    B, S, b = drafts.shape
    _check(lib().odb_block_step_static(model, cache, _dev_i32(drafts), block_off, b, S, tau, conf.data_ptr(),
                                       argmax.data_ptr(), unmask.data_ptr(), _stream()))
    return conf, argmax, unmask


def odb_prefill_logits(model: int, cache: int, tokens, resp_off: int, vocab: int):
    import torch
    B, L = tokens.shape
    logits = torch.empty((B, L - resp_off, vocab), dtype=torch.float32, device=tokens.device)
    _check(lib().odb_prefill_logits(model, cache, _dev_i32(tokens), L, resp_off, logits.data_ptr(), _stream()))
    return logits


def odb_block_step_logits(model: int, cache: int, drafts, block_off: int, vocab: int):
    import torch
    B, S, b = drafts.shape
    logits = torch.empty((B, S, b, vocab), dtype=torch.float32, device=drafts.device)
    _check(lib().odb_block_step_logits(model, cache, _dev_i32(drafts), block_off, b, S, logits.data_ptr(),
                                       _stream()))
    return logits


def odb_cache_read(cache: int, layer: int, kv: int, batch_index: int, pos0: int, n: int, n_heads: int,
                   head_dim: int) -> np.ndarray:
    out = np.empty((n, n_heads, head_dim), np.float32)
    _check(lib().odb_cache_read(cache, layer, kv, batch_index, pos0, n, out.ctypes.data))
    return out


# ---- paged K/V ------------------------------------------------------------------------------
# These calls run on the device of their tensors (all of a call's on one) and on that device's current stream.  A small one is
# bound by its host side (about 4 us for the launch itself), so structures are packed and not filled field by field, and
# checks look at each tensor once.

ROPE_SCALINGS = ("plain", "linear", "ntk", "yarn")
_PACK_PAGES, _PACK_QK_ROWS, _PACK_ATTENTION = (struct.Struct(f).pack for f in ("@PPiiiiiqqq", "@PPPiiiqqqPPfPiiiPPPqP", "@PPqqPPPPiiiifiiiiiPN"))
_PACK_QUANT_PAGES, _PACK_QUANT_ROWS = (struct.Struct(f).pack for f in ("@PPPPiiiiiiiqqqqq", "@PPPiiiqqqPPfPiiiPPqPPPPiiP"))
_torch = _raw_stream = None


def _load_torch():
    global _torch, _raw_stream, _DTYPES, _CODES
    import torch
    _torch = torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)          # (see _stream)
    _DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
    _CODES = {torch.int8: 3, torch.float8_e4m3fn: 4}
    return torch


def _not_ints(name, shape):
    raise TypeError("%s must be a contiguous int32 tensor of shape %s on the device of the others" % (name, shape))


def _ints(name, t, shape, index, i32):
    """Address of a contiguous int32 tensor of that shape on that device."""
    if t.dtype is not i32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        _not_ints(name, shape)
    return t.data_ptr()


def _on(index, call, *args):
    """call(*args, stream) with device `index` current."""
    if index < 0:
        raise OdbError("expected CUDA tensors")
    if _torch.cuda.current_device() == index:
        rc = call(*args, _raw_stream(index) if _raw_stream is not None else _stream())
        if rc:
            _check(rc)
    else:
        with _torch.cuda.device(index):
            _check(call(*args, _stream()))


def _pages(k_pages, v_pages):
    """Pools [n_pages, n_kv_heads, page_size, head_dim] of any strides whose channels follow each other, as a packed odb_pages."""
    shape, strides = k_pages.shape, k_pages.stride()
    if len(shape) != 4 or v_pages.shape != shape or v_pages.stride() != strides or strides[3] != 1:
        raise TypeError("k_pages and v_pages must be [n_pages, n_kv_heads, page_size, head_dim] with the same strides, the last one 1")
    if v_pages.dtype is not k_pages.dtype or v_pages.get_device() != k_pages.get_device() or k_pages.dtype not in _DTYPES:
        raise TypeError("k_pages and v_pages must be float16 or bfloat16, of one dtype and device")
    return _PACK_PAGES(k_pages.data_ptr(), v_pages.data_ptr(), shape[0], shape[2], shape[1], shape[3], _DTYPES[k_pages.dtype],
                       strides[0], strides[1], strides[2])


def _head_rows(name, t, index, dtype, shape):
    """Row stride of a [rows, heads, head_dim] tensor whose heads follow each other."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise TypeError("%s must be a %s tensor of shape %s on the device of the others" % (name, dtype, tuple(shape)))
    row, head, channel = t.stride()
    if channel != 1 or (head != shape[2] and shape[1] != 1):
        raise TypeError("the heads of a row of %s must follow each other" % name)
    return row if shape[0] > 1 else max(row, shape[1] * shape[2])


def odb_page_tables(held, wanted, tables, free_pages, n_free, page_size: int, n_pages: int, row_first=None, row_count=None,
                    rows_cap: int = 0, slots=None, positions=None, out=None):
    """held, wanted int32 [n]; tables int32 [n, columns] and free_pages int32 [n_pages], updated in place; n_free int32 [1];
    row_first, row_count int32 [n] or None -> (len int32 [n], cu_rows int32 [n + 1], slots, positions int32 [rows_cap],
    state int32 [4]).  `slots` and `positions` may be given (their length is then rows_cap; entries behind the last row
    stay, so a step over the whole buffers gives odb_qk_norm_rope row_end=cu_rows[n:]); buffers of this call's own hold -1 there.
    `out` = (len, cu_rows, state) may be given too."""
    torch = _torch or _load_torch()
    index, n, i32, (rows, columns) = held.get_device(), held.numel(), torch.int32, tables.shape if tables.dim() == 2 else (-1, -1)
    if rows != n:
        _not_ints("tables", "[n, columns]")
    if slots is None and positions is None:
        slots, positions = held.new_full((2, rows_cap), -1).unbind()
    elif slots is None:
        slots = held.new_full((rows_cap,), -1)
    cap = slots.numel()
    if positions is None:
        positions = held.new_full((cap,), -1)
    per = (n,)
    p_held = _ints("held", held, per, index, i32)
    if out is None:
        own = held.new_empty((2 * n + 5,))
        length, cu_rows, state = torch.split_with_sizes(own, (n, n + 1, 4))
        p_len = own.data_ptr()
        p_rows, p_state = p_len + 4 * n, p_len + 4 * (2 * n + 1)
    else:
        length, cu_rows, state = out
        p_len, p_rows, p_state = _ints("len", length, per, index, i32), _ints("cu_rows", cu_rows, (n + 1,), index, i32), _ints("state", state, (4,), index, i32)
    _on(index, lib().odb_page_tables, p_held, _ints("wanted", wanted, per, index, i32), n, page_size, _ints("tables", tables, (n, columns), index, i32),
        columns, _ints("free_pages", free_pages, (n_pages,), index, i32), n_pages, _ints("n_free", n_free, (1,), index, i32),
        None if row_first is None else _ints("row_first", row_first, per, index, i32),
        None if row_count is None else _ints("row_count", row_count, per, index, i32), p_len, p_rows, _ints("slots", slots, (cap,), index, i32),
        _ints("positions", positions, (cap,), index, i32), cap, p_state)
    return length, cu_rows, slots, positions, state


def odb_rope_table(n_pos: int, rot_dim: int, base: float, scaling: str = "plain", factor: float = 1.0, original_len: int = 0,
                   beta_fast: float = 32.0, beta_slow: float = 1.0, magnitude: float = 0.0, out=None, device=None):
    """-> float32 [n_pos, rot_dim / 2, 2] of (cos, sin).  scaling: "plain", "linear", "ntk" or "yarn"."""
    torch = _torch or _load_torch()
    if scaling not in ROPE_SCALINGS:
        raise ValueError("scaling is one of %s" % (ROPE_SCALINGS,))
    shape = (n_pos, rot_dim // 2, 2)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=device if device is not None else "cuda")
    elif out.dtype is not torch.float32 or out.shape != shape or not out.is_contiguous():
        raise TypeError("out must be a contiguous float32 tensor of shape %s" % (shape,))
    r = odb_rope(base, ROPE_SCALINGS.index(scaling), factor, original_len, beta_fast, beta_slow, magnitude)
    _on(out.get_device(), lib().odb_rope_table, out.data_ptr(), n_pos, rot_dim, ctypes.byref(r))
    return out


def odb_qk_norm_rope(q, k, v, k_pages, v_pages, table, positions, slots, q_gain=None, k_gain=None, eps: float = 1e-6,
                     interleaved: bool = False, out=None, row_end=None):
    """q [rows, n_heads, head_dim], k and v [rows, n_kv_heads, head_dim], float32 or the pools' dtype, rows of any stride (three
    parts of one buffer, say); k_pages, v_pages [n_pages, n_kv_heads, page_size, head_dim]; table float32 [n_pos, rot_dim / 2, 2];
    positions, slots int32 [rows]; gains float32 [head_dim] -> queries [rows, n_heads, head_dim] in the pools' dtype.  K/V of
    the rows go to the pools.  out may be q.  row_end int32 [1]: rows from this one on are padding."""
    torch = _torch or _load_torch()
    index, pages, dtype, i32, f32 = q.get_device(), _pages(k_pages, v_pages), q.dtype, torch.int32, torch.float32
    shape = rows, heads, dim = q.shape
    kv = (rows, k_pages.shape[1], dim)
    if k_pages.get_device() != index or dim != k_pages.shape[3] or dtype not in _DTYPES:
        raise TypeError("q and the pools must lie on one device and have heads of the same size, of float16, bfloat16 or float32")
    if out is None:
        out, out_row = q.new_empty(shape, dtype=k_pages.dtype), heads * dim
    else:
        out_row = _head_rows("out", out, index, k_pages.dtype, shape)
    if table.dtype is not f32 or table.dim() != 3 or table.shape[2] != 2 or table.get_device() != index or not table.is_contiguous():
        raise TypeError("table must be a contiguous float32 tensor [n_pos, rot_dim / 2, 2] on the device of the others")
    for gain in (q_gain, k_gain):
        if gain is not None and (gain.dtype is not f32 or gain.shape != (dim,) or gain.get_device() != index or not gain.is_contiguous()):
            raise TypeError("q_gain and k_gain must be contiguous float32 tensors [head_dim] on the device of the others")
    r = _PACK_QK_ROWS(q.data_ptr(), k.data_ptr(), v.data_ptr(), _DTYPES[dtype], rows, heads, _head_rows("q", q, index, dtype, shape),
                      _head_rows("k", k, index, dtype, kv), _head_rows("v", v, index, dtype, kv), 0 if q_gain is None else q_gain.data_ptr(),
                      0 if k_gain is None else k_gain.data_ptr(), eps, table.data_ptr(), table.shape[0], 2 * table.shape[1], bool(interleaved),
                      _ints("positions", positions, (rows,), index, i32), _ints("slots", slots, (rows,), index, i32), out.data_ptr(),
                      out_row, 0 if row_end is None else _ints("row_end", row_end, (1,), index, i32))
    if rows:
        _on(index, lib().odb_qk_norm_rope, r, pages)
    return out


def odb_paged_attention_workspace(attention, pages) -> int:
    """Of an odb_attention and odb_pages, or their bytes."""
    n = lib().odb_paged_attention_workspace(*(x if isinstance(x, bytes) else ctypes.byref(x) for x in (attention, pages)))
    if n < 0:
        _check(n)
    return n


def odb_paged_attention(q, k_pages, v_pages, tables, kv_len, *, causal: bool, cu_rows=None, first_pos=None, scale: Optional[float] = None,
                        window: int = 0, sinks: int = 0, max_rows: int = 0, max_len: int = 0, out=None, workspace=None):
    """q [rows, n_heads, head_dim] of the pages' dtype; tables int32 [n, columns]; kv_len int32 [n]; cu_rows int32 [n + 1] (None:
    one row per request); first_pos int32 [n] (None: the rows are the last positions); scale defaults to head_dim ** -0.5
    -> [rows, n_heads, head_dim].  max_rows and max_len, bounds of a request's rows and positions, choose the way of computing: give
    max_rows=1 for single tokens.  The workspace comes from torch's allocator unless a uint8 tensor is given."""
    _torch or _load_torch()
    pages = _pages(k_pages, v_pages)
    return _attention(odb_paged_attention_workspace, lib().odb_paged_attention, q, k_pages, pages, k_pages.dtype, tables, kv_len, causal, cu_rows, first_pos,
                      scale, window, sinks, max_rows, max_len, out, workspace)


def _attention(workspace_of, call, q, k_pages, pages, dtype, tables, kv_len, causal, cu_rows, first_pos, scale, window, sinks, max_rows, max_len, out, workspace):
    torch = _torch
    index, i32 = q.get_device(), torch.int32
    shape = rows, heads, dim = q.shape
    if k_pages.get_device() != index or dim != k_pages.shape[3]:
        raise TypeError("q and the pools must lie on one device and have heads of the same size")
    if tables.dim() != 2:
        _not_ints("tables", "[n, columns]")
    n, columns = tables.shape
    if cu_rows is None and rows != n:
        raise ValueError("without cu_rows every request has one row (%d rows, %d requests)" % (rows, n))
    q_row = _head_rows("q", q, index, dtype, shape)
    if out is None:
        out, out_row = q.new_empty(shape), heads * dim
    else:
        out_row = _head_rows("out", out, index, q.dtype, shape)
    fields = (q.data_ptr(), out.data_ptr(), q_row, out_row,
              0 if cu_rows is None else _ints("cu_rows", cu_rows, (n + 1,), index, i32),
              0 if first_pos is None else _ints("first_pos", first_pos, (n,), index, i32), _ints("kv_len", kv_len, (n,), index, i32),
              _ints("tables", tables, (n, columns), index, i32), columns, n, rows, heads, dim ** -0.5 if scale is None else scale, bool(causal),
              window, sinks, max_rows, max_len)
    if workspace is not None and (workspace.dtype is not torch.uint8 or workspace.get_device() != index or not workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous uint8 tensor on the device of the others")
    if rows == 0:
        return out
    a = _PACK_ATTENTION(*fields, 0, 0)
    need = workspace_of(a, pages)
    if need:
        if workspace is None:
            workspace = q.new_empty((need,), dtype=torch.uint8)
        a = _PACK_ATTENTION(*fields, workspace.data_ptr(), workspace.numel())
    _on(index, call, a, pages)
    return out


def _refuse_quant_pages(k_pages, v_pages, k_scale, v_scale):
    """Says what is wrong with pools that _quant_pages does not take."""
    strides = k_pages.stride()
    if len(strides) != 4 or v_pages.shape != k_pages.shape or v_pages.stride() != strides or strides[3] != 1:
        raise TypeError("k_pages and v_pages must be [n_pages, n_kv_heads, page_size, head_dim] with the same strides, the last one 1")
    if v_pages.dtype is not k_pages.dtype or v_pages.get_device() != k_pages.get_device() or k_pages.dtype not in _CODES:
        raise TypeError("k_pages and v_pages must be int8 or float8_e4m3fn, of one dtype and device")
    if any(t.dtype is not _torch.float32 or t.get_device() != k_pages.get_device() for t in (k_scale, v_scale)):
        raise TypeError("k_scale and v_scale must be float32, on the device of the codes")
    raise TypeError("k_scale and v_scale must be [n_pages, n_kv_heads, page_size / group] with the same strides, the last one 1")


def _quant_pages(k_pages, v_pages, k_scale, v_scale, index, dtype=0):
    """Pools of codes [n_pages, n_kv_heads, page_size, head_dim], int8 or float8_e4m3fn, and their scales, float32 [n_pages, n_kv_heads,
    page_size / group], all on device `index`, as a packed odb_quant_pages.  (One expression where all is well: what a call of a few rows
    takes is mostly this side of it.)"""
    shape, strides, s_shape, s_strides, codes, f32 = k_pages.shape, k_pages.stride(), k_scale.shape, k_scale.stride(), _CODES.get(k_pages.dtype), _torch.float32
    if (codes is None or len(shape) != 4 or v_pages.shape != shape or v_pages.stride() != strides or strides[3] != 1 or v_pages.dtype is not k_pages.dtype
            or len(s_shape) != 3 or v_scale.shape != s_shape or v_scale.stride() != s_strides or k_scale.dtype is not f32 or v_scale.dtype is not f32
            or s_shape[0] != shape[0] or s_shape[1] != shape[1] or s_shape[2] < 1 or shape[2] % s_shape[2] or (s_strides[2] != 1 and s_shape[2] != 1)
            or not k_pages.get_device() == v_pages.get_device() == k_scale.get_device() == v_scale.get_device()):
        _refuse_quant_pages(k_pages, v_pages, k_scale, v_scale)
    if k_pages.get_device() != index:
        raise TypeError("the pools and the other tensors must lie on one device")
    n_pages, heads, page, dim = shape
    return _PACK_QUANT_PAGES(k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), n_pages, page, heads, dim, codes,
                             page // s_shape[2], dtype, strides[0], strides[1], strides[2], s_strides[0], s_strides[1])


def odb_qk_norm_rope_quant(q, k, v, k_pages, v_pages, k_scale, v_scale, table, positions, tables, kv_len, *, cu_rows=None, first_pos=None, q_gain=None,
                           k_gain=None, eps: float = 1e-6, interleaved: bool = False, dtype=None, out=None, odd=None):
    """odb_qk_norm_rope into pages of 8-bit codes: k_pages, v_pages int8 or float8_e4m3fn [n_pages, n_kv_heads, page_size, head_dim], their
    scales float32 [n_pages, n_kv_heads, page_size / group].  The requests as in odb_paged_attention: tables int32 [n, columns], kv_len int32 [n]
    (with the rows), cu_rows int32 [n + 1] (None: one row per request), first_pos int32 [n] (None: the rows are the last positions); positions
    int32 [rows] are those of the angles -> queries [rows, n_heads, head_dim] of `dtype`, float16 or bfloat16 (that of out, or of q, where none
    is given).  odd int32 [1] becomes 1 where a value that is not finite was stored."""
    torch = _torch or _load_torch()
    index, given, i32, f32 = q.get_device(), q.dtype, torch.int32, torch.float32
    if dtype is None:
        dtype = out.dtype if out is not None else given
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise TypeError("queries become float16 or bfloat16: give dtype")
    stream = _here(index)
    if stream is not None:
        calls = _calls
        got = calls[1].store(calls[2], stream, index, q, k, v, k_pages, v_pages, k_scale, v_scale, table, positions, tables, kv_len, cu_rows, first_pos,
                             q_gain, k_gain, eps, interleaved, dtype is torch.bfloat16, out, odd)
        if got is not None:
            return _made(got)
    pages = _quant_pages(k_pages, v_pages, k_scale, v_scale, index, _DTYPES[dtype])
    shape = rows, heads, dim = q.shape
    kv = (rows, k_pages.shape[1], dim)
    if dim != k_pages.shape[3] or given not in _DTYPES:
        raise TypeError("q and the pools must have heads of the same size, q of float16, bfloat16 or float32")
    if tables.dim() != 2:
        _not_ints("tables", "[n, columns]")
    n, columns = tables.shape
    if cu_rows is None and rows != n:
        raise ValueError("without cu_rows every request has one row (%d rows, %d requests)" % (rows, n))
    if out is None:
        out, out_row = q.new_empty(shape, dtype=dtype), heads * dim
    else:
        out_row = _head_rows("out", out, index, dtype, shape)
    t_shape = table.shape
    if table.dtype is not f32 or len(t_shape) != 3 or t_shape[2] != 2 or table.get_device() != index or not table.is_contiguous():
        raise TypeError("table must be a contiguous float32 tensor [n_pos, rot_dim / 2, 2] on the device of the others")
    for gain in (q_gain, k_gain):
        if gain is not None and (gain.dtype is not f32 or gain.shape != (dim,) or gain.get_device() != index or not gain.is_contiguous()):
            raise TypeError("q_gain and k_gain must be contiguous float32 tensors [head_dim] on the device of the others")
    per = (n,)
    r = _PACK_QUANT_ROWS(q.data_ptr(), k.data_ptr(), v.data_ptr(), _DTYPES[given], rows, heads, _head_rows("q", q, index, given, shape),
                         _head_rows("k", k, index, given, kv), _head_rows("v", v, index, given, kv), 0 if q_gain is None else q_gain.data_ptr(),
                         0 if k_gain is None else k_gain.data_ptr(), eps, table.data_ptr(), t_shape[0], 2 * t_shape[1], bool(interleaved),
                         _ints("positions", positions, (rows,), index, i32), out.data_ptr(), out_row,
                         0 if cu_rows is None else _ints("cu_rows", cu_rows, (n + 1,), index, i32),
                         0 if first_pos is None else _ints("first_pos", first_pos, per, index, i32), _ints("kv_len", kv_len, per, index, i32),
                         _ints("tables", tables, (n, columns), index, i32), columns, n, 0 if odd is None else _ints("odd", odd, (1,), index, i32))
    if rows:
        _on(index, lib().odb_qk_norm_rope_quant, r, pages)
    return out


def odb_paged_read_quant(k_pages, v_pages, k_scale, v_scale, slots, dtype=None, out=None):
    """Values at slots int32 [rows] (outside the pool: zeros) -> (k, v), each [rows, n_kv_heads, head_dim] of dtype float16 (the default),
    bfloat16 or float32, or `out` = (k, v)."""
    torch = _torch or _load_torch()
    index = slots.get_device()
    stream = _here(index)
    if stream is not None and out is None:
        calls = _calls
        got = calls[1].read(calls[3], stream, index, k_pages, v_pages, k_scale, v_scale, slots, _DTYPES.get(dtype, -1) if dtype is not None else 0)
        if got is not None:
            return _made(got)
    pages = _quant_pages(k_pages, v_pages, k_scale, v_scale, index)
    if out is not None:
        dtype = out[0].dtype
    elif dtype is None:
        dtype = torch.float16
    if dtype not in _DTYPES:
        raise TypeError("values are read as float16, bfloat16 or float32")
    rows, (_, heads, _, dim) = slots.numel(), k_pages.shape
    if out is None:
        shape = (rows, heads, dim)
        k, v = slots.new_empty(shape, dtype=dtype), slots.new_empty(shape, dtype=dtype)
        k_row = v_row = heads * dim
    else:
        k, v = out
        k_row, v_row = (_head_rows(name, t, index, dtype, torch.Size((rows, heads, dim))) for name, t in (("out[0]", k), ("out[1]", v)))
    p_slots = _ints("slots", slots, (rows,), index, torch.int32)
    if rows:
        _on(index, lib().odb_paged_read_quant, pages, p_slots, rows, _DTYPES[dtype], k.data_ptr(), v.data_ptr(), k_row, v_row)
    return k, v


def odb_paged_attention_quant_workspace(attention, pages) -> int:
    """Of an odb_attention and odb_quant_pages, or their bytes."""
    n = lib().odb_paged_attention_quant_workspace(*(x if isinstance(x, bytes) else ctypes.byref(x) for x in (attention, pages)))
    if n < 0:
        _check(n)
    return n


def odb_paged_attention_quant(q, k_pages, v_pages, k_scale, v_scale, tables, kv_len, *, causal: bool, cu_rows=None, first_pos=None,
                              scale: Optional[float] = None, window: int = 0, sinks: int = 0, max_rows: int = 0, max_len: int = 0, out=None, workspace=None):
    """odb_paged_attention over pages of 8-bit codes (see odb_qk_norm_rope_quant); q float16 or bfloat16."""
    torch = _torch or _load_torch()
    if q.dtype is not torch.bfloat16 and q.dtype is not torch.float16:
        raise TypeError("q must be float16 or bfloat16")
    index = q.get_device()
    stream = _here(index)
    if stream is not None:
        calls = _calls
        got = calls[1].attention(calls[4], calls[5], stream, index, q, k_pages, v_pages, k_scale, v_scale, tables, kv_len, cu_rows, first_pos,
                                 k_pages.shape[3] ** -0.5 if scale is None else scale, causal, window, sinks, max_rows, max_len, out, workspace)
        if got is not None:
            return _made(got)
    pages = _quant_pages(k_pages, v_pages, k_scale, v_scale, index, _DTYPES[q.dtype])
    return _attention(odb_paged_attention_quant_workspace, lib().odb_paged_attention_quant, q, k_pages, pages, q.dtype, tables, kv_len, causal, cu_rows,
                      first_pos, scale, window, sinks, max_rows, max_len, out, workspace)


def odb_step_paged(model: int, tokens, k_pages, v_pages, tables, first_pos, kv_len, positions, slots, table, tau: Optional[float] = None,
                   skip: int = 0, head: bool = True, max_len: int = 0):
    """tokens int32 [n, b]; k_pages, v_pages float16 [n_layers, n_pages, n_heads, page_size, head_dim]; tables int32 [n, columns];
    first_pos, kv_len int32 [n]; positions, slots int32 [n * b]; table float32 [n_pos, head_dim / 2, 2] -> (conf f32, argmax int32,
    each [n, b - skip], unmask uint8 [n, b] or None): unmask with a threshold tau only; all None with head=False."""
    _torch or _load_torch()
    r, outs = _paged_rows(tokens, k_pages, v_pages, tables, first_pos, kv_len, positions, slots, table, tau, skip, head, max_len)
    _on(tokens.get_device(), lib().odb_step_paged, model, ctypes.byref(r), _pages(k_pages[0], v_pages[0]))
    return outs


def odb_step_paged_quant(model: int, tokens, k_pages, v_pages, k_scale, v_scale, tables, first_pos, kv_len, positions, table, tau: Optional[float] = None,
                         skip: int = 0, head: bool = True, max_len: int = 0):
    """odb_step_paged over pages of 8-bit codes: k_pages, v_pages int8 or float8_e4m3fn [n_layers, n_pages, n_heads, page_size, head_dim],
    k_scale, v_scale float32 [n_layers, n_pages, n_heads, page_size / group]."""
    _torch or _load_torch()
    r, outs = _paged_rows(tokens, k_pages, v_pages, tables, first_pos, kv_len, positions, None, table, tau, skip, head, max_len)
    if k_scale.dim() != 4 or k_scale.shape != v_scale.shape or k_scale.stride() != v_scale.stride() or k_scale.shape[0] != k_pages.shape[0]:
        raise TypeError("k_scale and v_scale must be [n_layers, n_pages, n_heads, page_size / group] with the same strides")
    index = tokens.get_device()
    pages = _quant_pages(k_pages[0], v_pages[0], k_scale[0], v_scale[0], index)
    _on(index, lib().odb_step_paged_quant, model, ctypes.byref(r), pages, k_scale.stride(0))
    return outs


def _paged_rows(tokens, k_pages, v_pages, tables, first_pos, kv_len, positions, slots, table, tau, skip, head, max_len):
    """An odb_paged_rows, and what it writes: (conf, argmax, unmask)."""
    torch = _torch
    index, i32 = tokens.get_device(), torch.int32
    n, b = tokens.shape
    if k_pages.dim() != 5 or k_pages.shape != v_pages.shape or k_pages.stride() != v_pages.stride() or k_pages.get_device() != index:
        raise TypeError("k_pages and v_pages must be [n_layers, n_pages, n_heads, page_size, head_dim] with the same strides, on the device of the others")
    if table.dtype is not torch.float32 or table.dim() != 3 or tuple(table.shape[1:]) != (k_pages.shape[4] // 2, 2) or table.get_device() != index or not table.is_contiguous():
        raise TypeError("table must be a contiguous float32 tensor [n_pos, head_dim / 2, 2] on the device of the others")
    if tables.dim() != 2:
        _not_ints("tables", "[n, columns]")
    if not 0 <= skip < b:
        raise ValueError("skip=%d outside [0, %d)" % (skip, b))
    conf = argmax = unmask = None
    if head:
        conf, argmax = tokens.new_empty((n, b - skip), dtype=torch.float32), tokens.new_empty((n, b - skip))
        unmask = None if tau is None else tokens.new_empty((n, b), dtype=torch.uint8)
    r = odb_paged_rows(_ints("tokens", tokens, (n, b), index, i32), n, b, _ints("first_pos", first_pos, (n,), index, i32),
                       _ints("kv_len", kv_len, (n,), index, i32), _ints("tables", tables, (n, tables.shape[1]), index, i32), tables.shape[1],
                       _ints("positions", positions, (n * b,), index, i32), 0 if slots is None else _ints("slots", slots, (n * b,), index, i32), table.data_ptr(),
                       table.shape[0],
                       k_pages.stride(0), skip, max_len, 0.0 if tau is None else tau, *(None if t is None else t.data_ptr() for t in (conf, argmax, unmask)),
                       k_pages.shape[0])
    return r, (conf, argmax, unmask)


def odb_set_option(model: int, option: int, value: int) -> None:
    _check(lib().odb_set_option(model, option, value))


def odb_model_status(model: int) -> None:
    _check(lib().odb_model_status(model))


def odb_profile_begin(model: int, kernel_class: int, max_launches: int) -> None:
    _check(lib().odb_profile_begin(model, kernel_class, max_launches))


def odb_profile_end(model: int) -> Tuple[int, float, float]:
    """-> (timed launches, sum of their event-pair durations in ms, sum of the empty pairs recorded behind them)."""
    n, ms, empty = ctypes.c_int(), ctypes.c_float(), ctypes.c_float()
    _check(lib().odb_profile_end(model, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(empty)))
    return n.value, ms.value, empty.value


def odb_profile_kernel(model: int, run, steps: int, kernel_class: int = 3, max_launches: int = 1 << 16) -> Dict:
    """Average on-stream duration of one kernel class over `steps` calls of run()."""
    odb_profile_begin(model, kernel_class, max_launches)
    try:
        for _ in range(steps):
            run()
    finally:
        n, ms, empty = odb_profile_end(model)
    return {"kernel": KERNEL_CLASSES[kernel_class], "launches": n, "avg_ms": ms / max(n, 1),
            "avg_empty_pair_ms": empty / max(n, 1)}


def bf16_bits_to_f32(bits: np.ndarray) -> np.ndarray:
    """Widening of bf16 bit patterns (pure reinterpretation, no arithmetic)."""
    return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32)
