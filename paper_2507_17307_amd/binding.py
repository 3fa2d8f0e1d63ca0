"""ctypes binding of librstitch.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/rstitch.h).
Torch tensors are used as device buffers; what crosses the boundary is their
``data_ptr()`` and the raw handle of torch's current HIP stream.  ``Model`` is a
convenience holder that keeps the borrowed buffers alive for the lifetime of the
C handle; it adds no arithmetic.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

RS_SLM, RS_LLM = 0, 1
FLAG_HI, FLAG_ACCEPT, FLAG_NEXT_LLM, FLAG_NONFINITE, FLAG_BADARG, FLAG_ABORTED, FLAG_ROUTER_STAY, FLAG_NO_PAGE = 1, 2, 4, 8, 16, 32, 64, 128

_HERE = os.path.dirname(os.path.abspath(__file__))


def library_path() -> str:
    return os.path.join(_HERE, "librstitch.so")


class RsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"rstitch status {status}: {message}")
        self.status = status


class RsConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab",
        "tied_lm_head", "max_ctx", "max_seqs", "max_rows")] + [("rms_eps", C.c_float), ("rope_theta", C.c_float)]


class _RsWeights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p)] + [
        (n, C.POINTER(C.c_void_p)) for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")]


class _RsPagedKv(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p)] + [(n, C.c_int32) for n in (
        "n_pages", "page_size", "n_slots", "max_pages", "n_kv_heads", "head_dim")]


class _RsPagePool(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p), ("page_ref", C.c_void_p)] + [(n, C.c_int32) for n in (
        "n_layers", "n_pages", "page_size", "n_slots", "max_pages", "n_kv_heads", "head_dim")]


class _RsRope(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("d_inv_freq", C.c_void_p), ("amplitude", C.c_float)]


class _RsRouterWeights(C.Structure):
    _fields_ = [("d", C.c_int32), ("r", C.c_int32), ("ln_eps", C.c_float)] + [
        (n, C.POINTER(C.c_void_p)) for n in ("w1", "b1", "w2", "b2")] + [
        (n, C.c_void_p) for n in ("ln_gain", "ln_bias", "w_head", "b_head")]


def _load() -> C.CDLL:
    path = library_path()
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
            "or python paper_2507_17307_amd/build.py). There is no fallback path.")
    lib = C.CDLL(path)
    vp, i32, i64, f32, f64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double, C.c_size_t
    lib.rs_last_error.restype = C.c_char_p
    lib.rs_last_error.argtypes = []
    lib.rs_abi_version.restype = i32
    lib.rs_abi_version.argtypes = []
    lib.rs_workspace_bytes.restype = sz
    lib.rs_workspace_bytes.argtypes = [C.POINTER(RsConfig)]
    lib.rs_kv_bytes.restype = sz
    lib.rs_kv_bytes.argtypes = [C.POINTER(RsConfig)]
    lib.rs_create_model.restype = i32
    lib.rs_create_model.argtypes = [C.POINTER(RsConfig), C.POINTER(_RsWeights), vp, vp, vp, sz, C.POINTER(vp)]
    lib.rs_destroy_model.restype = i32
    lib.rs_destroy_model.argtypes = [vp]
    lib.rs_decode_step.restype = i32
    lib.rs_decode_step.argtypes = [vp, i32, vp, vp, vp, vp, f32, i32, vp, vp, vp]
    lib.rs_catchup_prefill.restype = i32
    lib.rs_catchup_prefill.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, f32, i32, vp, vp, vp]
    lib.rs_route_scratch_bytes.restype = sz
    lib.rs_route_scratch_bytes.argtypes = [i32, i32]
    lib.rs_route.restype = i32
    lib.rs_route.argtypes = [vp, i32, i32, vp, f32, i32, vp, vp, sz, vp]
    lib.rs_set_sampling.restype = i32
    lib.rs_set_sampling.argtypes = [vp, i32, C.c_uint64]
    lib.rs_route_plus.restype = i32
    lib.rs_route_plus.argtypes = [vp, vp, i32, C.POINTER(_RsRouterWeights), i32, vp, vp, vp]
    lib.rs_route_static.restype = i32
    lib.rs_route_static.argtypes = [vp, i32, i32, vp, f32, i32, vp, vp]
    lib.rs_stitch_generate.restype = i32
    lib.rs_stitch_generate.argtypes = [vp, vp, i32, vp, i32, i32, i32, i32, vp, f32, i32, vp, i32, vp, vp]
    lib.rs_rope_frequencies.restype = i32
    lib.rs_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp, vp]
    lib.rs_rope_rows.restype = i32
    lib.rs_rope_rows.argtypes = [C.POINTER(_RsRope), i32, vp, i32, i32, i32, vp, i64, i32, vp, i64, vp]
    lib.rs_paged_append.restype = i32
    lib.rs_paged_append.argtypes = [C.POINTER(_RsPagedKv), i32, i32, vp, vp, vp, C.POINTER(_RsRope), i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp]
    lib.rs_paged_attention_scratch_bytes.restype = sz
    lib.rs_paged_attention_scratch_bytes.argtypes = [C.POINTER(_RsPagedKv), i32, i32, i32]
    lib.rs_paged_attention.restype = i32
    lib.rs_paged_attention.argtypes = [C.POINTER(_RsPagedKv), i32, i32, vp, vp, vp, i32, i32, vp, i64, f32, i32, vp, i64, vp, vp, vp, sz, vp]
    lib.rs_paged_workspace_bytes.restype = sz
    lib.rs_paged_workspace_bytes.argtypes = [C.POINTER(RsConfig), C.POINTER(_RsPagedKv)]
    lib.rs_create_model_paged.restype = i32
    lib.rs_create_model_paged.argtypes = [C.POINTER(RsConfig), C.POINTER(_RsWeights), C.POINTER(_RsPagedKv), vp, sz, C.POINTER(vp)]
    lib.rs_beam_select_scratch_bytes.restype = sz
    lib.rs_beam_select_scratch_bytes.argtypes = [i32, i32, i32, i32]
    lib.rs_beam_select.restype = i32
    lib.rs_beam_select.argtypes = [vp, i64, i32, i32, i32, i32, vp, vp, vp, i32, f64, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    pool = C.POINTER(_RsPagePool)
    lib.rs_pages_scratch_bytes.restype = sz
    lib.rs_pages_scratch_bytes.argtypes = [pool, i32]
    lib.rs_pages_reserve.restype = i32
    lib.rs_pages_reserve.argtypes = [pool, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.rs_pages_release.restype = i32
    lib.rs_pages_release.argtypes = [pool, i32, vp, vp, vp, vp, vp]
    lib.rs_pages_fork.restype = i32
    lib.rs_pages_fork.argtypes = [pool, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.rs_pages_copy.restype = i32
    lib.rs_pages_copy.argtypes = [pool, pool, i32, vp, vp, vp, vp]
    lib.rs_pages_compact.restype = i32
    lib.rs_pages_compact.argtypes = [pool, vp, vp, sz, vp]
    lib.rs_set_spin_limit.restype = i32
    lib.rs_set_spin_limit.argtypes = [vp, C.c_uint32]
    lib.rs_set_phase_timer.restype = i32
    lib.rs_set_phase_timer.argtypes = [vp, i32, i32, vp, vp]
    return lib


lib = _load()


def _check(status: int) -> None:
    if status != 0:
        raise RsError(status, rs_last_error())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# torch.cuda.current_stream() builds a stream object (2.7 us, of a call of rs_route on 1024 logits 6.8); its raw handle alone takes 0.2
_raw_stream, _raw_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ------------------------------------------------------------------ plain entry points
def rs_last_error() -> str:
    return lib.rs_last_error().decode()


def rs_abi_version() -> int:
    return lib.rs_abi_version()


def rs_workspace_bytes(cfg: RsConfig) -> int:
    return lib.rs_workspace_bytes(C.byref(cfg))


def rs_kv_bytes(cfg: RsConfig) -> int:
    return lib.rs_kv_bytes(C.byref(cfg))


def _marshal_weights(cfg: RsConfig, weights):
    n = cfg.n_layers
    arrs = {}
    for name in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down"):
        arrs[name] = (C.c_void_p * n)(*[getattr(l, name).data_ptr() for l in weights.layers])
    return _RsWeights(weights.embed.data_ptr(), weights.lm_head.data_ptr(), weights.final_norm.data_ptr(),
                      *[C.cast(arrs[k], C.POINTER(C.c_void_p)) for k in
                        ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")])


def rs_create_model(cfg: RsConfig, weights, kv_k: torch.Tensor, kv_v: torch.Tensor,
                    workspace: torch.Tensor) -> int:
    """weights: object with embed, lm_head, final_norm and layers[*].{attn_norm,w_qkv,w_o,mlp_norm,
    w_gate_up,w_down} as contiguous bf16 device tensors.  Returns the opaque handle."""
    w = _marshal_weights(cfg, weights)
    handle = C.c_void_p()
    _check(lib.rs_create_model(C.byref(cfg), C.byref(w), kv_k.data_ptr(), kv_v.data_ptr(), workspace.data_ptr(),
                               workspace.numel() * workspace.element_size(), C.byref(handle)))
    return handle.value


def rs_paged_workspace_bytes(cfg: RsConfig, cache: _RsPagedKv) -> int:
    return lib.rs_paged_workspace_bytes(C.byref(cfg), C.byref(cache))


def rs_create_model_paged(cfg: RsConfig, weights, cache: _RsPagedKv, workspace: torch.Tensor) -> int:
    """cache: the marshalled pages of all layers (PagedModel.cache_struct)."""
    w = _marshal_weights(cfg, weights)
    handle = C.c_void_p()
    _check(lib.rs_create_model_paged(C.byref(cfg), C.byref(w), C.byref(cache), workspace.data_ptr(), workspace.numel() * workspace.element_size(), C.byref(handle)))
    return handle.value


def rs_destroy_model(handle: int) -> None:
    _check(lib.rs_destroy_model(handle))


def rs_decode_step(handle: int, n_seqs: int, d_seq_slot, d_token, d_pos, d_logit_scale, tau: float, active: int,
                   d_out, d_logits=None, stream=None) -> None:
    _check(lib.rs_decode_step(handle, n_seqs, _ptr(d_seq_slot), _ptr(d_token), _ptr(d_pos), _ptr(d_logit_scale),
                              tau, active, _ptr(d_out), _ptr(d_logits), _stream(stream)))


def rs_catchup_prefill(handle: int, n_seqs: int, n_rows: int, d_seq_slot, d_tokens, d_span_offset, d_pos0,
                       d_logit_scale, tau: float, active: int, d_out, d_logits=None, stream=None) -> None:
    _check(lib.rs_catchup_prefill(handle, n_seqs, n_rows, _ptr(d_seq_slot), _ptr(d_tokens), _ptr(d_span_offset),
                                  _ptr(d_pos0), _ptr(d_logit_scale), tau, active, _ptr(d_out), _ptr(d_logits),
                                  _stream(stream)))


def rs_route_scratch_bytes(n: int, vocab: int) -> int:
    return lib.rs_route_scratch_bytes(n, vocab)


def rs_route(d_logits, n: int, vocab: int, d_logit_scale, tau: float, active: int, d_out, d_scratch,
             stream=None) -> None:
    _check(lib.rs_route(_ptr(d_logits), n, vocab, _ptr(d_logit_scale), tau, active, _ptr(d_out), _ptr(d_scratch),
                        0 if d_scratch is None else d_scratch.numel() * d_scratch.element_size(), _stream(stream)))


def rs_route_static(d_logits, n: int, vocab: int, d_logit_scale, tau: float, active: int, d_out, stream=None) -> None:
    _check(lib.rs_route_static(_ptr(d_logits), n, vocab, _ptr(d_logit_scale), tau, active, _ptr(d_out), _stream(stream)))


class RouterPlus:
    """Marshalled rs_router_weights: keeps the device tensors and the pointer arrays alive.
    weights: object with w1, b1, w2, b2 (lists of six bf16 device tensors), ln_gain, ln_bias, w_head, b_head."""

    def __init__(self, weights, ln_eps: float = 1e-5):
        self.weights = weights
        self._arrs = {n: (C.c_void_p * 6)(*[t.data_ptr() for t in getattr(weights, n)]) for n in ("w1", "b1", "w2", "b2")}
        r, d = weights.w1[0].shape
        self.struct = _RsRouterWeights(d, r, ln_eps, *[C.cast(self._arrs[n], C.POINTER(C.c_void_p)) for n in ("w1", "b1", "w2", "b2")],
                                       weights.ln_gain.data_ptr(), weights.ln_bias.data_ptr(), weights.w_head.data_ptr(),
                                       weights.b_head.data_ptr())


def rs_route_plus(handle: Optional[int], d_hidden, n_seqs: int, router: RouterPlus, active: int, d_out,
                  d_router_logits=None, stream=None) -> None:
    """d_out: tensor or raw address of the records to update."""
    out = d_out if isinstance(d_out, int) else _ptr(d_out)
    _check(lib.rs_route_plus(handle, _ptr(d_hidden), n_seqs, C.byref(router.struct), active, out,
                             _ptr(d_router_logits), _stream(stream)))


STITCH_RUNNING, STITCH_DONE, STITCH_TRACE_FULL, STITCH_FLAGGED, STITCH_ABORTED = range(5)
STITCH_RECORD_INTS = 10     # rs_stitch_record: model, pos0, n_rows, reserved, then the 6 words of rs_route_out
STITCH_RESULT_INTS = 8      # rs_stitch_result: status, n_tokens, n_records, seen_slm, seen_llm, active, n_target, reserved


def rs_stitch_generate(slm: int, llm: int, seq_slot: int, d_seq, n_prompt: int, n_new: int, seen_slm: int,
                       seen_llm: int, d_logit_scale, tau: float, eos: int, d_trace, max_records: int, d_result,
                       stream=None) -> None:
    """d_seq: int32 tensor [n_prompt + n_new]; d_trace: int32 tensor [max_records, 10]; d_result: int32 tensor [8]."""
    _check(lib.rs_stitch_generate(slm, llm, seq_slot, _ptr(d_seq), n_prompt, n_new, seen_slm, seen_llm,
                                  _ptr(d_logit_scale), tau, eos, _ptr(d_trace), max_records, _ptr(d_result),
                                  _stream(stream)))


def rs_set_sampling(handle: int, enabled: bool, key: int = 0) -> None:
    _check(lib.rs_set_sampling(handle, int(bool(enabled)), key & 0xFFFFFFFFFFFFFFFF))


# ------------------------------------------------------------------ caches in pages
RS_F32, RS_BF16, RS_SCORES_F64 = 0, 1, 256
ROPE_PLAIN, ROPE_LINEAR, ROPE_BY_PARTS = range(3)
_ROW_TYPES = {torch.float32: RS_F32, torch.bfloat16: RS_BF16}
_INT_TYPES = (torch.int32, torch.uint32)


def _rows(name: str, t: torch.Tensor, device: int):
    """(address, row stride) of a tensor [rows, heads, channels] whose heads lie back to back; the C side checks the rest.
    (The stride of a dimension of one element says nothing: a single row's is its length.)"""
    if t.dim() != 3 or not t.is_contiguous() and (t.stride(2) != 1 or t.stride(1) != t.shape[2] and t.shape[1] != 1):
        raise ValueError(f"{name} must be [rows, heads, head_dim] with the heads of a row back to back, not {tuple(t.shape)} with strides {t.stride()}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on {_device_name(device)}")
    return t.data_ptr(), t.stride(0) if t.shape[0] != 1 else t.shape[1] * t.shape[2]


def _ints(name: str, t: Optional[torch.Tensor], n: int, device: int) -> Optional[int]:
    """Address of n 32-bit integers."""
    if t is None:
        return None
    if t.dtype is not torch.int32 and t.dtype not in _INT_TYPES or not t.is_contiguous() or t.numel() < n or t.get_device() != device:
        raise ValueError(f"{name} must hold {n} contiguous 32-bit integers on {_device_name(device)}")
    return t.data_ptr()


def _device_name(device: int) -> str:
    return "the CPU" if device < 0 else f"cuda:{device}"


def _device_stream(device: int, stream) -> Optional[int]:
    """The launch goes to the current device, which has to be the tensors' own."""
    if stream is None and _raw_stream is not None and _raw_device is not None and 0 <= device == _raw_device():
        return _raw_stream(device)
    if device < 0:
        raise ValueError("tensors must be on a GPU")
    if device != (_raw_device() if _raw_device is not None else torch.cuda.current_device()):
        raise ValueError(f"tensors are on cuda:{device}, which is not the current device")
    return _stream(stream)


class PagedCache:
    """Marshalled rs_paged_kv over one layer's tensors, which it keeps alive: k [n_pages, n_kv_heads, page_size, head_dim] and
    v [n_pages, n_kv_heads, head_dim, page_size] bf16, page_table [n_slots, max_pages] int32, all contiguous on one device."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        if k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16 or k.dim() != 4 or v.shape != (k.shape[0], k.shape[1], k.shape[3], k.shape[2]):
            raise ValueError("k must be bf16 [pages, KV heads, positions, channels], v bf16 [pages, KV heads, channels, positions]")
        if page_table.dtype != torch.int32 or page_table.dim() != 2:
            raise ValueError("page_table must be int32 [slots, pages]")
        if not (k.is_contiguous() and v.is_contiguous() and page_table.is_contiguous()) or not k.device == v.device == page_table.device:
            raise ValueError("k, v and page_table must be contiguous and on one device")
        self.k, self.v, self.page_table, self.device = k, v, page_table, k.get_device()
        self.n_kv_heads, self.page_size, self.head_dim = k.shape[1], k.shape[2], k.shape[3]
        self.struct = _RsPagedKv(k.data_ptr(), v.data_ptr(), page_table.data_ptr(), k.shape[0], k.shape[2], page_table.shape[0],
                                 page_table.shape[1], k.shape[1], k.shape[3])
        self._ref = C.byref(self.struct)


class Rope:
    """Marshalled rs_rope over its frequencies (float64 [rot_dim / 2] on the GPU), which it keeps alive."""

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, amplitude: float = 1.0):
        if inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be contiguous float64 [rot_dim / 2]")
        self.inv_freq, self.device = inv_freq, inv_freq.get_device()
        self.struct = _RsRope(2 * inv_freq.numel(), int(bool(interleaved)), inv_freq.data_ptr(), amplitude)
        self._ref = C.byref(self.struct)


def rs_rope_frequencies(rot_dim: int, theta: float, kind: int = ROPE_PLAIN, factor: float = 1.0, original_ctx: float = 32768.0,
                        beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(float64 host tensor [rot_dim / 2], amplitude)."""
    freq, amp = torch.empty(max(rot_dim, 0) // 2, dtype=torch.float64), C.c_float()
    _check(lib.rs_rope_frequencies(rot_dim, theta, kind, factor, original_ctx, beta_fast, beta_slow, freq.data_ptr() or None, C.byref(amp)))
    return freq, amp.value


def rs_rope_rows(rope: Rope, d_pos: torch.Tensor, x: torch.Tensor, out: torch.Tensor, inverse: bool = False, stream=None) -> None:
    """x, out: [rows, heads, head_dim] of one type (out may be x); d_pos: int32 [rows]."""
    dev = x.get_device()
    if x.dtype not in _ROW_TYPES or out.dtype != x.dtype or out.shape != x.shape or rope.device != dev:
        raise ValueError("x and out must be fp32 or bf16, of one type, shape and device, which is the frequencies' too")
    px, sx = _rows("x", x, dev)
    po, so = _rows("out", out, dev)
    n, heads, hd = x.shape
    _check(lib.rs_rope_rows(rope._ref, n, _ints("d_pos", d_pos, n, dev), _ROW_TYPES[x.dtype], heads, hd, px, sx, int(bool(inverse)), po, so,
                            _device_stream(dev, stream)))


def _paged_rows(name: str, t: torch.Tensor, cache: PagedCache, n_rows: int, heads: int, dtype: torch.dtype):
    """_rows of a tensor that a call on `cache` takes."""
    if t.dtype is dtype and t.dim() == 3 and t.get_device() == cache.device:
        rows, h, hd = t.shape
        if rows >= n_rows and h == heads and hd == cache.head_dim:
            stride = t.stride()
            if stride[2] == 1 and stride[1] == hd:
                return t.data_ptr(), stride[0] if rows != 1 else h * hd
    if t.dtype != dtype or t.dim() != 3 or t.shape[0] < n_rows or t.shape[1] != heads or t.shape[2] != cache.head_dim:
        raise ValueError(f"{name} must be {dtype} and at least [{n_rows}, {heads}, {cache.head_dim}], not {t.dtype} {tuple(t.shape)}")
    return _rows(name, t, cache.device)


def _paged_type(q: torch.Tensor) -> int:
    if q.dtype not in _ROW_TYPES or q.dim() != 3:
        raise ValueError(f"q must be fp32 or bf16 [rows, heads, head_dim], not {q.dtype} {tuple(q.shape)}")
    return _ROW_TYPES[q.dtype]


def rs_paged_append(cache: PagedCache, n_seqs: int, n_rows: int, d_seq_slot, d_span_offset, d_pos0, rope: Optional[Rope], q, k, v, q_out,
                    d_flags=None, stream=None) -> None:
    """q, q_out: [rows, query heads, head_dim]; k, v: [rows, KV heads, head_dim]; views of one projection's rows do."""
    dev, kind, nq, nkv = cache.device, _paged_type(q), q.shape[1], cache.n_kv_heads
    pq, sq = _paged_rows("q", q, cache, n_rows, nq, q.dtype)
    pk, sk = _paged_rows("k", k, cache, n_rows, nkv, q.dtype)
    pv, sv = _paged_rows("v", v, cache, n_rows, nkv, q.dtype)
    po, so = _paged_rows("q_out", q_out, cache, n_rows, nq, q.dtype)
    if rope is not None and rope.device != dev:
        raise ValueError(f"the frequencies are on {_device_name(rope.device)}, the cache on {_device_name(dev)}")
    _check(lib.rs_paged_append(cache._ref, n_seqs, n_rows, _ints("d_seq_slot", d_seq_slot, n_seqs, dev),
                               _ints("d_span_offset", d_span_offset, n_seqs + 1, dev), _ints("d_pos0", d_pos0, n_seqs, dev),
                               None if rope is None else rope._ref, kind, nq, pq, sq, pk, sk, pv, sv, po, so,
                               _ints("d_flags", d_flags, n_seqs, dev), _device_stream(dev, stream)))


def rs_paged_attention_scratch_bytes(cache: PagedCache, n_seqs: int, n_rows: int, n_q_heads: int) -> int:
    return lib.rs_paged_attention_scratch_bytes(cache._ref, n_seqs, n_rows, n_q_heads)


def rs_paged_attention(cache: PagedCache, n_seqs: int, n_rows: int, d_seq_slot, d_span_offset, d_pos0, q, scale: float, window: int, out, d_lse, d_scratch,
                       d_flags=None, stream=None) -> None:
    """q, out: [rows, query heads, head_dim]; d_lse: fp32 [rows, query heads] or None; d_scratch: uint8."""
    dev, kind, nq = cache.device, _paged_type(q), q.shape[1]
    pq, sq = _paged_rows("q", q, cache, n_rows, nq, q.dtype)
    po, so = _paged_rows("out", out, cache, n_rows, nq, q.dtype)
    if d_lse is not None and (d_lse.dtype != torch.float32 or not d_lse.is_contiguous() or d_lse.numel() < n_rows * nq or d_lse.get_device() != dev):
        raise ValueError(f"d_lse must be contiguous fp32 [{n_rows}, {nq}] on {_device_name(dev)}")
    if d_scratch is None or d_scratch.get_device() != dev or not d_scratch.is_contiguous():
        raise ValueError(f"d_scratch must be a contiguous tensor on {_device_name(dev)}")
    _check(lib.rs_paged_attention(cache._ref, n_seqs, n_rows, _ints("d_seq_slot", d_seq_slot, n_seqs, dev),
                                  _ints("d_span_offset", d_span_offset, n_seqs + 1, dev), _ints("d_pos0", d_pos0, n_seqs, dev), kind, nq, pq, sq,
                                  scale, window, po, so, _ptr(d_lse), _ints("d_flags", d_flags, n_seqs, dev), d_scratch.data_ptr(),
                                  d_scratch.numel() * d_scratch.element_size(), _device_stream(dev, stream)))


# ------------------------------------------------------------------ beam search
def rs_beam_select_scratch_bytes(n_groups: int, n_beams: int, vocab: int, n_out: int) -> int:
    return lib.rs_beam_select_scratch_bytes(n_groups, n_beams, vocab, n_out)


def _floats(name: str, t: Optional[torch.Tensor], n: int, device: int, kind: torch.dtype = torch.float32) -> Optional[int]:
    """Address of n numbers of a type, fp32 by default."""
    if t is None:
        return None
    if t.dtype is not kind or not t.is_contiguous() or t.numel() < n or t.get_device() != device:
        raise ValueError(f"{name} must hold {n} contiguous {kind} numbers on {_device_name(device)}")
    return t.data_ptr()


def _scratch(t: torch.Tensor, device: int):
    """(address, bytes)"""
    if t is None or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"d_scratch must be a contiguous tensor on {_device_name(device)}")
    return t.data_ptr(), t.numel() * t.element_size()


def rs_beam_select(d_logits: torch.Tensor, n_groups: int, n_beams: int, d_logit_scale, d_score, d_last, eos: int, length_penalty: float, d_len, n_out: int,
                   d_parent, d_token, d_score_out, d_len_out, d_scratch, d_flags=None, stream=None) -> None:
    """d_logits: fp32 or bf16 [rows, vocab] with the values of a row side by side, at least n_groups * n_beams rows; d_logit_scale (or None): fp32,
    d_score: fp32 or fp64, d_last, d_len (or None): int32 of a row each; d_parent, d_token, d_len_out (or None): int32, d_score_out: d_score's type, of n_groups * n_out."""
    dev, rows, n = d_logits.get_device(), n_groups * n_beams, n_groups * n_out
    if d_logits.dtype not in _ROW_TYPES or d_logits.dim() != 2 or d_logits.shape[0] < rows or d_logits.stride(1) != 1 and d_logits.shape[1] != 1:
        raise ValueError(f"d_logits must be fp32 or bf16 [{rows}, vocab] with the values of a row side by side, not {d_logits.dtype} {tuple(d_logits.shape)}")
    vocab = d_logits.shape[1]
    stride = d_logits.stride(0) if d_logits.shape[0] != 1 else vocab
    wide = d_score is not None and d_score.dtype is torch.float64
    kind = torch.float64 if wide else torch.float32
    _check(lib.rs_beam_select(d_logits.data_ptr(), stride, _ROW_TYPES[d_logits.dtype] + (RS_SCORES_F64 if wide else 0), n_groups, n_beams, vocab, _floats("d_logit_scale", d_logit_scale, rows, dev),
                              _floats("d_score", d_score, rows, dev, kind), _ints("d_last", d_last, rows, dev), eos, length_penalty, _ints("d_len", d_len, rows, dev), n_out,
                              _ints("d_parent", d_parent, n, dev), _ints("d_token", d_token, n, dev), _floats("d_score_out", d_score_out, n, dev, kind),
                              _ints("d_len_out", d_len_out, n, dev), _ints("d_flags", d_flags, rows, dev), *_scratch(d_scratch, dev), _device_stream(dev, stream)))


class PagePool:
    """Marshalled rs_page_pool over its tensors, which it keeps alive: page_table int32 [slots, pages], page_ref int32 [pages] and, for the
    calls that move what is in the pages, k [layers, pages, KV heads, positions, channels] and v [layers, pages, KV heads, channels, positions]
    bf16; all contiguous on one device."""

    def __init__(self, page_table: torch.Tensor, page_ref: torch.Tensor, page_size: int, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_ref.dtype != torch.int32 or page_ref.dim() != 1:
            raise ValueError("page_table must be int32 [slots, pages], page_ref int32 [pages]")
        if (k is None) != (v is None):
            raise ValueError("give both k and v or neither")
        tensors = [page_table, page_ref] + ([] if k is None else [k, v])
        if any(not t.is_contiguous() or t.device != page_table.device for t in tensors):
            raise ValueError("page_table, page_ref, k and v must be contiguous and on one device")
        layers = heads = hd = 0
        if k is not None:
            if k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16 or k.dim() != 5 or k.shape[1] != page_ref.shape[0] or k.shape[3] != page_size \
                    or v.shape != (k.shape[0], k.shape[1], k.shape[2], k.shape[4], k.shape[3]):
                raise ValueError("k must be bf16 [layers, pages, KV heads, page_size, channels], v bf16 [layers, pages, KV heads, channels, page_size]")
            layers, heads, hd = k.shape[0], k.shape[2], k.shape[4]
        self.page_table, self.page_ref, self.page_size, self.k, self.v, self.device = page_table, page_ref, page_size, k, v, page_table.get_device()
        self.struct = _RsPagePool(_ptr(k), _ptr(v), page_table.data_ptr(), page_ref.data_ptr(), layers, page_ref.shape[0], page_size, page_table.shape[0],
                                  page_table.shape[1], heads, hd)
        self._ref = C.byref(self.struct)


def rs_pages_scratch_bytes(pool: PagePool, n: int) -> int:
    return lib.rs_pages_scratch_bytes(pool._ref, n)


def rs_pages_reserve(pool: PagePool, n: int, d_slot, d_from, d_to, d_scratch, d_flags=None, stream=None) -> None:
    dev = pool.device
    _check(lib.rs_pages_reserve(pool._ref, n, _ints("d_slot", d_slot, n, dev), _ints("d_from", d_from, n, dev), _ints("d_to", d_to, n, dev),
                                _ints("d_flags", d_flags, n, dev), *_scratch(d_scratch, dev), _device_stream(dev, stream)))


def rs_pages_release(pool: PagePool, n: int, d_slot, d_from, d_to, d_flags=None, stream=None) -> None:
    dev = pool.device
    _check(lib.rs_pages_release(pool._ref, n, _ints("d_slot", d_slot, n, dev), _ints("d_from", d_from, n, dev), _ints("d_to", d_to, n, dev),
                                _ints("d_flags", d_flags, n, dev), _device_stream(dev, stream)))


def rs_pages_fork(pool: PagePool, n_groups: int, n_beams: int, d_slot, d_parent, d_pos, d_pos_out, d_scratch, d_flags=None, stream=None) -> None:
    dev, n = pool.device, n_groups * n_beams
    _check(lib.rs_pages_fork(pool._ref, n_groups, n_beams, _ints("d_slot", d_slot, n, dev), _ints("d_parent", d_parent, n, dev), _ints("d_pos", d_pos, n, dev),
                             _ints("d_pos_out", d_pos_out, n, dev), _ints("d_flags", d_flags, n, dev), *_scratch(d_scratch, dev), _device_stream(dev, stream)))


def rs_pages_copy(to: PagePool, source: PagePool, n: int, d_src, d_dst, d_flags=None, stream=None) -> None:
    """Pages d_src of `source` to pages d_dst of `to`."""
    dev = to.device
    if source.device != dev:
        raise ValueError(f"the pools are on {_device_name(source.device)} and {_device_name(dev)}")
    _check(lib.rs_pages_copy(to._ref, source._ref, n, _ints("d_src", d_src, n, dev), _ints("d_dst", d_dst, n, dev), _ints("d_flags", d_flags, n, dev),
                             _device_stream(dev, stream)))


def rs_pages_compact(pool: PagePool, d_used, d_scratch, stream=None) -> None:
    dev = pool.device
    _check(lib.rs_pages_compact(pool._ref, _ints("d_used", d_used, 1, dev), *_scratch(d_scratch, dev), _device_stream(dev, stream)))


PHASE_QKV, PHASE_OPROJ, PHASE_GATEUP, PHASE_DOWN, PHASE_LMHEAD, PHASE_ATTN = range(6)


def rs_set_spin_limit(handle: int, polls: int) -> None:
    _check(lib.rs_set_spin_limit(handle, polls))


def rs_set_phase_timer(handle: int, phase: int, layer: int = 0, start_event: int = 0, stop_event: int = 0) -> None:
    """start_event / stop_event: raw hipEvent_t handles (integers); phase < 0 disarms."""
    _check(lib.rs_set_phase_timer(handle, phase, layer, start_event or None, stop_event or None))


# ------------------------------------------------------------------ records
@dataclass
class RouteOut:
    token: int
    flags: int
    h_nats: float
    h_norm: float
    max_logit: float
    log_z: float

    @property
    def hi(self) -> bool:
        return bool(self.flags & FLAG_HI)

    @property
    def accept(self) -> bool:
        return bool(self.flags & FLAG_ACCEPT)


def new_route_out(n: int, device="cuda") -> torch.Tensor:
    """Device buffer for n rs_route_out records (6 x 32-bit words each)."""
    return torch.zeros(n, 6, dtype=torch.int32, device=device)


def read_route_out(buf: torch.Tensor) -> List[RouteOut]:
    host = buf.cpu()
    ints, floats = host, host.view(torch.float32)
    return [RouteOut(int(ints[i, 0]), int(ints[i, 1]) & 0xFFFFFFFF, float(floats[i, 2]), float(floats[i, 3]),
                     float(floats[i, 4]), float(floats[i, 5])) for i in range(host.shape[0])]


# ------------------------------------------------------------------ buffer holder
def make_config(shape, max_ctx: int, max_seqs: int = 1, max_rows: int = 64) -> RsConfig:
    return RsConfig(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
                    shape.vocab, int(shape.tied_lm_head), max_ctx, max_seqs, max_rows, shape.rms_eps, shape.rope_theta)


class Model:
    """Owns the device buffers a C handle borrows (weights, KV caches, workspace) and small
    staging tensors for the per-call arrays."""

    def __init__(self, weights, max_ctx: int, max_seqs: int = 1, max_rows: int = 64, device="cuda"):
        self.shape = weights.shape
        self.weights = weights                      # bf16 tensors already on `device`
        max_ctx = (max_ctx + 7) // 8 * 8            # the library wants a multiple of 8
        self.cfg = make_config(self.shape, max_ctx, max_seqs, max_rows)
        kvb, wsb = rs_kv_bytes(self.cfg), rs_workspace_bytes(self.cfg)
        if kvb == 0 or wsb == 0:
            raise RsError(-1, rs_last_error())
        self.kv_k = torch.zeros(kvb // 2, dtype=torch.bfloat16, device=device)
        self.kv_v = torch.zeros(kvb // 2, dtype=torch.bfloat16, device=device)
        self.workspace = torch.zeros(wsb, dtype=torch.uint8, device=device)
        self.device = device
        self.handle = rs_create_model(self.cfg, weights, self.kv_k, self.kv_v, self.workspace)

    def close(self) -> None:
        if self.handle:
            rs_destroy_model(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv_view(self, which: str) -> torch.Tensor:
        """[layer, slot, kv_head, position, head_dim] view of a cache (V is stored transposed)."""
        c = self.cfg
        if which == "k":
            return self.kv_k.view(c.n_layers, c.max_seqs, c.n_kv_heads, c.max_ctx, c.head_dim)
        return self.kv_v.view(c.n_layers, c.max_seqs, c.n_kv_heads, c.head_dim, c.max_ctx).transpose(3, 4)

    def _i32(self, values: Sequence[int]) -> torch.Tensor:
        return torch.tensor(list(values), dtype=torch.int32, device=self.device)

    def decode_step(self, tokens: Sequence[int], positions: Sequence[int], tau: float, active: int,
                    scales: Optional[Sequence[float]] = None, slots: Optional[Sequence[int]] = None,
                    want_logits: bool = False):
        n = len(tokens)
        slots = list(range(n)) if slots is None else slots
        out = new_route_out(n, self.device)
        logits = torch.empty(n, self.cfg.vocab, dtype=torch.float32, device=self.device) if want_logits else None
        sc = None if scales is None else torch.tensor(list(scales), dtype=torch.float32, device=self.device)
        rs_decode_step(self.handle, n, self._i32(slots), self._i32(tokens), self._i32(positions), sc, tau, active,
                       out, logits)
        return (read_route_out(out), logits) if want_logits else read_route_out(out)

    def catchup_prefill(self, spans: Sequence[Sequence[int]], pos0: Sequence[int], tau: float, active: int,
                        scales: Optional[Sequence[float]] = None, slots: Optional[Sequence[int]] = None,
                        want_logits: bool = False):
        n = len(spans)
        slots = list(range(n)) if slots is None else slots
        off = [0]
        flat: List[int] = []
        for s in spans:
            flat.extend(s)
            off.append(len(flat))
        out = new_route_out(n, self.device)
        logits = torch.empty(n, self.cfg.vocab, dtype=torch.float32, device=self.device) if want_logits else None
        sc = None if scales is None else torch.tensor(list(scales), dtype=torch.float32, device=self.device)
        rs_catchup_prefill(self.handle, n, len(flat), self._i32(slots), self._i32(flat), self._i32(off),
                           self._i32(pos0), sc, tau, active, out, logits)
        return (read_route_out(out), logits) if want_logits else read_route_out(out)

    def forward_span(self, tokens: Sequence[int], pos0: int, tau: float, active: int, scale: float = 1.0,
                     slot: int = 0, want_logits: bool = False):
        """One sequence, any span length: chunks of max_rows through rs_catchup_prefill (a single
        token goes through rs_decode_step).  Returns the router record of the last chunk."""
        tokens = list(tokens)
        res = None
        mr = self.cfg.max_rows
        for s in range(0, len(tokens), mr):
            chunk = tokens[s:s + mr]
            if len(chunk) == 1:
                res = self.decode_step(chunk, [pos0 + s], tau, active, [scale], [slot], want_logits)
            else:
                res = self.catchup_prefill([chunk], [pos0 + s], tau, active, [scale], [slot], want_logits)
        return res


class PagedModel(Model):
    """A Model whose K/V cache is a pool of n_pages pages of page_size positions that its sequence slots draw from.

    reserve(slot, positions) gives a slot the pages for its first `positions` positions (the calls do not do it by
    themselves: the tokens a call feeds need their pages before it, and a sequence without them is flagged and left as it
    is), release(slot) gives them back.  Both write the page table
    on the current stream, after which calls on that stream see it.  page_pool() hands the pages over to the calls on
    pools of pages (rs_pages_reserve and the others), for sequences that branch; reserve and release are theirs from then on."""

    def __init__(self, weights, max_ctx: int, n_pages: int, page_size: int = 64, max_seqs: int = 1, max_rows: int = 64, device="cuda"):
        self.handle = 0
        if n_pages < 1 or page_size < 1:
            raise RsError(-1, "n_pages and page_size must be at least 1")
        self.shape = s = weights.shape
        self.weights = weights
        max_ctx = (max_ctx + 7) // 8 * 8
        self.cfg = make_config(s, max_ctx, max_seqs, max_rows)
        self.page_size, self.n_pages = page_size, n_pages
        self.pages_k = torch.zeros(s.n_layers, n_pages, s.n_kv_heads, page_size, s.head_dim, dtype=torch.bfloat16, device=device)
        self.pages_v = torch.zeros(s.n_layers, n_pages, s.n_kv_heads, s.head_dim, page_size, dtype=torch.bfloat16, device=device)
        self.page_table = torch.full((max_seqs, (max_ctx + page_size - 1) // page_size), -1, dtype=torch.int32, device=device)
        self.cache_struct = _RsPagedKv(self.pages_k.data_ptr(), self.pages_v.data_ptr(), self.page_table.data_ptr(), n_pages, page_size, max_seqs,
                                       self.page_table.shape[1], s.n_kv_heads, s.head_dim)
        wsb = rs_paged_workspace_bytes(self.cfg, self.cache_struct)
        if wsb == 0:
            raise RsError(-1, rs_last_error())
        self.workspace = torch.zeros(wsb, dtype=torch.uint8, device=device)
        self.device = device
        self._free = list(range(n_pages - 1, -1, -1))
        self._held: List[List[int]] = [[] for _ in range(max_seqs)]
        self._pool: Optional[PagePool] = None
        self.search_slots = 0                                    # slots 0 .. search_slots - 1 are beam searches'
        self.handle = rs_create_model_paged(self.cfg, weights, self.cache_struct, self.workspace)

    def page_pool(self) -> PagePool:
        """The pool over this model's pages and page table, with the pages that the slots hold counted."""
        if self._pool is None:
            count = torch.zeros(self.n_pages, dtype=torch.int32)
            for held in self._held:
                count[held] = 1
            self._pool = PagePool(self.page_table, count.to(self.device), self.page_size, self.pages_k, self.pages_v)
        return self._pool

    def _host_pages(self) -> None:
        if self._pool is not None:
            raise RsError(-1, "the pages are a pool's: use rs_pages_reserve and rs_pages_release")

    def reserve(self, slot: int, positions: int) -> None:
        self._host_pages()
        if not 0 <= slot < len(self._held):
            raise RsError(-1, f"slot {slot} out of range")
        held, more = self._held[slot], (positions + self.page_size - 1) // self.page_size - len(self._held[slot])
        if positions > self.cfg.max_ctx:
            raise RsError(-2, f"{positions} positions do not fit max_ctx {self.cfg.max_ctx}")
        if more <= 0:
            return
        if more > len(self._free):
            raise RsError(-2, f"{more} pages wanted, {len(self._free)} are free")
        at = len(held)
        held.extend(self._free.pop() for _ in range(more))
        self.page_table[slot, at:len(held)] = self._i32(held[at:])

    def release(self, slot: int) -> None:
        self._host_pages()
        if not 0 <= slot < len(self._held):
            raise RsError(-1, f"slot {slot} out of range")
        held = self._held[slot]
        self.page_table[slot].fill_(-1)
        self._free.extend(reversed(held))
        held.clear()

    def kv_view(self, which: str, slot: int = 0) -> torch.Tensor:
        """[layer, kv_head, position, head_dim]: a copy of the positions of a slot's pages, in order."""
        held = self._held[slot] if self._pool is None else [p for p in self.page_table[slot].tolist() if p >= 0]
        pages = torch.tensor(held, dtype=torch.long, device=self.device)
        t = self.pages_k[:, pages] if which == "k" else self.pages_v[:, pages].transpose(3, 4)
        return t.transpose(1, 2).flatten(2, 3)
