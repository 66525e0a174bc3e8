"""ctypes binding of liblookahead.so: argument marshalling only.

The functions carry the C names (la_init_model, la_kv_alloc, la_forward_layers,
la_unembed_argmax, la_ngram_accept, ...).  torch is used for device memory and
streams; every step of the path runs inside the library's kernels.  Importing
this module fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from operator import index

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblookahead.so")

LA_MAX_ROWS = 64
LA_F32, LA_BF16, LA_F16 = 0, 1, 2


class LaError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"liblookahead error {code}: {text}")
        self.code = code


class la_model_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float), ("dtype", C.c_int32)]


class la_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown", "g_attn", "g_mlp")]


class la_lookahead_desc(C.Structure):
    _fields_ = [("W", C.c_int32), ("N", C.c_int32), ("G", C.c_int32)]


class la_step_state(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("L", "c0", "n_cand", "Bp", "steps", "matched_steps", "n_emitted", "last_emitted",
                 "last_k", "last_m", "error", "reserved")] + \
               [("tok", C.c_int32 * LA_MAX_ROWS), ("pos", C.c_int32 * LA_MAX_ROWS),
                ("vis", C.c_uint64 * LA_MAX_ROWS), ("win", C.c_int32 * LA_MAX_ROWS),
                ("cand", C.c_int32 * LA_MAX_ROWS)]


class la_sampling(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p", "u", "u_index")] + [("n_u", C.c_int32)]


class la_adjust(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("req", "repetition", "presence", "frequency", "tokens", "n_tokens", "n_prompt", "draft", "first", "vis", "bias_token", "bias", "allowed",
                                          "allowed_index")] + \
               [(n, C.c_int64) for n in ("tokens_stride", "bias_stride", "allowed_stride")] + [(n, C.c_int32) for n in ("n_requests", "max_tokens", "n_bias", "n_allowed")]


class la_pages_desc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)] + \
               [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")]


class la_profile_entry(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int32), ("total_ms", C.c_float)]


STATE_BYTES = C.sizeof(la_step_state)
STATE_OFF = {n: getattr(la_step_state, n).offset for n, _ in la_step_state._fields_}

EXPORTS = [
    "la_init_model", "la_model_set_layer", "la_free_model", "la_kv_alloc", "la_kv_set_len", "la_kv_get_len",
    "la_kv_fill", "la_kv_read", "la_free_kv", "la_embed", "la_forward_layers", "la_unembed_argmax",
    "la_unembed_argmax_noalloc", "la_unembed_logits", "la_sample", "la_sample_workspace", "la_page_map", "la_paged_write", "la_paged_attend",
    "la_paged_attend_workspace", "la_forward_paged", "la_paged_copy", "la_tree_layout", "la_paged_tree_attend", "la_paged_tree_attend_workspace",
    "la_forward_tree", "la_tree_accept", "la_logits_adjust", "la_causal_layout", "la_set_barrier_timeout",
    "la_prefill", "la_jacobi_init", "la_jacobi_accept", "la_rtt_fixed_overhead", "la_rtt_project", "la_jacobi_project",
    "la_pool_alloc", "la_free_pool", "la_state_init", "la_ngram_accept", "la_lookahead_layout",
    "la_profile_enable", "la_profile_select", "la_profile_read", "la_profile_copy", "la_last_error",
]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2602_16760_amd.build` "
            "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
    sig = {
        "la_init_model": (i32, [C.POINTER(la_model_desc), C.POINTER(la_layer_weights), vp, vp, vp, vp, C.POINTER(vp)]),
        "la_model_set_layer": (i32, [vp, i32, C.POINTER(la_layer_weights), vp]),
        "la_free_model": (None, [vp]),
        "la_kv_alloc": (i32, [vp, i32, C.POINTER(vp)]),
        "la_kv_set_len": (i32, [vp, i32, vp]),
        "la_kv_get_len": (i32, [vp, C.POINTER(i32), vp]),
        "la_kv_fill": (i32, [vp, i32, i32, vp, vp, i32, vp]),
        "la_kv_read": (i32, [vp, i32, i32, i32, vp, vp, vp]),
        "la_free_kv": (None, [vp]),
        "la_embed": (i32, [vp, vp, i32, vp, vp]),
        "la_forward_layers": (i32, [vp, i32, i32, vp, i32, vp, vp, vp, vp]),
        "la_unembed_argmax": (i32, [vp, vp, i32, vp, vp, vp]),
        "la_unembed_argmax_noalloc": (i32, [vp, vp, i32, vp, vp, vp]),
        "la_unembed_logits": (i32, [vp, vp, i32, vp, i64, vp]),
        "la_sample_workspace": (C.c_size_t, [i32, i32]),
        "la_sample": (i32, [vp, i32, i64, i32, i32, vp, vp, vp, vp, C.c_size_t, vp]),
        "la_page_map": (i32, [vp, vp, i32, i32, vp, i64, i32, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp]),
        "la_paged_write": (i32, [vp, i32, vp, vp, i64, i64, vp, i32, vp]),
        "la_paged_attend_workspace": (C.c_size_t, [vp, i32, i32, i32]),
        "la_paged_attend": (i32, [vp, i32, vp, i64, i32, f32, vp, i64, i32, i32, vp, vp, i32, vp, i64, vp, C.c_size_t, vp]),
        "la_forward_paged": (i32, [vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, i64, i32, i32, vp]),
        "la_paged_copy": (i32, [vp, i32, i32, vp, vp, i32, i32, vp]),
        "la_tree_layout": (i32, [vp, vp, vp, i32, i32, vp, vp, vp]),
        "la_paged_tree_attend_workspace": (C.c_size_t, [vp, i32, i32, i32, i32]),
        "la_paged_tree_attend": (i32, [vp, i32, vp, i64, i32, f32, vp, i64, i32, i32, vp, vp, vp, i32, i32, vp, i64, vp, C.c_size_t, vp]),
        "la_forward_tree": (i32, [vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, i64, i32, i32, vp]),
        "la_tree_accept": (i32, [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]),
        "la_logits_adjust": (i32, [vp, i32, i64, i32, i32, vp, vp, i64, vp]),
        "la_pool_alloc": (i32, [i32, i32, i32, C.POINTER(vp)]),
        "la_free_pool": (None, [vp]),
        "la_state_init": (i32, [vp, vp, C.POINTER(la_lookahead_desc), vp, i32, i32, i32, vp, vp]),
        "la_ngram_accept": (i32, [vp, vp, C.POINTER(la_lookahead_desc), vp, vp, vp, i32, vp]),
        "la_prefill": (i32, [vp, vp, vp, i32, i32, vp]),
        "la_jacobi_init": (i32, [vp, i32, vp, i32, i32, vp, vp]),
        "la_jacobi_accept": (i32, [vp, i32, vp, vp, vp, i32, vp]),
        "la_lookahead_layout": (i32, [C.POINTER(la_lookahead_desc), i32, i32, i32, C.POINTER(C.c_int32), C.POINTER(C.c_uint64)]),
        "la_causal_layout": (i32, [i32, i32, C.POINTER(C.c_int32), C.POINTER(C.c_uint64)]),
        "la_set_barrier_timeout": (i32, [vp, C.c_uint]),
        "la_rtt_fixed_overhead": (i32, [C.c_double, C.c_double, C.POINTER(C.c_double)]),
        "la_rtt_project": (i32, [C.c_double, C.c_double, C.c_double, C.POINTER(C.c_double)]),
        "la_jacobi_project": (i32, [i32, C.c_double, C.c_double, C.POINTER(C.c_double)]),
        "la_profile_enable": (i32, [i32]),
        "la_profile_select": (i32, [C.c_char_p]),
        "la_profile_read": (i32, [C.POINTER(la_profile_entry), i32]),
        "la_profile_copy": (i32, [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
        "la_last_error": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def _check(rc):
    if rc != 0:
        raise LaError(rc, lib.la_last_error().decode())


_torch = torch._C


def _stream(stream=None):
    """Handle of `stream`, of the current stream without one.  (The stream object that torch.cuda.current_stream() makes for it
    costs 2.9 us, more than half of a launch, and torch.cuda.current_device() looks for the runtime's start first; a call of a small
    kernel waits for the host.  Both names are looked up here: a torch built without a GPU has neither, and the host functions need none.)"""
    if stream is None:
        return _torch._cuda_getCurrentRawStream(_torch._cuda_getDevice())
    return stream.cuda_stream


def _ptr(t):
    if t is None:
        return 0
    assert t.is_cuda and t.is_contiguous(), "device pointer arguments must be contiguous CUDA tensors"
    return t.data_ptr()


def to_device(a: np.ndarray) -> torch.Tensor:
    """numpy array -> device tensor with the same bytes (uint16/uint64 travel as int16/int64)."""
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    elif a.dtype == np.uint64:
        a = a.view(np.int64)
    elif a.dtype == np.uint32:
        a = a.view(np.int32)
    return torch.from_numpy(a).cuda()


def make_desc(shape) -> la_model_desc:
    return la_model_desc(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                         shape.d_ffn, shape.vocab, shape.rms_eps, shape.rope_theta,
                         {"f32": LA_F32, "bf16": LA_BF16, "f16": LA_F16}[shape.dtype])


def _layer_struct(w: dict) -> la_layer_weights:
    return la_layer_weights(*[_ptr(w[k]) for k in ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown", "g_attn", "g_mlp")])


class _Model(C.c_void_p):
    """A la_model handle and the widths of its rows."""
    d_model = vocab = None


# ---- thin wrappers, one per C entry point ---------------------------------------------
def la_init_model(shape, embed=None, g_final=None, unembed=None, stream=None):
    """Creates an empty model (layers are added with la_model_set_layer).  Returns the handle."""
    out = _Model()
    out.d_model, out.vocab = shape.d_model, shape.vocab
    d = make_desc(shape)
    _check(lib.la_init_model(C.byref(d), None, _ptr(embed), _ptr(g_final), _ptr(unembed), _stream(stream), C.byref(out)))
    return out


def la_model_set_layer(model, layer: int, w: dict, stream=None):
    s = _layer_struct(w)
    _check(lib.la_model_set_layer(model, layer, C.byref(s), _stream(stream)))


def la_free_model(model):
    lib.la_free_model(model)


def la_kv_alloc(model, max_len: int):
    out = C.c_void_p()
    _check(lib.la_kv_alloc(model, max_len, C.byref(out)))
    return out


def la_kv_set_len(kv, L: int, stream=None):
    _check(lib.la_kv_set_len(kv, L, _stream(stream)))


def la_kv_get_len(kv, stream=None) -> int:
    v = C.c_int(0)
    _check(lib.la_kv_get_len(kv, C.byref(v), _stream(stream)))
    return v.value


def la_kv_fill(kv, layer, row0, k, v, stream=None):
    _check(lib.la_kv_fill(kv, layer, row0, _ptr(k), _ptr(v), k.shape[0], _stream(stream)))


def la_kv_read(kv, layer, row0, n, k_out, v_out, stream=None):
    _check(lib.la_kv_read(kv, layer, row0, n, _ptr(k_out), _ptr(v_out), _stream(stream)))


def la_free_kv(kv):
    lib.la_free_kv(kv)


def la_embed(model, tok, hidden, stream=None):
    _check(lib.la_embed(model, _ptr(tok), hidden.shape[0], _ptr(hidden), _stream(stream)))


def la_forward_layers(model, layer_begin, layer_end, hidden, pos, vis, kv, stream=None):
    assert hidden.dtype == torch.float32 and pos.dtype == torch.int32 and vis.dtype == torch.int64
    _check(lib.la_forward_layers(model, layer_begin, layer_end, _ptr(hidden), hidden.shape[0], _ptr(pos), _ptr(vis),
                                 kv, _stream(stream)))


def la_unembed_argmax(model, hidden, ids, top2=None, stream=None):
    assert ids.dtype == torch.int32
    _check(lib.la_unembed_argmax(model, _ptr(hidden), hidden.shape[0], _ptr(ids), _ptr(top2), _stream(stream)))


def la_unembed_argmax_noalloc(model, hidden, ids, top2=None, stream=None):
    assert ids.dtype == torch.int32
    _check(lib.la_unembed_argmax_noalloc(model, _ptr(hidden), hidden.shape[0], _ptr(ids), _ptr(top2), _stream(stream)))


# ---- sampling and the shared cache: operators on plain tensors, of any model or none ---------------------
_DTYPES = {torch.float32: LA_F32, torch.bfloat16: LA_BF16, torch.float16: LA_F16}
_F32, _I32, _I64 = torch.float32, torch.int32, torch.int64


def _refuse(text):
    raise LaError(-1, text)


def _here(t, name):
    """Index of the current device, on which every tensor of the call has to be: the launch goes to one of its streams."""
    device = t.get_device()
    if device < 0 or device != _torch._cuda_getDevice():
        _refuse(f"{name} is on {t.device}, not on the current CUDA device")
    return device


def _array(t, name, dtype, shape, device):
    """Address of a contiguous array of that type and shape on that device."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        _refuse(f"{name}: need a contiguous {dtype} tensor of shape {tuple(shape)} on device {device}, got {t.dtype}, {tuple(t.shape)}, strides {t.stride()} on {t.device}")
    return t.data_ptr()


def _optional(t, name, dtype, shape, device):
    return None if t is None else _array(t, name, dtype, shape, device)


def _workspace(size, like, stream):
    """Memory for one call, out of the memory of the stream that runs it: what that stream did with it before is through when the call starts, and nobody
    is given it before the call is through.  (The current stream's may still be written by that stream.)"""
    if stream is None:
        return torch.empty(size, dtype=torch.uint8, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(size, dtype=torch.uint8, device=like.device)


def la_unembed_logits(model, hidden, logits, stream=None):
    """logits: float32 [Bp, vocab], rows may be strided."""
    device = _here(hidden, "hidden")
    n, V = hidden.shape[0], model.vocab
    if logits.get_device() != device or logits.dtype is not _F32 or logits.shape != (n, V) or (logits.stride(1) != 1 and V > 1):
        _refuse(f"logits: need float32 [{n}, {V}] with contiguous rows on device {device}, got {logits.dtype}, {tuple(logits.shape)}, strides {logits.stride()} on {logits.device}")
    _check(lib.la_unembed_logits(model, _array(hidden, "hidden", _F32, (n, model.d_model), device), n, logits.data_ptr(), logits.stride(0) if n > 1 else V, _stream(stream)))


@functools.lru_cache(maxsize=256)
def _sample_bytes(B, V):
    return lib.la_sample_workspace(B, V)


def la_sample(logits, u, ids, prob=None, temperature=None, top_k=None, top_p=None, min_p=None, u_index=None, stream=None):
    """ids[b] = a token of row b of logits [B, V] (float32, bfloat16 or float16, rows may be strided), drawn by u[b] (with u_index: by
    u[u_index[b]]).  temperature, top_p, min_p: float32 [B] or None; top_k, u_index: int32 [B] or None; prob: float32 [B] or None."""
    device = _here(logits, "logits")
    if logits.dim() != 2 or logits.dtype not in _DTYPES or (logits.stride(1) != 1 and logits.shape[1] > 1):
        _refuse("logits: need [B, V] of float32, bfloat16 or float16 with contiguous rows")
    B, V = logits.shape
    n = (B,)
    if u.dim() != 1:
        _refuse("u: need a float32 array")
    how = la_sampling(_optional(temperature, "temperature", _F32, n, device), _optional(top_k, "top_k", _I32, n, device), _optional(top_p, "top_p", _F32, n, device),
                      _optional(min_p, "min_p", _F32, n, device), _array(u, "u", _F32, n if u_index is None else u.shape, device), _optional(u_index, "u_index", _I32, n, device),
                      u.shape[0])
    size = _sample_bytes(B, V)
    ws = _workspace(size, logits, stream)
    _check(lib.la_sample(logits.data_ptr(), _DTYPES[logits.dtype], logits.stride(0) if B > 1 else V, B, V, C.byref(how), _array(ids, "ids", _I32, n, device),
                         _optional(prob, "prob", _F32, n, device), ws.data_ptr(), size, _stream(stream)))


def _lists(t, name, dtype, device, rows=None):
    """Address, row stride, number and length of lists [rows, n] (their rows may be strided)."""
    if t.dtype is not dtype or t.get_device() != device or t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (t.stride(1) != 1 and t.shape[1] > 1):
        _refuse(f"{name}: need {dtype} [{'n' if rows is None else rows}, n] with contiguous rows on device {device}, got {t.dtype}, {tuple(t.shape)}, strides {t.stride()} on {t.device}")
    R, n = t.shape
    return t.data_ptr(), t.stride(0) if R > 1 else n, R, n


def la_logits_adjust(logits, out, req=None, repetition=None, presence=None, frequency=None, tokens=None, n_tokens=None, n_prompt=None, draft=None, first=None, vis=None, bias=None,
                     bias_token=None, allowed=None, allowed_index=None, n_requests=None, stream=None):
    """out [B, V] = logits [B, V] (float32, bfloat16 or float16, rows may be strided; out may be logits) with penalties, biases and masks: see la.h.  repetition, presence, frequency:
    float32 [R]; tokens int32 [R, max_tokens] with n_tokens, n_prompt int32 [R]; draft int32 [B] with first int32 [R + 1] and vis int64 [B]; bias float32 [R, n_bias] with bias_token int32 of the
    same shape; allowed int32 [n_masks, ceil(V / 32)] with allowed_index int32 [B]; req int32 [B].  n_requests: R, where none of the arrays says it."""
    device = _here(logits, "logits")
    for t, name in ((logits, "logits"), (out, "out")):
        if t.dim() != 2 or t.dtype not in _DTYPES or (t.stride(1) != 1 and t.shape[1] > 1):
            _refuse(f"{name}: need [B, V] of float32, bfloat16 or float16 with contiguous rows")
    if out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != device:
        _refuse(f"out: need {logits.dtype} {tuple(logits.shape)} on device {device}, got {out.dtype}, {tuple(out.shape)} on {out.device}")
    B, V = logits.shape
    n = (B,)
    R = n_requests
    if R is None:
        of = repetition if repetition is not None else presence if presence is not None else frequency if frequency is not None else tokens if tokens is not None else bias
        R = of.shape[0] if of is not None and of.dim() else first.shape[0] - 1 if first is not None and first.dim() else B
    r = (R,)
    tokens_p = tokens_ld = most = lens_p = prompt_p = draft_p = first_p = vis_p = token_p = bias_p = bias_ld = n_bias = allowed_p = allowed_ld = n_allowed = index_p = 0
    if tokens is not None:
        tokens_p, tokens_ld, _, most = _lists(tokens, "tokens", _I32, device, R)
        lens_p, prompt_p = _optional(n_tokens, "n_tokens", _I32, r, device), _optional(n_prompt, "n_prompt", _I32, r, device)
    if draft is not None:
        draft_p, first_p, vis_p = _array(draft, "draft", _I32, n, device), _optional(first, "first", _I32, (R + 1,), device), _optional(vis, "vis", _I64, n, device)
    if bias is not None or bias_token is not None:
        if bias is None or bias_token is None or bias.shape != bias_token.shape:
            _refuse("bias, bias_token: need both, of one shape")
        bias_p, bias_ld, _, n_bias = _lists(bias, "bias", _F32, device, R)
        token_p, ld, _, _ = _lists(bias_token, "bias_token", _I32, device, R)
        if ld != bias_ld:
            _refuse("bias, bias_token: need rows of one stride")
    if allowed is not None:
        allowed_p, allowed_ld, n_allowed, words = _lists(allowed, "allowed", _I32, device)
        if words != (V + 31) // 32:
            _refuse(f"allowed: need {(V + 31) // 32} words a mask, got {words}")
        index_p = _optional(allowed_index, "allowed_index", _I32, n, device)
    how = la_adjust(_optional(req, "req", _I32, n, device), _optional(repetition, "repetition", _F32, r, device), _optional(presence, "presence", _F32, r, device),
                    _optional(frequency, "frequency", _F32, r, device), tokens_p, lens_p, prompt_p, draft_p, first_p, vis_p, token_p, bias_p, allowed_p, index_p, tokens_ld, bias_ld, allowed_ld,
                    R, most, n_bias, n_allowed)
    _check(lib.la_logits_adjust(logits.data_ptr(), _DTYPES[logits.dtype], logits.stride(0) if B > 1 else V, B, V, C.byref(how), out.data_ptr(), out.stride(0) if B > 1 else V,
                                _stream(stream)))


class la_pages:
    """Pages of K and V, both [n_layers, n_pages, n_kv_heads, page_size, head_dim], and the descriptor that calls on them take."""

    def __init__(self, k, v):
        if k.dim() != 5 or k.dtype not in _DTYPES or not k.is_cuda or not k.is_contiguous():
            _refuse("k: need a contiguous CUDA tensor [n_layers, n_pages, n_kv_heads, page_size, head_dim] of float32, bfloat16 or float16")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.get_device()
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.desc = la_pages_desc(k.data_ptr(), _array(v, "v", k.dtype, k.shape, self.device), self.n_layers, self.n_pages, self.page_size, self.n_kv_heads,
                                  self.head_dim, _DTYPES[k.dtype])
        self.ref = C.byref(self.desc)
        self._bytes = {}

    def _here(self):
        if self.device != _torch._cuda_getDevice():
            _refuse(f"the pages are on device {self.device}, not on the current CUDA device")
        return self.device

    def _rows(self, t, name, n, heads):
        """Address and row stride of [n, heads, head_dim] rows of the pages' type (the stride of a dimension of one says nothing)."""
        s = t.stride()
        if t.dtype is not self.dtype or t.get_device() != self.device or t.shape != (n, heads, self.head_dim) or s[2] != 1 or (s[1] != self.head_dim and heads > 1):
            _refuse(f"{name}: need {self.dtype} [{n}, {heads}, {self.head_dim}] with contiguous rows on device {self.device}, got {t.dtype}, {tuple(t.shape)}, strides {s} on {t.device}")
        return t.data_ptr(), s[0] if n > 1 else heads * self.head_dim

    def _tree_bytes(self, heads, blocks, requests, rows):
        """Workspace of a trees' attention call, by its sizes."""
        key = (heads, blocks, requests, rows)
        size = self._bytes.get(key)
        if size is None:
            size = self._bytes[key] = lib.la_paged_tree_attend_workspace(self.ref, heads, blocks, requests, rows)
        return size

    def _attend_bytes(self, heads, blocks, rows):
        """Workspace of an attention call, by its sizes."""
        key = (heads, blocks, rows)
        size = self._bytes.get(key)
        if size is None:
            size = self._bytes[key] = lib.la_paged_attend_workspace(self.ref, heads, blocks, rows)
        return size


def _table(table, device):
    if table.dtype is not _I32 or table.get_device() != device or table.dim() != 2 or (table.stride(1) != 1 and table.shape[1] > 1):
        _refuse(f"table: need int32 [n_requests, max_blocks] with contiguous rows on device {device}")
    R, blocks = table.shape
    return table.data_ptr(), table.stride(0) if R > 1 else blocks, R, blocks


def la_page_map(old_len, new_len, page_size, table, ring, heads_in, heads_out, slot, pos, req, first, stream=None):
    """Pages and slots of the requests' new tokens: see la.h.  All int32: old_len, new_len [R], table [R, max_blocks], ring [n_pages],
    heads_in, heads_out [4] = {head, free pages, rows, error}, slot, pos, req [max_rows], first [R + 1]."""
    device = _here(old_len, "old_len")
    tp, ld, R, blocks = _table(table, device)
    n, rows, n_pages = (R,), slot.shape, ring.numel()
    if slot.dim() != 1:
        _refuse("slot: need an int32 array")
    _check(lib.la_page_map(_array(old_len, "old_len", _I32, n, device), _array(new_len, "new_len", _I32, n, device), R, page_size, tp, ld, blocks,
                           _array(ring, "ring", _I32, (n_pages,), device), n_pages, _array(heads_in, "heads_in", _I32, (4,), device),
                           _array(heads_out, "heads_out", _I32, (4,), device), _array(slot, "slot", _I32, rows, device), _array(pos, "pos", _I32, rows, device),
                           _array(req, "req", _I32, rows, device), rows[0], _array(first, "first", _I32, (R + 1,), device), _stream(stream)))


def la_paged_write(pages, layer, k, v, slot, stream=None):
    """Rows of k, v [n, n_kv_heads, head_dim] (the rows themselves may be strided) into the slots slot [n] of one layer."""
    device, n = pages._here(), k.shape[0]
    kp, ldk = pages._rows(k, "k", n, pages.n_kv_heads)
    vp, ldv = pages._rows(v, "v", n, pages.n_kv_heads)
    _check(lib.la_paged_write(pages.ref, layer, kp, vp, ldk, ldv, _array(slot, "slot", _I32, (n,), device), n, _stream(stream)))


def la_paged_attend(pages, layer, q, table, req, pos, out, scale=None, stream=None):
    """out[b] = attention of q[b] over positions 0 .. pos[b] of request req[b] (None: request b); q, out [B, n_q_heads, head_dim], rows may be
    strided; scale None: head_dim ** -0.5."""
    device = pages._here()
    if q.dim() != 3:
        _refuse("q: need [B, n_q_heads, head_dim]")
    B, Hq, dh = q.shape
    qp, ldq = pages._rows(q, "q", B, Hq)
    op, ldo = pages._rows(out, "out", B, Hq)
    if B > 1 and ldo < Hq * dh:
        _refuse("out: rows overlap")
    tp, ld, R, blocks = _table(table, device)
    size = pages._attend_bytes(Hq, blocks, B)
    ws = _workspace(size, q, stream) if size else None
    _check(lib.la_paged_attend(pages.ref, layer, qp, ldq, Hq, dh ** -0.5 if scale is None else scale, tp, ld, R, blocks, _optional(req, "req", _I32, (B,), device),
                               _array(pos, "pos", _I32, (B,), device), B, op, ldo, ws.data_ptr() if size else None, size, _stream(stream)))


def la_paged_copy(pages, from_slot, to_slot, run=None, layers=None, stream=None):
    """K and V of slots from_slot to slots to_slot (int32, of one shape) in layers = (begin, end), None: all.  Two dimensions: each row is a run, whose sources are all read before one of its
    destinations is written; else runs of `run` (None: 1)."""
    device, n = pages._here(), from_slot.numel()
    if run is None:
        run = from_slot.shape[1] if from_slot.dim() == 2 else 1
    begin, end = (0, pages.n_layers) if layers is None else layers
    _check(lib.la_paged_copy(pages.ref, begin, end, _array(from_slot, "from_slot", _I32, from_slot.shape, device), _array(to_slot, "to_slot", _I32, from_slot.shape, device), n,
                             run if n else 1, _stream(stream)))


def la_tree_layout(parent, first, len, pos, vis, stream=None):
    """Positions and masks of the requests' trees: parent int32 [B], first int32 [R + 1], len int32 [R], pos int32 [B], vis int64 [B]."""
    device = _here(parent, "parent")
    n, R = parent.shape, len.numel()
    if parent.dim() != 1:
        _refuse("parent: need an int32 array")
    _check(lib.la_tree_layout(_array(parent, "parent", _I32, n, device), _array(first, "first", _I32, (R + 1,), device), _array(len, "len", _I32, (R,), device), R, n[0],
                              _array(pos, "pos", _I32, n, device), _array(vis, "vis", _I64, n, device), _stream(stream)))


def la_paged_tree_attend(pages, layer, q, table, first, len, vis, max_rows, out, scale=None, stream=None):
    """out[i] = attention of q[i], row i - first[r] of request r's block, over its len[r] committed positions and the block's rows of vis[i] (int64 [B]); q, out [B, n_q_heads, head_dim], rows
    may be strided; first int32 [R + 1], len int32 [R]; max_rows: rows of a request at most; scale None: head_dim ** -0.5."""
    device = pages._here()
    if q.dim() != 3:
        _refuse("q: need [B, n_q_heads, head_dim]")
    B, Hq, dh = q.shape
    qp, ldq = pages._rows(q, "q", B, Hq)
    op, ldo = pages._rows(out, "out", B, Hq)
    if B > 1 and ldo < Hq * dh:
        _refuse("out: rows overlap")
    tp, ld, R, blocks = _table(table, device)
    size = pages._tree_bytes(Hq, blocks, R, max_rows)
    ws = _workspace(size, q, stream) if size else None
    _check(lib.la_paged_tree_attend(pages.ref, layer, qp, ldq, Hq, dh ** -0.5 if scale is None else scale, tp, ld, R, blocks, _array(first, "first", _I32, (R + 1,), device),
                                    _array(len, "len", _I32, (R,), device), _array(vis, "vis", _I64, (B,), device), max_rows, B, op, ldo, ws.data_ptr() if size else None, size,
                                    _stream(stream)))


def la_tree_accept(parent, tok, ids, slot, first, len, n_new, new_len, last, out, from_slot, to_slot, limit=None, stream=None):
    """The path that each request commits: see la.h.  All int32: parent, tok, ids, slot [B], first [R + 1], len, limit (or None), n_new, new_len, last [R], out, from_slot, to_slot
    [R, max_path]."""
    device = _here(parent, "parent")
    n, R = parent.shape, len.numel()
    if parent.dim() != 1 or out.dim() != 2:
        _refuse("parent, out: need int32 [B] and [R, max_path]")
    r, path = (R,), (R, out.shape[1])
    _check(lib.la_tree_accept(_array(parent, "parent", _I32, n, device), _array(tok, "tok", _I32, n, device), _array(ids, "ids", _I32, n, device), _array(slot, "slot", _I32, n, device),
                              _array(first, "first", _I32, (R + 1,), device), _array(len, "len", _I32, r, device), _optional(limit, "limit", _I32, r, device), R, n[0], path[1],
                              _array(n_new, "n_new", _I32, r, device), _array(new_len, "new_len", _I32, r, device), _array(last, "last", _I32, r, device),
                              _array(out, "out", _I32, path, device), _array(from_slot, "from_slot", _I32, path, device), _array(to_slot, "to_slot", _I32, path, device), _stream(stream)))


def la_forward_paged(model, layer_begin, layer_end, hidden, pos, req, slot, pages, table, stream=None):
    """One token each of several requests through the layers: hidden float32 [B, d_model] in place, pos, req (None: row b is request b), slot int32 [B]."""
    device = pages._here()
    n = (hidden.shape[0],)
    tp, ld, R, blocks = _table(table, device)
    _check(lib.la_forward_paged(model, layer_begin, layer_end, _array(hidden, "hidden", _F32, (n[0], model.d_model), device), n[0], _array(pos, "pos", _I32, n, device), _optional(req, "req", _I32, n, device),
                                _array(slot, "slot", _I32, n, device), pages.ref, tp, ld, R, blocks, _stream(stream)))


def la_forward_tree(model, layer_begin, layer_end, hidden, pos, vis, slot, first, len, max_rows, pages, table, stream=None):
    """Rows of the requests' blocks through the layers: hidden float32 [B, d_model] in place, pos, slot int32 [B], vis int64 [B], first int32 [R + 1], len int32 [R]; max_rows: rows of a request
    at most."""
    device = pages._here()
    n = (hidden.shape[0],)
    tp, ld, R, blocks = _table(table, device)
    _check(lib.la_forward_tree(model, layer_begin, layer_end, _array(hidden, "hidden", _F32, (n[0], model.d_model), device), n[0], _array(pos, "pos", _I32, n, device),
                               _array(vis, "vis", _I64, n, device), _array(slot, "slot", _I32, n, device), _array(first, "first", _I32, (R + 1,), device), _array(len, "len", _I32, (R,), device),
                               max_rows, pages.ref, tp, ld, R, blocks, _stream(stream)))


def la_pool_alloc(vocab, N, G):
    out = C.c_void_p()
    _check(lib.la_pool_alloc(vocab, N, G, C.byref(out)))
    return out


def la_free_pool(pool):
    lib.la_free_pool(pool)


@functools.lru_cache(maxsize=64)
def _lookahead(W, N, G):
    """Reference to a descriptor, which the library only reads.  It is kept by three Python integers, the numbers that a call's arguments hold
    (operator.index): an argument itself may change in place (a 0-d tensor, whose hash is its identity) or have no hash (a 0-d array)."""
    return C.byref(la_lookahead_desc(W, N, G))


def la_state_init(pool, kv, W, N, G, prompt, Bp, seed_pool, state, stream=None):
    _check(lib.la_state_init(pool, kv, _lookahead(index(W), index(N), index(G)), _ptr(prompt), prompt.shape[0], Bp, int(seed_pool), _ptr(state),
                             _stream(stream)))


def la_ngram_accept(pool, kv, W, N, G, ids, state, emitted, max_total, stream=None):
    _check(lib.la_ngram_accept(pool, kv, _lookahead(index(W), index(N), index(G)), _ptr(ids), _ptr(state), _ptr(emitted), max_total, _stream(stream)))


def la_prefill(model, kv, tok, L0=0, stream=None):
    assert tok.dtype == torch.int32
    _check(lib.la_prefill(model, kv, _ptr(tok), tok.shape[0], L0, _stream(stream)))


def la_jacobi_init(kv, k, prompt, Bp, state, stream=None):
    _check(lib.la_jacobi_init(kv, k, _ptr(prompt), prompt.shape[0], Bp, _ptr(state), _stream(stream)))


def la_jacobi_accept(kv, k, ids, state, emitted, max_total, stream=None):
    _check(lib.la_jacobi_accept(kv, k, _ptr(ids), _ptr(state), _ptr(emitted), max_total, _stream(stream)))


def la_lookahead_layout(W, N, G, t, n_cand, Bp):
    """Host helper -> (pos int32[Bp], vis uint64[Bp]) numpy arrays."""
    d = la_lookahead_desc(W, N, G)
    pos = (C.c_int32 * Bp)()
    vis = (C.c_uint64 * Bp)()
    _check(lib.la_lookahead_layout(C.byref(d), t, n_cand, Bp, pos, vis))
    return np.array(pos, dtype=np.int32), np.array(vis, dtype=np.uint64)


def la_causal_layout(t, n):
    """Host helper -> (pos int32[n], vis uint64[n]) numpy arrays of a causal block of n tokens at position t."""
    pos = (C.c_int32 * n)()
    vis = (C.c_uint64 * n)()
    _check(lib.la_causal_layout(t, n, pos, vis))
    return np.array(pos, dtype=np.int32), np.array(vis, dtype=np.uint64)


def la_set_barrier_timeout(model, polls):
    _check(lib.la_set_barrier_timeout(model, polls))


def la_rtt_fixed_overhead(per_step_ms, rtt_ms) -> float:
    out = C.c_double(0.0)
    _check(lib.la_rtt_fixed_overhead(per_step_ms, rtt_ms, C.byref(out)))
    return out.value


def la_rtt_project(tokens_per_step, rtt_ms, fixed_ms) -> float:
    out = C.c_double(0.0)
    _check(lib.la_rtt_project(tokens_per_step, rtt_ms, fixed_ms, C.byref(out)))
    return out.value


def la_jacobi_project(k, iterations, rtt_ms) -> float:
    out = C.c_double(0.0)
    _check(lib.la_jacobi_project(k, iterations, rtt_ms, C.byref(out)))
    return out.value


def la_profile_enable(on: bool):
    _check(lib.la_profile_enable(int(on)))


def la_profile_select(name):
    _check(lib.la_profile_select(name.encode() if name else None))


def la_profile_read(cap=64):
    buf = (la_profile_entry * cap)()
    n = lib.la_profile_read(buf, cap)
    return {buf[i].name.decode(): (buf[i].launches, buf[i].total_ms) for i in range(n)}


def la_profile_copy(dst: torch.Tensor, src: torch.Tensor):
    _check(lib.la_profile_copy(dst.data_ptr(), src.data_ptr(), src.numel() * src.element_size(), _stream()))


# ---- state helpers (views of the published struct layout) ------------------------------
def new_state() -> torch.Tensor:
    return torch.zeros(STATE_BYTES, dtype=torch.uint8, device="cuda")


def state_field(state: torch.Tensor, name: str) -> torch.Tensor:
    """Device view of one field of la_step_state (no copy)."""
    off = STATE_OFF[name]
    if name == "vis":
        return state[off:off + 8 * LA_MAX_ROWS].view(torch.int64)
    if name in ("tok", "pos", "win", "cand"):
        return state[off:off + 4 * LA_MAX_ROWS].view(torch.int32)
    return state[off:off + 4].view(torch.int32)


def read_state(state: torch.Tensor) -> la_step_state:
    raw = bytes(state.cpu().numpy().tobytes())
    return la_step_state.from_buffer_copy(raw)
