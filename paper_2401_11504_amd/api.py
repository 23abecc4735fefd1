"""Thin ctypes binding of libtemplora.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/templora.h)
and passes device pointers of torch tensors straight through; no step of the
chunk update is computed in Python.  torch is used for device memory and the
HIP stream handle, nothing else.  If the shared library has not been built the
import of this module fails loudly: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtemplora.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2401_11504_amd.build` "
        "(the Temp-Lora path has no CPU or PyTorch fallback)")
_lib = C.CDLL(LIB_PATH)

TL_OK = 0
STATUS = {0: "TL_OK", -1: "TL_ERR_ARG", -2: "TL_ERR_SHAPE", -3: "TL_ERR_TOKEN_RANGE", -4: "TL_ERR_WINDOW",
          -5: "TL_ERR_NONFINITE", -6: "TL_ERR_DEVICE", -7: "TL_ERR_DISCARDED", -8: "TL_ERR_OOM"}
(FACTOR_A, FACTOR_B, GRAD_A, GRAD_B, M_A, M_B, V_A, V_B) = range(8)
PROJ = ("q", "k", "v", "o", "gate", "up", "down")


class TlError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class tl_model_cfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("d_head", C.c_int32),
                ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("max_tokens", C.c_int32), ("rms_eps", C.c_float),
                ("rope_base", C.c_float)]


class tl_lora_cfg(C.Structure):
    _fields_ = [("rank", C.c_int32), ("alpha", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("weight_decay", C.c_float), ("a_init_std", C.c_float), ("seed", C.c_uint64),
                ("dropout", C.c_float)]


class tl_train_cfg(C.Structure):
    _fields_ = [("n_ctx_max", C.c_int32), ("batch", C.c_int32), ("epochs", C.c_int32), ("warmup_steps", C.c_int32),
                ("lr", C.c_float)]


class tl_generate_cfg(C.Structure):
    _fields_ = [("window", C.c_int32), ("chunk", C.c_int32), ("train", tl_train_cfg)]


class tl_penalties(C.Structure):
    _fields_ = [("repetition", C.c_float), ("presence", C.c_float), ("frequency", C.c_float), ("last_n", C.c_int32)]


class tl_sampling(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float), ("seed", C.c_uint64)]


class tl_paged_mem(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("table", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("d_head", C.c_int32), ("n_seqs", C.c_int32), ("n_table", C.c_int32)]


class tl_cache8_mem(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("k_tail", C.c_void_p),
                ("v_tail", C.c_void_p), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("capacity", C.c_int32)]


_vp, _i32, _i64, _f32, _sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
_SIGS = {
    "tl_model_create": [C.POINTER(tl_model_cfg), C.POINTER(_vp), _vp, C.POINTER(_vp)],
    "tl_model_destroy": [_vp],
    "tl_lora_init": [_vp, C.POINTER(tl_lora_cfg), C.POINTER(_vp)],
    "tl_chunk_update": [_vp, _vp, _i32, _i32, _f32, C.POINTER(_f32), C.POINTER(_i32)],
    "tl_chunk_loss": [_vp, _vp, _i32, _i32, C.POINTER(_f32), C.POINTER(_i32)],
    "tl_chunk_train": [_vp, _vp, _i32, _i32, C.POINTER(tl_train_cfg), _vp, C.POINTER(_i32)],
    "tl_prefill": [_vp, _vp, _i32, C.POINTER(_i32), _vp],
    "tl_decode_step": [_vp, _i32, C.POINTER(_i32), _vp],
    "tl_kv_length": [_vp, C.POINTER(_i32)],
    "tl_generate": [_vp, _vp, _i32, _i32, C.POINTER(tl_generate_cfg), _vp, _vp, C.POINTER(_i32)],
    "tl_cache_reuse": [_vp, _i32],
    "tl_cache_8bit": [_vp, _i32],
    "tl_extend": [_vp, _vp, _i32, C.POINTER(_i32), _vp],
    "tl_get_kv": [_vp, _i32, _i32, _i32, _vp, _vp],
    "tl_set_penalties": [_vp, C.POINTER(tl_penalties)],
    "tl_set_sampling": [_vp, C.POINTER(tl_sampling)],
    "tl_set_bias": [_vp, _vp],
    "tl_set_allowed": [_vp, _vp],
    "tl_discard": [_vp],
    "tl_lora_free": [_vp],
    "tl_get_factor": [_vp, _i32, _i32, _i32, _vp, _sz],
    "tl_set_factor": [_vp, _i32, _i32, _i32, _vp, _sz],
    "tl_get_step": [_vp, C.POINTER(_i64)],
    "tl_get_nll": [_vp, _vp, _sz],
    "tl_get_dh": [_vp, _i32, _vp, _sz],
    "tl_keep_input_grad": [_vp, _i32],
    "tl_profile_enable": [_vp, _i32],
    "tl_profile_read": [_vp, C.POINTER(C.c_double), C.POINTER(_i64), C.POINTER(C.c_double)],
    "tl_layer_step": [_vp, _i32, _vp, _vp, _i32, _vp, _vp, _f32, _i32],
    "tl_linear_step": [_vp] * 5 + [_i32] * 4 + [_f32] * 6 + [_i32] + [_vp] * 6 + [_vp],
    "tl_linear_step_static": [_vp] * 5 + [_i32] * 4 + [_f32] * 6 + [_i32] + [_vp] * 6 + [_vp],
    "tl_k_gemm_nt": [_vp, _i32, _vp, _i32, _i32, _i32, _i32, _vp, _i32, _vp, _i32, _i32, _f32, _vp, _vp, _i32, _i32, _vp,
                     _sz, _vp],
    "tl_k_low_rank": [_vp, _i32, _vp, _i32, _i32, _i32, _i32, _i32, _f32, _vp, _vp, _sz, _vp],
    "tl_k_low_rank_plan": [_i32, _i32, _i32, _i32, _sz, C.c_char_p, _sz],
    "tl_k_frozen": [_vp, _i32, _vp, _i32, _i32, _i32, _i32, _vp, _i32, _vp, _i32, _i32, _i32, _vp, _vp, _i32, _i32, _vp, _sz, C.POINTER(_i32), _vp],
    "tl_k_frozen_plan": [_i32] * 5 + [_sz, _i32, C.c_char_p, _sz],
    "tl_k_gemm_nt_plan": [_i32, _i32, _i32, _i32, _sz, C.c_char_p, _sz, C.POINTER(_i32), C.POINTER(_i32)],
    "tl_k_linear_step_plan": [_i32] * 4 + [_f32, _i32, C.c_char_p, _sz],
    "tl_k_gemm_tn": [_vp, _i32, _vp, _i32, _i32, _i32, _i32, _f32, _vp, _i32, _vp],
    "tl_k_rmsnorm_fwd": [_vp, _vp, _i32, _i32, _f32, _vp, _vp],
    "tl_k_rmsnorm_bwd": [_vp, _vp, _vp, _vp, _i32, _i32, _f32, _vp, _vp, _vp],
    "tl_k_rope": [_vp, _i32, _i32, _i32, _i32, _f32, _i32, _i32, _vp],
    "tl_k_rope_table": [_vp, _i32, _i32, _i32, _i32, _f32, _i32, _i32, _vp, _sz, _vp],
    "tl_k_dropout": [_vp, _i32, _i32, _f32, C.c_uint64, _i64, _i32, _i32, _vp, _vp],
    "tl_k_swiglu_fwd": [_vp, _i32, _i32, _vp, _vp],
    "tl_k_swiglu_bwd": [_vp, _vp, _i32, _i32, _vp, _vp],
    "tl_k_gemv": [_vp, _i32, _vp, _i32, _i32, _vp, _vp, _i32, _i32, _f32, _vp, _vp, _i32, _vp],
    "tl_k_gemv_pre": [_vp, _i32, _i32, _i32, _i32, _vp, _vp, _f32, _vp, _vp, _vp, _vp],
    "tl_k_attention_decode": [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _sz, _vp],
    "tl_k_argmax": [_vp, _i32, _vp, _vp],
    "tl_k_cache8_append": [C.POINTER(tl_cache8_mem), _i32, _vp, _i32, _vp, _i32, _i32, _vp],
    "tl_k_cache8_read": [C.POINTER(tl_cache8_mem), _i32, _i32, _i32, _vp, _i32, _vp, _i32, _vp],
    "tl_k_attention_cache8": [C.POINTER(tl_cache8_mem), _i32, _vp, _i32, _i32, _i32, _vp, _i32, _vp, _sz, _vp],
    "tl_k_attention_cache8_plan": [_i32] * 5 + [_sz, C.c_char_p, _sz, C.POINTER(_i32), C.POINTER(_sz)],
    "tl_k_token_counts": [_vp, _i32, _i32, _i32, _i32, _i32, _vp, _i32, _vp],
    "tl_k_choose": [_vp, _i32, _i32, _i32, _vp, _i32, _f32, _f32, _f32, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _sz, _vp],
    "tl_k_sample": [_vp, _i32, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "tl_k_paged_append": [C.POINTER(tl_paged_mem), _vp, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _i32, _vp],
    "tl_k_attention_paged": [C.POINTER(tl_paged_mem), _vp, _i32, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _i32, _vp, _sz, _vp],
    "tl_k_attention_paged_plan": [_i32] * 6 + [_sz, C.POINTER(_i32), C.POINTER(_sz)],
    "tl_k_attention_weights": [_vp, _i32, _vp] + [_i32] * 6 + [_vp, _vp, _i32, _vp, _i32, _vp],
    "tl_k_paged_evict": [C.POINTER(tl_paged_mem), _vp, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _sz, _vp],
    "tl_k_attention_fwd": [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _i32, _vp, _vp],
    "tl_k_attention_bwd": [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp],
    "tl_k_cross_entropy": [_vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp],
    "tl_k_adamw": [_vp, _vp, _vp, _vp, _vp, _sz, _i64, _f32, _f32, _f32, _f32, _f32, _vp],
    "tl_k_embed": [_vp, _vp, _i32, _i32, _vp, _vp],
}
EXPORTS = tuple(_SIGS) + ("tl_warmup_lr", "tl_last_error", "tl_version")
for _n, _a in _SIGS.items():
    _f = getattr(_lib, _n)
    _f.argtypes = _a
    _f.restype = C.c_int
_lib.tl_warmup_lr.argtypes = [_f32, _i64, _i32]
_lib.tl_warmup_lr.restype = _f32
_lib.tl_last_error.restype = C.c_char_p
_lib.tl_version.restype = C.c_char_p


def tl_last_error() -> str:
    return _lib.tl_last_error().decode()


def tl_version() -> str:
    return _lib.tl_version().decode()


def _chk(status: int):
    if status != TL_OK:
        raise TlError(status, tl_last_error())


def _dp(t):
    """device pointer of a torch tensor (None -> NULL)"""
    if t is None:
        return None
    assert t.is_cuda and (t.dim() == 0 or t.stride(-1) == 1), "device tensor with unit inner stride expected"
    return C.c_void_p(t.data_ptr())


def current_stream_handle():
    # (torch.cuda.current_stream() builds an object: 2.8 us of every call, this 0.2)
    return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()))


# ------------------------------------------------------------------ life cycle
def tl_model_create(n_layers, d_model, n_heads, d_head, d_ffn, vocab, max_tokens, weight_tensors, rms_eps=1e-5,
                    rope_base=10000.0, stream=None):
    """weight_tensors: flat list in the order of the header (9 per layer, then embedding, final gain, lm_head;
    entries may be None where the header allows).  Returns an opaque model handle."""
    cfg = tl_model_cfg(n_layers, d_model, n_heads, d_head, d_ffn, vocab, max_tokens, rms_eps, rope_base)
    n = 9 * n_layers + 3
    assert len(weight_tensors) == n
    arr = (_vp * n)(*[(t.data_ptr() if t is not None else None) for t in weight_tensors])
    out = _vp()
    _chk(_lib.tl_model_create(C.byref(cfg), arr, stream if stream is not None else current_stream_handle(),
                              C.byref(out)))
    return out


def tl_model_destroy(model):
    _chk(_lib.tl_model_destroy(model))


def tl_lora_init(model, rank, alpha, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, a_init_std=0.02, seed=0,
                 dropout=0.0):
    cfg = tl_lora_cfg(rank, alpha, beta1, beta2, eps, weight_decay, a_init_std, seed, dropout)
    out = _vp()
    _chk(_lib.tl_lora_init(model, C.byref(cfg), C.byref(out)))
    return out


def _tok(tokens):
    a = np.ascontiguousarray(np.asarray(tokens), dtype=np.int32)
    return a, a.ctypes.data_as(_vp)


def tl_chunk_update(lora, tokens, n_ctx=0, lr=5e-5):
    """-> (loss, n_targets)"""
    a, p = _tok(tokens)
    loss, n = _f32(), _i32()
    _chk(_lib.tl_chunk_update(lora, p, a.size, n_ctx, lr, C.byref(loss), C.byref(n)))
    return loss.value, n.value


def tl_chunk_loss(lora, tokens, n_ctx=0):
    a, p = _tok(tokens)
    loss, n = _f32(), _i32()
    _chk(_lib.tl_chunk_loss(lora, p, a.size, n_ctx, C.byref(loss), C.byref(n)))
    return loss.value, n.value


def tl_chunk_train(lora, tokens, n_chunk, n_ctx_max=1024, batch=0, epochs=2, lr=5e-5, warmup_steps=0):
    """-> list of per-step losses (epochs * ceil(n_chunk / batch) of them)"""
    a, p = _tok(tokens)
    cfg = tl_train_cfg(n_ctx_max, batch, epochs, warmup_steps, lr)
    b = batch if 0 < batch < n_chunk else max(n_chunk, 1)
    losses = np.zeros(max(epochs, 1) * (-(-max(n_chunk, 1) // b)), dtype=np.float32)
    n = _i32()
    _chk(_lib.tl_chunk_train(lora, p, a.size, n_chunk, C.byref(cfg), losses.ctypes.data_as(_vp), C.byref(n)))
    return [float(x) for x in losses[:n.value]]


def tl_warmup_lr(lr, step, warmup_steps):
    return float(_lib.tl_warmup_lr(lr, step, warmup_steps))


def tl_prefill(lora, tokens, vocab=0):
    """-> (next_token, logits fp32[vocab] or None)"""
    a, p = _tok(tokens)
    nxt = _i32()
    logits = np.empty(vocab, np.float32) if vocab else None
    _chk(_lib.tl_prefill(lora, p, a.size, C.byref(nxt), logits.ctypes.data if vocab else None))
    return nxt.value, logits


def tl_decode_step(lora, token, vocab=0):
    """-> (next_token, logits fp32[vocab] or None)"""
    nxt = _i32()
    logits = np.empty(vocab, np.float32) if vocab else None
    _chk(_lib.tl_decode_step(lora, int(token), C.byref(nxt), logits.ctypes.data if vocab else None))
    return nxt.value, logits


def tl_generate(lora, prompt, n_new, window, chunk, n_ctx_max=1024, batch=0, epochs=2, lr=5e-5, warmup_steps=0):
    """-> (generated tokens int32[n_new], per-step training losses)"""
    a, p = _tok(prompt)
    cfg = tl_generate_cfg(window, chunk, tl_train_cfg(n_ctx_max, batch, epochs, warmup_steps, lr))
    out = np.zeros(max(n_new, 1), np.int32)
    b = batch if 0 < batch < chunk else max(chunk, 1)
    losses = np.zeros(max(1, (n_new // max(chunk, 1)) * max(epochs, 1) * (-(-max(chunk, 1) // b))), np.float32)
    n = _i32()
    _chk(_lib.tl_generate(lora, p, a.size, n_new, C.byref(cfg), out.ctypes.data_as(_vp), losses.ctypes.data_as(_vp),
                          C.byref(n)))
    return out[:n_new], [float(x) for x in losses[:n.value]]


def tl_cache_reuse(lora, on=True):
    _chk(_lib.tl_cache_reuse(lora, int(on)))


def tl_cache_8bit(lora, on=True):
    _chk(_lib.tl_cache_8bit(lora, int(on)))


def tl_extend(lora, tokens, vocab=0):
    """-> (next greedy token, logits of the last position or None)"""
    a, p = _tok(tokens)
    nxt = _i32()
    logits = np.empty(vocab, dtype=np.float32) if vocab else None
    _chk(_lib.tl_extend(lora, p, a.size, C.byref(nxt), logits.ctypes.data_as(_vp) if vocab else None))
    return nxt.value, logits


def tl_get_kv(lora, layer, first, n, d_model):
    """-> keys, values of tokens first .. first + n - 1: fp32 [n, d_model] each"""
    k, v = (np.empty((n, d_model), dtype=np.float32) for _ in range(2))
    _chk(_lib.tl_get_kv(lora, layer, first, n, k.ctypes.data_as(_vp), v.ctypes.data_as(_vp)))
    return k, v


def tl_set_penalties(lora, repetition=1.0, presence=0.0, frequency=0.0, last_n=0):
    """tl_set_penalties(lora) takes them off"""
    p = tl_penalties(repetition, presence, frequency, last_n)
    off = (repetition, presence, frequency) == (1.0, 0.0, 0.0)
    _chk(_lib.tl_set_penalties(lora, None if off else C.byref(p)))


def tl_set_sampling(lora, temperature=None, top_k=0, top_p=1.0, min_p=0.0, seed=0):
    """tl_set_sampling(lora) goes back to the greedy choice"""
    p = None if temperature is None else tl_sampling(temperature, top_k, top_p, min_p, seed)
    _chk(_lib.tl_set_sampling(lora, None if p is None else C.byref(p)))


def tl_set_bias(lora, bias, vocab):
    """bias: vocab numbers, or None"""
    a = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    assert a is None or a.size == vocab
    _chk(_lib.tl_set_bias(lora, None if a is None else a.ctypes.data_as(_vp)))


def tl_set_allowed(lora, allowed, vocab):
    """allowed: vocab truth values, or None"""
    if allowed is None:
        return _chk(_lib.tl_set_allowed(lora, None))
    bits = np.packbits(np.asarray(allowed, dtype=bool), bitorder="little")
    assert len(allowed) == vocab
    words = np.zeros(4 * ((vocab + 31) // 32), dtype=np.uint8)
    words[:bits.size] = bits
    _chk(_lib.tl_set_allowed(lora, words.ctypes.data_as(_vp)))


def tl_kv_length(lora):
    n = _i32()
    _chk(_lib.tl_kv_length(lora, C.byref(n)))
    return n.value


def tl_discard(lora):
    _chk(_lib.tl_discard(lora))


def tl_lora_free(lora):
    _chk(_lib.tl_lora_free(lora))


# ------------------------------------------------------------------ inspection
def tl_get_factor(lora, layer, proj, which, shape):
    out = np.empty(shape, dtype=np.float32)
    _chk(_lib.tl_get_factor(lora, layer, proj, which, out.ctypes.data_as(_vp), out.size))
    return out


def tl_set_factor(lora, layer, proj, which, values):
    a = np.ascontiguousarray(values, dtype=np.float32)
    _chk(_lib.tl_set_factor(lora, layer, proj, which, a.ctypes.data_as(_vp), a.size))


def tl_get_step(lora) -> int:
    s = _i64()
    _chk(_lib.tl_get_step(lora, C.byref(s)))
    return s.value


def tl_get_nll(lora, n_tokens):
    out = np.empty(n_tokens, dtype=np.float32)
    _chk(_lib.tl_get_nll(lora, out.ctypes.data_as(_vp), out.size))
    return out


def tl_get_dh(lora, boundary, n_tokens, d_model):
    out = np.empty((n_tokens, d_model), dtype=np.float32)
    _chk(_lib.tl_get_dh(lora, boundary, out.ctypes.data_as(_vp), out.size))
    return out


def tl_keep_input_grad(lora, on=True):
    _chk(_lib.tl_keep_input_grad(lora, int(on)))


def tl_profile_enable(lora, on=True):
    _chk(_lib.tl_profile_enable(lora, int(on)))


def tl_profile_read(lora):
    """-> (milliseconds, launches, flop) of the frozen-weight GEMM launches since the last read"""
    ms, n, fl = C.c_double(), _i64(), C.c_double()
    _chk(_lib.tl_profile_read(lora, C.byref(ms), C.byref(n), C.byref(fl)))
    return ms.value, n.value, fl.value


def tl_layer_step(lora, layer, h_in, dh_out, h_out, dh_in, lr=0.0, apply_adamw=False):
    _chk(_lib.tl_layer_step(lora, layer, _dp(h_in), _dp(dh_out), h_in.shape[0], _dp(h_out), _dp(dh_in), lr,
                            int(apply_adamw)))


def tl_linear_step(X, W, A, B, dY, s, lr, beta1, beta2, eps, weight_decay, apply_adamw, Y, dX, dA, dB, A_new, B_new,
                   stream=None):
    T, d_in = X.shape
    d_out, r = B.shape
    _chk(_lib.tl_linear_step(_dp(X), _dp(W), _dp(A), _dp(B), _dp(dY), T, d_in, d_out, r, s, lr, beta1, beta2, eps,
                             weight_decay, int(apply_adamw), _dp(Y), _dp(dX), _dp(dA), _dp(dB), _dp(A_new),
                             _dp(B_new), stream if stream is not None else current_stream_handle()))


def tl_linear_step_static(X, W, A, B, dY, s, lr, beta1, beta2, eps, weight_decay, apply_adamw, Y, dX, dA, dB, A_new,
                          B_new, stream=None):
    T, d_in = X.shape
    d_out, r = B.shape
    _chk(_lib.tl_linear_step_static(_dp(X), _dp(W), _dp(A), _dp(B), _dp(dY), T, d_in, d_out, r, s, lr, beta1, beta2, eps,
                                    weight_decay, int(apply_adamw), _dp(Y), _dp(dX), _dp(dA), _dp(dB), _dp(A_new),
                                    _dp(B_new), stream if stream is not None else current_stream_handle()))


# ------------------------------------------------------------------ single kernels (not synchronised)
def _s(stream):
    return stream if stream is not None else current_stream_handle()


def tl_k_gemm_nt(A, B, C_out, A2=None, B2=None, alpha=1.0, R=None, workspace=None, stream=None):
    M, K = A.shape
    N = B.shape[0]
    K2 = A2.shape[1] if A2 is not None else 0
    _chk(_lib.tl_k_gemm_nt(_dp(A), A.stride(0), _dp(B), B.stride(0), M, N, K, _dp(A2),
                           A2.stride(0) if A2 is not None else 0, _dp(B2), B2.stride(0) if B2 is not None else 0, K2,
                           alpha, _dp(R), _dp(C_out), C_out.stride(0), int(C_out.dtype == torch.float32),
                           _dp(workspace), workspace.numel() if workspace is not None else 0, _s(stream)))


def tl_k_low_rank(A, B, out, batch=1, alpha=1.0, workspace=None, stream=None):
    """A [M, batch K], B [batch N, K], out [M, batch N], all bf16"""
    M, K, N = A.shape[0], B.shape[1], B.shape[0] // batch
    _chk(_lib.tl_k_low_rank(_dp(A), A.stride(0), _dp(B), B.stride(0), M, N, K, batch, alpha, _dp(out), _dp(workspace),
                            workspace.numel() if workspace is not None else 0, _s(stream)))


def tl_k_low_rank_plan(M, N, K, batch=1, workspace_elems=0):
    """-> name of the tile"""
    buf = C.create_string_buffer(32)
    _chk(_lib.tl_k_low_rank_plan(M, N, K, batch, workspace_elems, buf, 32))
    return buf.value.decode()


def tl_k_frozen(A, B, out, A2=None, B2=None, R=None, batch=1, workspace=None, deferred=False, stream=None):
    """A [M, K], B [batch N, K], A2 [M, batch K2], B2 [batch N, K2]; out bf16 or fp32 [M, batch N], R fp32 of out's strides
    -> partial tiles left in the workspace (deferred), None otherwise"""
    parts = _i32(0) if deferred else None
    two = A2 is not None
    _chk(_lib.tl_k_frozen(_dp(A), A.stride(0), _dp(B), B.stride(0), A.shape[0], B.shape[0] // batch, A.shape[1], _dp(A2), A2.stride(0) if two else 0,
                          _dp(B2), B2.stride(0) if two else 0, B2.shape[1] if two else 0, batch, _dp(R), _dp(out), out.stride(0),
                          int(out.dtype == torch.float32), _dp(workspace), workspace.numel() if workspace is not None else 0,
                          C.byref(parts) if deferred else None, _s(stream)))
    return parts.value if deferred else None


def tl_k_frozen_plan(M, N, K, K2=0, batch=1, workspace_elems=0, deferred=False):
    """-> name of the tile"""
    buf = C.create_string_buffer(32)
    _chk(_lib.tl_k_frozen_plan(M, N, K, K2, batch, workspace_elems, int(deferred), buf, 32))
    return buf.value.decode()


def tl_k_gemm_nt_plan(M, N, K, K2=0, workspace_elems=0):
    """-> (configuration name, contraction split, launches)"""
    buf = C.create_string_buffer(32)
    sp, nl = _i32(0), _i32(0)
    _chk(_lib.tl_k_gemm_nt_plan(M, N, K, K2, workspace_elems, buf, 32, C.byref(sp), C.byref(nl)))
    return buf.value.decode(), sp.value, nl.value


def tl_k_linear_step_plan(T, d_in, d_out, r, s=1.0, one_by_one=False):
    """-> names of the kernels of H and dH and of the rest; one_by_one: of H, Y, dH, dX, dA, dB"""
    buf = C.create_string_buffer(128)
    _chk(_lib.tl_k_linear_step_plan(T, d_in, d_out, r, s, int(one_by_one), buf, 128))
    return buf.value.decode().split()


def tl_k_gemm_tn(P, Q, C_out, alpha=1.0, stream=None):
    T, Mo = P.shape
    No = Q.shape[1]
    _chk(_lib.tl_k_gemm_tn(_dp(P), P.stride(0), _dp(Q), Q.stride(0), T, Mo, No, alpha, _dp(C_out), C_out.stride(0),
                           _s(stream)))


def tl_k_rmsnorm_fwd(h, g, eps, y, stream=None):
    _chk(_lib.tl_k_rmsnorm_fwd(_dp(h), _dp(g), h.shape[0], h.shape[1], eps, _dp(y), _s(stream)))


def tl_k_rmsnorm_bwd(dy, h, g, dres, eps, dh_out, dh_out_bf16=None, stream=None):
    _chk(_lib.tl_k_rmsnorm_bwd(_dp(dy), _dp(h), _dp(g), _dp(dres), h.shape[0], h.shape[1], eps, _dp(dh_out),
                               _dp(dh_out_bf16), _s(stream)))


def tl_k_rope(x, n_heads, d_head, base=10000.0, pos0=0, sign=1, stream=None):
    _chk(_lib.tl_k_rope(_dp(x), x.stride(0), x.shape[0], n_heads, d_head, base, pos0, sign, _s(stream)))


def tl_k_rope_table(x, n_heads, d_head, table, base=10000.0, pos0=0, sign=1, stream=None):
    _chk(_lib.tl_k_rope_table(_dp(x), x.stride(0), x.shape[0], n_heads, d_head, base, pos0, sign, _dp(table),
                              table.numel(), _s(stream)))


def tl_k_dropout(x, y, p, seed, step, layer, group, stream=None):
    _chk(_lib.tl_k_dropout(_dp(x), x.shape[0], x.shape[1], p, seed, step, layer, group, _dp(y), _s(stream)))


def tl_k_swiglu_fwd(gu, a, stream=None):
    _chk(_lib.tl_k_swiglu_fwd(_dp(gu), gu.shape[0], gu.shape[1] // 2, _dp(a), _s(stream)))


def tl_k_swiglu_bwd(da, gu, dgu, stream=None):
    _chk(_lib.tl_k_swiglu_bwd(_dp(da), _dp(gu), gu.shape[0], gu.shape[1] // 2, _dp(dgu), _s(stream)))


def tl_k_gemv(W, x, y, lora_b=None, lora_h=None, rows_per_group=0, alpha=1.0, resid=None, stream=None):
    N, K = W.shape
    r = lora_b.shape[1] if lora_b is not None else 0
    _chk(_lib.tl_k_gemv(_dp(W), W.stride(0), _dp(x), N, K, _dp(lora_b), _dp(lora_h), r, rows_per_group, alpha, _dp(resid),
                        _dp(y), int(y.dtype == torch.float32), _s(stream)))


def tl_k_gemv_pre(W, y, mode, h=None, gain=None, eps=0.0, gu=None, x_out=None, stream=None):
    N, K = W.shape
    _chk(_lib.tl_k_gemv_pre(_dp(W), W.stride(0), N, K, mode, _dp(h), _dp(gain), eps, _dp(gu), _dp(x_out), _dp(y), _s(stream)))


def tl_k_attention_decode(q, k, v, n_heads, d_head, o, workspace=None, stream=None):
    _chk(_lib.tl_k_attention_decode(_dp(q), _dp(k), _dp(v), k.stride(0), k.shape[0], n_heads, d_head, _dp(o),
                                    _dp(workspace), workspace.numel() if workspace is not None else 0, _s(stream)))


def tl_k_argmax(x, out, stream=None):
    _chk(_lib.tl_k_argmax(_dp(x), x.numel(), _dp(out), _s(stream)))


class Cache8:
    """The memory of a key/value cache held in 8 bits (tl_cache8_mem in the header): six device tensors, kept alive here.
    k int8 [n_blocks, heads, d_head / 64, 64, 64], v int8 [n_blocks, heads, d_head, 64], scales fp32 [n_blocks, heads], tails bf16 as one block."""

    def __init__(self, k, v, k_scale, v_scale, k_tail, v_tail, capacity):
        nb, heads, d = v.shape[:3]
        want = {"k": ((nb, heads, d // 64, 64, 64), torch.int8), "v": ((nb, heads, d, 64), torch.int8),
                "k_scale": ((nb, heads), torch.float32), "v_scale": ((nb, heads), torch.float32),
                "k_tail": ((heads, d // 64, 64, 64), torch.bfloat16), "v_tail": ((heads, d, 64), torch.bfloat16)}
        self.tensors = dict(k=k, v=v, k_scale=k_scale, v_scale=v_scale, k_tail=k_tail, v_tail=v_tail)
        for name, (shape, dtype) in want.items():
            t = self.tensors[name]
            assert t.is_cuda and t.is_contiguous() and tuple(t.shape) == shape and t.dtype == dtype, f"{name}: {dtype} {shape} expected"
        assert 0 < capacity <= 64 * nb, "capacity beyond the blocks"
        self.n_kv_heads, self.d_head, self.capacity = heads, d, capacity
        self.width = heads * d
        self.mem = tl_cache8_mem(*[self.tensors[n].data_ptr() for n in want], heads, d, capacity)
        self.ref = C.byref(self.mem)

    @classmethod
    def empty(cls, n_kv_heads, d_head, capacity, device="cuda"):
        nb = -(-capacity // 64)
        new = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device=device)  # noqa: E731
        return cls(new(torch.int8, nb, n_kv_heads, d_head // 64, 64, 64), new(torch.int8, nb, n_kv_heads, d_head, 64),
                   new(torch.float32, nb, n_kv_heads), new(torch.float32, nb, n_kv_heads),
                   new(torch.bfloat16, n_kv_heads, d_head // 64, 64, 64), new(torch.bfloat16, n_kv_heads, d_head, 64), capacity)


def _rows2(a, b, dtype, width):
    """(address, row stride) of each of two tensors [n, width]"""
    assert a.shape == b.shape and a.dim() == 2 and a.shape[1] == width and a.dtype == b.dtype == dtype, f"{dtype} [n, {width}] expected"
    (la, ua), (lb, ub) = a.stride(), b.stride()
    assert a.is_cuda and b.is_cuda and ua == ub == 1, "device tensors with unit inner stride expected"
    return a.data_ptr(), la, b.data_ptr(), lb


def _ws(workspace):
    if workspace is None:
        return None, 0
    assert workspace.is_cuda and workspace.dtype == torch.float32 and workspace.is_contiguous(), "fp32 device scratch expected"
    return workspace.data_ptr(), workspace.numel()


def tl_k_cache8_append(cache, n_cached, k, v, stream=None):
    """k, v bf16 [n_new, n_kv_heads * d_head] -> tokens n_cached .. of the cache"""
    kp, ldk, vp, ldv = _rows2(k, v, torch.bfloat16, cache.width)
    _chk(_lib.tl_k_cache8_append(cache.ref, n_cached, kp, ldk, vp, ldv, k.shape[0], _s(stream)))


def tl_k_cache8_read(cache, n_cached, first, k_out, v_out, stream=None):
    """k_out, v_out fp32 [n, n_kv_heads * d_head] <- what the cache stands for, tokens first .. first + n - 1"""
    kp, ldk, vp, ldv = _rows2(k_out, v_out, torch.float32, cache.width)
    _chk(_lib.tl_k_cache8_read(cache.ref, n_cached, first, k_out.shape[0], kp, ldk, vp, ldv, _s(stream)))


def tl_k_attention_cache8(cache, n_keys, q, o, n_heads, workspace=None, stream=None):
    """q, o bf16 [n_rows, n_heads * d_head], the last n_rows of n_keys cached tokens"""
    qp, ldq, op, ldo = _rows2(q, o, torch.bfloat16, n_heads * cache.d_head)
    wp, n = _ws(workspace)
    _chk(_lib.tl_k_attention_cache8(cache.ref, n_keys, qp, ldq, q.shape[0], n_heads, op, ldo, wp, n, _s(stream)))


def tl_k_attention_cache8_plan(n_keys, n_rows, n_heads, n_kv_heads, d_head, workspace_elems=0):
    """-> (name of the kernel, ranges of keys, floats used of the workspace)"""
    buf, n, elems = C.create_string_buffer(32), _i32(0), _sz(0)
    _chk(_lib.tl_k_attention_cache8_plan(n_keys, n_rows, n_heads, n_kv_heads, d_head, workspace_elems, buf, 32, C.byref(n), C.byref(elems)))
    return buf.value.decode(), n.value, elems.value


def tl_k_token_counts(tokens, counts, add=0, stream=None):
    """tokens int32 [rows, n], counts int32 [rows, vocab]; add 0: set, 1: add, -1: take away"""
    (rows, n), (again, vocab) = tokens.shape, counts.shape
    (ldt, ut), (ldc, uc) = tokens.stride(), counts.stride()
    assert rows == again and tokens.dtype == counts.dtype == torch.int32 and tokens.is_cuda and counts.is_cuda, "int32 [rows, n], [rows, vocab] expected"
    assert (ut == 1 or n <= 1) and (uc == 1 or vocab == 1), "unit inner stride expected"
    _chk(_lib.tl_k_token_counts(tokens.data_ptr(), ldt, rows, n, vocab, add, counts.data_ptr(), ldc, _s(stream)))


def _row(t, dtype, rows, width):
    """(address, row stride) of [rows, width], of one row for all, or of nothing"""
    if t is None:
        return None, 0
    shape, stride = t.shape, t.stride()
    assert t.is_cuda and t.dtype == dtype and shape[-1] == width and (stride[-1] == 1 or width == 1), f"{dtype} [{rows}, {width}] expected"
    if len(shape) == 1:
        return t.data_ptr(), 0
    assert len(shape) == 2 and shape[0] == rows, f"{dtype} [{rows}, {width}] expected"
    return t.data_ptr(), stride[0]


def tl_k_choose(logits, counts, out, choice, repetition=1.0, presence=0.0, frequency=0.0, bias=None, allowed=None, workspace=None, stream=None):
    """logits fp32 [rows, vocab]; counts int32 and bias fp32 [rows, vocab] or [vocab], allowed int32 words of 32 bits, [rows, ceil(vocab / 32)] or
    one row, each or None; out fp32 like logits or None, choice int32 [rows] or None"""
    R, V = logits.shape
    lp, ldl = _row(logits, torch.float32, R, V)
    cp, ldc = _row(counts, torch.int32, R, V)
    bp, ldb = _row(bias, torch.float32, R, V)
    ap, lda = _row(allowed, torch.int32, R, (V + 31) // 32)
    op, ldo = _row(out, torch.float32, R, V)
    hp, _ = _row(choice, torch.int32, 1, R)
    wp, n = _ws(workspace)
    _chk(_lib.tl_k_choose(lp, ldl, R, V, cp, ldc, repetition, presence, frequency, bp, ldb, ap, lda, op, ldo, hp, wp, n, _s(stream)))


def _vec(t, dtype, n):
    """address of n elements, or of nothing"""
    if t is None:
        return None
    assert t.is_cuda and t.dtype == dtype and t.numel() == n and t.is_contiguous(), f"{dtype} [{n}] expected"
    return t.data_ptr()


def tl_k_sample(logits, params, u, choice, kept=None, prob=None, workspace=None, stream=None):
    """logits fp32 [rows, vocab]; params fp32 [rows, 4] or [4]: temperature, top_k, top_p, min_p; u fp32 [rows]; choice, kept int32 [rows], prob fp32 [rows]"""
    R, V = logits.shape
    lp, ldl = _row(logits, torch.float32, R, V)
    pp, ldp = _row(params, torch.float32, R, 4)
    wp, n = _ws(workspace)
    _chk(_lib.tl_k_sample(lp, ldl, R, V, pp, ldp, _vec(u, torch.float32, R), _vec(choice, torch.int32, R), _vec(kept, torch.int32, R),
                          _vec(prob, torch.float32, R), wp, n, _s(stream)))


class Paged:
    """The memory of a key/value cache on pages (tl_paged_mem in the header): three device tensors, kept alive here.
    k, v bf16 [n_pages, n_kv_heads, page_size, d_head], table int32 [n_seqs, n_table]."""

    def __init__(self, k, v, table):
        assert k.shape == v.shape and k.dim() == 4 and k.dtype == v.dtype == torch.bfloat16, "k, v: bf16 [n_pages, heads, page_size, d_head] expected"
        assert table.dim() == 2 and table.dtype == torch.int32, "table: int32 [n_seqs, n_table] expected"
        for t in (k, v, table):
            assert t.is_cuda and t.is_contiguous(), "contiguous device tensors expected"
        self.k, self.v, self.table = k, v, table
        self.n_pages, self.n_kv_heads, self.page_size, self.d_head = k.shape
        self.n_seqs, self.n_table = table.shape
        self.width = self.n_kv_heads * self.d_head
        self.mem = tl_paged_mem(k.data_ptr(), v.data_ptr(), table.data_ptr(), self.n_pages, self.page_size, self.n_kv_heads, self.d_head, self.n_seqs, self.n_table)
        self.ref = C.byref(self.mem)

    @classmethod
    def empty(cls, n_pages, n_kv_heads, page_size, d_head, n_seqs, n_table, device="cuda"):
        """pages without values, a table without pages"""
        k, v = (torch.empty(n_pages, n_kv_heads, page_size, d_head, dtype=torch.bfloat16, device=device) for _ in range(2))
        return cls(k, v, torch.full((n_seqs, n_table), -1, dtype=torch.int32, device=device))


def _slots(cache, *tensors):
    """(addresses, width) of tensors [n_seqs, n_kv_heads, width], None among them; (dtype, tensor) pairs"""
    width, out = None, []
    for dtype, t in tensors:
        if t is None:
            out.append(None)
            continue
        s = t.shape
        assert t.is_cuda and t.is_contiguous() and t.dtype == dtype and len(s) == 3 and s[:2] == (cache.n_seqs, cache.n_kv_heads), \
            f"{dtype} [{cache.n_seqs}, {cache.n_kv_heads}, slots] expected"
        assert width in (None, s[2]), "as many slots each expected"
        width = s[2]
        out.append(t.data_ptr())
    return out, width or 0


def tl_k_paged_append(cache, lengths, k, v, first_row=None, pos=None, weights=None, positions=None, stream=None):
    """k, v bf16 [n_rows, n_kv_heads * d_head] -> slots lengths[s] .. of sequence s = row, or of the rows first_row[s] .. first_row[s + 1] - 1;
    weights fp32, positions int32 [n_seqs, n_kv_heads, slots]: 0 and pos[row] at the new slots"""
    kp, ldk, vp, ldv = _rows2(k, v, torch.bfloat16, cache.width)
    n = k.shape[0]
    (wp, pp), width = _slots(cache, (torch.float32, weights), (torch.int32, positions))
    _chk(_lib.tl_k_paged_append(cache.ref, _vec(lengths, torch.int32, cache.n_seqs), kp, ldk, vp, ldv, _vec(first_row, torch.int32, cache.n_seqs + 1), n,
                                _vec(pos, torch.int32, n), wp, pp, width, _s(stream)))


def tl_k_attention_paged(cache, lengths, q, o, n_heads, max_len=None, weights_in=None, weights_out=None, workspace=None, stream=None):
    """q, o bf16 [n_seqs, n_heads * d_head]; no sequence is longer than max_len (None: than the table has room for);
    weights_out fp32 [n_seqs, n_kv_heads, slots] = weights_in (or 0) + what each slot got"""
    qp, ldq, op, ldo = _rows2(q, o, torch.bfloat16, n_heads * cache.d_head)
    assert q.shape[0] == cache.n_seqs, "one row a sequence expected"
    (ip, wp), width = _slots(cache, (torch.float32, weights_in), (torch.float32, weights_out))
    sp, n = _ws(workspace)
    _chk(_lib.tl_k_attention_paged(cache.ref, _vec(lengths, torch.int32, cache.n_seqs), cache.n_table * cache.page_size if max_len is None else max_len, qp, ldq,
                                   n_heads, op, ldo, ip, wp, width, sp, n, _s(stream)))


def tl_k_attention_paged_plan(max_len, n_seqs, n_heads, n_kv_heads, d_head, weights=False, workspace_elems=0):
    """-> (ranges of keys, floats of the workspace that are used, or needed where that is more)"""
    n, elems = _i32(0), _sz(0)
    _chk(_lib.tl_k_attention_paged_plan(max_len, n_seqs, n_heads, n_kv_heads, d_head, int(weights), workspace_elems, C.byref(n), C.byref(elems)))
    return n.value, elems.value


def tl_k_attention_weights(q, k, n_heads, n_kv_heads, lse, weights_in, weights_out, first_row=0, stream=None):
    """q bf16 [T, n_heads * d_head], k bf16 [T, n_kv_heads * d_head], lse fp32 [n_heads, T]; weights_in (or None), weights_out fp32 [n_kv_heads, T or more]"""
    T, d = q.shape[0], q.shape[1] // n_heads
    assert q.dtype == k.dtype == torch.bfloat16 and q.shape[1] == n_heads * d and tuple(k.shape) == (T, n_kv_heads * d), "bf16 [T, heads * d_head] expected"
    for w in (weights_in, weights_out):
        assert w is None or (w.dtype == torch.float32 and w.dim() == 2 and w.shape[0] == n_kv_heads and w.shape[1] >= T), "weights: fp32 [n_kv_heads, T] expected"
    _chk(_lib.tl_k_attention_weights(_dp(q), q.stride(0), _dp(k), k.stride(0), T, n_heads, n_kv_heads, d, first_row, _vec(lse, torch.float32, n_heads * T),
                                     _dp(weights_in), weights_in.stride(0) if weights_in is not None else 0, _dp(weights_out), weights_out.stride(0), _s(stream)))


def tl_k_paged_evict(cache, lengths, budget, n_recent, weights, positions, weights_out, positions_out, lengths_out, workspace, stream=None):
    """weights fp32, positions int32 [n_seqs, n_kv_heads, slots] and what they become (or the same tensors); lengths, lengths_out int32 [n_seqs] (or the same)"""
    (wp, pp, wo, po), width = _slots(cache, (torch.float32, weights), (torch.int32, positions), (torch.float32, weights_out), (torch.int32, positions_out))
    sp, n = _ws(workspace)
    _chk(_lib.tl_k_paged_evict(cache.ref, _vec(lengths, torch.int32, cache.n_seqs), budget, n_recent, wp, pp, width, wo, po,
                               _vec(lengths_out, torch.int32, cache.n_seqs), sp, n, _s(stream)))


def tl_k_attention_fwd(q, k, v, n_heads, d_head, o, lse, stream=None):
    _chk(_lib.tl_k_attention_fwd(_dp(q), _dp(k), _dp(v), q.stride(0), q.shape[0], n_heads, d_head, _dp(o),
                                 o.stride(0), _dp(lse), _s(stream)))


def tl_k_attention_bwd(q, k, v, o, d_o, lse, n_heads, d_head, dq, dk, dv, delta, stream=None):
    _chk(_lib.tl_k_attention_bwd(_dp(q), _dp(k), _dp(v), _dp(o), _dp(d_o), _dp(lse), q.stride(0), o.stride(0),
                                 q.shape[0], n_heads, d_head, _dp(dq), _dp(dk), _dp(dv), _dp(delta), _s(stream)))


def tl_k_cross_entropy(logits, labels, first_target, n_targets, nll, dlogits, loss_sum, stream=None):
    _chk(_lib.tl_k_cross_entropy(_dp(logits), _dp(labels), logits.shape[0], logits.shape[1], first_target, n_targets,
                                 _dp(nll), _dp(dlogits), _dp(loss_sum), _s(stream)))


def tl_k_adamw(p, g, m, v, shadow, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, stream=None):
    _chk(_lib.tl_k_adamw(_dp(p), _dp(g), _dp(m), _dp(v), _dp(shadow), p.numel(), step, lr, beta1, beta2, eps,
                         weight_decay, _s(stream)))


def tl_k_embed(E, tokens, h, stream=None):
    _chk(_lib.tl_k_embed(_dp(E), _dp(tokens), tokens.shape[0], E.shape[1], _dp(h), _s(stream)))
