"""ctypes binding of libadept.so (the C ABI in include/adept.h).

Argument marshalling only: every function takes torch tensors (device
memory) or None, passes their data pointers and the current HIP stream to the
library, and raises AdeptError on a non-zero status.  No computation happens
here.  Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libadept.so")

F32, BF16 = 0, 1
KV_F32, KV_BF16, KV_FP8 = 0, 1, 2
FAMILY_LLAMA, FAMILY_GPT2 = 0, 1
SIM_GLOBAL, SIM_LOCAL, SIM_BOTH = 0, 1, 2
METRICS = {"global": SIM_GLOBAL, "local": SIM_LOCAL, "both": SIM_BOTH}

_vp = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_sz = ctypes.c_size_t


class AdeptError(RuntimeError):
    pass


class ExitCfg(ctypes.Structure):
    _fields_ = [("delta", ctypes.c_double), ("min_exit_layer", _i32), ("n_layers", _i32),
                ("metric", _i32), ("prompt_level", _i32)]


class HsmWeights(ctypes.Structure):
    _fields_ = [("g0", _vp), ("conv", (ctypes.c_float * 3) * 3), ("conv_bias", ctypes.c_float),
                ("w1", _vp), ("b1", _vp), ("w2", _vp), ("b2", _vp), ("w3", _vp), ("b3", _vp),
                ("g1", _vp), ("w4", _vp), ("b4", _vp), ("g2", _vp)]


class LayerArgs(ctypes.Structure):
    _fields_ = [
        ("dtype", _i32), ("n_layers", _i32), ("d_model", _i32), ("n_heads", _i32),
        ("head_dim", _i32), ("d_ff", _i32), ("rms_eps", ctypes.c_float), ("exit", ExitCfg),
        ("w_qkv", _vp), ("w_o", _vp), ("w_gate", _vp),
        ("w_up", _vp), ("w_down", _vp), ("rope_cos", _vp), ("rope_sin", _vp),
        ("rope_max_pos", _i32),
        ("n_tok", _i32), ("max_active", _i32), ("n_seq", _i32), ("s_max", _i32),
        ("attn_tiles", _i32),
        ("h", _vp * 2), ("inertia", _vp), ("pos", _vp), ("seq", _vp), ("slot", _vp),
        ("active", _vp * 2), ("n_active", _vp * 2), ("exited", _vp), ("n_exited", _vp),
        ("exit_layer", _vp), ("exit_flag", _vp), ("sim_out", _vp), ("force_layer", _vp),
        ("k_cache", _vp), ("v_cache", _vp), ("n_slots", _i64),
        ("q_buf", _vp), ("attn_out", _vp), ("ffn_act", _vp),
        ("workspace", _vp), ("workspace_bytes", _sz), ("hsm", _vp),
        ("family", _i32), ("b_qkv", _vp), ("b_o", _vp), ("b_fc", _vp), ("b_proj", _vp),
        ("kv_fused", _i32),
    ]


class EncoderArgs(ctypes.Structure):
    _fields_ = [
        ("dtype", _i32), ("n_layers", _i32), ("d_model", _i32), ("n_heads", _i32),
        ("head_dim", _i32), ("d_ff", _i32), ("ln_eps", ctypes.c_float), ("exit", ExitCfg),
        ("w_qkv", _vp), ("b_qkv", _vp), ("w_o", _vp), ("b_o", _vp), ("ln1_g", _vp),
        ("ln1_b", _vp), ("w_in", _vp), ("b_in", _vp), ("w_out", _vp), ("b_out", _vp),
        ("ln2_g", _vp), ("ln2_b", _vp),
        ("n_tok", _i32), ("n_seq", _i32), ("seq_len", _i32), ("cls_stop", _i32),
        ("h", _vp * 2), ("inertia", _vp), ("pos", _vp), ("seq", _vp),
        ("active", _vp * 2), ("n_active", _vp * 2), ("exited", _vp), ("n_exited", _vp),
        ("exit_layer", _vp), ("exit_flag", _vp), ("sim_out", _vp), ("force_layer", _vp),
        ("key_live", _vp), ("key_len", _vp), ("k_buf", _vp), ("v_buf", _vp), ("q_buf", _vp),
        ("attn_out", _vp), ("y_buf", _vp), ("ffn_act", _vp),
        ("workspace", _vp), ("workspace_bytes", _sz),
    ]


class PagedKv(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("page_size", _i32),
                ("n_pages", _i32), ("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp)]


class QuantMat(ctypes.Structure):
    _fields_ = [("codes", _vp), ("scales", _vp)]


class QuantLayers(ctypes.Structure):
    _fields_ = [("qkv", QuantMat), ("o", QuantMat), ("gate", QuantMat), ("up", QuantMat),
                ("down", QuantMat)]


_SIGS = {
    "adept_abi_version": (_i32, []),
    "adept_last_error": (ctypes.c_char_p, []),
    "adept_rope_table": (_i32, [_i32, _i32, ctypes.c_double, _vp, _vp, _vp]),
    "adept_exit_test": (_i32, [_i32, _i32, _i32, ctypes.POINTER(ExitCfg), _vp, _vp, _i32, _vp,
                               _vp, _vp, _vp, _vp, _vp, _vp]),
    "adept_compact_workspace_bytes": (_sz, [_i32]),
    "adept_hsm_workspace_bytes": (_sz, [_i32, _i32]),
    "adept_hsm_forward": (_i32, [_i32, _i32, ctypes.c_float, ctypes.POINTER(HsmWeights), _vp, _vp,
                                 _i32, _vp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]),
    "adept_exit_prompt_level_workspace_bytes": (_sz, [_i32]),
    "adept_exit_prompt_level": (_i32, [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _sz, _vp]),
    "adept_compact": (_i32, [_i32, _i32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                             _vp]),
    "adept_kv_generate_workspace_bytes": (_sz, [_i32, _i32]),
    "adept_kv_generate": (_i32, [_i32, _i32, _i32, _i32, _i32, ctypes.c_float, _vp, _vp, _vp,
                                 _i32, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i32, _vp, _vp,
                                 _i64, _vp, _sz, _vp]),
    "adept_kv_generate_noalloc": (_i32, [_i32, _i32, _i32, _i32, _i32, ctypes.c_float, _vp, _vp,
                                         _vp, _i32, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i32,
                                         _vp, _vp, _i64, _vp]),
    "adept_kv_generate_layernorm_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "adept_kv_generate_layernorm": (_i32, [_i32, _i32, _i32, _i32, _i32, ctypes.c_float, _vp, _vp,
                                           _vp, _i32, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp,
                                           _i64, _vp, _sz, _vp]),
    "adept_fold_bias": (_i32, [_i32, _i32, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _vp]),
    "adept_embed_positions": (_i32, [_i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "adept_final_logits_layernorm": (_i32, [_i32, _i32, _i32, ctypes.c_float, _vp, _vp, _vp, _vp,
                                            _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "adept_attend_workspace_bytes": (_sz, [_i32, _i32, _i32, _i32, _i32]),
    "adept_attend": (_i32, [_i32, _i32, _i32, ctypes.c_float, _i32, _vp, _vp, _vp, _i32, _vp,
                            _vp, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "adept_paged_store": (_i32, [_i32, ctypes.POINTER(PagedKv), _vp, _i64, _vp, _i64, _vp, _vp,
                                 _i32, _vp, _vp]),
    "adept_paged_load": (_i32, [_i32, ctypes.POINTER(PagedKv), _vp, _vp, _i32, _vp, _i64, _vp,
                                _i64, _vp]),
    "adept_paged_attend_workspace_bytes": (_sz, [ctypes.POINTER(PagedKv), _i32, _i32, _i32, _i32]),
    "adept_paged_attend": (_i32, [_i32, ctypes.POINTER(PagedKv), _i32, ctypes.c_float, _i32, _vp,
                                  _vp, _vp, _i32, _vp, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _vp,
                                  _sz, _vp]),
    "adept_paged_copy": (_i32, [ctypes.POINTER(PagedKv), _i32, _vp, _vp, _vp, _vp, _i32, _vp]),
    "adept_verify_drafts_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "adept_verify_drafts": (_i32, [_i32, _i32, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp,
                                   _vp, _vp, _vp, _sz, _vp]),
    "adept_quant_codes_bytes": (_sz, [_i32, _i32]),
    "adept_quant_scales_bytes": (_sz, [_i32, _i32]),
    "adept_quant_pack": (_i32, [_i32, _i32, _i32, _vp, _i64, _vp, _vp, _vp]),
    "adept_quant_unpack": (_i32, [_i32, _i32, _i32, _vp, _vp, _vp, _i64, _vp]),
    "adept_quant_linear": (_i32, [_i32, _i32, _vp, _i64, _vp, _vp, _i32, _vp, _vp, _vp, _i32, _vp,
                                  _i64, _vp]),
    "adept_final_logits_quant": (_i32, [_i32, _i32, ctypes.c_float, _vp, _vp, _vp, _vp, _vp, _i32,
                                        _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "adept_layer_workspace_bytes": (_sz, [ctypes.POINTER(LayerArgs)]),
    "adept_layer_step": (_i32, [ctypes.POINTER(LayerArgs), _i32, _vp]),
    "adept_layer_paged_workspace_bytes": (_sz, [ctypes.POINTER(LayerArgs), ctypes.POINTER(PagedKv),
                                               _i32]),
    "adept_layer_step_paged": (_i32, [ctypes.POINTER(LayerArgs), ctypes.POINTER(PagedKv), _vp, _i32,
                                      _vp, _i32, _vp]),
    "adept_layer_quant_workspace_bytes": (_sz, [ctypes.POINTER(LayerArgs),
                                                ctypes.POINTER(QuantLayers),
                                                ctypes.POINTER(PagedKv), _i32]),
    "adept_layer_step_quant": (_i32, [ctypes.POINTER(LayerArgs), ctypes.POINTER(QuantLayers),
                                      ctypes.POINTER(PagedKv), _vp, _i32, _vp, _i32, _vp]),
    "adept_embed": (_i32, [_i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "adept_final_logits": (_i32, [_i32, _i32, _i32, ctypes.c_float, _vp, _vp, _vp, _vp, _vp,
                                  _i32, _vp, _vp, _vp, _vp, _vp]),
    "adept_argmax": (_i32, [_i32, _i32, _vp, _vp, _vp]),
    "adept_token_init": (_i32, [_i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp]),
    "adept_fold_gain": (_i32, [_i32, _i32, _i32, _i32, _vp, _i64, _vp, _i64, _vp]),
    "adept_encoder_workspace_bytes": (_sz, [ctypes.POINTER(EncoderArgs)]),
    "adept_encoder_layer_step": (_i32, [ctypes.POINTER(EncoderArgs), _i32, _vp]),
    "adept_encoder_embed": (_i32, [_i32, _i32, _i32, _i32, ctypes.c_float, _vp, _vp, _vp, _vp,
                                   _vp, _vp, _vp, _vp, _vp]),
    "adept_classify_head": (_i32, [_i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "adept_timing_enable": (_i32, [_i32]),
    "adept_timing_select": (_i32, [ctypes.c_char_p]),
    "adept_timing_reset": (None, []),
    "adept_timing_count": (_i32, []),
    "adept_timing_get": (_i32, [_i32, ctypes.c_char_p, _i32, ctypes.POINTER(_i64),
                                ctypes.POINTER(ctypes.c_double)]),
}

EXPORTED = tuple(_SIGS)
_lib = None


def lib():
    """Load libadept.so once (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise AdeptError(f"{LIB_PATH} not built: run python -m paper_2601_03700_amd.build")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(status, what):
    if status != 0:
        msg = lib().adept_last_error().decode(errors="replace")
        raise AdeptError(f"{what} failed with status {status}: {msg}")


def ptr(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def stream_handle(stream=None):
    if stream is not None:
        return stream.cuda_stream
    # the handle without the Stream object around it, which takes 2 us to make
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def dtype_code(t_or_str):
    if isinstance(t_or_str, str):
        return {"f32": F32, "bf16": BF16}[t_or_str]
    return {torch.float32: F32, torch.bfloat16: BF16}[t_or_str.dtype]


def exit_cfg(delta, n_layers, metric="global", min_exit_layer=1, prompt_level=False):
    return ExitCfg(float(delta), int(min_exit_layer), int(n_layers), METRICS[metric],
                   int(bool(prompt_level)))


# ----------------------------------------------------------------------------
# thin wrappers, one per entry point
# ----------------------------------------------------------------------------

def rope_table(max_pos, head_dim, theta, cos_out, sin_out, stream=None):
    _check(lib().adept_rope_table(max_pos, head_dim, theta, ptr(cos_out), ptr(sin_out),
                                  stream_handle(stream)), "adept_rope_table")


def exit_test(d_model, layer, cfg, active_rows, n_active, max_active, h_cur, h_prev, inertia,
              force_layer, exit_flag, sim_out=None, stream=None):
    _check(lib().adept_exit_test(dtype_code(h_cur), d_model, layer, ctypes.byref(cfg),
                                 ptr(active_rows), ptr(n_active), max_active, ptr(h_cur),
                                 ptr(h_prev), ptr(inertia), ptr(force_layer), ptr(exit_flag),
                                 ptr(sim_out), stream_handle(stream)), "adept_exit_test")


def exit_prompt_level_workspace_bytes(n_seq):
    return lib().adept_exit_prompt_level_workspace_bytes(n_seq)


def exit_prompt_level(active_rows, n_active, max_active, seq, pos, n_seq, exit_flag,
                      workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().adept_exit_prompt_level(ptr(active_rows), ptr(n_active), max_active, ptr(seq),
                                         ptr(pos), n_seq, ptr(exit_flag), ptr(workspace),
                                         ws_bytes, stream_handle(stream)),
           "adept_exit_prompt_level")


def hsm_weights(w):
    """HsmWeights from a dict of device tensors (bf16 matrices, biases and
    gains) plus the host 3x3 "conv" values and the "conv_b" scalar.  Keep the
    dict alive while the struct is used."""
    hw = HsmWeights()
    for k in ("g0", "w1", "b1", "w2", "b2", "w3", "b3", "g1", "w4", "b4", "g2"):
        setattr(hw, k, ptr(w[k]))
    for r in range(3):
        for t in range(3):
            hw.conv[r][t] = float(w["conv"][r][t])
    hw.conv_bias = float(w["conv_b"])
    return hw


def hsm_workspace_bytes(d_model, max_rows):
    return lib().adept_hsm_workspace_bytes(d_model, max_rows)


def hsm_forward(d_model, eps, hw, rows, n_rows, max_rows, h_cur, h_prev, inertia,
                inertia_updated, out, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().adept_hsm_forward(dtype_code(h_cur), d_model, eps, ctypes.byref(hw), ptr(rows),
                                   ptr(n_rows), max_rows, ptr(h_cur), ptr(h_prev), ptr(inertia),
                                   int(inertia_updated), ptr(out), ptr(workspace), ws_bytes,
                                   stream_handle(stream)),
           "adept_hsm_forward")


def compact_workspace_bytes(max_active):
    return lib().adept_compact_workspace_bytes(max_active)


def compact(layer, n_layers, exit_flag, active_rows, n_active, max_active, next_rows, n_next,
            exited_rows, n_exited, exit_layer, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().adept_compact(layer, n_layers, ptr(exit_flag), ptr(active_rows), ptr(n_active), max_active,
                               ptr(next_rows), ptr(n_next), ptr(exited_rows), ptr(n_exited),
                               ptr(exit_layer), ptr(workspace), ws_bytes, stream_handle(stream)),
           "adept_compact")


def kv_generate_workspace_bytes(n_layers, max_rows):
    return lib().adept_kv_generate_workspace_bytes(n_layers, max_rows)


def kv_generate(n_layers, d_model, n_heads, head_dim, eps, s_map, rows, n_rows, max_rows,
                exit_layer, cache_slot, pos, w_kv, w_kv_layer_stride, attn_gain, rope_cos,
                rope_sin, k_cache, v_cache, n_slots, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().adept_kv_generate(dtype_code(s_map), n_layers, d_model, n_heads, head_dim, eps,
                                   ptr(s_map), ptr(rows), ptr(n_rows), max_rows, ptr(exit_layer),
                                   ptr(cache_slot), ptr(pos), ptr(w_kv), w_kv_layer_stride,
                                   ptr(attn_gain), ptr(rope_cos), ptr(rope_sin),
                                   rope_cos.shape[0], ptr(k_cache), ptr(v_cache), n_slots,
                                   ptr(workspace), ws_bytes, stream_handle(stream)),
           "adept_kv_generate")


def kv_generate_noalloc(n_layers, d_model, n_heads, head_dim, eps, s_map, rows, n_rows, max_rows,
                        exit_layer, cache_slot, pos, w_kv, w_kv_layer_stride, attn_gain,
                        rope_cos, rope_sin, k_cache, v_cache, n_slots, stream=None):
    _check(lib().adept_kv_generate_noalloc(dtype_code(s_map), n_layers, d_model, n_heads,
                                           head_dim, eps, ptr(s_map), ptr(rows), ptr(n_rows),
                                           max_rows, ptr(exit_layer), ptr(cache_slot), ptr(pos),
                                           ptr(w_kv), w_kv_layer_stride, ptr(attn_gain),
                                           ptr(rope_cos), ptr(rope_sin), rope_cos.shape[0],
                                           ptr(k_cache), ptr(v_cache), n_slots,
                                           stream_handle(stream)),
           "adept_kv_generate_noalloc")


def kv_generate_layernorm_workspace_bytes(n_layers, max_rows, d_model):
    return lib().adept_kv_generate_layernorm_workspace_bytes(n_layers, max_rows, d_model)


def kv_generate_layernorm(n_layers, d_model, n_heads, head_dim, eps, s_map, rows, n_rows,
                          max_rows, exit_layer, cache_slot, w_kv, w_kv_layer_stride, b_kv,
                          b_kv_layer_stride, k_cache, v_cache, n_slots, workspace=None,
                          stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().adept_kv_generate_layernorm(dtype_code(s_map), n_layers, d_model, n_heads,
                                             head_dim, eps, ptr(s_map), ptr(rows), ptr(n_rows),
                                             max_rows, ptr(exit_layer), ptr(cache_slot),
                                             ptr(w_kv), w_kv_layer_stride, ptr(b_kv),
                                             b_kv_layer_stride, ptr(k_cache), ptr(v_cache),
                                             n_slots, ptr(workspace), ws_bytes,
                                             stream_handle(stream)),
           "adept_kv_generate_layernorm")


def fold_bias(w, shift, bias, stream=None):
    """In place: bias[l][o] += sum_c w[l][o][c] * shift[l][c] for a stacked
    w [L, rows, cols] (rows contiguous), shift [L, cols] and bias [L, rows]
    (row views with unit column stride)."""
    L, rows, cols = w.shape
    assert w.stride(2) == 1 and (rows == 1 or w.stride(1) == cols)
    assert shift.stride(-1) == 1 and bias.stride(-1) == 1 and bias.shape[-1] == rows
    _check(lib().adept_fold_bias(dtype_code(w), L, rows, cols, ptr(w), w.stride(0), ptr(shift),
                                 shift.stride(0), ptr(bias), bias.stride(0),
                                 stream_handle(stream)), "adept_fold_bias")


def embed_positions(n, d_model, vocab, max_pos, ids, pos, wte, wpe, h0, stream=None):
    _check(lib().adept_embed_positions(dtype_code(wte), n, d_model, vocab, max_pos, ptr(ids),
                                       ptr(pos), ptr(wte), ptr(wpe), ptr(h0),
                                       stream_handle(stream)), "adept_embed_positions")


def final_logits_layernorm(d_model, vocab, eps, h0, h1, exit_layer, rows, n_rows, max_rows, ln_g,
                           ln_b, lm_head, x_norm, logits, stream=None):
    _check(lib().adept_final_logits_layernorm(dtype_code(h0), d_model, vocab, eps, ptr(h0),
                                              ptr(h1), ptr(exit_layer), ptr(rows), ptr(n_rows),
                                              max_rows, ptr(ln_g), ptr(ln_b), ptr(lm_head),
                                              ptr(x_norm), ptr(logits), stream_handle(stream)),
           "adept_final_logits_layernorm")


def attend_workspace_bytes(max_active, n_seq, n_heads, head_dim, s_max):
    return lib().adept_attend_workspace_bytes(max_active, n_seq, n_heads, head_dim, s_max)


def attend(n_heads, head_dim, q, rows, n_active, max_active, pos, seq, n_seq, k_layer, v_layer,
           s_max, out, causal=True, key_len=None, key_live=None, workspace=None, scale=None,
           stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    scale = 1.0 / math.sqrt(head_dim) if scale is None else scale
    _check(lib().adept_attend(dtype_code(q), n_heads, head_dim, scale, int(bool(causal)), ptr(q),
                              ptr(rows), ptr(n_active), max_active, ptr(pos), ptr(seq), n_seq,
                              ptr(k_layer), ptr(v_layer), s_max, ptr(key_len), ptr(key_live),
                              ptr(out), ptr(workspace), ws_bytes, stream_handle(stream)),
           "adept_attend")


_KV_TYPES = {torch.float32: KV_F32, torch.bfloat16: KV_BF16, torch.uint8: KV_FP8,
             torch.float8_e4m3fn: KV_FP8}


def _need(cond, what, why):
    if not cond:
        raise AdeptError(f"{what}: {why}")


def _elsewhere(what):
    return AdeptError(f"{what}: tensors must be on the current HIP device")


def _ptrs(what, dev, *tensors):
    """Pointers of tensors (None: NULL) on device `dev`."""
    out = []
    for t in tensors:
        if t is None:
            out.append(None)
        elif t.get_device() == dev:
            out.append(t.data_ptr())
        else:
            raise _elsewhere(what)
    return out


def _i32_ptrs(what, dev, *tensors):
    """The same of contiguous int32 tensors."""
    out = []
    for t in tensors:
        if t is None:
            out.append(None)
        elif t.dtype is not torch.int32 or not t.is_contiguous():
            raise AdeptError(f"{what}: index tensors must be contiguous int32")
        elif t.get_device() == dev:
            out.append(t.data_ptr())
        else:
            raise _elsewhere(what)
    return out


def _device_of(what, kv):
    """The cache's device, which has to be the current one (the library launches on its streams)."""
    dev = kv.tensors[0].get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise _elsewhere(what)
    return dev


def _count(what, n_rows):
    """A count is the first number; an empty tensor's address would be that of no count."""
    if n_rows is not None and n_rows.numel() == 0:
        raise AdeptError(f"{what}: n_rows holds no number")


def paged_kv(k, v, page_size, k_scale=None, v_scale=None):
    """Descriptor of one layer's paged cache: k, v [n_slots, Hkv, hd] (f32, bf16, or e4m3 codes as
    uint8 / float8_e4m3fn with k_scale, v_scale uint8 [n_slots, Hkv]), contiguous, n_slots a
    multiple of page_size.  It holds the tensors."""
    _need(k.dim() == 3 and k.shape == v.shape and k.dtype == v.dtype and k.dtype in _KV_TYPES and
          k.is_contiguous() and v.is_contiguous(),
          "paged_kv", "k and v must be contiguous [n_slots, Hkv, hd] of one cache type")
    for t in (v, k_scale, v_scale):
        _need(t is None or t.device == k.device, "paged_kv", "one device for the whole cache")
    _need(page_size >= 1 and k.shape[0] % page_size == 0,
          "paged_kv", f"{k.shape[0]} slots are no multiple of the page size {page_size}")
    fp8 = _KV_TYPES[k.dtype] == KV_FP8
    _need(fp8 == (k_scale is not None) == (v_scale is not None),
          "paged_kv", "scales go with an 8-bit cache, and only with it")
    for s in (k_scale, v_scale) if fp8 else ():
        _need(s.dtype == torch.uint8 and s.shape == k.shape[:2] and s.is_contiguous(),
              "paged_kv", "scales must be contiguous uint8 [n_slots, Hkv]")
    kv = PagedKv(_KV_TYPES[k.dtype], k.shape[1], k.shape[2], page_size, k.shape[0] // page_size,
                 ptr(k), ptr(v), ptr(k_scale), ptr(v_scale))
    kv.tensors, kv.layers = (k, v, k_scale, v_scale), None
    return kv


def _rows(what, kv, dev, t, dtype):
    """Pointer and row stride of K or V rows [n, Hkv, hd] with contiguous heads."""
    n, heads, hd = t.shape if t.dim() == 3 else (0, 0, 0)
    row = heads * hd
    if heads != kv.n_kv_heads or hd != kv.head_dim or t.dtype is not dtype or (
            dtype is not torch.bfloat16 and dtype is not torch.float32):
        raise AdeptError(f"{what}: rows must be f32 or bf16 [n, {kv.n_kv_heads}, {kv.head_dim}]")
    if n > 1 or not t.is_contiguous():
        r, h, d = t.stride()
        if n and (d != 1 or (heads > 1 and h != hd)):
            raise AdeptError(f"{what}: the heads of a row must be contiguous")
        row = r if n > 1 else row
    if t.get_device() != dev:
        raise _elsewhere(what)
    return t.data_ptr(), row


def paged_store(kv, k, v, slot, rows=None, n_rows=None, stream=None):
    """Rows of k, v [n, Hkv, hd] (any row stride) into the slots slot[row] of the cache, quantised
    if it is an 8-bit one; rows: the listed rows only, n_rows (device int32 [1]): how many of
    them."""
    dev = _device_of("paged_store", kv)
    _count("paged_store", n_rows)
    kp, ks = _rows("paged_store", kv, dev, k, k.dtype)
    vp, vs = _rows("paged_store", kv, dev, v, k.dtype)
    sp, rp, np_ = _i32_ptrs("paged_store", dev, slot, rows, n_rows)
    n = k.shape[0]
    if v.shape[0] != n or slot.numel() != n:
        raise AdeptError("paged_store: one slot for each row")
    if rows is not None:
        n = rows.numel()
    _check(lib().adept_paged_store(dtype_code(k), ctypes.byref(kv), kp, ks, vp, vs, rp, np_, n, sp,
                                   stream_handle(stream)), "adept_paged_store")


def paged_load(kv, slot, k, v, n_rows=None, stream=None):
    """k[i], v[i] = the cache's values at slot[i] (k, v [n, Hkv, hd], any row stride)."""
    dev = _device_of("paged_load", kv)
    _count("paged_load", n_rows)
    kp, ks = _rows("paged_load", kv, dev, k, k.dtype)
    vp, vs = _rows("paged_load", kv, dev, v, k.dtype)
    sp, np_ = _i32_ptrs("paged_load", dev, slot, n_rows)
    n = slot.numel()
    if k.shape[0] < n or v.shape[0] < n:
        raise AdeptError("paged_load: fewer output rows than slots")
    _check(lib().adept_paged_load(dtype_code(k), ctypes.byref(kv), sp, np_, n, kp, ks, vp, vs,
                                  stream_handle(stream)), "adept_paged_load")


def paged_attend_workspace_bytes(kv, n_heads, max_active, n_seq, max_pages):
    return lib().adept_paged_attend_workspace_bytes(ctypes.byref(kv), n_heads, max_active, n_seq,
                                                    max_pages)


def paged_attend(kv, q, rows, n_active, max_active, pos, seq, n_seq, page_table, out, causal=True,
                 key_len=None, key_live=None, workspace=None, scale=None, stream=None):
    """Attention of the entries q [max_active, H, hd] over the paged cache kv; page_table int32
    [n_seq, max_pages].  workspace: uint8, paged_attend_workspace_bytes()."""
    dev = _device_of("paged_attend", kv)
    n, H, hd = q.shape if q.dim() == 3 else (-1, 0, 0)
    if not (n >= 0 and q.is_contiguous() and out.is_contiguous() and out.dtype is q.dtype and
            hd == kv.head_dim and n >= max_active and out.numel() >= max_active * H * hd and
            rows.numel() >= max_active and
            (q.dtype is torch.bfloat16 or q.dtype is torch.float32)):
        raise AdeptError("paged_attend: q and out must be contiguous [max_active, H, hd] of one type")
    if page_table.dim() != 2 or page_table.shape[0] != n_seq:
        raise AdeptError("paged_attend: page_table must be [n_seq, max_pages]")
    if key_len is not None and key_len.numel() != n_seq:
        raise AdeptError("paged_attend: one key_len for each sequence")
    if key_live is not None and not (key_live.dtype is torch.uint8 and key_live.is_contiguous() and
                                     key_live.numel() == kv.n_pages * kv.page_size):
        raise AdeptError("paged_attend: key_live must be uint8, one for each slot")
    qp, op, lp, wp = _ptrs("paged_attend", dev, q, out, key_live, workspace)
    rp, ap, pp, sp, tp, np_ = _i32_ptrs("paged_attend", dev, rows, n_active, pos, seq, page_table,
                                        key_len)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    _check(lib().adept_paged_attend(dtype_code(q), ctypes.byref(kv), H, scale, int(bool(causal)),
                                    qp, rp, ap, max_active, pp, sp, n_seq, tp, page_table.shape[1],
                                    np_, lp, op, wp, ws_bytes, stream_handle(stream)),
           "adept_paged_attend")


def paged_copy(kv, n_layers, src, dst, n_tokens=None, n_pages=None, stream=None):
    """Pages src[i] of n_layers layers (kv: paged_kv of the first, the others behind it) copied to
    pages dst[i], of each the first n_tokens[i] tokens; n_pages (device int32 [1]): how many of
    them.  The destinations are distinct and none of them is a source."""
    dev = _device_of("paged_copy", kv)
    _count("paged_copy", n_pages)
    sp, dp, tp, np_ = _i32_ptrs("paged_copy", dev, src, dst, n_tokens, n_pages)
    n = src.numel()
    if dst.numel() != n or (n_tokens is not None and n_tokens.numel() != n):
        raise AdeptError("paged_copy: one destination and one number of tokens for each page")
    if _layers_from(kv) < n_layers:
        raise AdeptError(f"paged_copy: {n_layers} layers, the cache has {kv.layers} from the "
                         "described one on")
    _check(lib().adept_paged_copy(ctypes.byref(kv), n_layers, sp, dp, tp, np_, n,
                                  stream_handle(stream)), "adept_paged_copy")


def verify_drafts_workspace_bytes(n_seq, max_draft, vocab):
    return lib().adept_verify_drafts_workspace_bytes(n_seq, max_draft, vocab)


def _logit_rows(what, t, n, per, vocab):
    """Row stride of logits [n, per, vocab] whose rows follow each other at one distance."""
    if t.dim() != 3 or t.shape != (n, per, vocab):
        raise AdeptError(f"{what}: logits must be [{n}, {per}, {vocab}]")
    if t.is_contiguous() or t.numel() == 0:
        return vocab
    s, r, e = t.stride()
    r = s if per == 1 else r
    if (vocab > 1 and e != 1) or (n > 1 and s != per * r):
        raise AdeptError(f"{what}: the rows of logits must be at one distance from each other")
    return r


def verify_drafts(target, draft, tokens, u, out_tokens, n_kept, n_draft=None, temperature=None,
                  workspace=None, stream=None):
    """How many of the drafted tokens [n, g] are kept and the token behind them: out_tokens
    [n, g+1], n_kept [n] int32.  target [n, g+1, V], draft [n, g, V] or None: logits of one type;
    u [n, g+1] f32 in [0, 1); n_draft [n] int32, temperature [n] f32.  workspace: uint8,
    verify_drafts_workspace_bytes()."""
    what = "verify_drafts"
    dev = target.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise _elsewhere(what)
    if target.dim() != 3 or target.shape[1] < 1 or target.dtype not in (torch.float32, torch.bfloat16):
        raise AdeptError(f"{what}: target must be f32 or bf16 [n, drafts + 1, vocab]")
    n, rows, V = target.shape
    ts, ds = _logit_rows(what, target, n, rows, V), V
    if draft is not None:
        if draft.dtype is not target.dtype:
            raise AdeptError(f"{what}: target and draft must be of one type")
        ds = _logit_rows(what, draft, n, rows - 1, V)
    for t, shape in ((tokens, (n, rows - 1)), (out_tokens, (n, rows)), (n_kept, (n,)), (u, (n, rows)),
                     (n_draft, (n,)), (temperature, (n,))):
        if t is not None and tuple(t.shape) != shape:
            raise AdeptError(f"{what}: a tensor of {shape} expected, not {tuple(t.shape)}")
    for t in (u, temperature):
        if t is not None and not (t.dtype is torch.float32 and t.is_contiguous()):
            raise AdeptError(f"{what}: u and temperature must be contiguous f32")
    xp, qp, up, mp, wp = _ptrs(what, dev, target, draft, u, temperature, workspace)
    tp, op, kp, np_ = _i32_ptrs(what, dev, tokens, out_tokens, n_kept, n_draft)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().adept_verify_drafts(dtype_code(target), n, rows - 1, V, xp, ts, qp, ds, tp, np_, mp,
                                     up, op, kp, wp, ws_bytes, stream_handle(stream)),
           "adept_verify_drafts")


class QuantWeights:
    """n_mats matrices [n, k] in 4 bits, in the library's order: codes and scales, uint8
    [n_mats, bytes]."""

    def __init__(self, n, k, codes, scales):
        # (the kernels go by n and k)
        for t, size in ((codes, lib().adept_quant_codes_bytes(n, k)),
                        (scales, lib().adept_quant_scales_bytes(n, k))):
            _need(size > 0 and t.dtype is torch.uint8 and t.dim() == 2 and t.shape[0] >= 1 and
                  t.shape[1] == size and t.is_contiguous(), "quant_weights",
                  f"matrices of {n} x {k} are contiguous uint8 [n_mats, {size}]")
        _need(codes.shape[0] == scales.shape[0] and codes.device == scales.device, "quant_weights",
              "codes and scales of as many matrices, on one device")
        self.n, self.k, self.codes, self.scales = n, k, codes, scales

    @property
    def n_mats(self):
        return self.codes.shape[0]


def quant_weights(n, k, device, n_mats=1):
    """Room for n_mats matrices [n, k], which quant_pack fills."""
    cb, sb = lib().adept_quant_codes_bytes(n, k), lib().adept_quant_scales_bytes(n, k)
    if cb == 0 or n_mats < 1:
        raise AdeptError(f"quant_weights: no matrix of {n} x {k}")
    return QuantWeights(n, k, torch.empty((n_mats, cb), dtype=torch.uint8, device=device),
                        torch.empty((n_mats, sb), dtype=torch.uint8, device=device))


def _matrix(what, qw, w, mat):
    dev = qw.codes.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise _elsewhere(what)
    if not 0 <= mat < qw.n_mats:
        raise AdeptError(f"{what}: matrix {mat} of {qw.n_mats}")
    if w is None:
        return dev, qw.codes.data_ptr() + mat * qw.codes.stride(0), \
            qw.scales.data_ptr() + mat * qw.scales.stride(0), None
    if (w.shape != (qw.n, qw.k) or w.dtype not in (torch.float32, torch.bfloat16) or
            (qw.k > 1 and w.stride(1) != 1)):
        raise AdeptError(f"{what}: the matrix must be f32 or bf16 [{qw.n}, {qw.k}] with contiguous rows")
    if w.get_device() != dev:
        raise _elsewhere(what)
    return dev, qw.codes.data_ptr() + mat * qw.codes.stride(0), \
        qw.scales.data_ptr() + mat * qw.scales.stride(0), w.stride(0) if qw.n > 1 else qw.k


def quant_pack(w, qw, mat=0, stream=None):
    """w [n, k] (f32 or bf16, any row stride) quantised into matrix `mat` of qw."""
    _, cp, sp, ld = _matrix("quant_pack", qw, w, mat)
    _check(lib().adept_quant_pack(dtype_code(w), qw.n, qw.k, ptr(w), ld, cp, sp,
                                  stream_handle(stream)), "adept_quant_pack")


def quant_unpack(qw, w, mat=0, stream=None):
    """w [n, k] = the values of matrix `mat` of qw."""
    _, cp, sp, ld = _matrix("quant_unpack", qw, w, mat)
    _check(lib().adept_quant_unpack(dtype_code(w), qw.n, qw.k, cp, sp, ptr(w), ld,
                                    stream_handle(stream)), "adept_quant_unpack")


def quant_linear_max_rows(n):
    """The most rows that a call (quant_linear, final_logits_quant) takes over n weight rows."""
    return min(64 * 65535, ((1 << 22) - 1) // (-(-n // 16) + 7) * 16)


def quant_linear(x, qw, y, mat=0, rows=None, n_rows=None, bias=None, stream=None):
    """y[i] = x[row] w^T + bias with matrix `mat` of qw, row = rows[i] (None: i); n_rows (device
    int32 [1]): how many.  x bf16 [m, k], y f32 or bf16 [rows, n], any row stride."""
    what = "quant_linear"
    dev, cp, sp, _ = _matrix(what, qw, None, mat)
    _count(what, n_rows)
    if x.dim() != 2 or x.shape[1] != qw.k or x.dtype is not torch.bfloat16 or x.stride(1) != 1:
        raise AdeptError(f"{what}: x must be bf16 [m, {qw.k}] with contiguous rows")
    n = x.shape[0] if rows is None else rows.numel()
    if (y.dim() != 2 or y.shape[0] < n or y.shape[1] != qw.n or (qw.n > 1 and y.stride(1) != 1) or
            y.dtype not in (torch.float32, torch.bfloat16)):
        raise AdeptError(f"{what}: y must be f32 or bf16 [{n}, {qw.n}] with contiguous rows")
    if bias is not None and not (bias.dtype is torch.bfloat16 and bias.shape == (qw.n,) and
                                 bias.is_contiguous()):
        raise AdeptError(f"{what}: bias must be contiguous bf16 [{qw.n}]")
    xp, yp, bp = _ptrs(what, dev, x, y, bias)
    rp, np_ = _i32_ptrs(what, dev, rows, n_rows)
    _check(lib().adept_quant_linear(qw.n, qw.k, xp, x.stride(0) if x.shape[0] > 1 else qw.k, rp, np_,
                                    n, cp, sp, bp, dtype_code(y), yp,
                                    y.stride(0) if y.shape[0] > 1 else qw.n, stream_handle(stream)),
           "adept_quant_linear")


def final_logits_quant(d_model, vocab, eps, h0, h1, exit_layer, rows, n_rows, max_rows, norm_gain,
                       norm_bias, qw, x_norm, logits, stream=None):
    """final_logits (norm_bias None) or final_logits_layernorm over a head in 4 bits."""
    _, cp, sp, _ = _matrix("final_logits_quant", qw, None, 0)
    if (qw.n, qw.k) != (vocab, d_model) or h0.dtype is not torch.bfloat16:
        raise AdeptError(f"final_logits_quant: a bf16 model and a head of {vocab} x {d_model} expected")
    _check(lib().adept_final_logits_quant(d_model, vocab, eps, ptr(h0), ptr(h1), ptr(exit_layer),
                                          ptr(rows), ptr(n_rows), max_rows, ptr(norm_gain),
                                          ptr(norm_bias), cp, sp, ptr(x_norm), ptr(logits),
                                          stream_handle(stream)), "adept_final_logits_quant")


def layer_workspace_bytes(args: LayerArgs):
    return lib().adept_layer_workspace_bytes(ctypes.byref(args))


def layer_step(args: LayerArgs, layer, stream=None):
    _check(lib().adept_layer_step(ctypes.byref(args), layer, stream_handle(stream)),
           "adept_layer_step")


def layer_paged_workspace_bytes(args: LayerArgs, kv, max_pages):
    return lib().adept_layer_paged_workspace_bytes(ctypes.byref(args), ctypes.byref(kv), max_pages)


def _layers_from(kv):
    """Layers of a cache from the described one on, by the memory behind its tensors."""
    if kv.layers is None:
        kv.layers = min((t.untyped_storage().nbytes() - t.storage_offset() * t.element_size()) //
                        max(t.numel() * t.element_size(), 1) for t in kv.tensors if t is not None)
    return kv.layers


def _paged_step(what, args, kv, page_table, cache_slot):
    if page_table.dim() != 2 or page_table.shape[0] < args.n_seq:
        raise AdeptError(f"{what}: page_table must be [n_seq, max_pages]")
    if cache_slot is not None and cache_slot.numel() < args.n_tok:
        raise AdeptError(f"{what}: one slot for each row")
    if _layers_from(kv) < args.n_layers:
        raise AdeptError(f"{what}: {args.n_layers} layers, the cache has "
                         f"{kv.layers} from the described one on")
    return _i32_ptrs(what, _device_of(what, kv), page_table, cache_slot)


def _layer_sizes(args):
    return args.d_model, args.n_heads * args.head_dim, args.d_ff, args.family


def quant_layers(args: LayerArgs, qkv, o, gate, up, down):
    """Descriptor of the layers' weights in 4 bits (QuantWeights of all layers each; up None in the
    GPT2 family), which it holds."""
    N = args.n_layers
    D, dq, F, family = _layer_sizes(args)
    q = QuantLayers()
    q.weights, q.sizes, q.layers = (qkv, o, gate, up, down), (D, dq, F, family), None
    for name, w, n, k in (("qkv", qkv, 3 * dq, D), ("o", o, D, dq), ("gate", gate, F, D),
                          ("up", up, F, D), ("down", down, D, F)):
        if w is None and name == "up" and family == FAMILY_GPT2:
            continue
        if w is None or (w.n, w.k) != (n, k) or w.n_mats < N:
            raise AdeptError(f"quant_layers: {name} must be {N} matrices of {n} x {k}")
        if w.codes.device != qkv.codes.device:
            raise AdeptError("quant_layers: weights on one device")
        q.layers = w.n_mats if q.layers is None else min(q.layers, w.n_mats)
        setattr(q, name, QuantMat(w.codes.data_ptr(), w.scales.data_ptr()))
    return q


def layer_quant_workspace_bytes(args: LayerArgs, weights, kv=None, max_pages=0):
    return lib().adept_layer_quant_workspace_bytes(
        ctypes.byref(args), ctypes.byref(weights), ctypes.byref(kv) if kv is not None else None,
        max_pages)


def layer_step_quant(args: LayerArgs, weights, layer, kv=None, page_table=None, cache_slot=None,
                     stream=None):
    """layer_step (kv None) or layer_step_paged with the weights in 4 bits as well (quant_layers)."""
    if args.n_layers > weights.layers or _layer_sizes(args) != weights.sizes:
        raise AdeptError(f"layer_step_quant: weights of {weights.layers} layers, width, H*hd, d_ff and "
                         f"family {weights.sizes}; the arguments have {args.n_layers}, "
                         f"{_layer_sizes(args)}")
    dev = weights.weights[0].codes.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise _elsewhere("layer_step_quant")
    tp = cp = None
    if kv is not None:
        tp, cp = _paged_step("layer_step_quant", args, kv, page_table, cache_slot)
    _check(lib().adept_layer_step_quant(ctypes.byref(args), ctypes.byref(weights),
                                        ctypes.byref(kv) if kv is not None else None, tp,
                                        page_table.shape[1] if kv is not None else 0, cp, layer,
                                        stream_handle(stream)), "adept_layer_step_quant")


def layer_step_paged(args: LayerArgs, kv, page_table, layer, cache_slot=None, stream=None):
    """layer_step over a paged cache; kv: paged_kv of its first layer, the others behind it;
    page_table int32 [n_seq, max_pages]; cache_slot int32, one for each row (8-bit caches)."""
    tp, cp = _paged_step("layer_step_paged", args, kv, page_table, cache_slot)
    _check(lib().adept_layer_step_paged(ctypes.byref(args), ctypes.byref(kv), tp,
                                        page_table.shape[1], cp, layer, stream_handle(stream)),
           "adept_layer_step_paged")


def embed(n, d_model, vocab, ids, table, h0, stream=None):
    _check(lib().adept_embed(dtype_code(table), n, d_model, vocab, ptr(ids), ptr(table), ptr(h0),
                             stream_handle(stream)), "adept_embed")


def final_logits(d_model, vocab, eps, h0, h1, exit_layer, rows, n_rows, max_rows, final_norm,
                 lm_head, x_norm, logits, stream=None):
    _check(lib().adept_final_logits(dtype_code(h0), d_model, vocab, eps, ptr(h0), ptr(h1),
                                    ptr(exit_layer), ptr(rows), ptr(n_rows), max_rows,
                                    ptr(final_norm), ptr(lm_head), ptr(x_norm), ptr(logits),
                                    stream_handle(stream)), "adept_final_logits")


def argmax(n, vocab, logits, out, stream=None):
    _check(lib().adept_argmax(n, vocab, ptr(logits), ptr(out), stream_handle(stream)),
           "adept_argmax")


def token_init(n_tok, n_layers, d_model, active, n_active, exit_layer, inertia=None, stream=None):
    _check(lib().adept_token_init(n_tok, n_layers, d_model, ptr(active), ptr(n_active),
                                  ptr(exit_layer), ptr(inertia), stream_handle(stream)),
           "adept_token_init")


def timing_enable(on=True):
    _check(lib().adept_timing_enable(1 if on else 0), "adept_timing_enable")


def timing_select(prefix=None):
    """Time only the launches whose kernel name starts with `prefix` (None: all)."""
    _check(lib().adept_timing_select(prefix.encode() if prefix else None),
           "adept_timing_select")


def timing_reset():
    lib().adept_timing_reset()


def encoder_workspace_bytes(args):
    return lib().adept_encoder_workspace_bytes(ctypes.byref(args))


def encoder_layer_step(args, layer, stream=None):
    _check(lib().adept_encoder_layer_step(ctypes.byref(args), layer, stream_handle(stream)),
           "adept_encoder_layer_step")


def encoder_embed(n, d_model, vocab, max_pos, eps, ids, pos, word_emb, pos_emb, type_emb, ln_g,
                  ln_b, out, stream=None):
    _check(lib().adept_encoder_embed(n, d_model, vocab, max_pos, eps, ptr(ids), ptr(pos),
                                     ptr(word_emb), ptr(pos_emb), ptr(type_emb), ptr(ln_g),
                                     ptr(ln_b), ptr(out), stream_handle(stream)),
           "adept_encoder_embed")


def classify_head(n_seq, seq_len, d_model, n_classes, h0, h1, exit_layer, w_cls, b_cls, logits,
                  stream=None):
    _check(lib().adept_classify_head(n_seq, seq_len, d_model, n_classes, ptr(h0), ptr(h1),
                                     ptr(exit_layer), ptr(w_cls), ptr(b_cls), ptr(logits),
                                     stream_handle(stream)), "adept_classify_head")


def timing_read():
    """{kernel name: (launches, total ms)} accumulated since the last reset."""
    L = lib()
    out = {}
    buf = ctypes.create_string_buffer(256)
    for i in range(L.adept_timing_count()):
        n, ms = _i64(0), ctypes.c_double(0.0)
        _check(L.adept_timing_get(i, buf, 256, ctypes.byref(n), ctypes.byref(ms)),
               "adept_timing_get")
        out[buf.value.decode()] = (int(n.value), float(ms.value))
    return out


def fold_gain(w, gain, stream=None):
    """In place: w[l][o][c] *= gain[l][c] for a stacked weight w [L, rows, cols]
    (or a [L, rows, cols] view with unit column stride) and gain [L, cols]."""
    L, rows, cols = w.shape
    assert w.stride(2) == 1 and gain.stride(-1) == 1 and gain.shape[-1] == cols
    if rows > 1:
        assert w.stride(1) == cols, "rows of each matrix must be contiguous"
    _check(lib().adept_fold_gain(dtype_code(w), L, rows, cols, ptr(w), w.stride(0), ptr(gain),
                                 gain.stride(0) if gain.dim() == 2 else 0, stream_handle(stream)),
           "adept_fold_gain")
