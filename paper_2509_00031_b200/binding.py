"""ctypes binding of libzoqat.so: the same names as include/zoqat.h, argument
marshalling only (torch tensors -> device pointers).  Every step of the path runs
in the CUDA library; there is no Python or CPU fallback - loading raises if the
library has not been built.
"""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libzoqat.so")

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_SMALL, ERR_CUDA, ERR_BAD_STATE, ERR_TIMEOUT = -1, -2, -3, -4, -5, -6
ARCH_LLAMA, ARCH_OPT = 0, 1
(ROLE_WQ, ROLE_WK, ROLE_WV, ROLE_WO, ROLE_W_GATE, ROLE_W_UP, ROLE_W_DOWN, ROLE_ATTN_NORM_G, ROLE_ATTN_NORM_B,
 ROLE_FFN_NORM_G, ROLE_FFN_NORM_B, ROLE_BQ, ROLE_BK, ROLE_BV, ROLE_BO, ROLE_B_FC1, ROLE_B_FC2, ROLE_EMBED,
 ROLE_POS_EMBED, ROLE_FINAL_NORM_G, ROLE_FINAL_NORM_B, ROLE_LM_HEAD) = range(22)
ROLE_SMOOTH_SCALE, ROLE_SMOOTH_SHIFT = 22, 26      # + quantisation point 0..3 (Section 4.2)
SMOOTH_POINTS = ("attn_in", "attn_out", "ffn_in", "ffn_out")
TENSOR_TRAINABLE, TENSOR_QUANTIZED, TENSOR_FROZEN_PACKED, TENSOR_ADAPTIVE = 1, 2, 4, 8
GEMM_TCGEN05, GEMM_SIMT, GEMM_TCGEN05_1CTA, GEMM_TCGEN05_I8 = 0, 1, 2, 3
BUF_RESIDUAL, BUF_QKV, BUF_ATTN, BUF_FFN, BUF_TOKEN_LOSS = range(5)
PROF_GEMM, PROF_WEIGHT, PROF_ACT, PROF_ATTENTION, PROF_LOSS, PROF_UPDATE = range(6)
TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3
PLAN_BAD_LENGTH, PLAN_NO_PAGES, PLAN_BAD_PAGE, PLAN_BAD_PARENT = 1, 2, 4, 8
PROF_NAMES = ["gemm", "weight_operand", "act_operand", "attention", "loss", "update"]

EXPORTS = [
    "zoqat_query_workspace", "zoqat_packed_bytes", "zoqat_model_create", "zoqat_model_destroy",
    "zoqat_prequantize_frozen", "zoqat_expand_frozen_bytes", "zoqat_expand_frozen", "zoqat_init_qparams", "zoqat_forward_loss", "zoqat_step", "zoqat_step_rates", "zoqat_step_deferred", "zoqat_step_rates_deferred", "zoqat_step_finish_deferred", "zoqat_step_finish_rates_deferred", "zoqat_flush_update", "zoqat_step_multi",
    "zoqat_step_begin", "zoqat_step_finish", "zoqat_step_finish_rates", "zoqat_step_host", "zoqat_step_host_deferred", "zoqat_apply_update", "zoqat_apply_update_rates", "zoqat_apply_update_multi", "zoqat_step_result",
    "zoqat_check", "zoqat_launch_count", "zoqat_profile_enable", "zoqat_profile_read", "zoqat_debug_buffer", "zoqat_debug_capture", "zoqat_debug_capture_bytes", "zoqat_status_string", "zoqat_last_error",
    "zoqat_op_philox_words", "zoqat_op_normal", "zoqat_op_weight_quant", "zoqat_op_weight_operand_pair",
    "zoqat_op_weight_operand_learned", "zoqat_op_smooth_perturb", "zoqat_op_smooth_act_operand", "zoqat_op_init_qparams",
    "zoqat_op_pack_frozen", "zoqat_op_unpack_operand", "zoqat_op_unpack_operand_i8", "zoqat_op_update", "zoqat_op_norm_act_operand",
    "zoqat_op_ffn_act_operand", "zoqat_op_gemm", "zoqat_op_gemm_silu_gate", "zoqat_op_gemm_i8", "zoqat_op_weight_operand_i8", "zoqat_op_norm_act_operand_i8", "zoqat_op_qkv_attention", "zoqat_op_attention_scratch_bytes", "zoqat_op_attention",
    "zoqat_op_head_loss_scratch_bytes",
    "zoqat_op_head_loss", "zoqat_op_head_loss_static",
    "zoqat_decode_bytes", "zoqat_decode_begin", "zoqat_decode_step", "zoqat_op_decode_gemv",
    "zoqat_op_cache_plan", "zoqat_op_cache_append", "zoqat_op_tree_attention_scratch_bytes", "zoqat_op_tree_attention",
    "zoqat_op_logit_rules", "zoqat_decode_tree_step",
    "zoqat_rotary_frequencies", "zoqat_op_rotary_append", "zoqat_op_prefix_attention_scratch_bytes", "zoqat_op_prefix_attention", "zoqat_op_beam_select", "zoqat_op_beam_reorder_scratch_bytes", "zoqat_op_beam_reorder",
    "zoqat_op_cache_copy", "zoqat_decode_prefix_step",
]


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("arch", "n_layers", "d_model", "n_heads", "d_ffn", "vocab", "max_batch", "max_seq",
                 "w_bits", "w_group", "a_bits", "gemm_impl")] + [("norm_eps", ctypes.c_float), ("rope_base", ctypes.c_float)]


class TensorDesc(ctypes.Structure):
    _fields_ = [("role", ctypes.c_int32), ("layer", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32), ("data", ctypes.c_void_p), ("packed", ctypes.c_void_p),
                ("qparams", ctypes.c_void_p)]


class StepResult(ctypes.Structure):
    _fields_ = [("loss_plus", ctypes.c_float), ("loss_minus", ctypes.c_float), ("proj_grad", ctypes.c_float),
                ("update_scale", ctypes.c_float), ("status", ctypes.c_int32), ("n_labels", ctypes.c_int32)]


class PagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in (
        "type", "n_pages", "page_size", "n_kv_heads", "d_head", "reserved")] + [(n, ctypes.c_int64) for n in (
            "page_stride", "slot_stride", "head_stride")]


class TreeBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("block_table", "kv_len", "row_start", "row_pos", "slot", "tree_mask")] + [
        (n, ctypes.c_int32) for n in ("batch", "max_pages", "mask_words", "reserved")]


class LogitRulesDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "row_request", "repetition", "presence", "frequency", "history", "history_len", "prompt_len", "bias_token", "bias_value", "bias_len",
        "allowed", "draft_token", "row_start", "tree_mask")] + [(n, ctypes.c_int64) for n in ("history_stride", "allowed_stride")] + [
            (n, ctypes.c_int32) for n in ("bias_stride", "mask_words", "batch", "reserved")]


class PrefixGroups(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("group_start", "prefix_len", "request_group")] + [(n, ctypes.c_int32) for n in ("groups", "reserved")]


class BeamReorder(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "parent", "kv_len", "block_table", "shared_len", "free_pages", "n_free", "history", "history_len", "token", "block_table_out", "kv_len_out",
        "free_pages_out", "n_free_out", "copy_from", "copy_to", "copy_len", "history_out", "history_len_out", "status")] + [
            ("history_stride", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("batch", "beams", "page_size", "n_pages", "max_pages", "free_capacity")]


class ZoqatError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"zoqat status {status}: {text}")
        self.status = status


_lib = None


def lib():
    """The loaded library.  Raises if libzoqat.so is missing: there is no fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: build it with `python -m paper_2509_00031_b200.build` "
                              "(the CUDA library is the only implementation of this path)")
        L = ctypes.CDLL(LIB_PATH)
        L.zoqat_status_string.restype = ctypes.c_char_p
        L.zoqat_last_error.restype = ctypes.c_char_p
        vp, i32, i64, u32, u64, f32, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint32,
                                           ctypes.c_uint64, ctypes.c_float, ctypes.c_size_t)
        P = ctypes.POINTER
        sigs = {
            "zoqat_query_workspace": [P(Config), P(sz)],
            "zoqat_packed_bytes": [i64, i64, i32, i32, P(sz), P(sz)],
            "zoqat_model_create": [P(Config), P(TensorDesc), i32, vp, sz, P(vp)],
            "zoqat_model_destroy": [vp],
            "zoqat_prequantize_frozen": [vp, vp],
            "zoqat_expand_frozen_bytes": [vp, P(sz)],
            "zoqat_expand_frozen": [vp, vp, sz, vp],
            "zoqat_init_qparams": [vp, vp],
            "zoqat_step_rates": [vp, vp, vp, i32, i32, u64, f32, f32, f32, f32, vp, vp],
            "zoqat_step_finish_rates": [vp, vp, u64, f32, f32, f32, f32, vp, vp],
            "zoqat_step_rates_deferred": [vp, vp, vp, i32, i32, u64, f32, f32, f32, f32, vp, vp],
            "zoqat_step_finish_rates_deferred": [vp, vp, u64, f32, f32, f32, f32, vp, vp],
            "zoqat_apply_update_rates": [vp, u64, f32, f32, f32, vp],
            "zoqat_op_weight_operand_learned": [vp, i64, i64, i32, i32, u64, u32, f32, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "zoqat_op_smooth_perturb": [vp, vp, i64, u64, u32, u32, f32, vp, vp],
            "zoqat_op_smooth_act_operand": [vp, i64, i64, i32, vp, vp, f32, i32, vp, i64, vp, vp, vp],
            "zoqat_op_init_qparams": [vp, i64, i64, i32, i32, vp, vp],
            "zoqat_forward_loss": [vp, vp, vp, i32, i32, u64, f32, vp, vp],
            "zoqat_step": [vp, vp, vp, i32, i32, u64, f32, f32, vp, vp],
            "zoqat_step_multi": [vp, vp, vp, i32, i32, u64, i32, f32, f32, vp, vp],
            "zoqat_step_deferred": [vp, vp, vp, i32, i32, u64, f32, f32, vp, vp],
            "zoqat_flush_update": [vp, vp],
            "zoqat_step_finish_deferred": [vp, vp, u64, f32, f32, vp, vp],
            "zoqat_step_host": [vp, vp, vp, i32, i32, u64, f32, f32, P(StepResult), vp],
            "zoqat_step_host_deferred": [vp, vp, vp, i32, i32, u64, f32, f32, P(StepResult), vp],
            "zoqat_step_begin": [vp, vp, vp, i32, i32, u64, f32, vp, vp],
            "zoqat_step_finish": [vp, vp, u64, f32, f32, vp, vp],
            "zoqat_apply_update": [vp, u64, f32, vp],
            "zoqat_apply_update_multi": [vp, P(u64), vp, i32, vp],
            "zoqat_step_result": [vp, vp, f32, f32, vp, vp],
            "zoqat_check": [vp, vp],
            "zoqat_launch_count": [vp, P(i64)],
            "zoqat_debug_buffer": [vp, i32, P(vp), P(sz)],
            "zoqat_debug_capture": [vp, vp, sz],
            "zoqat_debug_capture_bytes": [vp, i32, i32, i32, P(sz)],
            "zoqat_profile_enable": [vp, i32],
            "zoqat_profile_read": [vp, i32, P(ctypes.c_double), P(i64), vp],
            "zoqat_op_philox_words": [u64, u32, u64, u64, vp, vp],
            "zoqat_op_normal": [u64, u32, u64, vp, vp],
            "zoqat_op_weight_quant": [vp, i64, i64, i32, i32, u64, u32, f32, vp, vp, vp, vp, vp],
            "zoqat_op_weight_operand_pair": [vp, i64, i64, i32, i32, u64, u32, f32, vp, vp, vp],
            "zoqat_op_pack_frozen": [vp, i64, i64, i32, i32, vp, vp, vp],
            "zoqat_op_unpack_operand": [vp, vp, i64, i64, i32, i32, vp, vp],
            "zoqat_op_unpack_operand_i8": [vp, vp, i64, i64, i32, vp, vp, vp, vp],
            "zoqat_op_update": [vp, u64, u64, u32, f32, vp],
            "zoqat_op_norm_act_operand": [vp, i64, i64, i32, vp, vp, f32, i32, vp, vp, vp, vp],
            "zoqat_op_ffn_act_operand": [vp, i64, i64, i32, i32, vp, vp, vp],
            "zoqat_op_gemm": [vp, vp, i64, i64, i64, vp, vp, i32, i32, vp, i32, vp, vp],
            "zoqat_op_gemm_silu_gate": [vp, vp, i64, i64, i64, vp, vp, vp, vp, vp],
            "zoqat_op_gemm_i8": [vp, vp, i64, i64, i64, vp, vp, vp, i32, i32, vp, vp, vp, vp],
            "zoqat_op_weight_operand_i8": [vp, i64, i64, i32, u64, u32, f32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "zoqat_op_norm_act_operand_i8": [vp, i64, i64, i32, vp, vp, f32, i32, vp, vp, vp],
            "zoqat_op_attention_scratch_bytes": [i32, i32, i32, i32, P(sz)],
            "zoqat_op_qkv_attention": [vp, vp, i32, i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp],
            "zoqat_op_attention": [vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp],
            "zoqat_op_head_loss_scratch_bytes": [i64, i64, P(sz)],
            "zoqat_op_head_loss": [vp, vp, vp, i64, i64, i64, vp, vp, vp, vp, i32, vp, vp],
            "zoqat_op_head_loss_static": [vp, vp, vp, i64, i64, i64, vp, vp, vp, i32, vp, vp],
            "zoqat_decode_bytes": [vp, i32, i32, P(sz)],
            "zoqat_decode_begin": [vp, vp, sz, i32, i32, vp],
            "zoqat_decode_step": [vp, vp, i32, vp, vp, vp],
            "zoqat_op_decode_gemv": [vp, vp, i64, i64, i32, i32, vp, vp, i32, vp, i32, vp, vp, vp],
            "zoqat_op_cache_plan": [vp, vp, i32, i32, i32, vp, i32, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "zoqat_op_cache_append": [vp, i64, vp, vp, i32, i32, vp, vp, i32, P(PagedCache), vp, i64, vp, vp],
            "zoqat_op_tree_attention_scratch_bytes": [i32, i32, P(sz)],
            "zoqat_op_tree_attention": [vp, i64, P(PagedCache), vp, i32, vp, vp, vp, i32, i32, i32, i32, f32, vp, i64, vp, sz, vp, vp],
            "zoqat_decode_tree_step": [vp, vp, i32, P(TreeBatch), P(PagedCache), P(LogitRulesDesc), vp, vp, vp, sz, vp],
            "zoqat_op_logit_rules": [vp, i32, i64, i32, i32, P(LogitRulesDesc), vp, i64, vp, vp],
            "zoqat_rotary_frequencies": [i32, ctypes.c_double, i32, ctypes.c_double, i32, P(ctypes.c_double), P(f32)],
            "zoqat_op_rotary_append": [vp, i32, i64, vp, vp, i32, i32, vp, i32, i32, f32, vp, vp, f32, P(PagedCache), vp, i64, vp, vp],
            "zoqat_op_prefix_attention_scratch_bytes": [i32, i32, i32, i32, P(sz)],
            "zoqat_op_prefix_attention": [vp, i64, P(PagedCache), vp, i32, vp, vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, f32, vp, i64, vp, sz, vp, vp],
            "zoqat_op_beam_select": [vp, i32, i64, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp],
            "zoqat_op_beam_reorder_scratch_bytes": [i32, P(sz)],
            "zoqat_op_beam_reorder": [P(BeamReorder), vp, sz, vp],
            "zoqat_decode_prefix_step": [vp, vp, i32, P(TreeBatch), P(PrefixGroups), P(PagedCache), P(LogitRulesDesc), vp, vp, vp, sz, vp],
            "zoqat_op_cache_copy": [P(PagedCache), i32, vp, vp, vp, i32, vp, vp],
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status):
    if status != OK:
        raise ZoqatError(status, lib().zoqat_last_error().decode())


def _p(t):
    """Device (or host) pointer of a tensor, None -> NULL."""
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


# ---- single operations ---------------------------------------------------------------
def zoqat_op_philox_words(seed, tensor_id, blk0, nblk, out=None):
    out = torch.empty((nblk, 4), dtype=torch.int32, device="cuda") if out is None else out
    _check(lib().zoqat_op_philox_words(seed, tensor_id, blk0, nblk, _p(out), _stream()))
    return out


def zoqat_op_normal(seed, tensor_id, n):
    out = torch.empty(n, dtype=torch.float32, device="cuda")
    _check(lib().zoqat_op_normal(seed, tensor_id, n, _p(out), _stream()))
    return out


def zoqat_op_weight_quant(w, group, bits, seed=0, tensor_id=0, signed_eps=0.0, want_codes=True):
    rows, cols = w.shape
    operand = torch.empty((rows, cols), dtype=torch.bfloat16, device=w.device)
    codes = step = zp = None
    if want_codes and bits:
        codes = torch.empty((rows, cols), dtype=torch.uint8, device=w.device)
        step = torch.empty((rows, cols // group), dtype=torch.float32, device=w.device)
        zp = torch.empty((rows, cols // group), dtype=torch.int32, device=w.device)
    _check(lib().zoqat_op_weight_quant(_p(w), rows, cols, group, bits, seed, tensor_id, signed_eps,
                                       _p(codes), _p(step), _p(zp), _p(operand), _stream()))
    return codes, step, zp, operand


def zoqat_op_weight_operand_pair(w, group, bits, seed, tensor_id, eps):
    rows, cols = w.shape
    plus = torch.empty((rows, cols), dtype=torch.bfloat16, device=w.device)
    minus = torch.empty_like(plus)
    _check(lib().zoqat_op_weight_operand_pair(_p(w), rows, cols, group, bits, seed, tensor_id, eps, _p(plus), _p(minus), _stream()))
    return plus, minus


def zoqat_op_init_qparams(w, group, bits):
    """group = 0: one group per row."""
    rows, cols = w.shape
    theta = torch.empty((rows, cols // group if group else 1, 4), dtype=torch.float32, device=w.device)
    _check(lib().zoqat_op_init_qparams(_p(w), rows, cols, group, bits, _p(theta), _stream()))
    return theta


def zoqat_op_smooth_perturb(scale, shift, seed, scale_id, shift_id, eps):
    """-> float32 [2, 3, cols]: [sign][scale', shift', 1/scale']."""
    cols = scale.numel()
    out = torch.empty((2, 3, cols), dtype=torch.float32, device=scale.device)
    _check(lib().zoqat_op_smooth_perturb(_p(scale), _p(shift), cols, seed, scale_id, shift_id, eps, _p(out), _stream()))
    return out


def zoqat_op_weight_operand_learned(w, group, bits, seed, tensor_id, eps, theta=None, smooth=None, bias0=None,
                                    dual=True, want_codes=False):
    """-> (operand_plus, operand_minus or None, bias [signs, rows] or None, codes or None)."""
    rows, cols = w.shape
    plus = torch.empty((rows, cols), dtype=torch.bfloat16, device=w.device)
    minus = torch.empty_like(plus) if dual else None
    bias = None
    scratch = torch.empty(18 * rows * (cols // (group or 128)), dtype=torch.float32, device=w.device)
    if smooth is not None:
        bias = torch.empty((2 if dual else 1, rows), dtype=torch.float32, device=w.device)
    codes = torch.empty((rows, cols), dtype=torch.uint8, device=w.device) if want_codes else None
    _check(lib().zoqat_op_weight_operand_learned(_p(w), rows, cols, group, bits, seed, tensor_id, eps, _p(theta), _p(smooth),
                                                 _p(bias0), _p(bias), _p(scratch), _p(plus), _p(minus), _p(codes), _stream()))
    return plus, minus, bias, codes


def zoqat_op_smooth_act_operand(x, norm_kind, gain, bias, norm_eps, a_bits, smooth, rows_per_pass):
    rows, cols = x.shape
    operand = torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    row_step = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib().zoqat_op_smooth_act_operand(_p(x), rows, cols, norm_kind, _p(gain), _p(bias), norm_eps, a_bits, _p(smooth),
                                             rows_per_pass, _p(operand), _p(row_step), _stream()))
    return operand, row_step


def zoqat_packed_bytes(rows, cols, bits, group):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().zoqat_packed_bytes(rows, cols, bits, group, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def zoqat_op_pack_frozen(w, group, bits):
    rows, cols = w.shape
    cb, qb = zoqat_packed_bytes(rows, cols, bits, group)
    packed = torch.empty(cb, dtype=torch.uint8, device=w.device)
    qparams = torch.empty(qb // 4, dtype=torch.float32, device=w.device)
    _check(lib().zoqat_op_pack_frozen(_p(w), rows, cols, group, bits, _p(packed), _p(qparams), _stream()))
    return packed, qparams


def zoqat_op_unpack_operand(packed, qparams, rows, cols, group, bits):
    operand = torch.empty((rows, cols), dtype=torch.bfloat16, device=packed.device)
    _check(lib().zoqat_op_unpack_operand(_p(packed), _p(qparams), rows, cols, group, bits, _p(operand), _stream()))
    return operand


def zoqat_op_unpack_operand_i8(packed, qparams, rows, cols, bits):
    """Per-row packed tensor -> (int8 operand code - zero point, row steps, error word)."""
    operand = torch.empty((rows, cols), dtype=torch.int8, device=packed.device)
    steps = torch.empty(rows, dtype=torch.float32, device=packed.device)
    err = torch.zeros(1, dtype=torch.int32, device=packed.device)
    _check(lib().zoqat_op_unpack_operand_i8(_p(packed), _p(qparams), rows, cols, bits, _p(operand), _p(steps), _p(err), _stream()))
    return operand, steps, err


def zoqat_op_update(w, seed, tensor_id, scale):
    _check(lib().zoqat_op_update(_p(w), w.numel(), seed, tensor_id, scale, _stream()))
    return w


def zoqat_op_norm_act_operand(x, norm_kind, gain, bias, norm_eps, a_bits, want_normed=False):
    rows, cols = x.shape
    operand = torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    row_step = torch.empty(rows, dtype=torch.float32, device=x.device)
    normed = torch.empty_like(x) if want_normed else None
    _check(lib().zoqat_op_norm_act_operand(_p(x), rows, cols, norm_kind, _p(gain), _p(bias), norm_eps, a_bits,
                                           _p(operand), _p(row_step), _p(normed), _stream()))
    return operand, row_step, normed


def zoqat_op_ffn_act_operand(x, gated, a_bits):
    rows = x.shape[0]
    cols = x.shape[1] // 2 if gated else x.shape[1]
    operand = torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    row_step = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib().zoqat_op_ffn_act_operand(_p(x), rows, cols, int(gated), a_bits, _p(operand), _p(row_step), _stream()))
    return operand, row_step


def zoqat_op_gemm(a, b, row_step=None, bias=None, relu=False, out=None, accumulate=False, impl=GEMM_TCGEN05):
    M, K = a.shape
    N = b.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=a.device)
    err = torch.zeros(1, dtype=torch.int32, device=a.device)
    _check(lib().zoqat_op_gemm(_p(a), _p(b), M, N, K, _p(row_step), _p(bias), int(relu), int(accumulate), _p(out),
                               impl, _p(err), _stream()))
    return out, err


def zoqat_op_gemm_silu_gate(a, b_gate_up, row_step=None):
    M, K = a.shape
    F = b_gate_up.shape[0] // 2
    act = torch.empty((M, F), dtype=torch.float32, device=a.device)
    amax = torch.empty(M, dtype=torch.int32, device=a.device)
    err = torch.zeros(1, dtype=torch.int32, device=a.device)
    _check(lib().zoqat_op_gemm_silu_gate(_p(a), _p(b_gate_up), M, F, K, _p(row_step), _p(act), _p(amax), _p(err), _stream()))
    return act, amax.view(torch.float32), err


def zoqat_op_gemm_i8(a, b, col_step, row_step=None, bias=None, out=None, accumulate=False, gated=False):
    """a int8 [M, K], b int8 [N, K] -> (out fp32 [M, N] or [M, N/2] when gated, row maxima or None, error word)."""
    M, K = a.shape
    N = b.shape[0]
    if out is None:
        out = torch.empty((M, N // 2 if gated else N), dtype=torch.float32, device=a.device)
    amax = torch.empty(M, dtype=torch.int32, device=a.device) if gated else None
    err = torch.zeros(1, dtype=torch.int32, device=a.device)
    _check(lib().zoqat_op_gemm_i8(_p(a), _p(b), M, N, K, _p(row_step), _p(col_step), _p(bias), int(accumulate), int(gated),
                                  _p(out), _p(amax), _p(err), _stream()))
    return out, (amax.view(torch.float32) if gated else None), err


def zoqat_op_weight_operand_i8(w, bits, seed, tensor_id, eps, theta=None, smooth=None, bias0=None, dual=True):
    """-> (int8 operand of +eps, of -eps or None, steps [signs, rows], smoothed bias or None, error word)."""
    rows, cols = w.shape
    plus = torch.empty((rows, cols), dtype=torch.int8, device=w.device)
    minus = torch.empty_like(plus) if dual else None
    steps = torch.zeros((2 if dual else 1, rows), dtype=torch.float32, device=w.device)
    scratch = torch.empty(18 * rows * (cols // 128), dtype=torch.float32, device=w.device)
    bias = torch.empty((2 if dual else 1, rows), dtype=torch.float32, device=w.device) if smooth is not None else None
    err = torch.zeros(1, dtype=torch.int32, device=w.device)
    _check(lib().zoqat_op_weight_operand_i8(_p(w), rows, cols, bits, seed, tensor_id, eps, _p(theta), _p(smooth), _p(bias0),
                                            _p(bias), _p(scratch), _p(plus), _p(minus), _p(steps), _p(err), _stream()))
    return plus, minus, steps, bias, err


def zoqat_op_norm_act_operand_i8(x, norm_kind, gain, bias, norm_eps, a_bits):
    rows, cols = x.shape
    operand = torch.empty((rows, cols), dtype=torch.int8, device=x.device)
    row_step = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib().zoqat_op_norm_act_operand_i8(_p(x), rows, cols, norm_kind, _p(gain), _p(bias), norm_eps, a_bits,
                                              _p(operand), _p(row_step), _stream()))
    return operand, row_step


def zoqat_op_attention(qkv, batch, seq, n_heads, d_head, cos=None, sin=None, impl=GEMM_TCGEN05, scratch=None, err=None):
    out = torch.empty((batch * seq, n_heads * d_head), dtype=torch.float32, device=qkv.device)
    if impl == GEMM_TCGEN05:
        if scratch is None:
            nb = ctypes.c_size_t()
            _check(lib().zoqat_op_attention_scratch_bytes(batch, seq, n_heads, d_head, ctypes.byref(nb)))
            scratch = torch.empty(nb.value, dtype=torch.uint8, device=qkv.device)
        if err is None:
            err = torch.zeros(1, dtype=torch.int32, device=qkv.device)
    _check(lib().zoqat_op_attention(_p(qkv), batch, seq, n_heads, d_head, _p(cos), _p(sin), _p(out), impl, _p(scratch),
                                    _p(err), _stream()))
    return out, err


def zoqat_op_qkv_attention(a, b_qkv, batch, seq, n_heads, d_head, row_step=None, bias=None, cos=None, sin=None):
    """Fused q|k|v projection + attention; returns (out [batch*seq, d_model], err)."""
    K = a.shape[1]
    out = torch.empty((batch * seq, n_heads * d_head), dtype=torch.float32, device=a.device)
    nb = ctypes.c_size_t()
    _check(lib().zoqat_op_attention_scratch_bytes(batch, seq, n_heads, d_head, ctypes.byref(nb)))
    scratch = torch.empty(nb.value, dtype=torch.uint8, device=a.device)
    err = torch.zeros(1, dtype=torch.int32, device=a.device)
    _check(lib().zoqat_op_qkv_attention(_p(a), _p(b_qkv), batch, seq, n_heads, d_head, K, _p(row_step), _p(bias), _p(cos), _p(sin),
                                        _p(out), _p(scratch), _p(err), _stream()))
    return out, err


def zoqat_op_head_loss(a, b, labels, impl=GEMM_TCGEN05):
    T, d = a.shape
    V = b.shape[0]
    nb = ctypes.c_size_t()
    _check(lib().zoqat_op_head_loss_scratch_bytes(T, V, ctypes.byref(nb)))
    scratch = torch.empty(nb.value, dtype=torch.uint8, device=a.device)
    token_loss = torch.empty(T, dtype=torch.float32, device=a.device)
    loss_sum = torch.zeros(1, dtype=torch.float64, device=a.device)
    count = torch.zeros(1, dtype=torch.int32, device=a.device)
    err = torch.zeros(1, dtype=torch.int32, device=a.device)
    _check(lib().zoqat_op_head_loss(_p(a), _p(b), _p(labels), T, V, d, _p(token_loss), _p(loss_sum), _p(count),
                                    _p(scratch), impl, _p(err), _stream()))
    return token_loss, loss_sum, count, err


def zoqat_op_decode_gemv(packed, qparams, rows, cols, group, bits, act_codes, row_step, bias=None, out=None, accumulate=False):
    batch = act_codes.shape[0]
    if out is None:
        out = torch.empty((batch, rows), dtype=torch.float32, device=packed.device)
    scratch = torch.empty(rows * cols // 2 + 2 * batch * cols, dtype=torch.uint8, device=packed.device)
    _check(lib().zoqat_op_decode_gemv(_p(packed), _p(qparams), rows, cols, group, bits, _p(act_codes), _p(row_step), batch, _p(bias),
                                      int(accumulate), _p(out), _p(scratch), _stream()))
    return out


STATIC_SCRATCH_BYTES = 16 << 20


def zoqat_op_head_loss_static(a, b, labels, token_loss, loss_sum, count, err, impl=GEMM_TCGEN05):
    """zoqat_op_head_loss for callers that cannot allocate: the library's built-in scratch array is
    used, and every output tensor is supplied by the caller, so nothing is allocated here either."""
    T, d = a.shape
    V = b.shape[0]
    _check(lib().zoqat_op_head_loss_static(_p(a), _p(b), _p(labels), T, V, d, _p(token_loss), _p(loss_sum), _p(count),
                                           impl, _p(err), _stream()))
    return token_loss, loss_sum, count, err


# ---- serving drafted tokens over a paged cache ---------------------------------------------
_TYPES = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
_I32, _F32 = torch.int32, torch.float32


def _refuse(text):
    raise ZoqatError(ERR_INVALID_ARG, text)


def _here():
    """(index of the current device, its current stream): looked up once per call, these calls run in decode loops."""
    dev = torch.cuda.current_device()
    return dev, torch._C._cuda_getCurrentRawStream(dev)


def _flat(dev, name, t, dtype, n0, n1=None):
    """Address of a contiguous [n0] (or [n0, n1]) tensor of this type on device `dev`; sizes of -1 are free.  None -> NULL."""
    if t is None:
        return None
    s = t.shape
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        _refuse(f"{name}: a contiguous {dtype} tensor on the current CUDA device is needed")
    if len(s) != (1 if n1 is None else 2) or (n0 >= 0 and s[0] != n0) or (n1 is not None and n1 >= 0 and s[1] != n1):
        _refuse(f"{name}: shape {tuple(s)}, {(n0,) if n1 is None else (n0, n1)} is needed")
    return t.data_ptr()


def _ints(dev, *named):
    """Addresses of contiguous int32 tensors on device `dev`, each (name, tensor or None, shape)."""
    at = []
    for name, t, shape in named:
        if t is None:
            at.append(None)
        elif t.dtype is _I32 and t.shape == shape and t.get_device() == dev and t.is_contiguous():
            at.append(t.data_ptr())
        else:
            _refuse(f"{name}: a contiguous int32 tensor of shape {shape} on the current CUDA device is needed")
    return at


def _rows(dev, name, t, dtype, rows, heads, d_head):
    """(address, row stride) of [>= rows, heads, d_head] whose rows may stand apart."""
    s, st = t.shape, t.stride()
    if t.dtype is not dtype or t.get_device() != dev or len(s) != 3 or s[0] < rows or s[1] != heads or s[2] != d_head:
        _refuse(f"{name}: [{rows}, {heads}, {d_head}] of {dtype} on the current CUDA device is needed")
    if st[2] != 1 or (heads > 1 and st[1] != d_head):
        _refuse(f"{name}: heads must stand back to back")
    return t.data_ptr(), st[0] if s[0] > 1 else heads * d_head


def _caches(dev, k, v):
    s, st, ty = k.shape, k.stride(), _TYPES.get(k.dtype, -1)
    if ty < 0 or v.dtype is not k.dtype or k.get_device() != dev or v.get_device() != dev:
        _refuse("caches must both be float32, bfloat16 or float16 tensors on the current CUDA device")
    if len(s) != 4 or v.shape != s or v.stride() != st or st[3] != 1:
        _refuse("caches must be [n_pages, page_size, n_kv_heads, d_head] with the same strides and contiguous heads")
    return PagedCache(k.data_ptr(), v.data_ptr(), ty, s[0], s[1], s[2], s[3], 0, st[0], st[1], st[2])


def zoqat_op_cache_plan(cached_len, new_len, page_size, n_pages, free_pages, n_free, block_table, max_rows, parents=None, mask_words=0, out=None):
    """-> dict of int32 tensors: kv_len, row_start, row_request, row_pos, slot, n_free, status and, with mask_words, tree_mask.
    block_table is extended in place.  out: such a dict of an earlier call to write into (its status word is or-ed)."""
    dev, stream = _here()
    batch = cached_len.shape[0]
    if out is None:
        shapes = dict(kv_len=(batch,), row_start=(batch + 1,), row_request=(max_rows,), row_pos=(max_rows,), slot=(max_rows,), n_free=(1,))
        if mask_words:
            shapes["tree_mask"] = (max_rows, mask_words)
        out = {n: torch.empty(s, dtype=_I32, device=cached_len.device) for n, s in shapes.items()}
        out["status"] = torch.zeros(1, dtype=_I32, device=cached_len.device)
    _check(lib().zoqat_op_cache_plan(
        _flat(dev, "cached_len", cached_len, _I32, batch), _flat(dev, "new_len", new_len, _I32, batch), batch, page_size, n_pages,
        _flat(dev, "free_pages", free_pages, _I32, -1), free_pages.shape[0], _flat(dev, "n_free", n_free, _I32, 1),
        _flat(dev, "block_table", block_table, _I32, batch, -1), block_table.shape[1], _flat(dev, "parents", parents, _I32, max_rows), max_rows, mask_words,
        _flat(dev, "kv_len", out["kv_len"], _I32, batch), _flat(dev, "row_start", out["row_start"], _I32, batch + 1),
        _flat(dev, "row_request", out["row_request"], _I32, max_rows), _flat(dev, "row_pos", out["row_pos"], _I32, max_rows),
        _flat(dev, "slot", out["slot"], _I32, max_rows), _flat(dev, "tree_mask", out["tree_mask"], _I32, max_rows, mask_words) if mask_words else None,
        _flat(dev, "n_free", out["n_free"], _I32, 1), _flat(dev, "status", out["status"], _I32, 1), stream))
    return out


def zoqat_op_cache_append(qkv, row_pos, slot, k_cache, v_cache, n_heads, cos=None, sin=None, q_out=None, err=None):
    """qkv float32 [rows, (n_heads + 2 n_kv_heads) * d_head] -> (q_out [rows, n_heads, d_head] of the caches' type, err)."""
    dev, stream = _here()
    cache = _caches(dev, k_cache, v_cache)
    rows, dh, st = qkv.shape[0], cache.d_head, qkv.stride()
    if qkv.dtype is not _F32 or qkv.get_device() != dev or len(st) != 2 or qkv.shape[1] != (n_heads + 2 * cache.n_kv_heads) * dh or st[1] != 1:
        _refuse("qkv: float32 [rows, (n_heads + 2 n_kv_heads) * d_head] on the current CUDA device is needed")
    if q_out is None:
        q_out = torch.empty((rows, n_heads, dh), dtype=k_cache.dtype, device=qkv.device)
    if err is None:
        err = torch.zeros(1, dtype=_I32, device=qkv.device)
    q_ptr, q_stride = _rows(dev, "q_out", q_out, k_cache.dtype, rows, n_heads, dh)
    n_rope = cos.shape[0] if cos is not None else 0
    _check(lib().zoqat_op_cache_append(
        qkv.data_ptr(), st[0] if rows > 1 else qkv.shape[1], _flat(dev, "row_pos", row_pos, _I32, rows) if n_rope else None,
        _flat(dev, "slot", slot, _I32, rows), rows, n_heads, _flat(dev, "cos", cos, _F32, n_rope, dh // 2), _flat(dev, "sin", sin, _F32, n_rope, dh // 2),
        n_rope, cache, q_ptr, q_stride, _flat(dev, "err", err, _I32, 1), stream))
    return q_out, err


def zoqat_op_tree_attention(q, k_cache, v_cache, block_table, kv_len, row_start, tree_mask=None, scale=None, out=None, scratch=None, err=None):
    """q [rows, n_heads, d_head] of the caches' type -> (out of the same form, err).  scale: 1 / sqrt(d_head) by default."""
    dev, stream = _here()
    cache = _caches(dev, k_cache, v_cache)
    rows, heads, dh = q.shape
    batch = kv_len.shape[0]
    q_ptr, q_stride = _rows(dev, "q", q, k_cache.dtype, rows, heads, cache.d_head)
    words = 0
    if tree_mask is not None:
        words = tree_mask.shape[1]
        if tree_mask.shape[0] < rows:
            _refuse("tree_mask: too few rows")
    if out is None:
        out = torch.empty((rows, heads, dh), dtype=q.dtype, device=q.device)
    out_ptr, out_stride = _rows(dev, "out", out, k_cache.dtype, rows, heads, dh)
    if scratch is None:
        nb = ctypes.c_size_t()
        _check(lib().zoqat_op_tree_attention_scratch_bytes(cache.type, dh, ctypes.byref(nb)))
        scratch = torch.empty(nb.value, dtype=torch.uint8, device=q.device)
    if err is None:
        err = torch.zeros(1, dtype=_I32, device=q.device)
    if scratch.get_device() != dev or not scratch.is_contiguous():
        _refuse("scratch: a contiguous tensor on the current CUDA device is needed")
    _check(lib().zoqat_op_tree_attention(
        q_ptr, q_stride, cache, _flat(dev, "block_table", block_table, _I32, batch, -1), block_table.shape[1], _flat(dev, "kv_len", kv_len, _I32, batch),
        _flat(dev, "row_start", row_start, _I32, batch + 1), _flat(dev, "tree_mask", tree_mask, _I32, -1, words), words, batch, rows, heads,
        dh ** -0.5 if scale is None else scale, out_ptr, out_stride, scratch.data_ptr(), scratch.numel() * scratch.element_size(),
        _flat(dev, "err", err, _I32, 1), stream))
    return out, err


class LogitRules:
    """zoqat_logit_rules_t over tensors, which it keeps alive; every group may be left out."""
    __slots__ = ("desc", "tensors", "max_rows", "dev")

    def __init__(self, batch=None, row_request=None, repetition=None, presence=None, frequency=None, history=None, history_len=None,
                 prompt_len=None, bias_token=None, bias_value=None, bias_len=None, allowed=None, draft_token=None, row_start=None, tree_mask=None):
        if batch is None:
            sized = next((t for t in (history_len, repetition, presence, frequency, bias_len) if t is not None), None)
            if sized is None:
                _refuse("batch is needed when no rule is per request")
            batch = sized.shape[0]
        dev = self.dev = torch.cuda.current_device()
        n_bias = bias_token.shape[1] if bias_token is not None else 0
        self.tensors = (row_request, repetition, presence, frequency, history, history_len, prompt_len, bias_token, bias_value, bias_len, allowed,
                        draft_token, row_start, tree_mask)
        self.max_rows = min([t.shape[0] for t in (row_request, allowed, draft_token, tree_mask) if t is not None], default=1 << 30)
        self.desc = LogitRulesDesc(
            _flat(dev, "row_request", row_request, _I32, -1), _flat(dev, "repetition", repetition, _F32, batch), _flat(dev, "presence", presence, _F32, batch),
            _flat(dev, "frequency", frequency, _F32, batch), _flat(dev, "history", history, _I32, batch, -1), _flat(dev, "history_len", history_len, _I32, batch),
            _flat(dev, "prompt_len", prompt_len, _I32, batch), _flat(dev, "bias_token", bias_token, _I32, batch, n_bias),
            _flat(dev, "bias_value", bias_value, _F32, batch, n_bias), _flat(dev, "bias_len", bias_len, _I32, batch), _flat(dev, "allowed", allowed, _I32, -1, -1),
            _flat(dev, "draft_token", draft_token, _I32, -1), _flat(dev, "row_start", row_start, _I32, batch + 1), _flat(dev, "tree_mask", tree_mask, _I32, -1, -1),
            history.shape[1] if history is not None else 0, allowed.shape[1] if allowed is not None else 0, n_bias,
            tree_mask.shape[1] if tree_mask is not None else 0, batch, 0)


def zoqat_op_logit_rules(logits, rules, out=None, token=None, want_logits=True):
    """logits [rows, vocab] (rows may stand apart) -> (out of the same type or None, token int32 [rows]).  out may be logits."""
    dev, stream = _here()
    s, st, ty = logits.shape, logits.stride(), _TYPES.get(logits.dtype, -1)
    if ty < 0 or logits.get_device() != dev or rules.dev != dev or len(s) != 2 or st[1] != 1:
        _refuse("logits: [rows, vocab] of float32, bfloat16 or float16 on the current CUDA device (the rules' one) is needed")
    rows, vocab = s
    if rules.max_rows < rows:
        _refuse("rules: row_request, allowed, draft_token or tree_mask has too few rows")
    if out is None and want_logits:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    if token is None:
        token = torch.empty(rows, dtype=_I32, device=logits.device)
    out_ptr = out_ld = 0
    if out is not None:
        so = out.stride()
        if out.dtype is not logits.dtype or out.get_device() != dev or out.shape != s or so[1] != 1:
            _refuse("out: not like logits")
        out_ptr, out_ld = out.data_ptr(), so[0] if rows > 1 else max(so[0], vocab)
    _check(lib().zoqat_op_logit_rules(logits.data_ptr(), ty, st[0] if rows > 1 else max(st[0], vocab), rows, vocab, rules.desc, out_ptr, out_ld,
                                      _flat(dev, "token", token, _I32, rows), stream))
    return out, token


# ---- many continuations of one prompt --------------------------------------------------------
def rotary_frequencies(rot, base=10000.0, kind=ROTARY_PLAIN, factor=1.0, trained_len=0, device="cuda"):
    """-> (float64 tensor [rot / 2] of angles a position, magnitude): what zoqat_op_rotary_append takes."""
    freq, magnitude = (ctypes.c_double * max(1, rot // 2))(), ctypes.c_float()
    _check(lib().zoqat_rotary_frequencies(rot, base, kind, factor, trained_len, freq, ctypes.byref(magnitude)))
    return torch.tensor(list(freq), dtype=torch.float64).to(device), magnitude.value


def zoqat_op_rotary_append(qkv, row_pos, slot, k_cache, v_cache, n_heads, freq=None, interleaved=False, magnitude=1.0, q_gain=None, k_gain=None,
                           norm_eps=1e-6, q_out=None, err=None):
    """qkv [rows, (n_heads + 2 n_kv_heads) * d_head] -> (q_out [rows, n_heads, d_head] of the caches' type, err)."""
    dev, stream = _here()
    cache = _caches(dev, k_cache, v_cache)
    rows, dh, st, ty = qkv.shape[0], cache.d_head, qkv.stride(), _TYPES.get(qkv.dtype, -1)
    if ty < 0 or qkv.get_device() != dev or len(st) != 2 or qkv.shape[1] != (n_heads + 2 * cache.n_kv_heads) * dh or st[1] != 1:
        _refuse("qkv: [rows, (n_heads + 2 n_kv_heads) * d_head] of float32, bfloat16 or float16 on the current CUDA device is needed")
    if q_out is None:
        q_out = torch.empty((rows, n_heads, dh), dtype=k_cache.dtype, device=qkv.device)
    if err is None:
        err = torch.zeros(1, dtype=_I32, device=qkv.device)
    q_ptr, q_stride = _rows(dev, "q_out", q_out, k_cache.dtype, rows, n_heads, dh)
    rot = 2 * freq.shape[0] if freq is not None else 0
    _check(lib().zoqat_op_rotary_append(
        qkv.data_ptr(), ty, st[0] if rows > 1 else qkv.shape[1], _flat(dev, "row_pos", row_pos, _I32, rows) if rot else None,
        _flat(dev, "slot", slot, _I32, rows), rows, n_heads, _flat(dev, "freq", freq, torch.float64, -1), rot, int(interleaved), magnitude,
        _flat(dev, "q_gain", q_gain, _F32, dh), _flat(dev, "k_gain", k_gain, _F32, dh), norm_eps, cache, q_ptr, q_stride, _flat(dev, "err", err, _I32, 1), stream))
    return q_out, err


def prefix_attention_scratch(q, k_cache, rows=None):
    """Scratch of zoqat_op_prefix_attention for queries like q (or this many rows of them): for one call at a time."""
    nb = ctypes.c_size_t()
    _check(lib().zoqat_op_prefix_attention_scratch_bytes(_TYPES.get(k_cache.dtype, -1), k_cache.shape[3], q.shape[0] if rows is None else rows, q.shape[1], ctypes.byref(nb)))
    return torch.empty(nb.value, dtype=torch.uint8, device=q.device)


def zoqat_op_prefix_attention(q, k_cache, v_cache, block_table, kv_len, row_start, group_start, prefix_len, request_group, tree_mask=None, scale=None, out=None,
                              scratch=None, err=None):
    """zoqat_op_tree_attention for requests in groups (group_start int32 [groups + 1], request_group [batch]) that share their first prefix_len [groups]
    keys -> (out, err)."""
    dev, stream = _here()
    cache = _caches(dev, k_cache, v_cache)
    rows, heads, dh = q.shape
    batch, groups = kv_len.shape[0], prefix_len.shape[0]
    q_ptr, q_stride = _rows(dev, "q", q, k_cache.dtype, rows, heads, cache.d_head)
    words = 0
    if tree_mask is not None:
        words = tree_mask.shape[1]
        if tree_mask.shape[0] < rows:
            _refuse("tree_mask: too few rows")
    if out is None:
        out = torch.empty((rows, heads, dh), dtype=q.dtype, device=q.device)
    out_ptr, out_stride = _rows(dev, "out", out, k_cache.dtype, rows, heads, dh)
    if scratch is None:
        scratch = prefix_attention_scratch(q, k_cache)
    if err is None:
        err = torch.zeros(1, dtype=_I32, device=q.device)
    if scratch.get_device() != dev or not scratch.is_contiguous():
        _refuse("scratch: a contiguous tensor on the current CUDA device is needed")
    _check(lib().zoqat_op_prefix_attention(
        q_ptr, q_stride, cache, _flat(dev, "block_table", block_table, _I32, batch, -1), block_table.shape[1], _flat(dev, "kv_len", kv_len, _I32, batch),
        _flat(dev, "row_start", row_start, _I32, batch + 1), _flat(dev, "group_start", group_start, _I32, groups + 1), _flat(dev, "prefix_len", prefix_len, _I32, groups),
        _flat(dev, "request_group", request_group, _I32, batch), groups, _flat(dev, "tree_mask", tree_mask, _I32, -1, words), words, batch, rows, heads,
        dh ** -0.5 if scale is None else scale, out_ptr, out_stride, scratch.data_ptr(), scratch.numel() * scratch.element_size(),
        _flat(dev, "err", err, _I32, 1), stream))
    return out, err


def zoqat_op_beam_select(logits, scores, eos=None, out=None):
    """logits [batch * beams, vocab] (rows may stand apart), scores float32 [batch, beams] -> dict of [batch, beams]: beam, token, score of the
    continuations that go on, done_beam, done_token, done_score of those that end.  out: such a dict of an earlier call to write into."""
    dev, stream = _here()
    batch, beams = scores.shape
    s, st, ty = logits.shape, logits.stride(), _TYPES.get(logits.dtype, -1)
    if ty < 0 or logits.get_device() != dev or len(s) != 2 or st[1] != 1 or s[0] != batch * beams:
        _refuse("logits: [batch * beams, vocab] of float32, bfloat16 or float16 on the current CUDA device is needed")
    if out is None:
        names = dict(beam=_I32, token=_I32, score=_F32, done_beam=_I32, done_token=_I32, done_score=_F32)
        out = {n: torch.empty((batch, beams), dtype=t, device=logits.device) for n, t in names.items()}
    _check(lib().zoqat_op_beam_select(
        logits.data_ptr(), ty, st[0] if s[0] > 1 else max(st[0], s[1]), batch, beams, s[1], _flat(dev, "scores", scores, _F32, batch, beams),
        _flat(dev, "eos", eos, _I32, -1), eos.shape[0] if eos is not None else 0, _flat(dev, "beam", out["beam"], _I32, batch, beams),
        _flat(dev, "token", out["token"], _I32, batch, beams), _flat(dev, "score", out["score"], _F32, batch, beams),
        _flat(dev, "done_beam", out["done_beam"], _I32, batch, beams), _flat(dev, "done_token", out["done_token"], _I32, batch, beams),
        _flat(dev, "done_score", out["done_score"], _F32, batch, beams), stream))
    return out


def beam_reorder_scratch(parent):
    """Scratch of zoqat_op_beam_reorder for parents of this shape: for one call at a time."""
    nb = ctypes.c_size_t()
    _check(lib().zoqat_op_beam_reorder_scratch_bytes(parent.shape[0], ctypes.byref(nb)))
    return torch.empty(nb.value, dtype=torch.uint8, device=parent.device)


def zoqat_op_beam_reorder(parent, kv_len, block_table, page_size, n_pages, free_pages, n_free, shared_len=None, history=None, history_len=None, token=None,
                          out=None, scratch=None):
    """parent int32 [batch, beams]; kv_len [batch * beams], block_table [batch * beams, max_pages], history [batch * beams, any] -> dict of int32
    tensors: block_table, kv_len, free_pages, n_free, copy_from, copy_to, copy_len, status and, with history, history, history_len.  out: such a dict of
    an earlier call to write into (its status word is or-ed); its tensors are others than the inputs."""
    dev, stream = _here()
    batch, beams = parent.shape
    rows, m, cap = batch * beams, block_table.shape[1], free_pages.shape[0]
    stride = history.shape[1] if history is not None else 0
    if out is None:
        shapes = dict(block_table=(rows, m), kv_len=(rows,), free_pages=(cap,), n_free=(1,), copy_from=(rows,), copy_to=(rows,), copy_len=(rows,))
        if history is not None:
            shapes.update(history=(rows, stride), history_len=(rows,))
        out = {n: torch.full(s, -1, dtype=_I32, device=parent.device) for n, s in shapes.items()}
        out["status"] = torch.zeros(1, dtype=_I32, device=parent.device)
    if scratch is None:
        scratch = beam_reorder_scratch(parent)
    if scratch.get_device() != dev or not scratch.is_contiguous():
        _refuse("scratch: a contiguous tensor on the current CUDA device is needed")
    row, table, past = (rows,), (rows, m), (rows, stride)
    have = history is not None
    r = BeamReorder(*_ints(
        dev, ("parent", parent, (batch, beams)), ("kv_len", kv_len, row), ("block_table", block_table, table), ("shared_len", shared_len, (batch,)),
        ("free_pages", free_pages, (cap,)), ("n_free", n_free, (1,)), ("history", history, past), ("history_len", history_len, row),
        ("token", token, row if token is None or len(token.shape) == 1 else (batch, beams)), ("block_table_out", out["block_table"], table),
        ("kv_len_out", out["kv_len"], row), ("free_pages_out", out["free_pages"], (cap,)), ("n_free_out", out["n_free"], (1,)), ("copy_from", out["copy_from"], row),
        ("copy_to", out["copy_to"], row), ("copy_len", out["copy_len"], row), ("history_out", out["history"] if have else None, past),
        ("history_len_out", out["history_len"] if have else None, row), ("status", out["status"], (1,))), stride, batch, beams, page_size, n_pages, m, cap)
    _check(lib().zoqat_op_beam_reorder(r, scratch.data_ptr(), scratch.numel() * scratch.element_size(), stream))
    return out


class LayerCaches:
    """The caches of all layers, (k, v) each, described once for calls that take them together; keeps the tensors alive."""
    __slots__ = ("desc", "tensors", "dev")

    def __init__(self, caches):
        self.dev = torch.cuda.current_device()
        self.tensors = tuple((k, v) for k, v in caches)
        if not self.tensors:
            _refuse("caches: one layer at least is needed")
        self.desc = (PagedCache * len(self.tensors))(*[_caches(self.dev, k, v) for k, v in self.tensors])


def zoqat_op_cache_copy(layers, copy_from, copy_to, copy_len, err=None):
    """layers: LayerCaches; copy_from, copy_to, copy_len int32 [rows] -> err."""
    dev, stream = _here()
    rows = copy_from.shape[0]
    if layers.dev != dev:
        _refuse("caches must be on the current CUDA device")
    if err is None:
        err = torch.zeros(1, dtype=_I32, device=copy_from.device)
    _check(lib().zoqat_op_cache_copy(layers.desc, len(layers.desc), _flat(dev, "copy_from", copy_from, _I32, rows), _flat(dev, "copy_to", copy_to, _I32, rows),
                                     _flat(dev, "copy_len", copy_len, _I32, rows), rows, _flat(dev, "err", err, _I32, 1), stream))
    return err


# ---- the model handle -------------------------------------------------------------------
_LINEAR_ROLES = {"wq": ROLE_WQ, "wk": ROLE_WK, "wv": ROLE_WV, "wo": ROLE_WO, "w_gate": ROLE_W_GATE, "w_up": ROLE_W_UP,
                 "w_down": ROLE_W_DOWN, "fc1": ROLE_W_GATE, "fc2": ROLE_W_DOWN}
_VECTOR_ROLES = {"attn_norm_g": ROLE_ATTN_NORM_G, "attn_norm_b": ROLE_ATTN_NORM_B, "ffn_norm_g": ROLE_FFN_NORM_G,
                 "ffn_norm_b": ROLE_FFN_NORM_B, "bq": ROLE_BQ, "bk": ROLE_BK, "bv": ROLE_BV, "bo": ROLE_BO,
                 "b_fc1": ROLE_B_FC1, "b_fc2": ROLE_B_FC2}
_MODEL_ROLES = {"embed": ROLE_EMBED, "pos": ROLE_POS_EMBED, "final_norm_g": ROLE_FINAL_NORM_G,
                "final_norm_b": ROLE_FINAL_NORM_B, "lm_head": ROLE_LM_HEAD}


class ZoqatModel:
    """Owns the device tensors handed to zoqat_model_create and the opaque handle.

    params: dict of CUDA float32 tensors in the layout of ``synth.make_params``
    (model-level entries plus ``layers``: a list of per-layer dicts).
    first_trainable_layer: block linears of earlier layers are frozen; with
    packed_frozen=True they are FROZEN_PACKED (Section 4.3), else quantised on
    the fly from their fp32 values every pass.  trainable_names: the block linears
    that are trainable inside the trainable layers (None = all; Section 4.3 keeps
    only ("wq", "wv")); the others are frozen like the earlier layers.
    adaptive_quant / smoothing (Section 4.2): trainable block linears get learnable quantiser
    parameters (layer entry ``theta_<name>``, float32 [out, in/group, 4]; created here when absent -
    call zoqat_init_qparams() to fill them) and the trainable layers get smoothing vectors
    (``smooth_s_<point>``, ``smooth_d_<point>``; created as ones / zeros when absent).
    """

    def __init__(self, shape, params, max_batch, max_seq, gemm_impl=GEMM_TCGEN05, first_trainable_layer=0,
                 head_trainable=True, packed_frozen=False, norm_eps=1e-5, rope_base=10000.0, trainable_names=None,
                 adaptive_quant=False, smoothing=False):
        L = lib()
        self.shape = dict(shape)
        self.params = params
        self.cfg = Config(arch=ARCH_LLAMA if shape["arch"] == "llama" else ARCH_OPT, n_layers=shape["n_layers"],
                          d_model=shape["d_model"], n_heads=shape["n_heads"], d_ffn=shape["d_ffn"], vocab=shape["vocab"],
                          max_batch=max_batch, max_seq=max_seq, w_bits=shape["w_bits"], w_group=shape["w_group"],
                          a_bits=shape["a_bits"], gemm_impl=gemm_impl, norm_eps=norm_eps, rope_base=rope_base)
        self.gemm_impl = gemm_impl
        nbytes = ctypes.c_size_t()
        _check(L.zoqat_query_workspace(ctypes.byref(self.cfg), ctypes.byref(nbytes)))
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")
        self._keep = []
        descs = []
        for name, role in _MODEL_ROLES.items():
            if name in params:
                flags = TENSOR_TRAINABLE if (name == "lm_head" and head_trainable) else 0
                descs.append(TensorDesc(role, -1, flags, 0, params[name].data_ptr(), None, None))
        for l, P in enumerate(params["layers"]):
            if smoothing and l >= first_trainable_layer:
                for i, pt in enumerate(SMOOTH_POINTS):
                    n = shape["d_ffn"] if i == 3 else shape["d_model"]
                    P.setdefault("smooth_s_" + pt, torch.ones(n, dtype=torch.float32, device="cuda"))
                    P.setdefault("smooth_d_" + pt, torch.zeros(n, dtype=torch.float32, device="cuda"))
            for name, t in list(P.items()):
                if name.startswith("theta_"):
                    continue
                if name.startswith("smooth_s_") or name.startswith("smooth_d_"):
                    base = ROLE_SMOOTH_SCALE if name.startswith("smooth_s_") else ROLE_SMOOTH_SHIFT
                    descs.append(TensorDesc(base + SMOOTH_POINTS.index(name[9:]), l, 0, 0, t.data_ptr(), None, None))
                elif name in _LINEAR_ROLES:
                    if l >= first_trainable_layer and (trainable_names is None or name in trainable_names):
                        flags, th = TENSOR_TRAINABLE | TENSOR_QUANTIZED, None
                        if adaptive_quant:
                            ng = t.shape[1] // shape["w_group"] if shape["w_group"] else 1
                            th = P.setdefault("theta_" + name, torch.empty((t.shape[0], ng, 4), dtype=torch.float32, device="cuda"))
                            flags |= TENSOR_ADAPTIVE
                        descs.append(TensorDesc(_LINEAR_ROLES[name], l, flags, 0, t.data_ptr(), None,
                                                th.data_ptr() if th is not None else None))
                    elif packed_frozen:
                        cb, qb = zoqat_packed_bytes(t.shape[0], t.shape[1], shape["w_bits"], shape["w_group"])
                        pk = torch.empty(cb, dtype=torch.uint8, device="cuda")
                        qp = torch.empty(qb // 4, dtype=torch.float32, device="cuda")
                        self._keep += [pk, qp]
                        descs.append(TensorDesc(_LINEAR_ROLES[name], l, TENSOR_FROZEN_PACKED, 0, t.data_ptr(), pk.data_ptr(), qp.data_ptr()))
                    else:
                        descs.append(TensorDesc(_LINEAR_ROLES[name], l, TENSOR_QUANTIZED, 0, t.data_ptr(), None, None))
                else:
                    descs.append(TensorDesc(_VECTOR_ROLES[name], l, 0, 0, t.data_ptr(), None, None))
        arr = (TensorDesc * len(descs))(*descs)
        self.handle = ctypes.c_void_p()
        _check(L.zoqat_model_create(ctypes.byref(self.cfg), arr, len(descs), _p(self.workspace), nbytes.value,
                                    ctypes.byref(self.handle)))
        self.packed_bytes = sum(t.numel() * t.element_size() for t in self._keep)

    def close(self):
        if getattr(self, "handle", None):
            lib().zoqat_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def zoqat_prequantize_frozen(self):
        _check(lib().zoqat_prequantize_frozen(self.handle, _stream()))

    def zoqat_expand_frozen(self, on=True):
        """Expands the packed tensors once into byte operands (buffer kept alive by this object); on=False undoes it."""
        if not on:
            _check(lib().zoqat_expand_frozen(self.handle, None, 0, _stream()))
            self.expand_buffer = None
            return
        nb = ctypes.c_size_t()
        _check(lib().zoqat_expand_frozen_bytes(self.handle, ctypes.byref(nb)))
        self.expand_buffer = torch.empty(nb.value, dtype=torch.uint8, device="cuda")
        _check(lib().zoqat_expand_frozen(self.handle, _p(self.expand_buffer), nb.value, _stream()))

    def zoqat_decode_begin(self, batch, max_len):
        """Allocates the decode buffer (kept alive by this object) and converts the packed model for decoding."""
        nb = ctypes.c_size_t()
        _check(lib().zoqat_decode_bytes(self.handle, batch, max_len, ctypes.byref(nb)))
        self.decode_buffer = torch.empty(nb.value, dtype=torch.uint8, device="cuda")
        self.decode_batch = batch
        _check(lib().zoqat_decode_begin(self.handle, _p(self.decode_buffer), nb.value, batch, max_len, _stream()))
        return nb.value

    def zoqat_decode_step(self, tokens, pos, logits=None, next_token=None, want_logits=True):
        """tokens: int32 device tensor [batch].  Returns (logits [batch, vocab] or None, next_token [batch])."""
        if logits is None and want_logits:
            logits = torch.empty((self.decode_batch, self.shape["vocab"]), dtype=torch.float32, device="cuda")
        if next_token is None:
            next_token = torch.empty(self.decode_batch, dtype=torch.int32, device="cuda")
        _check(lib().zoqat_decode_step(self.handle, _p(tokens), pos, _p(logits), _p(next_token), _stream()))
        return logits, next_token

    def zoqat_decode_tree_step(self, tokens, plan, block_table, caches, rules=None, logits=None, next_token=None, scratch=None):
        """tokens int32 [rows] (1, 2, 4 or 8) at the rows of `plan` (the dict of zoqat_op_cache_plan); caches: (k, v) per layer, each
        [n_pages, page_size, n_heads, d_head]; rules: LogitRules or None.  Returns (logits [rows, vocab], next_token [rows])."""
        return self._tree_step(tokens, plan, block_table, None, caches, rules, logits, next_token, scratch)

    def zoqat_decode_prefix_step(self, tokens, plan, block_table, group_start, prefix_len, request_group, caches, rules=None, logits=None, next_token=None,
                                 scratch=None):
        """zoqat_decode_tree_step for requests in groups (group_start int32 [groups + 1], request_group [batch]) that share their first prefix_len
        [groups] keys."""
        return self._tree_step(tokens, plan, block_table, (group_start, prefix_len, request_group), caches, rules, logits, next_token, scratch)

    def _tree_step(self, tokens, plan, block_table, groups, caches, rules, logits, next_token, scratch):
        dev, stream = _here()
        rows, batch = tokens.shape[0], plan["kv_len"].shape[0]
        mask = plan.get("tree_mask")
        if len(caches) != self.shape["n_layers"]:
            _refuse("caches: one pair per layer is needed")
        if plan["row_pos"].shape[0] < rows or plan["slot"].shape[0] < rows or (mask is not None and mask.shape[0] < rows) or (
                rules is not None and (rules.max_rows < rows or rules.dev != dev)):
            _refuse("the plan or the rules have too few rows")
        tb = TreeBatch(_flat(dev, "block_table", block_table, _I32, batch, -1), _flat(dev, "kv_len", plan["kv_len"], _I32, batch),
                       _flat(dev, "row_start", plan["row_start"], _I32, batch + 1), _flat(dev, "row_pos", plan["row_pos"], _I32, -1),
                       _flat(dev, "slot", plan["slot"], _I32, -1), _flat(dev, "tree_mask", mask, _I32, -1, -1), batch, block_table.shape[1],
                       mask.shape[1] if mask is not None else 0, 0)
        descs = (PagedCache * len(caches))(*[_caches(dev, k, v) for k, v in caches])
        if logits is None:
            logits = torch.empty((rows, self.shape["vocab"]), dtype=torch.float32, device=tokens.device)
        if next_token is None:
            next_token = torch.empty(rows, dtype=torch.int32, device=tokens.device)
        if scratch is None:
            nb = ctypes.c_size_t()
            if groups is None:
                _check(lib().zoqat_op_tree_attention_scratch_bytes(descs[0].type, descs[0].d_head, ctypes.byref(nb)))
            else:
                _check(lib().zoqat_op_prefix_attention_scratch_bytes(descs[0].type, descs[0].d_head, rows, self.shape["n_heads"], ctypes.byref(nb)))
            scratch = torch.empty(nb.value, dtype=torch.uint8, device=tokens.device)
        rest = (descs, rules.desc if rules is not None else None, _flat(dev, "logits", logits, _F32, rows, self.shape["vocab"]),
                _flat(dev, "next_token", next_token, _I32, rows), scratch.data_ptr(), scratch.numel() * scratch.element_size(), stream)
        ids = _flat(dev, "tokens", tokens, _I32, rows)
        if groups is None:
            _check(lib().zoqat_decode_tree_step(self.handle, ids, rows, tb, *rest))
        else:
            start, length, of = groups
            n = length.shape[0]
            pg = PrefixGroups(_flat(dev, "group_start", start, _I32, n + 1), _flat(dev, "prefix_len", length, _I32, n), _flat(dev, "request_group", of, _I32, batch), n, 0)
            _check(lib().zoqat_decode_prefix_step(self.handle, ids, rows, tb, pg, *rest))
        return logits, next_token

    def zoqat_init_qparams(self):
        _check(lib().zoqat_init_qparams(self.handle, _stream()))

    def zoqat_step_rates(self, tokens, labels, seed, eps, lr, lr_quant, lr_smooth, result=None):
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        b, s = tokens.shape
        _check(lib().zoqat_step_rates(self.handle, _p(tokens), _p(labels), b, s, seed, eps, lr, lr_quant, lr_smooth,
                                      _p(result), _stream()))
        return result

    def zoqat_step_rates_deferred(self, tokens, labels, seed, eps, lr, lr_quant, lr_smooth, result=None):
        """zoqat_step_rates whose weight update rides on the next step's producers (or zoqat_flush_update)."""
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        b, s = tokens.shape
        _check(lib().zoqat_step_rates_deferred(self.handle, _p(tokens), _p(labels), b, s, seed, eps, lr, lr_quant, lr_smooth,
                                               _p(result), _stream()))
        return result

    def zoqat_step_finish_rates_deferred(self, sums, seed, eps, lr, lr_quant, lr_smooth, result=None):
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        _check(lib().zoqat_step_finish_rates_deferred(self.handle, _p(sums), seed, eps, lr, lr_quant, lr_smooth, _p(result), _stream()))
        return result

    def zoqat_step_finish_rates(self, sums, seed, eps, lr, lr_quant, lr_smooth, result=None):
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        _check(lib().zoqat_step_finish_rates(self.handle, _p(sums), seed, eps, lr, lr_quant, lr_smooth, _p(result), _stream()))
        return result

    def zoqat_apply_update_rates(self, seed, scale, scale_quant, scale_smooth):
        _check(lib().zoqat_apply_update_rates(self.handle, seed, scale, scale_quant, scale_smooth, _stream()))

    def zoqat_forward_loss(self, tokens, labels, seed, signed_eps, out=None):
        out = torch.empty(1, dtype=torch.float32, device="cuda") if out is None else out
        b, s = tokens.shape
        _check(lib().zoqat_forward_loss(self.handle, _p(tokens), _p(labels), b, s, seed, signed_eps, _p(out), _stream()))
        return out

    def zoqat_step(self, tokens, labels, seed, eps, lr, result=None):
        """result: int32/float32 device tensor of 6 words (zoqat_step_result_t)."""
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        b, s = tokens.shape
        _check(lib().zoqat_step(self.handle, _p(tokens), _p(labels), b, s, seed, eps, lr, _p(result), _stream()))
        return result

    def zoqat_step_deferred(self, tokens, labels, seed, eps, lr, result=None):
        """zoqat_step whose update is applied by the next deferred step (or zoqat_flush_update)."""
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        b, s = tokens.shape
        _check(lib().zoqat_step_deferred(self.handle, _p(tokens), _p(labels), b, s, seed, eps, lr, _p(result), _stream()))
        return result

    def zoqat_step_finish_deferred(self, sums, seed, eps, lr, result=None):
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        _check(lib().zoqat_step_finish_deferred(self.handle, _p(sums), seed, eps, lr, _p(result), _stream()))
        return result

    def zoqat_flush_update(self):
        _check(lib().zoqat_flush_update(self.handle, _stream()))

    def zoqat_step_multi(self, tokens, labels, seed, n_dirs, eps, lr, results=None):
        """results: float32 device tensor [n_dirs, 6] (one zoqat_step_result_t per direction)."""
        results = torch.empty((n_dirs, 6), dtype=torch.float32, device="cuda") if results is None else results
        b, s = tokens.shape
        _check(lib().zoqat_step_multi(self.handle, _p(tokens), _p(labels), b, s, seed, n_dirs, eps, lr, _p(results), _stream()))
        return results

    def zoqat_step_begin(self, tokens, labels, seed, eps, sums=None):
        """sums: float64 device tensor [3] = (sum L+, sum L-, labelled positions) of this shard."""
        sums = torch.empty(3, dtype=torch.float64, device="cuda") if sums is None else sums
        b, s = tokens.shape
        _check(lib().zoqat_step_begin(self.handle, _p(tokens), _p(labels), b, s, seed, eps, _p(sums), _stream()))
        return sums

    def zoqat_step_finish(self, sums, seed, eps, lr, result=None):
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        _check(lib().zoqat_step_finish(self.handle, _p(sums), seed, eps, lr, _p(result), _stream()))
        return result

    def zoqat_step_host(self, tokens_host, labels_host, seed, eps, lr, deferred=False):
        """tokens_host / labels_host: pinned (or pageable) CPU int32 tensors [batch, seq].  deferred: the update of the
        masters rides on the next step (zoqat_step_host_deferred)."""
        res = StepResult()
        b, s = tokens_host.shape
        fn = lib().zoqat_step_host_deferred if deferred else lib().zoqat_step_host
        _check(fn(self.handle, _p(tokens_host), _p(labels_host), b, s, seed, eps, lr, ctypes.byref(res), _stream()))
        return res

    def zoqat_apply_update(self, seed, scale):
        _check(lib().zoqat_apply_update(self.handle, seed, scale, _stream()))

    def zoqat_apply_update_multi(self, seeds, scales):
        """seeds: sequence of q integers (host); scales: float32 device tensor [q]."""
        q = len(seeds)
        arr = (ctypes.c_uint64 * q)(*[int(x) for x in seeds])
        _check(lib().zoqat_apply_update_multi(self.handle, arr, _p(scales), q, _stream()))

    def zoqat_step_result(self, sums, eps, lr, result=None):
        """Eq. (1) from the sums of zoqat_step_begin; no update."""
        result = torch.empty(6, dtype=torch.float32, device="cuda") if result is None else result
        _check(lib().zoqat_step_result(self.handle, _p(sums), eps, lr, _p(result), _stream()))
        return result

    def zoqat_check(self):
        _check(lib().zoqat_check(self.handle, _stream()))

    def zoqat_launch_count(self):
        n = ctypes.c_int64()
        _check(lib().zoqat_launch_count(self.handle, ctypes.byref(n)))
        return n.value

    def zoqat_profile_enable(self, on):
        """on: 0 off, 1 (or True) every category, 2 the GEMM launches only."""
        _check(lib().zoqat_profile_enable(self.handle, int(on)))

    def zoqat_profile_read(self, category):
        ms, n = ctypes.c_double(), ctypes.c_int64()
        _check(lib().zoqat_profile_read(self.handle, category, ctypes.byref(ms), ctypes.byref(n), _stream()))
        return ms.value, n.value

    def zoqat_debug_buffer(self, which, dtype=torch.float32):
        ptr, nb = ctypes.c_void_p(), ctypes.c_size_t()
        _check(lib().zoqat_debug_buffer(self.handle, which, ctypes.byref(ptr), ctypes.byref(nb)))
        off = ptr.value - self.workspace.data_ptr()
        return self.workspace[off:off + nb.value].view(dtype)


    def zoqat_debug_capture(self, batch, seq, passes=1):
        """Switches the quantiser capture on for forwards of this size (the buffer is allocated here and kept alive
        by this object); passes = 0 switches it off.  Returns the buffer (uint8) or None."""
        if passes == 0:
            _check(lib().zoqat_debug_capture(self.handle, None, 0))
            self.capture_buffer = None
            return None
        nb = ctypes.c_size_t()
        _check(lib().zoqat_debug_capture_bytes(self.handle, batch, seq, passes, ctypes.byref(nb)))
        self.capture_buffer = torch.zeros(nb.value, dtype=torch.uint8, device="cuda")
        _check(lib().zoqat_debug_capture(self.handle, _p(self.capture_buffer), nb.value))
        return self.capture_buffer

    def capture_records(self, rows_per_layer):
        """Splits the capture buffer of the last forward into records, in execution order:
        [(layer, point, input fp32 [rows, cols], operand bf16 [rows, cols], step fp32 [rows])], rows_per_layer[l] =
        rows materialised at layer l (passes * batch * seq; batch * seq inside a frozen prefix).  One entry more than
        the model has layers: the last one is the final norm (layer = n_layers, point 0: the vocabulary projection's
        bf16 operand, steps of 1)."""
        up = lambda n: (n + 255) // 256 * 256
        buf, off, out = self.capture_buffer, 0, []
        for l, rows in enumerate(rows_per_layer):
            for point in range(4 if l < self.shape["n_layers"] else 1):
                cols = self.shape["d_ffn"] if point == 3 else self.shape["d_model"]
                x = buf[off:off + rows * cols * 4].view(torch.float32).view(rows, cols); off += up(rows * cols * 4)
                if self.gemm_impl == GEMM_TCGEN05_I8 and l < self.shape["n_layers"]:     # signed bytes in the first half
                    op = buf[off:off + rows * cols].view(torch.int8).view(rows, cols)
                else:
                    op = buf[off:off + rows * cols * 2].view(torch.bfloat16).view(rows, cols)
                off += up(rows * cols * 2)
                st = buf[off:off + rows * 4].view(torch.float32); off += up(rows * 4)
                out.append((l, point, x, op, st))
        return out


def decode_step_result(result):
    """Device result record (6 x 32-bit words) -> dict on the host."""
    r = result.detach().cpu()
    f = r.view(torch.float32)
    i = r.view(torch.int32)
    return dict(loss_plus=float(f[0]), loss_minus=float(f[1]), proj_grad=float(f[2]), update_scale=float(f[3]),
                status=int(i[4]), n_labels=int(i[5]))


def params_to_device(params_np, device="cuda"):
    """numpy parameter dict (synth.make_params) -> dict of CUDA float32 tensors."""
    out = {k: torch.from_numpy(v).to(device) for k, v in params_np.items() if k != "layers"}
    out["layers"] = [{k: torch.from_numpy(v).to(device) for k, v in L.items()} for L in params_np["layers"]]
    return out
