"""ctypes binding of include/attn_softmax.h, lstm_stack.h, vocab_ops.h and kv_cache.h: same names, argument marshalling only.

PyTorch is used for device memory and streams; every step of the path runs in
the HIP library.  There is no fallback: if libattn_softmax.so is missing the
first call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libattn_softmax.so")
_lib = None

AS_F32, AS_BF16 = 0, 1
KC_F32, KC_BF16, KC_INT8, KC_E4M3 = 0, 1, 2, 3
AS_VIEW_ALPHA, AS_VIEW_CTX, AS_VIEW_HC, AS_VIEW_LOGITS, AS_VIEW_LSE, AS_VIEW_ROW_POS = range(6)
STATUS_NAMES = {0: "AS_OK", 1: "AS_ERR_NULL", 2: "AS_ERR_SHAPE", 3: "AS_ERR_DTYPE",
                4: "AS_ERR_WORKSPACE", 5: "AS_ERR_ALIGN", 6: "AS_ERR_HIP"}
STAGE_NAMES = ["gemm_q", "attn_score", "attn_softmax", "attn_ctx", "gemm_hc", "gemm_logits",
               "xent_stats", "xent_dlogits", "gemm_dwout", "gemm_dhc", "gemm_dwc", "gemm_dch",
               "attn_bwd", "attn_softmax_bwd", "gemm_dwa", "gemm_dh", "misc", "adam", "compact"]
AS_STATIC_SCRATCH_BYTES = 64 << 20
EXPORTS = ["attn_softmax_workspace_bytes", "attn_softmax_fwd", "attn_softmax_fwd_static", "attn_softmax_bwd", "attn_softmax_view",
           "attn_softmax_last_error", "attn_softmax_profile_enable", "attn_softmax_profile_read",
           "attn_softmax_profile_select", "attn_softmax_stream_probe",
           "attn_softmax_adam_step", "attn_softmax_step_workspace_bytes", "attn_softmax_step_prepare",
           "attn_softmax_step_fwd", "lstm_stack_workspace_bytes", "lstm_stack_fwd", "lstm_stack_bwd"]

VOCAB_EXPORTS = ["vocab_embed_workspace_bytes", "vocab_embed_fwd", "vocab_embed_bwd", "vocab_xent_workspace_bytes",
                 "vocab_xent_fwd", "vocab_xent_bwd", "vocab_distill_fwd", "vocab_distill_bwd", "vocab_verify_workspace_bytes", "vocab_verify"]

KV_EXPORTS = ["kv_cache_write", "kv_cache_read", "kv_cache_attn_workspace_bytes", "kv_cache_attn"]


class AttnSoftmaxError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


class AsShape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("S", ctypes.c_int32), ("B", ctypes.c_int32),
                ("H", ctypes.c_int32), ("V", ctypes.c_int32), ("pad_id", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("grad_scale", ctypes.c_float),
                ("dropout_p", ctypes.c_float), ("dropout_seed", ctypes.c_uint64),
                ("skip_pad_rows", ctypes.c_int32)]


class LsShape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("I", ctypes.c_int32), ("H", ctypes.c_int32),
                ("L", ctypes.c_int32), ("dtype", ctypes.c_int32), ("dropout_p", ctypes.c_float),
                ("dropout_seed", ctypes.c_uint64)]


class AsAdam(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("step", ctypes.c_int32)]


class VoEmbed(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("I", ctypes.c_int32), ("V", ctypes.c_int32), ("pad_id", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class VoShape(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("H", ctypes.c_int32), ("V", ctypes.c_int32), ("pad_id", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("grad_scale", ctypes.c_float)]


class VoTeacher(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("temperature", ctypes.c_float), ("scale", ctypes.c_float)]


class VoVerify(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("temperature", ctypes.c_float)]


class KcCache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int32), ("page", ctypes.c_int32), ("heads", ctypes.c_int32), ("D", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("cache_type", ctypes.c_int32), ("B", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


class KcAttn(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("max_len", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libattn_softmax.so (built by `python -m paper_1909_00562_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "or `python paper_1909_00562_amd/build.py`; there is no fallback path")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.attn_softmax_workspace_bytes.restype = sz
    lib.attn_softmax_workspace_bytes.argtypes = [ctypes.POINTER(AsShape)]
    lib.attn_softmax_fwd.restype = ctypes.c_int
    lib.attn_softmax_fwd.argtypes = [ctypes.POINTER(AsShape)] + [vp] * 14 + [vp, sz, vp]
    lib.attn_softmax_fwd_static.restype = ctypes.c_int
    lib.attn_softmax_fwd_static.argtypes = [ctypes.POINTER(AsShape)] + [vp] * 14 + [vp]
    lib.attn_softmax_bwd.restype = ctypes.c_int
    lib.attn_softmax_bwd.argtypes = [ctypes.POINTER(AsShape)] + [vp] * 8 + [vp, sz] + [vp] * 6 + [vp]
    lib.attn_softmax_view.restype = ctypes.c_int
    lib.attn_softmax_view.argtypes = [ctypes.POINTER(AsShape), vp, ctypes.c_int, ctypes.POINTER(vp),
                                      ctypes.POINTER(sz), ctypes.POINTER(ctypes.c_int64)]
    lib.attn_softmax_last_error.restype = ctypes.c_char_p
    lib.attn_softmax_last_error.argtypes = []
    lib.attn_softmax_profile_enable.restype = ctypes.c_int
    lib.attn_softmax_profile_enable.argtypes = [ctypes.c_int]
    lib.attn_softmax_profile_select.restype = ctypes.c_int
    lib.attn_softmax_profile_select.argtypes = [ctypes.c_uint64]
    lib.attn_softmax_profile_read.restype = ctypes.c_int
    lib.attn_softmax_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.attn_softmax_stream_probe.restype = ctypes.c_int
    lib.attn_softmax_stream_probe.argtypes = [ctypes.c_int, vp, vp, ctypes.c_int32, sz, vp]
    lib.attn_softmax_step_workspace_bytes.restype = sz
    lib.attn_softmax_step_workspace_bytes.argtypes = [ctypes.POINTER(AsShape)]
    lib.attn_softmax_step_prepare.restype = ctypes.c_int
    lib.attn_softmax_step_prepare.argtypes = [ctypes.POINTER(AsShape), vp, vp, vp, sz, vp]
    lib.attn_softmax_step_fwd.restype = ctypes.c_int
    lib.attn_softmax_step_fwd.argtypes = [ctypes.POINTER(AsShape)] + [vp] * 11 + [vp, sz, vp]
    lib.attn_softmax_adam_step.restype = ctypes.c_int
    lib.attn_softmax_adam_step.argtypes = [ctypes.POINTER(AsAdam), sz, vp, vp, vp, vp, vp, ctypes.c_int32, vp]
    lib.lstm_stack_workspace_bytes.restype = sz
    lib.lstm_stack_workspace_bytes.argtypes = [ctypes.POINTER(LsShape)]
    lib.lstm_stack_fwd.restype = ctypes.c_int
    lib.lstm_stack_fwd.argtypes = [ctypes.POINTER(LsShape)] + [vp] * 10 + [vp, sz, vp]
    lib.lstm_stack_bwd.restype = ctypes.c_int
    lib.lstm_stack_bwd.argtypes = [ctypes.POINTER(LsShape)] + [vp] * 7 + [vp, sz] + [vp] * 6 + [vp]
    pe, ps, pt = ctypes.POINTER(VoEmbed), ctypes.POINTER(VoShape), ctypes.POINTER(VoTeacher)
    lib.vocab_embed_workspace_bytes.restype = sz
    lib.vocab_embed_workspace_bytes.argtypes = [pe]
    lib.vocab_embed_fwd.restype = ctypes.c_int
    lib.vocab_embed_fwd.argtypes = [pe] + [vp] * 4
    lib.vocab_embed_bwd.restype = ctypes.c_int
    lib.vocab_embed_bwd.argtypes = [pe] + [vp] * 3 + [ctypes.c_int, vp, sz, vp]
    lib.vocab_xent_workspace_bytes.restype = sz
    lib.vocab_xent_workspace_bytes.argtypes = [ps, pt]
    lib.vocab_xent_fwd.restype = ctypes.c_int
    lib.vocab_xent_fwd.argtypes = [ps] + [vp] * 9 + [sz, vp]
    lib.vocab_xent_bwd.restype = ctypes.c_int
    lib.vocab_xent_bwd.argtypes = [ps] + [vp] * 3 + [sz] + [vp] * 4
    lib.vocab_distill_fwd.restype = ctypes.c_int
    lib.vocab_distill_fwd.argtypes = [ps, pt] + [vp] * 12 + [sz, vp]
    lib.vocab_distill_bwd.restype = ctypes.c_int
    lib.vocab_distill_bwd.argtypes = [ps, pt] + [vp] * 3 + [sz] + [vp] * 4
    pv, i32, i64 = ctypes.POINTER(VoVerify), ctypes.c_int32, ctypes.c_int64
    lib.vocab_verify_workspace_bytes.restype = sz
    lib.vocab_verify_workspace_bytes.argtypes = [pv]
    lib.vocab_verify.restype = ctypes.c_int
    lib.vocab_verify.argtypes = [pv, vp, i64, vp, i64] + [vp] * 6 + [sz, vp]
    pc, pa = ctypes.POINTER(KcCache), ctypes.POINTER(KcAttn)
    lib.kv_cache_write.restype = ctypes.c_int
    lib.kv_cache_write.argtypes = [pc, i32, vp, i64, vp, i64] + [vp] * 7 + [vp]
    lib.kv_cache_read.restype = ctypes.c_int
    lib.kv_cache_read.argtypes = [pc, i32] + [vp] * 9 + [vp]
    lib.kv_cache_attn_workspace_bytes.restype = sz
    lib.kv_cache_attn_workspace_bytes.argtypes = [pc, pa]
    lib.kv_cache_attn.restype = ctypes.c_int
    lib.kv_cache_attn.argtypes = [pc, pa, vp, i64] + [vp] * 9 + [sz, vp]
    _lib = lib
    return lib


def _ptr(x) -> Optional[int]:
    """Device/host address of a torch tensor, an int address, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _check(code: int):
    if code != 0:
        raise AttnSoftmaxError(code, attn_softmax_last_error())


def attn_softmax_last_error() -> str:
    return load_library().attn_softmax_last_error().decode()


def attn_softmax_workspace_bytes(shape: AsShape) -> int:
    return int(load_library().attn_softmax_workspace_bytes(ctypes.byref(shape)))


def attn_softmax_fwd(shape, h_dec, h_enc, src_len, W_a, W_c, W_out, b_out, targets, loss_sum, n_tok,
                     tok_loss, argmax, attn_mask, tgt_mask, workspace, workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().attn_softmax_fwd(
        ctypes.byref(shape) if shape is not None else None,
        _ptr(h_dec), _ptr(h_enc), _ptr(src_len), _ptr(W_a), _ptr(W_c), _ptr(W_out), _ptr(b_out), _ptr(targets),
        _ptr(loss_sum), _ptr(n_tok), _ptr(tok_loss), _ptr(argmax), _ptr(attn_mask), _ptr(tgt_mask),
        _ptr(workspace), int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def attn_softmax_fwd_static(shape, h_dec, h_enc, src_len, W_a, W_c, W_out, b_out, targets, loss_sum, n_tok,
                            tok_loss, argmax, attn_mask, tgt_mask, stream=0, check=True) -> int:
    """attn_softmax_fwd on the library's own static scratch (no workspace argument, nothing allocated)."""
    rc = load_library().attn_softmax_fwd_static(
        ctypes.byref(shape) if shape is not None else None,
        _ptr(h_dec), _ptr(h_enc), _ptr(src_len), _ptr(W_a), _ptr(W_c), _ptr(W_out), _ptr(b_out), _ptr(targets),
        _ptr(loss_sum), _ptr(n_tok), _ptr(tok_loss), _ptr(argmax), _ptr(attn_mask), _ptr(tgt_mask), stream or None)
    if check:
        _check(rc)
    return rc


def attn_softmax_bwd(shape, h_dec, h_enc, src_len, W_a, W_c, W_out, b_out, targets, workspace, workspace_bytes,
                     d_h_dec, d_h_enc, dW_a, dW_c, dW_out, db_out, stream=0, check=True) -> int:
    rc = load_library().attn_softmax_bwd(
        ctypes.byref(shape) if shape is not None else None,
        _ptr(h_dec), _ptr(h_enc), _ptr(src_len), _ptr(W_a), _ptr(W_c), _ptr(W_out), _ptr(b_out), _ptr(targets),
        _ptr(workspace), int(workspace_bytes),
        _ptr(d_h_dec), _ptr(d_h_enc), _ptr(dW_a), _ptr(dW_c), _ptr(dW_out), _ptr(db_out), stream or None)
    if check:
        _check(rc)
    return rc


def attn_softmax_view(shape, workspace, which: int):
    """Returns (address, bytes, row_stride_elements) of a saved activation."""
    p, n, ld = ctypes.c_void_p(), ctypes.c_size_t(), ctypes.c_int64()
    _check(load_library().attn_softmax_view(ctypes.byref(shape), _ptr(workspace), which, ctypes.byref(p),
                                            ctypes.byref(n), ctypes.byref(ld)))
    return int(p.value), int(n.value), int(ld.value)


def attn_softmax_step_workspace_bytes(shape: AsShape) -> int:
    return int(load_library().attn_softmax_step_workspace_bytes(ctypes.byref(shape)))


def attn_softmax_step_prepare(shape, h_enc, W_a, workspace, workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().attn_softmax_step_prepare(ctypes.byref(shape) if shape is not None else None, _ptr(h_enc),
                                                  _ptr(W_a), _ptr(workspace), workspace_bytes, stream)
    if check:
        _check(rc)
    return rc


def attn_softmax_step_fwd(shape, h_t, h_enc, src_len, W_c, W_out, b_out, targets, loss_sum, n_tok, tok_loss,
                          argmax, workspace, workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().attn_softmax_step_fwd(ctypes.byref(shape) if shape is not None else None, _ptr(h_t),
                                              _ptr(h_enc), _ptr(src_len), _ptr(W_c), _ptr(W_out), _ptr(b_out),
                                              _ptr(targets), _ptr(loss_sum), _ptr(n_tok), _ptr(tok_loss),
                                              _ptr(argmax), _ptr(workspace), workspace_bytes, stream)
    if check:
        _check(rc)
    return rc


def attn_softmax_adam_step(hyper: AsAdam, n: int, grad, master, m, v, weights_out, dtype: int, stream: int = 0,
                           check=True) -> int:
    rc = load_library().attn_softmax_adam_step(ctypes.byref(hyper) if hyper is not None else None, n, _ptr(grad),
                                               _ptr(master), _ptr(m), _ptr(v), _ptr(weights_out), dtype, stream)
    if check:
        _check(rc)
    return rc


def _ptr_array(tensors):
    """Host array of device addresses (one per layer); None stays NULL."""
    if tensors is None:
        return None
    arr = (ctypes.c_void_p * len(tensors))(*[_ptr(t) for t in tensors])
    return ctypes.cast(arr, ctypes.c_void_p), arr      # the second element keeps the array alive


def lstm_stack_workspace_bytes(shape: LsShape) -> int:
    return int(load_library().lstm_stack_workspace_bytes(ctypes.byref(shape)))


def lstm_stack_fwd(shape, x, lengths, W_ih, W_hh, b, h0, c0, y, hT, cT, workspace, workspace_bytes, stream=0,
                   check=True) -> int:
    """W_ih, W_hh, b: sequences of L device tensors (or addresses)."""
    arrs = [_ptr_array(a) for a in (W_ih, W_hh, b)]
    rc = load_library().lstm_stack_fwd(ctypes.byref(shape) if shape is not None else None, _ptr(x), _ptr(lengths),
                                       *[a[0] if a else None for a in arrs], _ptr(h0), _ptr(c0), _ptr(y), _ptr(hT),
                                       _ptr(cT), _ptr(workspace), int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def lstm_stack_bwd(shape, x, lengths, W_ih, W_hh, dy, dhT, dcT, workspace, workspace_bytes, dx, dW_ih, dW_hh, db,
                   dh0, dc0, stream=0, check=True) -> int:
    ins = [_ptr_array(a) for a in (W_ih, W_hh)]
    outs = [_ptr_array(a) for a in (dW_ih, dW_hh, db)]
    rc = load_library().lstm_stack_bwd(ctypes.byref(shape) if shape is not None else None, _ptr(x), _ptr(lengths),
                                       *[a[0] if a else None for a in ins], _ptr(dy), _ptr(dhT), _ptr(dcT),
                                       _ptr(workspace), int(workspace_bytes), _ptr(dx),
                                       *[a[0] if a else None for a in outs], _ptr(dh0), _ptr(dc0), stream or None)
    if check:
        _check(rc)
    return rc


def _ref(struct):
    return ctypes.byref(struct) if struct is not None else None


def _addresses(*tensors):
    """Device addresses of torch tensors (or int addresses, or None)."""
    return [t if t is None or type(t) is int else t.data_ptr() for t in tensors]


def vocab_embed_workspace_bytes(shape: VoEmbed) -> int:
    return int(load_library().vocab_embed_workspace_bytes(_ref(shape)))


def vocab_embed_fwd(shape, table, ids, x, stream=0, check=True) -> int:
    rc = load_library().vocab_embed_fwd(_ref(shape), *_addresses(table, ids, x), stream or None)
    if check:
        _check(rc)
    return rc


def vocab_embed_bwd(shape, ids, dy, d_table, accumulate, workspace, workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().vocab_embed_bwd(_ref(shape), *_addresses(ids, dy, d_table), int(accumulate),
                                        *_addresses(workspace), int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def vocab_xent_workspace_bytes(shape: VoShape, teacher=None) -> int:
    return int(load_library().vocab_xent_workspace_bytes(_ref(shape), _ref(teacher)))


def vocab_xent_fwd(shape, h, W, b, targets, loss_sum, n_tok, tok_loss, argmax, workspace, workspace_bytes, stream=0,
                   check=True) -> int:
    rc = load_library().vocab_xent_fwd(_ref(shape), *_addresses(h, W, b, targets, loss_sum, n_tok, tok_loss, argmax, workspace),
                                       int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def vocab_xent_bwd(shape, W, b, workspace, workspace_bytes, dh, dW, db, stream=0, check=True) -> int:
    rc = load_library().vocab_xent_bwd(_ref(shape), *_addresses(W, b, workspace), int(workspace_bytes), *_addresses(dh, dW, db),
                                       stream or None)
    if check:
        _check(rc)
    return rc


def vocab_distill_fwd(shape, teacher, h, W, b, targets, teacher_ids, teacher_logits, loss_sum, n_tok, distill_sum,
                      tok_loss, tok_distill, workspace, workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().vocab_distill_fwd(_ref(shape), _ref(teacher),
                                          *_addresses(h, W, b, targets, teacher_ids, teacher_logits, loss_sum, n_tok,
                                                      distill_sum, tok_loss, tok_distill, workspace),
                                          int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def vocab_distill_bwd(shape, teacher, W, b, workspace, workspace_bytes, dh, dW, db, stream=0, check=True) -> int:
    rc = load_library().vocab_distill_bwd(_ref(shape), _ref(teacher), *_addresses(W, b, workspace),
                                          int(workspace_bytes), *_addresses(dh, dW, db), stream or None)
    if check:
        _check(rc)
    return rc


def vocab_verify_workspace_bytes(shape: VoVerify) -> int:
    return int(load_library().vocab_verify_workspace_bytes(_ref(shape)))


def vocab_verify(shape, target, ld_target, draft, ld_draft, drafted, u_accept, u_next, n_accepted, words, workspace,
                 workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().vocab_verify(_ref(shape), *_addresses(target), int(ld_target), *_addresses(draft), int(ld_draft),
                                     *_addresses(drafted, u_accept, u_next, n_accepted, words, workspace),
                                     int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def kv_cache_write(cache, N, k, ld_k, v, ld_v, seq, pos, page_table, k_pages, v_pages, k_scales, v_scales, stream=0,
                   check=True) -> int:
    rc = load_library().kv_cache_write(_ref(cache), int(N), *_addresses(k), int(ld_k), *_addresses(v), int(ld_v),
                                       *_addresses(seq, pos, page_table, k_pages, v_pages, k_scales, v_scales), stream or None)
    if check:
        _check(rc)
    return rc


def kv_cache_read(cache, N, k_pages, v_pages, k_scales, v_scales, seq, pos, page_table, k, v, stream=0, check=True) -> int:
    rc = load_library().kv_cache_read(_ref(cache), int(N), *_addresses(k_pages, v_pages, k_scales, v_scales, seq, pos, page_table, k, v),
                                      stream or None)
    if check:
        _check(rc)
    return rc


def kv_cache_attn_workspace_bytes(cache: KcCache, attn: KcAttn) -> int:
    return int(load_library().kv_cache_attn_workspace_bytes(_ref(cache), _ref(attn)))


def kv_cache_attn(cache, attn, q, ld_q, k_pages, v_pages, k_scales, v_scales, page_table, lengths, out, lse, workspace,
                  workspace_bytes, stream=0, check=True) -> int:
    rc = load_library().kv_cache_attn(_ref(cache), _ref(attn), *_addresses(q), int(ld_q),
                                      *_addresses(k_pages, v_pages, k_scales, v_scales, page_table, lengths, out, lse, workspace),
                                      int(workspace_bytes), stream or None)
    if check:
        _check(rc)
    return rc


def attn_softmax_stream_probe(kind: int, buf, buf2, rows: int, row_bytes: int, stream=0, check=True) -> int:
    rc = load_library().attn_softmax_stream_probe(int(kind), _ptr(buf), _ptr(buf2), int(rows), int(row_bytes),
                                                  stream or None)
    if check:
        _check(rc)
    return rc


def attn_softmax_profile_enable(enable: bool):
    _check(load_library().attn_softmax_profile_enable(1 if enable else 0))


def attn_softmax_profile_select(stages) -> None:
    """Time only the named stages (names as in STAGE_NAMES) until profiling is enabled again."""
    mask = 0
    for name in stages:
        mask |= 1 << STAGE_NAMES.index(name)
    _check(load_library().attn_softmax_profile_select(mask))


def attn_softmax_profile_read() -> Dict[str, dict]:
    n = len(STAGE_NAMES)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(load_library().attn_softmax_profile_read(ms, cnt))
    return {STAGE_NAMES[i]: {"ms": ms[i], "launches": int(cnt[i])} for i in range(n)}


class DeviceBatch:
    """Device buffers for one batch: uploads the inputs, owns outputs and the
    workspace, and forwards to the C ABI.  No arithmetic happens here."""

    def __init__(self, inp, device="cuda:0", skip_pad_rows=False):
        import torch
        self.torch = torch
        self.inp = inp
        self.dev = torch.device(device)
        bf = inp.dtype == "bf16"
        self.shape = AsShape(inp.T, inp.S, inp.B, inp.H, inp.V, inp.pad_id, AS_BF16 if bf else AS_F32,
                             float(inp.grad_scale), float(getattr(inp, "dropout_p", 0.0)),
                             int(getattr(inp, "dropout_seed", 0)), 1 if skip_pad_rows else 0)
        tdt = torch.bfloat16 if bf else torch.float32
        self.tdt = tdt

        def up(a):   # values are already representable in the storage type
            return torch.from_numpy(np.ascontiguousarray(a)).to(tdt).to(self.dev)

        self.h_dec, self.h_enc = up(inp.h_dec), up(inp.h_enc)
        self.W_a, self.W_c, self.W_out, self.b_out = up(inp.W_a), up(inp.W_c), up(inp.W_out), up(inp.b_out)
        self.src_len = torch.from_numpy(inp.src_len.astype(np.int32)).to(self.dev)
        self.targets = torch.from_numpy(np.ascontiguousarray(inp.targets, dtype=np.int32)).to(self.dev)
        T, S, B, H, V = inp.T, inp.S, inp.B, inp.H, inp.V
        f32, i32, u8 = torch.float32, torch.int32, torch.uint8
        self.loss_sum = torch.zeros(1, dtype=f32, device=self.dev)
        self.n_tok = torch.zeros(1, dtype=i32, device=self.dev)
        self.tok_loss = torch.zeros(T, B, dtype=f32, device=self.dev)
        self.argmax = torch.zeros(T, B, dtype=i32, device=self.dev)
        self.attn_mask = torch.zeros(B, S, dtype=u8, device=self.dev)
        self.tgt_mask = torch.zeros(T, B, dtype=u8, device=self.dev)
        self.ws_bytes = attn_softmax_workspace_bytes(self.shape)
        if self.ws_bytes == 0:
            raise AttnSoftmaxError(2, "invalid shape for workspace")
        self.workspace = torch.empty(self.ws_bytes, dtype=u8, device=self.dev)
        self.d_h_dec = torch.empty(T, B, H, dtype=f32, device=self.dev)
        self.d_h_enc = torch.empty(S, B, H, dtype=f32, device=self.dev)
        self.dW_a = torch.empty(H, H, dtype=f32, device=self.dev)
        self.dW_c = torch.empty(H, 2 * H, dtype=f32, device=self.dev)
        self.dW_out = torch.empty(V, H, dtype=f32, device=self.dev)
        self.db_out = torch.empty(V, dtype=f32, device=self.dev)

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream(self.dev).cuda_stream)

    def fwd(self):
        attn_softmax_fwd(self.shape, self.h_dec, self.h_enc, self.src_len, self.W_a, self.W_c, self.W_out,
                         self.b_out, self.targets, self.loss_sum, self.n_tok, self.tok_loss, self.argmax,
                         self.attn_mask, self.tgt_mask, self.workspace, self.ws_bytes, self._stream())

    def bwd(self):
        attn_softmax_bwd(self.shape, self.h_dec, self.h_enc, self.src_len, self.W_a, self.W_c, self.W_out,
                         self.b_out, self.targets, self.workspace, self.ws_bytes, self.d_h_dec, self.d_h_enc,
                         self.dW_a, self.dW_c, self.dW_out, self.db_out, self._stream())

    def view(self, which: int):
        """Saved activation as a torch tensor aliasing the workspace.  With skip_pad_rows the logits and lse
        views are [N, V] / [N] with one row per non-pad position (AS_VIEW_ROW_POS maps (t, b) to its row)."""
        torch = self.torch
        addr, nbytes, ld = attn_softmax_view(self.shape, self.workspace, which)
        off = addr - self.workspace.data_ptr()
        raw = self.workspace[off:off + nbytes]
        T, S, B, H, V = self.inp.T, self.inp.S, self.inp.B, self.inp.H, self.inp.V
        if which == AS_VIEW_ALPHA:
            return raw.view(torch.float32).view(B, T, S)
        compact = self.shape.skip_pad_rows != 0
        if which == AS_VIEW_ROW_POS:
            return raw.view(torch.int32).view(T, B)
        if which == AS_VIEW_LSE:
            return raw.view(torch.float32).view(T * B) if compact else raw.view(torch.float32).view(T, B)
        if which in (AS_VIEW_CTX, AS_VIEW_HC):
            return raw.view(self.tdt).view(T, B, H)
        if which == AS_VIEW_LOGITS:
            if compact:
                return raw.view(self.tdt).view(T * B, ld)[:, :V]
            return raw.view(self.tdt).view(T, B, ld)[:, :, :V]
        raise ValueError(which)

    def sync(self):
        self.torch.cuda.synchronize(self.dev)


class DeviceLstm:
    """Device buffers for one side (encoder or decoder) of the stacked LSTM: uploads the inputs, owns the
    outputs and the workspace, and forwards to the C ABI.  No arithmetic happens here.
    x [T,B,I], lengths [B], W_ih / W_hh / b: lists of L arrays, h0 / c0 [L,B,H] or None (numpy, values already
    representable in the storage type)."""

    def __init__(self, x, lengths, W_ih, W_hh, b, h0=None, c0=None, dtype="f32", device="cuda:0", dropout_p=0.0,
                 dropout_seed=0):
        import torch
        self.torch = torch
        self.dev = torch.device(device)
        bf = dtype == "bf16"
        tdt = torch.bfloat16 if bf else torch.float32
        self.tdt = tdt
        T, B, I = x.shape
        L, H = len(W_ih), W_hh[0].shape[1]
        self.T, self.B, self.I, self.H, self.L = T, B, I, H, L
        self.shape = LsShape(T, B, I, H, L, AS_BF16 if bf else AS_F32, float(dropout_p), int(dropout_seed))
        f32 = torch.float32

        def up(a, dt=tdt):
            return torch.from_numpy(np.ascontiguousarray(a)).to(dt).to(self.dev)

        self.x = up(x)
        self.lengths = torch.from_numpy(np.asarray(lengths, dtype=np.int32)).to(self.dev)
        self.W_ih = [up(w) for w in W_ih]
        self.W_hh = [up(w) for w in W_hh]
        self.b = [up(v) for v in b]
        self.h0 = up(h0, f32) if h0 is not None else None
        self.c0 = up(c0, f32) if c0 is not None else None
        self.y = torch.empty(T, B, H, dtype=tdt, device=self.dev)
        self.hT = torch.empty(L, B, H, dtype=f32, device=self.dev)
        self.cT = torch.empty(L, B, H, dtype=f32, device=self.dev)
        self.ws_bytes = lstm_stack_workspace_bytes(self.shape)
        if self.ws_bytes == 0:
            raise AttnSoftmaxError(2, "invalid shape for the LSTM workspace")
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev)
        self.dx = torch.empty(T, B, I, dtype=f32, device=self.dev)
        self.dW_ih = [torch.empty(w.shape, dtype=f32, device=self.dev) for w in self.W_ih]
        self.dW_hh = [torch.empty(w.shape, dtype=f32, device=self.dev) for w in self.W_hh]
        self.db = [torch.empty(v.shape, dtype=f32, device=self.dev) for v in self.b]
        self.dh0 = torch.empty(L, B, H, dtype=f32, device=self.dev)
        self.dc0 = torch.empty(L, B, H, dtype=f32, device=self.dev)

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream(self.dev).cuda_stream)

    def fwd(self):
        lstm_stack_fwd(self.shape, self.x, self.lengths, self.W_ih, self.W_hh, self.b, self.h0, self.c0, self.y,
                       self.hT, self.cT, self.workspace, self.ws_bytes, self._stream())

    def bwd(self, dy, dhT=None, dcT=None):
        """dy [T,B,H], dhT / dcT [L,B,H]: float32 device tensors (or None)."""
        lstm_stack_bwd(self.shape, self.x, self.lengths, self.W_ih, self.W_hh, dy, dhT, dcT, self.workspace,
                       self.ws_bytes, self.dx, self.dW_ih, self.dW_hh, self.db, self.dh0, self.dc0, self._stream())

    def sync(self):
        self.torch.cuda.synchronize(self.dev)


def _as_dtype(t) -> int:
    import torch
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise AttnSoftmaxError(3, f"storage type {t.dtype}")
    return AS_BF16 if t.dtype == torch.bfloat16 else AS_F32


def _grad_dtype(grad_dtype, dtype: int) -> int:
    if grad_dtype not in (None, "f32", "bf16"):
        raise AttnSoftmaxError(3, f"gradient type {grad_dtype!r}")
    return dtype if grad_dtype is None else AS_BF16 if grad_dtype == "bf16" else AS_F32


class _DeviceOp:
    """Checks of the tensors that a call is given (shape, type, device, dense rows) and the stream it goes to: the
    current one of the tensors' device, with that device current for the call.  (Written for few interpreter steps: a
    decoder step's kernels take as long as the host needs for the call.)"""

    def _on(self, device):
        import torch
        if device.type != "cuda":
            raise AttnSoftmaxError(2, f"tensors are on {device}, expected a GPU")
        self.torch, self.dev, self.index = torch, device, device.index
        torch.cuda.init()
        # (the address of the current stream and the current device's number, without making objects of them)
        self.stream_of, self.current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        self.lib = load_library()
        self.workspace = None

    def _own_workspace(self):
        torch = self.torch
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.dev)
        self.home = torch.cuda.current_stream(self.dev).cuda_stream

    def _tensor(self, t, shape, dtype, name):
        if t is None:
            raise AttnSoftmaxError(1, f"{name} is None")
        if t.shape != shape:
            raise AttnSoftmaxError(2, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.dtype is not dtype:
            raise AttnSoftmaxError(3, f"{name} is {t.dtype}, expected {dtype}")
        if t.get_device() != self.index:
            raise AttnSoftmaxError(2, f"{name} is on {t.device}, expected {self.dev}")
        if not t.is_contiguous():
            raise AttnSoftmaxError(5, f"{name} is not dense row-major")
        return t.data_ptr()

    def _optional(self, t, shape, dtype, name):
        return None if t is None else self._tensor(t, shape, dtype, name)

    def _rows(self, t, shape, dtype, name, inner):
        """(address, elements from row to row) of a tensor whose first dimensions are rows the same distance apart, each dense with
        the strides `inner`: a part of a wider projection, or logits with padding."""
        if t is None:
            raise AttnSoftmaxError(1, f"{name} is None")
        if t.shape != shape:
            raise AttnSoftmaxError(2, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.dtype is not dtype:
            raise AttnSoftmaxError(3, f"{name} is {t.dtype}, expected {dtype}")
        if t.get_device() != self.index:
            raise AttnSoftmaxError(2, f"{name} is on {t.device}, expected {self.dev}")
        strides = t.stride()
        ahead = len(shape) - len(inner)
        if strides[ahead:] != inner:
            for n, stride, dense in zip(shape[ahead:], strides[ahead:], inner):
                if n != 1 and stride != dense:
                    raise AttnSoftmaxError(5, f"the rows of {name} are not dense")
        row = strides[ahead - 1]
        if shape[ahead - 1] == 1 or ahead == 2 and shape[0] > 1:
            a, b = (1, shape[0]) if ahead == 1 else shape[:2]      # (dimensions of one have any stride)
            if b == 1:
                whole = 16 // t.element_size()
                row = strides[0] if a > 1 else -(-inner[0] * shape[ahead] // whole) * whole
            elif a > 1 and strides[0] != b * row:
                raise AttnSoftmaxError(5, f"the rows of {name} are not the same distance apart")
        return t.data_ptr(), row

    def _call(self, function, *args):
        """function(*args, stream), for addresses that _tensor has checked.  The workspace is the handle's own, so the allocator is
        told here of a stream other than the one it was allocated on: a handle may be dropped while calls are on their way."""
        stream = self.stream_of(self.index)
        if self.workspace is not None and stream != self.home:
            self.workspace.record_stream(self.torch.cuda.current_stream(self.dev))
        if self.current_device() == self.index:
            rc = function(*args, stream or None)
        else:
            with self.torch.cuda.device(self.dev):
                rc = function(*args, stream or None)
        if rc:
            _check(rc)


class DeviceEmbed(_DeviceOp):
    """Embedding of N positions at a time (shorter batches: ids of -1 behind them, or a handle of their own length) in a table
    [V,I] (a device tensor, not copied): owns the workspace of the backward pass and forwards to the C ABI.  grad_dtype: "f32" or "bf16", the type of dy and of the table's gradient."""

    def __init__(self, table, N, pad_id=-1, scale=1.0, grad_dtype=None):
        self._on(table.device)
        torch = self.torch
        dtype = _as_dtype(table)
        V, I = table.shape
        self.table, self.tdt = table, table.dtype
        self._tensor(table, (V, I), self.tdt, "table")
        self.shape = VoEmbed(N, I, V, pad_id, dtype, _grad_dtype(grad_dtype, dtype), float(scale))
        self.shape_ref = ctypes.byref(self.shape)
        self.n, self.rows = (N,), (N, I)
        self.gdt = torch.bfloat16 if self.shape.grad_dtype == AS_BF16 else torch.float32
        self.ws_bytes = vocab_embed_workspace_bytes(self.shape)
        if self.ws_bytes == 0:
            raise AttnSoftmaxError(2, "invalid shape for the embedding")

    def fwd(self, ids, x=None):
        """x [N,I] = scale * table[ids]; ids [N] int32."""
        torch = self.torch
        if x is None:
            x = torch.empty(self.rows, dtype=self.tdt, device=self.dev)
        self._call(self.lib.vocab_embed_fwd, self.shape_ref, self.table.data_ptr(),
                   self._tensor(ids, self.n, torch.int32, "ids"), self._tensor(x, self.rows, self.tdt, "x"))
        return x

    def bwd(self, ids, dy, d_table=None, accumulate=False):
        """d_table [V,I] = (d_table +) scale * sums of the rows of dy [N,I] per word."""
        torch, s = self.torch, self.shape
        if d_table is None:
            if accumulate:
                raise AttnSoftmaxError(1, "d_table is None")
            d_table = torch.empty(s.V, s.I, dtype=self.gdt, device=self.dev)
        if self.workspace is None:
            self._own_workspace()
        self._call(self.lib.vocab_embed_bwd, self.shape_ref, self._tensor(ids, self.n, torch.int32, "ids"),
                   self._tensor(dy, self.rows, self.gdt, "dy"), self._tensor(d_table, (s.V, s.I), self.gdt, "d_table"),
                   int(accumulate), self.workspace.data_ptr(), self.ws_bytes)
        return d_table


class DeviceVocabLoss(_DeviceOp):
    """Cross-entropy (and, with K > 0, distillation from a teacher's top K logits) of N positions over a vocabulary with the
    projection W [V,H] and bias b [V] or None (device tensors, not copied): owns the workspace, which carries what a
    backward pass needs of the forward pass ahead of it, and forwards to the C ABI.  grad_dtype: "f32" or "bf16"."""

    def __init__(self, W, b, N, pad_id=-1, grad_scale=1.0, grad_dtype=None, K=0, temperature=1.0, distill_scale=1.0):
        self._on(W.device)
        torch = self.torch
        dtype = _as_dtype(W)
        V, H = W.shape
        self.W, self.b, self.tdt = W, b, W.dtype
        self._tensor(W, (V, H), self.tdt, "W")
        self._optional(b, (V,), self.tdt, "b")
        self.shape = VoShape(N, H, V, pad_id, dtype, _grad_dtype(grad_dtype, dtype), float(grad_scale))
        self.gdt = torch.bfloat16 if self.shape.grad_dtype == AS_BF16 else torch.float32
        self.teacher = VoTeacher(K, float(temperature), float(distill_scale)) if K else None
        self.refs = (ctypes.byref(self.shape),) + ((ctypes.byref(self.teacher),) if K else ())
        self.one, self.n, self.rows, self.entries = (1,), (N,), (N, H), (N, K)
        self.ws_bytes = vocab_xent_workspace_bytes(self.shape, self.teacher)
        if self.ws_bytes == 0:
            raise AttnSoftmaxError(2, "invalid shape for the vocabulary loss")
        self._own_workspace()
        self.done = False

    def _weights(self):
        return self.W.data_ptr(), None if self.b is None else self.b.data_ptr()

    def xent_fwd(self, h, targets, loss_sum, n_tok, tok_loss=None, argmax=None):
        if self.teacher is not None:
            raise AttnSoftmaxError(2, "this workspace is for distillation (K > 0): distill_fwd")
        f32, i32, check, n = self.torch.float32, self.torch.int32, self._tensor, self.n
        self._call(self.lib.vocab_xent_fwd, *self.refs, check(h, self.rows, self.tdt, "h"), *self._weights(),
                   check(targets, n, i32, "targets"), check(loss_sum, self.one, f32, "loss_sum"),
                   check(n_tok, self.one, i32, "n_tok"), self._optional(tok_loss, n, f32, "tok_loss"),
                   self._optional(argmax, n, i32, "argmax"), self.workspace.data_ptr(), self.ws_bytes)
        self.done = True

    def distill_fwd(self, h, targets, teacher_ids, teacher_logits, loss_sum, n_tok, distill_sum, tok_loss=None,
                    tok_distill=None):
        if self.teacher is None:
            raise AttnSoftmaxError(1, "no teacher (K = 0): xent_fwd")
        f32, i32, check, n = self.torch.float32, self.torch.int32, self._tensor, self.n
        self._call(self.lib.vocab_distill_fwd, *self.refs, check(h, self.rows, self.tdt, "h"), *self._weights(),
                   check(targets, n, i32, "targets"), check(teacher_ids, self.entries, i32, "teacher_ids"),
                   check(teacher_logits, self.entries, f32, "teacher_logits"), check(loss_sum, self.one, f32, "loss_sum"),
                   check(n_tok, self.one, i32, "n_tok"), check(distill_sum, self.one, f32, "distill_sum"),
                   self._optional(tok_loss, n, f32, "tok_loss"), self._optional(tok_distill, n, f32, "tok_distill"),
                   self.workspace.data_ptr(), self.ws_bytes)
        self.done = True

    def _bwd(self, function, dh, dW, db):
        s, gdt = self.shape, self.gdt
        if not self.done:
            raise AttnSoftmaxError(2, "a backward pass without the forward pass ahead of it")
        self._call(function, *self.refs, *self._weights(), self.workspace.data_ptr(), self.ws_bytes,
                   self._tensor(dh, self.rows, gdt, "dh"), self._tensor(dW, (s.V, s.H), gdt, "dW"),
                   self._optional(db, (s.V,), gdt, "db"))

    def xent_bwd(self, dh, dW, db=None):
        if self.teacher is not None:
            raise AttnSoftmaxError(2, "this workspace is for distillation (K > 0): distill_bwd")
        self._bwd(self.lib.vocab_xent_bwd, dh, dW, db)

    def distill_bwd(self, dh, dW, db=None):
        if self.teacher is None:
            raise AttnSoftmaxError(1, "no teacher (K = 0): xent_bwd")
        self._bwd(self.lib.vocab_distill_bwd, dh, dW, db)


class DeviceVocabVerify(_DeviceOp):
    """Verification of T drafted words of each of B sequences against the target's logits (vocab_ops.h): owns the workspace and
    forwards to the C ABI.  Shorter drafts end with ids outside the vocabulary (-1)."""

    def __init__(self, B, T, V, dtype="bf16", temperature=1.0, device="cuda:0"):
        import torch
        device = torch.device(device)
        self._on(torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device)
        if dtype not in ("f32", "bf16"):
            raise AttnSoftmaxError(3, f"logits of type {dtype!r}")
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.shape = VoVerify(B, T, V, AS_BF16 if dtype == "bf16" else AS_F32, float(temperature))
        self.ref = ctypes.byref(self.shape)
        self.b, self.bt, self.bt1, self.target_shape, self.draft_shape = (B,), (B, T), (B, T + 1), (B, T + 1, V), (B, T, V)
        self.ws_bytes = vocab_verify_workspace_bytes(self.shape)
        if self.ws_bytes == 0:
            raise AttnSoftmaxError(2, "invalid shape for the verification")
        self._own_workspace()

    def verify(self, target, draft, drafted, u_accept, u_next, n_accepted=None, words=None):
        """(n_accepted [B], words [B,T+1]) int32; target [B,T+1,V] and draft [B,T,V] logits, drafted [B,T] int32, u_accept [B,T]
        and u_next [B] float32 in [0,1)."""
        torch = self.torch
        f32, i32 = torch.float32, torch.int32
        if n_accepted is None:
            n_accepted = torch.empty(self.b, dtype=i32, device=self.dev)
        if words is None:
            words = torch.empty(self.bt1, dtype=i32, device=self.dev)
        check = self._tensor
        self._call(self.lib.vocab_verify, self.ref, *self._rows(target, self.target_shape, self.tdt, "target", (1,)),
                   *self._rows(draft, self.draft_shape, self.tdt, "draft", (1,)), check(drafted, self.bt, i32, "drafted"),
                   check(u_accept, self.bt, f32, "u_accept"), check(u_next, self.b, f32, "u_next"),
                   check(n_accepted, self.b, i32, "n_accepted"), check(words, self.bt1, i32, "words"),
                   self.workspace.data_ptr(), self.ws_bytes)
        return n_accepted, words


class DeviceKvCache(_DeviceOp):
    """A paged cache of keys and values (kv_cache.h): k_pages, v_pages [pages, heads, page, D] (device tensors, not copied) of float32,
    bfloat16, int8 or float8_e4m3fn, in 8 bits with scales [pages, heads, page] float32.  dtype: "f32" or "bf16", the type of what is
    written and read (in 8 bits; else the pages')."""

    def __init__(self, k_pages, v_pages, k_scales=None, v_scales=None, dtype=None):
        self._on(k_pages.device)
        torch = self.torch
        kinds = {torch.float32: KC_F32, torch.bfloat16: KC_BF16, torch.int8: KC_INT8, torch.float8_e4m3fn: KC_E4M3}
        if k_pages.dtype not in kinds:
            raise AttnSoftmaxError(3, f"storage type {k_pages.dtype}")
        kind = kinds[k_pages.dtype]
        coded = kind in (KC_INT8, KC_E4M3)
        own = {KC_F32: "f32", KC_BF16: "bf16"}.get(kind)
        dtype = own if dtype is None else dtype
        if dtype not in ("f32", "bf16") or (own is not None and dtype != own):
            raise AttnSoftmaxError(3, f"a cache of {k_pages.dtype} for values of type {dtype!r}")
        if k_pages.dim() != 4:
            raise AttnSoftmaxError(2, f"k_pages has shape {tuple(k_pages.shape)}, expected [pages, heads, page, D]")
        P, heads, page, D = k_pages.shape
        self.pages = (self._tensor(k_pages, k_pages.shape, k_pages.dtype, "k_pages"),
                      self._tensor(v_pages, k_pages.shape, k_pages.dtype, "v_pages"))
        if coded:
            self.pages += (self._tensor(k_scales, (P, heads, page), torch.float32, "k_scales"),
                           self._tensor(v_scales, (P, heads, page), torch.float32, "v_scales"))
        elif k_scales is not None or v_scales is not None:
            raise AttnSoftmaxError(1, "scales belong to caches in 8 bits")
        else:
            self.pages += (None, None)
        self.k_pages, self.v_pages, self.k_scales, self.v_scales = k_pages, v_pages, k_scales, v_scales
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.heads, self.D, self.page, self.inner = heads, D, page, (D, 1)
        self.shape = KcCache(P, page, heads, D, AS_BF16 if dtype == "bf16" else AS_F32, kind, 1, 1)
        self.described = (1, 1), ctypes.byref(self.shape)

    def _table(self, page_table):
        """The cache's description for this table, and the table's address."""
        if page_table is None or page_table.dim() != 2:
            raise AttnSoftmaxError(2 if page_table is not None else 1, "page_table is not [sequences, pages]")
        of = page_table.shape
        described, ref = self.described     # (replaced as a whole: another thread may be in a call with it)
        if of != described:
            c, (B, max_pages) = self.shape, of
            self.shape = c = KcCache(c.pages, c.page, c.heads, c.D, c.dtype, c.cache_type, B, max_pages)
            ref = ctypes.byref(c)
            self.described = of, ref
        return ref, self._tensor(page_table, of, self.torch.int32, "page_table")

    def write(self, k, v, seq, pos, page_table):
        """Rows n of k and v [N, heads, D] to token pos[n] of sequence seq[n] (int32); rows of no sequence (-1) are left out."""
        if seq is None:
            raise AttnSoftmaxError(1, "seq is None")
        i32, N = self.torch.int32, seq.shape[0]
        rows = (N, self.heads, self.D)
        k_at, ld_k = self._rows(k, rows, self.tdt, "k", self.inner)
        v_at, ld_v = self._rows(v, rows, self.tdt, "v", self.inner)
        seq, pos = self._tensor(seq, (N,), i32, "seq"), self._tensor(pos, (N,), i32, "pos")
        ref, table = self._table(page_table)
        if N:
            self._call(self.lib.kv_cache_write, ref, N, k_at, ld_k, v_at, ld_v, seq, pos, table, *self.pages)

    def read(self, seq, pos, page_table, k=None, v=None):
        """(k, v) [N, heads, D]: what the cache holds at token pos[n] of sequence seq[n] (int32), zeros where it is no place."""
        if seq is None:
            raise AttnSoftmaxError(1, "seq is None")
        torch, N = self.torch, seq.shape[0]
        rows = (N, self.heads, self.D)
        if k is None:
            k = torch.empty(rows, dtype=self.tdt, device=self.dev)
        if v is None:
            v = torch.empty(rows, dtype=self.tdt, device=self.dev)
        ref, table = self._table(page_table)
        at = (self._tensor(seq, (N,), torch.int32, "seq"), self._tensor(pos, (N,), torch.int32, "pos"), table,
              self._tensor(k, rows, self.tdt, "k"), self._tensor(v, rows, self.tdt, "v"))
        if N:
            self._call(self.lib.kv_cache_read, ref, N, *self.pages, *at)
        return k, v


class DeviceKvAttn(_DeviceOp):
    """Attention of the newest T tokens of B sequences over a DeviceKvCache: owns the workspace and forwards to the C ABI.
    max_len: no sequence is longer; window > 0: a token sees itself and the window - 1 ahead of it; scale: 1 / sqrt(D) by itself."""

    def __init__(self, cache, B, T, q_heads, max_len, window=0, scale=None):
        self._on(cache.dev)
        self.cache, self.tdt = cache, cache.tdt
        c = cache.shape
        self.shape = KcCache(c.pages, c.page, c.heads, c.D, c.dtype, c.cache_type, B, max(1, -(-max_len // c.page)))
        self.attn = KcAttn(T, q_heads, max_len, window, float(c.D ** -0.5 if scale is None else scale))
        self.attn_ref = ctypes.byref(self.attn)
        self.b, self.heads_shape, self.q_shape, self.inner = (B,), (B, T, q_heads), (B, T, q_heads, c.D), (c.D, 1)
        self.ws_bytes = kv_cache_attn_workspace_bytes(self.shape, self.attn)
        if self.ws_bytes == 0:
            raise AttnSoftmaxError(2, "invalid shape for the attention: " + attn_softmax_last_error())
        self._own_workspace()

    def fwd(self, q, page_table, lengths, out=None, lse=None):
        """out [B,T,q_heads,D] (and lse [B,T,q_heads] float32, if given); lengths [B] int32 with the new tokens, whose keys and values the
        cache holds; page_table [B, pages] int32 of pages for max_len tokens at least."""
        torch = self.torch
        if out is None:
            out = torch.empty(self.q_shape, dtype=self.tdt, device=self.dev)
        if page_table is None or page_table.dim() != 2 or page_table.shape[1] * self.shape.page < self.attn.max_len:
            raise AttnSoftmaxError(2, "page_table is not [sequences, pages for max_len tokens]")
        c, max_pages = self.shape, page_table.shape[1]
        if c.max_pages != max_pages:      # (never changed in place: another thread may be in a call with it)
            self.shape = c = KcCache(c.pages, c.page, c.heads, c.D, c.dtype, c.cache_type, c.B, max_pages)
        table = self._tensor(page_table, (c.B, max_pages), torch.int32, "page_table")
        self._call(self.lib.kv_cache_attn, ctypes.byref(c), self.attn_ref, *self._rows(q, self.q_shape, self.tdt, "q", self.inner), *self.cache.pages, table,
                   self._tensor(lengths, self.b, torch.int32, "lengths"), self._tensor(out, self.q_shape, self.tdt, "out"),
                   self._optional(lse, self.heads_shape, torch.float32, "lse"), self.workspace.data_ptr(), self.ws_bytes)
        return out
