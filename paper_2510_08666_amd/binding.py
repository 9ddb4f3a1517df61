"""ctypes binding of libdinfer.so: the same entry points as include/dinfer.h, argument marshalling only.

Every step of the path runs inside the HIP library; nothing here computes.  PyTorch is used only to own
device memory and to name the stream.  Importing this module without the built library raises.
"""
import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DINFER_LIB") or os.path.join(_HERE, "libdinfer.so")   # DINFER_LIB: another build of it

c_i32, c_u64, c_f32, c_vp, c_sz = ctypes.c_int32, ctypes.c_uint64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
c_i64 = ctypes.c_int64

F32, BF16 = 0, 1
(T_EMB, T_LM_HEAD, T_FINAL_GAIN, T_ATTN_GAIN, T_WQ, T_WK, T_WV, T_WO, T_FFN_GAIN, T_ROUTER, T_GATE, T_UP,
 T_DOWN) = range(13)
TENSOR_IDS = {"emb": T_EMB, "lm_head": T_LM_HEAD, "final_gain": T_FINAL_GAIN, "attn_gain": T_ATTN_GAIN, "wq": T_WQ,
              "wk": T_WK, "wv": T_WV, "wo": T_WO, "ffn_gain": T_FFN_GAIN, "w_router": T_ROUTER, "w_gate": T_GATE,
              "w_up": T_UP, "w_down": T_DOWN}

EXPORTS = ["dinfer_weights_bytes", "dinfer_kv_bytes", "dinfer_workspace_bytes", "dinfer_create", "dinfer_destroy",
           "dinfer_last_error", "dinfer_set_tensor", "dinfer_prefill", "dinfer_step", "dinfer_step_vicinity", "dinfer_step_credit", "dinfer_step_smooth", "dinfer_step_smooth_static", "dinfer_smooth_scratch_bytes",
           "dinfer_refresh_block", "dinfer_commit", "dinfer_generate",
           "dinfer_generate_block", "dinfer_kv_write", "dinfer_kv_read", "dinfer_debug_logits", "dinfer_debug_get",
           "dinfer_profile_every", "dinfer_profile_start", "dinfer_profile_stop", "dinfer_stream_read", "dinfer_debug_trace",
           "dinfer_debug_single_slice", "dinfer_generate_block_smooth", "dinfer_rotary_table_bytes", "dinfer_rotary_table",
           "dinfer_kv_append", "dinfer_attend", "dinfer_kv_score", "dinfer_kv_evict", "dinfer_step_scored",
           "dinfer_refresh_block_scored", "dinfer_attend_ruled", "dinfer_beam_scratch_bytes", "dinfer_beam_select",
           "dinfer_kv_fork", "dinfer_kv_compact"]
(STAGE_QKV, STAGE_ATTENTION, STAGE_OPROJ, STAGE_EXPERT_GATE_UP, STAGE_EXPERT_DOWN, STAGE_LM_HEAD,
 STAGE_ROUTER) = range(7)


class Config(ctypes.Structure):
    _fields_ = [(n, c_i32) for n in ("n_layers", "hidden", "n_heads", "head_dim", "n_experts", "top_k", "moe_inter",
                                     "vocab", "dtype", "page_size", "mask_id", "norm_topk", "max_pos")] + \
               [(n, c_f32) for n in ("rms_eps", "rope_theta", "logit_scale")]


class Decode(ctypes.Structure):
    _fields_ = [("threshold", c_f32), ("fixed_k", c_i32), ("hierarchical", c_i32), ("lower_bound", c_f32),
                ("skip_decided", c_i32)]


def _decode(threshold, fixed_k):
    """A Decode passes through; otherwise threshold decoding (or fixed-k when fixed_k > 0)."""
    if isinstance(threshold, Decode):
        return threshold
    return Decode(float(threshold), int(fixed_k), 0, 0.0, 0)


def hierarchical(threshold, lower_bound):
    """Decoder settings of hierarchical decoding."""
    return Decode(float(threshold), 0, 1, float(lower_bound), 0)


class Credit(ctypes.Structure):
    _fields_ = [("alpha", c_f32), ("beta", c_f32), ("gamma", c_f32)]


class SmoothSchedule(ctypes.Structure):
    _fields_ = [("alpha_init", c_f32), ("alpha_growth", c_f32), ("alpha_preset", c_f32), ("threshold_start", c_f32),
                ("threshold_decay", c_f32)]


class Rotary(ctypes.Structure):
    _fields_ = [(n, c_i32) for n in ("rotary_dim", "interleaved", "scaling", "original_positions")] + \
               [(n, ctypes.c_double) for n in ("theta", "factor", "beta_fast", "beta_slow", "magnitude")]


class CacheUse(ctypes.Structure):
    _fields_ = [("d_position", c_vp), ("d_score_in", c_vp), ("d_score_out", c_vp), ("score_stride", c_i32), ("decay", c_f32)]


class AttendRule(ctypes.Structure):
    _fields_ = [("block", c_i32), ("window", c_i32), ("d_prefix", c_vp), ("d_first", c_vp), ("d_end", c_vp), ("cap", c_f32),
                ("d_slope", c_vp)]


class State(ctypes.Structure):
    _fields_ = [("d_in", c_vp), ("d_out", c_vp), ("row_bytes", c_i64)]


ROTARY_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3}


def rotary(rotary_dim, interleaved=False, theta=10000.0, scaling="plain", factor=1.0, original_positions=0, beta_fast=0.0,
           beta_slow=0.0, magnitude=0.0):
    """A rotation of the first rotary_dim features of a head (see dinfer_rotary)."""
    return Rotary(int(rotary_dim), int(bool(interleaved)), ROTARY_SCALINGS[scaling], int(original_positions), float(theta),
                  float(factor), float(beta_fast), float(beta_slow), float(magnitude))


def rotary_table(rot, max_pos, device="cuda:0"):
    """Cosines and sines of positions 0 .. max_pos-1 as a [2][max_pos][rotary_dim / 2] device tensor."""
    n = lib.dinfer_rotary_table_bytes(ctypes.byref(rot), int(max_pos))
    if n == 0:
        raise DinferError(-1, last_error())
    t = torch.empty((2, int(max_pos), rot.rotary_dim // 2), dtype=torch.float32, device=device)
    with torch.cuda.device(t.device):      # (the kernel and its stream are the table's GPU's, whichever is current)
        _check(lib.dinfer_rotary_table(ctypes.byref(rot), int(max_pos), _ptr(t), n, _stream()))
    return t


CREDIT_CAP = 64


def commit(d_conf, d_argmax, d_block_tokens, d_mask, decode, d_n_committed):
    """The decoder alone on given confidences and candidate ids ([n_seq][block_len] device tensors)."""
    n_seq, block_len = d_block_tokens.shape
    _check(lib.dinfer_commit(_ptr(d_conf), _ptr(d_argmax), n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask),
                             ctypes.byref(decode), _ptr(d_n_committed), _stream()))


def beam_scratch(n_seq, n_rows, vocab, n_keep, device="cuda:0"):
    """Device scratch buffer of beam_select."""
    n = lib.dinfer_beam_scratch_bytes(int(n_seq), int(n_rows), int(vocab), int(n_keep))
    if n == 0:
        raise DinferError(-1, last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)


def beam_select(logits, score, row, token, score_out, scratch, hold=None):
    """The best candidates (row, token) of every sequence (see dinfer_beam_select): logits [n_seq][n_rows][vocab] (float32 or bfloat16, a
    sequence's rows as far apart as the others), score [n_seq][n_rows]; row, token, score_out [n_seq][n_keep] receive them."""
    if logits is None or logits.dim() != 3 or logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be a float32 or bfloat16 tensor of 3 dimensions")
    (ns, rows, vocab), (outer, stride, one) = logits.shape, logits.stride()
    index = logits.get_device()
    if index < 0 or one != 1 and vocab > 1 or ns > 1 and rows > 1 and outer != rows * stride:
        raise ValueError("logits must be rows of contiguous elements, equally far apart, on a GPU")
    if rows == 1:
        stride = outer if ns > 1 else max(vocab, 1)
    if row is None or row.dim() != 2:
        raise ValueError("row must be a tensor of 2 dimensions")
    keep = row.shape[1]
    for name, t, dtype, shape in (("score", score, torch.float32, (ns, rows)), ("row", row, torch.int32, (ns, keep)),
                                  ("token", token, torch.int32, (ns, keep)), ("score_out", score_out, torch.float32, (ns, keep)),
                                  ("hold", hold, torch.int32, (ns, rows))):
        if t is None and name == "hold":
            continue
        if t is None or t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor %s on the logits' device" % (name, dtype, list(shape)))
    if scratch is None or scratch.dtype is not torch.uint8 or scratch.get_device() != index or not scratch.is_contiguous():
        raise ValueError("scratch must be a contiguous uint8 tensor on the logits' device")
    with torch.cuda.device(index):
        _check(lib.dinfer_beam_select(_ptr(logits), BF16 if logits.dtype is torch.bfloat16 else F32, stride, ns, rows, vocab, _ptr(score),
                                      _ptr(hold), keep, _ptr(row), _ptr(token), _ptr(score_out), _ptr(scratch), scratch.numel(), _stream()))


class DinferError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("dinfer error %d: %s" % (code, msg))
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError("libdinfer.so is not built (run `python -m paper_2510_08666_amd.build`); "
                          "there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    L.dinfer_weights_bytes.restype = c_sz
    L.dinfer_weights_bytes.argtypes = [P(Config)]
    L.dinfer_kv_bytes.restype = c_sz
    L.dinfer_kv_bytes.argtypes = [P(Config), c_i32]
    L.dinfer_workspace_bytes.restype = c_sz
    L.dinfer_workspace_bytes.argtypes = [P(Config), c_i32, c_i32]
    L.dinfer_create.restype = c_i32
    L.dinfer_create.argtypes = [P(Config), c_vp, c_sz, c_vp, c_i32, c_vp, c_sz, c_i32, c_i32, c_vp, P(c_vp)]
    L.dinfer_destroy.restype = None
    L.dinfer_destroy.argtypes = [c_vp]
    L.dinfer_last_error.restype = ctypes.c_char_p
    L.dinfer_last_error.argtypes = []
    L.dinfer_set_tensor.restype = c_i32
    L.dinfer_set_tensor.argtypes = [c_vp, c_i32, c_i32, c_vp, c_sz, c_vp]
    L.dinfer_prefill.restype = c_i32
    L.dinfer_prefill.argtypes = [c_vp, c_i32, c_vp, c_vp, c_vp, c_i32, c_vp]
    L.dinfer_step.restype = c_i32
    L.dinfer_step.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), c_vp, c_vp, c_vp, c_vp]
    L.dinfer_smooth_scratch_bytes.restype = c_sz
    L.dinfer_smooth_scratch_bytes.argtypes = [P(Config), c_i32]
    L.dinfer_step_smooth.restype = c_i32
    L.dinfer_step_smooth.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), c_f32, c_vp, c_vp, c_sz,
                                     c_vp, c_vp, c_vp, c_vp]
    L.dinfer_generate_block_smooth.restype = c_i32
    L.dinfer_generate_block_smooth.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode),
                                               P(SmoothSchedule), c_vp, c_vp, c_sz, c_vp, c_vp, c_vp, c_i32, c_i32,
                                               P(c_i32), c_vp]
    L.dinfer_step_smooth_static.restype = c_i32
    L.dinfer_step_smooth_static.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), c_f32, c_vp,
                                            c_vp, c_vp, c_vp, c_vp]
    L.dinfer_step_credit.restype = c_i32
    L.dinfer_step_credit.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), P(Credit), c_vp, c_vp,
                                     c_vp, c_vp, c_vp, c_vp, c_vp]
    L.dinfer_step_vicinity.restype = c_i32
    L.dinfer_step_vicinity.argtypes = [c_vp, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), c_vp,
                                       c_vp, c_vp, c_vp]
    L.dinfer_refresh_block.restype = c_i32
    L.dinfer_refresh_block.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_i32, c_vp]
    L.dinfer_generate_block.restype = c_i32
    L.dinfer_generate_block.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), c_vp, c_vp, c_vp,
                                        c_i32, c_i32, c_i32, P(c_i32), c_vp]
    L.dinfer_rotary_table_bytes.restype = c_sz
    L.dinfer_rotary_table_bytes.argtypes = [P(Rotary), c_i32]
    L.dinfer_rotary_table.restype = c_i32
    L.dinfer_rotary_table.argtypes = [P(Rotary), c_i32, c_vp, c_sz, c_vp]
    L.dinfer_kv_append.restype = c_i32
    L.dinfer_kv_append.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_i32, c_vp, c_i64, c_vp, c_i64, c_vp, c_i64, c_i32,
                                   c_vp, c_vp, c_f32, P(Rotary), c_vp, c_i32, c_vp, c_vp, c_i64, c_vp]
    L.dinfer_attend.restype = c_i32
    L.dinfer_attend.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_i32, c_vp, c_i64, c_i32, c_vp, c_f32, c_vp, c_i64,
                                c_vp, c_vp]
    L.dinfer_kv_score.restype = c_i32
    L.dinfer_kv_score.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_i32, c_vp, c_i64, c_i32, c_vp, c_f32, c_vp, c_i32,
                                  c_f32, c_vp, c_vp, c_i32, c_vp]
    L.dinfer_kv_evict.restype = c_i32
    L.dinfer_kv_evict.argtypes = [c_vp, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_vp, c_i32, c_vp, c_vp, c_i32, c_vp, c_i32,
                                  c_vp, c_vp, c_vp, c_vp]
    L.dinfer_step_scored.restype = c_i32
    L.dinfer_step_scored.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), P(CacheUse), c_vp, c_vp,
                                     c_vp, c_vp]
    L.dinfer_refresh_block_scored.restype = c_i32
    L.dinfer_refresh_block_scored.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_i32, P(CacheUse), c_vp]
    L.dinfer_attend_ruled.restype = c_i32
    L.dinfer_attend_ruled.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_i32, c_vp, c_i64, c_i32, P(AttendRule), c_f32, c_vp,
                                      c_i64, c_vp, c_vp]
    L.dinfer_beam_scratch_bytes.restype = c_sz
    L.dinfer_beam_scratch_bytes.argtypes = [c_i32, c_i32, c_i32, c_i32]
    L.dinfer_beam_select.restype = c_i32
    L.dinfer_beam_select.argtypes = [c_vp, c_i32, c_i64, c_i32, c_i32, c_i32, c_vp, c_vp, c_i32, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    L.dinfer_kv_fork.restype = c_i32
    L.dinfer_kv_fork.argtypes = [c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, c_vp,
                                 c_vp, P(State), c_i32, c_vp]
    L.dinfer_kv_compact.restype = c_i32
    L.dinfer_kv_compact.argtypes = [c_vp, c_i32, c_vp, c_vp, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]
    L.dinfer_commit.restype = c_i32
    L.dinfer_commit.argtypes = [c_vp, c_vp, c_i32, c_i32, c_vp, c_vp, P(Decode), c_vp, c_vp]
    L.dinfer_generate.restype = c_i32
    L.dinfer_generate.argtypes = [c_vp, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_i32, P(Decode), c_i32, c_i32,
                                  c_vp, c_vp, c_vp, c_vp, P(c_i32), c_vp]
    L.dinfer_kv_write.restype = c_i32
    L.dinfer_kv_write.argtypes = [c_vp, c_i32, c_vp, c_i32, c_i32, c_vp, c_vp, c_vp]
    L.dinfer_kv_read.restype = c_i32
    L.dinfer_kv_read.argtypes = [c_vp, c_i32, c_vp, c_i32, c_i32, c_vp, c_vp, c_vp]
    L.dinfer_debug_logits.restype = c_i32
    L.dinfer_debug_logits.argtypes = [c_vp, c_i32, c_vp, c_vp]
    L.dinfer_debug_single_slice.restype = c_i32
    L.dinfer_debug_single_slice.argtypes = [c_i32]
    L.dinfer_debug_get.restype = c_i32
    L.dinfer_debug_get.argtypes = [c_vp, c_i32, c_vp, c_sz, c_vp]
    L.dinfer_profile_every.restype = c_i32
    L.dinfer_profile_every.argtypes = [c_vp, c_i32]
    L.dinfer_profile_start.restype = c_i32
    L.dinfer_profile_start.argtypes = [c_vp, c_i32]
    L.dinfer_profile_stop.restype = c_i32
    L.dinfer_profile_stop.argtypes = [c_vp, P(c_i32), P(c_f32)]
    L.dinfer_debug_trace.restype = c_i32
    L.dinfer_debug_trace.argtypes = [c_i32, c_vp, c_sz]
    L.dinfer_stream_read.restype = c_i32
    L.dinfer_stream_read.argtypes = [c_vp, c_sz, c_vp, c_vp]
    return L


lib = _load()


def last_error():
    return lib.dinfer_last_error().decode()


def _check(rc):
    if rc != 0:
        raise DinferError(rc, last_error())


def make_config(cfg, max_pos):
    """dinfer_config from an object with the model fields (n_layers, hidden, ..., dtype 'f32'|'bf16')."""
    return Config(cfg.n_layers, cfg.hidden, cfg.n_heads, cfg.head_dim, cfg.n_experts, cfg.top_k, cfg.moe_inter,
                  cfg.vocab, BF16 if cfg.dtype == "bf16" else F32, 16, cfg.mask_id, cfg.norm_topk, int(max_pos),
                  cfg.rms_eps, cfg.rope_theta, cfg.logit_scale)


def _stream():
    """Handle of the current stream (without the Stream object around it, which takes longer than a small kernel)."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def debug_single_slice(on):
    """Test switch: while on, no contraction shares a task's sum among workgroups."""
    _check(lib.dinfer_debug_single_slice(1 if on else 0))


def debug_trace(unit, n_wgs):
    """Phase timestamps [n_wgs][8] (uint64, 10 ns ticks) of a library built with DINFER_TRACE=<kernel id>."""
    import numpy as np
    out = np.zeros((n_wgs, 8), dtype=np.uint64)
    _check(lib.dinfer_debug_trace(int(unit), out.ctypes.data, out.nbytes))
    return out


def stream_read(d_buf, nbytes, d_sink):
    """One pass of the streaming-read probe over the first nbytes of a device tensor."""
    _check(lib.dinfer_stream_read(_ptr(d_buf), int(nbytes), _ptr(d_sink), _stream()))


class Context:
    """A dinfer context plus the three device buffers it lives in (allocated through torch)."""

    def __init__(self, cfg, n_pages, max_seqs, max_tokens, max_pos, device="cuda:0", weights_buffer=None):
        """weights_buffer: the `weights` tensor of another Context of the same configuration whose tensors are
        already loaded (the packed weights are position independent, so contexts may share them)."""
        self.cfg = cfg
        self.device = torch.device(device)
        self.ccfg = make_config(cfg, max_pos)
        wb = lib.dinfer_weights_bytes(self.ccfg)
        kb = lib.dinfer_kv_bytes(self.ccfg, n_pages)
        sb = lib.dinfer_workspace_bytes(self.ccfg, max_seqs, max_tokens)
        if wb == 0 or kb == 0 or sb == 0:
            raise DinferError(-1, last_error())
        self.n_pages, self.max_seqs, self.max_tokens = n_pages, max_seqs, max_tokens
        self._dtype = torch.bfloat16 if self.ccfg.dtype == BF16 else torch.float32
        self._index = self.device.index if self.device.index is not None else torch.cuda.current_device()
        if weights_buffer is not None:
            if weights_buffer.numel() < wb or weights_buffer.device != self.device:
                raise ValueError("weights_buffer does not fit this configuration")
            self.weights = weights_buffer
        else:
            self.weights = torch.empty(wb, dtype=torch.uint8, device=self.device)
        self.kv = torch.empty(kb, dtype=torch.uint8, device=self.device)
        self.ws = torch.empty(sb, dtype=torch.uint8, device=self.device)
        h = c_vp()
        _check(lib.dinfer_create(self.ccfg, _ptr(self.weights), self.weights.numel(), _ptr(self.kv), n_pages, _ptr(self.ws), sb, max_seqs,
                                 max_tokens, _stream(), ctypes.byref(h)))
        self.h = h

    def close(self):
        if self.h:
            torch.cuda.synchronize(self.device)
            lib.dinfer_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- weights
    def set_tensor(self, name, layer, array):
        """Upload one tensor given as a numpy array (float32, or uint16 bfloat16 bit patterns)."""
        a = np.ascontiguousarray(array)
        d = torch.from_numpy(a.reshape(-1).view(np.uint8)).to(self.device)
        _check(lib.dinfer_set_tensor(self.h, TENSOR_IDS[name], layer, _ptr(d), a.nbytes, _stream()))
        torch.cuda.current_stream().synchronize()     # d is released after the pack kernel has read it

    def load_weights(self, weights):
        for n in ("emb", "lm_head", "final_gain"):
            self.set_tensor(n, 0, weights[n])
        for l, lw in enumerate(weights["layers"]):
            for n, a in lw.items():
                self.set_tensor(n, l, a)

    # ---- the path
    def prefill(self, d_tokens, lens, d_page_table):
        h_lens = (c_i32 * len(lens))(*[int(x) for x in lens])
        _check(lib.dinfer_prefill(self.h, len(lens), _ptr(d_tokens), ctypes.cast(h_lens, c_vp), _ptr(d_page_table),
                                  d_page_table.shape[1], _stream()))

    def step(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, d_conf, d_argmax,
             d_n_committed):
        n_seq, block_len = d_block_tokens.shape
        dec = _decode(threshold, fixed_k)
        _check(lib.dinfer_step(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask), _ptr(d_prefix_len),
                               _ptr(d_page_table), d_page_table.shape[1], ctypes.byref(dec), _ptr(d_conf),
                               _ptr(d_argmax), _ptr(d_n_committed), _stream()))

    def smooth_scratch(self, max_tokens):
        """Device scratch buffer for step_smooth with up to max_tokens block tokens."""
        n = lib.dinfer_smooth_scratch_bytes(ctypes.byref(self.ccfg), int(max_tokens))
        if n == 0:
            raise DinferError(-1, "dinfer_smooth_scratch_bytes: unsupported size")
        return torch.empty(n, dtype=torch.uint8, device=self.device)

    def step_smooth(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, alpha, d_delta,
                    d_scratch, d_conf, d_argmax, d_n_committed):
        n_seq, block_len = d_block_tokens.shape
        dec = _decode(threshold, fixed_k)
        _check(lib.dinfer_step_smooth(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask), _ptr(d_prefix_len),
                                      _ptr(d_page_table), d_page_table.shape[1], ctypes.byref(dec), float(alpha),
                                      _ptr(d_delta), _ptr(d_scratch), d_scratch.numel(), _ptr(d_conf), _ptr(d_argmax),
                                      _ptr(d_n_committed), _stream()))

    def step_smooth_static(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, alpha, d_delta,
                           d_conf, d_argmax, d_n_committed):
        """step_smooth with the library's own static scratch: the call allocates nothing."""
        n_seq, block_len = d_block_tokens.shape
        dec = _decode(threshold, fixed_k)
        _check(lib.dinfer_step_smooth_static(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask),
                                             _ptr(d_prefix_len), _ptr(d_page_table), d_page_table.shape[1],
                                             ctypes.byref(dec), float(alpha), _ptr(d_delta), _ptr(d_conf),
                                             _ptr(d_argmax), _ptr(d_n_committed), _stream()))

    def step_credit(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, alpha, beta, gamma,
                    d_credit_ids, d_credit_val, d_credit_n, d_conf, d_argmax, d_n_committed):
        n_seq, block_len = d_block_tokens.shape
        dec = _decode(threshold, fixed_k)
        cr = Credit(float(alpha), float(beta), float(gamma))
        _check(lib.dinfer_step_credit(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask), _ptr(d_prefix_len),
                                      _ptr(d_page_table), d_page_table.shape[1], ctypes.byref(dec), ctypes.byref(cr),
                                      _ptr(d_credit_ids), _ptr(d_credit_val), _ptr(d_credit_n), _ptr(d_conf),
                                      _ptr(d_argmax), _ptr(d_n_committed), _stream()))

    def step_vicinity(self, d_block_tokens, d_vicinity_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k,
                      d_conf, d_argmax, d_n_committed):
        n_seq, block_len = d_block_tokens.shape
        look_back = d_vicinity_tokens.shape[1]
        dec = _decode(threshold, fixed_k)
        _check(lib.dinfer_step_vicinity(self.h, n_seq, block_len, look_back, _ptr(d_block_tokens),
                                        _ptr(d_vicinity_tokens), _ptr(d_mask), _ptr(d_prefix_len), _ptr(d_page_table),
                                        d_page_table.shape[1], ctypes.byref(dec), _ptr(d_conf), _ptr(d_argmax),
                                        _ptr(d_n_committed), _stream()))

    def refresh_block(self, d_block_tokens, d_prefix_len, d_page_table):
        n_seq, block_len = d_block_tokens.shape
        _check(lib.dinfer_refresh_block(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_prefix_len),
                                        _ptr(d_page_table), d_page_table.shape[1], _stream()))

    def generate_block(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, d_conf, d_argmax,
                       d_n_committed, max_steps, masked_hint=0, steps_per_wait=1):
        """The inner loop over the steps of a block; returns the number of steps that ran.  steps_per_wait: steps
        enqueued between two host waits when the step count depends on the data."""
        n_seq, block_len = d_block_tokens.shape
        dec = _decode(threshold, fixed_k)
        steps = c_i32(0)
        _check(lib.dinfer_generate_block(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask),
                                         _ptr(d_prefix_len), _ptr(d_page_table), d_page_table.shape[1],
                                         ctypes.byref(dec), _ptr(d_conf), _ptr(d_argmax), _ptr(d_n_committed),
                                         int(max_steps), int(masked_hint), int(steps_per_wait), ctypes.byref(steps),
                                         _stream()))
        return steps.value

    def generate_block_smooth(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, schedule, d_delta,
                              d_scratch, d_conf, d_argmax, d_n_committed, max_steps, steps_per_wait=1):
        """A block denoised with iteration smoothing; schedule = (alpha_init, alpha_growth, alpha_preset,
        threshold_start, threshold_decay).  Returns the number of steps that ran."""
        n_seq, block_len = d_block_tokens.shape
        dec = _decode(threshold, 0)
        sch = SmoothSchedule(*[float(v) for v in schedule])
        steps = c_i32(0)
        _check(lib.dinfer_generate_block_smooth(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask),
                                                _ptr(d_prefix_len), _ptr(d_page_table), d_page_table.shape[1],
                                                ctypes.byref(dec), ctypes.byref(sch), _ptr(d_delta), _ptr(d_scratch),
                                                d_scratch.numel(), _ptr(d_conf), _ptr(d_argmax), _ptr(d_n_committed),
                                                int(max_steps), int(steps_per_wait), ctypes.byref(steps), _stream()))
        return steps.value

    def generate(self, d_out, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, eos_id,
                 d_finished, d_conf, d_argmax, d_n_committed, steps_per_wait=1):
        """Outer loop over the blocks of d_out [n_seq][n_blocks * block_len]; returns the blocks that were run."""
        n_seq, block_len = d_block_tokens.shape
        n_blocks = d_out.shape[1] // block_len
        assert d_out.shape[1] == n_blocks * block_len and d_out.is_contiguous()
        dec = _decode(threshold, fixed_k)
        run = c_i32(0)
        _check(lib.dinfer_generate(self.h, n_seq, block_len, n_blocks, _ptr(d_out), _ptr(d_block_tokens), _ptr(d_mask),
                                   _ptr(d_prefix_len), _ptr(d_page_table), d_page_table.shape[1], ctypes.byref(dec),
                                   int(eos_id), int(steps_per_wait), _ptr(d_finished), _ptr(d_conf), _ptr(d_argmax),
                                   _ptr(d_n_committed), ctypes.byref(run), _stream()))
        return run.value

    # ---- operators on the paged cache (shapes: T = sum(lens) rows; see include/dinfer.h)
    def _raw_stream(self):
        return torch._C._cuda_getCurrentRawStream(self._index)

    def _rows(self, name, t, rows, heads):
        """Address and stride of a matrix of at least `rows` rows of heads * head_dim contiguous elements."""
        width = heads * self.cfg.head_dim
        if t is not None and t.dtype is self._dtype and t.dim() == 2 and t.get_device() == self._index:
            (n, m), (stride, one) = t.shape, t.stride()
            if n >= rows and m == width and one == 1:
                return t.data_ptr(), stride
        raise ValueError("%s must be a [%d][%d] tensor of the context's dtype and device, rows contiguous" % (name, rows, width))

    @staticmethod
    def _sizes(name, t, dims):
        """Sizes of a tensor that has `dims` of them."""
        if t is None or t.dim() != dims:
            raise ValueError("%s must be a tensor of %d dimensions" % (name, dims))
        return t.shape

    def _flat(self, name, t, dtype, *shape):
        """Address of a contiguous tensor of that type and these sizes (the first may be larger); None passes."""
        if t is None:
            return None
        if t.dtype is dtype and t.get_device() == self._index and t.is_contiguous():
            n = t.shape
            if n == shape or (len(n) == len(shape) and n[0] >= shape[0] and n[1:] == shape[1:]):
                return t.data_ptr()
        raise ValueError("%s must be a contiguous %s tensor %s on the context's device" % (name, dtype, list(shape)))

    def _tokens(self, lens, d_past, d_page_table):
        """The arguments that say which tokens join which sequences, and how many there are."""
        n, columns = len(lens), self._sizes("d_page_table", d_page_table, 2)[1]
        return ((n, (c_i32 * n)(*lens), self._flat("d_past", d_past, torch.int32, n),
                 self._flat("d_page_table", d_page_table, torch.int32, n, columns), columns), sum(lens))

    def _words(self, visible, T):
        if visible is not None and visible.dtype is torch.uint64:
            visible = visible.view(torch.int64)
        return self._flat("visible", visible, torch.int64, T)

    def kv_append(self, layer, lens, d_past, d_page_table, d_q, d_k, d_v, d_q_out, q_gain=None, k_gain=None, eps=1e-6,
                  rotary=None, rotary_table=None, positions=None):
        """Norms, rotates and stores a layer's new tokens; d_q_out receives the queries (d_q and d_q_out None: keys and values only)."""
        tok, T = self._tokens(lens, d_past, d_page_table)
        nh, hd = self.cfg.n_heads, self.cfg.head_dim
        nq = nh if d_q is None else self._sizes("d_q", d_q, 2)[1] // hd
        q, out = ((None, 0), (None, 0)) if d_q is None else (self._rows("d_q", d_q, T, nq), self._rows("d_q_out", d_q_out, T, nq))
        table_positions = 0
        if rotary is not None and rotary_table is not None:
            table_positions = self._sizes("rotary_table", rotary_table, 3)[1]
            self._flat("rotary_table", rotary_table, torch.float32, 2, table_positions, rotary.rotary_dim // 2)
        _check(lib.dinfer_kv_append(self.h, layer, *tok, *q, *self._rows("d_k", d_k, T, nh), *self._rows("d_v", d_v, T, nh), nq,
                                    self._flat("q_gain", q_gain, torch.float32, hd), self._flat("k_gain", k_gain, torch.float32, hd), eps,
                                    rotary, _ptr(rotary_table), table_positions, self._flat("positions", positions, torch.int32, T),
                                    *out, self._raw_stream()))

    def attend(self, layer, lens, d_past, d_page_table, d_q, d_out, visible=None, scale=0.0, lse=None):
        """Attention of the new tokens over the cache, their own keys as far as the words of `visible` [T] allow."""
        tok, T = self._tokens(lens, d_past, d_page_table)
        nq = self._sizes("d_q", d_q, 2)[1] // self.cfg.head_dim
        _check(lib.dinfer_attend(self.h, layer, *tok, *self._rows("d_q", d_q, T, nq), nq, self._words(visible, T), scale,
                                 *self._rows("d_out", d_out, T, nq), self._flat("lse", lse, torch.float32, T, nq), self._raw_stream()))

    def kv_score(self, layer, lens, d_past, d_page_table, d_q, d_score_out, score_in=None, decay=1.0, visible=None, scale=0.0,
                 lse=None):
        """Adds the attention weight of the new tokens to d_score_out [n_seq][n_heads][stride]; lse: what `attend` left for
        the same queries (None: worked out here)."""
        tok, T = self._tokens(lens, d_past, d_page_table)
        nq = self._sizes("d_q", d_q, 2)[1] // self.cfg.head_dim
        shape = (len(lens), self.cfg.n_heads, self._sizes("d_score_out", d_score_out, 3)[2])
        q = self._rows("d_q", d_q, T, nq)
        given = lse is not None
        if not given:
            lse = torch.empty((max(T, 1), nq), dtype=torch.float32, device=d_q.device)
        _check(lib.dinfer_kv_score(self.h, layer, *tok, *q, nq, self._words(visible, T), scale, self._flat("lse", lse, torch.float32, T, nq),
                                   given, decay, self._flat("score_in", score_in, torch.float32, *shape),
                                   self._flat("d_score_out", d_score_out, torch.float32, *shape), shape[2], self._raw_stream()))

    def kv_evict(self, first_layer, n_layers, keep, n_sink, n_recent, d_score, d_len, d_page_table, d_new_page_table, d_kept,
                 d_new_len, score_out=None):
        """Keeps `keep` positions per (layer, sequence, head) of d_score [n_layers][n_seq][n_heads][stride] in new pages."""
        (ns, columns), (_, new_columns) = self._sizes("d_page_table", d_page_table, 2), self._sizes("d_new_page_table", d_new_page_table, 2)
        nh, width, i32 = self.cfg.n_heads, self._sizes("d_score", d_score, 4)[3], torch.int32
        _check(lib.dinfer_kv_evict(self.h, first_layer, n_layers, ns, keep, n_sink, n_recent,
                                   self._flat("d_score", d_score, torch.float32, n_layers, ns, nh, width), width,
                                   self._flat("d_len", d_len, i32, ns), self._flat("d_page_table", d_page_table, i32, ns, columns), columns,
                                   self._flat("d_new_page_table", d_new_page_table, i32, ns, new_columns), new_columns,
                                   self._flat("d_kept", d_kept, i32, n_layers, ns, nh, keep),
                                   self._flat("score_out", score_out, torch.float32, n_layers, ns, nh, width),
                                   self._flat("d_new_len", d_new_len, i32, ns), self._raw_stream()))

    def attend_ruled(self, layer, lens, d_past, d_page_table, d_q, d_out, block=0, window=0, prefix=None, first=None, end=None, cap=0.0,
                     slope=None, scale=0.0, lse=None):
        """Attention of any number of new tokens over the cache under a rule (see dinfer_attend_rule): causal by blocks, window, prefix
        [n_seq], documents first, end [T], capped scores, slopes [query heads]."""
        tok, T = self._tokens(lens, d_past, d_page_table)
        nq, i32 = self._sizes("d_q", d_q, 2)[1] // self.cfg.head_dim, torch.int32
        rule = AttendRule(block, window, self._flat("prefix", prefix, i32, len(lens)), self._flat("first", first, i32, T),
                          self._flat("end", end, i32, T), cap, self._flat("slope", slope, torch.float32, nq))
        _check(lib.dinfer_attend_ruled(self.h, layer, *tok, *self._rows("d_q", d_q, T, nq), nq, rule, scale, *self._rows("d_out", d_out, T, nq),
                                       self._flat("lse", lse, torch.float32, T, nq), self._raw_stream()))

    def kv_fork(self, parent, d_len, d_held, d_page_table, refs, d_new_len, d_new_held, d_new_page_table, new_refs, short, room=0, rewrite=0,
                states=()):
        """The next sequences out of the present ones (see dinfer_kv_fork): parent [n_new]; d_len, d_held [n_old] and d_page_table
        [n_old][columns] (all None: no old ones); refs, new_refs [n_pages]; short [1]; states: pairs of tensors, a row per old and per
        new sequence."""
        i32 = torch.int32
        n_new, new_columns = self._sizes("d_new_page_table", d_new_page_table, 2)
        n_old, columns = (0, 0) if d_page_table is None else self._sizes("d_page_table", d_page_table, 2)
        rows = (State * len(states))() if states else None
        for k, (a, b) in enumerate(states):
            sa, sb = a.shape, b.shape
            if not (len(sa) > 0 and sa[1:] == sb[1:] and sa[0] >= n_old and sb[0] >= n_new and a.dtype is b.dtype and a.get_device() == self._index and
                    b.get_device() == self._index and a.is_contiguous() and b.is_contiguous()):
                raise ValueError("state %d must be two contiguous tensors on the context's device, a row of one type and size for each of %d old "
                                 "and %d new sequences" % (k, n_old, n_new))
            r = rows[k]
            r.d_in, r.d_out, r.row_bytes = a.data_ptr(), b.data_ptr(), b.numel() // sb[0] * b.element_size()
        _check(lib.dinfer_kv_fork(self.h, n_old, n_new, self._flat("parent", parent, i32, n_new), self._flat("d_len", d_len, i32, n_old),
                                  self._flat("d_held", d_held, i32, n_old), self._flat("d_page_table", d_page_table, i32, n_old, columns), columns,
                                  room, rewrite, self._flat("refs", refs, i32, self.n_pages), self._flat("d_new_len", d_new_len, i32, n_new),
                                  self._flat("d_new_held", d_new_held, i32, n_new),
                                  self._flat("d_new_page_table", d_new_page_table, i32, n_new, new_columns), new_columns,
                                  self._flat("new_refs", new_refs, i32, self.n_pages), self._flat("short", short, i32, 1), rows, len(states),
                                  self._raw_stream()))

    def kv_compact(self, d_held, d_page_table, refs, d_new_page_table, new_refs, moved, count):
        """Moves the pages in use to the front of the pool (see dinfer_kv_compact): moved [2][n_pages], count [2]."""
        i32, (ns, columns) = torch.int32, self._sizes("d_page_table", d_page_table, 2)
        _check(lib.dinfer_kv_compact(self.h, ns, self._flat("d_held", d_held, i32, ns), self._flat("d_page_table", d_page_table, i32, ns, columns),
                                     columns, self._flat("refs", refs, i32, self.n_pages),
                                     self._flat("d_new_page_table", d_new_page_table, i32, ns, columns),
                                     self._flat("new_refs", new_refs, i32, self.n_pages), self._flat("moved", moved, i32, 2, self.n_pages),
                                     self._flat("count", count, i32, 2), self._raw_stream()))

    def _cache_use(self, n_seq, position, score_in, score_out, decay):
        shape = (self.cfg.n_layers, n_seq, self.cfg.n_heads, 0 if score_out is None else self._sizes("score_out", score_out, 4)[3])
        return CacheUse(self._flat("position", position, torch.int32, n_seq), self._flat("score_in", score_in, torch.float32, *shape),
                        self._flat("score_out", score_out, torch.float32, *shape), shape[3], decay)

    def step_scored(self, d_block_tokens, d_mask, d_prefix_len, d_page_table, threshold, fixed_k, d_conf, d_argmax,
                    d_n_committed, position=None, score_in=None, score_out=None, decay=1.0):
        """step over a cache that may have been shortened; score_out [n_layers][n_seq][n_heads][stride] receives its scores."""
        n_seq, block_len = d_block_tokens.shape
        dec, use = _decode(threshold, fixed_k), self._cache_use(n_seq, position, score_in, score_out, decay)
        _check(lib.dinfer_step_scored(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_mask), _ptr(d_prefix_len),
                                      _ptr(d_page_table), d_page_table.shape[1], ctypes.byref(dec), ctypes.byref(use),
                                      _ptr(d_conf), _ptr(d_argmax), _ptr(d_n_committed), _stream()))

    def refresh_block_scored(self, d_block_tokens, d_prefix_len, d_page_table, position=None, score_in=None, score_out=None,
                             decay=1.0):
        n_seq, block_len = d_block_tokens.shape
        use = self._cache_use(n_seq, position, score_in, score_out, decay)
        _check(lib.dinfer_refresh_block_scored(self.h, n_seq, block_len, _ptr(d_block_tokens), _ptr(d_prefix_len),
                                               _ptr(d_page_table), d_page_table.shape[1], ctypes.byref(use), _stream()))

    # ---- KV rows in and out, test hooks
    def kv_write(self, layer, d_page_row, first_pos, d_k, d_v):
        _check(lib.dinfer_kv_write(self.h, layer, _ptr(d_page_row), first_pos, d_k.shape[0], _ptr(d_k), _ptr(d_v),
                                   _stream()))

    def kv_read(self, layer, d_page_row, first_pos, n_pos):
        D = self.cfg.n_heads * self.cfg.head_dim
        k = torch.empty((n_pos, D), dtype=torch.float32, device=self.device)
        v = torch.empty((n_pos, D), dtype=torch.float32, device=self.device)
        _check(lib.dinfer_kv_read(self.h, layer, _ptr(d_page_row), first_pos, n_pos, _ptr(k), _ptr(v), _stream()))
        return k, v

    def debug_logits(self, n_rows):
        out = torch.empty((n_rows, self.cfg.vocab), dtype=torch.float32, device=self.device)
        _check(lib.dinfer_debug_logits(self.h, n_rows, _ptr(out), _stream()))
        return out

    def profile_every(self, n_forwards):
        _check(lib.dinfer_profile_every(self.h, n_forwards))

    def profile_start(self, stage):
        _check(lib.dinfer_profile_start(self.h, stage))

    def profile_stop(self):
        """(launches recorded, summed milliseconds) of the profiled stage."""
        n, ms = c_i32(0), c_f32(0.0)
        _check(lib.dinfer_profile_stop(self.h, ctypes.byref(n), ctypes.byref(ms)))
        return n.value, ms.value

    def debug_get(self, what, shape, dtype):
        out = torch.empty(shape, dtype=dtype, device=self.device)
        _check(lib.dinfer_debug_get(self.h, what, _ptr(out), out.numel() * out.element_size(), _stream()))
        return out
