"""Python binding of the C ABI in include/rl_decode.h (argument marshalling only).

PyTorch supplies device memory (weights, KV pool, workspace, token and output
buffers) and the stream; every step of the decoder runs in the library's HIP
kernels.  There is no fallback: if librl_decode.so is missing or a call
fails, an exception is raised.
"""
import ctypes as C
import functools
import os
from typing import Dict, Optional, Sequence

import numpy as np
import torch

from .configs import ModelShape

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "librl_decode.so")

RL_OK, RL_ERR_INVALID_ARG, RL_ERR_UNSUPPORTED, RL_ERR_CAPACITY, RL_ERR_HIP, RL_ERR_STATE = range(6)
RL_DTYPE_FP32, RL_DTYPE_BF16 = 0, 1
RL_OPT_ATTN_CHUNK, RL_OPT_PROFILE, RL_OPT_GEMM_PLAN, RL_OPT_SHARED_PREFIX, RL_OPT_PREFILL_ATTENTION = 1, 2, 3, 4, 5
(RL_GEMM_DIRECT, RL_GEMM_GEMV, RL_GEMM_T256, RL_GEMM_T128X256, RL_GEMM_T128, RL_GEMM_T128_DEEP,
 RL_GEMM_GEMV_WIDE, RL_GEMM_T256_CUT) = 1, 2, 3, 4, 5, 6, 7, 9


def gemm_plan_code(kernel: int, splits: int = 0, second: int = 0) -> int:
    """Value of RL_OPT_GEMM_PLAN: tile kernel, split-K count, second-half kernel."""
    return int(kernel) | (int(splits) << 8) | (int(second) << 16)
KERNEL_CLASSES = ("embed", "rmsnorm", "gemm_qkv", "rope_append", "attention", "attn_combine",
                  "gemm_o", "gemm_gate_up", "gemm_down", "gemm_lm_head", "splitk_reduce", "sample",
                  "moe_route", "moe_experts")

EXPORTS = ("rl_decode_kv_bytes", "rl_decode_workspace_bytes", "rl_decode_create", "rl_decode_destroy",
           "rl_prefill", "rl_score", "rl_decode_step", "rl_sample_logits", "rl_release_slots",
           "rl_set_slot_lengths", "rl_slot_length", "rl_kv_free_pages", "rl_kv_offload_bytes", "rl_kv_offload", "rl_kv_onload",
           "rl_decode_rebind", "rl_decode_set_option", "rl_decode_kernel_stats",
           "rl_decode_reset_stats", "rl_decode_attn_plan_stats", "rl_probe_copy", "rl_probe_read", "rl_probe_mfma",
           "rl_probe_gumbel_bound",
           "rl_sample_logits_noalloc", "rl_logprob_workspace_bytes", "rl_token_logprobs",
           "rl_token_logprobs_backward", "rl_policy_workspace_bytes", "rl_policy_logits_workspace_bytes",
           "rl_policy_loss", "rl_policy_loss_logits", "rl_preference_workspace_bytes", "rl_preference_loss",
           "rl_rmsnorm_quant", "rl_quantise", "rl_gemm_quant_workspace_bytes", "rl_gemm_quant", "rl_kv_quant_bytes",
           "rl_kv_quant_append", "rl_kv_quant_read", "rl_attention_quant_workspace_bytes", "rl_attention_quant",
           "rl_decode_tune_gemms", "rl_decode_gemm_plan", "rl_status_string",
           "rl_decode_last_error")


class ModelConfig(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32),
                ("vocab", C.c_int32), ("dtype", C.c_int32), ("rms_eps", C.c_double),
                ("rope_theta", C.c_double), ("max_seqs", C.c_int32), ("max_ctx", C.c_int32),
                ("max_prefill_tokens", C.c_int32), ("kv_page_size", C.c_int32), ("kv_pages", C.c_int32),
                ("n_experts", C.c_int32), ("top_k", C.c_int32), ("expert_ffn", C.c_int32),
                ("reserved", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("embed", "attn_norm", "w_qkv", "w_o", "mlp_norm",
                                          "w_gate_up", "w_down", "final_norm", "lm_head",
                                          "w_router", "w_exp_gate_up", "w_exp_down")]


def _weights_struct(weights: Dict[str, torch.Tensor]) -> "Weights":
    """Device pointers of the weight tensors (absent ones NULL: the dense MLP
    of a mixture of experts, the experts of a dense model)."""
    w = Weights()
    for name, _ in Weights._fields_:
        setattr(w, name, weights[name].data_ptr() if name in weights else None)
    return w


class SampleParams(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("temperature", C.c_float), ("reserved", C.c_int32)]


class KernelStats(C.Structure):
    _fields_ = [("launches", C.c_int64), ("total_ms", C.c_double), ("alg_bytes", C.c_double),
                ("alg_flops", C.c_double), ("name", C.c_char * 48)]


class AttnPlanStats(C.Structure):
    _fields_ = [("steps", C.c_int64), ("items", C.c_int64), ("shared_items", C.c_int64),
                ("pair_items", C.c_int64), ("lds_workgroups", C.c_int64)]


class PolicyParams(C.Structure):
    _fields_ = [("clip_low", C.c_double), ("clip_high", C.c_double), ("dual_clip", C.c_double),
                ("kl_coef", C.c_double), ("entropy_coef", C.c_double), ("scale", C.c_double), ("kl", C.c_int32),
                ("aggregate", C.c_int32), ("token_advantages", C.c_int32), ("reserved", C.c_int32)]


class PolicyBatch(C.Structure):
    _fields_ = [("n", C.c_int32), ("n_seqs", C.c_int32), ("seq_offsets", C.c_void_p), ("old_logp", C.c_void_p),
                ("ref_logp", C.c_void_p), ("advantages", C.c_void_p), ("mask", C.c_void_p)]


class PreferenceParams(C.Structure):
    _fields_ = [("beta", C.c_double), ("label_smoothing", C.c_double), ("margin", C.c_double), ("scale", C.c_double),
                ("form", C.c_int32), ("average", C.c_int32)]


class Fp8Matrix(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("ld", C.c_int64), ("scales", C.c_void_p), ("ld_scales", C.c_int64)]


class KvFp8(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("page_table", C.c_void_p), ("n_seqs", C.c_int32), ("max_pages", C.c_int32),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


FP8_FORMS = {"rows": 0, "swiglu": 1, "tiles": 2}
KL_KINDS = {"k1": 1, "k2": 2, "k3": 3}
AGGREGATES = {"token_mean": 0, "sequence_mean": 1, "sum": 2}
PREFERENCE_FORMS = {"sigmoid": 0, "hinge": 1, "squared": 2}

_lib = None


def lib():
    """Load librl_decode.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2509_15965_amd.build`")
    L = C.CDLL(LIB_PATH)
    vp, i32, u64, sz = C.c_void_p, C.c_int32, C.c_uint64, C.c_size_t
    cfgp = C.POINTER(ModelConfig)
    L.rl_decode_kv_bytes.restype = sz
    L.rl_decode_kv_bytes.argtypes = [cfgp]
    L.rl_decode_workspace_bytes.restype = sz
    L.rl_decode_workspace_bytes.argtypes = [cfgp]
    L.rl_decode_create.restype = C.c_int
    L.rl_decode_create.argtypes = [cfgp, C.POINTER(Weights), vp, sz, vp, sz, vp, C.POINTER(vp)]
    L.rl_decode_destroy.restype = C.c_int
    L.rl_decode_destroy.argtypes = [vp]
    L.rl_prefill.restype = C.c_int
    L.rl_prefill.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, C.POINTER(SampleParams), vp, vp, vp]
    L.rl_score.restype = C.c_int
    L.rl_score.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, vp, vp, C.c_float, vp]
    L.rl_decode_step.restype = C.c_int
    L.rl_decode_step.argtypes = [vp, i32, vp, vp, vp, vp, C.POINTER(SampleParams), vp, vp, vp]
    L.rl_sample_logits.restype = C.c_int
    L.rl_sample_logits.argtypes = [vp, i32, vp, vp, vp, vp, C.POINTER(SampleParams), vp, vp]
    L.rl_release_slots.restype = C.c_int
    L.rl_release_slots.argtypes = [vp, i32, vp]
    L.rl_set_slot_lengths.restype = C.c_int
    L.rl_set_slot_lengths.argtypes = [vp, i32, vp, vp]
    L.rl_slot_length.restype = i32
    L.rl_slot_length.argtypes = [vp, i32]
    L.rl_kv_free_pages.restype = C.c_int64
    L.rl_kv_free_pages.argtypes = [vp]
    L.rl_kv_offload_bytes.restype = sz
    L.rl_kv_offload_bytes.argtypes = [vp, i32, vp]
    L.rl_kv_offload.restype = C.c_int
    L.rl_kv_offload.argtypes = [vp, i32, vp, vp, sz]
    L.rl_kv_onload.restype = C.c_int
    L.rl_kv_onload.argtypes = [vp, i32, vp, vp, vp, sz]
    L.rl_decode_rebind.restype = C.c_int
    L.rl_decode_rebind.argtypes = [vp, C.POINTER(Weights), vp, sz, vp, sz]
    L.rl_decode_set_option.restype = C.c_int
    L.rl_decode_set_option.argtypes = [vp, i32, C.c_int64]
    L.rl_decode_tune_gemms.restype = C.c_int
    L.rl_decode_tune_gemms.argtypes = [vp, i32, vp]
    L.rl_decode_gemm_plan.restype = C.c_int
    L.rl_decode_gemm_plan.argtypes = [vp, i32, i32, C.POINTER(C.c_int64), C.POINTER(C.c_float)]
    L.rl_decode_kernel_stats.restype = C.c_int
    L.rl_decode_kernel_stats.argtypes = [vp, i32, C.POINTER(KernelStats)]
    L.rl_decode_reset_stats.restype = C.c_int
    L.rl_decode_reset_stats.argtypes = [vp]
    L.rl_decode_attn_plan_stats.restype = C.c_int
    L.rl_decode_attn_plan_stats.argtypes = [vp, C.POINTER(AttnPlanStats)]
    L.rl_probe_copy.restype = C.c_int
    L.rl_probe_copy.argtypes = [vp, vp, sz, vp]
    L.rl_probe_read.restype = C.c_int
    L.rl_probe_read.argtypes = [vp, sz, i32, vp, vp]
    L.rl_probe_mfma.restype = C.c_int
    L.rl_probe_mfma.argtypes = [i32, i32, vp, vp]
    L.rl_sample_logits_noalloc.restype = C.c_int
    L.rl_sample_logits_noalloc.argtypes = [i32, i32, vp, i32, vp, vp, vp, C.POINTER(SampleParams), vp, vp, vp]
    L.rl_probe_gumbel_bound.restype = C.c_int
    L.rl_probe_gumbel_bound.argtypes = [C.c_uint32, C.c_uint64, i32, vp, vp, vp]
    i64 = C.c_int64
    L.rl_logprob_workspace_bytes.restype = sz
    L.rl_logprob_workspace_bytes.argtypes = [i32, i32]
    L.rl_token_logprobs.restype = C.c_int
    L.rl_token_logprobs.argtypes = [i32, i32, i32, vp, i64, vp, C.c_double, vp, vp, vp, vp, sz, vp]
    L.rl_token_logprobs_backward.restype = C.c_int
    L.rl_token_logprobs_backward.argtypes = [i32, i32, i32, vp, i64, vp, C.c_double, vp, vp, vp, vp, vp, i64, vp]
    L.rl_policy_workspace_bytes.restype = sz
    L.rl_policy_workspace_bytes.argtypes = [i32, i32]
    L.rl_policy_logits_workspace_bytes.restype = sz
    L.rl_policy_logits_workspace_bytes.argtypes = [i32, i32, i32]
    L.rl_policy_loss.restype = C.c_int
    L.rl_policy_loss.argtypes = [C.POINTER(PolicyBatch), C.POINTER(PolicyParams), vp, vp, vp, vp, vp, vp, sz, vp]
    L.rl_policy_loss_logits.restype = C.c_int
    L.rl_policy_loss_logits.argtypes = [C.POINTER(PolicyBatch), C.POINTER(PolicyParams), i32, i32, vp, i64, vp, C.c_double,
                                        vp, vp, vp, vp, i64, vp, sz, vp]
    L.rl_preference_workspace_bytes.restype = sz
    L.rl_preference_workspace_bytes.argtypes = [i32, i32]
    L.rl_preference_loss.restype = C.c_int
    L.rl_preference_loss.argtypes = [i32, i32, vp, vp, vp, vp, C.POINTER(PreferenceParams), vp, vp, vp, vp, sz, vp]
    mp, kp, f64 = C.POINTER(Fp8Matrix), C.POINTER(KvFp8), C.c_double
    L.rl_rmsnorm_quant.restype = C.c_int
    L.rl_rmsnorm_quant.argtypes = [i32, i32, i32, vp, i64, i32, vp, i64, i32, vp, f64, vp, i64, mp, vp]
    L.rl_quantise.restype = C.c_int
    L.rl_quantise.argtypes = [i32, i32, i32, i32, vp, i64, mp, vp]
    L.rl_gemm_quant_workspace_bytes.restype = sz
    L.rl_gemm_quant_workspace_bytes.argtypes = [i32, i32, i32]
    L.rl_gemm_quant.restype = C.c_int
    L.rl_gemm_quant.argtypes = [i32, i32, i32, mp, mp, i32, vp, i64, vp, sz, vp]
    L.rl_kv_quant_bytes.restype = sz
    L.rl_kv_quant_bytes.argtypes = [i32, i32, i32, i32]
    for f in (L.rl_kv_quant_append, L.rl_kv_quant_read):
        f.restype = C.c_int
        f.argtypes = [kp, i32, vp, vp, i32, vp, i64, vp, i64, vp]
    L.rl_attention_quant_workspace_bytes.restype = sz
    L.rl_attention_quant_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    L.rl_attention_quant.restype = C.c_int
    L.rl_attention_quant.argtypes = [kp, i32, vp, vp, i32, i32, vp, i64, i32, f64, vp, i64, vp, sz, vp]
    L.rl_status_string.restype = C.c_char_p
    L.rl_status_string.argtypes = [C.c_int]
    L.rl_decode_last_error.restype = C.c_char_p
    L.rl_decode_last_error.argtypes = [vp]
    _lib = L
    return L


class RLError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{lib().rl_status_string(status).decode()} ({status}): {msg}")
        self.status = status


def make_config(shape: ModelShape, max_seqs: int, max_ctx: int, max_prefill_tokens: int,
                kv_page_size: int = 0, kv_pages: int = 0) -> ModelConfig:
    c = ModelConfig()
    c.n_layers, c.hidden, c.n_q_heads = shape.n_layers, shape.hidden, shape.n_q_heads
    c.n_kv_heads, c.head_dim, c.ffn, c.vocab = shape.n_kv_heads, shape.head_dim, shape.ffn, shape.vocab
    c.dtype = RL_DTYPE_BF16 if shape.dtype == "bf16" else RL_DTYPE_FP32
    c.rms_eps, c.rope_theta = float(shape.rms_eps), float(shape.rope_theta)
    c.max_seqs, c.max_ctx, c.max_prefill_tokens = max_seqs, max_ctx, max_prefill_tokens
    c.kv_page_size, c.kv_pages, c.reserved = kv_page_size, kv_pages, 0
    c.n_experts, c.top_k, c.expert_ffn = shape.n_experts, shape.top_k, shape.expert_ffn
    return c


def kv_bytes(cfg: ModelConfig) -> int:
    return int(lib().rl_decode_kv_bytes(C.byref(cfg)))


def workspace_bytes(cfg: ModelConfig) -> int:
    return int(lib().rl_decode_workspace_bytes(C.byref(cfg)))


def _p(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _host_i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _host_u64(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.uint64))


class Engine:
    """One decode context: borrowed weights, a KV pool and a workspace
    allocated here with torch, and the current torch stream."""

    def __init__(self, shape: ModelShape, weights: Dict[str, torch.Tensor], max_seqs: int,
                 max_ctx: int, max_prefill_tokens: int, device="cuda", stream=None,
                 kv_page_size: int = 0, kv_pages: int = 0):
        L = lib()
        self.shape = shape
        self.cfg = make_config(shape, max_seqs, max_ctx, max_prefill_tokens, kv_page_size, kv_pages)
        self.kv_nbytes = kv_bytes(self.cfg)
        self.ws_nbytes = workspace_bytes(self.cfg)
        if self.kv_nbytes == 0 or self.ws_nbytes == 0:
            raise RLError(RL_ERR_INVALID_ARG, "configuration rejected")
        self.device = torch.device(device)
        self.kv = torch.empty(self.kv_nbytes, dtype=torch.uint8, device=self.device)
        self.ws = torch.empty(self.ws_nbytes, dtype=torch.uint8, device=self.device)
        self.weights = weights
        w = _weights_struct(weights)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = C.c_void_p()
        st = L.rl_decode_create(C.byref(self.cfg), C.byref(w), self.kv.data_ptr(), self.kv_nbytes,
                                self.ws.data_ptr(), self.ws_nbytes, self.stream.cuda_stream, C.byref(h))
        if st != RL_OK:
            raise RLError(st, "rl_decode_create failed")
        self.h = h

    # -- helpers ----------------------------------------------------------
    def _check(self, st: int, what: str):
        if st != RL_OK:
            raise RLError(st, f"{what}: {lib().rl_decode_last_error(self.h).decode()}")

    def close(self):
        if getattr(self, "h", None):
            lib().rl_decode_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- entry points -----------------------------------------------------
    def prefill(self, slots: Sequence[int], uids: Sequence[int], prompt_offsets: Sequence[int],
                tokens: torch.Tensor, out_tok: torch.Tensor, out_logp: torch.Tensor, *, group: int = 1,
                embeds: Optional[torch.Tensor] = None, forced: Optional[torch.Tensor] = None,
                seed: int = 0, temperature: float = 1.0, out_logits: Optional[torch.Tensor] = None):
        slots, uids, offs = _host_i32(slots), _host_u64(uids), _host_i32(prompt_offsets)
        n_prompts = len(offs) - 1
        sp = SampleParams(seed, temperature, 0)
        n_rows = 0 if embeds is None else int(embeds.shape[0])
        st = lib().rl_prefill(self.h, n_prompts, group, slots.ctypes.data, uids.ctypes.data,
                              offs.ctypes.data, _p(tokens), _p(embeds), n_rows, _p(forced), C.byref(sp),
                              _p(out_tok), _p(out_logp), _p(out_logits))
        self._check(st, "rl_prefill")

    def score(self, slots: Sequence[int], prompt_offsets: Sequence[int], prompt_tokens: torch.Tensor,
              resp_offsets: Sequence[int], resp_tokens: torch.Tensor, out_logp: torch.Tensor, *,
              group: int = 1, embeds: Optional[torch.Tensor] = None, temperature: float = 1.0):
        slots, poffs, roffs = _host_i32(slots), _host_i32(prompt_offsets), _host_i32(resp_offsets)
        n_rows = 0 if embeds is None else int(embeds.shape[0])
        st = lib().rl_score(self.h, len(poffs) - 1, group, slots.ctypes.data, poffs.ctypes.data,
                            _p(prompt_tokens), _p(embeds), n_rows, roffs.ctypes.data, _p(resp_tokens),
                            float(temperature), _p(out_logp))
        self._check(st, "rl_score")

    def step(self, slots: Sequence[int], uids: Sequence[int], in_tok: torch.Tensor, out_tok: torch.Tensor,
             out_logp: torch.Tensor, *, forced: Optional[torch.Tensor] = None, seed: int = 0,
             temperature: float = 1.0, out_logits: Optional[torch.Tensor] = None):
        slots, uids = _host_i32(slots), _host_u64(uids)
        sp = SampleParams(seed, temperature, 0)
        st = lib().rl_decode_step(self.h, len(slots), slots.ctypes.data, uids.ctypes.data, _p(in_tok),
                                  _p(forced), C.byref(sp), _p(out_tok), _p(out_logp), _p(out_logits))
        self._check(st, "rl_decode_step")

    def sample_logits(self, logits: torch.Tensor, uids: Sequence[int], pos_new: Sequence[int],
                      out_tok: torch.Tensor, out_logp: torch.Tensor, *, forced=None, seed: int = 0,
                      temperature: float = 1.0):
        uids, pos = _host_u64(uids), _host_i32(pos_new)
        sp = SampleParams(seed, temperature, 0)
        st = lib().rl_sample_logits(self.h, len(uids), _p(logits), uids.ctypes.data, pos.ctypes.data,
                                    _p(forced), C.byref(sp), _p(out_tok), _p(out_logp))
        self._check(st, "rl_sample_logits")

    def release(self, slots: Sequence[int]):
        s = _host_i32(slots)
        self._check(lib().rl_release_slots(self.h, len(s), s.ctypes.data), "rl_release_slots")

    def set_lengths(self, slots: Sequence[int], lengths: Sequence[int]):
        s, l = _host_i32(slots), _host_i32(lengths)
        self._check(lib().rl_set_slot_lengths(self.h, len(s), s.ctypes.data, l.ctypes.data),
                    "rl_set_slot_lengths")

    def slot_length(self, slot: int) -> int:
        return int(lib().rl_slot_length(self.h, slot))

    def kv_free_pages(self) -> int:
        """Free pages of a paged K/V pool (-1 for a contiguous pool)."""
        return int(lib().rl_kv_free_pages(self.h))

    def kv_offload_bytes(self, slots: Sequence[int]) -> int:
        s = _host_i32(slots)
        return int(lib().rl_kv_offload_bytes(self.h, len(s), s.ctypes.data))

    def kv_offload(self, slots: Sequence[int], host: torch.Tensor):
        """Live K/V of `slots` into `host` (a pinned uint8 CPU tensor)."""
        s = _host_i32(slots)
        self._check(lib().rl_kv_offload(self.h, len(s), s.ctypes.data, host.data_ptr(), host.numel()),
                    "rl_kv_offload")

    def kv_onload(self, slots: Sequence[int], lengths: Sequence[int], host: torch.Tensor):
        s, l = _host_i32(slots), _host_i32(lengths)
        self._check(lib().rl_kv_onload(self.h, len(s), s.ctypes.data, l.ctypes.data, host.data_ptr(),
                                       host.numel()), "rl_kv_onload")

    def rebind(self, weights: Dict[str, torch.Tensor], kv: torch.Tensor, ws: torch.Tensor):
        """Point the context at new device buffers (weights, KV pool, workspace)."""
        w = _weights_struct(weights)
        self._check(lib().rl_decode_rebind(self.h, C.byref(w), kv.data_ptr(), kv.numel(), ws.data_ptr(),
                                           ws.numel()), "rl_decode_rebind")
        self.weights, self.kv, self.ws = weights, kv, ws

    def set_option(self, option: int, value: int):
        self._check(lib().rl_decode_set_option(self.h, option, value), "rl_decode_set_option")

    def tune_gemms(self, sizes: Sequence[int]):
        """Measure the GEMM plans at these batch sizes (increasing); [] clears."""
        s = _host_i32(sizes)
        self._check(lib().rl_decode_tune_gemms(self.h, len(s), s.ctypes.data if len(s) else None),
                    "rl_decode_tune_gemms")

    def gemm_plan(self, kclass: str, rows: int):
        """(RL_OPT_GEMM_PLAN code, measured us per layer or -1) of a GEMM class at `rows` rows."""
        code, us = C.c_int64(0), C.c_float(0.0)
        self._check(lib().rl_decode_gemm_plan(self.h, KERNEL_CLASSES.index(kclass), rows, C.byref(code),
                                              C.byref(us)), "rl_decode_gemm_plan")
        return int(code.value), float(us.value)

    def kernel_stats(self) -> Dict[str, dict]:
        out = {}
        for k, name in enumerate(KERNEL_CLASSES):
            s = KernelStats()
            self._check(lib().rl_decode_kernel_stats(self.h, k, C.byref(s)), "rl_decode_kernel_stats")
            out[name] = {"launches": s.launches, "total_ms": s.total_ms, "alg_bytes": s.alg_bytes,
                         "alg_flops": s.alg_flops}
        return out

    def attn_plan_stats(self) -> Dict[str, int]:
        s = AttnPlanStats()
        self._check(lib().rl_decode_attn_plan_stats(self.h, C.byref(s)), "rl_decode_attn_plan_stats")
        return {name: int(getattr(s, name)) for name, _ in AttnPlanStats._fields_}

    def reset_stats(self):
        self._check(lib().rl_decode_reset_stats(self.h), "rl_decode_reset_stats")

    # -- KV pool views (layout of include/rl_decode.h) --------------------
    def kv_views(self):
        """(K, V) torch views of a contiguous pool: K [L][S][Hkv][cap][d],
        V [L][S][Hkv][cap/8][d][8] (8-position blocks), model dtype."""
        if self.cfg.kv_page_size:
            raise ValueError("a paged pool has no per-slot views")
        s = self.shape
        cap = (self.cfg.max_ctx + 31) // 32 * 32
        dt = torch.float32 if s.dtype == "fp32" else torch.bfloat16
        half = self.kv_nbytes // 2
        K = self.kv[:half].view(dt).view(s.n_layers, self.cfg.max_seqs, s.n_kv_heads, cap, s.head_dim)
        V = self.kv[half:].view(dt).view(s.n_layers, self.cfg.max_seqs, s.n_kv_heads, cap // 8, s.head_dim, 8)
        return K, V


def probe_copy(dst: torch.Tensor, src: torch.Tensor, nbytes: int, stream=None):
    stream = stream if stream is not None else torch.cuda.current_stream(dst.device)
    st = lib().rl_probe_copy(dst.data_ptr(), src.data_ptr(), nbytes, stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, "rl_probe_copy")


def probe_read(src: torch.Tensor, nbytes: int, out: torch.Tensor, stream=None):
    """Read-only stream of nbytes of src by out.numel() workgroups (out: int32, one word each)."""
    stream = stream if stream is not None else torch.cuda.current_stream(src.device)
    st = lib().rl_probe_read(src.data_ptr(), nbytes, out.numel(), out.data_ptr(), stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, "rl_probe_read")


def probe_mfma(n_blocks: int, iters: int, out: torch.Tensor, stream=None):
    """n_blocks x 4 waves x iters x 8 MFMA 32x32x16 bf16 (out: float32 [4 * n_blocks])."""
    if out.numel() < 4 * n_blocks or out.dtype != torch.float32:
        raise ValueError("out must hold 4 * n_blocks float32")
    stream = stream if stream is not None else torch.cuda.current_stream(out.device)
    st = lib().rl_probe_mfma(n_blocks, iters, out.data_ptr(), stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, "rl_probe_mfma")


def probe_gumbel_bound(lo: int, count: int, n_blocks: int = 4096, device="cuda"):
    """Run the sampler's noise-bound check over words [lo, lo + count);
    returns (violations, smallest margin of the fp32 bound)."""
    viol = torch.empty(n_blocks, dtype=torch.int32, device=device)
    mm = torch.empty(n_blocks, dtype=torch.float32, device=device)
    stream = torch.cuda.current_stream(torch.device(device))
    st = lib().rl_probe_gumbel_bound(int(lo), int(count), n_blocks, viol.data_ptr(), mm.data_ptr(),
                                     stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, "rl_probe_gumbel_bound")
    torch.cuda.synchronize(device)
    return int(viol.to(torch.int64).sum().item()), float(mm.min().item())


def sample_logits_noalloc(logits: torch.Tensor, uids: torch.Tensor, pos_new: torch.Tensor, out_tok: torch.Tensor,
                          out_logp: torch.Tensor, *, forced: Optional[torch.Tensor] = None, seed: int = 0,
                          temperature: float = 1.0, stream=None):
    """rl_sample_logits_noalloc: logits [n][ld] fp32, uids uint64 (int64
    tensor) and pos_new int32 on the device."""
    n, ld = int(logits.shape[0]), int(logits.stride(0))
    stream = stream if stream is not None else torch.cuda.current_stream(logits.device)
    sp = SampleParams(seed, temperature, 0)
    st = lib().rl_sample_logits_noalloc(n, int(logits.shape[1]), logits.data_ptr(), ld, uids.data_ptr(),
                                        pos_new.data_ptr(), _p(forced), C.byref(sp), out_tok.data_ptr(),
                                        out_logp.data_ptr(), stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, "rl_sample_logits_noalloc")


# -- training stage: losses and gradients on a caller's tensors ---------------
# Outputs are the caller's tensors.  Every tensor is contiguous but for logits
# and d_logits, whose rows may be apart (stride(0)).  Arguments are checked
# before anything is enqueued: ValueError for a tensor of the wrong type, size
# or device, RLError for what the library refuses.  `workspace`: a uint8
# tensor of at least the matching *_workspace_bytes; made here when None.

def _on(dev: int, name: str, t: Optional[torch.Tensor], dtype, numel: int, optional: bool = False):
    """Device pointer of a contiguous tensor of this type and size on GPU `dev`."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is missing")
    if t.dtype is dtype and t.get_device() == dev and t.numel() == numel < 1 << 31 and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be {dtype}, contiguous, of {numel} entries on cuda:{dev}, not {t.dtype} "
                     f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _mask_on(dev: int, mask: Optional[torch.Tensor], n: int):
    return _on(dev, "mask", mask, torch.bool if mask is not None and mask.dtype == torch.bool else torch.uint8, n, True)


def _rows_on(dev: int, name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None):
    """(pointer, row stride) of a float32 or bfloat16 matrix whose rows are contiguous."""
    if t.dim() != 2 or t.dtype not in (torch.float32, torch.bfloat16) or t.get_device() != dev or (
            like is not None and (t.dtype is not like.dtype or t.shape != like.shape)):
        raise ValueError(f"{name} must be a matrix of float32 or bfloat16 on cuda:{dev}"
                         + (f" like the logits ({tuple(like.shape)} {like.dtype})" if like is not None else "")
                         + f", not {t.dtype} {tuple(t.shape)} on {t.device}")
    n, V = t.shape
    ld = t.stride(0) if n > 1 else V
    if (V > 1 and t.stride(1) != 1) or ld < V or V >= 1 << 31:
        raise ValueError(f"{name}: entries of a row must be contiguous, fewer than 2^31, and rows apart: {tuple(t.shape)} "
                         f"with strides {t.stride()}")
    return t.data_ptr(), ld


def _gpu_of(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU")
    return t.get_device()


# the stream's handle without a Stream object around it (a sixth of a short call's time), where torch has it
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device   # the same without its check of the start-up


def _run_on(dev: int, stream, nbytes: int, workspace: Optional[torch.Tensor], call, what: str):
    """call(workspace pointer, its bytes, stream) with GPU `dev` current."""
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return _run_on(dev, stream, nbytes, workspace, call, what)
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{dev}")
    ws = None
    if workspace is not None:
        if workspace.dtype is not torch.uint8 or workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous uint8 tensor on cuda:{dev}")
        ws, nbytes = workspace.data_ptr(), workspace.numel()
    elif nbytes and stream is None:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr()
    elif nbytes:
        with torch.cuda.stream(stream):   # memory of that stream: the current one may still be using what it has freed
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        ws = workspace.data_ptr()
    st = call(ws, nbytes, _current_stream(dev) if stream is None else stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, what)


def _dtype_code(t: torch.Tensor) -> int:
    return RL_DTYPE_FP32 if t.dtype == torch.float32 else RL_DTYPE_BF16


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, out_logp: torch.Tensor, *,
                   out_entropy: Optional[torch.Tensor] = None, out_stats: Optional[torch.Tensor] = None,
                   temperature: float = 1.0, workspace: Optional[torch.Tensor] = None, stream=None):
    """rl_token_logprobs: log-probabilities of `targets` (int32 [n]) under
    logits [n][vocab], with the entropies and the statistics ([n][2]) that the
    backward pass takes."""
    dev = _gpu_of(logits, "logits")
    z, ld = _rows_on(dev, "logits", logits)
    n, V = logits.shape
    y = _on(dev, "targets", targets, torch.int32, n)
    lp = _on(dev, "out_logp", out_logp, torch.float32, n)
    ent = _on(dev, "out_entropy", out_entropy, torch.float32, n, True)
    st = _on(dev, "out_stats", out_stats, torch.float32, 2 * n, True)
    L = lib()
    _run_on(dev, stream, L.rl_logprob_workspace_bytes(n, V) if workspace is None else 0, workspace,
            lambda ws, nb, s: L.rl_token_logprobs(n, V, _dtype_code(logits), z, ld, y, temperature, lp, ent, st, ws, nb, s),
            "rl_token_logprobs")


def token_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, stats: torch.Tensor, d_logp: torch.Tensor,
                            d_logits: torch.Tensor, *, entropy: Optional[torch.Tensor] = None,
                            d_entropy: Optional[torch.Tensor] = None, temperature: float = 1.0, stream=None):
    """rl_token_logprobs_backward: d_logits (may be the logits) from the
    gradients of the log-probabilities and, with the forward's `entropy`, of
    the entropies."""
    dev = _gpu_of(logits, "logits")
    z, ld = _rows_on(dev, "logits", logits)
    dz, ldd = _rows_on(dev, "d_logits", d_logits, logits)
    n, V = logits.shape
    y = _on(dev, "targets", targets, torch.int32, n)
    st = _on(dev, "stats", stats, torch.float32, 2 * n)
    g = _on(dev, "d_logp", d_logp, torch.float32, n)
    ent = _on(dev, "entropy", entropy, torch.float32, n, True)
    ge = _on(dev, "d_entropy", d_entropy, torch.float32, n, True)
    L = lib()
    _run_on(dev, stream, 0, None,
            lambda ws, nb, s: L.rl_token_logprobs_backward(n, V, _dtype_code(logits), z, ld, y, temperature, st, ent, g,
                                                           ge, dz, ldd, s), "rl_token_logprobs_backward")


def _policy(dev, n: int, old_logp, advantages, token_advantages, seq_offsets, ref_logp, mask, clip_low, clip_high,
            dual_clip, kl, kl_coef, entropy_coef, aggregate, scale):
    """The structs of a policy loss over n tokens."""
    if kl not in KL_KINDS or aggregate not in AGGREGATES:
        raise ValueError(f"kl is one of {tuple(KL_KINDS)}, aggregate one of {tuple(AGGREGATES)}")
    k = 1 if seq_offsets is None else seq_offsets.numel() - 1
    if k < 1:
        raise ValueError("seq_offsets holds one entry more than there are sequences")
    batch = PolicyBatch(n, k, _on(dev, "seq_offsets", seq_offsets, torch.int32, k + 1, True),
                        _on(dev, "old_logp", old_logp, torch.float32, n),
                        _on(dev, "ref_logp", ref_logp, torch.float32, n, True),
                        _on(dev, "advantages", advantages, torch.float32, n if token_advantages else k),
                        _mask_on(dev, mask, n))
    params = PolicyParams(clip_low, clip_high, dual_clip, kl_coef, entropy_coef, scale, KL_KINDS[kl],
                          AGGREGATES[aggregate], int(bool(token_advantages)), 0)
    return batch, params


def policy_loss(logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, out_loss: torch.Tensor,
                d_logp: torch.Tensor, *, token_advantages: bool = False, seq_offsets: Optional[torch.Tensor] = None,
                ref_logp: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                mask: Optional[torch.Tensor] = None, d_entropy: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, dual_clip: float = 0.0, kl: str = "k3", kl_coef: float = 0.0,
                entropy_coef: float = 0.0, aggregate: str = "token_mean", scale: float = 1.0,
                workspace: Optional[torch.Tensor] = None, stream=None):
    """rl_policy_loss on packed tokens: out_loss [8] and the gradients of
    logp and entropy.  advantages: one a sequence, or with token_advantages
    one a token."""
    dev = _gpu_of(logp, "logp")
    n = logp.numel()
    lp = _on(dev, "logp", logp, torch.float32, n)
    ent = _on(dev, "entropy", entropy, torch.float32, n, True)
    out = _on(dev, "out_loss", out_loss, torch.float32, 8)
    g = _on(dev, "d_logp", d_logp, torch.float32, n)
    ge = _on(dev, "d_entropy", d_entropy, torch.float32, n, True)
    b, q = _policy(dev, n, old_logp, advantages, token_advantages, seq_offsets, ref_logp, mask, clip_low, clip_high,
                   dual_clip, kl, kl_coef, entropy_coef, aggregate, scale)
    L = lib()
    _run_on(dev, stream, L.rl_policy_workspace_bytes(n, b.n_seqs) if workspace is None else 0, workspace,
            lambda ws, nb, s: L.rl_policy_loss(C.byref(b), C.byref(q), lp, ent, out, g, ge, ws, nb, s), "rl_policy_loss")


def policy_loss_logits(logits: torch.Tensor, targets: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                       out_loss: torch.Tensor, out_logp: torch.Tensor, d_logits: torch.Tensor, *,
                       token_advantages: bool = False, seq_offsets: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                       mask: Optional[torch.Tensor] = None, out_entropy: Optional[torch.Tensor] = None,
                       temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2, dual_clip: float = 0.0,
                       kl: str = "k3", kl_coef: float = 0.0, entropy_coef: float = 0.0, aggregate: str = "token_mean",
                       scale: float = 1.0, workspace: Optional[torch.Tensor] = None, stream=None):
    """rl_policy_loss_logits: the policy loss of logits [n][vocab] and its
    gradient d_logits (may be the logits) in one call."""
    dev = _gpu_of(logits, "logits")
    z, ld = _rows_on(dev, "logits", logits)
    dz, ldd = _rows_on(dev, "d_logits", d_logits, logits)
    n, V = logits.shape
    y = _on(dev, "targets", targets, torch.int32, n)
    out = _on(dev, "out_loss", out_loss, torch.float32, 8)
    lp = _on(dev, "out_logp", out_logp, torch.float32, n)
    ent = _on(dev, "out_entropy", out_entropy, torch.float32, n, True)
    b, q = _policy(dev, n, old_logp, advantages, token_advantages, seq_offsets, ref_logp, mask, clip_low, clip_high,
                   dual_clip, kl, kl_coef, entropy_coef, aggregate, scale)
    L = lib()
    _run_on(dev, stream, L.rl_policy_logits_workspace_bytes(n, b.n_seqs, V) if workspace is None else 0, workspace,
            lambda ws, nb, s: L.rl_policy_loss_logits(C.byref(b), C.byref(q), V, _dtype_code(logits), z, ld, y,
                                                      temperature, out, lp, ent, dz, ldd, ws, nb, s),
            "rl_policy_loss_logits")


def preference_loss(logp: torch.Tensor, seq_offsets: torch.Tensor, out_loss: torch.Tensor, d_logp: torch.Tensor, *,
                    ref_logp: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                    out_rewards: Optional[torch.Tensor] = None, form: str = "sigmoid", average: bool = False,
                    beta: float = 0.1, label_smoothing: float = 0.0, margin: float = 0.0, scale: float = 1.0,
                    workspace: Optional[torch.Tensor] = None, stream=None):
    """rl_preference_loss on packed tokens: sequences 2p and 2p + 1 are pair
    p's chosen and rejected answers; out_loss [8] and the gradient of logp."""
    dev = _gpu_of(logp, "logp")
    n = logp.numel()
    lp = _on(dev, "logp", logp, torch.float32, n)
    P = (seq_offsets.numel() - 1) // 2
    if form not in PREFERENCE_FORMS:
        raise ValueError(f"form is one of {tuple(PREFERENCE_FORMS)}")
    offs = _on(dev, "seq_offsets", seq_offsets, torch.int32, 2 * P + 1)
    ref = _on(dev, "ref_logp", ref_logp, torch.float32, n, True)
    m = _mask_on(dev, mask, n)
    out = _on(dev, "out_loss", out_loss, torch.float32, 8)
    rew = _on(dev, "out_rewards", out_rewards, torch.float32, 2 * P, True)
    g = _on(dev, "d_logp", d_logp, torch.float32, n)
    q = PreferenceParams(beta, label_smoothing, margin, scale, PREFERENCE_FORMS[form], int(average))
    L = lib()
    _run_on(dev, stream, L.rl_preference_workspace_bytes(n, P) if workspace is None else 0, workspace,
            lambda ws, nb, s: L.rl_preference_loss(n, P, offs, lp, ref, m, C.byref(q), out, rew, g, ws, nb, s),
            "rl_preference_loss")


# -- rollout in 8 bits: norm, quantiser, product, cache and attention ----------
# Codes: float8_e4m3fn (or uint8) [rows][whole blocks of 128]; scale bytes:
# float8_e8m0fnu (or uint8) [rows, or tiles of 128 rows][blocks or more].  Rows
# may be apart (stride(0)).  As above: ValueError for a tensor of the wrong
# type, size or device, RLError for what the library refuses.

_CODES = (torch.float8_e4m3fn, torch.uint8)
_SCALES = (torch.float8_e8m0fnu, torch.uint8)


def fp8_blocks(k: int) -> int:
    """Blocks of 128 codes of a row of k entries."""
    return (int(k) + 127) // 128


def empty_fp8(rows: int, k: int, *, weight: bool = False, device="cuda"):
    """(codes, scales) with room for [rows][k] in 8 bits: a scale for each block of a row, or for each tile of a weight."""
    kb = fp8_blocks(k)
    codes = torch.empty(rows, 128 * kb, dtype=torch.float8_e4m3fn, device=device)
    scales = torch.empty(fp8_blocks(rows) if weight else rows, (kb + 3) // 4 * 4, dtype=torch.uint8, device=device)
    return codes, scales.view(torch.float8_e8m0fnu)


def _bytes_on(dev: int, name: str, t: torch.Tensor, dtypes, rows: int, width: int):
    """(pointer, row stride) of a matrix of bytes with this many rows of at least `width`."""
    shape, st = t.shape, t.stride()
    if len(shape) == 2 and shape[0] == rows and shape[1] >= width and t.dtype in dtypes and t.get_device() == dev:
        w = shape[1]
        ld = st[0] if rows > 1 else max(w, st[0])
        if ld >= w and (st[1] == 1 or w < 2):
            return t.data_ptr(), ld
    raise ValueError(f"{name} must be {rows} rows, apart, of {width} or more contiguous {' or '.join(map(str, dtypes))} on "
                     f"cuda:{dev}, not {t.dtype} {tuple(shape)} with strides {st} on {t.device}")


def _fp8_on(dev: int, name: str, codes: torch.Tensor, scales: torch.Tensor, rows: int, k: int, weight: bool = False) -> Fp8Matrix:
    kb = (k + 127) // 128
    c, ld = _bytes_on(dev, name, codes, _CODES, rows, 128 * kb)
    b, lds = _bytes_on(dev, name, scales, _SCALES, (rows + 127) // 128 if weight else rows, kb)
    return Fp8Matrix(c, ld, b, lds)


def _numbers_on(dev: int, name: str, t: torch.Tensor, rows: Optional[int] = None, width: Optional[int] = None):
    """(pointer, row stride, rows, entries, rl_dtype) of float32 or bfloat16 rows."""
    shape, st, dt = t.shape, t.stride(), t.dtype
    if len(shape) == 2 and (dt is torch.bfloat16 or dt is torch.float32) and t.get_device() == dev:
        n, w = shape
        ld = st[0] if n > 1 else w
        if (rows is None or (n == rows and w == width)) and ld >= w and w < 1 << 31 and (st[1] == 1 or w < 2):
            return t.data_ptr(), ld, n, w, RL_DTYPE_BF16 if dt is torch.bfloat16 else RL_DTYPE_FP32
    size = "" if rows is None else f"{rows} rows of {width} entries, "
    raise ValueError(f"{name} must be a matrix of float32 or bfloat16, {size}rows apart and of contiguous entries, on cuda:{dev}, "
                     f"not {dt} {tuple(shape)} with strides {st} on {t.device}")


def _launch_on(dev: int, stream, what: str, call, *args):
    """call(*args, stream) with GPU `dev` current: a call without a workspace."""
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return _launch_on(dev, stream, what, call, *args)
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{dev}")
    st = call(*args, _current_stream(dev) if stream is None else stream.cuda_stream)
    if st != RL_OK:
        raise RLError(st, what)


def rmsnorm_quant(x: torch.Tensor, weight: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, *,
                add: Optional[torch.Tensor] = None, out_sum: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None):
    """rl_rmsnorm_quant: rows of x (+ add, the sum to out_sum, which may be x)
    normed, times weight, in 8 bits."""
    dev = _gpu_of(x, "x")
    xp, ldx, n, H, dt = _numbers_on(dev, "x", x)
    wdt = weight.dtype
    if weight.dim() != 1 or (wdt is not torch.bfloat16 and wdt is not torch.float32):
        raise ValueError(f"weight must be a vector of float32 or bfloat16, not {wdt} {tuple(weight.shape)}")
    w = _on(dev, "weight", weight, wdt, H)
    ap, lda, adt = None, 0, dt
    if add is not None:
        ap, lda, _, _, adt = _numbers_on(dev, "add", add, n, H)
    sp, lds = None, 0
    if out_sum is not None:
        sp, lds, _, _, sdt = _numbers_on(dev, "out_sum", out_sum, n, H)
        if sdt != dt:
            raise ValueError(f"out_sum must be {x.dtype} as x is, not {out_sum.dtype}")
    out = _fp8_on(dev, "codes", codes, scales, n, H)
    _launch_on(dev, stream, "rl_rmsnorm_quant", lib().rl_rmsnorm_quant, n, H, dt, xp, ldx, adt, ap, lda,
               RL_DTYPE_BF16 if wdt is torch.bfloat16 else RL_DTYPE_FP32, w, eps, sp, lds, C.byref(out))


def quantise(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, *, form: str = "rows", stream=None):
    """rl_quantise: rows of x, silu(first half) * second half of its rows
    ("swiglu"), or a weight in tiles of 128 x 128 ("tiles"), in 8 bits."""
    if form not in FP8_FORMS:
        raise ValueError(f"form is one of {tuple(FP8_FORMS)}")
    dev = _gpu_of(x, "x")
    xp, ldx, n, k, dt = _numbers_on(dev, "x", x)
    if form == "swiglu":
        if k % 2:
            raise ValueError("the two halves of a row are of one size")
        k //= 2
    out = _fp8_on(dev, "codes", codes, scales, n, k, form == "tiles")
    _launch_on(dev, stream, "rl_quantise", lib().rl_quantise, FP8_FORMS[form], n, k, dt, xp, ldx, C.byref(out))


def gemm_quant(a: torch.Tensor, a_scales: torch.Tensor, w: torch.Tensor, w_scales: torch.Tensor, out: torch.Tensor, *,
             workspace: Optional[torch.Tensor] = None, stream=None):
    """rl_gemm_quant: out [m][n] = a [m][k] times the weight w [n][k] (tiles),
    both in whole blocks of 128 codes."""
    dev = _gpu_of(out, "out")
    o, ldo, m, n, dt = _numbers_on(dev, "out", out)
    k = a.shape[-1] if a.dim() == 2 else 0
    if k < 1 or k % 128:
        raise ValueError(f"a must hold rows of whole blocks of 128 codes, not {tuple(a.shape)}")
    A, W = _fp8_on(dev, "a", a, a_scales, m, k), _fp8_on(dev, "w", w, w_scales, n, k, True)
    if w.shape[1] != k:
        raise ValueError(f"a has rows of {k} codes, w of {w.shape[1]}")
    L = lib()
    need = L.rl_gemm_quant_workspace_bytes(m, n, k) if workspace is None else 0
    if workspace is None and not need:
        _launch_on(dev, stream, "rl_gemm_quant", L.rl_gemm_quant, m, n, k, C.byref(A), C.byref(W), dt, o, ldo, None, 0)
        return
    _run_on(dev, stream, need, workspace,
            lambda ws, nb, s: L.rl_gemm_quant(m, n, k, C.byref(A), C.byref(W), dt, o, ldo, ws, nb, s), "rl_gemm_quant")


def _counts(*numbers: int) -> bool:
    """Whether C takes them all as they are: ctypes cuts a number to its 32 bits without a word."""
    return all(-1 << 31 <= i < 1 << 31 for i in numbers)


def kv_quant_bytes(n_pages: int, page_size: int, n_kv_heads: int, head_dim: int) -> int:
    if not _counts(n_pages, page_size, n_kv_heads, head_dim):
        return 0
    return int(lib().rl_kv_quant_bytes(n_pages, page_size, n_kv_heads, head_dim))


def _heads_on(dev: int, name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None):
    """(pointer, row stride) of [n][heads][d] whose heads lie one after the other."""
    shape, st, dt = t.shape, t.stride(), t.dtype
    if len(shape) == 3 and (dt is torch.bfloat16 or dt is torch.float32) and t.get_device() == dev and (
            like is None or (dt is like.dtype and shape == like.shape)):
        n, h, d = shape
        ld = st[0] if n > 1 else h * d
        if (st[2] == 1 or d < 2) and (st[1] == d or h < 2) and ld >= h * d:
            return t.data_ptr(), ld
    raise ValueError(f"{name} must be [n][heads][d] of float32 or bfloat16 on cuda:{dev}, a token's heads contiguous and tokens apart"
                     + (f", like the other ({tuple(like.shape)} {like.dtype})" if like is not None else "")
                     + f", not {dt} {tuple(shape)} with strides {st} on {t.device}")


@functools.lru_cache(maxsize=64)
def _kv_page_bytes(page_size: int, heads: int, d: int) -> int:
    return kv_quant_bytes(1, page_size, heads, d)


def _cache_on(dev: int, pool: torch.Tensor, page_table: torch.Tensor, page_size: int, heads: int, d: int) -> KvFp8:
    one = _kv_page_bytes(page_size, heads, d)
    if not one:
        raise ValueError(f"no cache of pages of {page_size} positions with {heads} heads of {d}")
    shape = page_table.shape
    if len(shape) != 2:
        raise ValueError(f"page_table must be [sequences][pages], not {tuple(shape)}")
    n_pages = pool.numel() // one
    if pool.dtype is not torch.uint8 or pool.get_device() != dev or not pool.is_contiguous() or not 0 < n_pages < 1 << 31:
        raise ValueError(f"pool must be a contiguous uint8 tensor of whole pages ({one} bytes) on cuda:{dev}, not {pool.dtype} "
                         f"{tuple(pool.shape)} on {pool.device}")
    table = _on(dev, "page_table", page_table, torch.int32, shape[0] * shape[1])
    return KvFp8(pool.data_ptr(), table, shape[0], shape[1], n_pages, page_size, heads, d)


def _kv_call(name: str, dev: int, pool, page_table, seqs, positions, k, v, page_size, stream):
    kp, ldk = _heads_on(dev, "k", k)
    vp, ldv = _heads_on(dev, "v", v, k)
    n, h, d = k.shape
    cache = _cache_on(dev, pool, page_table, page_size, h, d)
    sq, ps = _on(dev, "seqs", seqs, torch.int32, n), _on(dev, "positions", positions, torch.int32, n)
    _launch_on(dev, stream, name, getattr(lib(), name), C.byref(cache), n, sq, ps, _dtype_code(k), kp, ldk, vp, ldv)


def kv_quant_append(pool: torch.Tensor, page_table: torch.Tensor, seqs: torch.Tensor, positions: torch.Tensor, k: torch.Tensor,
                  v: torch.Tensor, *, page_size: int, stream=None):
    """rl_kv_quant_append: keys and values [n][kv-heads][d] of tokens (seqs[i],
    positions[i]) into the pool (uint8, kv_quant_bytes of it)."""
    _kv_call("rl_kv_quant_append", _gpu_of(pool, "pool"), pool, page_table, seqs, positions, k, v, page_size, stream)


def kv_quant_read(pool: torch.Tensor, page_table: torch.Tensor, seqs: torch.Tensor, positions: torch.Tensor, out_k: torch.Tensor,
                out_v: torch.Tensor, *, page_size: int, stream=None):
    """rl_kv_quant_read: those tokens' keys and values as numbers."""
    _kv_call("rl_kv_quant_read", _gpu_of(pool, "pool"), pool, page_table, seqs, positions, out_k, out_v, page_size, stream)


def attention_quant(pool: torch.Tensor, page_table: torch.Tensor, q: torch.Tensor, lengths: torch.Tensor, out: torch.Tensor, *,
                  page_size: int, n_kv_heads: int, max_length: int, scale: float, seqs: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None):
    """rl_attention_quant: q and out [n][q-heads][d]; row i attends over the first
    lengths[i] <= max_length positions of sequence seqs[i] (of i without seqs)."""
    dev = _gpu_of(q, "q")
    qp, ldq = _heads_on(dev, "q", q)
    op, ldo = _heads_on(dev, "out", out, q)
    n, h, d = q.shape
    if not _counts(max_length):
        raise ValueError(f"max_length must be a count of 32 bits, not {max_length}")
    cache = _cache_on(dev, pool, page_table, page_size, n_kv_heads, d)
    ln, sq = _on(dev, "lengths", lengths, torch.int32, n), _on(dev, "seqs", seqs, torch.int32, n, True)
    L = lib()
    _run_on(dev, stream, L.rl_attention_quant_workspace_bytes(n, n_kv_heads, h, d, max_length) if workspace is None else 0, workspace,
            lambda ws, nb, s: L.rl_attention_quant(C.byref(cache), n, sq, ln, max_length, _dtype_code(q), qp, ldq, h, scale, op, ldo,
                                                 ws, nb, s), "rl_attention_quant")
