"""Thin ctypes binding of liblede (include/lede.h).

Argument marshalling only: every step of decoding runs in the library's HIP
kernels.  PyTorch provides device memory (the weight arena, KV pool,
workspace and weight staging buffers) and the stream handle.  There is no
fallback: if liblede.so is missing or no GPU is present, the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblede.so")

LEDE_OK, LEDE_E_ARG, LEDE_E_STATE, LEDE_E_KV_FULL, LEDE_E_CTX_OVERFLOW, LEDE_E_HIP, LEDE_E_UNSUPPORTED = \
    0, -1, -2, -3, -4, -5, -6
STATUS = {0: "OK", -1: "E_ARG", -2: "E_STATE", -3: "E_KV_FULL", -4: "E_CTX_OVERFLOW", -5: "E_HIP",
          -6: "E_UNSUPPORTED"}

T_EMBED, T_FINAL_NORM, T_HEAD, T_ATTN_NORM, T_WQ, T_WK, T_WV, T_WO, T_FFN_NORM, T_WG, T_WU, T_WD, \
    T_QNET_W1, T_QNET_B1, T_QNET_W2, T_QNET_B2, T_EXIT_W1, T_EXIT_B1, T_EXIT_W2, T_EXIT_B2 = range(20)
LAYER_KINDS = {"attn_norm": T_ATTN_NORM, "wq": T_WQ, "wk": T_WK, "wv": T_WV, "wo": T_WO,
               "ffn_norm": T_FFN_NORM, "wg": T_WG, "wu": T_WU, "wd": T_WD}


class LedeConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float), ("rope_base", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("max_ctx", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("qnet_hidden", ctypes.c_int32), ("n_exits", ctypes.c_int32),
                ("n_lengths", ctypes.c_int32), ("exits", ctypes.c_int32 * 64), ("lengths", ctypes.c_int32 * 16),
                ("k_max", ctypes.c_int32), ("exit_qnet_hidden", ctypes.c_int32)]


class LedeProfEntry(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double), ("bytes", ctypes.c_double), ("launches", ctypes.c_int64)]


K_NCLASS = 10
K_NAMES = ["linear_vec", "linear_mfma", "attention", "norm", "qnet", "accept", "draft_phase", "verify_phase",
           "linear_vec_gx", "linear_mfma_lx"]
# rocprofv3 kernel symbol of each linear timing class (bf16 models)
K_SYMBOLS = {"linear_vec": "lede::k_linear<1, 0>", "linear_mfma": "lede::k_linear<1, 2>",
             "linear_vec_gx": "lede::k_linear<1, 1>", "linear_mfma_lx": "lede::k_linear<1, 3>"}


LAYER_TENSORS = 9  # LEDE_LAYER_TENSORS: attn_norm, wq, wk, wv, wo, ffn_norm, wg, wu, wd
LAYER_ORDER = ["attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "wg", "wu", "wd"]
LOGITS_VERIFY, LOGITS_DRAFT = 0, 1


class LedeWeights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p), ("head", ctypes.c_void_p),
                ("first_layer", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("layer", ctypes.POINTER(ctypes.c_void_p)),
                ("qnet_w1", ctypes.c_void_p), ("qnet_b1", ctypes.c_void_p), ("qnet_w2", ctypes.c_void_p),
                ("qnet_b2", ctypes.c_void_p), ("exit_w1", ctypes.c_void_p), ("exit_b1", ctypes.c_void_p),
                ("exit_w2", ctypes.c_void_p), ("exit_b2", ctypes.c_void_p)]


class LedeAction(ctypes.Structure):
    _fields_ = [("l", ctypes.c_int32), ("k", ctypes.c_int32)]


class LedeStepRecord(ctypes.Structure):
    _fields_ = [("l", ctypes.c_int32), ("k_req", ctypes.c_int32), ("k_eff", ctypes.c_int32),
                ("accepted", ctypes.c_int32), ("n_emitted", ctypes.c_int32), ("tokens", ctypes.c_int32 * 17),
                ("drafts", ctypes.c_int32 * 16), ("q_action", ctypes.c_int32), ("q_max", ctypes.c_float),
                ("reward", ctypes.c_float), ("seq_len", ctypes.c_int32), ("pending", ctypes.c_int32)]


EXPORTED = ["lede_region_bytes", "lede_create", "lede_destroy", "lede_last_error", "lede_load_tensor",
            "lede_set_free_list", "lede_set_options", "lede_prefill", "lede_set_pending", "lede_truncate",
            "lede_draft", "lede_verify", "lede_step", "lede_get_kv_state", "lede_debug_read",
            "lede_prof_enable", "lede_prof_read", "lede_op_tiled_bytes", "lede_op_repack", "lede_op_linear",
            "lede_op_read_probe", "lede_op_read_groups", "lede_step_sampled", "lede_op_sample", "lede_step_policy", "lede_set_trace",
            "lede_get_trace", "lede_set_verify_reuse", "lede_dqn_region_bytes", "lede_dqn_create", "lede_dqn_destroy",
            "lede_dqn_last_error", "lede_dqn_init", "lede_dqn_push", "lede_dqn_record", "lede_dqn_end_episode",
            "lede_dqn_update", "lede_dqn_sync_target", "lede_dqn_act", "lede_dqn_read", "lede_step_submit",
            "lede_step_collect", "lede_load_weights", "lede_debug_logits", "lede_debug_inject_failure", "lede_op_sample_noalloc",
            "lede_op_cache_bytes", "lede_op_cache_plan", "lede_op_cache_append", "lede_op_cache_read",
            "lede_op_cache_attention_bytes", "lede_op_cache_attention", "lede_op_logprobs_bytes", "lede_op_logprobs",
            "lede_op_cache_fork", "lede_op_cache_own", "lede_op_cache_copy", "lede_op_cache_free", "lede_op_cache_compact",
            "lede_op_quant_bytes", "lede_op_quantize", "lede_op_quant_pack", "lede_op_quant_linear",
            "lede_op_head_loss_bytes", "lede_op_head_loss", "lede_op_head_loss_grad_bytes", "lede_op_head_loss_grad"]
MAX_IN_FLIGHT = 2
SAMPLE_SLOTS = 16
SAMPLE_STRIDE = 33

_lib = None


def load(path: str = LIB_PATH):
    """Load liblede.so and declare its signatures.  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("liblede.so not built (run __graft_entry__.build()): %s" % path)
    L = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    P = ctypes.POINTER
    L.lede_region_bytes.argtypes = [P(LedeConfig), P(sz), P(sz), P(sz)]
    L.lede_create.argtypes = [P(LedeConfig), vp, sz, vp, sz, vp, sz, P(vp)]
    L.lede_destroy.argtypes = [vp]
    L.lede_destroy.restype = None
    L.lede_last_error.argtypes = [vp]
    L.lede_last_error.restype = ctypes.c_char_p
    L.lede_load_tensor.argtypes = [vp, i32, i32, vp, vp]
    L.lede_load_weights.argtypes = [vp, P(LedeWeights), vp]
    L.lede_debug_logits.argtypes = [vp, i32, P(ctypes.c_float), sz, P(i32), vp]
    L.lede_debug_inject_failure.argtypes = [vp, i32]
    L.lede_set_free_list.argtypes = [vp, P(i32), i32]
    L.lede_set_options.argtypes = [vp, i32, i32]
    L.lede_set_verify_reuse.argtypes = [vp, i32]
    L.lede_prefill.argtypes = [vp, P(i32), i32, vp, P(i32)]
    L.lede_set_pending.argtypes = [vp, i32, vp]
    L.lede_truncate.argtypes = [vp, i32, vp]
    L.lede_draft.argtypes = [vp, i32, i32, vp, P(i32)]
    L.lede_verify.argtypes = [vp, vp, P(i32), P(i32), P(i32), P(i32)]
    L.lede_step.argtypes = [vp, P(LedeAction), i32, i32, vp, P(LedeStepRecord)]
    L.lede_step_submit.argtypes = [vp, P(LedeAction), i32, i32, vp]
    L.lede_step_collect.argtypes = [vp, vp, P(LedeStepRecord)]
    L.lede_get_kv_state.argtypes = [vp, P(i32), P(i32), P(i32), i32, P(i32)]
    L.lede_debug_read.argtypes = [vp, i32, P(ctypes.c_float), sz, P(i32), vp]
    L.lede_prof_enable.argtypes = [vp, i32]
    L.lede_prof_read.argtypes = [vp, P(LedeProfEntry), i32]
    L.lede_op_tiled_bytes.argtypes = [i32, i32, i32]
    L.lede_op_tiled_bytes.restype = sz
    L.lede_op_repack.argtypes = [i32, vp, i32, i32, vp, vp]
    L.lede_op_linear.argtypes = [i32, vp, i32, i32, vp, i32, i32, vp, i32, vp]
    L.lede_op_read_probe.argtypes = [vp, sz, vp, i32, vp, P(ctypes.c_float)]
    L.lede_op_read_groups.argtypes = [vp, i32, i32, vp, vp, P(ctypes.c_float)]
    L.lede_step_sampled.argtypes = [vp, P(LedeAction), i32, i32, ctypes.c_float, P(ctypes.c_float), vp,
                                    P(LedeStepRecord)]
    L.lede_op_sample.argtypes = [vp, i32, ctypes.c_float, ctypes.c_float, P(i32), vp]
    L.lede_op_sample_noalloc.argtypes = [vp, i32, i32, i32, ctypes.c_float, P(ctypes.c_float), P(i32), vp]
    L.lede_step_policy.argtypes = [vp, i32, vp, P(LedeStepRecord)]
    L.lede_set_trace.argtypes = [vp, P(ctypes.c_float), i32, vp]
    L.lede_get_trace.argtypes = [vp, P(ctypes.c_float), P(i32), vp]
    fp = P(ctypes.c_float)
    L.lede_dqn_region_bytes.argtypes = [P(LedeDqnConfig)]
    L.lede_dqn_region_bytes.restype = sz
    L.lede_dqn_create.argtypes = [P(LedeDqnConfig), vp, sz, P(vp)]
    L.lede_dqn_destroy.argtypes = [vp]
    L.lede_dqn_destroy.restype = None
    L.lede_dqn_last_error.argtypes = [vp]
    L.lede_dqn_last_error.restype = ctypes.c_char_p
    L.lede_dqn_init.argtypes = [vp, vp, vp]
    L.lede_dqn_push.argtypes = [vp, vp, i32, vp]
    L.lede_dqn_record.argtypes = [vp, vp, i32, vp]
    L.lede_dqn_end_episode.argtypes = [vp, vp]
    L.lede_dqn_update.argtypes = [vp, vp, vp, vp, fp]
    L.lede_dqn_sync_target.argtypes = [vp, vp]
    L.lede_dqn_act.argtypes = [vp, vp, vp, vp]
    L.lede_dqn_read.argtypes = [vp, i32, fp, sz, P(i32), vp]
    i64, f32 = ctypes.c_int64, ctypes.c_float
    L.lede_op_cache_bytes.argtypes = [i32] * 3
    L.lede_op_head_loss_bytes.argtypes = L.lede_op_head_loss_grad_bytes.argtypes = [i32, i32, i32, i32]
    L.lede_op_head_loss.argtypes = [i32, vp, i64, i32, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp]
    L.lede_op_head_loss_grad.argtypes = [i32, vp, i64, i32, vp, i64, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    L.lede_op_quant_bytes.argtypes = [i32, i32, i32]
    L.lede_op_quantize.argtypes = [i32, vp, i64, i32, i32, i32, vp, vp, vp]
    L.lede_op_quant_pack.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    L.lede_op_quant_linear.argtypes = [i32, vp, i32, i32, i32, vp, i64, i32, i32, vp, i64, vp]
    L.lede_op_cache_fork.argtypes = [vp, vp, vp, vp, i32, vp, i32, vp, i32, vp, vp]
    L.lede_op_cache_own.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, i32, vp, i32, vp, i32, vp, vp]
    L.lede_op_cache_copy.argtypes = [vp, vp, i32, vp, i32, i32, i32, vp]
    L.lede_op_cache_free.argtypes = [vp, vp, i32, vp, i32, vp, vp, i32, vp, i32, vp, vp]
    L.lede_op_cache_compact.argtypes = [vp, i32, vp, i32, vp, vp, i32, vp, i32, vp, i32, vp, vp]
    L.lede_op_cache_plan.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]
    L.lede_op_cache_append.argtypes = [i32, vp, i64, vp, i64, vp, i32, vp, i32, i32, i32, vp]
    L.lede_op_cache_read.argtypes = [i32, vp, i32, i32, i32, vp, i32, vp, i64, vp, i64, vp]
    L.lede_op_cache_attention_bytes.argtypes = [i32] * 8
    L.lede_op_cache_attention.argtypes = [i32, vp, i64, vp, i32, vp, i32, vp, vp, i32, i32, i32, i32, i32, f32, i32, i32,
                                          vp, i64, vp, sz, vp]
    L.lede_op_logprobs_bytes.argtypes = [i32] * 3
    L.lede_op_logprobs.argtypes = [i32, vp, i64, i32, i32, f32, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    sizes = ("lede_op_cache_bytes", "lede_op_cache_attention_bytes", "lede_op_logprobs_bytes", "lede_op_quant_bytes",
             "lede_op_head_loss_bytes", "lede_op_head_loss_grad_bytes")
    for name in sizes:
        getattr(L, name).restype = sz
    for name in EXPORTED:
        if name not in sizes + ("lede_destroy", "lede_last_error", "lede_op_tiled_bytes", "lede_dqn_region_bytes",
                                "lede_dqn_destroy", "lede_dqn_last_error"):
            getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


class LedeDqnConfig(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("capacity", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("n_step", ctypes.c_int32), ("gamma", ctypes.c_float), ("lr", ctypes.c_float),
                ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("adam_eps", ctypes.c_float),
                ("sigma0", ctypes.c_float)]


class LedeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("%s (%d): %s" % (STATUS.get(code, "?"), code, msg))
        self.code = code


def make_config(model, max_ctx: int, n_pages: Optional[int] = None, k_max: int = 15,
                exit_hidden: int = 0) -> LedeConfig:
    """lede_config from a model shape (any object with the ModelConfig fields);
    exit_hidden > 0 adds the paper's exit policy (its candidate layers are the
    model's exits)."""
    c = LedeConfig()
    c.n_layers, c.d_model, c.n_heads = model.n_layers, model.d_model, model.n_heads
    c.n_kv_heads, c.head_dim, c.ffn_dim, c.vocab = model.n_kv_heads, model.head_dim, model.ffn_dim, model.vocab
    c.rms_eps, c.rope_base = model.rms_eps, model.rope_base
    c.dtype = 1 if model.dtype == "bf16" else 0
    c.max_ctx, c.page_size = max_ctx, 64
    c.n_pages = n_pages if n_pages is not None else -(-max_ctx // 64)
    c.qnet_hidden = model.qnet_hidden
    c.n_exits, c.n_lengths = len(model.exits), len(model.lengths)
    for i, e in enumerate(model.exits):
        c.exits[i] = e
    for i, k in enumerate(model.lengths):
        c.lengths[i] = k
    c.k_max = k_max
    c.exit_qnet_hidden = exit_hidden
    return c


def _i32p(a):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


@dataclass
class StepRecord:
    l: int
    k_req: int
    k_eff: int
    accepted: int
    emitted: List[int]
    drafts: List[int]
    q_action: int
    q_max: float
    reward: float
    seq_len: int
    pending: int


class Engine:
    """A liblede context over torch-allocated device regions."""

    def __init__(self, model, max_ctx: int, n_pages: Optional[int] = None, k_max: int = 15, device: int = 0,
                 exit_hidden: int = 0):
        import torch
        self.torch = torch
        self.L = load()
        self.model = model
        self.cfg = make_config(model, max_ctx, n_pages, k_max, exit_hidden)
        wb, kvb, wsb = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        self._check(self.L.lede_region_bytes(ctypes.byref(self.cfg), ctypes.byref(wb), ctypes.byref(kvb),
                                             ctypes.byref(wsb)), None)
        self.region_bytes = (wb.value, kvb.value, wsb.value)
        dev = torch.device("cuda", device)
        self.device = dev
        self.weights = torch.empty(wb.value, dtype=torch.uint8, device=dev)
        self.kv = torch.empty(kvb.value, dtype=torch.uint8, device=dev)
        self.ws = torch.empty(wsb.value, dtype=torch.uint8, device=dev)
        h = ctypes.c_void_p()
        self._check(self.L.lede_create(ctypes.byref(self.cfg), self.weights.data_ptr(), wb.value,
                                       self.kv.data_ptr(), kvb.value, self.ws.data_ptr(), wsb.value,
                                       ctypes.byref(h)), None)
        self.ctx = h

    # -- plumbing ----------------------------------------------------------
    @property
    def stream(self):
        return ctypes.c_void_p(self.torch.cuda.current_stream(self.device).cuda_stream)

    def _check(self, rc: int, ctx):
        if rc != LEDE_OK:
            msg = self.L.lede_last_error(ctx).decode() if ctx is not None else ""
            raise LedeError(rc, msg)

    def close(self):
        if getattr(self, "ctx", None):
            self.L.lede_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- weights -------------------------------------------------------------
    def load_tensor(self, kind: int, layer: int, host: np.ndarray):
        t = self.torch
        a = np.ascontiguousarray(host)
        if a.dtype == np.uint16:
            a = a.view(np.int16)
        dev = t.from_numpy(a).to(self.device)
        self._check(self.L.lede_load_tensor(self.ctx, kind, layer, dev.data_ptr(), self.stream), self.ctx)
        t.cuda.current_stream(self.device).synchronize()

    def _dev(self, host: np.ndarray):
        a = np.ascontiguousarray(host)
        if a.dtype == np.uint16:
            a = a.view(np.int16)
        return self.torch.from_numpy(a).to(self.device)

    def lede_load_weights(self, weights: Optional[dict] = None, qnet: Optional[dict] = None,
                          exit_qnet: Optional[dict] = None, first_layer: int = 0, n_layers: int = 0):
        """One lede_load_weights call: the tensors given (host arrays in the
        lede_inputs.weights() layout) are staged on the device and repacked;
        absent ones are left as they are.  Layers [first_layer, first_layer +
        n_layers) come from weights["layers"]."""
        keep = []

        def ptr(host):
            if host is None:
                return None
            if isinstance(host, self.torch.Tensor) and host.device == self.device:
                keep.append(host)  # already staged on the device
                return host.data_ptr()
            d = self._dev(host)
            keep.append(d)
            return d.data_ptr()

        w = LedeWeights()
        weights = weights or {}
        w.embed, w.final_norm, w.head = (ptr(weights.get(n)) for n in ("embed", "final_norm", "head"))
        w.first_layer, w.n_layers = first_layer, n_layers
        table = (ctypes.c_void_p * max(1, n_layers * LAYER_TENSORS))()
        layers = weights.get("layers", [])
        for j in range(n_layers):
            if first_layer + j >= len(layers):
                break  # the library checks the range against the model
            for t, name in enumerate(LAYER_ORDER):
                table[j * LAYER_TENSORS + t] = ptr(layers[first_layer + j][name])
        w.layer = ctypes.cast(table, ctypes.POINTER(ctypes.c_void_p))
        f32 = lambda a: None if a is None else ptr(np.ascontiguousarray(a, dtype=np.float32))  # noqa: E731
        if qnet is not None:
            w.qnet_w1, w.qnet_b1, w.qnet_w2, w.qnet_b2 = (f32(qnet[n]) for n in ("w1", "b1", "w2", "b2"))
        if exit_qnet is not None:
            w.exit_w1, w.exit_b1, w.exit_w2, w.exit_b2 = (f32(exit_qnet[n]) for n in ("w1", "b1", "w2", "b2"))
        self._check(self.L.lede_load_weights(self.ctx, ctypes.byref(w), self.stream), self.ctx)
        self.torch.cuda.current_stream(self.device).synchronize()
        del keep

    def load_weights(self, weights: dict, qnet: Optional[dict] = None, staging_bytes: int = 16 << 30):
        """weights: lede_inputs.weights() layout; qnet: lede_inputs.qnet_weights().
        Through lede_load_weights: the embedding, head and Q-network in one
        call, then the layers in groups whose staging copies take at most
        staging_bytes of device memory."""
        self.lede_load_weights({n: weights[n] for n in ("embed", "final_norm", "head")}, qnet)
        layers = weights["layers"]
        per_layer = max(1, sum(np.asarray(a).nbytes for a in layers[0].values())) if layers else 1
        group = max(1, staging_bytes // per_layer)
        for j0 in range(0, len(layers), group):
            n = min(group, len(layers) - j0)
            self.lede_load_weights({"layers": layers}, first_layer=j0, n_layers=n)

    # -- C-ABI calls (same names) --------------------------------------------------
    def lede_set_options(self, use_graphs: int = 0, debug: int = 0):
        self._check(self.L.lede_set_options(self.ctx, use_graphs, debug), self.ctx)

    def lede_set_verify_reuse(self, enable: bool = True):
        self._check(self.L.lede_set_verify_reuse(self.ctx, int(enable)), self.ctx)

    def lede_set_free_list(self, order: Sequence[int]):
        a = np.ascontiguousarray(order, dtype=np.int32)
        self._check(self.L.lede_set_free_list(self.ctx, _i32p(a), len(a)), self.ctx)

    def lede_prefill(self, tokens: Sequence[int]) -> int:
        a = np.ascontiguousarray(tokens, dtype=np.int32)
        nxt = ctypes.c_int32()
        self._check(self.L.lede_prefill(self.ctx, _i32p(a), len(a), self.stream, ctypes.byref(nxt)), self.ctx)
        return nxt.value

    def lede_set_pending(self, token: int):
        self._check(self.L.lede_set_pending(self.ctx, token, self.stream), self.ctx)

    def lede_truncate(self, new_len: int):
        self._check(self.L.lede_truncate(self.ctx, new_len, self.stream), self.ctx)

    def lede_draft(self, l: int, k: int, read: bool = True) -> Optional[List[int]]:
        out = np.zeros(max(k, 1), dtype=np.int32)
        self._check(self.L.lede_draft(self.ctx, l, k, self.stream, _i32p(out) if read else None), self.ctx)
        return [int(x) for x in out[:k]] if read else None

    def lede_verify(self):
        """Returns (accepted, emitted tokens, verify argmax of every row)."""
        acc, ne = ctypes.c_int32(), ctypes.c_int32()
        toks = np.zeros(17, dtype=np.int32)
        ver = np.zeros(17, dtype=np.int32)
        self._check(self.L.lede_verify(self.ctx, self.stream, ctypes.byref(acc), _i32p(toks), ctypes.byref(ne),
                                       _i32p(ver)), self.ctx)
        return acc.value, [int(x) for x in toks[:ne.value]], ver

    @staticmethod
    def _record(rec) -> StepRecord:
        return StepRecord(l=rec.l, k_req=rec.k_req, k_eff=rec.k_eff, accepted=rec.accepted,
                          emitted=[rec.tokens[i] for i in range(rec.n_emitted)],
                          drafts=[rec.drafts[i] for i in range(rec.k_eff)], q_action=rec.q_action,
                          q_max=rec.q_max, reward=rec.reward, seq_len=rec.seq_len, pending=rec.pending)

    def lede_step(self, action=None, n_remaining: int = 1 << 30, log_qnet: bool = True) -> StepRecord:
        rec = LedeStepRecord()
        act = LedeAction(int(action[0]), int(action[1])) if action is not None else None
        self._check(self.L.lede_step(self.ctx, ctypes.byref(act) if act is not None else None, int(log_qnet),
                                     int(n_remaining), self.stream, ctypes.byref(rec)), self.ctx)
        return self._record(rec)

    def lede_step_submit(self, action, n_remaining: int = 1 << 30, log_qnet: bool = True) -> None:
        """Queue a forced greedy step; at most MAX_IN_FLIGHT wait for lede_step_collect."""
        act = LedeAction(int(action[0]), int(action[1]))
        self._check(self.L.lede_step_submit(self.ctx, ctypes.byref(act), int(log_qnet), int(n_remaining),
                                            self.stream), self.ctx)

    def lede_step_collect(self) -> StepRecord:
        """The record of the oldest submitted step (waits for it)."""
        rec = LedeStepRecord()
        self._check(self.L.lede_step_collect(self.ctx, self.stream, ctypes.byref(rec)), self.ctx)
        return self._record(rec)

    def lede_step_sampled(self, action, temperature: float, uniforms, n_remaining: int = 1 << 30,
                          log_qnet: bool = True) -> StepRecord:
        """A speculative-sampling step; uniforms: SAMPLE_STRIDE floats in [0, 1)."""
        rec = LedeStepRecord()
        act = LedeAction(int(action[0]), int(action[1])) if action is not None else None
        u = np.ascontiguousarray(uniforms, dtype=np.float32)
        if u.size != SAMPLE_STRIDE:
            raise ValueError("need %d uniforms" % SAMPLE_STRIDE)
        self._check(self.L.lede_step_sampled(self.ctx, ctypes.byref(act) if act is not None else None,
                                             int(log_qnet), int(n_remaining), float(temperature),
                                             u.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), self.stream,
                                             ctypes.byref(rec)), self.ctx)
        return self._record(rec)

    def load_exit_qnet(self, w: dict):
        """The exit policy's Q-network: lede_inputs.exit_qnet_weights() layout."""
        self.lede_load_weights(exit_qnet=w)

    def lede_step_policy(self, n_remaining: int = 1 << 30) -> StepRecord:
        rec = LedeStepRecord()
        self._check(self.L.lede_step_policy(self.ctx, int(n_remaining), self.stream, ctypes.byref(rec)), self.ctx)
        return self._record(rec)

    def policy_log(self) -> np.ndarray:
        """Decisions of the last lede_step_policy: rows of (kind, layer / draft,
        C_5, H, C_trace, Q(continue), Q(exit), action)."""
        out, rows = self.lede_debug_read(4, (64 + 12) * 8)
        return out[:rows * 8].reshape(rows, 8)

    def lede_set_trace(self, values):
        v = np.ascontiguousarray(values, dtype=np.float32)
        self._check(self.L.lede_set_trace(self.ctx, v.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), len(v),
                                          self.stream), self.ctx)

    def lede_get_trace(self) -> np.ndarray:
        v = np.zeros(20, dtype=np.float32)
        n = ctypes.c_int32()
        self._check(self.L.lede_get_trace(self.ctx, v.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                          ctypes.byref(n), self.stream), self.ctx)
        return v[:n.value]

    def lede_get_kv_state(self):
        """(seq_len, pending, block table)."""
        sl, pend, n = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        cap = self.cfg.max_ctx // 64 + 2
        bt = np.zeros(cap, dtype=np.int32)
        self._check(self.L.lede_get_kv_state(self.ctx, ctypes.byref(sl), ctypes.byref(pend), _i32p(bt), cap,
                                             ctypes.byref(n)), self.ctx)
        return sl.value, pend.value, [int(x) for x in bt[:n.value]]

    def lede_debug_read(self, which: int, n_floats: int) -> np.ndarray:
        out = np.zeros(n_floats, dtype=np.float32)
        rows = ctypes.c_int32()
        self._check(self.L.lede_debug_read(self.ctx, which, out.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                           n_floats, ctypes.byref(rows), self.stream), self.ctx)
        return out, rows.value

    def lede_debug_logits(self, which: int = LOGITS_VERIFY) -> np.ndarray:
        """Logits of the last verify / prefill head (LOGITS_VERIFY) or of the
        last step's draft heads (LOGITS_DRAFT), [rows][vocab]."""
        V = self.model.vocab
        out = np.zeros(16 * V, dtype=np.float32)
        rows = ctypes.c_int32()
        self._check(self.L.lede_debug_logits(self.ctx, int(which), out.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                             out.size, ctypes.byref(rows), self.stream), self.ctx)
        return out[:rows.value * V].reshape(rows.value, V)

    def lede_debug_inject_failure(self, n_ops: int):
        """The (n_ops + 1)-th device operation of the next calls fails with
        E_HIP before it is issued (one-shot; n_ops < 0 disables)."""
        self._check(self.L.lede_debug_inject_failure(self.ctx, int(n_ops)), self.ctx)

    def lede_prof_enable(self, level: int):
        """0 off, 1 draft / verify phases only, 2 phases and every launch."""
        self._check(self.L.lede_prof_enable(self.ctx, int(level)), self.ctx)

    def lede_prof_read(self, reset: bool = True) -> dict:
        arr = (LedeProfEntry * K_NCLASS)()
        self._check(self.L.lede_prof_read(self.ctx, arr, int(reset)), self.ctx)
        return {K_NAMES[i]: {"ms": arr[i].ms, "bytes": arr[i].bytes, "launches": arr[i].launches}
                for i in range(K_NCLASS)}

    def logits(self, which: int = 0) -> np.ndarray:
        """Debug logits of the last verify/prefill head (which=0) or of the
        last draft passes (which=3), shape [rows][vocab]."""
        V = self.model.vocab
        out, rows = self.lede_debug_read(which, 16 * V)
        return out[:rows * V].reshape(rows, V)


# ---- single-op helpers (kernel-level tests) ----------------------------------------

def op_linear(W, x, use_mfma: bool):
    """y = x W^T through the library's tiled linear kernels.  W [N][K] and x
    [M][K] are torch tensors on the GPU (float32 or bfloat16)."""
    import torch
    L = load()
    dtype = 1 if W.dtype == torch.bfloat16 else 0
    N, K = W.shape
    M = x.shape[0]
    tiled = torch.empty(L.lede_op_tiled_bytes(dtype, N, K), dtype=torch.uint8, device=W.device)
    y = torch.empty(M, N, dtype=torch.float32, device=W.device)
    s = ctypes.c_void_p(torch.cuda.current_stream(W.device).cuda_stream)
    rc = L.lede_op_repack(dtype, W.data_ptr(), N, K, tiled.data_ptr(), s)
    if rc:
        raise LedeError(rc, "op_repack")
    # rows padded with zeros to the tile width, which the kernels read whole
    tk = 32 if dtype == 1 else 16
    ldx = -(-K // tk) * tk
    xp = torch.zeros(M, ldx, dtype=x.dtype, device=x.device)
    xp[:, :K] = x
    rc = L.lede_op_linear(dtype, tiled.data_ptr(), N, K, xp.data_ptr(), ldx, M, y.data_ptr(), int(use_mfma), s)
    if rc:
        raise LedeError(rc, "op_linear")
    return y


def op_read_probe(buf, grid: int = 0) -> float:
    """Kernel milliseconds for one read of the whole GPU tensor buf (its byte
    size a multiple of 16) with the weight-streaming loads."""
    import torch
    L = load()
    nbytes = buf.numel() * buf.element_size()
    grid = grid or 256 * 16
    sink = torch.empty(grid, dtype=torch.int32, device=buf.device)
    ms = ctypes.c_float()
    s = ctypes.c_void_p(torch.cuda.current_stream(buf.device).cuda_stream)
    rc = L.lede_op_read_probe(buf.data_ptr(), nbytes, sink.data_ptr(), int(grid), s, ctypes.byref(ms))
    if rc:
        raise LedeError(rc, "op_read_probe")
    return ms.value


def op_read_groups(buf, n_groups: int, tiles: int) -> float:
    """Kernel milliseconds for reading n_groups x tiles 1 KiB tiles at the start
    of the GPU tensor buf with the one-row linear kernel's load structure."""
    import torch
    L = load()
    if n_groups * tiles * 1024 > buf.numel() * buf.element_size():
        raise LedeError(LEDE_E_ARG, "buffer smaller than n_groups x tiles KiB")
    sink = torch.empty(n_groups, dtype=torch.int32, device=buf.device)
    ms = ctypes.c_float()
    s = ctypes.c_void_p(torch.cuda.current_stream(buf.device).cuda_stream)
    rc = L.lede_op_read_groups(buf.data_ptr(), int(n_groups), int(tiles), sink.data_ptr(), s, ctypes.byref(ms))
    if rc:
        raise LedeError(rc, "op_read_groups")
    return ms.value


def op_sample(logits, temperature: float, u: float) -> int:
    """One inverse-CDF draw from softmax(logits / temperature) by the
    library's sampling kernel; logits is a float32 GPU tensor of one row."""
    import torch
    L = load()
    tok = ctypes.c_int32()
    s = ctypes.c_void_p(torch.cuda.current_stream(logits.device).cuda_stream)
    x = logits.contiguous()
    rc = L.lede_op_sample(x.data_ptr(), x.numel(), float(temperature), float(u), ctypes.byref(tok), s)
    if rc:
        raise LedeError(rc, "op_sample")
    return tok.value


def op_sample_noalloc(logits, temperature: float, u) -> List[int]:
    """One inverse-CDF draw per row of the float32 GPU tensor logits [rows][V]
    (rows <= 32) with the uniforms u [rows], through the entry point that
    allocates nothing."""
    import torch
    L = load()
    x = logits.contiguous()
    rows, V = x.shape
    uu = np.ascontiguousarray(u, dtype=np.float32)
    out = np.zeros(max(rows, 1), dtype=np.int32)
    s = ctypes.c_void_p(torch.cuda.current_stream(x.device).cuda_stream)
    rc = L.lede_op_sample_noalloc(x.data_ptr(), rows, V, V, float(temperature),
                                  uu.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), _i32p(out), s)
    if rc:
        raise LedeError(rc, "op_sample_noalloc")
    return [int(t) for t in out[:rows]]


# ---- a batch of requests over one paged 8-bit cache ----------------------------------

def _call(device, what: str, fn, *args):
    """fn(*args, current stream of device) with that device current; a status
    other than OK raises."""
    import torch
    index = device.index
    _need(index is not None, what + ": tensors on the GPU")
    stream = torch._C._cuda_getCurrentRawStream   # (torch.cuda.current_stream builds an object: 1.9 us against 0.1)
    if index == torch._C._cuda_getDevice():       # (torch.cuda.current_device checks for initialisation first: 0.7 us against 0.2)
        rc = fn(*args, stream(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, stream(index))
    if rc:
        raise LedeError(rc, what)


def _need(ok: bool, what: str):
    if not ok:
        raise LedeError(LEDE_E_ARG, what)


def _dense(device, dtype, *tensors) -> bool:
    index = -1 if device.index is None else device.index
    for t in tensors:
        if t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
            return False
    return True


def _dtype_code(torch, dtype) -> int:
    if dtype is torch.bfloat16:
        return 1
    _need(dtype is torch.float32, "dtype must be float32 or bfloat16")
    return 0


def _row_stride(x, heads: int, head_dim: int, what: str) -> int:
    """Elements between the rows of x [rows][heads][head_dim], whose heads are dense."""
    rows, h, d = x.shape
    r, sh, sd = x.stride()
    _need(h == heads and d == head_dim and sd == 1 and (sh == d or h == 1), what)
    return r if rows > 1 else max(r, h * d)


class Cache:
    """One layer's paged 8-bit K/V cache: n_pages pages of 64 tokens, in
    `region`, a uint8 GPU tensor of lede_op_cache_bytes (allocated and cleared
    when not given)."""

    def __init__(self, n_pages: int, n_kv: int, head_dim: int, device: int = 0, region=None):
        import torch
        nbytes = load().lede_op_cache_bytes(n_pages, n_kv, head_dim)
        if nbytes == 0:
            raise LedeError(LEDE_E_UNSUPPORTED, "cache of %d pages, %d heads of %d" % (n_pages, n_kv, head_dim))
        if region is None:
            region = torch.zeros(nbytes, dtype=torch.uint8, device=torch.device("cuda", device))
        _need(region.dtype == torch.uint8 and region.is_contiguous() and region.numel() >= nbytes, "cache region")
        self.region, self.n_pages, self.n_kv, self.head_dim = region, n_pages, n_kv, head_dim
        self.device = region.device


@dataclass
class CachePlan:
    kv_lens: object
    held: object
    row_start: object
    slots: object
    status: object   # code, rows, place in the free list after the call, first failing sequence


def op_cache_plan(seq_lens, new_lens, held, free_pages, free_head, tables, max_rows: int,
                  out: Optional[CachePlan] = None) -> CachePlan:
    """Pages and slots of a pass in which sequence s gets new_lens[s] tokens
    behind seq_lens[s] cached ones (int32 GPU tensors; tables [n_seqs][width]
    is updated).  `out` reuses a plan's tensors, which may be the inputs'
    own (kv_lens is seq_lens, held is held, free_head is status[2:3]); of
    longer slots the first max_rows are written, and only those are the plan's."""
    import torch
    dev, n, max_rows = seq_lens.device, seq_lens.numel(), int(max_rows)
    _need(_dense(dev, torch.int32, seq_lens, new_lens, held, free_pages, free_head, tables) and tables.dim() == 2
          and new_lens.numel() == n and held.numel() == n and tables.shape[0] == n and free_head.numel() == 1 and max_rows >= 0,
          "op_cache_plan")
    if out is None:
        buf = torch.empty(3 * n + 5, dtype=torch.int32, device=dev)
        kv_lens, held_out, row_start, status = buf.split_with_sizes((n, n, n + 1, 4))
        out = CachePlan(kv_lens, held_out, row_start, torch.empty(max_rows, dtype=torch.int64, device=dev), status)
    else:
        _need(_dense(dev, torch.int32, out.kv_lens, out.held, out.row_start, out.status)
              and _dense(dev, torch.int64, out.slots) and out.kv_lens.numel() == n and out.held.numel() == n
              and out.row_start.numel() == n + 1 and out.slots.numel() >= max_rows and out.status.numel() == 4,
              "op_cache_plan: out")
    _call(dev, "op_cache_plan", load().lede_op_cache_plan, seq_lens.data_ptr(), new_lens.data_ptr(), held.data_ptr(), n,
          free_pages.data_ptr(), free_pages.numel(), free_head.data_ptr(), tables.data_ptr(), tables.shape[1], max_rows,
          out.kv_lens.data_ptr(), out.held.data_ptr(), out.row_start.data_ptr(), out.slots.data_ptr(), out.status.data_ptr())
    return out


def _int32(sizes: int, what: str):
    """sizes: the bits of all that a call takes as 32-bit numbers (ctypes cuts larger ones off without a word)."""
    if sizes >> 31:
        raise LedeError(LEDE_E_UNSUPPORTED, what + ": sizes of 2^31 or more")


def _status(torch, status, n: int, device, what: str):
    if status is None:
        return torch.empty(n, dtype=torch.int32, device=device)
    _need(_dense(device, torch.int32, status) and status.numel() == n, what + ": status")
    return status


def op_cache_fork(source, seq_lens, held, tables, shares, lens=None, status=None):
    """Sequence s with source[s] = r >= 0 becomes the first lens[s] tokens of
    sequence r (all of them without `lens`) and shares its pages; -1 leaves it.
    int32 GPU tensors; seq_lens, held, tables [n_seqs][width] and shares
    [n_pages] are updated.  Returns status [3]: code, entries shared, first
    failing sequence."""
    import torch
    dev, n = seq_lens.device, seq_lens.numel()
    _need(_dense(dev, torch.int32, source, seq_lens, held, tables, shares) and tables.dim() == 2 and source.numel() == n
          and held.numel() == n and tables.shape[0] == n
          and (lens is None or (_dense(dev, torch.int32, lens) and lens.numel() == n)), "op_cache_fork")
    _int32(n | tables.shape[1] | shares.numel(), "op_cache_fork")
    status = _status(torch, status, 3, dev, "op_cache_fork")
    _call(dev, "op_cache_fork", load().lede_op_cache_fork, source.data_ptr(), None if lens is None else lens.data_ptr(),
          seq_lens.data_ptr(), held.data_ptr(), n, tables.data_ptr(), tables.shape[1], shares.data_ptr(), shares.numel(),
          status.data_ptr())
    return status


@dataclass
class CacheMoves:
    pairs: object    # [max_moves][2]: page, page that gets its content; -1 behind the last
    status: object   # code, moves, place in the free list after the call, first failing sequence (compact: live pages)


def _moves(torch, out, max_moves: int, device, what: str) -> CacheMoves:
    if out is None:
        return CacheMoves(torch.empty(max_moves, 2, dtype=torch.int32, device=device), torch.empty(4, dtype=torch.int32, device=device))
    _need(_dense(device, torch.int32, out.pairs, out.status) and out.pairs.numel() == 2 * max_moves and out.status.numel() == 4,
          what + ": out")
    return out


def op_cache_own(seq_lens, new_lens, held, free_pages, free_head, tables, shares, max_moves: int,
                 out: Optional[CacheMoves] = None) -> CacheMoves:
    """Before new_lens[s] tokens are appended behind seq_lens[s]: the held pages
    that they fall into become the sequence's alone (tables and shares are
    updated).  Pages whose content has to follow are listed for op_cache_copy;
    max_moves = n_seqs always suffices."""
    import torch
    dev, n, max_moves = seq_lens.device, seq_lens.numel(), int(max_moves)
    _need(_dense(dev, torch.int32, seq_lens, new_lens, held, free_pages, free_head, tables, shares) and tables.dim() == 2
          and new_lens.numel() == n and held.numel() == n and tables.shape[0] == n and free_head.numel() == 1 and max_moves >= 0,
          "op_cache_own")
    _int32(n | free_pages.numel() | tables.shape[1] | shares.numel() | max_moves, "op_cache_own")
    out = _moves(torch, out, max_moves, dev, "op_cache_own")
    _call(dev, "op_cache_own", load().lede_op_cache_own, seq_lens.data_ptr(), new_lens.data_ptr(), held.data_ptr(), n,
          free_pages.data_ptr(), free_pages.numel(), free_head.data_ptr(), tables.data_ptr(), tables.shape[1], shares.data_ptr(),
          shares.numel(), out.pairs.data_ptr(), max_moves, out.status.data_ptr())
    return out


def op_cache_copy(cache: Cache, pairs, count):
    """Page pairs[i][0] of the cache to page pairs[i][1], for the first
    count[0] of the pairs [max_moves][2] (int32; moves.pairs and
    moves.status[1:2] of op_cache_own and op_cache_compact); once a layer."""
    import torch
    dev = cache.device
    _need(_dense(dev, torch.int32, pairs, count) and pairs.dim() == 2 and pairs.shape[1] == 2 and count.numel() == 1, "op_cache_copy")
    _int32(pairs.shape[0], "op_cache_copy")
    _call(dev, "op_cache_copy", load().lede_op_cache_copy, pairs.data_ptr(), count.data_ptr(), pairs.shape[0], cache.region.data_ptr(),
          cache.n_pages, cache.n_kv, cache.head_dim)


def op_cache_free(seq_lens, held, free_pages, free_head, tables, shares, status=None):
    """Pages that the sequences' seq_lens[s] tokens do not need (all of them
    where that is 0) are given back; held, shares and free_pages are updated.
    Returns status [4]: code, pages freed, place in the free list after the
    call, first failing sequence (free_head may be its [2:3])."""
    import torch
    dev, n = seq_lens.device, seq_lens.numel()
    _need(_dense(dev, torch.int32, seq_lens, held, free_pages, free_head, tables, shares) and tables.dim() == 2 and held.numel() == n
          and tables.shape[0] == n and free_head.numel() == 1, "op_cache_free")
    _int32(n | free_pages.numel() | tables.shape[1] | shares.numel(), "op_cache_free")
    status = _status(torch, status, 4, dev, "op_cache_free")
    _call(dev, "op_cache_free", load().lede_op_cache_free, seq_lens.data_ptr(), held.data_ptr(), n, free_pages.data_ptr(),
          free_pages.numel(), free_head.data_ptr(), tables.data_ptr(), tables.shape[1], shares.data_ptr(), shares.numel(),
          status.data_ptr())
    return status


def op_cache_compact(held, free_pages, free_head, tables, shares, max_moves: int, out: Optional[CacheMoves] = None) -> CacheMoves:
    """The pages that the tables' held entries name become the pool's first
    ones (tables, shares and free_pages are updated); the moves are listed for
    op_cache_copy; max_moves = n_pages // 2 always suffices."""
    import torch
    dev, n, max_moves = held.device, held.numel(), int(max_moves)
    _need(_dense(dev, torch.int32, held, free_pages, free_head, tables, shares) and tables.dim() == 2 and tables.shape[0] == n
          and free_head.numel() == 1 and max_moves >= 0, "op_cache_compact")
    _int32(n | free_pages.numel() | tables.shape[1] | shares.numel() | max_moves, "op_cache_compact")
    out = _moves(torch, out, max_moves, dev, "op_cache_compact")
    _call(dev, "op_cache_compact", load().lede_op_cache_compact, held.data_ptr(), n, free_pages.data_ptr(), free_pages.numel(),
          free_head.data_ptr(), tables.data_ptr(), tables.shape[1], shares.data_ptr(), shares.numel(), out.pairs.data_ptr(), max_moves,
          out.status.data_ptr())
    return out


def op_cache_append(cache: Cache, k, v, slots):
    """Rows k and v [rows][n_kv][head_dim] (any row stride that is a multiple
    of 16 bytes) into the cache at slots (int64)."""
    import torch
    dev, kv, hd, n = cache.device, cache.n_kv, cache.head_dim, slots.numel()
    _need(_dense(dev, torch.int64, slots) and k.dim() == 3 and v.dim() == 3 and k.shape[0] == n and v.shape[0] == n
          and k.device == dev and v.device == dev and k.dtype == v.dtype, "op_cache_append")
    _call(dev, "op_cache_append", load().lede_op_cache_append, _dtype_code(torch, k.dtype), k.data_ptr(),
          _row_stride(k, kv, hd, "op_cache_append: k"), v.data_ptr(), _row_stride(v, kv, hd, "op_cache_append: v"),
          slots.data_ptr(), n, cache.region.data_ptr(), cache.n_pages, kv, hd)


def op_cache_read(cache: Cache, slots, dtype, out=None):
    """(k, v) [rows][n_kv][head_dim] of `dtype` that the cache holds at slots
    (int64); `out` gives the two tensors."""
    import torch
    dev, kv, hd, n = cache.device, cache.n_kv, cache.head_dim, slots.numel()
    code = _dtype_code(torch, dtype)
    k, v = torch.empty(2, n, kv, hd, dtype=dtype, device=dev).unbind(0) if out is None else out
    _need(_dense(dev, torch.int64, slots) and k.dim() == 3 and v.dim() == 3 and k.shape[0] == n and v.shape[0] == n
          and k.device == dev and v.device == dev and k.dtype == dtype and v.dtype == dtype, "op_cache_read")
    _call(dev, "op_cache_read", load().lede_op_cache_read, code, cache.region.data_ptr(), cache.n_pages, kv, hd,
          slots.data_ptr(), n, k.data_ptr(), _row_stride(k, kv, hd, "op_cache_read: k"), v.data_ptr(),
          _row_stride(v, kv, hd, "op_cache_read: v"))
    return k, v


def _workspace(torch, need: int, workspace, device, what: str):
    """(tensor, address, bytes) of the workspace, the caller's or one of `need` bytes."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _need(workspace.device == device and workspace.is_contiguous(), what)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def op_cache_attention(cache: Cache, q, tables, kv_lens, row_start, max_new: int, max_kv: int, scale: Optional[float] = None,
                       out=None, workspace=None):
    """Causal attention of q [rows][n_heads][head_dim], the rows row_start[s] ..
    row_start[s + 1] - 1 being the last of the kv_lens[s] cached tokens of
    sequence s, over the pages of tables [n_seqs][width] (int32).  max_new and
    max_kv: the largest numbers of rows and of tokens expected.  `scale` is
    head_dim ** -0.5 when not given.  Rows of a new `out` that no sequence has
    are undefined; a given one's (q itself is taken) are left as they are."""
    import torch
    dev, kv, hd, n = cache.device, cache.n_kv, cache.head_dim, kv_lens.numel()
    max_new, max_kv = int(max_new), int(max_kv)
    _need(_dense(dev, torch.int32, tables, kv_lens, row_start) and q.dim() == 3 and q.device == dev and tables.dim() == 2
          and tables.shape[0] == n and row_start.numel() == n + 1, "op_cache_attention")
    rows, heads, _ = q.shape
    ldq = _row_stride(q, heads, hd, "op_cache_attention: q")
    if out is None:
        out = torch.empty(rows, heads, hd, dtype=q.dtype, device=dev)
        ldo = heads * hd
    else:
        _need(out.dtype == q.dtype and out.shape == q.shape and out.device == dev, "op_cache_attention: out")
        ldo = _row_stride(out, heads, hd, "op_cache_attention: out")
    L, code = load(), _dtype_code(torch, q.dtype)
    need = L.lede_op_cache_attention_bytes(code, n, rows, heads, kv, hd, max_new, max_kv)
    ws, ws_at, ws_bytes = _workspace(torch, need, workspace, dev, "op_cache_attention: workspace")
    _call(dev, "op_cache_attention", L.lede_op_cache_attention, code, q.data_ptr(), ldq,
          cache.region.data_ptr(), cache.n_pages, tables.data_ptr(), tables.shape[1], kv_lens.data_ptr(),
          row_start.data_ptr(), n, rows, heads, kv, hd, hd ** -0.5 if scale is None else scale, max_new, max_kv,
          out.data_ptr(), ldo, ws_at, ws_bytes)
    return out


@dataclass
class Logprobs:
    logprobs: object
    ranks: object
    entropy: object
    top_ids: object
    top_logprobs: object


def op_logprobs(logits, tokens, n_top: int = 0, temperature: float = 1.0, workspace=None) -> Logprobs:
    """Log probabilities under softmax(logits / temperature) of the given token
    of each row (int32 [rows]; None: no token), its rank, the row's entropy and
    its n_top most likely tokens.  logits [rows][V] is float32 or bfloat16, of
    any row stride."""
    import torch
    dev = logits.device
    n_top = int(n_top)
    rows, V = logits.shape
    ld, step = logits.stride()
    _need((step == 1 or V == 1) and (tokens is None or (_dense(dev, torch.int32, tokens) and tokens.numel() == rows)),
          "op_logprobs")
    _need(0 <= n_top <= V, "op_logprobs: n_top")
    given, m, f32 = tokens is not None, rows * n_top, torch.float32
    buf = torch.empty(3 * rows + 2 * m, dtype=torch.int32, device=dev)      # (one allocation, split and seen as fp32: 0.9 us less than two)
    logprobs, entropy, top, ranks, ids = buf.split_with_sizes((rows, rows, m, rows, m))
    L = load()
    ws, ws_at, ws_bytes = _workspace(torch, L.lede_op_logprobs_bytes(rows, V, n_top), workspace, dev, "op_logprobs: workspace")
    at = buf.data_ptr()
    at_ranks = at + 4 * (2 * rows + m)
    _call(dev, "op_logprobs", L.lede_op_logprobs, _dtype_code(torch, logits.dtype), logits.data_ptr(),
          ld if rows > 1 else max(ld, V), rows, V, temperature, tokens.data_ptr() if given else None, n_top,
          at if given else None, at_ranks if given else None, at + 4 * rows, at_ranks + 4 * rows, at + 8 * rows, ws_at, ws_bytes)
    return Logprobs(logprobs.view(f32) if given else None, ranks if given else None, entropy.view(f32), ids.view(rows, n_top),
                    top.view(f32).view(rows, n_top))


# ---- linear products with 4-bit weights ---------------------------------------------

def _matrix_stride(x, what: str) -> int:
    """Elements between the rows of x [rows][columns], whose columns are dense."""
    rows, cols = x.shape
    r, c = x.stride()
    _need(c == 1 or cols == 1, what)
    return r if rows > 1 else max(r, cols)


def op_quantize(w, group: int = 64):
    """(codes, scales) of weights w [N][K] (float32 or bfloat16, any row
    stride): e2m1 codes, two a byte, uint8 [N][ceil(K / 2)], and a bfloat16
    scale for every `group` (32, 64 or 128) columns, [N][ceil(K / group)]."""
    import torch
    _need(w.dim() == 2, "op_quantize")
    (N, K), dev = w.shape, w.device
    ld = _matrix_stride(w, "op_quantize")
    _int32(N | K | group, "op_quantize")
    if load().lede_op_quant_bytes(N, K, group) == 0:
        raise LedeError(LEDE_E_UNSUPPORTED, "op_quantize: %d x %d, group %d" % (N, K, group))
    codes = torch.empty(N, (K + 1) // 2, dtype=torch.uint8, device=dev)
    scales = torch.empty(N, -(-K // group), dtype=torch.bfloat16, device=dev)
    _call(dev, "op_quantize", load().lede_op_quantize, _dtype_code(torch, w.dtype), w.data_ptr(), ld, N, K, group, codes.data_ptr(),
          scales.data_ptr())
    return codes, scales


class QuantMatrix:
    """A matrix [N][K] of 4-bit weights, packed for op_quant_linear from codes
    and scales as op_quantize gives them (which may go afterwards)."""

    def __init__(self, codes, scales, K: int, group: int):
        import torch
        N, dev = codes.shape[0], codes.device
        _int32(N | K | group, "QuantMatrix")
        nbytes = load().lede_op_quant_bytes(N, K, group)
        if nbytes == 0:
            raise LedeError(LEDE_E_UNSUPPORTED, "4-bit matrix of %d x %d, group %d" % (N, K, group))
        _need(_dense(dev, torch.uint8, codes) and _dense(dev, torch.bfloat16, scales) and codes.shape == (N, (K + 1) // 2)
              and scales.shape == (N, -(-K // group)), "QuantMatrix")
        self.packed = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        self.N, self.K, self.group, self.device = N, K, group, dev
        _call(dev, "QuantMatrix", load().lede_op_quant_pack, codes.data_ptr(), scales.data_ptr(), N, K, group, self.packed.data_ptr())


def op_quant_linear(matrix: QuantMatrix, x, dtype=None, out=None):
    """x W^T for rows x [M][K] (float32 or bfloat16, any row stride) and a
    matrix of 4-bit weights: [M][N] of `dtype` (x's when not given); `out`
    gives the tensor, of any row stride."""
    import torch
    dev, N, K = matrix.device, matrix.N, matrix.K
    _need(x.dim() == 2 and x.shape[1] == K and x.device == dev, "op_quant_linear")
    M, ldx = x.shape[0], _matrix_stride(x, "op_quant_linear: x")
    _int32(M, "op_quant_linear")
    if out is None:
        out = torch.empty(M, N, dtype=dtype or x.dtype, device=dev)
        ldy = N
    else:
        _need(out.shape == (M, N) and out.device == dev and (dtype is None or out.dtype == dtype), "op_quant_linear: out")
        ldy = _matrix_stride(out, "op_quant_linear: out")
    _call(dev, "op_quant_linear", load().lede_op_quant_linear, _dtype_code(torch, x.dtype), matrix.packed.data_ptr(), N, K, matrix.group,
          x.data_ptr(), ldx, M, _dtype_code(torch, out.dtype), out.data_ptr(), ldy)
    return out


# ---- the vocabulary head's loss, without the logits -----------------------------------

@dataclass
class HeadLoss:
    loss: object   # float32 [rows]; 0 where the target lies outside the vocabulary
    lse: object    # float32 [rows]


def _head_inputs(torch, hidden, head, targets, what: str):
    dev = hidden.device
    _need(hidden.dim() == 2 and head.dim() == 2 and hidden.shape[1] == head.shape[1] and head.device == dev and head.dtype == hidden.dtype
          and _dense(dev, torch.int32, targets) and targets.numel() == hidden.shape[0], what)
    _int32(hidden.shape[0] | hidden.shape[1] | head.shape[0], what)
    return (_dtype_code(torch, hidden.dtype), hidden.shape[0], head.shape[0], hidden.shape[1], _matrix_stride(hidden, what),
            _matrix_stride(head, what))


def _head_supported(nbytes: int, M: int, V: int, K: int, what: str):
    if nbytes == 0 and M > 0:
        raise LedeError(LEDE_E_UNSUPPORTED, "%s: %d rows, %d x %d" % (what, M, V, K))


def op_head_loss(hidden, head, targets, workspace=None) -> HeadLoss:
    """-log softmax(hidden head^T)[target] of every row of hidden [M][K], and
    its log of the sum, without the logits; head [V][K] of the same dtype
    (float32 or bfloat16), targets int32 [M] (outside [0, V): the row is left
    out).  Rows lie at multiples of 16 bytes; K is a multiple of 8."""
    import torch
    dev = hidden.device
    code, M, V, K, ldh, ldw = _head_inputs(torch, hidden, head, targets, "op_head_loss")
    L = load()
    need = L.lede_op_head_loss_bytes(code, M, V, K)
    _head_supported(need, M, V, K, "op_head_loss")
    loss, lse = torch.empty(2, M, dtype=torch.float32, device=dev).unbind(0)
    ws, ws_at, ws_bytes = _workspace(torch, need, workspace, dev, "op_head_loss: workspace")
    _call(dev, "op_head_loss", L.lede_op_head_loss, code, hidden.data_ptr(), ldh, M, head.data_ptr(), ldw, V, K, targets.data_ptr(),
          loss.data_ptr(), lse.data_ptr(), ws_at, ws_bytes)
    return HeadLoss(loss, lse)


def op_head_loss_grad(hidden, head, targets, lse, weights=None, want_hidden: bool = True, want_head: bool = True, out=None,
                      workspace=None):
    """(d_hidden, d_head): the gradient of sum(weights * loss) (float32 [M],
    all 1 when not given) with the lse of op_head_loss; None for one that is
    not wanted.  `out` gives the two tensors (or None in a place)."""
    import torch
    dev = hidden.device
    code, M, V, K, ldh, ldw = _head_inputs(torch, hidden, head, targets, "op_head_loss_grad")
    _need(_dense(dev, torch.float32, lse) and lse.numel() == M
          and (weights is None or (_dense(dev, torch.float32, weights) and weights.numel() == M)), "op_head_loss_grad")
    L = load()
    need = L.lede_op_head_loss_grad_bytes(code, M, V, K)
    _head_supported(need, M, V, K, "op_head_loss_grad")
    if out is None:
        out = (torch.empty(M, K, dtype=hidden.dtype, device=dev) if want_hidden else None,
               torch.empty(V, K, dtype=hidden.dtype, device=dev) if want_head else None)
    dh, dw = out
    for t, n in ((dh, M), (dw, V)):
        _need(t is None or (t.shape == (n, K) and t.dtype == hidden.dtype and t.device == dev), "op_head_loss_grad: out")
    ws, ws_at, ws_bytes = _workspace(torch, need, workspace, dev, "op_head_loss_grad: workspace")
    _call(dev, "op_head_loss_grad", L.lede_op_head_loss_grad, code, hidden.data_ptr(), ldh, M, head.data_ptr(), ldw, V, K,
          targets.data_ptr(), lse.data_ptr(), None if weights is None else weights.data_ptr(),
          None if dh is None else dh.data_ptr(), 0 if dh is None else _matrix_stride(dh, "op_head_loss_grad: out"),
          None if dw is None else dw.data_ptr(), 0 if dw is None else _matrix_stride(dw, "op_head_loss_grad: out"), ws_at, ws_bytes)
    return dh, dw


def dqn_noise_count(hidden: int) -> int:
    """Standard normals one network draw takes: eps_in, eps_out of both layers."""
    return 2 * hidden + 5


def dqn_param_count(hidden: int) -> int:
    """Entries of [mu, sigma] of the 3 -> H -> 2 network."""
    return 2 * (6 * hidden + 2)


class Dqn:
    """A liblede policy trainer (lede_dqn_*) over a torch-allocated region."""

    def __init__(self, hidden: int = 16, capacity: int = 1 << 16, batch: int = 32, n_step: int = 3,
                 gamma: float = 0.99, lr: float = 6.25e-5, beta1: float = 0.9, beta2: float = 0.999,
                 adam_eps: float = 1.5e-4, sigma0: float = 0.1, device: int = 0):
        import torch
        self.torch = torch
        self.L = load()
        self.cfg = LedeDqnConfig(hidden, capacity, batch, n_step, gamma, lr, beta1, beta2, adam_eps, sigma0)
        nbytes = self.L.lede_dqn_region_bytes(ctypes.byref(self.cfg))
        if nbytes == 0:
            raise LedeError(LEDE_E_ARG, "invalid trainer configuration")
        self.device = torch.device("cuda", device)
        self.region = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        rc = self.L.lede_dqn_create(ctypes.byref(self.cfg), self.region.data_ptr(), nbytes, ctypes.byref(h))
        if rc != LEDE_OK:
            raise LedeError(rc, "lede_dqn_create")
        self.q = h

    @property
    def stream(self):
        return ctypes.c_void_p(self.torch.cuda.current_stream(self.device).cuda_stream)

    def _check(self, rc: int):
        if rc != LEDE_OK:
            raise LedeError(rc, self.L.lede_dqn_last_error(self.q).decode())

    def _dev(self, a):
        """A device fp32 copy of a host array (kept alive by the caller)."""
        return self.torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(self.device)

    def close(self):
        if getattr(self, "q", None):
            self.L.lede_dqn_destroy(self.q)
            self.q = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def lede_dqn_init(self, u):
        d = self._dev(u)
        self._check(self.L.lede_dqn_init(self.q, d.data_ptr(), self.stream))
        self.torch.cuda.current_stream(self.device).synchronize()

    def lede_dqn_push(self, transitions):
        t = np.ascontiguousarray(transitions, dtype=np.float32).reshape(-1, 6)
        d = self._dev(t)
        self._check(self.L.lede_dqn_push(self.q, d.data_ptr(), len(t), self.stream))
        self.torch.cuda.current_stream(self.device).synchronize()

    def lede_dqn_record(self, engine, episode_end: bool = False):
        self._check(self.L.lede_dqn_record(self.q, engine.ctx, int(episode_end), self.stream))

    def lede_dqn_end_episode(self):
        self._check(self.L.lede_dqn_end_episode(self.q, self.stream))

    def lede_dqn_update(self, u, noise, want_loss: bool = True):
        """u: [batch] uniforms m / 2^24, noise: [2][2H + 5] normals, host
        arrays or device tensors; returns the loss (or None)."""
        t = self.torch
        ud = u if isinstance(u, t.Tensor) else self._dev(u)
        nd = noise if isinstance(noise, t.Tensor) else self._dev(noise)
        loss = ctypes.c_float()
        self._check(self.L.lede_dqn_update(self.q, ud.data_ptr(), nd.data_ptr(), self.stream,
                                           ctypes.byref(loss) if want_loss else None))
        return loss.value if want_loss else None

    def lede_dqn_sync_target(self):
        self._check(self.L.lede_dqn_sync_target(self.q, self.stream))

    def lede_dqn_act(self, engine, noise=None):
        nd = None if noise is None else self._dev(noise)
        self._check(self.L.lede_dqn_act(self.q, engine.ctx, None if nd is None else nd.data_ptr(), self.stream))
        self.torch.cuda.current_stream(self.device).synchronize()

    def lede_dqn_read(self, which: int) -> np.ndarray:
        """0 online [mu, sigma], 1 target, 2 Adam m, 3 Adam v; 4 transitions [count][6]."""
        cap = dqn_param_count(self.cfg.hidden) if which < 4 else self.cfg.capacity * 6
        out = np.zeros(cap, dtype=np.float32)
        n = ctypes.c_int32()
        self._check(self.L.lede_dqn_read(self.q, which, out.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), cap,
                                         ctypes.byref(n), self.stream))
        return out[:n.value] if which < 4 else out[:n.value * 6].reshape(n.value, 6)
