"""Thin ctypes binding of ``libatspeed.so`` (the C ABI in include/atspeed.h).

Argument marshalling only: every step of the verification call runs in the CUDA library.  PyTorch
supplies device memory (weights, inputs, outputs) and the CUDA stream.  There is no CPU fallback:
if the library is missing or fails to load, every entry point raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "_build", "libatspeed.so")

OK, E_ARG, E_SHAPE, E_OOM, E_CUDA, E_TIMEOUT, E_STATE, E_UNSUPPORTED = 0, -1, -2, -3, -4, -5, -6, -7
STRICT, RELAXED = 0, 1
NORM_MASKED, NORM_FULL = 0, 1
PLAIN_TOPK, PLAIN_SAMPLE, SD_STRICT, SD_RELAXED = 0, 1, 2, 3
PLAN_OK, PLAN_NO_PAGES, PLAN_LIMIT = 0, 1, 2
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

EXPORTS = [
    "atspeed_create", "atspeed_destroy", "atspeed_last_error", "atspeed_prefill", "atspeed_begin_step",
    "atspeed_draft_step", "atspeed_verify", "atspeed_draft_step_logits", "atspeed_verify_logits",
    "atspeed_beam_search", "atspeed_set_early_reject", "atspeed_profile", "atspeed_profile_read", "atspeed_tree_shape", "atspeed_debug_tree",
    "atspeed_debug_node_logits", "atspeed_debug_node_lse", "atspeed_debug_buffer", "atspeed_set_tree", "atspeed_op_workspace_bytes", "atspeed_op_gemm",
    "atspeed_op_gemm_noalloc", "atspeed_op_status", "atspeed_op_gemm_swiglu", "atspeed_op_rmsnorm", "atspeed_op_attention_scratch", "atspeed_op_attention",
    "atspeed_op_batch_plan", "atspeed_op_rope_append", "atspeed_op_tree_attention_workspace", "atspeed_op_tree_attention",
    "atspeed_op_adjust_logits", "atspeed_op_capture_id", "atspeed_op_beam_select_workspace", "atspeed_op_beam_select",
    "atspeed_op_fork_pages", "atspeed_op_copy_pages", "atspeed_op_compact_tokens",
]


class AtSpeedError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"atspeed status {status}: {msg}")
        self.status = status


class ModelDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int), ("d_model", ctypes.c_int), ("n_heads", ctypes.c_int),
                ("d_ffn", ctypes.c_int), ("vocab", ctypes.c_int), ("rms_eps", ctypes.c_float),
                ("rope_theta", ctypes.c_float), ("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("lm_head", ctypes.c_void_p), ("attn_norm", ctypes.POINTER(ctypes.c_void_p)),
                ("wqkv", ctypes.POINTER(ctypes.c_void_p)), ("wo", ctypes.POINTER(ctypes.c_void_p)),
                ("mlp_norm", ctypes.POINTER(ctypes.c_void_p)), ("wgate_up", ctypes.POINTER(ctypes.c_void_p)),
                ("wdown", ctypes.POINTER(ctypes.c_void_p))]


class ItemsDesc(ctypes.Structure):
    _fields_ = [("n_items", ctypes.c_int), ("L", ctypes.c_int), ("codes_per_level", ctypes.c_int),
                ("code_base", ctypes.c_int), ("h_codes", ctypes.POINTER(ctypes.c_int32))]


class Limits(ctypes.Structure):
    _fields_ = [("max_users", ctypes.c_int), ("max_prompt", ctypes.c_int), ("max_K", ctypes.c_int),
                ("max_N", ctypes.c_int), ("max_gamma", ctypes.c_int)]


class DecodeOpts(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int), ("N", ctypes.c_int), ("gamma", ctypes.c_int), ("norm", ctypes.c_int),
                ("philox_seed", ctypes.c_uint64)]


class KvPages(ctypes.Structure):
    _fields_ = [("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("k_type", ctypes.c_int), ("v_type", ctypes.c_int),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("n_kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3)]


_KV_PACK = struct.Struct("@PPiiiiiiqqqqqq").pack
assert struct.calcsize("@PPiiiiiiqqqqqq") == ctypes.sizeof(KvPages)


class LogitRulesDesc(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int)] + [(f, ctypes.c_void_p) for f in (
        "d_hist", "d_hist_off", "d_prompt_len", "d_repetition", "d_frequency", "d_presence", "d_temperature", "d_bias_off",
        "d_bias_tok", "d_bias_val", "d_grammar")] + [("grammar_stride", ctypes.c_int64), ("n_states", ctypes.c_int),
                                                     ("d_tree_tok", ctypes.c_void_p), ("d_cu_q", ctypes.c_void_p)]


class BeamsDesc(ctypes.Structure):
    _fields_ = [("d_logits", ctypes.c_void_p), ("ld", ctypes.c_int64), ("type", ctypes.c_int), ("R", ctypes.c_int), ("vocab", ctypes.c_int),
                ("n_req", ctypes.c_int), ("width", ctypes.c_int), ("norm", ctypes.c_int), ("d_cu_beam", ctypes.c_void_p),
                ("d_score", ctypes.c_void_p), ("d_final", ctypes.c_void_p), ("d_state", ctypes.c_void_p), ("d_grammar", ctypes.c_void_p),
                ("grammar_stride", ctypes.c_int64), ("n_states", ctypes.c_int), ("d_token", ctypes.c_void_p),
                ("d_parent", ctypes.c_void_p), ("d_out_score", ctypes.c_void_p)]


class PageForkDesc(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int) for f in ("n_old", "n_new", "table_width", "page_size", "n_pages", "free_size")] + [(f, ctypes.c_void_p) for f in (
        "d_table", "d_kv_len", "d_q_len", "d_old_state", "d_parent", "d_length", "d_ref", "d_free", "d_n_free", "d_used", "d_new_table",
        "d_new_len", "d_new_state", "d_src", "d_dst", "d_new_ref", "d_new_free", "d_new_n_free")]


# (packed whole and passed by address: as arguments of their own the fields of a fork take 2 us more)
_BEAMS_PACK, _FORK_PACK = struct.Struct("@PqiiiiiiPPPPPqiPPP").pack, struct.Struct("@iiiiii18P").pack
assert struct.calcsize("@PqiiiiiiPPPPPqiPPP") == ctypes.sizeof(BeamsDesc) and struct.calcsize("@iiiiii18P") == ctypes.sizeof(PageForkDesc)

_lib: Optional[ctypes.CDLL] = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads the CUDA library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libatspeed.so not built ({path}); run __graft_entry__.build() first")
    lib = ctypes.CDLL(path)
    vp, i32p, fp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float)
    c_int = ctypes.c_int
    sig = {
        "atspeed_create": (c_int, [ctypes.POINTER(ModelDesc), ctypes.POINTER(ModelDesc), ctypes.POINTER(ItemsDesc),
                                   ctypes.POINTER(Limits), ctypes.POINTER(vp)]),
        "atspeed_destroy": (None, [vp]),
        "atspeed_last_error": (ctypes.c_char_p, [vp]),
        "atspeed_prefill": (c_int, [vp, vp, c_int, vp, i32p]),
        "atspeed_begin_step": (c_int, [vp, vp, ctypes.POINTER(DecodeOpts)]),
        "atspeed_draft_step": (c_int, [vp, vp, ctypes.POINTER(DecodeOpts), c_int]),
        "atspeed_verify": (c_int, [vp, vp, ctypes.POINTER(DecodeOpts), c_int, vp, vp, vp, vp]),
        "atspeed_draft_step_logits": (c_int, [vp, vp, ctypes.POINTER(DecodeOpts), c_int, fp]),
        "atspeed_verify_logits": (c_int, [vp, vp, ctypes.POINTER(DecodeOpts), c_int, fp, vp, vp, vp, vp]),
        "atspeed_beam_search": (c_int, [vp, vp, c_int, vp, i32p, ctypes.POINTER(DecodeOpts), c_int, vp, vp, i32p]),
        "atspeed_set_early_reject": (c_int, [vp, c_int]),
        "atspeed_profile": (c_int, [vp, c_int]),
        "atspeed_profile_read": (c_int, [vp, c_int, i32p, ctypes.POINTER(ctypes.c_double),
                                         ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]),
        "atspeed_tree_shape": (c_int, [vp, i32p, i32p, i32p, i32p]),
        "atspeed_debug_tree": (c_int, [vp, i32p, fp, fp, i32p]),
        "atspeed_debug_node_logits": (c_int, [vp, c_int, c_int, c_int, fp]),
        "atspeed_debug_node_lse": (c_int, [vp, c_int, c_int, c_int, fp]),
        "atspeed_debug_buffer": (c_int, [vp, c_int, c_int, vp, ctypes.c_size_t]),
        "atspeed_set_tree": (c_int, [vp, vp, c_int, i32p, i32p, i32p, fp, fp]),
        "atspeed_op_workspace_bytes": (ctypes.c_size_t, []),
        "atspeed_op_gemm": (c_int, [vp, vp, vp, c_int, c_int, c_int, c_int, vp, c_int, c_int, vp]),
        "atspeed_op_gemm_noalloc": (c_int, [vp, vp, vp, c_int, c_int, c_int, c_int, vp, c_int, c_int]),
        "atspeed_op_gemm_swiglu": (c_int, [vp, vp, vp, c_int, c_int, c_int, c_int, vp, c_int, vp]),
        "atspeed_op_status": (c_int, [vp, vp]),
        "atspeed_op_rmsnorm": (c_int, [vp, vp, vp, c_int, c_int, ctypes.c_float, vp, c_int]),
        "atspeed_op_attention_scratch": (ctypes.c_size_t, [c_int, c_int, c_int, c_int]),
        "atspeed_op_attention": (c_int, [vp, vp, vp, vp, c_int, c_int, c_int, c_int, c_int, i32p, i32p, i32p, i32p,
                                         vp, vp]),
        "atspeed_op_batch_plan": (c_int, [vp, c_int, vp, vp, vp, c_int, vp, c_int, vp, vp, c_int, c_int, vp, vp, vp, vp,
                                          vp, vp, vp, vp]),
        "atspeed_op_rope_append": (c_int, [vp, vp, c_int, ctypes.c_int64, c_int, c_int, ctypes.POINTER(KvPages), vp, vp,
                                           ctypes.c_float, vp, ctypes.c_int64]),
        "atspeed_op_tree_attention_workspace": (ctypes.c_size_t, []),
        "atspeed_op_tree_attention": (c_int, [vp, ctypes.POINTER(KvPages), vp, ctypes.c_int64, c_int, c_int, c_int, vp, vp,
                                              vp, c_int, vp, c_int, ctypes.c_float, vp, ctypes.c_int64, vp, vp]),
        "atspeed_op_capture_id": (ctypes.c_uint64, [vp]),
        "atspeed_op_adjust_logits": (c_int, [vp, vp, c_int, ctypes.c_int64, c_int, c_int, vp,
                                             ctypes.POINTER(LogitRulesDesc), vp, c_int, vp, vp, c_int, ctypes.c_int64]),
        "atspeed_op_beam_select_workspace": (ctypes.c_size_t, [c_int, c_int, c_int]),
        "atspeed_op_beam_select": (c_int, [vp, ctypes.c_char_p, vp]),   # (an atspeed_beams and an atspeed_page_fork as bytes)
        "atspeed_op_fork_pages": (c_int, [vp, ctypes.c_char_p]),
        "atspeed_op_copy_pages": (c_int, [vp, ctypes.POINTER(KvPages), c_int, c_int, vp, vp, vp]),
        "atspeed_op_compact_tokens": (c_int, [vp, ctypes.POINTER(KvPages), c_int, c_int, c_int, vp, vp, vp, vp, vp, c_int, vp, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _i32(a) -> ctypes.Array:
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _check(status: int, ctx=None):
    if status != OK:
        lib = load()
        msg = lib.atspeed_last_error(ctx)
        raise AtSpeedError(status, msg.decode() if msg else "")


def weights_to_device(weights: Dict[str, np.ndarray], device="cuda") -> Dict[str, torch.Tensor]:
    """float32 arrays holding bf16 values -> bf16 device tensors (exact)."""
    return {k: torch.from_numpy(np.ascontiguousarray(v)).to(device=device, dtype=torch.bfloat16)
            for k, v in weights.items()}


def _model_desc(spec, w: Dict[str, torch.Tensor]):
    L = spec.n_layers
    arrs = {}
    for key in ("attn_norm", "wqkv", "wo", "mlp_norm", "wgate_up", "wdown"):
        ptrs = [w[f"layers.{l}.{key}"].data_ptr() for l in range(L)]
        arrs[key] = (ctypes.c_void_p * L)(*ptrs)
    d = ModelDesc(spec.n_layers, spec.d_model, spec.n_heads, spec.d_ffn, spec.vocab, spec.rms_eps, spec.rope_theta,
                  w["embed"].data_ptr(), w["final_norm"].data_ptr(), w["lm_head"].data_ptr(),
                  arrs["attn_norm"], arrs["wqkv"], arrs["wo"], arrs["mlp_norm"], arrs["wgate_up"], arrs["wdown"])
    return d, arrs


def opts(K: int, N: int, gamma: int, seed: int = 0, norm: int = NORM_MASKED) -> DecodeOpts:
    return DecodeOpts(K, N, gamma, norm, seed)


class Context:
    """One atspeed_ctx: borrowed device weights, the item trie and every device buffer."""

    def __init__(self, target_spec, target_w: Dict[str, torch.Tensor], draft_spec, draft_w,
                 items: np.ndarray, code_base: int, max_users: int, max_prompt: int, max_K: int, max_N: int,
                 max_gamma: int):
        lib = load()
        self._lib = lib
        self._keep = [target_w, draft_w]
        td, ta = _model_desc(target_spec, target_w)
        self._keep += [td, ta]
        dd = None
        if draft_spec is not None:
            dd, da = _model_desc(draft_spec, draft_w)
            self._keep += [dd, da]
        it = np.ascontiguousarray(items, dtype=np.int32)
        self._keep.append(it)
        idesc = ItemsDesc(it.shape[0], it.shape[1], 256, code_base, it.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
        lim = Limits(max_users, max_prompt, max_K, max_N, max_gamma)
        self.max_N = max_N
        out = ctypes.c_void_p()
        st = lib.atspeed_create(ctypes.byref(td), ctypes.byref(dd) if dd is not None else None, ctypes.byref(idesc),
                                ctypes.byref(lim), ctypes.byref(out))
        _check(st, None)
        self.ptr = out.value
        self.n_users = 0

    def close(self):
        if getattr(self, "ptr", None):
            self._lib.atspeed_destroy(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- calls -----------------------------------------------------------------------------------
    def prefill(self, tokens: torch.Tensor, offsets: Sequence[int], stream=None):
        off, offp = _i32(offsets)
        self.n_users = len(offsets) - 1
        _check(self._lib.atspeed_prefill(self.ptr, _stream(stream), self.n_users, tokens.data_ptr(), offp), self.ptr)

    def begin_step(self, o: DecodeOpts, stream=None):
        _check(self._lib.atspeed_begin_step(self.ptr, _stream(stream), ctypes.byref(o)), self.ptr)

    def draft_step(self, o: DecodeOpts, mode: int, stream=None):
        _check(self._lib.atspeed_draft_step(self.ptr, _stream(stream), ctypes.byref(o), mode), self.ptr)

    def verify(self, o: DecodeOpts, mode: int, stream=None):
        B, K = self.n_users, o.K
        dev = torch.device("cuda")
        acc = torch.empty(B, dtype=torch.int32, device=dev)
        depth = torch.empty(B, dtype=torch.int32, device=dev)
        beams = torch.empty(B, K, 4, dtype=torch.int32, device=dev)
        scores = torch.empty(B, K, dtype=torch.float32, device=dev)
        _check(self._lib.atspeed_verify(self.ptr, _stream(stream), ctypes.byref(o), mode, acc.data_ptr(),
                                        depth.data_ptr(), beams.data_ptr(), scores.data_ptr()), self.ptr)
        return acc, depth, beams, scores

    def draft_step_logits(self, o: DecodeOpts, mode: int, logits: np.ndarray, stream=None):
        """logits [n_users][width][1024]: draft item-code logits of the previous level's slots."""
        lg = np.ascontiguousarray(logits, np.float32)
        _check(self._lib.atspeed_draft_step_logits(self.ptr, _stream(stream), ctypes.byref(o), mode,
                                                   lg.ctypes.data_as(ctypes.POINTER(ctypes.c_float))), self.ptr)

    def verify_logits(self, o: DecodeOpts, mode: int, logits: np.ndarray, stream=None):
        """logits [n_users][K + gamma*N][1024]: target item-code logits of every node slot."""
        B, K = self.n_users, o.K
        dev = torch.device("cuda")
        acc = torch.empty(B, dtype=torch.int32, device=dev)
        depth = torch.empty(B, dtype=torch.int32, device=dev)
        beams = torch.empty(B, K, 4, dtype=torch.int32, device=dev)
        scores = torch.empty(B, K, dtype=torch.float32, device=dev)
        lg = np.ascontiguousarray(logits, np.float32)
        _check(self._lib.atspeed_verify_logits(self.ptr, _stream(stream), ctypes.byref(o), mode,
                                               lg.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), acc.data_ptr(),
                                               depth.data_ptr(), beams.data_ptr(), scores.data_ptr()), self.ptr)
        return acc, depth, beams, scores

    def beam_search(self, tokens: torch.Tensor, offsets: Sequence[int], o: DecodeOpts, mode: int, stream=None,
                    items_out: Optional[torch.Tensor] = None, scores_out: Optional[torch.Tensor] = None):
        B = len(offsets) - 1
        self.n_users = B
        dev = torch.device("cuda")
        items = items_out if items_out is not None else torch.empty(B, o.K, 4, dtype=torch.int32, device=dev)
        scores = scores_out if scores_out is not None else torch.empty(B, o.K, dtype=torch.float32, device=dev)
        stats = np.zeros((B, 3), dtype=np.int32)
        off, offp = _i32(offsets)
        _check(self._lib.atspeed_beam_search(self.ptr, _stream(stream), B, tokens.data_ptr(), offp, ctypes.byref(o),
                                             mode, items.data_ptr(), scores.data_ptr(),
                                             stats.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))), self.ptr)
        return items, scores, stats

    def set_early_reject(self, enable: bool):
        _check(self._lib.atspeed_set_early_reject(self.ptr, 1 if enable else 0), self.ptr)

    def profile(self, enable: bool):
        _check(self._lib.atspeed_profile(self.ptr, 1 if enable else 0), self.ptr)

    def profile_read(self, kind: int):
        n = ctypes.c_int32()
        ms, by, fl = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
        _check(self._lib.atspeed_profile_read(self.ptr, kind, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(by),
                                              ctypes.byref(fl)), self.ptr)
        return {"launches": n.value, "ms": ms.value, "bytes": by.value, "flops": fl.value}

    # -- introspection -----------------------------------------------------------------------------
    def tree_shape(self):
        B = self.n_users
        depth = np.zeros(B, np.int32)
        levels = np.zeros(B, np.int32)
        si = np.zeros(1, np.int32)
        sl = np.zeros(1, np.int32)
        p = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        _check(self._lib.atspeed_tree_shape(self.ptr, p(depth), p(levels), p(si), p(sl)), self.ptr)
        return depth, levels, int(si[0]), int(sl[0])

    def debug_tree(self, gamma: int):
        depth, levels, si, sl = self.tree_shape()
        B = self.n_users
        stride = si + gamma * sl
        path = np.zeros((B, stride, 4), np.int32)
        sq = np.zeros((B, stride), np.float32)
        sp = np.zeros((B, stride), np.float32)
        cnt = np.zeros((B, gamma + 1), np.int32)
        _check(self._lib.atspeed_debug_tree(self.ptr, path.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                            sq.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                            sp.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                            cnt.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))), self.ptr)
        return {"path": path, "sq": sq, "sp": sp, "count": cnt, "slots_in": si, "slots_lvl": sl, "depth": depth,
                "levels": levels}

    def debug_buffer(self, which: int, buf: int, dtype, count: int) -> np.ndarray:
        out = np.zeros(count, dtype=dtype)
        _check(self._lib.atspeed_debug_buffer(self.ptr, which, buf, out.ctypes.data, out.nbytes), self.ptr)
        return out

    def node_logits(self, which: int, user: int, slot: int) -> np.ndarray:
        out = np.zeros(1024, np.float32)
        _check(self._lib.atspeed_debug_node_logits(self.ptr, which, user, slot,
                                                   out.ctypes.data_as(ctypes.POINTER(ctypes.c_float))), self.ptr)
        return out

    def node_lse(self, which: int, user: int, slot: int) -> float:
        out = np.zeros(1, np.float32)
        _check(self._lib.atspeed_debug_node_lse(self.ptr, which, user, slot,
                                                out.ctypes.data_as(ctypes.POINTER(ctypes.c_float))), self.ptr)
        return float(out[0])

    def set_tree(self, counts: np.ndarray, parents: np.ndarray, codes: np.ndarray, sq: np.ndarray,
                 draft_logits: Optional[np.ndarray] = None, stream=None):
        """counts [B][n_levels]; parents/codes/sq [B][n_levels][max_N]; draft_logits
        [B][n_levels][max_N][1024] (logits of the parents on levels 0 .. n_levels-1) or None."""
        n_levels = counts.shape[1]
        c, cp = _i32(counts)
        p, pp = _i32(parents)
        k, kp = _i32(codes)
        s = np.ascontiguousarray(sq, np.float32)
        dl = None if draft_logits is None else np.ascontiguousarray(draft_logits, np.float32)
        _check(self._lib.atspeed_set_tree(self.ptr, _stream(stream), n_levels, cp, pp, kp,
                                          s.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                          None if dl is None else dl.ctypes.data_as(ctypes.POINTER(ctypes.c_float))),
               self.ptr)


# ---------------------------------------------------------------------------------------------------
# stateless operators
# ---------------------------------------------------------------------------------------------------
_ws: Dict[int, torch.Tensor] = {}


def op_workspace(device: int = 0) -> torch.Tensor:
    if device not in _ws:
        n = load().atspeed_op_workspace_bytes()
        _ws[device] = torch.zeros(n, dtype=torch.uint8, device=f"cuda:{device}")
    return _ws[device]


def op_gemm(W: torch.Tensor, X: torch.Tensor, T: int, Y: Optional[torch.Tensor] = None, accumulate=False,
            stream=None) -> torch.Tensor:
    M, K = W.shape
    if Y is None:   # (every value is written unless it is added to)
        Y = (torch.zeros if accumulate else torch.empty)(T, M, dtype=torch.float32, device=W.device)
    _check(load().atspeed_op_gemm(_stream(stream), W.data_ptr(), X.data_ptr(), M, K, T, X.shape[0], Y.data_ptr(),
                                  Y.shape[1], 1 if accumulate else 0, op_workspace().data_ptr()))
    return Y


def op_gemm_noalloc(W: torch.Tensor, X: torch.Tensor, T: int, Y: Optional[torch.Tensor] = None, accumulate=False,
                    stream=None) -> torch.Tensor:
    """atspeed_op_gemm without a workspace argument (the library's fixed scratch array is used)."""
    M, K = W.shape
    if Y is None:   # (every value is written unless it is added to)
        Y = (torch.zeros if accumulate else torch.empty)(T, M, dtype=torch.float32, device=W.device)
    _check(load().atspeed_op_gemm_noalloc(_stream(stream), W.data_ptr(), X.data_ptr(), M, K, T, X.shape[0],
                                          Y.data_ptr(), Y.shape[1], 1 if accumulate else 0))
    return Y


def op_status(noalloc: bool = False, stream=None) -> int:
    """atspeed_op_status: synchronises, reads and clears the device error word of the op GEMMs'
    workspace (noalloc: those of the allocation-free scratch and of the attention); returns the status
    code (0 = no device error)."""
    ws = None if noalloc else op_workspace().data_ptr()
    status = int(load().atspeed_op_status(_stream(stream), ws))
    if noalloc and status != 0:   # a call that gave up leaves its counters as they are
        for device in {d for d, _ in _tree_ws}:   # (from here, not from their streams: some may be gone)
            torch.cuda.synchronize(device)
        for w in _tree_ws.values():
            w[:TREE_ATTENTION_COUNTER_BYTES].zero_()
        for device in {d for d, _ in _tree_ws}:
            torch.cuda.synchronize(device)
    return status


def op_gemm_swiglu(W: torch.Tensor, X: torch.Tensor, T: int, stream=None) -> torch.Tensor:
    F2, K = W.shape
    out = torch.empty(T, F2 // 2, dtype=torch.bfloat16, device=W.device)
    _check(load().atspeed_op_gemm_swiglu(_stream(stream), W.data_ptr(), X.data_ptr(), F2 // 2, K, T, X.shape[0],
                                         out.data_ptr(), out.shape[1], op_workspace().data_ptr()))
    return out


def op_rmsnorm(h: torch.Tensor, g: torch.Tensor, eps: float, stream=None) -> torch.Tensor:
    T, d = h.shape
    x = torch.empty(T, d, dtype=torch.bfloat16, device=h.device)
    _check(load().atspeed_op_rmsnorm(_stream(stream), h.data_ptr(), g.data_ptr(), T, d, eps, x.data_ptr(), d))
    return x


def op_attention(q: torch.Tensor, kc: torch.Tensor, vc: torch.Tensor, n_heads: int, head_dim: int, P: int,
                 pages: Sequence[int], vis: Sequence[int], path_rows: Optional[np.ndarray] = None,
                 n_path: Optional[Sequence[int]] = None, stream=None) -> torch.Tensor:
    lib = load()
    T = q.shape[0]
    out = torch.empty(T, n_heads * head_dim, dtype=torch.bfloat16, device=q.device)
    scratch = torch.empty(lib.atspeed_op_attention_scratch(T, n_heads, head_dim, P), dtype=torch.uint8,
                          device=q.device)
    pg, pgp = _i32(pages if len(pages) else [0])
    vv, vvp = _i32(vis)
    pr = prp = npth = npp = None   # (no counts: no path keys, and nothing to pass)
    if n_path is not None:
        pr, prp = _i32(np.zeros((T, 4), np.int32) if path_rows is None else path_rows)
        npth, npp = _i32(n_path)
    _check(lib.atspeed_op_attention(_stream(stream), q.data_ptr(), kc.data_ptr(), vc.data_ptr(), kc.shape[0], T,
                                    n_heads, head_dim, P, pgp, vvp, prp, npp, out.data_ptr(), scratch.data_ptr()))
    return out


# ---------------------------------------------------------------------------------------------------
# a serving step over a batch of requests: plan, cache append, tree attention, logit rules
# ---------------------------------------------------------------------------------------------------
def _refuse(what: str):
    """Arguments that the C ABI cannot see (types, shapes, devices) are refused as it refuses its own."""
    raise AtSpeedError(E_ARG, what)


def _gpu(t: torch.Tensor, stream: Optional[torch.cuda.Stream]) -> int:
    """The GPU of a call: its tensors' and its stream's, and the current one, on which the library launches.  (By numbers: ten
    comparisons of torch.device objects cost a call a microsecond more.)"""
    gpu = t.get_device()
    if gpu < 0 or gpu != torch._C._cuda_getDevice() or (stream is not None and stream.device.index != gpu):
        _refuse(f"tensors on {t.device}, stream on {'it' if stream is None else stream.device}: not both the current device")
    return gpu


def _tensor(t: Optional[torch.Tensor], dtype, n: int, what: str, gpu: int) -> Optional[int]:
    """The address of a contiguous tensor on a GPU of the given type with n elements or more; None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or t.get_device() != gpu or not t.is_contiguous():
        _refuse(f"{what}: {dtype} on GPU {gpu}, contiguous, {n} elements or more, not {tuple(t.shape)} {t.dtype} {t.device}")
    return t.data_ptr()


def _given(t: Optional[torch.Tensor], dtype, n: int, what: str, gpu: int) -> int:
    """The same for an argument that has to be there."""
    if t is None:
        _refuse(f"{what}: missing")
    return _tensor(t, dtype, n, what, gpu)


def _outputs(device, stream, *specs) -> List[torch.Tensor]:
    """Tensors (shape, dtype) for a call on `stream` to write.  They are of that stream's memory: what was given back on the
    current one may still be read there.  The current stream, which uses them next, is recorded."""
    if stream is None:
        return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in specs]
    here = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        out = [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in specs]
    for t in out:
        t.record_stream(here)
    return out


def _raw_stream(stream: Optional[torch.cuda.Stream], device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream


def _kv_pages(kc: torch.Tensor, vc: torch.Tensor, gpu: int) -> KvPages:
    """Caches [pages][page_size][kv heads][head_dim], any strides but the last (a head-by-head cache: transpose(1, 2))."""
    shape, ks, vs = kc.shape, kc.stride(), vc.stride()
    kt, vt = _DTYPES.get(kc.dtype), _DTYPES.get(vc.dtype)
    if (len(shape) != 4 or shape != vc.shape or ks[3] != 1 or vs[3] != 1 or kt is None or vt is None or kc.get_device() != gpu or
            vc.get_device() != gpu):
        _refuse(f"caches: two [pages][page_size][heads][head_dim] on GPU {gpu}, not {tuple(shape)} {kc.dtype} {kc.device} and "
                f"{tuple(vc.shape)} {vc.dtype} {vc.device}")
    return KvPages.from_buffer_copy(_KV_PACK(kc.data_ptr(), vc.data_ptr(), kt, vt, shape[0], shape[1], shape[2], shape[3],
                                             ks[0], ks[1], ks[2], vs[0], vs[1], vs[2]))   # (0.5 us; field by field 1.3)


def _pitch(t: torch.Tensor, width: int) -> int:
    """Elements from a row of `width` to the next; the stride of a single row means nothing."""
    return t.stride(0) if t.shape[0] != 1 else width


class BatchPlan:
    """Outputs of op_batch_plan (see atspeed_op_batch_plan)."""
    __slots__ = ("cu_q", "ctx_len", "state", "pages", "req", "pos", "slot", "mask")

    def __init__(self, cu_q, ctx_len, state, pages, req, pos, slot, mask):
        self.cu_q = cu_q          # [n + 1] int32
        self.ctx_len = ctx_len    # [n] int32, -1: not served
        self.state = state        # [n] int32, PLAN_*
        self.pages = pages        # [2] int32: used, taken
        self.req = req            # [T] int32
        self.pos = pos            # [T] int32
        self.slot = slot          # [T] int64, -1: not served
        self.mask = mask          # [T][words] int32 bit patterns (trees), or None

    @property
    def used(self) -> torch.Tensor:
        """[] int32, pages taken from the front of the free list."""
        return self.pages[0]

    @property
    def taken(self) -> torch.Tensor:
        """[] int32, pages that the requests up to the last served one ask for, those of the passed-over ones included."""
        return self.pages[1]


def op_batch_plan(q_len: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, free: torch.Tensor,
                  n_free: torch.Tensor, page_size: int, max_tokens: int, parent: Optional[torch.Tensor] = None,
                  mask_words: int = 0, stream=None) -> BatchPlan:
    """Pages, slots, positions and tree masks of a step from the requests' lengths; block_table is extended in place."""
    n, T, i32, dev, gpu = q_len.numel(), max_tokens, torch.int32, q_len.device, _gpu(q_len, stream)
    if block_table.dim() != 2 or block_table.shape[0] != n or T <= 0 or n == 0 or (parent is not None and mask_words <= 0):
        _refuse(f"{n} requests, {T} tokens, block_table {tuple(block_table.shape)}, {mask_words} mask words")
    q_ptr, kv_ptr = _given(q_len, i32, n, "q_len", gpu), _given(kv_len, i32, n, "kv_len", gpu)
    up_ptr = _tensor(parent, i32, T, "parent", gpu)
    table_ptr = _given(block_table, i32, n, "block_table", gpu)
    free_ptr, n_free_ptr = _given(free, i32, 0, "free", gpu), _given(n_free, i32, 1, "n_free", gpu)
    if free.numel() == 0:   # (n_free is 0: nothing is read of an address that has to be there)
        free_ptr = n_free_ptr
    cu_q, ctx_len, state, pages, req, pos, slot, *trees = _outputs(
        dev, stream, (n + 1, i32), (n, i32), (n, i32), (2, i32), (T, i32), (T, i32), (T, torch.int64),
        *([((T, mask_words), i32)] if parent is not None else []))
    mask = trees[0] if trees else None
    _check(load().atspeed_op_batch_plan(_raw_stream(stream, dev), n, q_ptr, kv_ptr, up_ptr, page_size, table_ptr,
                                        block_table.shape[1], free_ptr, n_free_ptr, T, mask_words, cu_q.data_ptr(),
                                        ctx_len.data_ptr(), state.data_ptr(), pages.data_ptr(), req.data_ptr(), pos.data_ptr(),
                                        slot.data_ptr(), _ptr(mask)))
    return BatchPlan(cu_q, ctx_len, state, pages, req, pos, slot, mask)


def op_rope_append(qkv: torch.Tensor, n_heads: int, kc: torch.Tensor, vc: torch.Tensor, slot: torch.Tensor,
                   pos: Optional[torch.Tensor] = None, theta: float = 10000.0, stream=None) -> torch.Tensor:
    """Rotates q and k of fused QKV rows [T][(heads + 2 kv heads) * head_dim], stores k and v by slot, returns q
    [T][heads][head_dim]."""
    dev, gpu = qkv.device, _gpu(qkv, stream)
    pages = _kv_pages(kc, vc, gpu)
    hd, src = pages.head_dim, _DTYPES.get(qkv.dtype)
    if qkv.dim() != 2 or src is None or qkv.stride(1) != 1 or qkv.shape[1] != (n_heads + 2 * pages.n_kv_heads) * hd:
        _refuse(f"qkv: [T][({n_heads} + 2 * {pages.n_kv_heads}) * {hd}], not {tuple(qkv.shape)} {qkv.dtype}")
    T = qkv.shape[0]
    q, = _outputs(dev, stream, ((T, n_heads, hd), kc.dtype))
    _check(load().atspeed_op_rope_append(_raw_stream(stream, dev), qkv.data_ptr(), src, _pitch(qkv, qkv.shape[1]), T, n_heads, pages,
                                         _given(slot, torch.int64, T, "slot", gpu), _tensor(pos, torch.int32, T, "pos", gpu), theta,
                                         q.data_ptr() if n_heads else None, n_heads * hd))
    return q


_tree_ws: Dict[Tuple[int, int], torch.Tensor] = {}
_graph_ws: Dict[Tuple[int, int], Tuple[int, torch.Tensor]] = {}   # of the last capture that a stream was part of
TREE_ATTENTION_COUNTER_BYTES = 4096


def _new_tree_workspace(device, stream: int) -> torch.Tensor:
    """Allocated and its counters zeroed on the stream whose calls use it, so that both come before them."""
    on = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(on):
        w = torch.empty(load().atspeed_op_tree_attention_workspace(), dtype=torch.uint8, device=device)
        w[:TREE_ATTENTION_COUNTER_BYTES].zero_()
    return w


def op_tree_attention_workspace(device, stream: int) -> torch.Tensor:
    """The attention's workspace of one stream (calls on one stream follow each other; two streams' would not).  Calls that are
    captured have one of their own, whatever the stream had before: a graph is replayed on any stream, beside this one's calls
    and other graphs.  It is of the graph's own memory, and the graph clears its counters before the first call."""
    key = (device.index or 0, stream)
    capture = load().atspeed_op_capture_id(stream)
    if capture:
        if _graph_ws.get(key, (0, None))[0] != capture:
            _graph_ws[key] = (capture, _new_tree_workspace(device, stream))
        return _graph_ws[key][1]
    if key not in _tree_ws:
        _tree_ws[key] = _new_tree_workspace(device, stream)
    return _tree_ws[key]


def op_tree_attention(q: torch.Tensor, kc: torch.Tensor, vc: torch.Tensor, cu_q: torch.Tensor, ctx_len: torch.Tensor,
                      block_table: torch.Tensor, mask: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of q [T][heads][head_dim] (rows any stride apart) over the batch's paged caches and, by the mask's bits
    (None: causal), the step's own tokens.  scale: 1 / sqrt(head_dim) by default.  Rows of no request (those past the last
    token of a padded step) are not written: without out they hold whatever the memory held."""
    dev, gpu = q.device, _gpu(q, stream)
    pages = _kv_pages(kc, vc, gpu)
    n, hd = ctx_len.numel(), pages.head_dim
    if q.dim() != 3 or q.dtype is not kc.dtype or q.shape[2] != hd or q.stride(2) != 1 or (q.stride(1) != hd and q.shape[1] != 1):
        _refuse(f"q: [T][heads][{hd}] of {kc.dtype}, each row contiguous, not {tuple(q.shape)} {q.dtype}")
    T, H, _ = q.shape
    if out is None:
        out, = _outputs(dev, stream, (q.shape, q.dtype))
    elif (out.shape != q.shape or out.dtype is not q.dtype or out.stride(2) != 1 or (out.stride(1) != hd and H != 1) or
          out.get_device() != gpu):
        _refuse(f"out: as q {tuple(q.shape)} {q.dtype} on {dev}, each row contiguous, not {tuple(out.shape)} {out.dtype} "
                f"{out.device}")
    if block_table.dim() != 2 or block_table.shape[0] < n or (mask is not None and (mask.dim() != 2 or mask.shape[0] < T)):
        _refuse(f"block_table: [{n}][width] and mask: [{T}][words], not {tuple(block_table.shape)} and "
                f"{None if mask is None else tuple(mask.shape)}")
    st = _raw_stream(stream, dev)
    _check(load().atspeed_op_tree_attention(st, pages, q.data_ptr(), _pitch(q, H * hd), H, n, T,
                                            _given(cu_q, torch.int32, n + 1, "cu_q", gpu),
                                            _given(ctx_len, torch.int32, 1, "ctx_len", gpu),
                                            _given(block_table, torch.int32, n, "block_table", gpu), block_table.shape[1],
                                            _tensor(mask, torch.int32, T, "mask", gpu), mask.shape[1] if mask is not None else 0,
                                            hd ** -0.5 if scale is None else scale, out.data_ptr(), _pitch(out, H * hd),
                                            _tensor(lse, torch.float32, T * H, "lse", gpu),
                                            op_tree_attention_workspace(dev, st).data_ptr()))
    return out


class LogitRules:
    """The per-request rules of op_adjust_logits (see atspeed_logit_rules); None leaves a rule out.  Keeps the tensors alive."""

    def __init__(self, n_req: Optional[int] = None, hist=None, hist_off=None, prompt_len=None, repetition=None, frequency=None,
                 presence=None, temperature=None, bias_off=None, bias_tok=None, bias_val=None, grammar=None, tree_tok=None,
                 cu_q=None):
        if n_req is None:
            n_req = next((t.numel() for t in (repetition, frequency, presence, temperature, prompt_len) if t is not None),
                         next((t.numel() - 1 for t in (hist_off, bias_off, cu_q) if t is not None), 0))
        if grammar is not None and grammar.dim() != 2:
            _refuse(f"grammar: [states][words], not {tuple(grammar.shape)}")
        if bias_tok is not None and bias_tok.numel() == 0:   # (lists without an entry have no address)
            bias_off = bias_tok = bias_val = None
        f32, i32 = torch.float32, torch.int32
        self._keep = (hist, hist_off, prompt_len, repetition, frequency, presence, temperature, bias_off, bias_tok, bias_val,
                      grammar, tree_tok, cu_q)
        self.n_req = n_req
        gpu = self.gpu = next((t.get_device() for t in self._keep if t is not None), None)   # (no tensor: of any)
        if gpu == -1:
            _refuse("rules on the CPU")
        self.desc = LogitRulesDesc(
            n_req, _tensor(hist, i32, 0, "hist", gpu), _tensor(hist_off, i32, n_req + 1, "hist_off", gpu),
            _tensor(prompt_len, i32, n_req, "prompt_len", gpu), _tensor(repetition, f32, n_req, "repetition", gpu),
            _tensor(frequency, f32, n_req, "frequency", gpu), _tensor(presence, f32, n_req, "presence", gpu),
            _tensor(temperature, f32, n_req, "temperature", gpu), _tensor(bias_off, i32, n_req + 1, "bias_off", gpu),
            _tensor(bias_tok, i32, 0, "bias_tok", gpu),
            _tensor(bias_val, f32, 0 if bias_tok is None else bias_tok.numel(), "bias_val", gpu),
            _tensor(grammar, i32, 0, "grammar", gpu),
            0 if grammar is None else grammar.shape[1], 0 if grammar is None else grammar.shape[0],
            _tensor(tree_tok, i32, 0, "tree_tok", gpu), _tensor(cu_q, i32, n_req + 1, "cu_q", gpu))


def op_adjust_logits(logits: torch.Tensor, req: torch.Tensor, rules: LogitRules, mask: Optional[torch.Tensor] = None,
                     state: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, out_dtype=None,
                     stream=None) -> torch.Tensor:
    """Rules on logits [R][vocab] (rows any stride apart) of requests req [R]; out may be logits itself."""
    it, dev, gpu = _DTYPES.get(logits.dtype), logits.device, _gpu(logits, stream)
    if logits.dim() != 2 or it is None or (logits.stride(1) != 1 and logits.shape[1] != 1):
        _refuse(f"logits: [R][vocab], not {tuple(logits.shape)} {logits.dtype}")
    R, V = logits.shape
    if rules.gpu not in (None, gpu):
        _refuse(f"rules on GPU {rules.gpu}, logits on {dev}")
    if out is None:
        out, = _outputs(dev, stream, ((R, V), out_dtype or logits.dtype))
    ot = _DTYPES.get(out.dtype)
    if out.shape != logits.shape or ot is None or out.get_device() != gpu or (out.stride(1) != 1 and V != 1):
        _refuse(f"out: [{R}][{V}] on {dev}, not {tuple(out.shape)} {out.dtype} {out.device}")
    if mask is not None and (mask.dim() != 2 or mask.shape[0] < R):
        _refuse(f"mask: [{R}][words], not {tuple(mask.shape)}")
    _check(load().atspeed_op_adjust_logits(_raw_stream(stream, dev), logits.data_ptr(), it, _pitch(logits, V), R, V,
                                           _given(req, torch.int32, R, "req", gpu), rules.desc,
                                           _tensor(mask, torch.int32, R, "mask", gpu), mask.shape[1] if mask is not None else 0,
                                           _tensor(state, torch.int32, R, "state", gpu), out.data_ptr(), ot, _pitch(out, V)))
    return out


# ---------------------------------------------------------------------------------------------------
# what follows a step's logits: beam selection, fork of block tables, copies of pages, compaction of an accepted path
# ---------------------------------------------------------------------------------------------------
# Memory of the stream that a call is on (or of the graph that captures it), given back after the call: what comes there next comes
# after it.  (As a tensor, as a torch without these two has it, it takes 1.4 us more.)
_raw_alloc = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_alloc", None)
_raw_delete = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_delete", None)


class BeamChoice:
    """Outputs of op_beam_select [n][width], best first (see atspeed_op_beam_select)."""
    __slots__ = ("token", "parent", "score")

    def __init__(self, token, parent, score):
        self.token = token      # int32, -1: no continuation
        self.parent = parent    # int32, the row of the logits, -1: none
        self.score = score      # float32, -infinity: none


def op_beam_select(logits: torch.Tensor, cu_beam: torch.Tensor, width: int, score: Optional[torch.Tensor] = None,
                   final: Optional[torch.Tensor] = None, grammar: Optional[torch.Tensor] = None,
                   state: Optional[torch.Tensor] = None, norm: int = NORM_MASKED, stream=None) -> BeamChoice:
    """The best continuations of each request's beams, rows cu_beam[b] .. cu_beam[b + 1] - 1 of logits [R][vocab] (any stride apart)."""
    it, dev, gpu = _DTYPES.get(logits.dtype), logits.device, _gpu(logits, stream)
    if logits.dim() != 2 or it is None or (logits.stride(1) != 1 and logits.shape[1] != 1):
        _refuse(f"logits: [R][vocab], not {tuple(logits.shape)} {logits.dtype}")
    (R, V), n, i32, f32 = logits.shape, cu_beam.numel() - 1, torch.int32, torch.float32
    if n < 1 or R < 1 or V < 1 or width < 1 or (state is None) != (grammar is None) or (grammar is not None and grammar.dim() != 2):
        _refuse(f"{n} requests, {R} rows of {V}, width {width}, state {'missing' if state is None else 'given'}, grammar "
                f"{'missing' if grammar is None else tuple(grammar.shape)}")
    lib = load()
    cu_ptr, score_ptr = _given(cu_beam, i32, 2, "cu_beam", gpu), _tensor(score, f32, R, "score", gpu) or 0
    final_ptr, state_ptr = _tensor(final, i32, R, "final", gpu) or 0, _tensor(state, i32, R, "state", gpu) or 0
    words, states, grammar_ptr = 0, 0, 0
    if grammar is not None:
        states, words = grammar.shape
        grammar_ptr = _tensor(grammar, i32, 1, "grammar", gpu)
    token, parent, out = _outputs(dev, stream, ((n, width), i32), ((n, width), i32), ((n, width), f32))
    beams = _BEAMS_PACK(logits.data_ptr(), _pitch(logits, V), it, R, V, n, width, norm, cu_ptr, score_ptr, final_ptr, state_ptr, grammar_ptr,
                        words, states, token.data_ptr(), parent.data_ptr(), out.data_ptr())
    st, size = _raw_stream(stream, dev), lib.atspeed_op_beam_select_workspace(R, V, width)
    if _raw_alloc is None or _raw_delete is None:
        whole, = _outputs(dev, stream, ((size,), torch.uint8))
        _check(lib.atspeed_op_beam_select(st, beams, whole.data_ptr()))
        return BeamChoice(token, parent, out)
    ws = _raw_alloc(size, st)
    try:
        _check(lib.atspeed_op_beam_select(st, beams, ws))
    finally:
        _raw_delete(ws)
    return BeamChoice(token, parent, out)


class PageFork:
    """Outputs of op_fork_pages (see atspeed_op_fork_pages)."""
    __slots__ = ("table", "kv_len", "state", "src", "dst", "ref", "free", "n_free")

    def __init__(self, table, kv_len, state, src, dst, ref, free, n_free):
        self.table = table      # [m][width] int32, -1 behind a row's pages
        self.kv_len = kv_len    # [m] int32, -1: not served
        self.state = state      # [m] int32, PLAN_*
        self.src = src          # [m] int32, page to copy from, -1: none
        self.dst = dst          # [m] int32, page to copy to, -1: none
        self.ref = ref          # [pages] int32, who holds a page
        self.free = free        # [pages] int32, free pages, -1 behind them
        self.n_free = n_free    # [1] int32


def op_fork_pages(table: torch.Tensor, kv_len: torch.Tensor, ref: torch.Tensor, free: torch.Tensor, n_free: torch.Tensor,
                  page_size: int, q_len: Optional[torch.Tensor] = None, state: Optional[torch.Tensor] = None,
                  used: Optional[torch.Tensor] = None, parent: Optional[torch.Tensor] = None,
                  length: Optional[torch.Tensor] = None, out: Optional[PageFork] = None, stream=None) -> PageFork:
    """New rows of block tables, page counts and free list from old ones, which stay as they are.  used: the plan's count of pages
    taken (BatchPlan.pages or .used); out: a fork of the same sizes to write into, not the one that the inputs are from."""
    i32, dev, gpu = torch.int32, table.device, _gpu(table, stream)
    n, pages = kv_len.numel(), ref.numel()
    if table.dim() != 2 or table.shape[0] != n or n < 1 or pages < 1 or (parent is None and length is not None and length.numel() != n):
        _refuse(f"{n} rows, table {tuple(table.shape)}, {pages} pages, {'no parents' if parent is None else parent.numel()}")
    m, width, room = n if parent is None else parent.numel(), table.shape[1], free.numel() or -1
    n_free_ptr = _given(n_free, i32, 1, "n_free", gpu)
    ins = (_given(table, i32, n, "table", gpu), _given(kv_len, i32, n, "kv_len", gpu), _tensor(q_len, i32, n, "q_len", gpu) or 0,
           _tensor(state, i32, n, "state", gpu) or 0, _tensor(parent, i32, 1, "parent", gpu) or 0, _tensor(length, i32, m, "length", gpu) or 0,
           _given(ref, i32, pages, "ref", gpu),
           _given(free, i32, 0, "free", gpu) if room > 0 else n_free_ptr,   # (of an empty list nothing is read, whatever n_free is)
           n_free_ptr, _tensor(used, i32, 1, "used", gpu) or 0)
    if out is None:   # (one tensor and views of it, the counts at its start: eight tensors take longer)
        cells = m * width
        whole, = _outputs(dev, stream, ((2 * pages + cells + 4 * m + 1,), i32))
        new_ref, new_free, new_table, new_len, new_state, src, dst, left = whole.split_with_sizes((pages, pages, cells, m, m, m, m, 1))
        out, at = PageFork(new_table.view(m, width), new_len, new_state, src, dst, new_ref, new_free, left), whole.data_ptr()
        rows = at + 8 * pages + 4 * cells
        outs = (at + 8 * pages, rows, rows + 4 * m, rows + 8 * m, rows + 12 * m, at, at + 4 * pages, rows + 16 * m)
    else:
        if out.table.shape != (m, width):
            _refuse(f"out.table: [{m}][{width}], not {tuple(out.table.shape)}")
        sizes = (m * width, m, m, m, m, pages, pages, 1)
        outs = [_given(getattr(out, k), i32, size, "out." + k, gpu) for k, size in zip(PageFork.__slots__, sizes)]
    _check(load().atspeed_op_fork_pages(_raw_stream(stream, dev), _FORK_PACK(n, m, width, page_size, pages, room, *ins, *outs)))
    return out


class CacheLayers:
    """All layers' caches, [(K, V), ..] of one geometry, each [pages][page_size][kv heads][head_dim] (any strides but the last): what
    op_copy_pages and op_compact_tokens move rows in.  Made once; keeps the tensors alive."""

    def __init__(self, caches: Sequence[Tuple[torch.Tensor, torch.Tensor]]):
        if not caches:
            _refuse("no layers")
        self._keep = [tuple(c) for c in caches]
        self.device = caches[0][0].device
        self.gpu = caches[0][0].get_device()
        if self.gpu < 0:
            _refuse("caches on the CPU")
        self.n = len(caches)
        self.desc = (KvPages * self.n)(*[_kv_pages(k, v, self.gpu) for k, v in caches])

    def _on(self, stream) -> int:
        if self.gpu != torch._C._cuda_getDevice() or (stream is not None and stream.device.index != self.gpu):
            _refuse(f"caches on {self.device}, stream on {'it' if stream is None else stream.device}: not both the current device")
        return self.gpu


def op_copy_pages(layers: CacheLayers, src: torch.Tensor, dst: torch.Tensor, length: Optional[torch.Tensor] = None,
                  stream=None) -> None:
    """The first ((length - 1) mod page size) + 1 tokens (None: all) of pages src to pages dst, K and V of all layers; -1: none."""
    gpu, n, i32 = layers._on(stream), src.numel(), torch.int32
    if not 0 < n < 1 << 31:
        _refuse(f"{n} pages")
    _check(load().atspeed_op_copy_pages(_raw_stream(stream, layers.device), layers.desc, layers.n, n, _given(src, i32, n, "src", gpu),
                                        _given(dst, i32, n, "dst", gpu), _tensor(length, i32, n, "length", gpu)))


def op_compact_tokens(layers: CacheLayers, slot: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor, keep: torch.Tensor,
                      n_keep: torch.Tensor, state: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Moves the kept ones keep [n][..] (n_keep [n] of them, ascending) of each request's new tokens behind the cached ones, K and V of
    all layers; slot, cu_q, state: the plan's.  Returns the cached tokens of each request [n]."""
    gpu, n, i32 = layers._on(stream), kv_len.numel(), torch.int32
    if not 0 < n < 1 << 31 or keep.dim() != 2 or keep.shape[0] != n or not 0 < keep.shape[1] < 1 << 31 or slot.numel() < 1:
        _refuse(f"{n} requests, {slot.numel()} slots, keep {tuple(keep.shape)}")
    ins = (min(slot.numel(), (1 << 31) - 1), _given(slot, torch.int64, 1, "slot", gpu), _given(cu_q, i32, n + 1, "cu_q", gpu), _given(kv_len, i32, n, "kv_len", gpu),
           _tensor(state, i32, n, "state", gpu), _given(keep, i32, n, "keep", gpu), keep.shape[1], _given(n_keep, i32, n, "n_keep", gpu))
    new_len, = _outputs(layers.device, stream, ((n,), i32))
    _check(load().atspeed_op_compact_tokens(_raw_stream(stream, layers.device), layers.desc, layers.n, n, *ins, new_len.data_ptr()))
    return new_len
