"""ctypes binding of the C ABI in include/blockserve.h (argument marshalling only).

PyTorch provides device memory and the CUDA stream; every step of the path runs
in the library's kernels.  Importing this module without the built library, or
creating an engine without a CUDA device, raises: there is no CPU path.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Dict, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# BS_DEBUG_LIB=1 selects the bounds-checked build (paper_2607_08930_b200.build.build(debug=True))
DEBUG_LIB = bool(os.environ.get("BS_DEBUG_LIB"))
LIB_PATH = os.path.join(_HERE, "libblockserve_dbg.so" if DEBUG_LIB else "libblockserve.so")
BUILD_BOUNDS_CHECK = 1

BS_OK, BS_E_ARG, BS_E_STATE, BS_E_BUDGET, BS_E_KV_FULL, BS_E_CUDA, BS_E_TIMEOUT, BS_E_UNKNOWN_REQ = (
    0, -1, -2, -3, -4, -5, -6, -7)
SUFFIX_FULL, SUFFIX_NONE = 0, 1
REFRESH_EVERY_BLOCK, REFRESH_AT_ADMISSION = 0, 1
REQ_QUEUED, REQ_ACTIVE, REQ_FINISHED = 0, 1, 2

(DBG_HEADER, DBG_ROW_SLOT, DBG_ROW_MASK, DBG_ROW_S, DBG_ROW_KV_BASE, DBG_CU_Q, DBG_TOK_ROW, DBG_TOK_POS,
 DBG_TOK_KV, DBG_LM_TOK, DBG_LM_ROW, DBG_LM_SLOT, DBG_PREV_LM_ROW, DBG_PREV_LM_SLOT, DBG_PREV_TOK,
 DBG_PREV_CONF, DBG_PREV_COMMIT, DBG_PREV_LOGITS, DBG_REQ_ID_OF_ROW, DBG_KV_ROW) = range(20)


FAMILIES = ("index", "embed_norm", "gemm_qkv", "rope_kv", "attention", "gemm_o", "gemm_gate_up", "gemm_down",
            "gemm_lm_head", "confidence", "attention_refresh")


class BsConfig(C.Structure):
    _fields_ = [("n_layers", C.c_int), ("d_model", C.c_int), ("n_q_heads", C.c_int), ("n_kv_heads", C.c_int),
                ("head_dim", C.c_int), ("d_ffn", C.c_int), ("vocab", C.c_int), ("mask_id", C.c_int),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("block_len", C.c_int), ("tau", C.c_float),
                ("token_budget", C.c_longlong), ("max_batch", C.c_int), ("max_requests", C.c_int),
                ("max_row_tokens", C.c_int), ("kv_capacity_tokens", C.c_longlong), ("suffix_mode", C.c_int),
                ("sort_queue", C.c_int), ("steps_per_block", C.c_int), ("eos_id", C.c_int),
                ("static_groups", C.c_int), ("async_advance", C.c_int), ("refresh_policy", C.c_int),
                ("keep_logits", C.c_int)]


class BsWeights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("wqkv", C.POINTER(C.c_void_p)), ("wo", C.POINTER(C.c_void_p)), ("w_gate", C.POINTER(C.c_void_p)),
                ("w_up", C.POINTER(C.c_void_p)), ("w_down", C.POINTER(C.c_void_p)),
                ("norm1", C.POINTER(C.c_void_p)), ("norm2", C.POINTER(C.c_void_p))]


class BsSizes(C.Structure):
    _fields_ = [("kv_bytes", C.c_size_t), ("workspace_bytes", C.c_size_t), ("state_bytes", C.c_size_t)]


class BsStats(C.Structure):
    _fields_ = [("steps", C.c_longlong), ("cycles", C.c_longlong), ("sum_active", C.c_longlong),
                ("committed", C.c_longlong), ("packed_tokens", C.c_longlong), ("lm_rows", C.c_longlong),
                ("kernel_launches", C.c_longlong), ("row_steps", C.c_longlong), ("active_row_steps", C.c_longlong)]


class BsLogitRules(C.Structure):
    _fields_ = [("vocab", C.c_int), ("n_reqs", C.c_int), ("mask_id", C.c_int), ("row_req", C.c_void_p), ("ctx", C.c_void_p),
                ("ctx_total", C.c_longlong), ("ctx_begin", C.c_void_p), ("ctx_gen", C.c_void_p), ("ctx_end", C.c_void_p),
                ("repetition", C.c_void_p), ("presence", C.c_void_p), ("frequency", C.c_void_p), ("bias_at", C.c_void_p),
                ("bias_tok", C.c_void_p), ("bias_val", C.c_void_p), ("bias_total", C.c_longlong), ("allowed", C.c_void_p),
                ("allowed_ld", C.c_longlong), ("n_masks", C.c_int), ("row_mask", C.c_void_p)]


EXPORTS = ["bs_query_sizes", "bs_init_model", "bs_admit", "bs_evict_refill", "bs_denoise_step", "bs_block_done",
           "bs_read_tokens", "bs_get_stats", "bs_set_profiling", "bs_get_profile", "bs_destroy", "bs_last_error", "bs_build_flags", "bs_debug_read", "bs_debug_inject_timeout",
           "bs_debug_force_commit", "bs_debug_snapshot", "bs_debug_restore", "bs_op_gemm", "bs_op_gemm_cluster_splits",
           "bs_op_rmsnorm", "bs_op_rope_kv", "bs_op_rope_kv_static", "bs_op_attention_q_tile", "bs_op_attention", "bs_op_confidence",
           "bs_op_lm_head_confidence", "bs_op_lm_head_confidence_scratch_bytes", "bs_rope_table", "bs_op_qk_norm_rope_kv",
           "bs_op_qk_norm_rope_kv8", "bs_op_kv8_read", "bs_op_attention_kv8", "bs_op_attention_kv8_scratch_bytes",
           "bs_op_attention_kv8_uses_scratch", "bs_op_quant_i8", "bs_op_gemm_i8", "bs_op_logit_rules",
           "bs_op_rules_confidence"]

_lib = None


def lib() -> C.CDLL:
    """Load the CUDA library (built in-tree by paper_2607_08930_b200/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2607_08930_b200.build` "
                               "(the engine has no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        vp, ip, i, f, ll = C.c_void_p, C.POINTER(C.c_int), C.c_int, C.c_float, C.c_longlong
        L.bs_query_sizes.argtypes = [C.POINTER(BsConfig), C.POINTER(BsSizes)]
        L.bs_init_model.argtypes = [C.POINTER(BsConfig), C.POINTER(BsWeights), vp, vp, vp, vp, C.POINTER(vp)]
        L.bs_admit.argtypes = [vp, ll, ip, i, i, f, i, ip]
        L.bs_evict_refill.argtypes = [vp, ip, ip, ip]
        L.bs_denoise_step.argtypes = [vp, ip]
        L.bs_block_done.argtypes = [vp, ip, C.POINTER(C.c_ubyte)]
        L.bs_read_tokens.argtypes = [vp, ll, ip, i, ip, ip]
        L.bs_get_stats.argtypes = [vp, C.POINTER(BsStats)]
        L.bs_set_profiling.argtypes = [vp, i]
        L.bs_get_profile.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(ll), C.POINTER(C.c_double),
                                     C.POINTER(C.c_double)]
        L.bs_destroy.argtypes = [vp]
        L.bs_destroy.restype = None
        L.bs_last_error.argtypes = [vp]
        L.bs_last_error.restype = C.c_char_p
        L.bs_build_flags.argtypes = []
        L.bs_debug_read.argtypes = [vp, i, i, i, vp, C.c_size_t, C.POINTER(C.c_size_t)]
        L.bs_debug_inject_timeout.argtypes = [vp]
        L.bs_debug_force_commit.argtypes = [vp, i, C.c_ulonglong, vp]
        L.bs_debug_snapshot.argtypes = [vp, vp, C.c_size_t, C.POINTER(C.c_size_t)]
        L.bs_debug_restore.argtypes = [vp, vp, C.c_size_t]
        L.bs_op_gemm.argtypes = [vp, i, vp, vp, vp, i, i, i, i, i, vp, vp, C.c_size_t, vp, vp]
        L.bs_op_gemm_cluster_splits.argtypes = [i, i, i, i]
        L.bs_op_rmsnorm.argtypes = [vp, vp, vp, vp, i, i, f, vp]
        L.bs_op_rope_kv.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, f, i, vp, vp]
        L.bs_op_rope_kv_static.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, f, i, vp]
        L.bs_op_attention_q_tile.argtypes = [i, i, i]
        L.bs_op_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, ll, i, i, i, vp, C.c_size_t, vp, vp]
        L.bs_op_confidence.argtypes = [vp, i, i, i, vp, vp, vp]
        L.bs_op_lm_head_confidence_scratch_bytes.argtypes = [i, i]
        L.bs_op_lm_head_confidence_scratch_bytes.restype = C.c_size_t
        L.bs_op_lm_head_confidence.argtypes = [vp, i, vp, i, i, i, vp, i, vp, C.c_size_t, vp, vp, vp, vp, vp]
        L.bs_rope_table.argtypes = [vp, i, i, f]
        L.bs_op_qk_norm_rope_kv.argtypes = [vp, vp, vp, f, vp, vp, vp, i, vp, vp, ll, i, i, i, i, vp, i, vp, vp]
        L.bs_op_qk_norm_rope_kv8.argtypes = [vp, vp, vp, f, vp, vp, vp, vp, vp, i, vp, i, vp, vp, vp, vp, ll, i, i, i, i,
                                             vp, i, vp, vp]
        L.bs_op_kv8_read.argtypes = [vp, vp, vp, vp, ll, vp, vp, vp, i, i, i, i, vp, vp, vp, vp]
        L.bs_op_attention_kv8_scratch_bytes.argtypes = [i, i, i]
        L.bs_op_attention_kv8_scratch_bytes.restype = C.c_size_t
        L.bs_op_attention_kv8_uses_scratch.argtypes = [i] * 7
        L.bs_op_attention_kv8.argtypes = [vp, i, vp, vp, vp, vp, ll, vp, vp, vp, vp, i, i, i, i, i, i, i, vp, C.c_size_t,
                                          vp, vp]
        L.bs_op_quant_i8.argtypes = [vp, i, ll, vp, i, vp, f, vp, ll, vp, i, i, vp, vp]
        L.bs_op_gemm_i8.argtypes = [vp, ll, vp, vp, ll, vp, vp, vp, vp, ll, i, i, i, i, vp, vp]
        L.bs_op_logit_rules.argtypes = [vp, i, ll, vp, ll, i, vp, vp, vp]
        L.bs_op_rules_confidence.argtypes = [vp, i, ll, i, vp, vp, vp, vp, vp]
        _lib = L
    return _lib


class BlockServeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"blockserve error {code}: {msg}")
        self.code = code


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _check_op(rc: int, name: str) -> None:
    if rc != BS_OK:
        raise BlockServeError(rc, f"{name} failed")


def make_config(shape, block_len: int, tau: float, token_budget: int, max_batch: int, max_requests: int,
                max_row_tokens: int, kv_capacity_tokens: int, suffix_mode: int = SUFFIX_FULL,
                sort_queue: bool = True, steps_per_block: int = 0, eos_id: int = -1,
                static_groups: bool = False, keep_logits: bool = False, async_advance: bool = False,
                refresh_policy: int = 0) -> BsConfig:
    return BsConfig(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
                    shape.vocab, shape.mask_id, shape.rms_eps, shape.rope_theta, block_len, tau, token_budget,
                    max_batch, max_requests, max_row_tokens, kv_capacity_tokens, suffix_mode, int(sort_queue),
                    int(steps_per_block), int(eos_id), int(static_groups), int(async_advance), int(refresh_policy),
                    int(keep_logits))


def query_sizes(cfg: BsConfig) -> BsSizes:
    out = BsSizes()
    rc = lib().bs_query_sizes(C.byref(cfg), C.byref(out))
    if rc != BS_OK:
        raise BlockServeError(rc, (lib().bs_last_error(None) or b"").decode())
    return out


class Engine:
    """Owns the torch buffers an engine borrows and forwards calls to the C ABI."""

    def __init__(self, cfg: BsConfig, weights: Dict[str, object], device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the block-denoising engine has no CPU fallback")
        self.L = lib()
        self.cfg = cfg
        self.device = torch.device(device)
        sz = query_sizes(cfg)
        self.sizes = sz
        with torch.cuda.device(self.device):
            self.kv = torch.empty(sz.kv_bytes, dtype=torch.uint8, device=self.device)
            self.workspace = torch.empty(sz.workspace_bytes, dtype=torch.uint8, device=self.device)
            self.state = torch.empty(sz.state_bytes, dtype=torch.uint8, device=self.device)
            self.weights = weights        # keep the tensors alive
            n = cfg.n_layers
            arrs = {}
            for name in ("wqkv", "wo", "w_gate", "w_up", "w_down", "norm1", "norm2"):
                ts = weights[name]
                assert len(ts) == n and all(t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous() for t in ts)
                arrs[name] = (C.c_void_p * n)(*[t.data_ptr() for t in ts])
            self._arrs = arrs
            w = BsWeights(weights["embed"].data_ptr(), weights["lm_head"].data_ptr(),
                          weights["final_norm"].data_ptr(),
                          *[C.cast(arrs[k], C.POINTER(C.c_void_p)) for k in
                            ("wqkv", "wo", "w_gate", "w_up", "w_down", "norm1", "norm2")])
            h = C.c_void_p()
            rc = self.L.bs_init_model(C.byref(cfg), C.byref(w), self.kv.data_ptr(), self.workspace.data_ptr(),
                                      self.state.data_ptr(), _stream(), C.byref(h))
        if rc != BS_OK:
            raise BlockServeError(rc, (self.L.bs_last_error(None) or b"").decode())
        self.h = h

    def _chk(self, rc: int) -> None:
        if rc != BS_OK:
            raise BlockServeError(rc, (self.L.bs_last_error(self.h) or b"").decode())

    def admit(self, req_id: int, prompt: Sequence[int], g: int, alpha: float, start_block: int = 0,
              gen_prefix: Optional[Sequence[int]] = None) -> None:
        pr = np.ascontiguousarray(prompt, dtype=np.int32)
        gp = None if gen_prefix is None else np.ascontiguousarray(gen_prefix, dtype=np.int32)
        ip = C.POINTER(C.c_int)
        self._chk(self.L.bs_admit(self.h, req_id, pr.ctypes.data_as(ip), len(pr), g, alpha, start_block,
                                  None if gp is None else gp.ctypes.data_as(ip)))

    def evict_refill(self):
        a, b, c = C.c_int(), C.c_int(), C.c_int()
        self._chk(self.L.bs_evict_refill(self.h, C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def denoise_step(self, want_count: bool = False) -> Optional[int]:
        if want_count:
            n = C.c_int()
            self._chk(self.L.bs_denoise_step(self.h, C.byref(n)))
            return n.value
        self._chk(self.L.bs_denoise_step(self.h, None))
        return None

    def block_done(self) -> bool:
        d = C.c_int()
        self._chk(self.L.bs_block_done(self.h, C.byref(d), None))
        return bool(d.value)

    def rows_done(self) -> np.ndarray:
        d = C.c_int()
        buf = (C.c_ubyte * self.cfg.max_batch)()
        self._chk(self.L.bs_block_done(self.h, C.byref(d), buf))
        return np.frombuffer(buf, dtype=np.uint8).copy()

    def read_tokens(self, req_id: int):
        n, st = C.c_int(), C.c_int()
        self._chk(self.L.bs_read_tokens(self.h, req_id, None, 0, C.byref(n), C.byref(st)))
        out = np.empty(n.value, dtype=np.int32)
        self._chk(self.L.bs_read_tokens(self.h, req_id, out.ctypes.data_as(C.POINTER(C.c_int)), n.value,
                                        C.byref(n), C.byref(st)))
        return out, st.value

    def stats(self) -> BsStats:
        s = BsStats()
        self._chk(self.L.bs_get_stats(self.h, C.byref(s)))
        return s

    def inject_timeout(self) -> None:
        self._chk(self.L.bs_debug_inject_timeout(self.h))

    def force_commit(self, row: int, positions: Dict[int, int]) -> None:
        """Commit block position -> token for the given active row (debugging aid)."""
        toks = np.zeros(64, dtype=np.int32)
        bits = 0
        for j, t in positions.items():
            toks[j] = t
            bits |= 1 << j
        self._chk(self.L.bs_debug_force_commit(self.h, row, bits, toks.ctypes.data))

    def snapshot(self) -> np.ndarray:
        """Engine state between block cycles as bytes (token rows + scheduler state; the KV cache is rebuilt)."""
        n = C.c_size_t(0)
        self._chk(self.L.bs_debug_snapshot(self.h, None, 0, C.byref(n)))
        buf = np.empty(n.value, dtype=np.uint8)
        self._chk(self.L.bs_debug_snapshot(self.h, buf.ctypes.data, buf.nbytes, C.byref(n)))
        return buf[:n.value]

    def restore(self, snap: np.ndarray) -> None:
        snap = np.ascontiguousarray(snap, dtype=np.uint8)
        self._chk(self.L.bs_debug_restore(self.h, snap.ctypes.data, snap.nbytes))

    def set_profiling(self, on: bool) -> None:
        self._chk(self.L.bs_set_profiling(self.h, int(on)))

    def profile(self) -> Dict[str, Dict[str, float]]:
        """Per kernel family: device ms, launches, algorithmic flops and bytes since profiling was enabled."""
        n = len(FAMILIES)
        ms, fl, by = (C.c_double * n)(), (C.c_double * n)(), (C.c_double * n)()
        la = (C.c_longlong * n)()
        self._chk(self.L.bs_get_profile(self.h, ms, la, fl, by))
        return {FAMILIES[i]: dict(ms=ms[i], launches=int(la[i]), flops=fl[i], bytes=by[i]) for i in range(n)}

    def debug(self, what: int, dtype=np.int32, arg0: int = 0, arg1: int = 0, cap: int = 1 << 16) -> np.ndarray:
        buf = np.empty(cap, dtype=np.uint8)
        n = C.c_size_t()
        self._chk(self.L.bs_debug_read(self.h, what, arg0, arg1, buf.ctypes.data, cap, C.byref(n)))
        return buf[:n.value].view(dtype).copy()

    def run(self, max_cycles: int = 1 << 30) -> int:
        """Algorithm 1 until the pending queue and the active set are empty."""
        cycles = 0
        while cycles < max_cycles:
            _, _, n = self.evict_refill()
            if n == 0:
                break
            while True:
                self.denoise_step()
                if self.block_done():
                    break
            cycles += 1
        return cycles

    def close(self) -> None:
        if getattr(self, "h", None):
            self.L.bs_destroy(self.h)      # synchronises the engine's stream
            self.h = None
            self.kv = self.workspace = self.state = None    # give the arenas back to the allocator

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def engine_for_workload(wl, weights, *, kv_capacity_tokens: Optional[int] = None, suffix_mode: int = SUFFIX_FULL,
                        sort_queue: bool = True, steps_per_block: int = 0, eos_id: int = -1,
                        static_groups: bool = False, keep_logits: bool = False, async_advance: bool = False,
                        refresh_policy: int = 0, device: str = "cuda:0") -> Engine:
    """Size an engine for a bs_inputs.Workload (the caller still admits the requests)."""
    mrt = wl.max_row_tokens
    if kv_capacity_tokens is None:
        rows = sorted((r.p + r.g for r in wl.requests), reverse=True)[:wl.max_batch]
        kv_capacity_tokens = sum(rows)
        if wl.token_budget > 0:       # Eq. 1 bounds |A| * width; rows are at most width + g long
            kv_capacity_tokens = min(kv_capacity_tokens, wl.token_budget + wl.max_batch * max(r.g for r in wl.requests))
    cfg = make_config(wl.shape, wl.block_len, wl.tau, wl.token_budget, wl.max_batch, len(wl.requests), mrt,
                      max(kv_capacity_tokens, mrt), suffix_mode, sort_queue, steps_per_block, eos_id, static_groups,
                      keep_logits, async_advance, refresh_policy)
    return Engine(cfg, weights, device)


# ---- single operations -------------------------------------------------------------------------------------

def op_gemm(A: torch.Tensor, W: torch.Tensor, mode: int = 0, W2: Optional[torch.Tensor] = None,
            C_out: Optional[torch.Tensor] = None, row_scale: Optional[torch.Tensor] = None,
            scratch: Optional[torch.Tensor] = None, error_flag: Optional[torch.Tensor] = None) -> torch.Tensor:
    M, K = A.shape
    N = W.shape[0]
    if C_out is None:
        C_out = torch.empty(M, N, dtype=torch.bfloat16 if mode in (0, 3) else torch.float32, device=A.device)
    _check_op(lib().bs_op_gemm(A.data_ptr(), A.stride(0), W.data_ptr(), _ptr(W2), C_out.data_ptr(), C_out.stride(0),
                               M, N, K, mode, _ptr(row_scale), _ptr(scratch),
                               0 if scratch is None else scratch.numel() * scratch.element_size(),
                               _ptr(error_flag), _stream()), "bs_op_gemm")
    return C_out


def op_gemm_cluster_splits(M: int, N: int, K: int, mode: int) -> int:
    """CTA pairs that share each output tile's K range inside one cluster for this op_gemm call (0: another plan)."""
    return int(lib().bs_op_gemm_cluster_splits(M, N, K, mode))


def op_rmsnorm(x: torch.Tensor, w: torch.Tensor, eps: float, idx: Optional[torch.Tensor] = None) -> torch.Tensor:
    M = x.shape[0] if idx is None else idx.shape[0]
    y = torch.empty(M, x.shape[1], dtype=torch.bfloat16, device=x.device)
    _check_op(lib().bs_op_rmsnorm(x.data_ptr(), _ptr(idx), w.data_ptr(), y.data_ptr(), M, x.shape[1], eps, _stream()),
              "bs_op_rmsnorm")
    return y


def op_rope_kv(qkv, tok_pos, tok_kv, kcache, vcache, hq, hkv, dh, theta, max_pos) -> None:
    scratch = torch.empty(max_pos * dh, dtype=torch.float32, device=qkv.device)
    _check_op(lib().bs_op_rope_kv(qkv.data_ptr(), tok_pos.data_ptr(), tok_kv.data_ptr(), kcache.data_ptr(),
                                  vcache.data_ptr(), qkv.shape[0], hq, hkv, dh, theta, max_pos, scratch.data_ptr(),
                                  _stream()), "bs_op_rope_kv")
    torch.cuda.current_stream().synchronize()


ROPE_STATIC_MAX_FLOATS = 512 * 1024


def op_rope_kv_static(qkv, tok_pos, tok_kv, kcache, vcache, hq, hkv, dh, theta, max_pos) -> int:
    """bs_op_rope_kv for callers that cannot allocate: the cos/sin table lives inside the library (at most
    ROPE_STATIC_MAX_FLOATS = max_pos * head_dim floats).  Nothing is allocated here either: the wrapper only
    passes the caller's pointers through.  Returns the status code (BS_E_ARG when the table would not fit)."""
    return lib().bs_op_rope_kv_static(qkv.data_ptr(), tok_pos.data_ptr(), tok_kv.data_ptr(), kcache.data_ptr(),
                                      vcache.data_ptr(), qkv.shape[0], hq, hkv, dh, theta, max_pos, _stream())


def attention_plan(cu_q: torch.Tensor, vis: torch.Tensor, hq: int, hkv: int, dh: int = 128):
    """Work-item prefix over rows (q-tiles) and the launch scalars of bs_op_attention; involves a device-to-host
    copy, so callers that launch repeatedly build it once."""
    qt = lib().bs_op_attention_q_tile(hq, hkv, dh)
    cu = cu_q.detach().cpu().numpy().astype(np.int64)
    tiles = np.zeros(len(cu), dtype=np.int32)
    tiles[1:] = np.cumsum((cu[1:] - cu[:-1] + qt - 1) // qt)
    return dict(cu_tile=torch.from_numpy(tiles).to(cu_q.device), n_tiles=int(tiles[-1]),
                max_vis=int(vis.max().item()) if len(vis) else 0,
                max_nq=int((cu[1:] - cu[:-1]).max()) if len(cu) > 1 else 0)


def op_attention(qkv, kcache, vcache, cu_q, kv_base, vis, hq, hkv, dh, scratch: Optional[torch.Tensor] = None,
                 plan=None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    plan = plan or attention_plan(cu_q, vis, hq, hkv, dh)
    if out is None:
        out = torch.empty(qkv.shape[0], hq * dh, dtype=torch.bfloat16, device=qkv.device)
    _check_op(lib().bs_op_attention(qkv.data_ptr(), kcache.data_ptr(), vcache.data_ptr(), out.data_ptr(),
                                    cu_q.data_ptr(), plan["cu_tile"].data_ptr(), kv_base.data_ptr(), vis.data_ptr(),
                                    len(cu_q) - 1, plan["n_tiles"], qkv.shape[0], plan["max_vis"], plan["max_nq"],
                                    kcache.shape[0], hq, hkv, dh, _ptr(scratch),
                                    0 if scratch is None else scratch.numel() * scratch.element_size(),
                                    None, _stream()), "bs_op_attention")
    return out


def lm_head_confidence_buffers(M: int, V: int, device) -> dict:
    """Buffers of op_lm_head_confidence, for callers that launch repeatedly."""
    nbytes = lib().bs_op_lm_head_confidence_scratch_bytes(M, V)
    return dict(scratch=torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device), nbytes=nbytes,
                tok=torch.empty(M, dtype=torch.int32, device=device),
                conf=torch.empty(M, dtype=torch.float32, device=device),
                flag=torch.zeros(1, dtype=torch.int32, device=device))


def op_lm_head_confidence(hf: torch.Tensor, W: torch.Tensor, row_scale: torch.Tensor, mask_id: int,
                          want_logits: bool = False, buffers: Optional[dict] = None):
    """LM head with the confidence pass in its epilogue: (tok int32 [M], conf fp32 [M], logits fp32 [M, V] or None).
    With `buffers` (from lm_head_confidence_buffers) nothing is allocated and the stream is not synchronised."""
    M, K = hf.shape
    V = W.shape[0]
    b = buffers or lm_head_confidence_buffers(M, V, hf.device)
    logits = torch.empty(M, V, dtype=torch.float32, device=hf.device) if want_logits else None
    _check_op(lib().bs_op_lm_head_confidence(hf.data_ptr(), hf.stride(0), W.data_ptr(), M, V, K, row_scale.data_ptr(),
                                             mask_id, b["scratch"].data_ptr(), b["nbytes"], b["tok"].data_ptr(),
                                             b["conf"].data_ptr(), _ptr(logits), b["flag"].data_ptr(), _stream()),
              "bs_op_lm_head_confidence")
    if buffers is None:
        torch.cuda.current_stream().synchronize()
        if int(b["flag"].item()):
            raise BlockServeError(BS_E_TIMEOUT, "a bounded device-side wait ran out")
    return b["tok"], b["conf"], logits


def op_confidence(logits: torch.Tensor, mask_id: int):
    n, V = logits.shape
    tok = torch.empty(n, dtype=torch.int32, device=logits.device)
    conf = torch.empty(n, dtype=torch.float32, device=logits.device)
    _check_op(lib().bs_op_confidence(logits.data_ptr(), n, V, mask_id, tok.data_ptr(), conf.data_ptr(), _stream()),
              "bs_op_confidence")
    return tok, conf


# ---- per-head norms with the rotation, and the 8-bit KV cache -----------------------------------------------------

KV8_BLOCK, KV8_MAX_ROWS = 32, 1024      # BS_KV8_BLOCK, BS_KV8_MAX_ROWS
_BF16, _F32, _I32, _E4M3, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)      # the handle alone: a fiftieth of the Stream object's cost
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _refuse(name: str, why: str) -> None:
    raise BlockServeError(BS_E_ARG, f"{name}: {why}")


def _need(name: str, dev: int, dtype: torch.dtype, least: int, args: str, *tensors) -> None:
    """Every tensor (named by the words of `args`): contiguous, on device `dev`, `dtype`, at least `least` elements."""
    for t in tensors:
        if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or t.numel() < least:
            arg = args.split()[next(i for i, u in enumerate(tensors) if u is t)]
            _refuse(name, f"{arg} must be a contiguous {dtype} tensor of at least {least} elements on the operator's "
                          f"device, got {tuple(t.shape)} {t.dtype} on {t.device}")


def _call(name: str, dev: int, fn, *args) -> None:
    """The library's kernels go to the current stream of the tensors' device, whatever device is current."""
    if dev < 0:
        _refuse(name, "the operators run on CUDA tensors only")
    if _current_device() == dev:
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc != BS_OK:
        _check_op(rc, name)


def rope_table(max_pos: int, dh: int, theta: float, device="cuda") -> torch.Tensor:
    """cos / sin table [max_pos, dh / 2, 2] of the operators below (angles evaluated in double): built once per model."""
    t = torch.empty(max_pos, dh // 2, 2, dtype=_F32)
    _check_op(lib().bs_rope_table(t.data_ptr(), max_pos, dh, theta), "bs_rope_table")
    return t.to(device)


def kv8_cache(kv_rows: int, hkv: int, dh: int, device="cuda"):
    """(k8, v8, k_scale, v_scale) of an 8-bit cache: e4m3 codes [kv_rows / 32, hkv, 32, dh] and one power-of-two scale
    for each block of 32 rows and head.  kv_rows is rounded up to whole blocks; the contents are not initialised (rows
    are valid once written)."""
    n = (kv_rows + KV8_BLOCK - 1) // KV8_BLOCK
    return (torch.empty(n, hkv, KV8_BLOCK, dh, dtype=_E4M3, device=device),
            torch.empty(n, hkv, KV8_BLOCK, dh, dtype=_E4M3, device=device),
            torch.empty(n, hkv, dtype=_F32, device=device), torch.empty(n, hkv, dtype=_F32, device=device))


def _kv8_shape(name: str, dev: int, k8, v8, k_scale, v_scale):
    """(kv_rows, kv heads, head_dim) of an 8-bit cache."""
    shape = k8.shape
    blocks, hkv, rows, dh = shape if len(shape) == 4 else (0, 0, 0, 0)
    scales = (blocks, hkv)
    if rows != KV8_BLOCK or v8.shape != shape or k_scale.shape != scales or v_scale.shape != scales:
        _refuse(name, "an 8-bit cache is codes [blocks, kv heads, 32, head_dim] and scales [blocks, kv heads]")
    # (all in one expression: a call of a small batch costs the host more than the device; what is wrong is found below)
    if not (k8.dtype is v8.dtype is _E4M3 and k_scale.dtype is v_scale.dtype is _F32 and blocks and hkv and dh and
            k8.get_device() == v8.get_device() == k_scale.get_device() == v_scale.get_device() == dev and
            k8.is_contiguous() and v8.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()):
        _need(name, dev, _E4M3, 1, "k8 v8", k8, v8)
        _need(name, dev, _F32, 1, "k_scale v_scale", k_scale, v_scale)
    return blocks * KV8_BLOCK, hkv, dh


def _rows_of(name: str, dev: int, args: str, cu, *tensors) -> int:
    """Number of rows of an index set: cu [n + 1] and tensors of at least n elements."""
    n = cu.numel() - 1
    if cu.dtype is not _I32 or n < 0 or cu.get_device() != dev or not cu.is_contiguous():
        _need(name, dev, _I32, 1, args, cu)
    for t in tensors:
        if t.dtype is not _I32 or t.numel() < n or t.get_device() != dev or not t.is_contiguous():
            _need(name, dev, _I32, n, args.partition(" ")[2], *tensors)
    return n


def _row_stride(name: str, dev: int, arg: str, t: torch.Tensor, rows: int, width: int) -> int:
    """Row stride of a bf16 matrix of at least `rows` rows of `width` adjacent elements."""
    shape = t.shape
    if len(shape) != 2 or t.dtype is not _BF16 or t.get_device() != dev or shape[0] < rows or shape[1] < width or \
            (t.stride(1) != 1 and t.numel() > 0):
        _refuse(name, f"{arg} must be a bfloat16 matrix of at least {rows} rows of {width} adjacent elements on the "
                      f"operator's device, got {tuple(t.shape)} {t.dtype} on {t.device}")
    if rows <= 1:
        return width
    ld = t.stride(0)
    if ld > 0x7fffffff:                       # (ctypes would pass its low bits on)
        _refuse(name, f"{arg}'s row stride of {ld} elements does not fit 31 bits")
    return ld


def _norm_inputs(name: str, dev: int, qkv, q_gain, k_gain, tok_pos, hq, hkv, dh, rope, q_out, error_flag):
    shape, width = qkv.shape, (hq + 2 * hkv) * dh
    if len(shape) != 2 or shape[1] != width or rope.dim() != 3 or rope.shape[1:] != (dh // 2, 2):
        _refuse(name, f"qkv must be [M, {width}] and rope_table [max_pos, {dh // 2}, 2]")
    M = shape[0]
    if not (qkv.dtype is _BF16 and tok_pos.dtype is _I32 and rope.dtype is _F32 and tok_pos.numel() >= M and
            qkv.get_device() == tok_pos.get_device() == rope.get_device() == dev and qkv.is_contiguous() and
            tok_pos.is_contiguous() and rope.is_contiguous() and rope.numel() >= dh):
        _need(name, dev, _BF16, 0, "qkv", qkv)
        _need(name, dev, _I32, M, "tok_pos", tok_pos)
        _need(name, dev, _F32, dh, "rope_table", rope)
    if (q_gain is None) != (k_gain is None):
        _refuse(name, "q_gain and k_gain are given together or not at all")
    if q_gain is not None:
        if not (q_gain.dtype is k_gain.dtype is _BF16 and q_gain.get_device() == k_gain.get_device() == dev and
                q_gain.is_contiguous() and k_gain.is_contiguous() and q_gain.numel() >= dh and k_gain.numel() >= dh):
            _need(name, dev, _BF16, dh, "q_gain k_gain", q_gain, k_gain)
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    if q_out is None:
        return M, torch.empty(M, hq * dh, dtype=_BF16, device=qkv.device), hq * dh
    return M, q_out, _row_stride(name, dev, "q_out", q_out, M, hq * dh)


def op_qk_norm_rope_kv(qkv, q_gain, k_gain, eps: float, tok_pos, tok_kv, kcache, vcache, hq: int, hkv: int, dh: int,
                       rope_table, q_out: Optional[torch.Tensor] = None,
                       error_flag: Optional[torch.Tensor] = None) -> torch.Tensor:
    """RMS norm of every query and key head (gains bf16 [dh], or None for both: no norm), rotation at tok_pos, K / V to
    rows tok_kv of the bf16 caches [kv_rows, hkv, dh] (tok_kv < 0: the token is skipped).  Returns the queries
    [M, hq * dh]; q_out = qkv rotates in place.  error_flag (int32 [1]) gets >= 100 where an index was out of range."""
    name, dev = "bs_op_qk_norm_rope_kv", qkv.get_device()
    M, q_out, ld = _norm_inputs(name, dev, qkv, q_gain, k_gain, tok_pos, hq, hkv, dh, rope_table, q_out, error_flag)
    shape = kcache.shape
    rows = shape[0] if len(shape) == 3 else 0
    if shape != (rows, hkv, dh) or vcache.shape != shape:
        _refuse(name, f"the caches must be [kv_rows, {hkv}, {dh}]")
    if not (kcache.dtype is vcache.dtype is _BF16 and tok_kv.dtype is _I32 and rows and tok_kv.numel() >= M and
            kcache.get_device() == vcache.get_device() == tok_kv.get_device() == dev and
            kcache.is_contiguous() and vcache.is_contiguous() and tok_kv.is_contiguous()):
        _need(name, dev, _BF16, 1, "kcache vcache", kcache, vcache)
        _need(name, dev, _I32, M, "tok_kv", tok_kv)
    _call(name, dev, (_lib or lib()).bs_op_qk_norm_rope_kv, qkv.data_ptr(), _ptr(q_gain), _ptr(k_gain), eps,
          tok_pos.data_ptr(), tok_kv.data_ptr(), q_out.data_ptr(), ld, kcache.data_ptr(), vcache.data_ptr(),
          rows, M, hq, hkv, dh, rope_table.data_ptr(), rope_table.shape[0], _ptr(error_flag))
    return q_out


def op_qk_norm_rope_kv8(qkv, q_gain, k_gain, eps: float, tok_pos, cu_q, kv_base, kv_at, kv_len, k8, v8, k_scale, v_scale,
                        hq: int, hkv: int, dh: int, rope_table, q_out: Optional[torch.Tensor] = None,
                        error_flag: Optional[torch.Tensor] = None) -> torch.Tensor:
    """op_qk_norm_rope_kv with the 8-bit cache of kv8_cache(): row i's tokens [cu_q[i], cu_q[i+1]) go to cache positions
    kv_at[i].. of its slab (kv_base[i], a multiple of 32), where positions [0, kv_len[i]) held valid rows before.
    Blocks it touches are re-scaled over everything valid in them."""
    name, dev = "bs_op_qk_norm_rope_kv8", qkv.get_device()
    M, q_out, ld = _norm_inputs(name, dev, qkv, q_gain, k_gain, tok_pos, hq, hkv, dh, rope_table, q_out, error_flag)
    rows, heads, width = _kv8_shape(name, dev, k8, v8, k_scale, v_scale)
    if heads != hkv or width != dh:
        _refuse(name, f"the cache holds {heads} heads of {width}, not {hkv} of {dh}")
    n = _rows_of(name, dev, "cu_q kv_base kv_at kv_len", cu_q, kv_base, kv_at, kv_len)
    _call(name, dev, (_lib or lib()).bs_op_qk_norm_rope_kv8, qkv.data_ptr(), _ptr(q_gain), _ptr(k_gain), eps,
          tok_pos.data_ptr(), cu_q.data_ptr(), kv_base.data_ptr(), kv_at.data_ptr(), kv_len.data_ptr(), n,
          q_out.data_ptr(), ld, k8.data_ptr(), v8.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), rows, M, hq, hkv, dh,
          rope_table.data_ptr(), rope_table.shape[0], _ptr(error_flag))
    return q_out


def op_kv8_read(k8, v8, k_scale, v_scale, cu, kv_base, kv_at, total: int, k_out: Optional[torch.Tensor] = None,
                v_out: Optional[torch.Tensor] = None, error_flag: Optional[torch.Tensor] = None):
    """Cache positions [kv_at[i], kv_at[i] + cu[i+1] - cu[i]) of every row, packed: bf16 (K, V) [total, hkv, dh]."""
    name, dev = "bs_op_kv8_read", k8.get_device()
    rows, hkv, dh = _kv8_shape(name, dev, k8, v8, k_scale, v_scale)
    n = _rows_of(name, dev, "cu kv_base kv_at", cu, kv_base, kv_at)
    if total < 0:
        _refuse(name, "total must not be negative")
    if k_out is None:
        k_out = torch.empty(total, hkv, dh, dtype=_BF16, device=k8.device)
    else:
        _need(name, dev, _BF16, total * hkv * dh, "k_out", k_out)
    if v_out is None:
        v_out = torch.empty_like(k_out) if k_out.shape == (total, hkv, dh) else k_out.new_empty(total, hkv, dh)
    else:
        _need(name, dev, _BF16, total * hkv * dh, "v_out", v_out)
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    _call(name, dev, (_lib or lib()).bs_op_kv8_read, k8.data_ptr(), v8.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
          rows, cu.data_ptr(), kv_base.data_ptr(), kv_at.data_ptr(), n, total, hkv, dh, k_out.data_ptr(), v_out.data_ptr(),
          _ptr(error_flag))
    return k_out, v_out


@functools.lru_cache(maxsize=None)
def attention_kv8_scratch_bytes(hq: int, hkv: int, dh: int) -> int:
    return max(256, lib().bs_op_attention_kv8_scratch_bytes(hq, hkv, dh))


@functools.lru_cache(maxsize=4096)
def _kv8_uses_scratch(n: int, M: int, max_nq: int, max_vis: int, hq: int, hkv: int, dh: int) -> bool:
    return lib().bs_op_attention_kv8_uses_scratch(n, M, max_nq, max_vis, hq, hkv, dh) != 0


def attention_kv8_scratch(hq: int, hkv: int, dh: int, device="cuda") -> torch.Tensor:
    """Scratch of op_attention_kv8, for callers that keep it (calls that share it must be ordered)."""
    return torch.empty(attention_kv8_scratch_bytes(hq, hkv, dh), dtype=_U8, device=device)


def op_attention_kv8(q, k8, v8, k_scale, v_scale, cu_q, kv_base, vis, hq: int, max_nq: int = 0, max_vis: int = 0,
                     scratch: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     error_flag: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of packed queries (q [M, >= hq * dh]: q_out of the operators above, or a qkv buffer) over their rows'
    cache positions [0, vis[i]) of the 8-bit cache; rows with vis = 0 give zeros.  max_nq / max_vis (0: unknown): the
    largest number of query tokens and of visible positions of a row: any value gives the same result, but calls without
    them can take several times as long.  Without `scratch` it comes from torch's allocator."""
    name, dev = "bs_op_attention_kv8", q.get_device()
    rows, hkv, dh = _kv8_shape(name, dev, k8, v8, k_scale, v_scale)
    M = q.shape[0]
    ld = _row_stride(name, dev, "q", q, M, hq * dh)
    n = _rows_of(name, dev, "cu_q kv_base vis", cu_q, kv_base, vis)
    if n > KV8_MAX_ROWS:
        _refuse(name, f"at most {KV8_MAX_ROWS} rows, got {n}")
    if out is None:
        out = torch.empty(M, hq * dh, dtype=_BF16, device=q.device)
    else:
        _need(name, dev, _BF16, M * hq * dh, "out", out)
    if scratch is not None:
        _need(name, dev, _U8, 0, "scratch", scratch)
    elif _kv8_uses_scratch(n, M, max_nq, max_vis, hq, hkv, dh):
        scratch = torch.empty(attention_kv8_scratch_bytes(hq, hkv, dh), dtype=_U8, device=q.device)
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    _call(name, dev, (_lib or lib()).bs_op_attention_kv8, q.data_ptr(), ld, k8.data_ptr(), v8.data_ptr(),
          k_scale.data_ptr(), v_scale.data_ptr(), rows, out.data_ptr(), cu_q.data_ptr(), kv_base.data_ptr(), vis.data_ptr(),
          n, M, max_nq, max_vis, hq, hkv, dh, _ptr(scratch),
          0 if scratch is None else scratch.numel(), _ptr(error_flag))
    return out


# ---- projections in 8-bit integers --------------------------------------------------------------------------------

I8_MAX_K, RULES_MAX_VOCAB = 131071, 524288      # BS_I8_MAX_K, BS_RULES_MAX_VOCAB
_I8 = torch.int8
_TYPES = {torch.bfloat16: 0, torch.float32: 1}  # BS_BF16, BS_F32


def _stride_of(t: torch.Tensor) -> int:
    """Row stride of a matrix of adjacent elements (a single row has the width's)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _rows_of_codes(name: str, dev: int, arg: str, t: torch.Tensor) -> int:
    """Row stride of an int8 matrix whose rows start at multiples of 16 bytes."""
    shape = t.shape
    if len(shape) != 2 or t.dtype is not _I8 or t.get_device() != dev or (shape[1] > 1 and t.stride(1) != 1):
        _refuse(name, f"{arg} must be an int8 matrix of adjacent elements on the operator's device, got {tuple(shape)} "
                      f"{t.dtype} on {t.device}")
    if shape[0] <= 1:
        return (shape[1] + 15) // 16 * 16
    return t.stride(0)


def i8_codes(rows: int, K: int, device="cuda") -> torch.Tensor:
    """Uninitialised int8 codes [rows, K] whose rows start at multiples of 16 bytes."""
    ld = (K + 15) // 16 * 16
    t = torch.empty(rows, ld, dtype=_I8, device=device)
    return t if ld == K else t[:, :K]


def op_quant_i8(x: torch.Tensor, gain: Optional[torch.Tensor] = None, eps: float = 1e-6, idx: Optional[torch.Tensor] = None,
                codes: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                error_flag: Optional[torch.Tensor] = None):
    """(codes int8 [M, K], scale fp32 [M]) of the rows of x (bf16 or fp32 [rows, K], any row stride), or of its rows
    idx[m]; with `gain` (bf16 [K]) of their RMS norms.  Weights are laid out by the same call: a row is an output channel.
    error_flag (int32 [1]) gets >= 100 where an idx was out of range (the row is left as it was)."""
    name, dev, shape = "bs_op_quant_i8", x.get_device(), x.shape
    type_ = _TYPES.get(x.dtype)
    if type_ is None or len(shape) != 2 or (shape[1] > 1 and x.stride(1) != 1):
        _refuse(name, f"x must be a bfloat16 or float32 matrix of adjacent elements, got {tuple(shape)} {x.dtype}")
    rows, K = shape
    M = rows
    if idx is not None:
        _need(name, dev, _I32, 0, "idx", idx)
        M = idx.numel()
    if gain is not None:
        _need(name, dev, _BF16, K, "gain", gain)
    if codes is None:
        ldc = (K + 15) // 16 * 16
        codes = torch.empty((M, ldc), dtype=_I8, device=x.device)
        if ldc != K:
            codes = codes[:, :K]
    else:
        if codes.shape != (M, K):
            _refuse(name, f"codes must be [{M}, {K}], got {tuple(codes.shape)}")
        ldc = _rows_of_codes(name, dev, "codes", codes)
    if scale is None:
        scale = torch.empty(M, dtype=_F32, device=x.device)
    elif scale.dtype is not _F32 or scale.get_device() != dev or not scale.is_contiguous() or scale.numel() < M:
        _need(name, dev, _F32, M, "scale", scale)
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    _call(name, dev, (_lib or lib()).bs_op_quant_i8, x.data_ptr(), type_, x.stride(0) if rows > 1 else K, _ptr(idx), rows,
          _ptr(gain), eps, codes.data_ptr(), ldc, scale.data_ptr(), M, K, _ptr(error_flag))
    return codes, scale


def op_gemm_i8(a: torch.Tensor, a_scale: torch.Tensor, W: torch.Tensor, w_scale: torch.Tensor, mode: int = 0,
               W2: Optional[torch.Tensor] = None, w2_scale: Optional[torch.Tensor] = None,
               C_out: Optional[torch.Tensor] = None, error_flag: Optional[torch.Tensor] = None) -> torch.Tensor:
    """z = (a @ W.T) * w_scale * a_scale[:, None] of int8 codes a [M, K], W [N, K] (rows at multiples of 16 bytes, as
    op_quant_i8 gives them), with the modes of op_gemm: 0 bf16, 1 added to fp32 C_out, 2 fp32, 3 bf16 silu(z) * z2 with
    W2 [N, K] and w2_scale."""
    name, dev = "bs_op_gemm_i8", a.get_device()
    lda, ldw = _rows_of_codes(name, dev, "a", a), _rows_of_codes(name, dev, "W", W)
    (M, K), (N, width) = a.shape, W.shape
    if width != K or (mode == 3) != (W2 is not None):
        _refuse(name, f"W must be [N, {K}], and W2 is given in mode 3 only")
    if not (a_scale.dtype is w_scale.dtype is _F32 and a_scale.get_device() == w_scale.get_device() == dev and
            a_scale.is_contiguous() and w_scale.is_contiguous() and a_scale.numel() >= M and w_scale.numel() >= N):
        _need(name, dev, _F32, M, "a_scale", a_scale)
        _need(name, dev, _F32, N, "w_scale", w_scale)
    if W2 is not None:
        if w2_scale is None or W2.shape != W.shape or _rows_of_codes(name, dev, "W2", W2) != ldw:
            _refuse(name, "W2 must have W's shape and strides, with w2_scale")
        _need(name, dev, _F32, N, "w2_scale", w2_scale)
    dtype = _F32 if mode in (1, 2) else _BF16
    if C_out is None:
        if mode == 1:
            _refuse(name, "mode 1 adds to C_out")
        C_out = torch.empty((M, N), dtype=dtype, device=a.device)
        ldc = N
    else:
        if C_out.shape != (M, N) or C_out.dtype is not dtype or C_out.get_device() != dev or (N > 1 and C_out.stride(1) != 1):
            _refuse(name, f"C_out must be a {dtype} matrix [{M}, {N}] of adjacent elements on the operator's device, got "
                          f"{tuple(C_out.shape)} {C_out.dtype} on {C_out.device}")
        ldc = _stride_of(C_out)
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    _call(name, dev, (_lib or lib()).bs_op_gemm_i8, a.data_ptr(), lda, a_scale.data_ptr(), W.data_ptr(), ldw, w_scale.data_ptr(),
          _ptr(W2), _ptr(w2_scale), C_out.data_ptr(), ldc, M, N, K, mode, _ptr(error_flag))
    return C_out


# ---- constrained decoding: rules on logits ------------------------------------------------------------------------

class LogitRules:
    """The rules of a batch, made once by logit_rules(); the tensors that it names are read at every call, so their
    contents may be updated in between."""

    __slots__ = ("struct", "ref", "tensors", "dev", "rows", "vocab")

    def __init__(self, struct: BsLogitRules, tensors, dev: int, rows: Optional[int]):
        self.struct, self.ref, self.tensors, self.dev, self.rows = struct, C.addressof(struct), tensors, dev, rows
        self.vocab = struct.vocab


def logit_rules(vocab: int, row_req: Optional[torch.Tensor], n_reqs: int, mask_id: int = -1, ctx: Optional[torch.Tensor] = None,
                ctx_begin: Optional[torch.Tensor] = None, ctx_gen: Optional[torch.Tensor] = None,
                ctx_end: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                presence: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                bias_at: Optional[torch.Tensor] = None, bias_tok: Optional[torch.Tensor] = None,
                bias_val: Optional[torch.Tensor] = None, allowed: Optional[torch.Tensor] = None,
                row_mask: Optional[torch.Tensor] = None) -> LogitRules:
    """Rules of constrained decoding for rows of logits [rows, vocab].

    row_req int32 [rows]: request of a row (-1: only the grammar applies; None: row r is request r).  Request i's context
    is ctx[ctx_begin[i] : ctx_end[i]] (int32), generated from ctx_gen[i] on; repetition, presence and frequency penalties
    fp32 [n_reqs]; its biases bias_val at the ascending tokens bias_tok, entries bias_at[i] .. bias_at[i + 1].  allowed
    int32 [masks, ceil(vocab / 32)]: bit v % 32 of word v // 32 set where token v is allowed; row_mask int32 [rows]: mask of
    a row (-1: none; None: row r has mask r).  mask_id is never chosen and not counted as context."""
    name = "logit_rules"
    given = [t for t in (row_req, ctx, ctx_begin, ctx_gen, ctx_end, repetition, presence, frequency, bias_at, bias_tok, bias_val,
                         allowed, row_mask) if t is not None]
    dev = given[0].get_device() if given else -1
    if dev < 0 and given:
        _refuse(name, "the rules' tensors are CUDA tensors")
    if not 1 <= vocab <= RULES_MAX_VOCAB or n_reqs < 0 or not -1 <= mask_id < vocab:
        _refuse(name, f"vocab must lie in [1, {RULES_MAX_VOCAB}], mask_id in [-1, vocab), got {vocab} and {mask_id}")
    rows = None                                   # most rows that the rules know, where they are listed by row
    for arg, t in (("row_req", row_req), ("row_mask", row_mask)):
        if t is not None:
            _need(name, dev, _I32, 0, arg, t)
            rows = t.numel() if rows is None else min(rows, t.numel())
    if row_req is None:
        rows = n_reqs if rows is None else min(rows, n_reqs)
    if ctx is not None:
        _need(name, dev, _I32, 0, "ctx", ctx)
        if ctx_begin is None or ctx_gen is None or ctx_end is None:
            _refuse(name, "ctx needs ctx_begin, ctx_gen and ctx_end")
        _need(name, dev, _I32, n_reqs, "ctx_begin ctx_gen ctx_end", ctx_begin, ctx_gen, ctx_end)
        _need(name, dev, _F32, n_reqs, "repetition presence frequency", *[t for t in (repetition, presence, frequency) if t is not None])
    elif not (ctx_begin is ctx_gen is ctx_end is repetition is presence is frequency is None):
        _refuse(name, "penalties need a context (ctx)")
    if bias_at is not None:
        if bias_tok is None or bias_val is None or bias_tok.numel() != bias_val.numel():
            _refuse(name, "bias_at needs bias_tok and bias_val of one length")
        _need(name, dev, _I32, n_reqs + 1, "bias_at", bias_at)
        _need(name, dev, _I32, 0, "bias_tok", bias_tok)
        _need(name, dev, _F32, 0, "bias_val", bias_val)
    elif bias_tok is not None or bias_val is not None:
        _refuse(name, "biases need bias_at")
    if allowed is not None:
        words = (vocab + 31) // 32
        if allowed.dim() != 2 or allowed.dtype is not _I32 or allowed.get_device() != dev or allowed.shape[1] < words or \
                allowed.stride(1) != 1:
            _refuse(name, f"allowed must be an int32 matrix of at least {words} adjacent words a mask on the operator's device")
        if row_mask is None:
            rows = allowed.shape[0] if rows is None else min(rows, allowed.shape[0])
    elif row_mask is not None:
        _refuse(name, "row_mask needs allowed")
    p = _ptr
    # (a tensor without elements has no address of its own, and NULL would be an absent rule)
    s = BsLogitRules(vocab, n_reqs, mask_id, p(row_req), p(ctx) or p(ctx_begin), 0 if ctx is None else ctx.numel(), p(ctx_begin),
                     p(ctx_gen), p(ctx_end), p(repetition), p(presence), p(frequency), p(bias_at), p(bias_tok), p(bias_val),
                     0 if bias_tok is None else bias_tok.numel(), p(allowed) or p(row_mask),
                     0 if allowed is None else (allowed.stride(0) if allowed.shape[0] > 1 else allowed.shape[1]),
                     0 if allowed is None else allowed.shape[0], p(row_mask))
    return LogitRules(s, given, dev, rows)


def _ruled_logits(name: str, logits: torch.Tensor, rules: LogitRules):
    """(device, type, row stride, rows) of logits that the rules fit."""
    dev, shape = logits.get_device(), logits.shape
    type_ = _TYPES.get(logits.dtype)
    if type_ is None or len(shape) != 2 or shape[1] != rules.vocab or (shape[1] > 1 and logits.stride(1) != 1):
        _refuse(name, f"logits must be a bfloat16 or float32 matrix [rows, {rules.vocab}] of adjacent elements, got "
                      f"{tuple(shape)} {logits.dtype}")
    if rules.dev not in (-1, dev):
        _refuse(name, "the rules' tensors are on another device than the logits")
    if rules.rows is not None and shape[0] > rules.rows:
        _refuse(name, f"{shape[0]} rows of logits, but rules for {rules.rows}")
    return dev, type_, _stride_of(logits), shape[0]


def op_logit_rules(logits: torch.Tensor, rules: LogitRules, out: Optional[torch.Tensor] = None,
                   error_flag: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The logits (fp32 or bf16 [rows, vocab]) after the rules: repetition, frequency and presence penalties, biases, then
    -inf where the grammar or mask_id forbids.  In place, or to `out` (the same type).  error_flag (int32 [1]) gets >= 100
    where an index was out of range."""
    name = "bs_op_logit_rules"
    dev, type_, ld, rows = _ruled_logits(name, logits, rules)
    if out is None:
        out = logits
    elif out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != dev or \
            (out.shape[1] > 1 and out.stride(1) != 1):
        _refuse(name, f"out must be a {logits.dtype} matrix {tuple(logits.shape)} of adjacent elements on the operator's device")
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    _call(name, dev, (_lib or lib()).bs_op_logit_rules, logits.data_ptr(), type_, ld, out.data_ptr(), _stride_of(out), rows,
          rules.ref, _ptr(error_flag))
    return out


def op_rules_confidence(logits: torch.Tensor, rules: LogitRules, tok: Optional[torch.Tensor] = None,
                        conf: Optional[torch.Tensor] = None, error_flag: Optional[torch.Tensor] = None):
    """op_confidence under the rules, without storing logits: (tok int32 [rows], conf fp32 [rows]); a row of which nothing
    is left gives -1 and 0."""
    name = "bs_op_rules_confidence"
    dev, type_, ld, rows = _ruled_logits(name, logits, rules)
    if tok is None:
        tok = torch.empty(rows, dtype=_I32, device=logits.device)
    else:
        _need(name, dev, _I32, rows, "tok", tok)
    if conf is None:
        conf = torch.empty(rows, dtype=_F32, device=logits.device)
    else:
        _need(name, dev, _F32, rows, "conf", conf)
    if error_flag is not None:
        _need(name, dev, _I32, 1, "error_flag", error_flag)
    _call(name, dev, (_lib or lib()).bs_op_rules_confidence, logits.data_ptr(), type_, ld, rows, rules.ref, tok.data_ptr(),
          conf.data_ptr(), _ptr(error_flag))
    return tok, conf
