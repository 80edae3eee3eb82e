"""ctypes binding of libpvf.so: the same calls as include/pvf.h, arguments marshalled from
torch tensors (device memory) and Python numbers.  No step of the method runs here.

The library must have been built (paper_2601_12247_amd/build.py); loading fails loudly
otherwise.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpvf.so")

PVF_F32, PVF_BF16 = 0, 1
MX_E4M3, MX_E2M1 = 0, 1   # PVF_MX_E4M3, PVF_MX_E2M1
MX_GEMM, MX_SWIGLU, MX_W4 = 0, 1, 2   # PVF_MX_CALL_*
PVF_ROUTES_PLAN, PVF_ROUTES_AR, PVF_ROUTES_CAL, PVF_ROUTES_XRANDOM, PVF_ROUTES_XPLANNING = 1, 2, 4, 8, 16
PVF_ROUTE_NONE, PVF_ROUTE_PLAN, PVF_ROUTE_AR, PVF_ROUTE_CAL = 0, 1, 2, 3
ROUTE_NONE, ROUTE_PLAN, ROUTE_AR = 0, 1, 2
PAGE_WORKSPACE = 1 << 26   # PVF_PAGE_WORKSPACE
MAX_K = 32          # PVF_MAX_K of include/pvf.h
STATUS = {0: "PVF_OK", -1: "PVF_EINVAL", -2: "PVF_ESHAPE", -3: "PVF_ENOMEM", -4: "PVF_EHIP",
          -5: "PVF_ENOTIMPL"}

# every symbol include/pvf.h declares
EXPORTS = ["pvf_create", "pvf_destroy", "pvf_last_error", "pvf_workspace_bytes", "pvf_profile_begin",
           "pvf_profile_end", "pvf_forward",
           "pvf_epilogue", "pvf_round", "pvf_state_init", "pvf_decode", "pvf_stage1", "pvf_gemm",
           "pvf_gemm_swiglu", "pvf_rmsnorm", "pvf_rope_attention", "pvf_fill_normal", "pvf_entropy",
           "pvf_plan_vocab_select", "pvf_qkv_attention", "pvf_rope_attention_noalloc", "pvf_round_sync", "pvf_ctx_gemm",
           "pvf_ctx_gemm_swiglu", "pvf_quant_mx", "pvf_add_rmsnorm_mx", "pvf_gemm_mx", "pvf_gemm_mx_swiglu", "pvf_gemm_w4",
           "pvf_gemm_mx_instance", "pvf_page_extend", "pvf_page_trim", "pvf_page_store", "pvf_page_attention_workspace",
           "pvf_page_attention"]


class PvfError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class ModelCfgC(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("d_ff", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("mask_id", C.c_int32)]


class DecodeCfgC(C.Structure):
    _fields_ = [("tau_high", C.c_float), ("tau_plan_lo", C.c_float), ("tau_plan_hi", C.c_float),
                ("tau_ar_lo", C.c_float), ("logit_scale", C.c_float), ("K", C.c_int32),
                ("block_len", C.c_int32), ("prompt_len", C.c_int32), ("gen_len", C.c_int32),
                ("routes", C.c_int32), ("n_sparse", C.c_int32), ("seed", C.c_uint32), ("kv_cache", C.c_int32)]


class WeightsC(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("out_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("attn_norm", C.POINTER(C.c_void_p)), ("wqkv", C.POINTER(C.c_void_p)),
                ("wo", C.POINTER(C.c_void_p)), ("ffn_norm", C.POINTER(C.c_void_p)),
                ("w_gate_up", C.POINTER(C.c_void_p)), ("w_down", C.POINTER(C.c_void_p))]


class StateC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("canvas", "n_drafts", "draft_route", "fill_pos", "fill_tok", "k_active", "n_ws_blocks",
                 "conf",
                 "tok", "accept", "winner", "n_commit", "done", "ent", "dh", "cal_n", "cal_m", "cal_a",
                 "cal_vig")]


class StatsC(C.Structure):
    _fields_ = [("rounds", C.c_int32), ("seq_forwards", C.c_int32), ("n_base", C.c_int64),
                ("n_plan", C.c_int64), ("n_ar", C.c_int64), ("drafts_proposed", C.c_int64),
                ("drafts_accepted", C.c_int64), ("ms_total", C.c_double)]


PROF_CATEGORIES = ("gemm", "attention", "stage1", "forward", "stage2")


class ProfileC(C.Structure):
    _fields_ = [("ms", C.c_double * 5), ("flops", C.c_double * 5), ("bytes", C.c_double * 5),
                ("launches", C.c_int64 * 5)]


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2601_12247_amd.build` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        L.pvf_last_error.restype = C.c_char_p
        L.pvf_last_error.argtypes = [C.c_void_p]
        L.pvf_workspace_bytes.restype = C.c_int64
        L.pvf_workspace_bytes.argtypes = [C.c_void_p]
        L.pvf_destroy.restype = None
        L.pvf_destroy.argtypes = [C.c_void_p]
        L.pvf_profile_begin.argtypes = [C.c_void_p]
        L.pvf_profile_end.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(ProfileC)]
        L.pvf_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(ModelCfgC), C.POINTER(WeightsC),
                                 C.c_int32, C.c_int32, C.c_int32]
        L.pvf_forward.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                  C.c_void_p, C.c_int32, C.c_void_p]
        L.pvf_epilogue.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                   C.c_int32, C.c_int32, C.c_void_p, C.POINTER(DecodeCfgC),
                                   C.POINTER(StateC)]
        L.pvf_round.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                C.POINTER(DecodeCfgC), C.POINTER(StateC), C.c_int32]
        L.pvf_round_sync.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                     C.POINTER(DecodeCfgC), C.POINTER(StateC), C.c_int32, C.POINTER(C.c_int32)]
        L.pvf_state_init.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                     C.POINTER(DecodeCfgC), C.POINTER(StateC)]
        L.pvf_decode.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                 C.POINTER(DecodeCfgC), C.POINTER(StateC), C.c_void_p,
                                 C.POINTER(StatsC)]
        L.pvf_stage1.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int32,
                                 C.c_int32, C.c_float, C.c_void_p, C.c_void_p]
        L.pvf_entropy.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int32,
                                  C.c_int32, C.c_float, C.c_void_p]
        L.pvf_plan_vocab_select.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                            C.c_int32, C.c_int32, C.c_uint32, C.c_uint32, C.c_float,
                                            C.c_float, C.c_void_p]
        L.pvf_gemm.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                               C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
        L.pvf_ctx_gemm.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
        L.pvf_ctx_gemm_swiglu.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_int32, C.c_int32, C.c_int32]
        L.pvf_gemm_swiglu.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_int32, C.c_int32, C.c_int32]
        L.pvf_rmsnorm.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_int32, C.c_int32, C.c_float]
        L.pvf_rope_attention.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32,
                                         C.c_int32, C.c_int32, C.c_int32, C.c_float]
        L.pvf_rope_attention_noalloc.argtypes = L.pvf_rope_attention.argtypes
        L.pvf_qkv_attention.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_float]
        L.pvf_quant_mx.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32]
        L.pvf_add_rmsnorm_mx.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_int32, C.c_int32, C.c_float]
        L.pvf_gemm_mx.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
        L.pvf_gemm_mx_swiglu.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
        L.pvf_gemm_w4.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_int32, C.c_int32, C.c_int32]
        L.pvf_gemm_mx_instance.argtypes = [C.c_int32] * 7 + [C.POINTER(C.c_int32)] * 2
        p, i, i64, f = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        L.pvf_page_extend.argtypes = [p, p, p, p, i, p, i, i64, i, p, i, p, i] + [p] * 7
        L.pvf_page_trim.argtypes = [p, p, p, i, p, i, i64, i, p, i, p, p, p, p]
        L.pvf_page_store.argtypes = [p, i, p, i64, p, p, i, i, i, i, f, p, i64, p, p, i, i, i64, i64]
        L.pvf_page_attention_workspace.argtypes = [i] * 8
        L.pvf_page_attention_workspace.restype = i64
        L.pvf_page_attention.argtypes = [p, i, p, i64, p, p, i, i, i64, i64, p, i, i64, p, p, i, i, i, i, i, i, f, p, i64, p, i64]
        L.pvf_fill_normal.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_uint64,
                                      C.c_float, C.c_float]
        for name in EXPORTS:
            fn = getattr(L, name)
            if name not in ("pvf_last_error", "pvf_workspace_bytes", "pvf_destroy", "pvf_page_attention_workspace"):
                fn.restype = C.c_int32
        _lib = L
    return _lib


def _check(status: int, ctx: Optional[int] = None) -> None:
    if status != 0:
        raise PvfError(status, lib().pvf_last_error(ctx).decode())


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return PVF_F32
    if t == torch.bfloat16:
        return PVF_BF16
    raise TypeError(f"unsupported dtype {t}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensor required"
    return t.data_ptr()


@dataclass
class DecodeCfg:
    block_len: int
    prompt_len: int
    gen_len: int
    tau_high: float = 0.9
    tau_plan_lo: float = 0.2
    tau_plan_hi: float = 0.65
    tau_ar_lo: float = 0.1
    logit_scale: float = 1.0
    K: int = 3
    routes: int = 3
    n_sparse: int = 0
    seed: int = 0
    kv_cache: int = 0

    @property
    def T(self) -> int:
        return self.prompt_len + self.gen_len

    @property
    def R(self) -> int:
        return min((4 if self.n_sparse > 0 else 2) * self.block_len, self.gen_len)

    def c(self) -> DecodeCfgC:
        return DecodeCfgC(self.tau_high, self.tau_plan_lo, self.tau_plan_hi, self.tau_ar_lo,
                          self.logit_scale, self.K, self.block_len, self.prompt_len, self.gen_len,
                          self.routes, self.n_sparse, self.seed, self.kv_cache)


class State:
    """Device buffers of pvf_state for G groups (allocated with torch)."""

    def __init__(self, G: int, cfg: DecodeCfg, device="cuda", vocab: Optional[int] = None):
        K, T, R = cfg.K, cfg.T, cfg.R
        i32 = dict(dtype=torch.int32, device=device)
        self.G, self.cfg = G, cfg
        self.canvas = torch.zeros(G, 1 + K, T, **i32)
        self.n_drafts = torch.zeros(G, **i32)
        self.draft_route = torch.zeros(G, **i32)
        self.fill_pos = torch.full((G, max(K, 1)), -1, **i32)
        self.fill_tok = torch.full((G, max(K, 1)), -1, **i32)
        self.k_active = torch.zeros(G, **i32)
        self.n_ws_blocks = torch.ones(G, **i32)
        self.conf = torch.zeros(G, 1 + K, R, dtype=torch.float32, device=device)
        self.tok = torch.zeros(G, 1 + K, R, **i32)
        self.accept = torch.zeros(G, max(K, 1), dtype=torch.uint8, device=device)
        self.winner = torch.zeros(G, **i32)
        self.n_commit = torch.zeros(G, 3, **i32)
        self.done = torch.zeros(G, **i32)
        # calibration members (App. A.2): allocated only for the calibration trajectory
        self.ent = self.dh = self.cal_n = self.cal_m = self.cal_a = self.cal_vig = None
        if cfg.routes & PVF_ROUTES_CAL:
            assert vocab is not None, "the calibration trajectory needs vocab for the token statistics"
            self.ent = torch.zeros(G, 1 + K, R, dtype=torch.float32, device=device)
            self.dh = torch.zeros(G, max(K, 1), dtype=torch.float64, device=device)
            self.cal_n = torch.zeros(vocab, **i32)
            self.cal_m = torch.zeros(vocab, **i32)
            self.cal_a = torch.zeros(vocab, **i32)
            self.cal_vig = torch.zeros(vocab, dtype=torch.float64, device=device)

    def c(self) -> StateC:
        return StateC(*[_ptr(getattr(self, n)) for n, _ in StateC._fields_])

    def live_seqs(self) -> int:
        """sum over live groups of 1 + n_drafts (synchronises)."""
        nd, dn = self.n_drafts.cpu(), self.done.cpu()
        return int(((1 + nd) * (1 - dn)).sum())


class Context:
    """pvf_ctx: keeps the weight tensors alive and owns the library workspace."""

    def __init__(self, n_layers: int, d_model: int, n_heads: int, d_ff: int, vocab: int,
                 mask_id: int, weights: Dict, max_seqs: int, max_T: int, max_rows: int,
                 rms_eps: float = 1e-5, rope_theta: float = 10000.0):
        self.weights = weights
        dt = weights["embed"].dtype
        self.dtype = dt
        self.vocab, self.mask_id, self.d_model = vocab, mask_id, d_model
        self.model = ModelCfgC(n_layers, d_model, n_heads, d_ff, vocab, _dtype_code(dt), rms_eps,
                               rope_theta, mask_id)
        layers: List[Dict] = weights["layers"]
        assert len(layers) == n_layers

        def arr(name):
            a = (C.c_void_p * n_layers)(*[_ptr(l[name]) for l in layers])
            return a

        self._arrs = {n: arr(n) for n in ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down")}
        wc = WeightsC(_ptr(weights["embed"]), _ptr(weights["out_head"]), _ptr(weights["final_norm"]),
                      *[C.cast(self._arrs[n], C.POINTER(C.c_void_p)) for n in
                        ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down")])
        h = C.c_void_p()
        _check(lib().pvf_create(C.byref(h), C.byref(self.model), C.byref(wc), max_seqs, max_T, max_rows))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().pvf_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def workspace_bytes(self) -> int:
        return lib().pvf_workspace_bytes(self.handle)

    def profile_begin(self) -> None:
        _check(lib().pvf_profile_begin(self.handle), self.handle)

    def profile_end(self) -> Dict[str, Dict[str, float]]:
        p = ProfileC()
        _check(lib().pvf_profile_end(self.handle, _stream(), C.byref(p)), self.handle)
        return {name: {"ms": p.ms[i], "flops": p.flops[i], "bytes": p.bytes[i], "launches": p.launches[i]}
                for i, name in enumerate(PROF_CATEGORIES)}

    # ---- GEMMs as the context launches them (weight-streaming kernels for few rows) ----
    def gemm(self, A: torch.Tensor, W: torch.Tensor, residual: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
        M, K = A.shape
        N = W.shape[0]
        assert W.shape[1] == K and A.dtype == self.dtype
        if out is None:
            out = torch.empty(M, N, dtype=A.dtype, device=A.device)
        _check(lib().pvf_ctx_gemm(self.handle, _stream(), _ptr(A), _ptr(W), _ptr(out), _ptr(residual), M, N, K),
               self.handle)
        return out

    def gemm_swiglu(self, A: torch.Tensor, W: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        M, K = A.shape
        ff = W.shape[0] // 2
        if out is None:
            out = torch.empty(M, ff, dtype=A.dtype, device=A.device)
        _check(lib().pvf_ctx_gemm_swiglu(self.handle, _stream(), _ptr(A), _ptr(W), _ptr(out), M, ff, K), self.handle)
        return out

    # ---- the four calls -------------------------------------------------------------
    def forward(self, tokens: torch.Tensor, row_pos: torch.Tensor) -> torch.Tensor:
        S, T = tokens.shape
        R = row_pos.shape[1]
        logits = torch.empty(S, R, self.vocab, dtype=self.dtype, device=tokens.device)
        _check(lib().pvf_forward(self.handle, _stream(), _ptr(tokens), S, T, _ptr(row_pos), R,
                                 _ptr(logits)), self.handle)
        return logits

    def round(self, state: State, plan_bitmap: torch.Tensor, n_seq: int = 0) -> None:
        cfgc, stc = state.cfg.c(), state.c()
        _check(lib().pvf_round(self.handle, _stream(), state.G, _ptr(plan_bitmap), C.byref(cfgc),
                               C.byref(stc), n_seq), self.handle)

    def round_sync(self, state: State, plan_bitmap: torch.Tensor, n_seq: int = 0):
        """pvf_round_sync: one round and its status words; returns a list of G tuples
        (done, n_drafts, committed by threshold, by planning, by AR)."""
        cfgc, stc = state.cfg.c(), state.c()
        buf = (C.c_int32 * (5 * state.G))()
        _check(lib().pvf_round_sync(self.handle, _stream(), state.G, _ptr(plan_bitmap), C.byref(cfgc),
                                    C.byref(stc), n_seq, buf), self.handle)
        return [tuple(buf[5 * g: 5 * g + 5]) for g in range(state.G)]

    def state_init(self, state: State, prompt: torch.Tensor) -> None:
        cfgc, stc = state.cfg.c(), state.c()
        _check(lib().pvf_state_init(self.handle, _stream(), _ptr(prompt), state.G, C.byref(cfgc),
                                    C.byref(stc)), self.handle)

    def decode(self, state: State, prompt: torch.Tensor, plan_bitmap: torch.Tensor):
        cfgc, stc, stats = state.cfg.c(), state.c(), StatsC()
        out = torch.empty(state.G, state.cfg.T, dtype=torch.int32, device=prompt.device)
        _check(lib().pvf_decode(self.handle, _stream(), _ptr(prompt), state.G, _ptr(plan_bitmap),
                                C.byref(cfgc), C.byref(stc), _ptr(out), C.byref(stats)), self.handle)
        return out, stats


def epilogue(logits: torch.Tensor, state: State, plan_bitmap: torch.Tensor, vocab: int,
             mask_id: int, ctx: Optional[Context] = None) -> None:
    """pvf_epilogue over logits [G, 1+K, R, V]."""
    cfgc, stc = state.cfg.c(), state.c()
    h = ctx.handle if ctx is not None else None
    _check(lib().pvf_epilogue(h, _stream(), _ptr(logits), _dtype_code(logits.dtype), state.G, vocab,
                              mask_id, _ptr(plan_bitmap), C.byref(cfgc), C.byref(stc)), h)


# ---- building blocks ---------------------------------------------------------------------
def stage1(logits: torch.Tensor, mask_id: int, logit_scale: float, conf: Optional[torch.Tensor] = None,
           tok: Optional[torch.Tensor] = None):
    n, V = logits.shape
    if conf is None:
        conf = torch.empty(n, dtype=torch.float32, device=logits.device)
    if tok is None:
        tok = torch.empty(n, dtype=torch.int32, device=logits.device)
    _check(lib().pvf_stage1(_stream(), _ptr(logits), _dtype_code(logits.dtype), n, V, mask_id,
                            logit_scale, _ptr(conf), _ptr(tok)))
    return conf, tok


def entropy(logits: torch.Tensor, mask_id: int, logit_scale: float = 1.0) -> torch.Tensor:
    """H_i (nats) of softmax(logit_scale * logits[i]) over all ids but mask_id; logits [n, V]."""
    n, V = logits.shape
    ent = torch.empty(n, dtype=torch.float32, device=logits.device)
    _check(lib().pvf_entropy(_stream(), _ptr(logits), _dtype_code(logits.dtype), n, V, mask_id,
                             logit_scale, _ptr(ent)))
    return ent


def plan_vocab_select(cal_n: torch.Tensor, cal_m: torch.Tensor, cal_a: torch.Tensor, cal_vig: torch.Tensor,
                      mask_id: int, n_min: int = 50, m_min: int = 20, rho_ver: float = 0.9,
                      gamma_vig: float = 0.03) -> torch.Tensor:
    """Filtering rule of App. A.2 on the accumulated token statistics -> planning bitmap."""
    V = cal_n.numel()
    bitmap = torch.empty((V + 31) // 32, dtype=torch.int32, device=cal_n.device)
    _check(lib().pvf_plan_vocab_select(_stream(), _ptr(cal_n), _ptr(cal_m), _ptr(cal_a), _ptr(cal_vig), V,
                                       mask_id, n_min, m_min, rho_ver, gamma_vig, _ptr(bitmap)))
    return bitmap


def gemm(A: torch.Tensor, W: torch.Tensor, residual: Optional[torch.Tensor] = None,
         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    M, K = A.shape
    N = W.shape[0]
    assert W.shape[1] == K
    if out is None:
        out = torch.empty(M, N, dtype=A.dtype, device=A.device)
    _check(lib().pvf_gemm(_stream(), _dtype_code(A.dtype), _ptr(A), _ptr(W), _ptr(out),
                          _ptr(residual), M, N, K))
    return out


def gemm_swiglu(A: torch.Tensor, W: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    M, K = A.shape
    ff = W.shape[0] // 2
    if out is None:
        out = torch.empty(M, ff, dtype=A.dtype, device=A.device)
    _check(lib().pvf_gemm_swiglu(_stream(), _dtype_code(A.dtype), _ptr(A), _ptr(W), _ptr(out), M, ff, K))
    return out


def rmsnorm(x: torch.Tensor, gain: torch.Tensor, eps: float) -> torch.Tensor:
    M, d = x.shape
    out = torch.empty_like(x)
    _check(lib().pvf_rmsnorm(_stream(), _dtype_code(x.dtype), _ptr(x), _ptr(gain), _ptr(out), M, d, eps))
    return out


# ---- block-scaled rows -------------------------------------------------------------------
# Codes are float8_e4m3fn tensors [rows, Kp], or uint8 [rows, Kp / 2] with two e2m1 codes a byte (even element low); scales are
# float8_e8m0fnu tensors [Kp / 128, rows, 4]; Kp = mx_width(K).
def mx_width(K: int) -> int:
    return (K + 127) // 128 * 128


def mx_empty(rows: int, K: int, fmt: int = MX_E4M3, device="cuda"):
    """Uninitialised codes and scales for rows of K elements."""
    Kp = mx_width(K)
    codes = (torch.empty(rows, Kp, dtype=torch.float8_e4m3fn, device=device) if fmt == MX_E4M3 else
             torch.empty(rows, Kp // 2, dtype=torch.uint8, device=device))
    return codes, torch.empty(Kp // 128, rows, 4, dtype=torch.float8_e8m0fnu, device=device)


def _mx_format(codes: torch.Tensor, scales: torch.Tensor, rows: int, Kp: int) -> int:
    """The format of checked codes and scales."""
    if codes.dtype is torch.float8_e4m3fn:
        fmt, width = MX_E4M3, Kp
    else:
        assert codes.dtype is torch.uint8, f"codes are float8_e4m3fn or uint8, not {codes.dtype}"
        fmt, width = MX_E2M1, Kp // 2
    assert codes.shape == (rows, width), f"codes of {rows} rows of {Kp}: {tuple(codes.shape)}"
    assert scales.dtype is torch.float8_e8m0fnu and scales.shape == (Kp // 128, rows, 4), \
        f"scales of {rows} rows of {Kp}: {scales.dtype} {tuple(scales.shape)}"
    return fmt


def _mx_call(fn, tensors, *args) -> None:
    """fn(stream, *args) on the device that the tensors are on.  Costs a microsecond beside the launch, so the device and its stream are asked
    for as numbers: torch.cuda.current_stream() takes three."""
    dev = tensors[0].get_device()
    for t in tensors:
        assert t is None or (t.get_device() == dev and t.is_contiguous()), "contiguous tensors on one device required"
    assert dev >= 0, "device-resident tensors required"
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            status = fn(torch._C._cuda_getCurrentRawStream(dev), *args)
    else:
        status = fn(torch._C._cuda_getCurrentRawStream(dev), *args)
    if status:
        _check(status)


def _p(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def quant_mx(x: torch.Tensor, fmt: int = MX_E4M3, out=None):
    """(codes, scales) of rows x [M, K] in MX_E4M3 or MX_E2M1; out = (codes, scales) to write into (mx_empty)."""
    M, K = x.shape
    codes, scales = mx_empty(M, K, fmt, x.device) if out is None else out
    assert _mx_format(codes, scales, M, mx_width(K)) == fmt, "out is of the other format"
    _mx_call(lib().pvf_quant_mx, (x, codes, scales), _dtype_code(x.dtype), x.data_ptr(), fmt, codes.data_ptr(), scales.data_ptr(), M, K)
    return codes, scales


def add_rmsnorm_mx(x: torch.Tensor, gain: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                   sum_out: Optional[torch.Tensor] = None, out=None):
    """(h, codes, scales): h = x + residual (x itself without a residual), codes and scales (MX_E4M3) of RMSNorm(h) * gain.
    sum_out (may be x or residual) receives h; out = (codes, scales)."""
    M, d = x.shape
    codes, scales = mx_empty(M, d, MX_E4M3, x.device) if out is None else out
    assert _mx_format(codes, scales, M, mx_width(d)) == MX_E4M3, "the norm writes MX_E4M3"
    if residual is not None and sum_out is None:
        sum_out = torch.empty_like(x)
    dtype, shape = x.dtype, x.shape
    assert gain.dtype is dtype and gain.shape == (d,), "gain is [d] of x's type"
    assert residual is None or (residual.dtype is dtype and residual.shape == shape), "the residual is like x"
    assert sum_out is None or (sum_out.dtype is dtype and sum_out.shape == shape), "the sum is like x"
    _mx_call(lib().pvf_add_rmsnorm_mx, (x, residual, gain, sum_out, codes, scales), _dtype_code(x.dtype), x.data_ptr(), _p(residual),
             gain.data_ptr(), _p(sum_out), codes.data_ptr(), scales.data_ptr(), M, d, eps)
    return x if sum_out is None else sum_out, codes, scales


def gemm_mx(A: torch.Tensor, a_scales: torch.Tensor, W: torch.Tensor, w_scales: torch.Tensor,
            residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """A W^T (+ residual) of MX_E4M3 rows A and weights W in either format; `dtype` where neither out nor residual has one."""
    (M, Kp), N = A.shape, W.shape[0]
    assert _mx_format(A, a_scales, M, Kp) == MX_E4M3 and Kp % 128 == 0, "A is MX_E4M3"
    fmt = _mx_format(W, w_scales, N, Kp)
    if out is None:
        out = torch.empty(M, N, dtype=dtype if residual is None else residual.dtype, device=A.device)
    assert out.shape == (M, N), "the result is [M, N]"
    assert residual is None or (residual.dtype is out.dtype and residual.shape == out.shape), "the residual is like the result"
    _mx_call(lib().pvf_gemm_mx, (A, a_scales, W, w_scales, out, residual), fmt, _dtype_code(out.dtype), A.data_ptr(), a_scales.data_ptr(),
             W.data_ptr(), w_scales.data_ptr(), out.data_ptr(), _p(residual), M, N, Kp)
    return out


def gemm_mx_swiglu(A: torch.Tensor, a_scales: torch.Tensor, W: torch.Tensor, w_scales: torch.Tensor, out=None):
    """(codes, scales), MX_E4M3, of silu(A W_gate^T) * (A W_up^T), W [2 * ff, Kp] (rows gate | up); out = (codes, scales)."""
    (M, Kp), ff = A.shape, W.shape[0] // 2
    assert _mx_format(A, a_scales, M, Kp) == MX_E4M3 and Kp % 128 == 0, "A is MX_E4M3"
    assert W.shape[0] == 2 * ff, "rows gate | up"
    fmt = _mx_format(W, w_scales, 2 * ff, Kp)
    codes, scales = mx_empty(M, ff, MX_E4M3, A.device) if out is None else out
    assert _mx_format(codes, scales, M, mx_width(ff)) == MX_E4M3, "the activation is MX_E4M3"
    _mx_call(lib().pvf_gemm_mx_swiglu, (A, a_scales, W, w_scales, codes, scales), fmt, A.data_ptr(), a_scales.data_ptr(), W.data_ptr(),
             w_scales.data_ptr(), codes.data_ptr(), scales.data_ptr(), M, ff, Kp)
    return codes, scales


def gemm_w4(x: torch.Tensor, W: torch.Tensor, w_scales: torch.Tensor, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x W^T (+ residual) of rows x [M, K] (float32 / bfloat16) and MX_E2M1 weights."""
    (M, K), N = x.shape, W.shape[0]
    assert _mx_format(W, w_scales, N, mx_width(K)) == MX_E2M1, "W is MX_E2M1"
    if out is None:
        out = torch.empty(M, N, dtype=x.dtype, device=x.device)
    assert out.dtype is x.dtype and out.shape == (M, N), "the result is [M, N] of x's type"
    assert residual is None or (residual.dtype is x.dtype and residual.shape == out.shape), "the residual is like the result"
    _mx_call(lib().pvf_gemm_w4, (x, W, w_scales, out, residual), _dtype_code(x.dtype), x.data_ptr(), W.data_ptr(), w_scales.data_ptr(),
             out.data_ptr(), _p(residual), M, N, K)
    return out


def gemm_mx_instance(call: int, M: int, N: int, K: int, w_fmt: int = MX_E4M3, dtype: torch.dtype = torch.bfloat16, aligned: bool = True):
    """(index, count): the kernel instance that gemm_mx, gemm_mx_swiglu (N = ff) or gemm_w4 (call = MX_GEMM, MX_SWIGLU, MX_W4) takes, of those that
    it chooses from; aligned: whether x of gemm_w4 begins at a multiple of 16 bytes."""
    index, count = C.c_int32(), C.c_int32()
    _check(lib().pvf_gemm_mx_instance(call, w_fmt, _dtype_code(dtype), int(aligned), M, N, K, C.byref(index), C.byref(count)))
    return index.value, count.value


# ---- keys and values in pages --------------------------------------------------------------
# A cache is a pair of tensors [n_pages, Hkv, page_size, d_head], pages contiguous but for the distance between them (stride(0)); a table is
# int32 [B, width], its rows apart by stride(0): the library refuses a table whose rows overlap, as an expanded one's do (one row for all requests: copy it).
# Lengths, counts, positions and slots are int32.  Tables may be of pages of any size, page_store and page_attention take multiples of 8.  These calls may stand in a loop of single tokens, where what a check costs counts:
# conditions are written out in one expression, and what does not fit is looked at again to say what it was.
_i32_t = torch.int32


def _misfit(dev: int, sizes) -> None:
    """Says which of the (name, tensor, elements) does not fit: contiguous int32 tensors on device dev."""
    assert dev >= 0, "device-resident tensors required"
    for name, t, n in sizes:
        assert t.dtype is _i32_t and t.numel() == n and t.is_contiguous() and t.get_device() == dev, \
            f"{name}: int32 [{n}] on device {dev} required, not {t.dtype} {tuple(t.shape)} on {t.device}"
    raise AssertionError("the table is int32 [B, width] beside the lengths, its rows contiguous")


def _page_call(fn, dev: int, args) -> None:
    """fn(stream, *args) on device dev."""
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            status = fn(torch._C._cuda_getCurrentRawStream(dev), *args)
    else:
        status = fn(torch._C._cuda_getCurrentRawStream(dev), *args)
    if status:
        _check(status)


def _check_cache(k: torch.Tensor, v: torch.Tensor, dtype: torch.dtype, dev: int) -> None:
    assert dev >= 0, "device-resident tensors required"
    assert k.dim() == 4 and v.shape == k.shape and k.dtype is dtype and v.dtype is dtype and k.get_device() == dev and v.get_device() == dev, \
        "caches are [n_pages, Hkv, page_size, d_head] of the rows' type, beside them"
    _, Hkv, P, dh = k.shape
    for c in (k, v):
        s = c.stride()
        assert (dh == 1 or s[3] == 1) and (P == 1 or s[2] == dh) and (Hkv == 1 or s[1] == P * dh), "what is in a page is contiguous"


def _check_rows(x: torch.Tensor, shape, dtype: torch.dtype, dev: int, name: str) -> None:
    """x [rows, heads, d_head], rows apart at will."""
    assert tuple(x.shape) == tuple(shape) and x.dtype is dtype and x.get_device() == dev and (shape[2] == 1 or x.stride(2) == 1) and \
        (shape[1] <= 1 or x.stride(1) == shape[2]), f"{name} is {tuple(shape)} of {dtype}, heads contiguous: {tuple(x.shape)} {x.dtype} {x.stride()}"


def page_extend(seq_len: torch.Tensor, n_rows: torch.Tensor, table: torch.Tensor, free_pages: torch.Tensor, n_free: torch.Tensor, page_size: int,
                start: Optional[torch.Tensor] = None, rows: Optional[int] = None, out=None):
    """Pages for the n_rows[b] rows that each request computes next, at positions start[b] .. (None: behind its seq_len[b] tokens); table is written.
    Returns (seq_len, n_free, cu_rows [B + 1], admitted [B], place [B + 1], pos [rows], slot [rows]), or writes them into `out`, such a tuple;
    `rows` counts the rows in all and is needed without `out`.  seq_len and n_free of `out` may be the inputs themselves."""
    dev, B, i32 = seq_len.get_device(), seq_len.numel(), _i32_t
    if out is None:
        assert rows is not None, "rows, or out, is needed"
        new = lambda n: torch.empty(n, dtype=i32, device=seq_len.device)  # noqa: E731
        out = (new(B), new(1), new(B + 1), new(B), new(B + 1), new(rows), new(rows))
    len_out, free_out, cu, admitted, place, pos, slot = out
    M, cap, (TB, width) = pos.numel(), free_pages.numel(), table.shape
    assert rows is None or rows == M, "rows of `out`"
    stride = table.stride(0) if B > 1 else width
    if not (dev >= 0 and seq_len.dtype is i32 and n_rows.dtype is i32 and len_out.dtype is i32 and admitted.dtype is i32 and cu.dtype is i32 and
            place.dtype is i32 and pos.dtype is i32 and slot.dtype is i32 and n_free.dtype is i32 and free_out.dtype is i32 and free_pages.dtype is i32 and
            table.dtype is i32 and TB == B and (width <= 1 or table.stride(1) == 1) and table.get_device() == dev and
            n_rows.numel() == B and len_out.numel() == B and admitted.numel() == B and cu.numel() == B + 1 and place.numel() == B + 1 and slot.numel() == M and
            n_free.numel() == 1 and free_out.numel() == 1 and
            seq_len.is_contiguous() and n_rows.is_contiguous() and len_out.is_contiguous() and admitted.is_contiguous() and cu.is_contiguous() and
            place.is_contiguous() and pos.is_contiguous() and slot.is_contiguous() and free_pages.is_contiguous() and
            n_rows.get_device() == dev and len_out.get_device() == dev and admitted.get_device() == dev and cu.get_device() == dev and
            place.get_device() == dev and pos.get_device() == dev and slot.get_device() == dev and n_free.get_device() == dev and
            free_out.get_device() == dev and free_pages.get_device() == dev):
        _misfit(dev, (("seq_len", seq_len, B), ("n_rows", n_rows, B), ("seq_len of out", len_out, B), ("admitted", admitted, B), ("cu_rows", cu, B + 1),
                      ("place", place, B + 1), ("pos", pos, M), ("slot", slot, M), ("n_free", n_free, 1), ("n_free of out", free_out, 1), ("free_pages", free_pages, cap)))
    if start is not None and not (start.dtype is i32 and start.numel() == B and start.is_contiguous() and start.get_device() == dev):
        _misfit(dev, (("start", start, B),))
    _page_call(lib().pvf_page_extend, dev, (
        seq_len.data_ptr(), None if start is None else start.data_ptr(), n_rows.data_ptr(), B, table.data_ptr(), width, stride, page_size,
        free_pages.data_ptr(), cap, n_free.data_ptr(), M, len_out.data_ptr(), free_out.data_ptr(), cu.data_ptr(), admitted.data_ptr(), place.data_ptr(),
        pos.data_ptr(), slot.data_ptr()))
    return out


def page_trim(seq_len: torch.Tensor, keep: torch.Tensor, table: torch.Tensor, free_pages: torch.Tensor, n_free: torch.Tensor, page_size: int, out=None):
    """Pages behind the first keep[b] tokens of each request go back to free_pages, which is written.  Returns (seq_len, n_free, place [B + 1]), or
    writes them into `out`; seq_len (also keep) and n_free of `out` may be the inputs themselves."""
    dev, B, i32 = seq_len.get_device(), seq_len.numel(), _i32_t
    if out is None:
        new = lambda n: torch.empty(n, dtype=i32, device=seq_len.device)  # noqa: E731
        out = (new(B), new(1), new(B + 1))
    len_out, free_out, place = out
    cap, (TB, width) = free_pages.numel(), table.shape
    stride = table.stride(0) if B > 1 else width
    if not (dev >= 0 and seq_len.dtype is i32 and keep.dtype is i32 and len_out.dtype is i32 and place.dtype is i32 and n_free.dtype is i32 and
            free_out.dtype is i32 and free_pages.dtype is i32 and table.dtype is i32 and TB == B and (width <= 1 or table.stride(1) == 1) and
            table.get_device() == dev and keep.numel() == B and len_out.numel() == B and place.numel() == B + 1 and n_free.numel() == 1 and
            free_out.numel() == 1 and seq_len.is_contiguous() and keep.is_contiguous() and len_out.is_contiguous() and place.is_contiguous() and
            free_pages.is_contiguous() and keep.get_device() == dev and len_out.get_device() == dev and place.get_device() == dev and
            n_free.get_device() == dev and free_out.get_device() == dev and free_pages.get_device() == dev):
        _misfit(dev, (("seq_len", seq_len, B), ("keep", keep, B), ("seq_len of out", len_out, B), ("place", place, B + 1), ("n_free", n_free, 1),
                      ("n_free of out", free_out, 1), ("free_pages", free_pages, cap)))
    _page_call(lib().pvf_page_trim, dev, (
        seq_len.data_ptr(), keep.data_ptr(), B, table.data_ptr(), width, stride, page_size, free_pages.data_ptr(), cap,
        n_free.data_ptr(), len_out.data_ptr(), free_out.data_ptr(), place.data_ptr()))
    return out


def page_store(qkv: torch.Tensor, pos: torch.Tensor, slot: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, rope_theta: float,
               q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotated q [M, H, d_head] of qkv [M, (H + 2 Hkv) * d_head] (rows may lie apart), whose rotated keys and values go to their slots; H follows from the
    caches.  q_out may be strided by rows, also the q part of qkv itself."""
    dev, (M, wide), dtype, i32 = qkv.get_device(), qkv.shape, qkv.dtype, _i32_t
    shape = k_cache.shape
    assert len(shape) == 4, "caches are [n_pages, Hkv, page_size, d_head]"
    n_pages, Hkv, P, dh = shape
    H = wide // dh - 2 * Hkv
    assert H >= 0 and wide == (H + 2 * Hkv) * dh, "rows are q | k | v of whole heads"
    if q_out is None:
        q_out = torch.empty(M, H, dh, dtype=dtype, device=qkv.device)
    (x0, x1), (q0, q1, q2), (k0, k1, k2, k3), (v0, v1, v2, v3) = qkv.stride(), q_out.stride(), k_cache.stride(), v_cache.stride()
    if not (dev >= 0 and k3 == 1 and v3 == 1 and k2 == dh and v2 == dh and k1 == P * dh and v1 == k1 and v_cache.shape == shape and k_cache.dtype is dtype and
            v_cache.dtype is dtype and k_cache.get_device() == dev and v_cache.get_device() == dev):
        _check_cache(k_cache, v_cache, dtype, dev)
    if not (q2 == 1 and q1 == dh and q_out.shape == (M, H, dh) and q_out.dtype is dtype and q_out.get_device() == dev):
        _check_rows(q_out, (M, H, dh), dtype, dev, "q_out")
    assert x1 == 1 or wide == 1, "rows are contiguous"
    if not (pos.dtype is i32 and slot.dtype is i32 and pos.numel() == M and slot.numel() == M and pos.is_contiguous() and slot.is_contiguous() and
            pos.get_device() == dev and slot.get_device() == dev):
        _misfit(dev, (("pos", pos, M), ("slot", slot, M)))
    one, few = M <= 1, n_pages <= 1
    _page_call(lib().pvf_page_store, dev, (
        _dtype_code(dtype), qkv.data_ptr(), 0 if one else x0, pos.data_ptr(), slot.data_ptr(), M, H, Hkv, dh, rope_theta, q_out.data_ptr(), 0 if one else q0,
        k_cache.data_ptr(), v_cache.data_ptr(), n_pages, P, 0 if few else k0, 0 if few else v0))
    return q_out


def page_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, table: torch.Tensor) -> int:
    """Bytes of workspace that page_attention wants for such tensors (PAGE_WORKSPACE suffices for any)."""
    M, H, dh = q.shape
    n = lib().pvf_page_attention_workspace(_dtype_code(q.dtype), table.shape[0], M, H, k_cache.shape[1], dh, table.shape[1], k_cache.shape[2])
    if n < 0:
        _check(n)
    return n


def page_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, seq_len: torch.Tensor,
                   cu_rows: Optional[torch.Tensor] = None, causal: bool = False, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(scale * q k^T) v of rows q [M, H, d_head] against the seq_len[b] tokens of their request: rows cu_rows[b] .. cu_rows[b + 1] - 1 are request b's
    (None: one row each).  causal: a request's rows are its last tokens and see no later ones.  scale: d_head^-0.5 by default.  q and out may be strided
    by rows, out may be q.  workspace: uint8, for callers who keep one (PAGE_WORKSPACE bytes); calls that overlap need one each."""
    dev, (M, H, dh), dtype, B, i32, shape = q.get_device(), q.shape, q.dtype, seq_len.numel(), _i32_t, k_cache.shape
    assert len(shape) == 4 and shape[3] == dh, "caches are [n_pages, Hkv, page_size, d_head], d_head that of q"
    n_pages, Hkv, P, _ = shape
    if out is None:
        out = torch.empty(M, H, dh, dtype=dtype, device=q.device)
    (q0, q1, q2), (o0, o1, o2), (k0, k1, k2, k3), (v0, v1, v2, v3) = q.stride(), out.stride(), k_cache.stride(), v_cache.stride()
    if not (dev >= 0 and k3 == 1 and v3 == 1 and k2 == dh and v2 == dh and k1 == P * dh and v1 == k1 and v_cache.shape == shape and k_cache.dtype is dtype and
            v_cache.dtype is dtype and k_cache.get_device() == dev and v_cache.get_device() == dev):
        _check_cache(k_cache, v_cache, dtype, dev)
    if not (q2 == 1 and q1 == dh):
        _check_rows(q, (M, H, dh), dtype, dev, "q")
    if not (o2 == 1 and o1 == dh and out.shape == (M, H, dh) and out.dtype is dtype and out.get_device() == dev):
        _check_rows(out, (M, H, dh), dtype, dev, "out")
    TB, width = table.shape
    stride = table.stride(0) if B > 1 else width
    if not (seq_len.dtype is i32 and seq_len.is_contiguous() and table.dtype is i32 and TB == B and (width <= 1 or table.stride(1) == 1) and table.get_device() == dev):
        _misfit(dev, (("seq_len", seq_len, B),))
    if cu_rows is not None and not (cu_rows.dtype is i32 and cu_rows.numel() == B + 1 and cu_rows.is_contiguous() and cu_rows.get_device() == dev):
        _misfit(dev, (("cu_rows", cu_rows, B + 1),))
    assert seq_len.get_device() == dev, "lengths lie beside q"
    if workspace is None:
        workspace = torch.empty(page_attention_workspace(q, k_cache, table), dtype=torch.uint8, device=q.device)
    assert workspace.dtype is torch.uint8 and workspace.is_contiguous() and workspace.get_device() == dev, "the workspace is uint8, beside q"
    one, few = M <= 1, n_pages <= 1
    _page_call(lib().pvf_page_attention, dev, (
        _dtype_code(dtype), q.data_ptr(), 0 if one else q0, k_cache.data_ptr(), v_cache.data_ptr(), n_pages, P, 0 if few else k0, 0 if few else v0,
        table.data_ptr(), width, stride, seq_len.data_ptr(), None if cu_rows is None else cu_rows.data_ptr(), B, M, H, Hkv, dh,
        1 if causal else 0, dh ** -0.5 if scale is None else scale, out.data_ptr(), 0 if one else o0, workspace.data_ptr(), workspace.numel()))
    return out


def rope_attention(qkv: torch.Tensor, S: int, T: int, n_heads: int, d_head: int,
                   rope_theta: float) -> torch.Tensor:
    """qkv [S*T, 3*d] is rotated in place; returns the attention output [S*T, d]."""
    assert qkv.shape == (S * T, 3 * n_heads * d_head) and qkv.is_contiguous()
    out = torch.empty(S * T, n_heads * d_head, dtype=qkv.dtype, device=qkv.device)
    _check(lib().pvf_rope_attention(_stream(), _dtype_code(qkv.dtype), _ptr(qkv), _ptr(out), S, T,
                                    n_heads, d_head, rope_theta))
    return out


def rope_attention_noalloc(qkv: torch.Tensor, out: torch.Tensor, S: int, T: int, n_heads: int, d_head: int,
                           rope_theta: float) -> torch.Tensor:
    """pvf_rope_attention_noalloc: like rope_attention, into the caller's `out`; the library allocates nothing."""
    assert qkv.shape == (S * T, 3 * n_heads * d_head) and qkv.is_contiguous()
    assert out.shape == (S * T, n_heads * d_head) and out.dtype == qkv.dtype
    _check(lib().pvf_rope_attention_noalloc(_stream(), _dtype_code(qkv.dtype), _ptr(qkv), _ptr(out), S, T,
                                            n_heads, d_head, rope_theta))
    return out


def qkv_attention(x: torch.Tensor, wqkv: torch.Tensor, S: int, T: int, n_heads: int, d_head: int,
                  rope_theta: float, vt: Optional[torch.Tensor] = None):
    """(qkv [S*T, 3d] with q, k rotated; attention output [S*T, d]) of x [S*T, d]; vt [S, H, d_head, T]
    (optional) receives the key-contiguous copy of v where the fused projection epilogue writes one."""
    d = n_heads * d_head
    assert x.shape == (S * T, d) and wqkv.shape == (3 * d, d) and x.is_contiguous() and wqkv.is_contiguous()
    assert wqkv.dtype == x.dtype
    qkv = torch.empty(S * T, 3 * d, dtype=x.dtype, device=x.device)
    out = torch.empty(S * T, d, dtype=x.dtype, device=x.device)
    if vt is not None:
        assert vt.shape == (S, n_heads, d_head, T) and vt.dtype == x.dtype
    _check(lib().pvf_qkv_attention(_stream(), _dtype_code(x.dtype), _ptr(x), _ptr(wqkv), _ptr(qkv), _ptr(vt), _ptr(out),
                                   S, T, n_heads, d_head, rope_theta))
    return qkv, out


def fill_normal(dst: torch.Tensor, seed: int, mean: float = 0.0, std: float = 0.02) -> None:
    _check(lib().pvf_fill_normal(_stream(), _dtype_code(dst.dtype), _ptr(dst), dst.numel(), seed,
                                 mean, std))
