"""ctypes mirror of include/dllm_rps.h and the loader of libdllm_rps.so.

The library is required: there is no fallback.  Importing this module fails
with ImportError if the in-tree shared object has not been built.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdllm_rps.so")
MARSHAL_PATH = os.path.join(HERE, "_marshal.so")

DLLM_MAX_TOPK = 16
RPS_MAX_PIVOTS = 16
RPS_MAX_BRANCH = 16
RPS_MAX_MASKED = 1024

DLLM_F32, DLLM_BF16 = 0, 1
RPS_PIVOT_PAPER, RPS_PIVOT_BAND = 0, 1
DLLM_PROF_CLASSES = 10
PROF_NAMES = ("embed", "rmsnorm", "gemm_qkv", "attention", "gemm_o", "gemm_gateup", "gemm_down", "lmhead",
              "lmhead_merge", "other")

STATUS = {0: "DLLM_OK", 1: "DLLM_EINVAL", 2: "DLLM_ESHAPE", 3: "DLLM_EDTYPE", 4: "DLLM_ENOMEM",
          5: "DLLM_EHIP", 6: "DLLM_EUNSUPPORTED"}

i32, f32, f64, vp, sz = C.c_int32, C.c_float, C.c_double, C.c_void_p, C.c_size_t


class ModelDesc(C.Structure):
    _fields_ = [("n_layers", i32), ("d_model", i32), ("n_heads", i32), ("head_dim", i32), ("d_ffn", i32),
                ("vocab", i32), ("mask_id", i32), ("rope_base", f32), ("rms_eps", f32), ("dtype", i32),
                ("max_pos", i32)]


class Weights(C.Structure):
    _fields_ = [("emb", vp), ("lm_head", vp), ("wqkv", C.POINTER(vp)), ("wo", C.POINTER(vp)),
                ("wgu", C.POINTER(vp)), ("wdown", C.POINTER(vp))]


class StatsC(C.Structure):
    _fields_ = [("H", vp), ("lse", vp), ("lmax", vp), ("argmax", vp), ("topk_id", vp), ("topk_logit", vp),
                ("k", i32)]


class KvCache(C.Structure):
    _fields_ = [("k", vp), ("vt", vp), ("len", i32), ("cap", i32)]


class KvPagesC(C.Structure):
    _fields_ = [("k", vp), ("vt", vp), ("refs", vp), ("table", vp), ("len", vp), ("n_layers", i32),
                ("n_pages", i32), ("n_kv_heads", i32), ("head_dim", i32), ("page_len", i32), ("max_seqs", i32),
                ("max_blocks", i32), ("dtype", i32)]


class Rows(C.Structure):
    _fields_ = [("p", vp), ("seq", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


class AttentionPlan(C.Structure):
    _fields_ = [(f, i32) for f in ("way", "prefix_rows", "prefix_ranges", "prefix_keys", "tail_rows", "tail_ranges",
                                   "tail_keys")]


class RotaryC(C.Structure):
    _fields_ = [("freq", vp), ("q_gain", vp), ("k_gain", vp), ("head_dim", i32), ("dim", i32), ("layout", i32),
                ("norm", i32), ("amplitude", f32), ("eps", f32)]


class Probe(C.Structure):
    _fields_ = [("row", vp), ("token", vp), ("logit", vp), ("n", i32)]


class RpsParams(C.Structure):
    _fields_ = [("mode", i32), ("k_max", i32), ("tau_pivot", f32), ("pct_lo", f32), ("pct_hi", f32),
                ("n_pivots", i32), ("r", f32), ("n_cand", i32), ("max_branch", i32)]


class RpsPlan(C.Structure):
    _fields_ = [("n_pivots", i32), ("n_branch", i32), ("pivot_row", i32 * RPS_MAX_PIVOTS),
                ("pivot_pos", i32 * RPS_MAX_PIVOTS), ("n_cand", i32 * RPS_MAX_PIVOTS),
                ("br_pivot", i32 * RPS_MAX_BRANCH), ("br_row", i32 * RPS_MAX_BRANCH),
                ("br_pos", i32 * RPS_MAX_BRANCH), ("br_token", i32 * RPS_MAX_BRANCH),
                ("br_logp", f32 * RPS_MAX_BRANCH)]


class RpsDecision(C.Structure):
    _fields_ = [("commit", i32), ("branch", i32), ("pivot_row", i32), ("pivot_pos", i32), ("token", i32),
                ("delta", f32), ("second_delta", f32), ("n_masked", i32)]


# name -> (restype, argtypes); the same names as the C ABI
SIGNATURES = {
    "dllm_abi_version": (i32, []),
    "dllm_last_error": (C.c_char_p, []),
    "dllm_status_string": (C.c_char_p, [i32]),
    "dllm_model_create": (i32, [C.POINTER(ModelDesc), C.POINTER(Weights), C.POINTER(vp)]),
    "dllm_model_destroy": (None, [vp]),
    "dllm_workspace_bytes": (sz, [vp, i32, i32, i32]),
    "dllm_workspace_bytes_packed": (sz, [vp, i32, i32, i32, i32]),
    "dllm_forward": (i32, [vp, vp, i32, i32, i32, C.POINTER(KvCache), C.POINTER(KvCache), vp, i32, vp, f32,
                           C.POINTER(Probe), C.POINTER(StatsC), vp, sz, vp]),
    "dllm_forward_packed": (i32, [vp, vp, i32, i32, i32, i32, i32, C.POINTER(KvCache), vp, i32, vp, f32,
                                  C.POINTER(Probe), C.POINTER(StatsC), vp, sz, vp]),
    "vocab_entropy_topk_workspace_bytes": (sz, [i32, i32]),
    "vocab_entropy_topk": (i32, [vp, vp, i32, i32, i32, i32, vp, f32, i32, C.POINTER(StatsC), vp, sz, vp]),
    "vocab_entropy_topk_noalloc": (i32, [vp, vp, i32, i32, i32, i32, vp, f32, i32, C.POINTER(StatsC), vp]),
    "dllm_workspace_bytes_pages": (sz, [vp, i32, i32, i32]),
    "dllm_forward_pages": (i32, [vp, vp, i32, i32, C.POINTER(KvPagesC), vp, i32, i32, i32, vp, i32, vp, f32,
                                 C.POINTER(Probe), C.POINTER(StatsC), vp, sz, vp]),
    "kv_pages_init": (i32, [C.POINTER(KvPagesC), vp]),
    "kv_pages_grow": (i32, [C.POINTER(KvPagesC), vp, vp, i32, vp, vp]),
    "kv_pages_fork": (i32, [C.POINTER(KvPagesC), vp, vp, vp, i32, vp, vp]),
    "kv_pages_free": (i32, [C.POINTER(KvPagesC), vp, vp, i32, vp, vp]),
    "kv_pages_compact_workspace_bytes": (sz, [C.POINTER(KvPagesC)]),
    "kv_pages_compact": (i32, [C.POINTER(KvPagesC), vp, vp, sz, vp]),
    "kv_pages_write": (i32, [C.POINTER(KvPagesC), i32, vp, i32, i32, vp, C.POINTER(Rows), C.POINTER(Rows), vp]),
    "kv_pages_attention_workspace_bytes": (sz, [C.POINTER(KvPagesC), i32, i32, i32]),
    "kv_pages_attention": (i32, [C.POINTER(KvPagesC), i32, vp, i32, i32, vp, i32, C.POINTER(Rows), C.POINTER(Rows),
                                 i32, i32, i32, i32, f32, vp, sz, vp]),
    "kv_pages_attention_plan": (i32, [C.POINTER(KvPagesC), i32, i32, i32, i32, i32, C.POINTER(AttentionPlan)]),
    "dllm_rotary_frequencies": (i32, [i32, f64, i32, f64, f64, f64, f64, C.POINTER(f64), C.POINTER(f32)]),
    "rotary_rows": (i32, [C.POINTER(RotaryC), i32, vp, i32, i32, i32, vp, i32, C.POINTER(Rows), C.POINTER(Rows), i32,
                          C.POINTER(Rows), C.POINTER(Rows), vp]),
    "kv_pages_append": (i32, [C.POINTER(KvPagesC), i32, vp, i32, i32, vp, C.POINTER(RotaryC), vp, i32, C.POINTER(Rows),
                              C.POINTER(Rows), C.POINTER(Rows), C.POINTER(Rows), vp]),
    "kv_pages_tree": (i32, [C.POINTER(KvPagesC), vp, i32, i32, vp, vp, vp, vp, vp]),
    "kv_pages_attention_tree": (i32, [C.POINTER(KvPagesC), i32, vp, i32, i32, vp, i32, C.POINTER(Rows), C.POINTER(Rows),
                                      vp, i32, i32, i32, f32, vp, sz, vp]),
    "kv_pages_attention_tree_plan": (i32, [C.POINTER(KvPagesC), i32, i32, i32, i32, i32, C.POINTER(AttentionPlan)]),
    "kv_pages_accept_workspace_bytes": (sz, [C.POINTER(KvPagesC), i32, i32]),
    "kv_pages_accept": (i32, [C.POINTER(KvPagesC), vp, i32, i32, vp, vp, i32, vp, vp, vp, sz, vp]),
    "dllm_profile_begin": (i32, [vp, i32]),
    "dllm_profile_begin_classes": (i32, [vp, i32, C.c_uint32]),
    "dllm_profile_end": (i32, [vp, C.POINTER(f32), C.POINTER(i32)]),
    "dllm_mfma_ceiling": (i32, [i32, C.POINTER(f32), vp]),
    "rps_select_pivots": (i32, [C.POINTER(StatsC), vp, i32, C.POINTER(RpsParams), vp, vp]),
    "rps_build_branches": (i32, [vp, i32, vp, i32, i32, vp, vp]),
    "rps_build_packed": (i32, [vp, i32, vp, i32, i32, i32, vp, vp]),
    "rps_lookahead_score": (i32, [C.POINTER(StatsC), C.POINTER(StatsC), i32, i32, vp, vp, f32, vp, vp, vp, vp]),
    "rps_commit": (i32, [vp, i32, vp, i32, C.POINTER(StatsC), vp, C.POINTER(StatsC), i32, C.POINTER(StatsC), f32,
                         vp, vp, vp, vp]),
    "sched_commit": (i32, [vp, i32, vp, i32, C.POINTER(StatsC), i32, i32, vp, vp, vp, vp]),
}

SCHED_TOP_CONFIDENCE, SCHED_LOW_ENTROPY = 0, 1
KV_PAGES_OK, KV_PAGES_ESEQ, KV_PAGES_ELEN, KV_PAGES_ESHARED, KV_PAGES_EFULL = 0, 1, 2, 3, 4
KV_PAGES_EPATH = 5
KV_WAY_ENTRIES, KV_WAY_PARTS, KV_WAY_PAIRS = 0, 1, 2
KV_MAX_PAGES, KV_MAX_SEQS, KV_MAX_POSITIONS = 1 << 20, 1024, 1 << 30
KV_MAX_HEADS, KV_MAX_LAYERS, KV_MAX_ROWS, KV_MAX_HEAD_ROWS = 1024, 65536, 1 << 20, 1 << 26
KV_TREE_MAX_ROWS = 1024
ROTARY_HALVES, ROTARY_PAIRS = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_RAMP = 0, 1, 2, 3


def require(*paths: str):
    for path in paths:
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: the HIP library must be built first "
                              "(python -c 'import __graft_entry__ as g; g.build()')")


def load(path: str = LIB_PATH):
    require(path)
    lib = C.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


class DllmError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status
