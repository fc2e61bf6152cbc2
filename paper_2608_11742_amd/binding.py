"""Python binding of libdllm_rps: argument marshalling only.

Every function has the name of the C entry point it calls and takes torch
tensors (device memory) instead of raw pointers.  Torch provides device
memory and the current stream; every step of the computation runs in the
library's HIP kernels.  A non-zero status raises DllmError with the
library's message.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import _abi
_abi.require(_abi.LIB_PATH, _abi.MARSHAL_PATH)   # _marshal is linked with the library
from . import _marshal  # noqa: E402
from ._abi import (DllmError, ModelDesc, Weights, StatsC, KvCache, Probe, RpsParams, RpsPlan, RpsDecision,
                   DLLM_F32, DLLM_BF16, RPS_PIVOT_PAPER, RPS_PIVOT_BAND, DLLM_MAX_TOPK, RPS_MAX_BRANCH)  # noqa: E402

_LIB = None
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def lib():
    global _LIB
    if _LIB is None:
        _LIB = _abi.load()
    return _LIB


def _check(status: int):
    if status != 0:
        raise DllmError(status, lib().dllm_last_error().decode())


def _p(t):
    # an address as a plain int: the declared argument types convert it
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        # the current stream's handle without the Stream object that
        # torch.cuda.current_stream() builds around it (7 us a call)
        return _raw_stream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return stream


# ---------------------------------------------------------------- device buffers

class Stats:
    """Per-position statistics of R rows in device memory (dllm_stats)."""

    def __init__(self, R: int, k: int = DLLM_MAX_TOPK, device="cuda", _views=None):
        if _views is not None:
            self.H, self.lse, self.lmax, self.argmax, self.topk_id, self.topk_logit = _views
        else:
            f = dict(dtype=torch.float32, device=device)
            i = dict(dtype=torch.int32, device=device)
            self.H = torch.empty(R, **f)
            self.lse = torch.empty(R, **f)
            self.lmax = torch.empty(R, **f)
            self.argmax = torch.empty(R, **i)
            self.topk_id = torch.empty(R, k, **i)
            self.topk_logit = torch.empty(R, k, **f)
        self.k = self.topk_id.shape[1]

    @property
    def R(self) -> int:
        return self.H.shape[0]

    def rows(self, start: int, n: int) -> "Stats":
        sl = slice(start, start + n)
        return Stats(0, _views=(self.H[sl], self.lse[sl], self.lmax[sl], self.argmax[sl], self.topk_id[sl],
                                self.topk_logit[sl]))

    def c(self) -> StatsC:
        return StatsC(self.H.data_ptr(), self.lse.data_ptr(), self.lmax.data_ptr(), self.argmax.data_ptr(),
                      self.topk_id.data_ptr(), self.topk_logit.data_ptr(), self.k)

    def fill_(self, value: float):
        for t in (self.H, self.lse, self.lmax, self.topk_logit):
            t.fill_(value)
        self.argmax.fill_(-1)
        self.topk_id.fill_(-1)
        return self

    def numpy(self) -> dict:
        return {n: getattr(self, n).cpu().numpy() for n in ("H", "lse", "lmax", "argmax", "topk_id", "topk_logit")}


def new_plan(device="cuda"):
    return torch.zeros(C.sizeof(RpsPlan), dtype=torch.uint8, device=device)


def new_decision(device="cuda"):
    return torch.zeros(C.sizeof(RpsDecision), dtype=torch.uint8, device=device)


def read_plan(t) -> RpsPlan:
    return RpsPlan.from_buffer_copy(t.cpu().numpy().tobytes())


def read_decision(t) -> RpsDecision:
    return RpsDecision.from_buffer_copy(t.cpu().numpy().tobytes())


def plan_field_ptr(plan, name: str) -> int:
    """Device address of an array field of a device-resident rps_plan."""
    return plan.data_ptr() + getattr(RpsPlan, name).offset


def params(mode="band", k_max=10, tau_pivot=0.9, pct_lo=25.0, pct_hi=75.0, n_pivots=1, r=0.1, n_cand=10,
           max_branch=RPS_MAX_BRANCH) -> RpsParams:
    m = RPS_PIVOT_BAND if mode == "band" else RPS_PIVOT_PAPER
    return RpsParams(m, k_max, tau_pivot, pct_lo, pct_hi, n_pivots, r, n_cand, max_branch)


# ---------------------------------------------------------------- model

def dllm_model_create(desc: ModelDesc, weights: dict):
    """weights: emb, lm_head, wqkv, wo, wgu, wdown (lists of per-layer device tensors)."""
    L = desc.n_layers
    arrs = {}
    for name in ("wqkv", "wo", "wgu", "wdown"):
        a = (C.c_void_p * L)(*[w.data_ptr() for w in weights[name]])
        arrs[name] = a
    w = Weights(weights["emb"].data_ptr(), weights["lm_head"].data_ptr(),
                C.cast(arrs["wqkv"], C.POINTER(C.c_void_p)), C.cast(arrs["wo"], C.POINTER(C.c_void_p)),
                C.cast(arrs["wgu"], C.POINTER(C.c_void_p)), C.cast(arrs["wdown"], C.POINTER(C.c_void_p)))
    handle = C.c_void_p()
    _check(lib().dllm_model_create(C.byref(desc), C.byref(w), C.byref(handle)))
    return handle


def dllm_model_destroy(handle):
    lib().dllm_model_destroy(handle)


def dllm_profile_begin(handle, max_launches: int = 20000, classes=None):
    """classes: optional iterable of kernel-class names (PROF_NAMES) to bracket; default all."""
    if classes is None:
        _check(lib().dllm_profile_begin(handle, max_launches))
        return
    mask = 0
    for name in classes:
        mask |= 1 << _abi.PROF_NAMES.index(name)
    _check(lib().dllm_profile_begin_classes(handle, max_launches, mask))


def dllm_profile_end(handle) -> dict:
    """{kernel class: (total ms, launches)} of the launches since dllm_profile_begin."""
    ms = (C.c_float * _abi.DLLM_PROF_CLASSES)()
    n = (C.c_int32 * _abi.DLLM_PROF_CLASSES)()
    _check(lib().dllm_profile_end(handle, ms, n))
    return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(_abi.PROF_NAMES)}


def dllm_mfma_ceiling(random_operands: bool = True, stream=None) -> float:
    """Sustained bf16 MFMA rate of the device on a register-only loop, TFLOP/s
    (random_operands: different random operands at every instruction)."""
    out = C.c_float(0.0)
    _check(lib().dllm_mfma_ceiling(1 if random_operands else 0, C.byref(out), _stream(stream)))
    return float(out.value)


def dllm_workspace_bytes(handle, batch: int, seq: int, n_lm_pos: int) -> int:
    return lib().dllm_workspace_bytes(handle, batch, seq, n_lm_pos)


def dllm_workspace_bytes_packed(handle, shared_len: int, block_len: int, n_branch: int, n_lm_pos: int) -> int:
    return lib().dllm_workspace_bytes_packed(handle, shared_len, block_len, n_branch, n_lm_pos)


def dllm_forward(handle, tokens, lm_pos, out: Stats, ws, pos_offset: int = 0, row_scale=None, scale: float = 1.0,
                 kv_prefix: KvCache | None = None, kv_out: KvCache | None = None, probe: Probe | None = None,
                 n_lm_pos: int | None = None, stream=None):
    batch, seq = tokens.shape
    n_lm = lm_pos.shape[0] if n_lm_pos is None else n_lm_pos
    _check(lib().dllm_forward(handle, _p(tokens), batch, seq, pos_offset,
                              None if kv_prefix is None else C.byref(kv_prefix),
                              None if kv_out is None else C.byref(kv_out), _p(lm_pos), n_lm, _p(row_scale),
                              scale, None if probe is None else C.byref(probe), C.byref(out.c()), _p(ws),
                              ws.numel() * ws.element_size(), _stream(stream)))


def dllm_forward_packed(handle, tokens, shared_len: int, block_start: int, block_len: int, n_branch: int, lm_pos,
                        out: Stats, ws, pos_offset: int = 0, kv_prefix: KvCache | None = None, row_scale=None,
                        scale: float = 1.0, probe: Probe | None = None, n_lm_pos: int | None = None, stream=None):
    """Packed lookahead forward: tokens [shared_len + n_branch * block_len] (one
    sequence); out receives (1 + n_branch) * n_lm_pos rows (shared, then each branch)."""
    n_lm = lm_pos.shape[0] if n_lm_pos is None else n_lm_pos
    _check(lib().dllm_forward_packed(handle, _p(tokens), shared_len, block_start, block_len, n_branch, pos_offset,
                                     None if kv_prefix is None else C.byref(kv_prefix), _p(lm_pos), n_lm,
                                     _p(row_scale), scale, None if probe is None else C.byref(probe),
                                     C.byref(out.c()), _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


def vocab_entropy_topk_workspace_bytes(R: int, vocab: int) -> int:
    return lib().vocab_entropy_topk_workspace_bytes(R, vocab)


def vocab_entropy_topk(hidden, w_lm, out: Stats, ws, row_scale=None, scale: float = 1.0, mask_id: int = -1,
                       stream=None):
    R, d = hidden.shape
    V = w_lm.shape[0]
    dt = DLLM_BF16 if hidden.dtype == torch.bfloat16 else DLLM_F32
    _check(lib().vocab_entropy_topk(_p(hidden), _p(w_lm), R, d, V, dt, _p(row_scale), scale, mask_id,
                                    C.byref(out.c()), _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


def vocab_entropy_topk_noalloc(hidden, w_lm, out: Stats, row_scale=None, scale: float = 1.0, mask_id: int = -1,
                               stream=None):
    R, d = hidden.shape
    V = w_lm.shape[0]
    dt = DLLM_BF16 if hidden.dtype == torch.bfloat16 else DLLM_F32
    _check(lib().vocab_entropy_topk_noalloc(_p(hidden), _p(w_lm), R, d, V, dt, _p(row_scale), scale, mask_id,
                                            C.byref(out.c()), _stream(stream)))


# ---------------------------------------------------------------- paged key/value cache

class KvPages:
    """Device arrays of a paged key/value cache (dllm_kv_pages).

    k [layers, pages, kv heads, page_len, head_dim] bf16 or fp32; vt [layers,
    pages, kv heads, head_dim, page_len] float16 for bf16 keys, else fp32;
    refs [pages], table [max_seqs, max_blocks], len [max_seqs] int32.
    """

    def __init__(self, k, vt, refs, table, len):
        L, n_pages, heads, page_len, hd = k.shape
        v_dtype = {torch.bfloat16: torch.float16, torch.float32: torch.float32}.get(k.dtype)
        if v_dtype is None or vt.dtype != v_dtype or tuple(vt.shape) != (L, n_pages, heads, hd, page_len):
            raise ValueError("k must be bf16 with float16 vt, or fp32 with fp32 vt, vt transposed within the pages")
        if any(t.dtype != torch.int32 for t in (refs, table, len)):
            raise ValueError("refs, table and len must be int32")
        if refs.shape != (n_pages,) or table.dim() != 2 or len.shape != table.shape[:1]:
            raise ValueError("refs [pages], table [max_seqs, max_blocks], len [max_seqs]")
        if any(t.device != k.device or not t.is_contiguous() for t in (k, vt, refs, table, len)):
            raise ValueError("the arrays must be contiguous tensors of one device")
        self.k, self.vt, self.refs, self.table, self.len = k, vt, refs, table, len
        self.page_len, self.head_dim, self.n_kv_heads, self.dtype = page_len, hd, heads, k.dtype
        self.device, self._index, self._scale = k.device, k.get_device(), hd ** -0.5
        self._c = _abi.KvPagesC(k.data_ptr(), vt.data_ptr(), refs.data_ptr(), table.data_ptr(), len.data_ptr(), L,
                                n_pages, heads, hd, page_len, table.shape[0], table.shape[1],
                                DLLM_BF16 if k.dtype == torch.bfloat16 else DLLM_F32)
        self._ref, self._at = C.byref(self._c), C.addressof(self._c)

    @classmethod
    def empty(cls, n_layers: int, n_pages: int, n_kv_heads: int, page_len: int, head_dim: int, max_seqs: int,
              max_blocks: int, dtype=torch.bfloat16, device="cuda"):
        """New arrays, every page free and every sequence empty (kv_pages_init)."""
        i = dict(dtype=torch.int32, device=device)
        v_dtype = torch.float16 if dtype == torch.bfloat16 else dtype
        pages = cls(torch.empty(n_layers, n_pages, n_kv_heads, page_len, head_dim, dtype=dtype, device=device),
                    torch.empty(n_layers, n_pages, n_kv_heads, head_dim, page_len, dtype=v_dtype, device=device),
                    torch.empty(n_pages, **i), torch.empty(max_seqs, max_blocks, **i), torch.empty(max_seqs, **i))
        kv_pages_init(pages)
        return pages


_I32, _Rows = torch.int32, _abi.Rows
# of a process that has tensors on a device: without the check for a first use
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _ids(pages: KvPages, t, n: int):
    """Address of an int32 list of n entries beside the pages' arrays."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.get_device() != pages._index or t.numel() != n or not t.is_contiguous():
        raise ValueError("sequence lists, counts and status are contiguous int32 tensors, one value an entry, beside the pages")
    return t.data_ptr()


def _rows(pages: KvPages, t, n: int, rows: int, heads: int, name: str):
    """t [n, rows, heads, head_dim], any strides over contiguous head_dim, as dllm_rows."""
    seq, row, head, one = t.stride()
    if one != 1 or t.dtype is not pages.dtype or t.get_device() != pages._index:
        raise ValueError(f"{name} must have contiguous rows, and the type and device of the pages' keys")
    # a dimension of one has no stride to speak of
    return _Rows(t.data_ptr(), seq if n > 1 else 0, row if rows > 1 else 0, head if heads > 1 else 0)


def _scratch(pages: KvPages, ws):
    """Address and size of a workspace beside the pages."""
    if ws.get_device() != pages._index or not ws.is_contiguous():
        raise ValueError("the workspace must be contiguous and beside the pages")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _page_stream(pages: KvPages, stream):
    dev = _current_device()
    if dev != pages._index:
        raise ValueError("the pages are on another device than the current one")
    if stream is None:
        return _raw_stream(dev)
    if isinstance(stream, torch.cuda.Stream) and stream.device_index != dev:
        raise ValueError("the stream is of another device than the pages")
    return _stream(stream)


def kv_pages_init(pages: KvPages, stream=None):
    _check(lib().kv_pages_init(pages._ref, _page_stream(pages, stream)))


def kv_pages_grow(pages: KvPages, seqs, add, status, stream=None):
    """Sequences seqs[i] grow by add[i] positions; status (int32, device) receives a KV_PAGES_ code."""
    n = seqs.numel()
    _check(lib().kv_pages_grow(pages._ref, _ids(pages, seqs, n), _ids(pages, add, n), n, _ids(pages, status, 1),
                               _page_stream(pages, stream)))


def kv_pages_fork(pages: KvPages, src, dst, status, keep=None, stream=None):
    """Empty sequences dst[i] become the first keep[i] positions of src[i] (all of them without keep)."""
    n = src.numel()
    _check(lib().kv_pages_fork(pages._ref, _ids(pages, src, n), _ids(pages, dst, n), _ids(pages, keep, n), n,
                               _ids(pages, status, 1), _page_stream(pages, stream)))


def kv_pages_free(pages: KvPages, seqs, status, keep=None, stream=None):
    """Sequences seqs[i] keep their first keep[i] positions (none without keep)."""
    n = seqs.numel()
    _check(lib().kv_pages_free(pages._ref, _ids(pages, seqs, n), _ids(pages, keep, n), n, _ids(pages, status, 1),
                               _page_stream(pages, stream)))


def kv_pages_compact_workspace_bytes(pages: KvPages) -> int:
    return lib().kv_pages_compact_workspace_bytes(pages._ref)


def kv_pages_compact(pages: KvPages, n_used, ws, stream=None):
    """Pages in use move to ids 0 .. n_used-1 (n_used: int32, device)."""
    _check(lib().kv_pages_compact(pages._ref, _ids(pages, n_used, 1), *_scratch(pages, ws),
                                  _page_stream(pages, stream)))


def kv_pages_write(pages: KvPages, layer: int, seqs, k, v, n_rows=None, stream=None):
    """k, v [entries, rows, kv heads, head_dim]: the last n_rows[b] (or all rows) positions of sequence seqs[b]."""
    n, rows, heads, hd = shape = k.shape
    if v.shape != shape or heads != pages.n_kv_heads or hd != pages.head_dim:
        raise ValueError("k and v need the pages' heads and head_dim and the same shape")
    _check(lib().kv_pages_write(pages._ref, layer, _ids(pages, seqs, n), n, rows, _ids(pages, n_rows, n),
                                _rows(pages, k, n, rows, heads, "k"), _rows(pages, v, n, rows, heads, "v"),
                                _page_stream(pages, stream)))


def kv_pages_attention_workspace_bytes(pages: KvPages, n: int, max_rows: int, n_heads: int) -> int:
    return lib().kv_pages_attention_workspace_bytes(pages._ref, n, max_rows, n_heads)


def kv_pages_attention(pages: KvPages, layer: int, seqs, q, out, ws, n_rows=None, prefix_seq: int = 0,
                       shared_len: int = 0, max_len: int | None = None, causal: bool = False,
                       scale: float | None = None, stream=None):
    """q, out [entries, rows, heads, head_dim]; see kv_pages_attention in dllm_rps.h.

    max_len defaults to the tables' length, scale to 1 / sqrt(head_dim)."""
    n, rows, heads, hd = shape = q.shape
    if out.shape != shape or hd != pages.head_dim:
        raise ValueError("q and out need the pages' head_dim and the same shape")
    if max_len is None:
        max_len = pages.table.shape[1] * pages.page_len
    _check(lib().kv_pages_attention(pages._ref, layer, _ids(pages, seqs, n), n, rows, _ids(pages, n_rows, n), heads,
                                    _rows(pages, q, n, rows, heads, "q"),
                                    _rows(pages, out, n, rows, heads, "out"), prefix_seq,
                                    shared_len, max_len, int(causal), pages._scale if scale is None else scale,
                                    *_scratch(pages, ws), _page_stream(pages, stream)))


def kv_pages_attention_plan(pages: KvPages, n: int, max_rows: int, n_heads: int, shared_len: int = 0,
                            max_len: int | None = None):
    """How kv_pages_attention divides a call of these sizes (way, and rows, ranges and keys of its parts)."""
    if max_len is None:
        max_len = pages.table.shape[1] * pages.page_len
    plan = _abi.AttentionPlan()
    _check(lib().kv_pages_attention_plan(pages._ref, n, max_rows, n_heads, shared_len, max_len, C.byref(plan)))
    return plan


# ---------------------------------------------------------------- rotary positions, drafts

_SCALINGS = {None: _abi.ROTARY_PLAIN, "linear": _abi.ROTARY_LINEAR, "base": _abi.ROTARY_BASE, "ramp": _abi.ROTARY_RAMP}
_LAYOUTS = {"halves": _abi.ROTARY_HALVES, "pairs": _abi.ROTARY_PAIRS}


def dllm_rotary_frequencies(dim: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                            original_len: float = 4096.0, slow: float = 1.0, fast: float = 32.0):
    """(frequencies in radians a position, amplitude) of a rotation of dim elements; scaling "linear", "base" or "ramp"."""
    if scaling not in _SCALINGS:
        raise ValueError("scaling is None, linear, base or ramp")
    freq, amplitude = (C.c_double * max(1, dim // 2))(), C.c_float()
    _check(lib().dllm_rotary_frequencies(dim, base, _SCALINGS[scaling], factor, original_len, slow, fast, freq,
                                         C.byref(amplitude)))
    return list(freq), float(amplitude.value)


class Rotary:
    """Rotation of heads to their positions, after a norm by head (dllm_rotary).

    dim: rotated elements of a head (default all), layout "halves" or "pairs",
    scaling as in dllm_rotary_frequencies; freq [dim / 2] stands for base and
    scaling (with amplitude 1), amplitude gives another factor.  norm: heads are normed first, with
    gains q_gain and k_gain [head_dim] where given."""

    def __init__(self, head_dim: int, dim: int | None = None, base: float = 10000.0, layout: str = "halves",
                 scaling: str | None = None, factor: float = 1.0, original_len: float = 4096.0, slow: float = 1.0,
                 fast: float = 32.0, freq=None, amplitude: float | None = None, norm: bool = False, eps: float = 1e-5,
                 q_gain=None, k_gain=None, device="cuda"):
        dim = head_dim if dim is None else dim
        if layout not in _LAYOUTS or scaling not in _SCALINGS:
            raise ValueError("layout is halves or pairs, scaling None, linear, base or ramp")
        if head_dim not in (64, 128) or not 0 <= dim <= head_dim or dim % 16:
            raise ValueError("head_dim is 64 or 128, dim a multiple of 16 up to it")
        if not norm and (q_gain is not None or k_gain is not None):
            raise ValueError("gains belong to a norm")
        own = 1.0
        if freq is None and dim:
            freq, own = dllm_rotary_frequencies(dim, base, scaling, factor, original_len, slow, fast)
        freq = torch.as_tensor([] if freq is None else freq, dtype=torch.float64)
        if tuple(freq.shape) != (dim // 2,):
            raise ValueError("one frequency for every pair of rotated elements")
        self.freq = (freq if dim else torch.zeros(1, dtype=torch.float64)).to(device).contiguous()
        self.device, self._index = self.freq.device, self.freq.get_device()
        self.q_gain, self.k_gain = q_gain, k_gain
        for g in (q_gain, k_gain):
            if g is not None and (g.dtype != torch.float32 or tuple(g.shape) != (head_dim,) or not g.is_contiguous()
                                  or g.device != self.device):
                raise ValueError("gains are contiguous fp32 tensors [head_dim] beside the frequencies")
        self.head_dim, self.dim, self.amplitude = head_dim, dim, own if amplitude is None else amplitude
        self._c = _abi.RotaryC(self.freq.data_ptr(), _p(q_gain), _p(k_gain), head_dim, dim, _LAYOUTS[layout], int(norm),
                               self.amplitude, eps)
        self._at = C.addressof(self._c)


# These are called once a layer and token: _marshal reads the tensors natively
# (types, devices, shapes and strides checked, ValueError where they do not fit).

def rotary_rows(rot: Rotary, q, q_out, k=None, k_out=None, pos=None, pos_offset: int = 0, n_rows=None, stream=None):
    """q [entries, rows, heads, head_dim] (and k, with heads of its own) normed and rotated into q_out (and k_out);
    pos [entries, rows], or row i is at pos_offset + i.  The outputs may be the inputs."""
    status = _marshal.rotary_rows(rot._at, rot._index, q, q_out, k, k_out, pos, pos_offset, n_rows,
                                  None if stream is None else _page_stream(rot, stream))
    if status:
        _check(status)


def kv_pages_append(pages: KvPages, layer: int, seqs, k, v, rot: Rotary, q=None, q_out=None, pos=None, n_rows=None,
                    stream=None):
    """kv_pages_write with k normed and rotated on the way; q [entries, rows, heads, head_dim] likewise into q_out.
    pos [entries, rows]: positions of the rotation, by default those of the rows.  entries * rows * (heads + key heads)
    is KV_MAX_HEAD_ROWS at most."""
    status = _marshal.kv_pages_append(pages._at, pages._index, layer, seqs, n_rows, rot._at, rot._index, pos, q, q_out,
                                      k, v, None if stream is None else _page_stream(pages, stream))
    if status:
        _check(status)


def kv_pages_tree(pages: KvPages, seqs, parent, mask, pos=None, n_rows=None, stream=None):
    """parent [entries, rows]: the row that each drafted row follows, or -1.  Written: mask [entries, rows,
    (rows + 31) // 32], the rows that each sees, as bits; pos [entries, rows], the rows' positions."""
    status = _marshal.kv_pages_tree(pages._at, pages._index, seqs, n_rows, parent, mask, pos,
                                    None if stream is None else _page_stream(pages, stream))
    if status:
        _check(status)


def kv_pages_attention_tree(pages: KvPages, layer: int, seqs, q, out, mask, ws, n_rows=None, prefix_seq: int = 0,
                            shared_len: int = 0, max_len: int | None = None, scale: float | None = None, stream=None):
    """kv_pages_attention of the last rows of each sequence, which see what is before them and the rows in their mask."""
    status = _marshal.kv_pages_attention_tree(pages._at, pages._index, layer, seqs, n_rows, q, out, mask, prefix_seq,
                                              shared_len, max_len, scale, ws,
                                              None if stream is None else _page_stream(pages, stream))
    if status:
        _check(status)


def kv_pages_attention_tree_plan(pages: KvPages, n: int, max_rows: int, n_heads: int, shared_len: int = 0,
                                 max_len: int | None = None):
    """How kv_pages_attention_tree divides a call of these sizes, as kv_pages_attention_plan."""
    if max_len is None:
        max_len = pages.table.shape[1] * pages.page_len
    plan = _abi.AttentionPlan()
    _check(lib().kv_pages_attention_tree_plan(pages._ref, n, max_rows, n_heads, shared_len, max_len, C.byref(plan)))
    return plan


def kv_pages_accept_workspace_bytes(pages: KvPages, n: int, max_path: int) -> int:
    return lib().kv_pages_accept_workspace_bytes(pages._ref, n, max_path)


def kv_pages_accept(pages: KvPages, seqs, path, n_path, status, ws, rows: int, n_rows=None, stream=None):
    """Of the last n_rows[i] (or `rows`) positions of seqs[i] those of the rows path[i][:n_path[i]], which ascend, are
    kept, in every layer, and the others given back."""
    code = _marshal.kv_pages_accept(pages._at, pages._index, seqs, rows, n_rows, path, n_path, status, ws,
                                    None if stream is None else _page_stream(pages, stream))
    if code:
        _check(code)


def dllm_workspace_bytes_pages(handle, batch: int, seq: int, n_lm_pos: int) -> int:
    return lib().dllm_workspace_bytes_pages(handle, batch, seq, n_lm_pos)


def dllm_forward_pages(handle, tokens, pages: KvPages, seqs, lm_pos, out: Stats, ws, prefix_seq: int = 0,
                       shared_len: int = 0, max_len: int | None = None, row_scale=None, scale: float = 1.0,
                       probe: Probe | None = None, n_lm_pos: int | None = None, stream=None):
    """tokens [batch, seq]: the last seq positions of the sequences seqs of `pages`."""
    batch, seq = tokens.shape
    n_lm = lm_pos.shape[0] if n_lm_pos is None else n_lm_pos
    if max_len is None:
        max_len = pages.table.shape[1] * pages.page_len
    _check(lib().dllm_forward_pages(handle, _p(tokens), batch, seq, pages._ref, _ids(pages, seqs, batch), prefix_seq,
                                    shared_len, max_len, _p(lm_pos), n_lm, _p(row_scale), scale,
                                    None if probe is None else C.byref(probe), C.byref(out.c()), *_scratch(pages, ws),
                                    _page_stream(pages, stream)))


# ---------------------------------------------------------------- scheduler

def rps_select_pivots(base: Stats, m_pos, n_m: int, prm: RpsParams, plan, stream=None):
    _check(lib().rps_select_pivots(C.byref(base.c()), _p(m_pos), n_m, C.byref(prm), _p(plan), _stream(stream)))


def rps_build_branches(tokens, plan, anchor_first: bool, capacity: int, out, stream=None):
    _check(lib().rps_build_branches(_p(tokens), tokens.shape[-1], _p(plan), int(anchor_first), capacity, _p(out),
                                    _stream(stream)))


def rps_build_packed(tokens, plan, block_start: int, block_len: int, capacity: int, out, stream=None):
    """out[seq + capacity * block_len]: tokens, then one block copy per branch slot."""
    _check(lib().rps_build_packed(_p(tokens), tokens.shape[-1], _p(plan), block_start, block_len, capacity, _p(out),
                                  _stream(stream)))


def rps_lookahead_score(anchor: Stats, branches: Stats, branch_offset: int, n_m: int, plan, lam: float, dec,
                        anchor_logit=None, scores=None, deltas=None, stream=None):
    _check(lib().rps_lookahead_score(C.byref(anchor.c()), C.byref(branches.c()), branch_offset, n_m, _p(plan),
                                     _p(anchor_logit), lam, _p(scores), _p(deltas), _p(dec), _stream(stream)))


def rps_commit(tokens, m_pos, n_m: int, base: Stats, tau: float, n_m_out, committed, n_committed, dec=None,
               branches: Stats | None = None, branch_offset: int = 0, anchor: Stats | None = None, stream=None):
    _check(lib().rps_commit(_p(tokens), tokens.shape[-1], _p(m_pos), n_m, C.byref(base.c()), _p(dec),
                            None if branches is None else C.byref(branches.c()), branch_offset,
                            None if anchor is None else C.byref(anchor.c()), tau, _p(n_m_out), _p(committed),
                            _p(n_committed), _stream(stream)))


def sched_commit(tokens, m_pos, n_m: int, stats: Stats, rule: int, k: int, n_m_out, committed, n_committed,
                 stream=None):
    """Baseline scheduler commit (Eq. 2, top-k by confidence or by lowest entropy)."""
    _check(lib().sched_commit(_p(tokens), tokens.shape[-1], _p(m_pos), n_m, C.byref(stats.c()), rule, k,
                              _p(n_m_out), _p(committed), _p(n_committed), _stream(stream)))
