// Host side of the C ABI: argument validation, workspace planning and the
// stream-ordered launch sequence of one denoising forward and of the
// scheduler calls.  Nothing here allocates except dllm_model_create.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <string>
#include <vector>

#include "dllm_rps.h"
#include "kernels.h"

using namespace dllm;

struct dllm_model {
  dllm_model_desc desc;
  const void* emb;
  const void* lm_head;
  // Largest split-K and LM-head workspace of a forward of at most 64 (i + 1)
  // rows, filled as far as a query has needed it: smaller launches can take
  // more parts and need more than larger ones
  struct UpTo {
    static constexpr int kKept = 1024;
    size_t bytes[kKept];
    int n = 0;
  };
  mutable UpTo part_max, lm_max;
  mutable std::mutex upto_mu;
  std::vector<const void*> wqkv, wo, wgu, wdown;
  float2* rope;
  // kernel timing (dllm_profile_begin / end)
  std::vector<hipEvent_t> prof_ev;   // 2 per launch
  std::vector<int> prof_cls;
  int prof_used = 0;
  bool prof_on = false;
  uint32_t prof_mask = ~0u;   // classes bracketed while profiling
};

namespace {

// Brackets one launch with events when profiling is on.
struct ProfScope {
  dllm_model* m;
  hipStream_t s;
  int idx = -1;
  ProfScope(dllm_model* m_, hipStream_t s_, int cls) : m(m_), s(s_) {
    if (!m->prof_on || !((m->prof_mask >> cls) & 1u) || m->prof_used >= int(m->prof_cls.size())) return;
    idx = m->prof_used++;
    m->prof_cls[idx] = cls;
    (void)hipEventRecord(m->prof_ev[2 * idx], s);
  }
  ~ProfScope() {
    if (idx >= 0) (void)hipEventRecord(m->prof_ev[2 * idx + 1], s);
  }
};

}  // namespace

namespace {

thread_local std::string g_err;

dllm_status fail(dllm_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
dllm_status fail(dllm_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return s;
}

dllm_status hip_check(hipError_t e, const char* what) {
  if (e == hipSuccess) return DLLM_OK;
  return fail(DLLM_EHIP, "%s: %s", what, hipGetErrorString(e));
}

#define TRY_HIP(expr, what)                         \
  do {                                              \
    dllm_status st_ = hip_check((expr), (what));    \
    if (st_ != DLLM_OK) return st_;                 \
  } while (0)

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
int elem_bytes(int dtype) { return dtype == DLLM_BF16 ? 2 : 4; }

StatsOut to_out(const dllm_stats& s) {
  return StatsOut{s.H, s.lse, s.lmax, s.argmax, s.topk_id, s.topk_logit, s.k};
}

dllm_status check_stats(const dllm_stats* s, const char* name) {
  if (!s) return fail(DLLM_EINVAL, "%s is NULL", name);
  if (!s->H || !s->lse || !s->lmax || !s->argmax || !s->topk_id || !s->topk_logit)
    return fail(DLLM_EINVAL, "%s has a NULL array", name);
  if (s->k < 1 || s->k > DLLM_MAX_TOPK) return fail(DLLM_EINVAL, "%s.k = %d outside 1..%d", name, s->k, DLLM_MAX_TOPK);
  return DLLM_OK;
}

// Workspace layout of one forward (256-byte aligned regions).
struct FwdLayout {
  size_t x, a, q, k, vt, f, hl, lm, lmsrc, part, attn, rope, total;
  int vt_ld;
};

// split-K parts of the four projections of a forward over M rows, and the
// partial-tile workspace they share (one projection at a time)
struct GemmSplits {
  int qkv, o, gu, down;
  size_t bytes;
};

// splits as planned for M rows, bytes for `rows` of them
GemmSplits plan_gemms(const dllm_model_desc& d, int M, int rows) {
  const int dt = d.dtype;
  auto cdiv = [](int a, int b) { return (a + b - 1) / b; };
  const int tq = cdiv(3 * d.d_model, 256), to = cdiv(d.d_model, 256), tg = cdiv(d.d_ffn, 128);
  GemmSplits g;
  g.qkv = gemm_splits(GEMM_KIND_QKV, M, 3 * d.d_model, d.d_model, dt);
  g.o = gemm_splits(GEMM_KIND_RESID, M, d.d_model, d.d_model, dt);
  g.gu = d.d_ffn % 4 ? 1 : gemm_splits(GEMM_KIND_GATEUP, M, 2 * d.d_ffn, d.d_model, dt);
  g.down = gemm_splits(GEMM_KIND_RESID, M, d.d_model, d.d_ffn, dt);
  g.bytes = std::max(std::max(gemm_partial_bytes(rows, tq, g.qkv), gemm_partial_bytes(rows, to, g.o)),
                     std::max(gemm_partial_bytes(rows, tg, g.gu), gemm_partial_bytes(rows, to, g.down)));
  return g;
}
GemmSplits plan_gemms(const dllm_model_desc& d, int M) { return plan_gemms(d, M, M); }

// Row counts 64 i + 1 .. 64 i + 64 have the same tiles in every launch, and
// parts that only get dearer with the rows (their traffic), so the first of
// them has the most parts.
constexpr int kEnvRows = 64;
constexpr int kMaxRows = 1 << 24;   // of one forward
// the largest of bytes_of(0) .. bytes_of(n - 1), n >= 1; the first kKept running maxima stay with the model
template <class F>
size_t max_upto(const dllm_model* m, dllm_model::UpTo& u, int n, F bytes_of) {
  const int kept = std::min(n, dllm_model::UpTo::kKept);
  size_t b;
  {
    std::lock_guard<std::mutex> lock(m->upto_mu);
    for (; u.n < kept; ++u.n) u.bytes[u.n] = std::max(u.n ? u.bytes[u.n - 1] : 0, bytes_of(u.n));
    b = u.bytes[kept - 1];
  }
  for (int i = kept; i < n; ++i) b = std::max(b, bytes_of(i));
  return b;
}
// largest split-K workspace of a forward of at most M rows
size_t part_bytes_upto(const dllm_model* m, int M) {
  return max_upto(m, m->part_max, (M + kEnvRows - 1) / kEnvRows,
                  [&](int i) { return plan_gemms(m->desc, kEnvRows * i + 1, kEnvRows * (i + 1)).bytes; });
}
// and of its LM head over at most R rows (past the kept ones it grows with R)
size_t lm_bytes_upto(const dllm_model* m, int R) {
  auto own = [&](int r) { return lmhead_workspace(m->desc.dtype, r, m->desc.vocab); };
  const int n = std::min((R + kEnvRows - 1) / kEnvRows, dllm_model::UpTo::kKept);
  return std::max(max_upto(m, m->lm_max, n, [&](int i) { return own(kEnvRows * (i + 1)); }), own(R));
}

// packed lookahead layout of one forward (see dllm_forward_packed)
struct Packing {
  int S, b0, B, n_branch;
};

// Regions of a forward with `lm`, `part` and `attn` bytes for the LM head's
// partials, the split-K parts and the attention's key ranges; the others grow
// with batch, seq and R, the LM-head rows of the call (batch * n_lm_pos, or
// (1 + n_branch) * n_lm_pos packed).  paged: rows with positions
// of their own, which take a row each of the rotary table.
FwdLayout layout_forward(const dllm_model_desc& d, int batch, int seq, int R, size_t lm, size_t part, size_t attn,
                         bool paged = false) {
  FwdLayout L;
  const size_t T = elem_bytes(d.dtype);
  const size_t M = size_t(batch) * seq;
  L.vt_ld = int(align_up(seq, 8));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    size_t o = off;
    off = align_up(off + bytes, 256);
    return o;
  };
  L.x = take(M * d.d_model * 4);
  L.a = take(M * d.d_model * T);
  L.q = take(M * d.d_model * T);
  L.k = take(M * d.d_model * T);
  L.vt = take(size_t(batch) * d.n_heads * d.head_dim * L.vt_ld * T);
  L.f = take(M * d.d_ffn * T);
  L.hl = take(size_t(R) * d.d_model * T);
  L.lm = take(lm);
  L.lmsrc = take(size_t(R) * 8);
  L.part = take(part);
  L.attn = attn ? take(attn) : 0;
  L.rope = paged ? take(M * d.head_dim / 2 * sizeof(float2)) : 0;
  L.total = off;
  return L;
}

// what one forward needs
FwdLayout plan_forward(const dllm_model_desc& d, int batch, int seq, int R) {
  return layout_forward(d, batch, seq, R, lmhead_workspace(d.dtype, R, d.vocab), plan_gemms(d, batch * seq).bytes,
                        attn_partial_bytes(batch, d.n_heads, seq, d.head_dim));
}

// the heads and types of a model's pages, as far as the attention's workspace goes by them
dllm_kv_pages pages_shape(const dllm_model_desc& d) {
  dllm_kv_pages p{};
  p.n_layers = d.n_layers;
  p.n_kv_heads = d.n_heads;
  p.head_dim = d.head_dim;
  p.dtype = d.dtype;
  return p;
}

// what one forward over pages needs
FwdLayout plan_forward_pages(const dllm_model_desc& d, int batch, int seq, int R) {
  return layout_forward(d, batch, seq, R, lmhead_workspace(d.dtype, R, d.vocab), plan_gemms(d, batch * seq).bytes,
                        paged_attention_workspace(pages_shape(d), batch, seq, d.n_heads), true);
}

// what it and every forward of no more sequences, positions and LM-head rows
// needs (arguments past kMaxRows are refused by the forward)
size_t workspace_upto(const dllm_model* m, int64_t batch, int64_t seq, int64_t R) {
  const dllm_model_desc& d = m->desc;
  const int b = int(std::min<int64_t>(batch, kMaxRows)), s = int(std::min<int64_t>(seq, kMaxRows)),
            M = int(std::min<int64_t>(int64_t(b) * s, kMaxRows)), r = int(std::min<int64_t>(R, kMaxRows));
  return layout_forward(d, b, s, r, lm_bytes_upto(m, r), part_bytes_upto(m, M),
                        attn_partial_bytes_upto(M, d.n_heads, d.head_dim)).total;
}

// the same over pages: every forward of no more entries, rows and LM-head rows
size_t workspace_pages_upto(const dllm_model* m, int32_t batch, int32_t seq, int64_t R) {
  const dllm_model_desc& d = m->desc;
  const int b = std::min(batch, KV_MAX_SEQS), s = std::min(seq, kMaxRows),
            M = int(std::min<int64_t>(int64_t(b) * s, kMaxRows)), r = int(std::min<int64_t>(R, kMaxRows));
  return layout_forward(d, b, s, r, lm_bytes_upto(m, r), part_bytes_upto(m, M),
                        paged_attention_workspace_upto(pages_shape(d), b, s, d.n_heads), true).total;
}

}  // namespace

extern "C" {

int32_t dllm_abi_version(void) { return DLLM_ABI_VERSION; }

const char* dllm_last_error(void) { return g_err.c_str(); }

const char* dllm_status_string(dllm_status s) {
  switch (s) {
    case DLLM_OK: return "ok";
    case DLLM_EINVAL: return "invalid argument";
    case DLLM_ESHAPE: return "unsupported shape";
    case DLLM_EDTYPE: return "unknown dtype";
    case DLLM_ENOMEM: return "workspace too small";
    case DLLM_EHIP: return "HIP runtime error";
    case DLLM_EUNSUPPORTED: return "unsupported";
  }
  return "unknown status";
}

dllm_status dllm_model_create(const dllm_model_desc* desc, const dllm_weights* w, dllm_model** out) {
  if (!desc || !w || !out) return fail(DLLM_EINVAL, "dllm_model_create: NULL argument");
  *out = nullptr;
  const dllm_model_desc& d = *desc;
  if (d.dtype != DLLM_F32 && d.dtype != DLLM_BF16) return fail(DLLM_EDTYPE, "dtype %d", d.dtype);
  if (d.n_layers < 1 || d.n_heads < 1 || d.vocab < 2 || d.d_ffn < 1 || d.max_pos < 1)
    return fail(DLLM_ESHAPE, "non-positive model size");
  if (d.head_dim != 64 && d.head_dim != 128) return fail(DLLM_ESHAPE, "head_dim %d not in {64, 128}", d.head_dim);
  if (d.d_model != d.n_heads * d.head_dim) return fail(DLLM_ESHAPE, "d_model != n_heads * head_dim");
  if (d.d_model % 256 || d.d_model > 8192) return fail(DLLM_ESHAPE, "d_model %% 256 != 0 or d_model > 8192");
  if (d.d_ffn % 128) return fail(DLLM_ESHAPE, "d_ffn %% 128 != 0");
  if (d.mask_id < 0 || d.mask_id >= d.vocab) return fail(DLLM_EINVAL, "mask_id outside [0, vocab)");
  if (!(d.rms_eps > 0.f) || !(d.rope_base > 1.f)) return fail(DLLM_EINVAL, "rms_eps / rope_base");
  const size_t T = elem_bytes(d.dtype);
  if (size_t(d.vocab) * d.d_model * T >= (size_t(1) << 32) || size_t(2) * d.d_ffn * d.d_model * T >= (size_t(1) << 32))
    return fail(DLLM_ESHAPE, "a weight matrix exceeds 4 GiB");
  if (!w->emb || !w->lm_head || !w->wqkv || !w->wo || !w->wgu || !w->wdown)
    return fail(DLLM_EINVAL, "NULL weight pointer");
  for (int l = 0; l < d.n_layers; ++l)
    if (!w->wqkv[l] || !w->wo[l] || !w->wgu[l] || !w->wdown[l]) return fail(DLLM_EINVAL, "NULL weight of layer %d", l);

  // rotary table in double precision: angle = pos * base^(-2j/hd)
  const int half = d.head_dim / 2;
  std::vector<float2> tab(size_t(d.max_pos) * half);
  for (int p = 0; p < d.max_pos; ++p)
    for (int j = 0; j < half; ++j) {
      const double ang = double(p) * std::pow(double(d.rope_base), -2.0 * j / d.head_dim);
      tab[size_t(p) * half + j] = make_float2(float(std::cos(ang)), float(std::sin(ang)));
    }
  float2* rope = nullptr;
  TRY_HIP(hipMalloc(&rope, tab.size() * sizeof(float2)), "hipMalloc(rope table)");
  hipError_t e = hipMemcpy(rope, tab.data(), tab.size() * sizeof(float2), hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipFree(rope);
    return hip_check(e, "hipMemcpy(rope table)");
  }
  dllm_model* m = new dllm_model;
  m->desc = d;
  m->emb = w->emb;
  m->lm_head = w->lm_head;
  m->wqkv.assign(w->wqkv, w->wqkv + d.n_layers);
  m->wo.assign(w->wo, w->wo + d.n_layers);
  m->wgu.assign(w->wgu, w->wgu + d.n_layers);
  m->wdown.assign(w->wdown, w->wdown + d.n_layers);
  m->rope = rope;
  *out = m;
  return DLLM_OK;
}

void dllm_model_destroy(dllm_model* m) {
  if (!m) return;
  for (hipEvent_t e : m->prof_ev) (void)hipEventDestroy(e);
  (void)hipFree(m->rope);
  delete m;
}

dllm_status dllm_profile_begin(dllm_model* m, int32_t max_launches) {
  return dllm_profile_begin_classes(m, max_launches, ~0u);
}

dllm_status dllm_profile_begin_classes(dllm_model* m, int32_t max_launches, uint32_t class_mask) {
  if (!m || max_launches < 1) return fail(DLLM_EINVAL, "dllm_profile_begin: NULL model or max_launches < 1");
  if (class_mask == 0) return fail(DLLM_EINVAL, "dllm_profile_begin_classes: empty class mask");
  m->prof_mask = class_mask;
  const size_t need = size_t(2) * max_launches;
  while (m->prof_ev.size() < need) {
    hipEvent_t e;
    TRY_HIP(hipEventCreate(&e), "hipEventCreate");
    m->prof_ev.push_back(e);
  }
  m->prof_cls.assign(max_launches, 0);
  m->prof_used = 0;
  m->prof_on = true;
  return DLLM_OK;
}

dllm_status dllm_profile_end(dllm_model* m, float* ms, int32_t* launches) {
  if (!m || !ms || !launches) return fail(DLLM_EINVAL, "dllm_profile_end: NULL argument");
  if (!m->prof_on) return fail(DLLM_EINVAL, "dllm_profile_end without dllm_profile_begin");
  m->prof_on = false;
  for (int c = 0; c < DLLM_PROF_CLASSES; ++c) {
    ms[c] = 0.f;
    launches[c] = 0;
  }
  for (int i = 0; i < m->prof_used; ++i) {
    TRY_HIP(hipEventSynchronize(m->prof_ev[2 * i + 1]), "hipEventSynchronize");
    float t = 0.f;
    TRY_HIP(hipEventElapsedTime(&t, m->prof_ev[2 * i], m->prof_ev[2 * i + 1]), "hipEventElapsedTime");
    ms[m->prof_cls[i]] += t;
    launches[m->prof_cls[i]] += 1;
  }
  m->prof_used = 0;
  return DLLM_OK;
}

dllm_status dllm_mfma_ceiling(int32_t random_operands, float* tflops, dllm_stream stream) {
  if (!tflops) return fail(DLLM_EINVAL, "dllm_mfma_ceiling: NULL tflops");
  hipStream_t s = static_cast<hipStream_t>(stream);
  int dev = 0, cus = 0;
  TRY_HIP(hipGetDevice(&dev), "hipGetDevice");
  TRY_HIP(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev), "hipDeviceGetAttribute");
  const int wg = 2 * std::max(cus, 1);
  double flop = 0.0;
  TRY_HIP(dllm::mfma_calibration(random_operands != 0, 2000, wg, &flop, s), "mfma_calibration (warm-up)");
  hipEvent_t e0, e1;
  TRY_HIP(hipEventCreate(&e0), "hipEventCreate");
  if (hipEventCreate(&e1) != hipSuccess) {
    (void)hipEventDestroy(e0);
    return fail(DLLM_EHIP, "hipEventCreate");
  }
  float ms = 0.f;
  hipError_t e = hipEventRecord(e0, s);
  if (e == hipSuccess) e = dllm::mfma_calibration(random_operands != 0, 20000, wg, &flop, s);
  if (e == hipSuccess) e = hipEventRecord(e1, s);
  if (e == hipSuccess) e = hipEventSynchronize(e1);
  if (e == hipSuccess) e = hipEventElapsedTime(&ms, e0, e1);
  (void)hipEventDestroy(e0);
  (void)hipEventDestroy(e1);
  TRY_HIP(e, "mfma_calibration");
  *tflops = ms > 0.f ? float(flop / (double(ms) * 1e-3) / 1e12) : 0.f;
  return DLLM_OK;
}

size_t dllm_workspace_bytes(const dllm_model* m, int32_t batch, int32_t seq, int32_t n_lm_pos) {
  if (!m || batch < 1 || seq < 1 || n_lm_pos < 1) return 0;
  return workspace_upto(m, batch, seq, int64_t(batch) * n_lm_pos);
}

size_t dllm_workspace_bytes_pages(const dllm_model* m, int32_t batch, int32_t seq, int32_t n_lm_pos) {
  if (!m || batch < 1 || seq < 1 || n_lm_pos < 1) return 0;
  return workspace_pages_upto(m, batch, seq, int64_t(batch) * n_lm_pos);
}

size_t dllm_workspace_bytes_packed(const dllm_model* m, int32_t shared_len, int32_t block_len, int32_t n_branch,
                                   int32_t n_lm_pos) {
  if (!m || shared_len < 1 || block_len < 1 || n_branch < 0 || n_lm_pos < 1) return 0;
  return workspace_upto(m, 1, int64_t(shared_len) + int64_t(n_branch) * block_len, (int64_t(1) + n_branch) * n_lm_pos);
}

namespace {

// a batch over pages (see dllm_forward_pages); pages have been checked
struct Paging {
  const dllm_kv_pages* pages;
  const int32_t* seqs;
  int prefix_seq, shared_len, max_len;
};

dllm_status forward_impl(dllm_model* m, const int32_t* tokens, int32_t batch, int32_t seq, int32_t pos_offset,
                         const dllm_kv_cache* kv_prefix, const dllm_kv_cache* kv_out, const int32_t* lm_pos,
                         int32_t n_lm_pos, const float* row_scale, float scale, const dllm_probe* probe,
                         const dllm_stats* out, void* ws, size_t ws_bytes, dllm_stream stream, const Packing* pk,
                         const Paging* pg = nullptr) {
  if (!m) return fail(DLLM_EINVAL, "dllm_forward: NULL model");
  if (!tokens || !lm_pos || !ws) return fail(DLLM_EINVAL, "dllm_forward: NULL tokens, lm_pos or ws");
  dllm_status st = check_stats(out, "out");
  if (st != DLLM_OK) return st;
  const dllm_model_desc& d = m->desc;
  if (batch < 1 || seq < 1 || n_lm_pos < 1 || n_lm_pos > (pk ? pk->S : seq))
    return fail(DLLM_ESHAPE, "batch %d seq %d n_lm_pos %d", batch, seq, n_lm_pos);
  const int n_pos = pk ? pk->S : seq;   // distinct positions of the call
  if (pos_offset < 0 || pos_offset + n_pos > d.max_pos)
    return fail(DLLM_ESHAPE, "positions %d..%d exceed max_pos %d", pos_offset, pos_offset + n_pos - 1, d.max_pos);
  if (pk) {
    if (batch != 1 || kv_out) return fail(DLLM_EINVAL, "packed lookahead: batch 1, no kv_out");
    if (pk->S < 1 || pk->B < 1 || (pk->B & (pk->B - 1)) || pk->n_branch < 0 || seq != pk->S + pk->n_branch * pk->B ||
        pk->b0 < 0 || pk->b0 + pk->B > pk->S)
      return fail(DLLM_ESHAPE, "packed lookahead: shared %d block %d..%d, seq %d", pk->S, pk->b0, pk->b0 + pk->B - 1,
                  seq);
  }
  if (!std::isfinite(scale)) return fail(DLLM_EINVAL, "scale is not finite");
  const size_t T = elem_bytes(d.dtype);
  const size_t M = size_t(batch) * seq;
  if (M * std::max(d.d_model, d.d_ffn) * T >= (size_t(1) << 32) || M > size_t(kMaxRows))
    return fail(DLLM_ESHAPE, "batch * seq too large");
  if (kv_prefix) {
    if (!kv_prefix->k || !kv_prefix->vt) return fail(DLLM_EINVAL, "kv_prefix has a NULL array");
    if (kv_prefix->len < 1 || kv_prefix->len > kv_prefix->cap || kv_prefix->cap % 8)
      return fail(DLLM_ESHAPE, "kv_prefix len %d cap %d (need 1 <= len <= cap, cap %% 8 == 0)", kv_prefix->len,
                  kv_prefix->cap);
  }
  if (kv_out) {
    if (!kv_out->k || !kv_out->vt) return fail(DLLM_EINVAL, "kv_out has a NULL array");
    if (batch != 1) return fail(DLLM_ESHAPE, "kv_out needs batch == 1");
    if (pos_offset + seq > kv_out->cap || kv_out->cap % 8) return fail(DLLM_ESHAPE, "kv_out capacity");
  }
  if (probe && probe->n > 0 && (!probe->row || !probe->token || !probe->logit))
    return fail(DLLM_EINVAL, "probe has a NULL array");
  // LM-head rows: every sequence's n_lm_pos rows; packed: the anchor's, then each branch's
  const int R = (pk ? 1 + pk->n_branch : batch) * n_lm_pos;
  const FwdLayout L = pg ? plan_forward_pages(d, batch, seq, R) : plan_forward(d, batch, seq, R);
  if (ws_bytes < L.total) return fail(DLLM_ENOMEM, "workspace %zu < %zu bytes", ws_bytes, L.total);

  hipStream_t s = static_cast<hipStream_t>(stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  float* x = reinterpret_cast<float*>(base + L.x);
  void* a = base + L.a;
  void* q = base + L.q;
  void* k = base + L.k;
  void* vt = base + L.vt;
  void* f = base + L.f;
  void* hl = base + L.hl;
  const int dm = d.d_model, F = d.d_ffn, H = d.n_heads, hd = d.head_dim, dt = d.dtype;
  const int Mi = int(M), vt_ld = pg ? int(align_up(M, 8)) : L.vt_ld;
  const GemmSplits gs = plan_gemms(d, Mi);
  float* part = reinterpret_cast<float*>(base + L.part);
  // the residual projections leave their partials to the RMSNorm that follows
  const SplitK sk_qkv{part, gs.qkv}, sk_o{part, gs.o}, sk_gu{part, gs.gu}, sk_down{part, gs.down};
  const int np_d = (dm + 255) / 256 * 256;   // partial row pitch of the d-wide projections
  int pending = 0;                            // split-K parts of x not yet added (0: none)
  // gathered row of each LM-head row (indexed modulo lm_n, per sequence) and
  // its row-scale index (its in-sequence position)
  const int32_t* lm_row = lm_pos;
  const int32_t* rs_idx = lm_pos;
  int lm_n = n_lm_pos;
  if (pk) {
    int32_t* rows = reinterpret_cast<int32_t*>(base + L.lmsrc);
    ProfScope ps(m, s, DLLM_PROF_OTHER);
    TRY_HIP(packed_lm_rows(pk->S, pk->b0, pk->B, pk->n_branch, lm_pos, n_lm_pos, rows, rows + R, s),
            "packed LM-head rows");
    lm_row = rows;
    rs_idx = rows + R;
    lm_n = R;
  }
  float2* rope_rows = reinterpret_cast<float2*>(base + L.rope);
  if (pg) {
    ProfScope ps(m, s, DLLM_PROF_OTHER);
    TRY_HIP(pages_rope_rows(*pg->pages, pg->seqs, batch, seq, d.max_pos, m->rope, hd / 2, rope_rows, s), "rope rows");
  }

  {
    ProfScope ps(m, s, DLLM_PROF_EMBED);
    TRY_HIP(embed_rmsnorm(dt, tokens, Mi, m->emb, dm, d.vocab, d.rms_eps, x, a, s), "embed_rmsnorm");
  }
  // a = rmsnorm(x), first adding the pending split-K partials of the last residual projection
  auto norm_into_a = [&]() -> dllm_status {
    ProfScope ps(m, s, DLLM_PROF_RMSNORM);
    if (pending > 1)
      TRY_HIP(resid_rmsnorm(dt, part, pending, np_d, Mi, x, dm, d.rms_eps, Mi, nullptr, 1, seq, a, s),
              "resid_rmsnorm");
    else
      TRY_HIP(rmsnorm(dt, x, dm, d.rms_eps, Mi, nullptr, 1, seq, a, s), "rmsnorm");
    pending = 0;
    return DLLM_OK;
  };
  for (int l = 0; l < d.n_layers; ++l) {
    if (l > 0)   // layer 0's comes with the embedding
      if (dllm_status e = norm_into_a(); e != DLLM_OK) return e;
    QkvOut qo{q, k, vt, seq, L.vt_ld, pos_offset, H, hd, dm, m->rope};
    if (pk) {
      qo.pack_S = pk->S;
      qo.pack_b0 = pk->b0;
      qo.pack_B = pk->B;
    }
    if (pg) {   // one sequence of all rows, each at its own row of the gathered table: q, k [H][M][hd], vt [H][hd][M]
      qo.seq = Mi;
      qo.vt_ld = vt_ld;
      qo.rope = rope_rows;
    }
    {
      ProfScope ps(m, s, DLLM_PROF_GEMM_QKV);
      TRY_HIP(gemm_qkv(dt, a, dm, m->wqkv[l], Mi, dm, qo, s, &sk_qkv), "gemm_qkv");
    }
    if (kv_out) {
      const size_t lay = size_t(l) * H * kv_out->cap * hd * T;
      ProfScope ps(m, s, DLLM_PROF_OTHER);
      TRY_HIP(kv_store(dt, k, vt, H, seq, hd, L.vt_ld, static_cast<uint8_t*>(kv_out->k) + lay,
                       static_cast<uint8_t*>(kv_out->vt) + lay, kv_out->cap, pos_offset, s),
              "kv_store");
    }
    if (pg) {
      // this layer's keys and values into the pages, then over all of them
      const int64_t entry = int64_t(seq) * hd, head = int64_t(Mi) * hd;
      {
        ProfScope ps(m, s, DLLM_PROF_OTHER);
        TRY_HIP(pages_write_vt(*pg->pages, l, pg->seqs, batch, seq, dllm_rows{k, entry, hd, head}, vt, vt_ld, s),
                "pages_write");
      }
      PagedAttn pa{};
      pa.p = *pg->pages;
      pa.layer = l;
      pa.seqs = pg->seqs;
      pa.n = batch;
      pa.max_rows = seq;
      pa.heads = H;
      pa.q = dllm_rows{q, entry, hd, head};
      pa.out = dllm_rows{a, int64_t(seq) * dm, dm, hd};
      pa.prefix_seq = pg->prefix_seq;
      pa.shared_len = pg->shared_len;
      pa.max_len = pg->max_len;
      pa.scale = 1.0f / sqrtf(float(hd));
      pa.part = reinterpret_cast<float*>(base + L.attn);
      ProfScope ps(m, s, DLLM_PROF_ATTENTION);
      TRY_HIP(paged_attention(pa, s), "attention over pages");
    }
    AttnArgs aa{};
    aa.q = q;
    aa.k = k;
    aa.vt = vt;
    aa.B = batch;
    aa.H = H;
    aa.Sq = seq;
    aa.hd = hd;
    aa.vt_ld = L.vt_ld;
    if (kv_prefix) {
      const size_t lay = size_t(l) * H * kv_prefix->cap * hd * T;
      aa.kp = static_cast<const uint8_t*>(kv_prefix->k) + lay;
      aa.vpt = static_cast<const uint8_t*>(kv_prefix->vt) + lay;
      aa.p_len = kv_prefix->len;
      aa.p_cap = kv_prefix->cap;
    }
    aa.o = a;
    if (L.attn) aa.kv_part = reinterpret_cast<float*>(base + L.attn);
    if (pk) {
      aa.pack_S = pk->S;
      aa.pack_b0 = pk->b0;
      aa.pack_B = pk->B;
    }
    if (!pg) {
      ProfScope ps(m, s, DLLM_PROF_ATTENTION);
      TRY_HIP(attention(dt, aa, s), "attention");
    }
    {
      ProfScope ps(m, s, DLLM_PROF_GEMM_O);
      TRY_HIP(gemm_resid(dt, a, dm, m->wo[l], dm, Mi, dm, dm, x, dm, s, &sk_o), "gemm_o");
      pending = sk_o.splits;
    }
    if (dllm_status e = norm_into_a(); e != DLLM_OK) return e;
    {
      ProfScope ps(m, s, DLLM_PROF_GEMM_GATEUP);
      TRY_HIP(gemm_swiglu(dt, a, dm, m->wgu[l], Mi, F, dm, f, s, &sk_gu), "gemm_swiglu");
    }
    {
      ProfScope ps(m, s, DLLM_PROF_GEMM_DOWN);
      TRY_HIP(gemm_resid(dt, f, F, m->wdown[l], F, Mi, dm, F, x, dm, s, &sk_down), "gemm_down");
      pending = sk_down.splits;
    }
  }
  {
    ProfScope ps(m, s, DLLM_PROF_RMSNORM);
    if (pending > 1)
      TRY_HIP(resid_rmsnorm(dt, part, pending, np_d, Mi, x, dm, d.rms_eps, R, lm_row, lm_n, seq, hl, s),
              "final resid_rmsnorm");
    else
      TRY_HIP(rmsnorm(dt, x, dm, d.rms_eps, R, lm_row, lm_n, seq, hl, s), "final rmsnorm");
  }
  {
    ProfScope ps(m, s, DLLM_PROF_LMHEAD);
    TRY_HIP(lmhead_partials(dt, hl, m->lm_head, R, dm, d.vocab, row_scale, rs_idx, lm_n, n_pos, scale,
                            d.mask_id, base + L.lm, s),
            "lm head");
  }
  {
    ProfScope ps(m, s, DLLM_PROF_LMHEAD_MERGE);
    TRY_HIP(lmhead_merge(dt, R, d.vocab, to_out(*out), base + L.lm, s), "lm head merge");
  }
  if (probe && probe->n > 0) {
    ProfScope ps(m, s, DLLM_PROF_OTHER);
    TRY_HIP(probe_logits(dt, hl, m->lm_head, dm, d.vocab, R, probe->row, probe->token, probe->n, row_scale, rs_idx,
                         lm_n, n_pos, scale, probe->logit, s),
            "probe");
  }
  return DLLM_OK;
}

}  // namespace

dllm_status dllm_forward(dllm_model* m, const int32_t* tokens, int32_t batch, int32_t seq, int32_t pos_offset,
                         const dllm_kv_cache* kv_prefix, const dllm_kv_cache* kv_out, const int32_t* lm_pos,
                         int32_t n_lm_pos, const float* row_scale, float scale, const dllm_probe* probe,
                         const dllm_stats* out, void* ws, size_t ws_bytes, dllm_stream stream) {
  return forward_impl(m, tokens, batch, seq, pos_offset, kv_prefix, kv_out, lm_pos, n_lm_pos, row_scale, scale, probe,
                      out, ws, ws_bytes, stream, nullptr);
}

dllm_status dllm_forward_packed(dllm_model* m, const int32_t* tokens, int32_t shared_len, int32_t block_start,
                                int32_t block_len, int32_t n_branch, int32_t pos_offset, const dllm_kv_cache* kv_prefix,
                                const int32_t* lm_pos, int32_t n_lm_pos, const float* row_scale, float scale,
                                const dllm_probe* probe, const dllm_stats* out, void* ws, size_t ws_bytes,
                                dllm_stream stream) {
  if (n_branch < 0 || block_len < 1 || shared_len < 1)
    return fail(DLLM_ESHAPE, "packed lookahead: shared %d, %d branches of %d", shared_len, n_branch, block_len);
  const Packing pk{shared_len, block_start, block_len, n_branch};
  return forward_impl(m, tokens, 1, shared_len + n_branch * block_len, pos_offset, kv_prefix, nullptr, lm_pos,
                      n_lm_pos, row_scale, scale, probe, out, ws, ws_bytes, stream, &pk);
}

size_t vocab_entropy_topk_workspace_bytes(int32_t R, int32_t vocab) {
  if (R < 1 || vocab < 2) return 0;
  return std::max(lmhead_workspace(DLLM_F32, R, vocab), lmhead_workspace(DLLM_BF16, R, vocab));
}

dllm_status vocab_entropy_topk(const void* hidden, const void* w_lm, int32_t R, int32_t d, int32_t vocab,
                               int32_t dtype, const float* row_scale, float scale, int32_t mask_id,
                               const dllm_stats* out, void* ws, size_t ws_bytes, dllm_stream stream) {
  if (!hidden || !w_lm || !ws) return fail(DLLM_EINVAL, "vocab_entropy_topk: NULL hidden, w_lm or ws");
  if (dtype != DLLM_F32 && dtype != DLLM_BF16) return fail(DLLM_EDTYPE, "dtype %d", dtype);
  dllm_status st = check_stats(out, "out");
  if (st != DLLM_OK) return st;
  if (R < 1 || vocab < 2 || d < 1) return fail(DLLM_ESHAPE, "R %d vocab %d d %d", R, vocab, d);
  const int kstage = dtype == DLLM_BF16 ? 64 : 32;
  if (d % kstage) return fail(DLLM_ESHAPE, "d %% %d != 0", kstage);
  const size_t T = elem_bytes(dtype);
  if (size_t(vocab) * d * T >= (size_t(1) << 32) || size_t(R) * d * T >= (size_t(1) << 32))
    return fail(DLLM_ESHAPE, "operand exceeds 4 GiB");
  if (mask_id >= vocab) return fail(DLLM_EINVAL, "mask_id >= vocab");
  if (!std::isfinite(scale)) return fail(DLLM_EINVAL, "scale is not finite");
  const size_t need = vocab_entropy_topk_workspace_bytes(R, vocab);
  if (ws_bytes < need) return fail(DLLM_ENOMEM, "workspace %zu < %zu bytes", ws_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  TRY_HIP(lmhead_partials(dtype, hidden, w_lm, R, d, vocab, row_scale, nullptr, R, R, scale, mask_id, ws, s),
          "vocab_entropy_topk");
  return hip_check(lmhead_merge(dtype, R, vocab, to_out(*out), ws, s), "vocab_entropy_topk merge");
}

// ---------------------------------------------------------------- allocation-free LM head

// Partial statistics of vocab_entropy_topk_noalloc, held by every device the
// library runs on until the process ends.  Host code never passes the array's
// name to a kernel (on the host it is only a stand-in for the symbol): the
// device address comes from hipGetSymbolAddress, once per device.
static __device__ __align__(256) uint8_t scratch[DLLM_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch[kMaxDevices] = {};

// Device address of `scratch` on device `dev`, looked up on the first call
// for that device with the device current.
dllm_status scratch_address(int dev, void** out) {
  if (dev < 0 || dev >= kMaxDevices) return fail(DLLM_EUNSUPPORTED, "device %d beyond %d devices", dev, kMaxDevices);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch[dev]) {
    int cur = -1;
    TRY_HIP(hipGetDevice(&cur), "hipGetDevice");
    if (cur != dev) TRY_HIP(hipSetDevice(dev), "hipSetDevice");
    void* p = nullptr;
    const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (cur != dev) (void)hipSetDevice(cur);
    TRY_HIP(e, "hipGetSymbolAddress(scratch)");
    if (!p) return fail(DLLM_EHIP, "hipGetSymbolAddress(scratch) returned NULL");
    g_scratch[dev] = p;
  }
  *out = g_scratch[dev];
  return DLLM_OK;
}

}  // namespace

dllm_status vocab_entropy_topk_noalloc(const void* hidden, const void* w_lm, int32_t R, int32_t d, int32_t vocab,
                                       int32_t dtype, const float* row_scale, float scale, int32_t mask_id,
                                       const dllm_stats* out, dllm_stream stream) {
  if (R < 1 || vocab < 2) return fail(DLLM_ESHAPE, "R %d vocab %d", R, vocab);
  const size_t need = vocab_entropy_topk_workspace_bytes(R, vocab);
  if (need > size_t(DLLM_NOALLOC_SCRATCH_BYTES))
    return fail(DLLM_ENOMEM, "vocab_entropy_topk_noalloc: R %d x vocab %d needs %zu bytes of partials, beyond the "
                "%zu-byte device scratch", R, vocab, need, size_t(DLLM_NOALLOC_SCRATCH_BYTES));
  hipStream_t s = static_cast<hipStream_t>(stream);
  int dev = -1;
  if (s) {
    TRY_HIP(hipStreamGetDevice(s, &dev), "hipStreamGetDevice");
  } else {
    TRY_HIP(hipGetDevice(&dev), "hipGetDevice");
  }
  void* ws = nullptr;
  dllm_status st = scratch_address(dev, &ws);
  if (st != DLLM_OK) return st;
  // every partial slot the merge reads is written by the partials kernel of
  // the same call: nothing in the scratch has to start at zero
  return vocab_entropy_topk(hidden, w_lm, R, d, vocab, dtype, row_scale, scale, mask_id, out, ws,
                            size_t(DLLM_NOALLOC_SCRATCH_BYTES), stream);
}

dllm_status rps_select_pivots(const dllm_stats* base, const int32_t* m_pos, int32_t n_m, const rps_params* prm,
                              rps_plan* plan, dllm_stream stream) {
  dllm_status st = check_stats(base, "base");
  if (st != DLLM_OK) return st;
  if (!m_pos || !prm || !plan) return fail(DLLM_EINVAL, "rps_select_pivots: NULL argument");
  if (n_m < 1 || n_m > RPS_MAX_MASKED) return fail(DLLM_ESHAPE, "n_m %d outside 1..%d", n_m, RPS_MAX_MASKED);
  if (prm->mode != RPS_PIVOT_PAPER && prm->mode != RPS_PIVOT_BAND) return fail(DLLM_EINVAL, "mode %d", prm->mode);
  if (prm->k_max < 1 || prm->k_max > base->k) return fail(DLLM_EINVAL, "k_max %d outside 1..k", prm->k_max);
  if (prm->n_cand < 1 || prm->n_cand > prm->k_max) return fail(DLLM_EINVAL, "n_cand %d outside 1..k_max", prm->n_cand);
  if (prm->n_pivots < 1 || prm->n_pivots > RPS_MAX_PIVOTS) return fail(DLLM_EINVAL, "n_pivots %d", prm->n_pivots);
  if (prm->max_branch < 1 || prm->max_branch > RPS_MAX_BRANCH) return fail(DLLM_EINVAL, "max_branch %d", prm->max_branch);
  if (!(prm->r >= 0.f) || !(prm->pct_lo >= 0.f) || !(prm->pct_hi <= 100.f) || !(prm->pct_lo <= prm->pct_hi) ||
      !std::isfinite(prm->tau_pivot))
    return fail(DLLM_EINVAL, "r / percentile / tau_pivot out of range");
  return hip_check(rps_select(to_out(*base), m_pos, n_m, *prm, plan, static_cast<hipStream_t>(stream)),
                   "rps_select_pivots");
}

dllm_status rps_build_branches(const int32_t* tokens, int32_t seq, const rps_plan* plan, int32_t anchor_first,
                               int32_t capacity, int32_t* out, dllm_stream stream) {
  if (!tokens || !plan || !out) return fail(DLLM_EINVAL, "rps_build_branches: NULL argument");
  if (seq < 1 || capacity < 1 || capacity > RPS_MAX_BRANCH + 1)
    return fail(DLLM_ESHAPE, "seq %d capacity %d", seq, capacity);
  return hip_check(rps_branches(tokens, seq, plan, anchor_first ? 1 : 0, capacity, out,
                                static_cast<hipStream_t>(stream)),
                   "rps_build_branches");
}

dllm_status rps_build_packed(const int32_t* tokens, int32_t seq, const rps_plan* plan, int32_t block_start,
                             int32_t block_len, int32_t capacity, int32_t* out, dllm_stream stream) {
  if (!tokens || !plan || !out) return fail(DLLM_EINVAL, "rps_build_packed: NULL argument");
  if (seq < 1 || capacity < 0 || capacity > RPS_MAX_BRANCH || block_len < 1 || block_start < 0 ||
      block_start + block_len > seq)
    return fail(DLLM_ESHAPE, "rps_build_packed: seq %d block %d..%d capacity %d", seq, block_start,
                block_start + block_len - 1, capacity);
  return hip_check(rps_branches_packed(tokens, seq, plan, block_start, block_len, capacity, out,
                                       static_cast<hipStream_t>(stream)),
                   "rps_build_packed");
}

dllm_status rps_lookahead_score(const dllm_stats* anchor, const dllm_stats* branches, int32_t branch_offset,
                                int32_t n_m, const rps_plan* plan, const float* anchor_logit, float lambda,
                                float* scores, float* deltas, rps_decision* dec, dllm_stream stream) {
  dllm_status st = check_stats(anchor, "anchor");
  if (st == DLLM_OK) st = check_stats(branches, "branches");
  if (st != DLLM_OK) return st;
  if (!plan || !dec) return fail(DLLM_EINVAL, "rps_lookahead_score: NULL plan or dec");
  if (n_m < 1 || n_m > RPS_MAX_MASKED) return fail(DLLM_ESHAPE, "n_m %d", n_m);
  if (branch_offset < 0 || branch_offset > 1) return fail(DLLM_EINVAL, "branch_offset %d", branch_offset);
  if (!(lambda >= 0.f) || !std::isfinite(lambda)) return fail(DLLM_EINVAL, "lambda must be finite and >= 0");
  return hip_check(rps_score(to_out(*anchor), to_out(*branches), branch_offset, n_m, plan, anchor_logit, lambda,
                             scores, deltas, dec, static_cast<hipStream_t>(stream)),
                   "rps_lookahead_score");
}

dllm_status rps_commit(int32_t* tokens, int32_t seq, int32_t* m_pos, int32_t n_m, const dllm_stats* base,
                       const rps_decision* dec,
                       const dllm_stats* branches, int32_t branch_offset, const dllm_stats* anchor, float tau,
                       int32_t* n_m_out, int32_t* committed, int32_t* n_committed, dllm_stream stream) {
  dllm_status st = check_stats(base, "base");
  if (st != DLLM_OK) return st;
  if (!tokens || !m_pos || !n_m_out || !committed || !n_committed)
    return fail(DLLM_EINVAL, "rps_commit: NULL argument");
  if (n_m < 1 || n_m > RPS_MAX_MASKED) return fail(DLLM_ESHAPE, "n_m %d", n_m);
  if (seq < 1) return fail(DLLM_ESHAPE, "seq %d", seq);
  if (dec) {
    st = check_stats(branches, "branches");
    if (st != DLLM_OK) return st;
    if (branches->k != base->k) return fail(DLLM_EINVAL, "branches.k != base.k");
    if (branch_offset < 0 || branch_offset > 1) return fail(DLLM_EINVAL, "branch_offset %d", branch_offset);
  }
  if (anchor) {
    st = check_stats(anchor, "anchor");
    if (st != DLLM_OK) return st;
    if (anchor->k != base->k) return fail(DLLM_EINVAL, "anchor.k != base.k");
  }
  if (std::isnan(tau)) return fail(DLLM_EINVAL, "tau is NaN");
  StatsOut bo = to_out(*base);
  StatsOut br = dec ? to_out(*branches) : StatsOut{};
  StatsOut an = anchor ? to_out(*anchor) : StatsOut{};
  return hip_check(rps_commit_step(tokens, seq, m_pos, n_m, bo, dec, dec ? &br : nullptr, branch_offset,
                                   anchor ? &an : nullptr, tau, n_m_out, committed, n_committed,
                                   static_cast<hipStream_t>(stream)),
                   "rps_commit");
}

dllm_status sched_commit(int32_t* tokens, int32_t seq, int32_t* m_pos, int32_t n_m, const dllm_stats* stats,
                         int32_t rule, int32_t k, int32_t* n_m_out, int32_t* committed, int32_t* n_committed,
                         dllm_stream stream) {
  dllm_status st = check_stats(stats, "stats");
  if (st != DLLM_OK) return st;
  if (!tokens || !m_pos || !n_m_out || !committed || !n_committed)
    return fail(DLLM_EINVAL, "sched_commit: NULL argument");
  if (rule != SCHED_TOP_CONFIDENCE && rule != SCHED_LOW_ENTROPY) return fail(DLLM_EINVAL, "rule %d", rule);
  if (k < 1) return fail(DLLM_EINVAL, "k %d", k);
  if (n_m < 1 || n_m > RPS_MAX_MASKED) return fail(DLLM_ESHAPE, "n_m %d", n_m);
  if (seq < 1) return fail(DLLM_ESHAPE, "seq %d", seq);
  return hip_check(sched_commit_step(tokens, seq, m_pos, n_m, to_out(*stats), rule, k, n_m_out, committed,
                                     n_committed, static_cast<hipStream_t>(stream)),
                   "sched_commit");
}

// ---------------------------------------------------------------- paged key/value cache

namespace {

dllm_status check_pages(const dllm_kv_pages* p, const char* who) {
  if (!p) return fail(DLLM_EINVAL, "%s: NULL pages", who);
  if (!p->k || !p->vt || !p->refs || !p->table || !p->len) return fail(DLLM_EINVAL, "%s: pages has a NULL array", who);
  if (p->dtype != DLLM_F32 && p->dtype != DLLM_BF16) return fail(DLLM_EDTYPE, "%s: dtype %d", who, p->dtype);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(DLLM_ESHAPE, "%s: head_dim %d not in {64, 128}", who, p->head_dim);
  if (p->page_len < 16 || p->page_len > 256 || (p->page_len & (p->page_len - 1)))
    return fail(DLLM_ESHAPE, "%s: page_len %d not in {16, 32, 64, 128, 256}", who, p->page_len);
  if (p->n_layers < 1 || p->n_layers > KV_MAX_LAYERS || p->n_kv_heads < 1 || p->n_kv_heads > KV_MAX_HEADS || p->n_pages < 1 ||
      p->n_pages > KV_MAX_PAGES || p->max_seqs < 1 || p->max_seqs > KV_MAX_SEQS || p->max_blocks < 1 ||
      p->max_blocks > KV_MAX_POSITIONS / p->page_len)
    return fail(DLLM_ESHAPE, "%s: %d layers, %d pages, %d heads, %d sequences of %d pages", who, p->n_layers,
                p->n_pages, p->n_kv_heads, p->max_seqs, p->max_blocks);
  if ((reinterpret_cast<uintptr_t>(p->k) | reinterpret_cast<uintptr_t>(p->vt)) % 16)
    return fail(DLLM_EINVAL, "%s: k and vt need 16-byte alignment", who);
  return DLLM_OK;
}

dllm_status check_entries(const void* seqs, int32_t n, const char* who) {
  if (!seqs) return fail(DLLM_EINVAL, "%s: NULL sequences", who);
  if (n < 1 || n > KV_MAX_SEQS) return fail(DLLM_ESHAPE, "%s: %d entries outside 1..%d", who, n, KV_MAX_SEQS);
  return DLLM_OK;
}

dllm_status check_rows(const dllm_rows* r, int dtype, const char* who, const char* name) {
  if (!r || !r->p) return fail(DLLM_EINVAL, "%s: NULL %s", who, name);
  const int64_t T = elem_bytes(dtype);
  const int64_t most = int64_t(1) << 40;   // of a stride; products with 2^24 rows stay inside 64 bits
  if (r->seq < 0 || r->row < 0 || r->head < 0 || r->seq > most || r->row > most || r->head > most)
    return fail(DLLM_ESHAPE, "%s: strides of %s outside 0..2^40", who, name);
  if (reinterpret_cast<uintptr_t>(r->p) % 16 || r->seq * T % 16 || r->row * T % 16 || r->head * T % 16)
    return fail(DLLM_EINVAL, "%s: %s needs 16-byte aligned rows", who, name);
  return DLLM_OK;
}

// Whether two of the n * rows * heads rows of hd elements share one.  Strides
// that nest (each at least what the smaller ones reach over) cannot; for others
// the distances of all pairs are gone through: of two dims one by one, of the
// third the nearest multiple (at most 2^19 steps, as the sizes' product is at most 2^26).
bool rows_overlap(const dllm_rows& r, int n, int rows, int heads, int64_t hd) {
  struct Dim {
    int64_t stride, size;
  } d[3] = {{r.seq, n}, {r.row, rows}, {r.head, heads}};
  for (Dim& x : d)
    if (x.size == 1) x.stride = 0;
  std::sort(d, d + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  int64_t reach = hd;
  bool nested = true;
  for (const Dim& x : d) {
    nested = nested && (x.size == 1 || x.stride >= reach);
    reach += x.stride * (x.size - 1);
  }
  if (nested) return false;
  std::sort(d, d + 3, [](const Dim& a, const Dim& b) { return a.size < b.size; });
  const Dim &a = d[0], &b = d[1], &c = d[2];
  for (int64_t i = 0; i < a.size; ++i)
    for (int64_t j = i ? 1 - b.size : 0; j < b.size; ++j) {
      const int64_t t = i * a.stride + j * b.stride;   // k of the third: |t - k stride| < hd, not all of i, j, k 0
      if (c.stride == 0) {
        if (std::abs(t) < hd && (i || j || c.size > 1)) return true;
        continue;
      }
      for (int64_t k = t / c.stride - 1; k <= t / c.stride + 1; ++k)
        if (std::abs(k) < c.size && (i || j || k) && std::abs(t - k * c.stride) < hd) return true;
    }
  return false;
}

}  // namespace

dllm_status kv_pages_init(const dllm_kv_pages* pages, dllm_stream stream) {
  dllm_status st = check_pages(pages, "kv_pages_init");
  if (st != DLLM_OK) return st;
  return hip_check(pages_init(*pages, static_cast<hipStream_t>(stream)), "kv_pages_init");
}

dllm_status kv_pages_grow(const dllm_kv_pages* pages, const int32_t* seqs, const int32_t* add, int32_t n,
                          int32_t* status, dllm_stream stream) {
  dllm_status st = check_pages(pages, "kv_pages_grow");
  if (st == DLLM_OK) st = check_entries(seqs, n, "kv_pages_grow");
  if (st != DLLM_OK) return st;
  if (!add || !status) return fail(DLLM_EINVAL, "kv_pages_grow: NULL add or status");
  return hip_check(pages_grow(*pages, seqs, add, n, status, static_cast<hipStream_t>(stream)), "kv_pages_grow");
}

dllm_status kv_pages_fork(const dllm_kv_pages* pages, const int32_t* src, const int32_t* dst, const int32_t* keep,
                          int32_t n, int32_t* status, dllm_stream stream) {
  dllm_status st = check_pages(pages, "kv_pages_fork");
  if (st == DLLM_OK) st = check_entries(src, n, "kv_pages_fork");
  if (st == DLLM_OK) st = check_entries(dst, n, "kv_pages_fork");
  if (st != DLLM_OK) return st;
  if (!status) return fail(DLLM_EINVAL, "kv_pages_fork: NULL status");
  return hip_check(pages_fork(*pages, src, dst, keep, n, status, static_cast<hipStream_t>(stream)), "kv_pages_fork");
}

dllm_status kv_pages_free(const dllm_kv_pages* pages, const int32_t* seqs, const int32_t* keep, int32_t n,
                          int32_t* status, dllm_stream stream) {
  dllm_status st = check_pages(pages, "kv_pages_free");
  if (st == DLLM_OK) st = check_entries(seqs, n, "kv_pages_free");
  if (st != DLLM_OK) return st;
  if (!status) return fail(DLLM_EINVAL, "kv_pages_free: NULL status");
  return hip_check(pages_free(*pages, seqs, keep, n, status, static_cast<hipStream_t>(stream)), "kv_pages_free");
}

size_t kv_pages_compact_workspace_bytes(const dllm_kv_pages* pages) {
  return check_pages(pages, "kv_pages_compact_workspace_bytes") == DLLM_OK ? pages_compact_workspace(pages->n_pages) : 0;
}

dllm_status kv_pages_compact(const dllm_kv_pages* pages, int32_t* n_used, void* ws, size_t ws_bytes,
                             dllm_stream stream) {
  dllm_status st = check_pages(pages, "kv_pages_compact");
  if (st != DLLM_OK) return st;
  if (!n_used) return fail(DLLM_EINVAL, "kv_pages_compact: NULL n_used");
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 16) return fail(DLLM_EINVAL, "kv_pages_compact: ws NULL or not 16-byte aligned");
  const size_t need = pages_compact_workspace(pages->n_pages);
  if (ws_bytes < need) return fail(DLLM_ENOMEM, "workspace %zu < %zu bytes", ws_bytes, need);
  return hip_check(pages_compact(*pages, n_used, ws, static_cast<hipStream_t>(stream)), "kv_pages_compact");
}

dllm_status kv_pages_write(const dllm_kv_pages* pages, int32_t layer, const int32_t* seqs, int32_t n,
                           int32_t max_rows, const int32_t* n_rows, const dllm_rows* k, const dllm_rows* v,
                           dllm_stream stream) {
  dllm_status st = check_pages(pages, "kv_pages_write");
  if (st == DLLM_OK) st = check_entries(seqs, n, "kv_pages_write");
  if (st == DLLM_OK) st = check_rows(k, pages->dtype, "kv_pages_write", "k");
  if (st == DLLM_OK) st = check_rows(v, pages->dtype, "kv_pages_write", "v");
  if (st != DLLM_OK) return st;
  if (layer < 0 || layer >= pages->n_layers) return fail(DLLM_ESHAPE, "kv_pages_write: layer %d", layer);
  if (max_rows < 1 || max_rows > KV_MAX_ROWS) return fail(DLLM_ESHAPE, "kv_pages_write: max_rows %d", max_rows);
  return hip_check(pages_write(*pages, layer, seqs, n, max_rows, n_rows, *k, *v, static_cast<hipStream_t>(stream)),
                   "kv_pages_write");
}

namespace {

dllm_status check_attention(const dllm_kv_pages* pages, int32_t n, int32_t max_rows, int32_t n_heads,
                            const char* who) {
  dllm_status st = check_pages(pages, who);
  if (st != DLLM_OK) return st;
  if (n < 1 || n > KV_MAX_SEQS) return fail(DLLM_ESHAPE, "%s: %d entries outside 1..%d", who, n, KV_MAX_SEQS);
  if (max_rows < 1 || max_rows > KV_MAX_ROWS) return fail(DLLM_ESHAPE, "%s: max_rows %d", who, max_rows);
  if (n_heads < 1 || n_heads > KV_MAX_HEADS || n_heads % pages->n_kv_heads)
    return fail(DLLM_ESHAPE, "%s: %d heads over %d key heads", who, n_heads, pages->n_kv_heads);
  if (int64_t(n) * max_rows * n_heads > KV_MAX_HEAD_ROWS)
    return fail(DLLM_ESHAPE, "%s: %d x %d rows of %d heads", who, n, max_rows, n_heads);
  return DLLM_OK;
}

}  // namespace

size_t kv_pages_attention_workspace_bytes(const dllm_kv_pages* pages, int32_t n, int32_t max_rows, int32_t n_heads) {
  if (check_attention(pages, n, max_rows, n_heads, "kv_pages_attention_workspace_bytes") != DLLM_OK) return 0;
  return paged_attention_workspace(*pages, n, max_rows, n_heads);
}

namespace {

// both attentions: checks and launch (mask NULL: full or causal rows)
dllm_status attend(const char* who, const dllm_kv_pages* pages, int32_t layer, const int32_t* seqs, int32_t n,
                   int32_t max_rows, const int32_t* n_rows, int32_t n_heads, const dllm_rows* q, const dllm_rows* out,
                   bool causal, const uint32_t* mask, int32_t prefix_seq, int32_t shared_len, int32_t max_len,
                   float scale, void* ws, size_t ws_bytes, dllm_stream stream) {
  dllm_status st = check_attention(pages, n, max_rows, n_heads, who);
  if (st == DLLM_OK) st = check_entries(seqs, n, who);
  if (st == DLLM_OK) st = check_rows(q, pages->dtype, who, "q");
  if (st == DLLM_OK) st = check_rows(out, pages->dtype, who, "out");
  if (st != DLLM_OK) return st;
  const int64_t hd = pages->head_dim;
  if ((n > 1 && out->seq < hd) || (max_rows > 1 && out->row < hd) || (n_heads > 1 && out->head < hd))
    return fail(DLLM_ESHAPE, "%s: rows of out overlap", who);
  if (layer < 0 || layer >= pages->n_layers) return fail(DLLM_ESHAPE, "%s: layer %d", who, layer);
  if (shared_len < 0 || max_len < 0) return fail(DLLM_ESHAPE, "%s: shared_len %d max_len %d", who, shared_len, max_len);
  if (shared_len > 0 && (prefix_seq < 0 || prefix_seq >= pages->max_seqs))
    return fail(DLLM_EINVAL, "%s: prefix_seq %d outside 0..%d", who, prefix_seq, pages->max_seqs - 1);
  if (!(scale > 0.f) || !std::isfinite(scale)) return fail(DLLM_EINVAL, "%s: scale must be finite and > 0", who);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 16) return fail(DLLM_EINVAL, "%s: ws NULL or not 16-byte aligned", who);
  const size_t need = paged_attention_workspace(*pages, n, max_rows, n_heads);
  if (ws_bytes < need) return fail(DLLM_ENOMEM, "workspace %zu < %zu bytes", ws_bytes, need);
  // which rows of ragged entries are written is known on the device alone
  if (!n_rows && rows_overlap(*out, n, max_rows, n_heads, hd))
    return fail(DLLM_ESHAPE, "%s: rows of out overlap", who);
  PagedAttn a{};
  a.p = *pages;
  a.layer = layer;
  a.seqs = seqs;
  a.n_rows = n_rows;
  a.n = n;
  a.max_rows = max_rows;
  a.heads = n_heads;
  a.q = *q;
  a.out = *out;
  a.prefix_seq = prefix_seq;
  a.shared_len = shared_len;
  a.max_len = max_len;
  a.causal = causal;
  a.mask = mask;
  a.scale = scale;
  a.part = static_cast<float*>(ws);
  return hip_check(paged_attention(a, static_cast<hipStream_t>(stream)), who);
}

}  // namespace

dllm_status kv_pages_attention(const dllm_kv_pages* pages, int32_t layer, const int32_t* seqs, int32_t n,
                               int32_t max_rows, const int32_t* n_rows, int32_t n_heads, const dllm_rows* q,
                               const dllm_rows* out, int32_t prefix_seq, int32_t shared_len, int32_t max_len,
                               int32_t causal, float scale, void* ws, size_t ws_bytes, dllm_stream stream) {
  return attend("kv_pages_attention", pages, layer, seqs, n, max_rows, n_rows, n_heads, q, out, causal != 0, nullptr,
                prefix_seq, shared_len, max_len, scale, ws, ws_bytes, stream);
}

dllm_status kv_pages_attention_tree(const dllm_kv_pages* pages, int32_t layer, const int32_t* seqs, int32_t n,
                                    int32_t max_rows, const int32_t* n_rows, int32_t n_heads, const dllm_rows* q,
                                    const dllm_rows* out, const uint32_t* mask, int32_t prefix_seq,
                                    int32_t shared_len, int32_t max_len, float scale, void* ws, size_t ws_bytes,
                                    dllm_stream stream) {
  const char* who = "kv_pages_attention_tree";
  if (!mask) return fail(DLLM_EINVAL, "%s: NULL mask", who);
  if (max_rows > KV_TREE_MAX_ROWS) return fail(DLLM_ESHAPE, "%s: max_rows %d > %d", who, max_rows, KV_TREE_MAX_ROWS);
  return attend(who, pages, layer, seqs, n, max_rows, n_rows, n_heads, q, out, false, mask, prefix_seq, shared_len,
                max_len, scale, ws, ws_bytes, stream);
}

namespace {

dllm_status plan_of(const char* who, const dllm_kv_pages* pages, int32_t n, int32_t max_rows, int32_t n_heads,
                    int32_t shared_len, int32_t max_len, bool tree, kv_attention_plan* plan) {
  dllm_status st = check_attention(pages, n, max_rows, n_heads, who);
  if (st != DLLM_OK) return st;
  if (!plan) return fail(DLLM_EINVAL, "%s: NULL plan", who);
  if (shared_len < 0 || max_len < 0) return fail(DLLM_ESHAPE, "%s: shared_len %d max_len %d", who, shared_len, max_len);
  PagedAttn a{};
  a.p = *pages;
  a.n = n;
  a.max_rows = max_rows;
  a.heads = n_heads;
  a.shared_len = shared_len;
  a.max_len = max_len;
  *plan = paged_attention_plan(a, tree);
  return DLLM_OK;
}

}  // namespace

dllm_status kv_pages_attention_plan(const dllm_kv_pages* pages, int32_t n, int32_t max_rows, int32_t n_heads,
                                    int32_t shared_len, int32_t max_len, kv_attention_plan* plan) {
  return plan_of("kv_pages_attention_plan", pages, n, max_rows, n_heads, shared_len, max_len, false, plan);
}

dllm_status kv_pages_attention_tree_plan(const dllm_kv_pages* pages, int32_t n, int32_t max_rows, int32_t n_heads,
                                         int32_t shared_len, int32_t max_len, kv_attention_plan* plan) {
  const char* who = "kv_pages_attention_tree_plan";
  if (max_rows > KV_TREE_MAX_ROWS) return fail(DLLM_ESHAPE, "%s: max_rows %d > %d", who, max_rows, KV_TREE_MAX_ROWS);
  return plan_of(who, pages, n, max_rows, n_heads, shared_len, max_len, true, plan);
}

dllm_status dllm_forward_pages(dllm_model* m, const int32_t* tokens, int32_t batch, int32_t seq,
                               const dllm_kv_pages* pages, const int32_t* seqs, int32_t prefix_seq,
                               int32_t shared_len, int32_t max_len, const int32_t* lm_pos, int32_t n_lm_pos,
                               const float* row_scale, float scale, const dllm_probe* probe, const dllm_stats* out,
                               void* ws, size_t ws_bytes, dllm_stream stream) {
  if (!m) return fail(DLLM_EINVAL, "dllm_forward_pages: NULL model");
  const dllm_model_desc& d = m->desc;
  dllm_status st = check_attention(pages, batch, seq, d.n_heads, "dllm_forward_pages");
  if (st == DLLM_OK) st = check_entries(seqs, batch, "dllm_forward_pages");
  if (st != DLLM_OK) return st;
  if (pages->dtype != d.dtype) return fail(DLLM_EDTYPE, "dllm_forward_pages: pages of dtype %d, model %d", pages->dtype, d.dtype);
  if (pages->n_layers != d.n_layers || pages->n_kv_heads != d.n_heads || pages->head_dim != d.head_dim)
    return fail(DLLM_ESHAPE, "dllm_forward_pages: pages of %d layers and %d heads of %d", pages->n_layers,
                pages->n_kv_heads, pages->head_dim);
  if (shared_len < 0 || max_len < 0)
    return fail(DLLM_ESHAPE, "dllm_forward_pages: shared_len %d max_len %d", shared_len, max_len);
  if (shared_len > 0 && (prefix_seq < 0 || prefix_seq >= pages->max_seqs))
    return fail(DLLM_EINVAL, "dllm_forward_pages: prefix_seq %d outside 0..%d", prefix_seq, pages->max_seqs - 1);
  if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(DLLM_EINVAL, "dllm_forward_pages: ws not 16-byte aligned");
  const Paging pg{pages, seqs, prefix_seq, shared_len, max_len};
  return forward_impl(m, tokens, batch, seq, 0, nullptr, nullptr, lm_pos, n_lm_pos, row_scale, scale, probe, out, ws,
                      ws_bytes, stream, nullptr, &pg);
}

// ---------------------------------------------------------------- rotary positions, drafts

dllm_status dllm_rotary_frequencies(int32_t dim, double base, int32_t scaling, double factor, double original_len,
                                    double slow, double fast, double* freq, float* amplitude) {
  const char* who = "dllm_rotary_frequencies";
  if (!freq || !amplitude) return fail(DLLM_EINVAL, "%s: NULL freq or amplitude", who);
  if (dim < 2 || dim % 2) return fail(DLLM_ESHAPE, "%s: dim %d", who, dim);
  if (!(base > 0.0) || !std::isfinite(base)) return fail(DLLM_EINVAL, "%s: base must be finite and > 0", who);
  if (scaling < DLLM_ROTARY_PLAIN || scaling > DLLM_ROTARY_RAMP) return fail(DLLM_EINVAL, "%s: scaling %d", who, scaling);
  if (scaling != DLLM_ROTARY_PLAIN && !(factor >= 1.0 && std::isfinite(factor)))
    return fail(DLLM_EINVAL, "%s: factor must be finite and at least 1", who);
  if (scaling == DLLM_ROTARY_RAMP &&
      !(original_len > 0.0 && std::isfinite(original_len) && slow >= 0.0 && fast > slow && std::isfinite(fast)))
    return fail(DLLM_EINVAL, "%s: a ramp needs original_len > 0 and 0 <= slow < fast", who);
  constexpr double kTurn = 6.283185307179586;
  if (scaling == DLLM_ROTARY_BASE && dim > 2) base *= std::pow(factor, double(dim) / (dim - 2));
  for (int32_t j = 0; j < dim / 2; ++j) {
    double f = std::pow(base, -2.0 * j / dim);
    if (scaling == DLLM_ROTARY_LINEAR) f /= factor;
    if (scaling == DLLM_ROTARY_RAMP) {
      const double stay = std::min(1.0, std::max(0.0, (original_len * f / kTurn - slow) / (fast - slow)));
      f *= stay + (1.0 - stay) / factor;
    }
    freq[j] = f;
  }
  *amplitude = scaling == DLLM_ROTARY_RAMP ? float(0.1 * std::log(factor) + 1.0) : 1.0f;
  return DLLM_OK;
}

namespace {

dllm_status check_rotary(const dllm_rotary* r, const char* who) {
  if (!r) return fail(DLLM_EINVAL, "%s: NULL rot", who);
  if (r->head_dim != 64 && r->head_dim != 128)
    return fail(DLLM_ESHAPE, "%s: head_dim %d not in {64, 128}", who, r->head_dim);
  if (r->dim < 0 || r->dim > r->head_dim || r->dim % 16)
    return fail(DLLM_ESHAPE, "%s: dim %d is no multiple of 16 in 0..%d", who, r->dim, r->head_dim);
  if (r->layout != DLLM_ROTARY_HALVES && r->layout != DLLM_ROTARY_PAIRS)
    return fail(DLLM_EINVAL, "%s: layout %d", who, r->layout);
  if (r->dim > 0 && (!r->freq || reinterpret_cast<uintptr_t>(r->freq) % 8))
    return fail(DLLM_EINVAL, "%s: freq NULL or not 8-byte aligned", who);
  if (!std::isfinite(r->amplitude)) return fail(DLLM_EINVAL, "%s: amplitude must be finite", who);
  if (r->norm && (!(r->eps > 0.f) || !std::isfinite(r->eps)))
    return fail(DLLM_EINVAL, "%s: eps must be finite and > 0", who);
  if (r->norm && (reinterpret_cast<uintptr_t>(r->q_gain) | reinterpret_cast<uintptr_t>(r->k_gain)) % 16)
    return fail(DLLM_EINVAL, "%s: gains need 16-byte alignment", who);
  return DLLM_OK;
}

// rows that are rotated into `out`: in place, or to rows that do not overlap
dllm_status check_turned(const dllm_rows* in, const dllm_rows* out, int dtype, int n, int max_rows, bool ragged,
                         int heads, int head_dim, const char* who, const char* name) {
  dllm_status st = check_rows(in, dtype, who, name);
  if (st == DLLM_OK) st = check_rows(out, dtype, who, name);
  if (st != DLLM_OK) return st;
  if (in->p == out->p && ((n > 1 && in->seq != out->seq) || (max_rows > 1 && in->row != out->row) ||
                          (heads > 1 && in->head != out->head)))
    return fail(DLLM_EINVAL, "%s: %s in place needs the same strides in and out", who, name);
  if ((n > 1 && out->seq < head_dim) || (max_rows > 1 && out->row < head_dim) || (heads > 1 && out->head < head_dim) ||
      (!ragged && rows_overlap(*out, n, max_rows, heads, head_dim)))
    return fail(DLLM_ESHAPE, "%s: output rows of %s overlap", who, name);
  return DLLM_OK;
}

dllm_status check_sizes(int32_t n, int32_t max_rows, int32_t q_heads, int32_t k_heads, const char* who) {
  if (n < 1 || n > KV_MAX_SEQS) return fail(DLLM_ESHAPE, "%s: %d entries outside 1..%d", who, n, KV_MAX_SEQS);
  if (max_rows < 1 || max_rows > KV_MAX_ROWS) return fail(DLLM_ESHAPE, "%s: max_rows %d", who, max_rows);
  if (q_heads < 0 || q_heads > KV_MAX_HEADS || k_heads < 0 || k_heads > KV_MAX_HEADS || q_heads + k_heads < 1 ||
      int64_t(n) * max_rows * (q_heads + k_heads) > KV_MAX_HEAD_ROWS)
    return fail(DLLM_ESHAPE, "%s: %d x %d rows of %d and %d heads", who, n, max_rows, q_heads, k_heads);
  return DLLM_OK;
}

}  // namespace

dllm_status rotary_rows(const dllm_rotary* rot, int32_t dtype, const int32_t* pos, int32_t pos_offset, int32_t n,
                        int32_t max_rows, const int32_t* n_rows, int32_t q_heads, const dllm_rows* q,
                        const dllm_rows* q_out, int32_t k_heads, const dllm_rows* k, const dllm_rows* k_out,
                        dllm_stream stream) {
  const char* who = "rotary_rows";
  dllm_status st = check_rotary(rot, who);
  if (st != DLLM_OK) return st;
  if (dtype != DLLM_F32 && dtype != DLLM_BF16) return fail(DLLM_EDTYPE, "%s: dtype %d", who, dtype);
  st = check_sizes(n, max_rows, q_heads, k_heads, who);
  if (st == DLLM_OK && q_heads)
    st = check_turned(q, q_out, dtype, n, max_rows, n_rows != nullptr, q_heads, rot->head_dim, who, "q");
  if (st == DLLM_OK && k_heads)
    st = check_turned(k, k_out, dtype, n, max_rows, n_rows != nullptr, k_heads, rot->head_dim, who, "k");
  if (st != DLLM_OK) return st;
  RotaryRows a{};
  a.rot = *rot;
  a.pos = pos;
  a.pos_offset = pos_offset;
  a.n = n;
  a.max_rows = max_rows;
  a.n_rows = n_rows;
  a.q_heads = q_heads;
  a.k_heads = k_heads;
  if (q_heads) a.q = *q, a.q_out = *q_out;
  if (k_heads) a.k = *k, a.k_out = *k_out;
  return hip_check(dllm::rotary_rows(dtype, a, static_cast<hipStream_t>(stream)), who);
}

dllm_status kv_pages_append(const dllm_kv_pages* pages, int32_t layer, const int32_t* seqs, int32_t n,
                            int32_t max_rows, const int32_t* n_rows, const dllm_rotary* rot, const int32_t* pos,
                            int32_t n_heads, const dllm_rows* q, const dllm_rows* q_out, const dllm_rows* k,
                            const dllm_rows* v, dllm_stream stream) {
  const char* who = "kv_pages_append";
  dllm_status st = check_pages(pages, who);
  if (st == DLLM_OK) st = check_entries(seqs, n, who);
  if (st == DLLM_OK) st = check_rotary(rot, who);
  if (st != DLLM_OK) return st;
  if (rot->head_dim != pages->head_dim)
    return fail(DLLM_ESHAPE, "%s: rotation of heads of %d, pages of %d", who, rot->head_dim, pages->head_dim);
  st = check_sizes(n, max_rows, n_heads, pages->n_kv_heads, who);
  if (st == DLLM_OK) st = check_rows(k, pages->dtype, who, "k");
  if (st == DLLM_OK) st = check_rows(v, pages->dtype, who, "v");
  if (st == DLLM_OK && n_heads)
    st = check_turned(q, q_out, pages->dtype, n, max_rows, n_rows != nullptr, n_heads, rot->head_dim, who, "q");
  if (st != DLLM_OK) return st;
  if (layer < 0 || layer >= pages->n_layers) return fail(DLLM_ESHAPE, "%s: layer %d", who, layer);
  RotaryRows a{};
  a.rot = *rot;
  a.pos = pos;
  a.n = n;
  a.max_rows = max_rows;
  a.n_rows = n_rows;
  a.q_heads = n_heads;
  a.k_heads = pages->n_kv_heads;
  if (n_heads) a.q = *q, a.q_out = *q_out;
  a.k = *k;
  return hip_check(pages_append(*pages, layer, seqs, a, *v, static_cast<hipStream_t>(stream)), who);
}

dllm_status kv_pages_tree(const dllm_kv_pages* pages, const int32_t* seqs, int32_t n, int32_t max_rows,
                          const int32_t* n_rows, const int32_t* parent, uint32_t* mask, int32_t* pos,
                          dllm_stream stream) {
  const char* who = "kv_pages_tree";
  dllm_status st = check_pages(pages, who);
  if (st == DLLM_OK) st = check_entries(seqs, n, who);
  if (st != DLLM_OK) return st;
  if (!parent || !mask) return fail(DLLM_EINVAL, "%s: NULL parent or mask", who);
  if (max_rows < 1 || max_rows > KV_TREE_MAX_ROWS)
    return fail(DLLM_ESHAPE, "%s: max_rows %d outside 1..%d", who, max_rows, KV_TREE_MAX_ROWS);
  return hip_check(pages_tree(*pages, seqs, n, max_rows, n_rows, parent, mask, pos, static_cast<hipStream_t>(stream)),
                   who);
}

size_t kv_pages_accept_workspace_bytes(const dllm_kv_pages* pages, int32_t n, int32_t max_path) {
  if (check_pages(pages, "kv_pages_accept_workspace_bytes") != DLLM_OK || n < 1 || n > KV_MAX_SEQS || max_path < 1 ||
      max_path > KV_TREE_MAX_ROWS)
    return 0;
  return size_t(n) * max_path * sizeof(int32_t);
}

dllm_status kv_pages_accept(const dllm_kv_pages* pages, const int32_t* seqs, int32_t n, int32_t max_rows,
                            const int32_t* n_rows, const int32_t* path, int32_t max_path, const int32_t* n_path,
                            int32_t* status, void* ws, size_t ws_bytes, dllm_stream stream) {
  const char* who = "kv_pages_accept";
  dllm_status st = check_pages(pages, who);
  if (st == DLLM_OK) st = check_entries(seqs, n, who);
  if (st != DLLM_OK) return st;
  if (!path || !n_path || !status) return fail(DLLM_EINVAL, "%s: NULL path, n_path or status", who);
  if (max_rows < 1 || max_rows > KV_MAX_ROWS) return fail(DLLM_ESHAPE, "%s: max_rows %d", who, max_rows);
  if (max_path < 1 || max_path > KV_TREE_MAX_ROWS)
    return fail(DLLM_ESHAPE, "%s: max_path %d outside 1..%d", who, max_path, KV_TREE_MAX_ROWS);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 16) return fail(DLLM_EINVAL, "%s: ws NULL or not 16-byte aligned", who);
  const size_t need = kv_pages_accept_workspace_bytes(pages, n, max_path);
  if (ws_bytes < need) return fail(DLLM_ENOMEM, "workspace %zu < %zu bytes", ws_bytes, need);
  return hip_check(pages_accept(*pages, seqs, n, max_rows, n_rows, path, max_path, n_path, status, ws,
                                static_cast<hipStream_t>(stream)),
                   who);
}

}  // extern "C"
