// Attention over the pages of one layer: softmax(scale q k^T) v for the rows
// of a batch of sequences, one pass over the keys with a running maximum m,
// sum l and output o per row.
//
// One wave a row and head: a lane takes one key of 64 (its score), then one
// or two dims (its part of o).
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace dllm {

namespace {

constexpr int kRowWaves = 4;

__device__ __forceinline__ float load_v(const float* p) { return *p; }
__device__ __forceinline__ float load_v(const bf16_t* p) { return f16_lo(p->bits); }

template <typename T, int HD>
__global__ __launch_bounds__(kRowWaves * kWave) void row_attn_kernel(PagedAttn a) {
  __shared__ float sq[kRowWaves][HD], sp[kRowWaves][kWave];
  const dllm_kv_pages& p = a.p;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int h = blockIdx.y, b = blockIdx.z, i = blockIdx.x * kRowWaves + wave;
  const int s = a.seqs[b];
  const int rows = a.n_rows ? min(max(a.n_rows[b], 0), a.max_rows) : a.max_rows;
  if (i >= rows) return;
  const bool known = s >= 0 && s < p.max_seqs;
  const int most = p.max_blocks * p.page_len;
  const int held = known ? min(max(p.len[s], 0), most) : 0;
  const int limit = a.causal ? max(0, min(held, held - rows + i + 1)) : held;
  const bool has_prefix = a.shared_len > 0 && a.prefix_seq >= 0 && a.prefix_seq < p.max_seqs;
  const int shared = has_prefix ? min(a.shared_len, min(max(p.len[a.prefix_seq], 0), most)) / p.page_len * p.page_len : 0;
  const size_t layer = size_t(a.layer) * p.n_pages;
  const int kvh = h / (a.heads / p.n_kv_heads);
  auto page_of = [&](int pos) {
    const int32_t* t = p.table + size_t(pos < shared ? a.prefix_seq : s) * p.max_blocks;
    return (layer + min(max(t[pos / p.page_len], 0), p.n_pages - 1)) * p.n_kv_heads + kvh;
  };
  const T* q = static_cast<const T*>(a.q.p) + b * a.q.seq + i * a.q.row + h * a.q.head;
  for (int d = lane; d < HD; d += kWave) sq[wave][d] = load_f(q + d);
  __builtin_amdgcn_wave_barrier();
  float m = -INFINITY, l = 0.f, o[HD / kWave] = {};
  for (int t = 0; t < limit; t += kWave) {
    float x = -INFINITY;
    if (t + lane < limit) {
      const T* k = static_cast<const T*>(p.k) + (page_of(t + lane) * p.page_len + (t + lane) % p.page_len) * HD;
      float dot = 0.f;
      for (int d = 0; d < HD; ++d) dot = fmaf(sq[wave][d], load_f(k + d), dot);
      x = dot * a.scale;
    }
    const float top = fmaxf(m, wave_max(x)), ref = top == -INFINITY ? 0.f : top;
    const float e = expf(x - ref), alpha = expf(m - ref);
    m = top;
    l = l * alpha + wave_sum(e);
    sp[wave][lane] = e;
    __builtin_amdgcn_wave_barrier();
    for (int c = 0; c < HD / kWave; ++c) o[c] *= alpha;
    for (int j = 0; j < min(kWave, limit - t); ++j) {
      const T* v = static_cast<const T*>(p.vt) + page_of(t + j) * HD * p.page_len + (t + j) % p.page_len;
      for (int c = 0; c < HD / kWave; ++c)
        o[c] = fmaf(sp[wave][j], load_v(v + (c * kWave + lane) * p.page_len), o[c]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  T* out = static_cast<T*>(a.out.p) + b * a.out.seq + i * a.out.row + h * a.out.head;
  for (int c = 0; c < HD / kWave; ++c) store_f(out + c * kWave + lane, limit > 0 ? o[c] / l : 0.f);
}

}  // namespace

size_t paged_attention_workspace(const dllm_kv_pages&, int, int, int) { return 16; }

hipError_t paged_attention(const PagedAttn& a, hipStream_t s) {
  const dim3 grid(cdiv(a.max_rows, kRowWaves), a.heads, a.n), block(kRowWaves * kWave);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
    return hipGetLastError();
  };
  if (a.p.dtype == DLLM_BF16)
    return a.p.head_dim == 128 ? launch(row_attn_kernel<bf16_t, 128>) : launch(row_attn_kernel<bf16_t, 64>);
  return a.p.head_dim == 128 ? launch(row_attn_kernel<float, 128>) : launch(row_attn_kernel<float, 64>);
}

}  // namespace dllm
