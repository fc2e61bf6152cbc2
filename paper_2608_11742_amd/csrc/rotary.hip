// Queries and keys normed by head and rotated, in memory or on the way into the
// pages of a layer, where the values go with them.
//
// A wave takes a row and some of its heads.  Its lanes compute the row's
// angles, one pair of elements each, once for all heads: a position times a
// frequency in turns, less the nearest quarter, in 64 bits (at position 2^30 a
// turn is then known to 2^-23), sine and cosine of the rest in 32, exchanged
// through LDS.  Then a lane holds two 16-byte chunks of a head that are each
// other's partners (or, in pairs, hold them), so nothing but the norm's sum
// crosses lanes, and each element is read and written once.
//
// Values of an append are transposed through LDS in tiles of 64 positions by
// workgroups of their own in the same launch.
//
// Bound by memory.  16 x 512 rows of 32 + 8 heads of 128, normed: 168 MB read and
// written in 30.3 us, the rate of a large copy (34 us) passed a little because
// what was written before is partly in the last-level cache; with values into
// pages 201 MB in 48.5 us (floor 41), 33 where the rows are in that cache.  9 single
// tokens take 5.7 us, a launch and its dependent loads.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace dllm {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// what a launch rotates: queries, then keys
struct Rotation {
  dllm_rotary rot;
  const int32_t* pos;   // nullable
  int pos_offset;
  int n, max_rows, q_heads, k_heads;
  const int32_t* n_rows;
  dllm_rows q, q_out, k, k_out;   // (an append's k_out is the pages)
  int parts, steps;               // waves of a row, steps of heads each takes
};
// the cache that an append's rows go to
struct Append {
  dllm_kv_pages p;
  int layer;
  const int32_t* seqs;
  dllm_rows v;
  bool heads_first;
  int turn_wgs, tiles;
};

__device__ __forceinline__ int rows_of(const int32_t* n_rows, int b, int max_rows) {
  return n_rows ? min(max(n_rows[b], 0), max_rows) : max_rows;
}

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// sum over groups of N neighbouring lanes
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  v += moved<0xb1>(v);                          // lane ^ 1
  v += moved<0x4e>(v);                          // lane ^ 2
  if constexpr (N >= 8) v += moved<0x141>(v);   // a lane of the other four of eight
  if constexpr (N >= 16) v += moved<0x140>(v);  // a lane of the other eight of sixteen
  return v;
}

template <typename T, int HD>
struct Heads {
  static constexpr int E = Elem<T>::per_chunk;
  static constexpr int U = HD / (2 * E);   // lanes of a head
  static constexpr int HS = kWave / U;     // heads of a step
  static constexpr bool kHalf = sizeof(T) == 2;

  bool turns, pairs;   // this lane's elements are rotated, in pairs of neighbours
  int e0, e1;          // first elements of its two chunks
  float c[E], s[E];    // of its pairs

  // cs: the wave's exchange, HD / 2 pairs
  __device__ __forceinline__ void angles(const dllm_rotary& rot, int64_t pos, float2* cs) {
    const int lane = threadIdx.x & 63, u = lane % U, half = rot.dim / 2;
    pairs = rot.layout == DLLM_ROTARY_PAIRS;
    turns = u * E < half;
    e0 = turns && !pairs ? u * E : 2 * u * E;
    e1 = turns && !pairs ? e0 + half : e0 + E;
    if (half == 0) return;
    if (lane < half) {
      const double t = double(pos) * (rot.freq[lane] * 0.6366197723675814);   // quarter turns
      const double q = rint(t);
      float sn, cn;
      sincospif(0.5f * float(t - q), &sn, &cn);
      const int quarter = int(int64_t(q) & 3);
      const float x = quarter & 1 ? -sn : cn, y = quarter & 1 ? cn : sn;
      const float a = quarter & 2 ? -rot.amplitude : rot.amplitude;
      cs[lane] = float2{a * x, a * y};
    }
    // a wave's LDS operations are done in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const f32x4* mine = reinterpret_cast<const f32x4*>(cs + (turns ? u * E : 0));
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const f32x4 x = mine[i];
      c[2 * i] = x[0];
      s[2 * i] = x[1];
      c[2 * i + 1] = x[2];
      s[2 * i + 1] = x[3];
    }
  }

  __device__ __forceinline__ static void unpack(u32x4 w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kHalf) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
  __device__ __forceinline__ static u32x4 pack(const float* x) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = kHalf ? pack_bf16x2(x[2 * i], x[2 * i + 1]) : __float_as_uint(x[i]);
    return w;
  }

  // the lane's chunks of a head, in and out
  __device__ __forceinline__ void turn(u32x4& a, u32x4& b, const dllm_rotary& rot, const float (&g)[2 * E]) const {
    float x[2 * E];
    unpack(a, x);
    unpack(b, x + E);
    if (rot.norm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) sum = fmaf(x[i], x[i], sum);
      const float r = 1.0f / sqrtf(group_sum<U>(sum) * (1.0f / HD) + rot.eps);
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) x[i] = x[i] * r * g[i];
    }
    if (turns) {
      if (pairs) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float y = x[2 * i], z = x[2 * i + 1];
          x[2 * i] = c[i] * y - s[i] * z;
          x[2 * i + 1] = s[i] * y + c[i] * z;
        }
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float y = x[i], z = x[E + i];
          x[i] = c[i] * y - s[i] * z;
          x[E + i] = s[i] * y + c[i] * z;
        }
      }
    }
    a = pack(x);
    b = pack(x + E);
  }

  // Heads h0, h0 + 1, .. of a row from `in` to `out`, `steps` steps.  Rows that are
  // rotated in memory are read past the caches (kOnce; 16 x 512 rows of 40 heads
  // of 128: 35.6 us, 37.7 with plain loads).  An append's are not (51.8 against
  // 48.9), and neither stores past them: 41 us by itself, but 4 more for the
  // attention that reads the rows next than the 8 it saves.
  template <bool kOnce>
  __device__ __forceinline__ void heads(const dllm_rotary& rot, const float* gain, const T* in, int64_t in_head, T* out,
                                        int64_t out_head, int h0, int n_heads, int steps) const {
    float g[2 * E];
#pragma unroll
    for (int i = 0; i < 2 * E; ++i) g[i] = 1.f;
    if (rot.norm && gain) {
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(gain + e0 + i), z = *reinterpret_cast<const f32x4*>(gain + e1 + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          g[i + k] = y[k];
          g[E + i + k] = z[k];
        }
      }
    }
    for (int st = 0; st < steps; ++st) {
      const int h = h0 + st * HS + int(threadIdx.x & 63) / U, at = min(h, n_heads - 1);
      const T* src = in + at * in_head;
      const u32x4 *pa = reinterpret_cast<const u32x4*>(src + e0), *pb = reinterpret_cast<const u32x4*>(src + e1);
      u32x4 a = kOnce ? __builtin_nontemporal_load(pa) : *pa, b = kOnce ? __builtin_nontemporal_load(pb) : *pb;
      turn(a, b, rot, g);
      if (h < n_heads) {
        T* dst = out + h * out_head;
        *reinterpret_cast<u32x4*>(dst + e0) = a;
        *reinterpret_cast<u32x4*>(dst + e1) = b;
      }
    }
  }
};

// Wave item `x` of the launch: a row, and its share of the steps over heads.
template <typename T, int HD, bool kAppend>
__device__ __forceinline__ void turn_row(const Rotation& r, const Append& w, int x, float2* cs) {
  using H = Heads<T, HD>;
  const int part = x % r.parts, row = x / r.parts;
  if (row >= r.n * r.max_rows) return;
  const int b = row / r.max_rows, i = row % r.max_rows;
  const int count = rows_of(r.n_rows, b, r.max_rows);
  if (i >= count) return;
  int64_t at = r.pos_offset + int64_t(i);
  int seq = 0;
  if constexpr (kAppend) {
    seq = w.seqs[b];
    if (seq < 0 || seq >= w.p.max_seqs) return;
    at = min(max(w.p.len[seq], 0), w.p.max_blocks * w.p.page_len) - count + i;
  }
  const int q_steps = (r.q_heads + H::HS - 1) / H::HS, k_steps = (r.k_heads + H::HS - 1) / H::HS;
  const int s0 = part * r.steps, s1 = min(s0 + r.steps, q_steps + k_steps);
  H lanes;
  lanes.angles(r.rot, r.pos ? int64_t(r.pos[row]) : at, cs);
  if (s0 < q_steps) {
    const T* in = static_cast<const T*>(r.q.p) + b * r.q.seq + i * r.q.row;
    T* out = static_cast<T*>(r.q_out.p) + b * r.q_out.seq + i * r.q_out.row;
    lanes.template heads<!kAppend>(r.rot, r.rot.q_gain, in, r.q.head, out, r.q_out.head, s0 * H::HS, r.q_heads, min(s1, q_steps) - s0);
  }
  if (s1 <= q_steps) return;
  const int k0 = max(s0 - q_steps, 0);
  const T* in = static_cast<const T*>(r.k.p) + b * r.k.seq + i * r.k.row;
  T* out;
  int64_t head;
  if constexpr (kAppend) {
    // the row's page, if it is this sequence's alone and no later entry writes it
    if (at < 0) return;
    bool later = false;
    for (int o = b + 1 + int(threadIdx.x & 63); o < r.n; o += kWave) later |= w.seqs[o] == seq;
    if (__any(later)) return;
    const int page = w.p.table[size_t(seq) * w.p.max_blocks + int(at) / w.p.page_len];
    if (page < 0 || page >= w.p.n_pages || w.p.refs[page] > 1) return;
    head = int64_t(w.p.page_len) * HD;
    out = static_cast<T*>(w.p.k) + (size_t(w.layer) * w.p.n_pages + page) * w.p.n_kv_heads * head +
          (int(at) & (w.p.page_len - 1)) * HD;
  } else {
    head = r.k_out.head;
    out = static_cast<T*>(r.k_out.p) + b * r.k_out.seq + i * r.k_out.row;
  }
  lanes.template heads<!kAppend>(r.rot, r.rot.k_gain, in, r.k.head, out, head, k0 * H::HS, r.k_heads, s1 - q_steps - k0);
}

// Grids of two dimensions: the most rows there may be are 2^24 workgroups, 2^32
// threads, one more than a dimension can have.
dim3 grid_of(int64_t wgs) {
  const int64_t most = 1 << 22;
  return dim3(uint32_t(std::min(wgs, most)), uint32_t((wgs + most - 1) / most));
}
__device__ __forceinline__ int workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }

template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotation r) {
  __shared__ __attribute__((aligned(16))) float2 cs[kWaves][HD / 2];
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  turn_row<T, HD, false>(r, Append{}, workgroup() * kWaves + wave, cs[wave]);
}

constexpr int kTile = 64;   // positions of a workgroup's values, from a multiple of 64: pages are cut there too

// Values of entry b and one head in the positions of tile `tile`, through LDS so
// that each dim's positions are stored together, 16 bytes at a time where the
// rows fill them.
template <typename T, int HD>
struct Values {
  static constexpr int E = Elem<T>::per_chunk;
  static constexpr int CR = HD / E;                      // chunks per row
  static constexpr int PITCH = HD + 4 / int(sizeof(T));  // LDS row of one position: an odd number of words
  struct Shared {
    T sv[kTile * PITCH];
    int page_of[kTile / 16];
  };

  __device__ static void run(const Rotation& r, const Append& w, int b, int h, int tile, Shared& sh) {
    const dllm_kv_pages& p = w.p;
    const int tid = threadIdx.x, s = w.seqs[b];
    if (s < 0 || s >= p.max_seqs) return;
    int later = 0;
    for (int i = b + 1 + tid; i < r.n; i += kThreads) later |= w.seqs[i] == s;
    const int held = min(max(p.len[s], 0), p.max_blocks * p.page_len);
    const int first = held - rows_of(r.n_rows, b, r.max_rows);   // position of row 0 (can be negative)
    const int lo = max(first, 0), t0 = lo / kTile * kTile + tile * kTile;
    const int from = max(lo, t0), to = min(held, t0 + kTile);
    if (__syncthreads_or(later) || from >= to) return;
    if (tid < kTile / 16) {
      const int pos = t0 + tid * 16;
      int page = -1;
      if (pos + 16 > from && pos < to) {
        page = p.table[size_t(s) * p.max_blocks + pos / p.page_len];
        if (page >= p.n_pages || (page >= 0 && p.refs[page] > 1)) page = -1;
      }
      sh.page_of[tid] = page;
    }
    const int count = to - from;
    const T* vs = static_cast<const T*>(w.v.p) + int64_t(b) * w.v.seq + int64_t(h) * w.v.head +
                  int64_t(from - first) * w.v.row;
    for (int c = tid; c < count * CR; c += kThreads) {
      const int i = c / CR, e = c % CR * E;
      const u32x4 x = *reinterpret_cast<const u32x4*>(vs + int64_t(i) * w.v.row + e);
      uint32_t* row = reinterpret_cast<uint32_t*>(sh.sv + (from - t0 + i) * PITCH + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) row[k] = x[k];
    }
    __syncthreads();
    // 8 consecutive positions of one dim; 8 lanes side by side hold the tile's 64
    const int c0 = (from - t0) >> 3, nc = ((to - t0 + 7) >> 3) - c0;
    for (int c = tid; c < nc * HD; c += kThreads) {
      const int d = c / nc, at = (c0 + c % nc) * 8, page = sh.page_of[at >> 4];
      if (page < 0) continue;
      T* dst = static_cast<T*>(p.vt) +
               (((size_t(w.layer) * p.n_pages + page) * p.n_kv_heads + h) * HD + d) * p.page_len +
               ((t0 + at) & (p.page_len - 1));
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = load_f(sh.sv + min(max(at + i, from - t0), to - t0 - 1) * PITCH + d);
      if (at >= from - t0 && at + 8 <= to - t0) {
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<u32x4*>(dst) =
              u32x4{pack_values(x[0], x[1]), pack_values(x[2], x[3]), pack_values(x[4], x[5]), pack_values(x[6], x[7])};
        } else {
          reinterpret_cast<f32x4*>(dst)[0] = f32x4{x[0], x[1], x[2], x[3]};
          reinterpret_cast<f32x4*>(dst)[1] = f32x4{x[4], x[5], x[6], x[7]};
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (at + i >= from - t0 && at + i < to - t0) store_value(dst + i, x[i]);
      }
    }
  }
};

template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void append_kernel(Rotation r, Append w) {
  __shared__ union {
    __attribute__((aligned(16))) float2 cs[kWaves][HD / 2];
    typename Values<T, HD>::Shared values;
  } sh;
  const int x = workgroup(), wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  // the two kinds in even turns: with either first, the other's waits at the end
  // are not covered (16 x 512 rows of 32 + 8 + 8 heads: 49.5 us, 51 with queries and keys first)
  const int heads = w.p.n_kv_heads, values = w.tiles * heads * r.n, all = values + w.turn_wgs;
  if (x >= all) return;
  const int y = int(int64_t(x) * values / all);
  if (y == int(int64_t(x + 1) * values / all)) {
    turn_row<T, HD, true>(r, w, (x - y) * kWaves + wave, sh.cs[wave]);
    return;
  }
  const int b = y / (heads * w.tiles), z = y % (heads * w.tiles);
  const int h = w.heads_first ? z % heads : z / w.tiles, tile = w.heads_first ? z / heads : z % w.tiles;
  Values<T, HD>::run(r, w, b, h, tile, sh.values);
}

// How the steps over a row's heads are shared: a wave takes them all where the
// rows alone fill the chip.
constexpr int kCus = 256;
template <typename T, int HD>
void divide(Rotation& r) {
  const int steps = cdiv(r.q_heads, Heads<T, HD>::HS) + cdiv(r.k_heads, Heads<T, HD>::HS);
  const int64_t rows = int64_t(r.n) * r.max_rows;
  r.parts = int(std::max<int64_t>(1, std::min<int64_t>(steps, 16 * kCus / rows)));
  r.steps = cdiv(steps, r.parts);
  r.parts = cdiv(steps, r.steps);
}

Rotation rotation_of(const RotaryRows& a) {
  Rotation r{};
  r.rot = a.rot;
  r.pos = a.pos;
  r.pos_offset = a.pos_offset;
  r.n = a.n;
  r.max_rows = a.max_rows;
  r.n_rows = a.n_rows;
  r.q_heads = a.q_heads;
  r.k_heads = a.k_heads;
  r.q = a.q;
  r.q_out = a.q_out;
  r.k = a.k;
  r.k_out = a.k_out;
  return r;
}

template <typename T, int HD>
hipError_t launch_rows(Rotation r, hipStream_t s) {
  divide<T, HD>(r);
  const int64_t items = int64_t(r.n) * r.max_rows * r.parts;
  hipLaunchKernelGGL((rotary_kernel<T, HD>), grid_of((items + kWaves - 1) / kWaves), dim3(kThreads), 0, s, r);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_append(Rotation r, Append w, hipStream_t s) {
  divide<T, HD>(r);
  const int64_t items = int64_t(r.n) * r.max_rows * r.parts;
  w.turn_wgs = int((items + kWaves - 1) / kWaves);
  w.tiles = (r.max_rows + kTile - 2) / kTile + 1;
  w.heads_first = w.tiles == 2;
  const int64_t all = w.turn_wgs + int64_t(w.tiles) * w.p.n_kv_heads * r.n;
  hipLaunchKernelGGL((append_kernel<T, HD>), grid_of(all), dim3(kThreads), 0, s, r, w);
  return hipGetLastError();
}

}  // namespace

hipError_t rotary_rows(int dtype, const RotaryRows& a, hipStream_t s) {
  const Rotation r = rotation_of(a);
  if (dtype == DLLM_BF16) return a.rot.head_dim == 128 ? launch_rows<bf16_t, 128>(r, s) : launch_rows<bf16_t, 64>(r, s);
  return a.rot.head_dim == 128 ? launch_rows<float, 128>(r, s) : launch_rows<float, 64>(r, s);
}

hipError_t pages_append(const dllm_kv_pages& p, int layer, const int32_t* seqs, const RotaryRows& a, const dllm_rows& v,
                        hipStream_t s) {
  const Rotation r = rotation_of(a);
  Append w{};
  w.p = p;
  w.layer = layer;
  w.seqs = seqs;
  w.v = v;
  if (p.dtype == DLLM_BF16) return p.head_dim == 128 ? launch_append<bf16_t, 128>(r, w, s) : launch_append<bf16_t, 64>(r, w, s);
  return p.head_dim == 128 ? launch_append<float, 128>(r, w, s) : launch_append<float, 64>(r, w, s);
}

}  // namespace dllm
