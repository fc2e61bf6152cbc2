// Paged key/value cache: reference counts, tables and lengths on the device,
// pages copied and rows written.
//
// A call that changes tables is planned by one workgroup of 1024 threads: it
// checks the sequences (thread i: entry i), sums the pages they need, and
// counts the free pages with one contiguous run of page ids per wave, 64 at a
// time by ballot, so that a free page's rank in id order is the counts before
// its wave's run plus the bits before it; the page of rank r goes to the entry
// whose range of needs holds r.  The check comes before any store: a call that
// fails changes nothing.  What moves pages or many table entries is done by a
// second, chip-wide launch that reads the plan.  A plan is bound by the latency
// of three dependent loads and two scans (4 us up to 8192 pages, 280 GB of the
// 8B-class shape's; 8 us at 32768, 150 at 2^20), the second launch by memory.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace dllm {

namespace {

constexpr int kPlanThreads = 1024;   // = KV_MAX_SEQS: one entry a thread
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kNoError = 1 << 30;

static_assert(kPlanThreads >= KV_MAX_SEQS, "one entry of a call per thread");

struct PlanShared {
  int wave_sum[kPlanWaves];
  int err;
  uint32_t seen[KV_MAX_SEQS / 32];
  int off[KV_MAX_SEQS], first[KV_MAX_SEQS], seq[KV_MAX_SEQS];
};

// exclusive prefix sum over the workgroup, and the total
__device__ __forceinline__ int block_scan(int v, PlanShared& sh, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  __syncthreads();   // an earlier scan's sums have been read
  if (lane == kWave - 1) sh.wave_sum[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int t = sh.wave_sum[w];
    before += w < wave ? t : 0;
    total += t;
  }
  return before + x - v;
}

__device__ __forceinline__ void plan_begin(PlanShared& sh) {
  if (threadIdx.x == 0) sh.err = kNoError;
  for (int i = threadIdx.x; i < KV_MAX_SEQS / 32; i += kPlanThreads) sh.seen[i] = 0;
  __syncthreads();
}

// the entry's sequence, or an error where it is out of range or listed before
__device__ __forceinline__ int check_seq(const dllm_kv_pages& p, int s, PlanShared& sh, int& err) {
  if (s < 0 || s >= p.max_seqs) {
    err = KV_PAGES_ESEQ;
    return -1;
  }
  if (atomicOr(&sh.seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1u) err = KV_PAGES_ESEQ;
  return s;
}

// the lowest code of any thread
__device__ __forceinline__ int plan_error(int err, PlanShared& sh) {
  if (err != kNoError) atomicMin(&sh.err, err);
  __syncthreads();
  return sh.err;
}

__device__ __forceinline__ int blocks_of(int positions, int page_len) { return (positions + page_len - 1) / page_len; }

// positions a sequence holds, inside its table
__device__ __forceinline__ int held_of(const dllm_kv_pages& p, int s) {
  return min(max(p.len[s], 0), p.max_blocks * p.page_len);
}

// this wave's run of page ids
struct Run {
  int lo, hi;
};
__device__ __forceinline__ Run run_of(const dllm_kv_pages& p) {
  const int ids = (p.n_pages + kPlanThreads - 1) / kPlanThreads * kWave;
  const int lo = min(__builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6) * ids, p.n_pages);
  return Run{lo, min(lo + ids, p.n_pages)};
}
// f(first id, bits of the used ones) for every 64 ids of a run, the counts of
// 512 on their way together; ids past the run are neither used nor free.  f
// returns whether to go on.
template <class F>
__device__ __forceinline__ void for_ids(const dllm_kv_pages& p, Run r, F&& f) {
  constexpr int kBatch = 8;
  const int lane = threadIdx.x & 63;
  for (int i0 = r.lo; i0 < r.hi; i0 += kBatch * kWave) {
    int refs[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) refs[u] = p.refs[min(i0 + u * kWave + lane, p.n_pages - 1)];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = i0 + u * kWave;
      if (i >= r.hi || !f(i, __ballot(refs[u] > 0))) return;
    }
  }
}
// bits of the ids i .. i + 63 that lie in lo .. hi - 1
__device__ __forceinline__ uint64_t inside(int i, int lo, int hi) {
  const int a = min(max(lo - i, 0), 64), b = min(max(hi - i, 0), 64);
  const uint64_t below_b = b == 64 ? ~uint64_t(0) : (uint64_t(1) << b) - 1;
  return a == 64 ? 0 : below_b & ~((uint64_t(1) << a) - 1);
}
// bits below this lane's
__device__ __forceinline__ int bits_before(uint64_t m) {
  return __popcll(m & ((uint64_t(1) << (threadIdx.x & 63)) - 1));
}
__device__ __forceinline__ int count_free(const dllm_kv_pages& p, Run r) {
  int n = 0;
  for_ids(p, r, [&](int i, uint64_t used) {
    n += __popcll(inside(i, r.lo, r.hi) & ~used);
    return true;
  });
  return n;
}

// sum of the waves' counts, and of those before this wave
__device__ __forceinline__ int wave_scan(int n, PlanShared& sh, int& total) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();   // earlier sums have been read
  if ((threadIdx.x & 63) == 0) sh.wave_sum[wave] = n;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int t = sh.wave_sum[w];
    before += w < wave ? t : 0;
    total += t;
  }
  return __builtin_amdgcn_readfirstlane(before);
}

// Pages for the plan's entries: entry i (this thread's) needs `need` pages as
// blocks first .. of sequence seq; n_free: the free pages of this wave's run.
// False (and nothing stored) if the pool has fewer free ones.
__device__ __forceinline__ bool take_pages(const dllm_kv_pages& p, PlanShared& sh, Run run, int n_free, int seq,
                                           int first, int need) {
  const int tid = threadIdx.x;
  int total, have;
  // needs past the pool fail below as they are; up to there 1024 of them sum up to less than 2^31
  const int off = block_scan(min(need, p.n_pages + 1), sh, total);
  sh.off[tid] = off;
  sh.first[tid] = first;
  sh.seq[tid] = seq;
  int rank0 = wave_scan(n_free, sh, have);   // its barriers publish off, first and seq too
  if (total > have) return false;
  if (n_free == 0 || rank0 >= total) return true;
  for_ids(p, run, [&](int i0, uint64_t used) {
    const uint64_t free = inside(i0, run.lo, run.hi) & ~used;
    const int rank = rank0 + bits_before(free);
    rank0 += __popcll(free);
    if ((free >> (tid & 63) & 1) && rank < total) {
      // the last entry whose needs start at or before this rank (entries that need nothing share their start with the next)
      int a = 0, b = kPlanThreads;
      while (b - a > 1) {
        const int m = (a + b) >> 1;
        if (sh.off[m] <= rank) a = m;
        else b = m;
      }
      const int page = i0 + (tid & 63);
      p.table[size_t(sh.seq[a]) * p.max_blocks + sh.first[a] + rank - sh.off[a]] = page;
      p.refs[page] = 1;
    }
    return rank0 < total;
  });
  return true;
}

__global__ __launch_bounds__(256) void pages_init_kernel(dllm_kv_pages p) {
  const size_t entries = size_t(p.max_seqs) * p.max_blocks, step = size_t(gridDim.x) * 256;
  const size_t t = size_t(blockIdx.x) * 256 + threadIdx.x;
  for (size_t i = t; i < entries; i += step) p.table[i] = -1;
  for (size_t i = t; i < size_t(p.n_pages); i += step) p.refs[i] = 0;
  for (size_t i = t; i < size_t(p.max_seqs); i += step) p.len[i] = 0;
}

__global__ __launch_bounds__(kPlanThreads) void pages_grow_kernel(dllm_kv_pages p, const int32_t* __restrict__ seqs,
                                                                  const int32_t* __restrict__ add, int n,
                                                                  int32_t* status) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x;
  int err = kNoError, s = -1, held = 0, more = 0;
  const int want_s = tid < n ? seqs[tid] : 0, want_a = tid < n ? add[tid] : 0;
  const Run run = run_of(p);
  const int n_free = count_free(p, run);   // with the lists on their way
  plan_begin(sh);
  if (tid < n) {
    s = check_seq(p, want_s, sh, err);
    more = want_a;
    if (s >= 0) held = held_of(p, s);
    if (err == kNoError && (more < 0 || int64_t(held) + more > int64_t(p.max_blocks) * p.page_len)) err = KV_PAGES_ELEN;
  }
  err = plan_error(err, sh);
  if (err == kNoError) {
    const int first = blocks_of(held, p.page_len);
    const int need = tid < n ? blocks_of(held + more, p.page_len) - first : 0;
    if (!take_pages(p, sh, run, n_free, s, first, need)) err = KV_PAGES_EFULL;
    else if (tid < n) p.len[s] = held + more;
  }
  if (tid == 0) *status = err == kNoError ? KV_PAGES_OK : err;
}

// Fork plan: checks, cut pages' copies allocated, lengths of the new
// sequences; fork_apply_kernel fills their tables and the copies.
__global__ __launch_bounds__(kPlanThreads) void pages_fork_kernel(dllm_kv_pages p, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ dst,
                                                                  const int32_t* __restrict__ keep, int n,
                                                                  int32_t* status) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x;
  int err = kNoError, d = -1, m = 0;
  const int from = tid < n ? src[tid] : 0, to = tid < n ? dst[tid] : 0, cut = keep && tid < n ? keep[tid] : 0;
  const Run run = run_of(p);
  const int n_free = count_free(p, run);
  plan_begin(sh);
  if (tid < n) {
    d = check_seq(p, to, sh, err);
    if (from < 0 || from >= p.max_seqs || (d >= 0 && p.len[d] != 0)) err = KV_PAGES_ESEQ;
    if (err == kNoError) {
      const int held = held_of(p, from);
      m = keep ? cut : held;
      if (m < 0 || m > held) err = KV_PAGES_ELEN;
    }
  }
  err = plan_error(err, sh);   // every length has been read before one is stored
  if (err == kNoError) {
    const int need = tid < n && m % p.page_len ? 1 : 0;
    if (!take_pages(p, sh, run, n_free, d, m / p.page_len, need)) err = KV_PAGES_EFULL;
    else if (tid < n) p.len[d] = m;
  }
  if (tid == 0) *status = err == kNoError ? KV_PAGES_OK : err;
}

// one page array (keys or values of one layer) is copied in units of 16 KB
constexpr int kCopyThreads = 256;
constexpr int kCopyRegs = 4;
constexpr int kCopyUnit = kCopyThreads * kCopyRegs * 16;

// unit u of the copy of a page's arrays: (array, layer, 16 KB part)
__device__ __forceinline__ void copy_unit(const dllm_kv_pages& p, size_t page_bytes, int parts, int u, int from,
                                          int to) {
  const int part = u % parts, layer = (u / parts) >> 1;
  uint8_t* base = static_cast<uint8_t*>((u / parts) & 1 ? p.vt : p.k) + size_t(layer) * p.n_pages * page_bytes;
  const u32x4* s = reinterpret_cast<const u32x4*>(base + size_t(from) * page_bytes);
  u32x4* d = reinterpret_cast<u32x4*>(base + size_t(to) * page_bytes);
  const int n = int(page_bytes / 16), c0 = part * (kCopyUnit / 16) + int(threadIdx.x);
  u32x4 v[kCopyRegs];
#pragma unroll
  for (int i = 0; i < kCopyRegs; ++i) v[i] = s[min(c0 + i * kCopyThreads, n - 1)];
#pragma unroll
  for (int i = 0; i < kCopyRegs; ++i)
    if (c0 + i * kCopyThreads < n) d[c0 + i * kCopyThreads] = v[i];
}

// Workgroups first .. of the grid share the units of every entry's cut page;
// the others (blockIdx.x < n * row_wgs) fill the tables.
__global__ __launch_bounds__(kCopyThreads) void fork_apply_kernel(dllm_kv_pages p, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ dst, int n, int row_wgs,
                                                                  size_t page_bytes, int parts,
                                                                  const int32_t* __restrict__ status) {
  if (*status != KV_PAGES_OK) return;
  if (int(blockIdx.x) < n * row_wgs) {
    const int i = blockIdx.x / row_wgs;
    const int32_t* from = p.table + size_t(src[i]) * p.max_blocks;
    int32_t* to = p.table + size_t(dst[i]) * p.max_blocks;
    const int whole = p.len[dst[i]] / p.page_len;
    for (int j = (blockIdx.x % row_wgs) * kCopyThreads + threadIdx.x; j < whole; j += row_wgs * kCopyThreads) {
      const int page = from[j];
      to[j] = page;
      if (page >= 0 && page < p.n_pages) atomicAdd(p.refs + page, 1);
    }
    return;
  }
  const int units = p.n_layers * 2 * parts;
  for (int64_t t = int(blockIdx.x) - n * row_wgs; t < int64_t(n) * units; t += int(gridDim.x) - n * row_wgs) {
    const int i = int(t / units);
    const int s = src[i], d = dst[i], m = p.len[d], j = m / p.page_len;
    if (m % p.page_len == 0) continue;
    const int from = p.table[size_t(s) * p.max_blocks + j], to = p.table[size_t(d) * p.max_blocks + j];
    if (from < 0 || from >= p.n_pages) continue;
    copy_unit(p, page_bytes, parts, int(t % units), from, to);
  }
}

// entries j0 .. of a sequence's table that hold a page give it back
__device__ __forceinline__ void drop_entry(const dllm_kv_pages& p, int s, int j) {
  int32_t* e = p.table + size_t(s) * p.max_blocks + j;
  const int page = *e;
  if (page < 0) return;
  *e = -1;
  if (page < p.n_pages) atomicSub(p.refs + page, 1);
}

__global__ __launch_bounds__(kPlanThreads) void pages_free_kernel(dllm_kv_pages p, const int32_t* __restrict__ seqs,
                                                                  const int32_t* __restrict__ keep, int n,
                                                                  int32_t* status, bool drop_here) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x;
  int err = kNoError, s = -1, m = 0;
  const int want = tid < n ? seqs[tid] : 0, cut = keep && tid < n ? keep[tid] : 0;
  plan_begin(sh);
  if (tid < n) {
    s = check_seq(p, want, sh, err);
    m = keep ? cut : 0;
    if (err == kNoError) {
      const int held = held_of(p, s);
      if (m < 0 || m > held) {
        err = KV_PAGES_ELEN;
      } else if (m < held && m % p.page_len) {
        const int page = p.table[size_t(s) * p.max_blocks + m / p.page_len];
        if (page >= 0 && page < p.n_pages && p.refs[page] > 1) err = KV_PAGES_ESHARED;
      }
    }
  }
  sh.seq[tid] = s;
  sh.first[tid] = m;
  err = plan_error(err, sh);
  if (err == kNoError) {
    if (tid < n) p.len[s] = m;
    if (drop_here)
      for (int t = tid; t < n * p.max_blocks; t += kPlanThreads) {
        const int i = t / p.max_blocks, j = t % p.max_blocks;
        if (j >= blocks_of(sh.first[i], p.page_len)) drop_entry(p, sh.seq[i], j);
      }
  }
  if (tid == 0) *status = err == kNoError ? KV_PAGES_OK : err;
}

__global__ __launch_bounds__(256) void free_apply_kernel(dllm_kv_pages p, const int32_t* __restrict__ seqs,
                                                         const int32_t* __restrict__ status) {
  if (*status != KV_PAGES_OK) return;
  const int s = seqs[blockIdx.y], first = blocks_of(p.len[s], p.page_len);
  for (int j = first + blockIdx.x * 256 + threadIdx.x; j < p.max_blocks; j += gridDim.x * 256) drop_entry(p, s, j);
}

// Compaction plan in the workspace: [0] pages moved, then their new ids by
// old id (from n_used on), the old ids and the new ones by rank.
struct CompactPlan {
  int32_t* moved;
  int32_t* new_id;
  int32_t* from;
  int32_t* to;
};
__host__ __device__ CompactPlan compact_plan(void* ws, int n_pages) {
  int32_t* w = static_cast<int32_t*>(ws);
  return CompactPlan{w, w + 16, w + 16 + n_pages, w + 16 + 2 * size_t(n_pages)};
}

__global__ __launch_bounds__(kPlanThreads) void pages_compact_kernel(dllm_kv_pages p, int32_t* n_used, CompactPlan c) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const Run run = run_of(p);
  int total, holes, moved;
  int h = count_free(p, run), m = run.hi - run.lo - h;
  wave_scan(m, sh, total);
  // below `total` free ids are filled, from there on used ones move
  const int mid = min(max(total, run.lo), run.hi);
  h = m = 0;
  for_ids(p, run, [&](int i, uint64_t used) {
    h += __popcll(inside(i, run.lo, mid) & ~used);
    m += __popcll(inside(i, mid, run.hi) & used);
    return true;
  });
  h = wave_scan(h, sh, holes);
  m = wave_scan(m, sh, moved);   // as many holes below as used pages past them
  if (moved == 0) {   // nothing to list
    if (tid == 0) {
      *n_used = total;
      *c.moved = 0;
    }
    return;
  }
  for_ids(p, run, [&](int i, uint64_t used) {
    const uint64_t hole = inside(i, run.lo, mid) & ~used, move = inside(i, mid, run.hi) & used;
    if (hole >> lane & 1) c.to[h + bits_before(hole)] = i + lane;
    if (move >> lane & 1) c.from[m + bits_before(move)] = i + lane;
    h += __popcll(hole);
    m += __popcll(move);
    return true;
  });
  __syncthreads();
  for (int r = tid; r < moved; r += kPlanThreads) {
    const int a = c.from[r], b = c.to[r];
    c.new_id[a] = b;
    p.refs[b] = p.refs[a];
    p.refs[a] = 0;
  }
  if (tid == 0) {
    *n_used = total;
    *c.moved = moved;
  }
}

__global__ __launch_bounds__(kCopyThreads) void compact_apply_kernel(dllm_kv_pages p, const int32_t* __restrict__ n_used,
                                                                     CompactPlan c, size_t page_bytes, int parts) {
  const int total = *n_used, moved = *c.moved;
  if (moved == 0) return;
  const size_t entries = size_t(p.max_seqs) * p.max_blocks, step = size_t(gridDim.x) * kCopyThreads;
  for (size_t i = size_t(blockIdx.x) * kCopyThreads + threadIdx.x; i < entries; i += step) {
    const int page = p.table[i];
    if (page >= total && page < p.n_pages) p.table[i] = c.new_id[page];
  }
  const int units = p.n_layers * 2 * parts;
  for (int64_t t = blockIdx.x; t < int64_t(moved) * units; t += gridDim.x) {
    const int r = int(t / units);
    copy_unit(p, page_bytes, parts, int(t % units), c.from[r], c.to[r]);
  }
}

// ---------------------------------------------------------------- rows

constexpr int kWriteThreads = 256;
constexpr int kWriteTile = 64;   // positions per workgroup, from a multiple of 64: pages are cut there too

// values as the pages of bf16 models hold them: rounded to binary16, past its
// range the largest of their sign (what saturating first gives), a NaN as it is
// (the median that saturates elsewhere returns the lowest of the others for one)
__device__ __forceinline__ uint32_t pack_values(float a, float b) {
  typedef _Float16 half2v __attribute__((ext_vector_type(2)));
  const half2v most = {65504, 65504}, v = __builtin_bit_cast(half2v, pack_f16x2(a, b));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_maximum(__builtin_elementwise_minimum(v, most), -most));
}
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(bf16_t* p, float v) { p->bits = uint16_t(pack_values(v, 0.f)); }

__device__ __forceinline__ int row_count(const int32_t* n_rows, int b, int max_rows) {
  return n_rows ? min(max(n_rows[b], 0), max_rows) : max_rows;
}

// Tile t of entry b and one head: keys go row by row as they are; values pass
// through LDS so that each dim's positions are stored together, 8 positions
// (16 bytes) at a time where the rows fill them.  A tile's page ids are looked
// up once, by the first lanes.  With kT the values come transposed ([dim][row],
// v.row elements a dim) in the type of the pages and are only shifted into place.
// Bound by memory: 16 x 512 rows of 32 heads of 128, 268 MB read and written, in
// 55 us, 64 x 512 in 257 (4.2 TB/s).  A sequence's rows take one tile more than
// they fill if they start inside one.  Workgroups go to the 8 XCDs in turn: with
// the tiles of a head first, the second of two would leave every other XCD idle,
// so there the heads come first (64 x 32 rows 26 us -> 21, 64 x 64 equal); with
// more tiles that costs 3 % (64 x 512 rows 266 us).
template <typename T, typename TV, int HD, bool kT>
__global__ __launch_bounds__(kWriteThreads) void pages_write_kernel(dllm_kv_pages p, int layer,
                                                                    const int32_t* __restrict__ seqs, int n,
                                                                    int max_rows, const int32_t* __restrict__ n_rows,
                                                                    dllm_rows k, dllm_rows v, bool heads_first) {
  constexpr int E = 16 / int(sizeof(T));          // elements per 16 bytes
  constexpr int CR = HD / E;                      // chunks per row
  constexpr int PITCH = HD + 4 / int(sizeof(T));  // LDS row of one position: an odd number of words
  __shared__ T sv[kT ? 1 : kWriteTile * PITCH];
  __shared__ int page_of[kWriteTile / 16];
  const int tid = threadIdx.x, b = blockIdx.z, h = heads_first ? blockIdx.x : blockIdx.y;
  const int tile = heads_first ? blockIdx.y : blockIdx.x;
  const int s = seqs[b];
  if (s < 0 || s >= p.max_seqs) return;
  int later = 0;
  for (int i = b + 1 + tid; i < n; i += kWriteThreads) later |= seqs[i] == s;
  const int held = min(max(p.len[s], 0), p.max_blocks * p.page_len);
  const int first = held - row_count(n_rows, b, max_rows);   // position of row 0 (can be negative)
  const int lo = max(first, 0), t0 = lo / kWriteTile * kWriteTile + tile * kWriteTile;
  const int from = max(lo, t0), to = min(held, t0 + kWriteTile);
  if (__syncthreads_or(later) || from >= to) return;
  if (tid < kWriteTile / 16) {
    const int pos = t0 + tid * 16;
    int page = -1;
    if (pos + 16 > from && pos < to) {
      page = p.table[size_t(s) * p.max_blocks + pos / p.page_len];
      if (page >= p.n_pages || (page >= 0 && p.refs[page] > 1)) page = -1;
    }
    page_of[tid] = page;
  }
  __syncthreads();
  const size_t head = (size_t(layer) * p.n_pages) * p.n_kv_heads + h;   // + page * n_kv_heads
  const int count = to - from;
  const T* ks = static_cast<const T*>(k.p) + int64_t(b) * k.seq + int64_t(h) * k.head + int64_t(from - first) * k.row;
  const T* vs = static_cast<const T*>(v.p) + int64_t(b) * v.seq + int64_t(h) * v.head +
                int64_t(from - first) * (kT ? 1 : v.row);
  for (int c = tid; c < count * CR; c += kWriteThreads) {
    const int r = c / CR, e = c % CR * E, at = from - t0 + r;
    const u32x4 kv = *reinterpret_cast<const u32x4*>(ks + int64_t(r) * k.row + e);
    u32x4 vv;
    if constexpr (!kT) vv = *reinterpret_cast<const u32x4*>(vs + int64_t(r) * v.row + e);
    const int page = page_of[at >> 4];
    if (page >= 0) {
      T* dst = static_cast<T*>(p.k) + (head + size_t(page) * p.n_kv_heads) * p.page_len * HD;
      *reinterpret_cast<u32x4*>(dst + ((t0 + at) & (p.page_len - 1)) * HD + e) = kv;
    }
    if constexpr (!kT) {
      uint32_t* row = reinterpret_cast<uint32_t*>(sv + at * PITCH + e);
#pragma unroll
      for (int w = 0; w < 4; ++w) row[w] = vv[w];
    }
  }
  __syncthreads();
  // 8 consecutive positions of one dim; 8 lanes side by side hold the tile's 64
  const int c0 = (from - t0) >> 3, c1 = (to - t0 + 7) >> 3, nc = c1 - c0;
  for (int w = tid; w < nc * HD; w += kWriteThreads) {
    const int d = w / nc, at = (c0 + w % nc) * 8, page = page_of[at >> 4];
    if (page < 0) continue;
    TV* dst = static_cast<TV*>(p.vt) + ((head + size_t(page) * p.n_kv_heads) * HD + d) * p.page_len +
              ((t0 + at) & (p.page_len - 1));
    const bool full = at >= from - t0 && at + 8 <= to - t0;
    auto row_of = [&](int i) { return min(max(at + i, from - t0), to - t0 - 1); };
    if constexpr (kT) {
      TV x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = vs[int64_t(d) * v.row + row_of(i) - (from - t0)];
      if (full) {
        constexpr int W = int(sizeof(TV)) * 8 / 16;
        u32x4 y[W];
        __builtin_memcpy(y, x, sizeof x);
#pragma unroll
        for (int i = 0; i < W; ++i) reinterpret_cast<u32x4*>(dst)[i] = y[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (at + i >= from - t0 && at + i < to - t0) dst[i] = x[i];
      }
    } else {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = load_f(sv + row_of(i) * PITCH + d);
      if (full) {
        if constexpr (sizeof(TV) == 2) {
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
}

__global__ __launch_bounds__(256) void rope_rows_kernel(dllm_kv_pages p, const int32_t* __restrict__ seqs, int n,
                                                        int rows, int max_pos, const float2* __restrict__ rope,
                                                        int half, float2* __restrict__ out) {
  const int t = blockIdx.x * 256 + threadIdx.x, row = t / half, c = t % half;
  if (row >= n * rows) return;
  const int s = seqs[row / rows];
  const int held = s >= 0 && s < p.max_seqs ? p.len[s] : 0;
  out[t] = rope[size_t(min(max(held - rows + row % rows, 0), max_pos - 1)) * half + c];
}

size_t page_bytes_of(const dllm_kv_pages& p) {
  return size_t(p.n_kv_heads) * p.page_len * p.head_dim * (p.dtype == DLLM_BF16 ? 2 : 4);
}

constexpr int kCopyWgs = 2048;        // 8 workgroups of a copy on every CU
constexpr int kDropHere = 32 * 1024;  // table entries one workgroup clears by itself

}  // namespace

hipError_t pages_init(const dllm_kv_pages& p, hipStream_t s) {
  hipLaunchKernelGGL(pages_init_kernel, dim3(256), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t pages_grow(const dllm_kv_pages& p, const int32_t* seqs, const int32_t* add, int n, int32_t* status,
                      hipStream_t s) {
  hipLaunchKernelGGL(pages_grow_kernel, dim3(1), dim3(kPlanThreads), 0, s, p, seqs, add, n, status);
  return hipGetLastError();
}

hipError_t pages_fork(const dllm_kv_pages& p, const int32_t* src, const int32_t* dst, const int32_t* keep, int n,
                      int32_t* status, hipStream_t s) {
  hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(kPlanThreads), 0, s, p, src, dst, keep, n, status);
  const size_t bytes = page_bytes_of(p);
  const int parts = int((bytes + kCopyUnit - 1) / kCopyUnit);
  const int row_wgs = std::min(cdiv(p.max_blocks, kCopyThreads), 8);
  const int copy_wgs = int(std::min<int64_t>(int64_t(n) * p.n_layers * 2 * parts, kCopyWgs));
  hipLaunchKernelGGL(fork_apply_kernel, dim3(n * row_wgs + copy_wgs), dim3(kCopyThreads), 0, s, p, src, dst, n,
                     row_wgs, bytes, parts, status);
  return hipGetLastError();
}

hipError_t pages_free(const dllm_kv_pages& p, const int32_t* seqs, const int32_t* keep, int n, int32_t* status,
                      hipStream_t s) {
  const bool here = int64_t(n) * p.max_blocks <= kDropHere;
  hipLaunchKernelGGL(pages_free_kernel, dim3(1), dim3(kPlanThreads), 0, s, p, seqs, keep, n, status, here);
  if (!here)
    hipLaunchKernelGGL(free_apply_kernel, dim3(std::min(cdiv(p.max_blocks, 256), 64), n), dim3(256), 0, s, p, seqs,
                       status);
  return hipGetLastError();
}

size_t pages_compact_workspace(int n_pages) { return (16 + 3 * size_t(n_pages)) * sizeof(int32_t); }

hipError_t pages_compact(const dllm_kv_pages& p, int32_t* n_used, void* ws, hipStream_t s) {
  const CompactPlan c = compact_plan(ws, p.n_pages);
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kPlanThreads), 0, s, p, n_used, c);
  const size_t bytes = page_bytes_of(p);
  const int parts = int((bytes + kCopyUnit - 1) / kCopyUnit);
  const int64_t most = std::max<int64_t>(int64_t(p.n_pages / 2) * p.n_layers * 2 * parts,
                                         (int64_t(p.max_seqs) * p.max_blocks + kCopyThreads - 1) / kCopyThreads);
  hipLaunchKernelGGL(compact_apply_kernel, dim3(int(std::min<int64_t>(std::max<int64_t>(most, 1), kCopyWgs))),
                     dim3(kCopyThreads), 0, s, p, n_used, c, bytes, parts);
  return hipGetLastError();
}

namespace {

template <bool kT>
hipError_t launch_write(const dllm_kv_pages& p, int layer, const int32_t* seqs, int n, int max_rows,
                        const int32_t* n_rows, const dllm_rows& k, const dllm_rows& v, hipStream_t s) {
  const int tiles = (max_rows + kWriteTile - 2) / kWriteTile + 1, heads = p.n_kv_heads;
  const bool heads_first = tiles == 2;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, heads_first ? dim3(heads, tiles, n) : dim3(tiles, heads, n), dim3(kWriteThreads), 0, s, p,
                       layer, seqs, n, max_rows, n_rows, k, v, heads_first);
    return hipGetLastError();
  };
  if (p.dtype == DLLM_BF16)
    return p.head_dim == 128 ? launch(pages_write_kernel<bf16_t, bf16_t, 128, kT>)
                             : launch(pages_write_kernel<bf16_t, bf16_t, 64, kT>);
  return p.head_dim == 128 ? launch(pages_write_kernel<float, float, 128, kT>)
                           : launch(pages_write_kernel<float, float, 64, kT>);
}

}  // namespace

hipError_t pages_write(const dllm_kv_pages& p, int layer, const int32_t* seqs, int n, int max_rows,
                       const int32_t* n_rows, const dllm_rows& k, const dllm_rows& v, hipStream_t s) {
  return launch_write<false>(p, layer, seqs, n, max_rows, n_rows, k, v, s);
}

hipError_t pages_write_vt(const dllm_kv_pages& p, int layer, const int32_t* seqs, int n, int rows, const dllm_rows& k,
                          const void* vt, int vt_ld, hipStream_t s) {
  const dllm_rows v{const_cast<void*>(vt), rows, vt_ld, int64_t(p.head_dim) * vt_ld};
  return launch_write<true>(p, layer, seqs, n, rows, nullptr, k, v, s);
}

hipError_t pages_rope_rows(const dllm_kv_pages& p, const int32_t* seqs, int n, int rows, int max_pos,
                           const float2* rope, int half, float2* out, hipStream_t s) {
  const int wgs = int((int64_t(n) * rows * half + 255) / 256);
  hipLaunchKernelGGL(rope_rows_kernel, dim3(wgs), dim3(256), 0, s, p, seqs, n, rows, max_pos, rope, half, out);
  return hipGetLastError();
}

}  // namespace dllm
