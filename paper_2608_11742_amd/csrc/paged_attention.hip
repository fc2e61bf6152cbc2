// Attention over the pages of one layer: softmax(scale q k^T) v for the rows
// of a batch of sequences.
//
// softmax over a set of keys is carried as (m, l, o): an exponent reference,
// the sum of 2^(x - m) and the unnormalised output; two disjoint sets join as
// m = max(m1, m2), l = l1 2^(m1 - m) + l2 2^(m2 - m), o alike.  So the keys of
// a row may be divided freely:
//   prefix   the positions that the whole batch shares.  The rows of all
//            entries (and of the query heads of one key head) are stacked, so
//            that a key tile is read once for all of them.
//   tail     each entry's own positions after them, for its own rows.  The
//            tail of an entry that ends inside the prefix starts with the key
//            range that it ends in: a weight of 0 would not cancel values past
//            its end that are infinite or no number, and a tail's are cut there.
// and each of the two over workgroups by ranges of keys, where there are few
// rows.  Every range leaves a record per row, and a merge joins them in order;
// with one range in all the workgroup writes the output itself.  Where the
// entries are few, short or fill their workgroups, reading the prefix again for
// each of them costs less than a join: then every entry's range starts at
// position 0 and takes its pages from the prefix's table first.
//
// Three kernels, by the number of stacked rows (MI355X; floors by the rates of
// a large copy, 4.9 TB/s, and a large bf16 product, 1190 TFLOP/s):
//   narrow   up to 32 rows: bound by the keys and values it streams.  The
//            waves share the rows and take the key steps in turn; a step's
//            fragments come straight from memory into registers, K of the
//            next step while the softmax runs, V after it (no LDS, no
//            barrier), and the waves' states are joined through LDS at the
//            end.  Single tokens of 4 sequences up to 120000 long, 8 key heads
//            of 128: 217 us, 5.7 TB/s.
//   wide     128 rows, 32 a wave (bf16).  Tiles of 64 keys go through a
//            two-slot LDS ring, copied one tile ahead, on 32 x 32 MFMAs.  16 x
//            32 rows of 32 heads over 30011 positions: 318 us, 0.80 PFLOP/s,
//            floor 213.  Matrix units are busy 43% of it and vector ALUs 37%:
//            products and softmax alone take 177 us, fragment reads from LDS
//            add 50, the copies 85 and the join of the ranges 15.
//   pairs    two entries' 32 rows each (bf16): prefix and own tails in one
//            launch that writes the output.  16 x 32 rows over 1024: 21 us, of
//            which 7 are spent before and after the keys, 1.4 on every 128
//            positions and 2.5 on the tail; floor 7.4.
// Scores are computed transposed (S^T = K Q^T): a lane then holds one row's
// scores, and with the key order below its probabilities are, as they lie in
// its registers, the operand of o^T += V^T P^T.  The exponent reference is set
// to 8 (log2 units) under a row's largest score and stands until a weight may
// pass 2^15, so o is rescaled rarely.  Weights of bf16 models are rounded to
// binary16 for the product with binary16 values: 11 significant bits down to
// 2^-22 of the row's largest, and off by 2^-33 of it at most below, so that a
// million keys that weigh 2^-25 each are not lost beside one that weighs 1.  The
// sums l and products o are held in 32 bits; wide and pairs sum the weights as
// rounded, narrow before.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "mainloop.h"

namespace dllm {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 64;       // keys of a wide tile; ranges are whole tiles
constexpr int kNarrowRows = 32;
constexpr float kFirst = 8.f, kMost = 15.f;   // log2 of a row's largest weight when its reference moves, and ever
// floats per record: HD output values, m, l, padding to 16 bytes
constexpr int record(int hd) { return hd + 4; }

// How a part's keys and rows are divided: row tiles, key ranges and keys per range
struct Part {
  int row_tiles, ranges, range;
};

// what a call's kernels share
struct Job {
  PagedAttn a;
  float scale_log2;   // scale * log2(e)
  int group;          // query heads per key head
  Part prefix, tail;
  bool stacked;       // the prefix is a part of its own; else each tail starts at position 0
  bool direct;        // one range in all: the output itself
};

__device__ __forceinline__ int most_positions(const PagedAttn& a) { return a.p.max_blocks * a.p.page_len; }

// whole pages of the prefix (0: none)
__device__ __forceinline__ int shared_of(const PagedAttn& a) {
  if (a.shared_len <= 0) return 0;
  const int held = min(max(a.p.len[a.prefix_seq], 0), most_positions(a));
  return min(a.shared_len, held) & ~(a.p.page_len - 1);
}

struct Entry {
  int seq, held, rows;   // sequence (-1: none), its positions, rows of the entry
};
__device__ __forceinline__ Entry entry_of(const PagedAttn& a, int b) {
  Entry e;
  const int s = a.seqs[b];
  e.seq = s >= 0 && s < a.p.max_seqs ? s : -1;
  e.held = e.seq >= 0 ? min(max(a.p.len[e.seq], 0), most_positions(a)) : 0;
  e.rows = a.n_rows ? min(max(a.n_rows[b], 0), a.max_rows) : a.max_rows;
  return e;
}
// of the `shared` positions, those that the entry takes with the others', which are in steps of `range`
__device__ __forceinline__ int stacked_of(const Entry& e, int shared, int range) {
  return e.held >= shared ? shared : e.held / range * range;
}
// positions that row i of the entry sees
__device__ __forceinline__ int limit_of(const PagedAttn& a, const Entry& e, int i) {
  return a.causal ? max(0, min(e.held, e.held - e.rows + i + 1)) : e.held;
}

// a table's row, read on the scalar unit: uniform, and not written here
typedef const __attribute__((address_space(4))) int32_t* table_t;
__device__ __forceinline__ table_t table_row(const PagedAttn& a, int seq) {
  return (table_t)(a.p.table + size_t(seq) * a.p.max_blocks);
}

// A workgroup's share: rows row0 .. (stacked as ((entry * max_rows) + row) *
// group + query head) of key head `head`, keys k0 .. k1 - 1, record index.
// Pages of positions before `split` are `before`'s, then `after`'s.
struct Share {
  int row0, row_end, head, k0, k1, part, split;
  table_t before, after;
  __device__ __forceinline__ int page(int pos, int shift, int last_block) const {
    return (pos < split ? before : after)[min(pos >> shift, last_block)];
  }
};

// Workgroup x of a part: its item (a key range of one head) and row tile.
// Workgroups go to the 8 XCDs in turn; the row tiles of an item, which read the
// same keys, take the same XCD one after the other, so that one L2 fetches them
// once (16 x 32 rows over 30011 positions, 4 row tiles: a tile's copies came
// from HBM up to 4 times before).
struct Item {
  int item, tile;
};
__device__ __forceinline__ Item item_of(int x, int row_tiles) {
  return Item{x / (8 * row_tiles) * 8 + x % 8, x / 8 % row_tiles};
}
int blocks_of(int items, int row_tiles) { return cdiv(items, 8) * 8 * row_tiles; }

// False if the share is empty.
__device__ __forceinline__ bool share_of(const Job& j, int x, bool in_prefix, int tile_rows, Share& w) {
  const PagedAttn& a = j.a;
  const int per = a.max_rows * j.group;   // stacked rows of one entry
  const Part& part = in_prefix ? j.prefix : j.tail;
  const Item it = item_of(x, part.row_tiles);
  w.head = it.item % a.p.n_kv_heads;
  const int t = it.item / a.p.n_kv_heads, r = t % part.ranges, b = t / part.ranges;
  if (b >= (in_prefix ? 1 : a.n)) return false;   // items are filled up to whole rounds of XCDs
  const int s = shared_of(a);
  if (in_prefix) {
    w.row0 = it.tile * tile_rows;
    w.row_end = a.n * per;
    w.k0 = r * part.range;
    w.k1 = min(w.k0 + part.range, s);
    w.part = r;
    w.split = 0;
    w.before = w.after = table_row(a, a.prefix_seq);
    return w.k0 < w.k1;
  }
  const Entry e = entry_of(a, b);
  w.row0 = b * per + it.tile * tile_rows;
  w.row_end = (b + 1) * per;
  w.k0 = (j.stacked ? stacked_of(e, s, j.prefix.range) : 0) + r * part.range;
  w.k1 = r + 1 == part.ranges ? e.held : min(w.k0 + part.range, e.held);
  w.part = j.prefix.ranges + r;
  w.split = s;
  w.before = table_row(a, a.prefix_seq);
  w.after = table_row(a, __builtin_amdgcn_readfirstlane(max(e.seq, 0)));
  // an entry without positions still has its rows set to 0 where nothing is joined
  return w.row0 < b * per + e.rows * j.group && (w.k0 < w.k1 || j.direct);
}

// a stacked row's place
struct RowAt {
  int b, i, g;
};
__device__ __forceinline__ RowAt row_at(const Job& j, int row) {
  RowAt r;
  r.g = row % j.group;
  const int t = row / j.group;
  r.b = t / j.a.max_rows;
  r.i = t % j.a.max_rows;
  return r;
}

__device__ __forceinline__ float* record_of(const Job& j, int part, const RowAt& r, int kvh, int hd) {
  const size_t row = (size_t(r.b) * j.a.max_rows + r.i) * j.a.heads + kvh * j.group + r.g;
  return j.a.part + (size_t(part) * j.a.n * j.a.max_rows * j.a.heads + row) * record(hd);
}

// lane l's value of lanes l, l ^ 32 joined
__device__ __forceinline__ float pair_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
// of lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_max(float x) {
  const float m = pair_max(x);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  const float m = pair_sum(x);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ---------------------------------------------------------------- narrow

// NQB blocks of 16 rows.  A key step is KS keys in blocks of 16; bf16 keys of
// a 32-key half are gathered so that output element i of lane group g in
// block kk is key 8 g + 4 kk + i: the lane's 8 probabilities of the half are 8
// consecutive keys, one 16-byte chunk of a V^T row.
template <typename T, int HD, int NQB>
struct Narrow {
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr int E = 16 / int(sizeof(T));             // elements per chunk
  static constexpr int CK = HD / E;                         // chunks per key row
  // a step's K takes 64 registers at most, its V as many; half of that beside the state of two row blocks
  // (and with fp32, whose steps the products bound: shorter ones come out more even)
  static constexpr int kRegs = NQB == 1 && kHalf ? 16 : 8;
  static constexpr int KS = kRegs * 1024 / (HD * int(sizeof(T))) < 64 ? kRegs * 1024 / (HD * int(sizeof(T))) : 64;
  static constexpr int NB = KS / 16;                        // 16-key blocks of a step
  static constexpr int QS = CK / 4;                         // MFMA steps over head_dim
  static constexpr int NDB = HD / 16;
  static constexpr int NV = KS / (4 * E);                   // V chunks per dim row and lane
  static constexpr int STATE = NDB * 4 + 2;                 // floats a lane hands over per 16 rows
  static constexpr int SMEM = kWaves * STATE * kWave * 4;

  __device__ __forceinline__ static int key_of(int kb, int r) {
    if constexpr (kHalf) return 32 * (kb >> 1) + 8 * (r >> 2) + 4 * (kb & 1) + (r & 3);
    else return 16 * kb + r;
  }

  __device__ static void run(const Job& j, const Share& w, uint8_t* lds) {
    float* smem = reinterpret_cast<float*>(lds);
    const PagedAttn& a = j.a;
    const int kvh = w.head;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int fr = lane & 15, g = lane >> 4;
    const int shift = 31 - __builtin_clz(a.p.page_len), pmask = a.p.page_len - 1;
    const size_t head_stride = size_t(a.p.page_len) * HD;
    const size_t page_stride = head_stride * a.p.n_kv_heads;
    const size_t base = (size_t(a.layer) * a.p.n_pages * a.p.n_kv_heads + kvh) * head_stride;
    const T* K = static_cast<const T*>(a.p.k) + base;
    const T* V = static_cast<const T*>(a.p.vt) + base;
    const int last_block = max(w.k1 - 1, 0) >> shift;

    RowAt at[NQB];
    u32x4 qf[NQB][QS];
    int lim[NQB], rows[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      at[qb] = row_at(j, min(w.row0 + 16 * qb + fr, w.row_end - 1));
      const Entry e = entry_of(a, at[qb].b);
      lim[qb] = min(limit_of(a, e, at[qb].i), w.k1);
      rows[qb] = e.rows;
    }

    // table entries of a step's 16-key groups (past the last key: its page
    // again), brought into the pool where they are used: loads do not wait here
    auto pages_at = [&](int k0, int (&id)[NB]) {
#pragma unroll
      for (int i = 0; i < NB; ++i) id[i] = w.page(k0 + 16 * i, shift, last_block);
    };
    auto in_pool = [&](int p) { return min(max(p, 0), a.p.n_pages - 1); };
    u32x4 kf[NB][QS], vf[NDB][NV];
    auto load_k = [&](int k0, const int (&id)[NB]) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const int key = key_of(kb, fr);
        const int page = in_pool(kHalf ? (fr < 8 ? id[kb & ~1] : id[kb | 1]) : id[kb]);
        const T* row = K + page * page_stride + ((k0 + key) & pmask) * HD;
#pragma unroll
        for (int st = 0; st < QS; ++st) kf[kb][st] = *reinterpret_cast<const u32x4*>(row + (4 * st + g) * E);
      }
    };
    auto load_v = [&](int k0, const int (&id)[NB]) {
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        const int key = (4 * c + g) * E;   // first of this lane's chunk
        const int page = in_pool(kHalf ? (g < 2 ? id[2 * c] : id[2 * c + 1]) : id[c]);
        const T* row = V + page * page_stride + size_t(fr) * a.p.page_len + ((k0 + key) & pmask);
#pragma unroll
        for (int db = 0; db < NDB; ++db)
          vf[db][c] = *reinterpret_cast<const u32x4*>(row + 16 * db * a.p.page_len);
      }
    };

    f32x4 o[NDB][NQB];
    float m[NQB], l[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      m[qb] = -INFINITY;
      l[qb] = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int k0 = w.k0 + wave * KS;
    int id[NB];
    if (k0 < w.k1) {
      pages_at(k0, id);
      load_k(k0, id);
    }
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      const T* q = static_cast<const T*>(a.q.p) + at[qb].b * a.q.seq + at[qb].i * a.q.row +
                   (kvh * j.group + at[qb].g) * a.q.head;
#pragma unroll
      for (int st = 0; st < QS; ++st) qf[qb][st] = *reinterpret_cast<const u32x4*>(q + (4 * st + g) * E);
    }
    if (k0 < w.k1) load_v(k0, id);
    for (; k0 < w.k1; k0 += kWaves * KS) {
      const int next = k0 + kWaves * KS;
      const bool more = next < w.k1;
      if (more) pages_at(next, id);
      f32x4 sc[NB][NQB];
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          sc[kb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int st = 0; st < QS; ++st) Mfma<T>::run(sc[kb][qb], kf[kb][st], qf[qb][st]);
        }
      if (more) load_k(next, id);
      bool all = true;
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) all = all && k0 + KS <= lim[qb];
      if (!__all(all)) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (k0 + key_of(kb, 4 * g + i) >= lim[qb]) sc[kb][qb][i] = -INFINITY;
      }
      bool moved = false;
      float alpha[NQB];
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[kb][qb][i]);
        top = quad_max(top) * j.scale_log2;
        const float mn = top > m[qb] + kMost ? top - kFirst : m[qb];
        const float ref = mn == -INFINITY ? 0.f : mn;   // a row that has seen no key yet: exponents 2^-inf
        alpha[qb] = __builtin_amdgcn_exp2f(m[qb] - ref);
        moved = moved || mn != m[qb];
        m[qb] = mn;
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sc[kb][qb][i] = __builtin_amdgcn_exp2f(fmaf(sc[kb][qb][i], j.scale_log2, -ref));
            sum += sc[kb][qb][i];
          }
        l[qb] = l[qb] * alpha[qb] + sum;
      }
      if (__any(moved)) {
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
          for (int db = 0; db < NDB; ++db) o[db][qb] *= alpha[qb];
      }
      if (k0 + KS > w.k1) {   // values past the last key: whatever they are, times 0
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          const int left = w.k1 - (k0 + (4 * c + g) * E);   // valid elements of this lane's chunks
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t keep = kHalf ? (left > 2 * x + 1 ? ~0u : left > 2 * x ? 0xffffu : 0u) : (left > x ? ~0u : 0u);
#pragma unroll
            for (int db = 0; db < NDB; ++db) vf[db][c][x] &= keep;
          }
        }
      }
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          u32x4 pf;
          if constexpr (kHalf) {
            pf = u32x4{pack_f16x2(sc[2 * c][qb][0], sc[2 * c][qb][1]), pack_f16x2(sc[2 * c][qb][2], sc[2 * c][qb][3]),
                       pack_f16x2(sc[2 * c + 1][qb][0], sc[2 * c + 1][qb][1]),
                       pack_f16x2(sc[2 * c + 1][qb][2], sc[2 * c + 1][qb][3])};
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[i] = __float_as_uint(sc[c][qb][i]);
          }
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            if constexpr (kHalf) MfmaF16::run(o[db][qb], vf[db][c], pf);
            else Mfma<float>::run(o[db][qb], vf[db][c], pf);
          }
        }
      if (more) load_v(next, id);
    }

    // join the waves' states, 16 rows at a time: wave w sums dim blocks w, w + 4, ..
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      float* mine = smem + wave * STATE * kWave + lane;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[(4 * db + i) * kWave] = o[db][qb][i];
      mine[(STATE - 2) * kWave] = m[qb];
      mine[(STATE - 1) * kWave] = quad_sum(l[qb]);
      __syncthreads();
      float mw[kWaves], top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        mw[v] = smem[(v * STATE + STATE - 2) * kWave + lane];
        top = fmaxf(top, mw[v]);
      }
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        mw[v] = __builtin_amdgcn_exp2f(mw[v] - ref);
        sum += smem[(v * STATE + STATE - 1) * kWave + lane] * mw[v];
      }
      const int row = w.row0 + 16 * qb + fr;
      const bool live = row < w.row_end && at[qb].i < rows[qb];
      const float inv = lim[qb] > 0 ? 1.f / sum : 0.f;
      T* out = static_cast<T*>(a.out.p) + at[qb].b * a.out.seq + at[qb].i * a.out.row +
               (kvh * j.group + at[qb].g) * a.out.head;
      float* rec = record_of(j, w.part, at[qb], kvh, HD);
      for (int db = wave; db < NDB; db += kWaves) {
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] += smem[(v * STATE + 4 * db + i) * kWave + lane] * mw[v];
        if (!live) continue;
        if (j.direct) {
#pragma unroll
          for (int i = 0; i < 4; ++i) store_f(out + 16 * db + 4 * g + i, lim[qb] > 0 ? x[i] * inv : 0.f);
        } else {
          *reinterpret_cast<f32x4*>(rec + 16 * db + 4 * g) = x;
        }
      }
      if (live && !j.direct && wave == 0 && g == 0) {
        rec[HD] = top;
        rec[HD + 1] = sum;
      }
      if (qb + 1 < NQB) __syncthreads();
    }
  }
};

// ---------------------------------------------------------------- wide

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

// 16 bytes per lane from global memory straight into LDS (lane l: lds + 16 l)
__device__ __forceinline__ void copy16(const void* src, uint32_t lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src),
                                   reinterpret_cast<__attribute__((address_space(3))) void*>(static_cast<uintptr_t>(lds)),
                                   16, 0, 0);
}

// Tiles of 64 bf16 keys in LDS, for 32 x 32 MFMAs.  MFMA row r of a 32-key half
// is key r with bits 2 and 3 exchanged: output registers 8 s .. 8 s + 7 of lane
// half f are then keys 16 s + 8 f .. + 7, the chunk of V^T that this lane half
// multiplies in step s.
template <int HD>
struct Tile {
  static constexpr int RB = HD * 2;                 // bytes of a key row
  static constexpr int CK = RB / 16;                // chunks of a key row
  static constexpr int KB = kTile * RB;             // K tile; V^T tile: HD rows of 128 bytes
  static constexpr int BYTES = 2 * KB;
  static constexpr int KROWS = kWave / CK;          // key rows of one 1 KB copy
  static constexpr int QS = HD / 16;                // MFMA steps over head_dim
  static constexpr int NDB = HD / 32;

  // chunk c of row r lies in slot c ^ swizzle(r): the 16 rows that 16 lanes
  // read together fall on different banks (64 of 4 bytes: a 256-byte row, or
  // two rows of 128)
  __device__ __forceinline__ static int kswz(int r) { return CK == 16 ? r & 15 : (r >> 1) & 7; }
  __device__ __forceinline__ static int vswz(int d) { return (d >> 1) & 7; }
  // key within its 32 of MFMA row r
  __device__ __forceinline__ static int key_of(int r) { return (r & 0x13) | ((r & 4) << 1) | ((r & 8) >> 1); }

  // one wave's part (`wave` of four) of copying a tile
  struct Copier {
    static constexpr int IC = KB / 1024 / kWaves;   // copies the wave issues for K, and for V
    const uint8_t* K;
    const uint8_t* V;
    size_t page_bytes;
    int wave, lane, page_len, n_pages, shift, last_block;

    __device__ __forceinline__ Copier(const PagedAttn& a, int head, int wave_, int end) : wave(wave_) {
      lane = threadIdx.x & 63;
      page_len = a.p.page_len;
      n_pages = a.p.n_pages;
      shift = 31 - __builtin_clz(page_len);
      last_block = max(end - 1, 0) >> shift;
      const size_t head_bytes = size_t(page_len) * RB;
      page_bytes = head_bytes * a.p.n_kv_heads;
      const size_t base = (size_t(a.layer) * n_pages * a.p.n_kv_heads + head) * head_bytes;
      K = static_cast<const uint8_t*>(a.p.k) + base;
      V = static_cast<const uint8_t*>(a.p.vt) + base;
    }
    __device__ __forceinline__ int in_pool(int p) const { return min(max(p, 0), n_pages - 1); }
    // table entries of the tile's 16-key groups (past the last key: its page
    // again), brought into the pool where they are used: loads do not wait here
    __device__ __forceinline__ void pages_at(const Share& w, int k0, int (&id)[4]) const {
#pragma unroll
      for (int i = 0; i < 4; ++i) id[i] = w.page(k0 + 16 * i, shift, last_block);
    }
    __device__ __forceinline__ void issue(int k0, const int (&id)[4], uint32_t dst) const {
      const int pmask = page_len - 1, kr = lane / CK, vd = lane >> 3, vc = (lane & 7) ^ vswz(8 * wave + vd);
#pragma unroll
      for (int i = 0; i < IC; ++i) {
        const int grp = i * kWaves + wave, r = grp * KROWS + kr;
        // a copy's rows share a 16-key group, one of C over the waves
        constexpr int C = kWaves * KROWS / 16;
        const int u = wave * KROWS / 16, sub = i * C + u;
        const int even = id[i * C], odd = id[i * C + C - 1];
        const int page = in_pool(u ? odd : even);
        const uint8_t* src = K + page * page_bytes + ((k0 + sub * 16) & pmask) * RB;
        copy16(src + (r & 15) * RB + ((lane % CK) ^ kswz(r)) * 16, dst + grp * 1024);
      }
      const int page = in_pool(vc < 4 ? (vc < 2 ? id[0] : id[1]) : (vc < 6 ? id[2] : id[3]));
      const uint8_t* src = V + page * page_bytes + size_t(vd) * (page_len * 2) + ((k0 + 8 * vc) & pmask) * 2;
#pragma unroll
      for (int i = 0; i < IC; ++i) {
        const int grp = i * kWaves + wave;
        copy16(src + size_t(grp) * 8 * (page_len * 2), dst + KB + grp * 1024);
      }
    }
  };

  // values of keys from `left` on (whatever they are) set to 0, by `threads` threads
  __device__ __forceinline__ static void zero_values(uint8_t* sv, int t, int threads, int left) {
    for (int c = t; c < HD * 8; c += threads) {
      const int d = c >> 3, n = left - 8 * (c & 7);
      if (n >= 8) continue;
      u32x4* p = reinterpret_cast<u32x4*>(sv + d * 128 + (((c & 7) ^ vswz(d)) << 4));
      u32x4 x = *p;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] &= n > 2 * i + 1 ? ~0u : n > 2 * i ? 0xffffu : 0u;
      *p = x;
    }
  }
  __device__ __forceinline__ static u32x4 key_chunk(const uint8_t* sk, int h, int st, int lane) {
    const int r = 32 * h + key_of(lane & 31);
    return *reinterpret_cast<const u32x4*>(sk + r * RB + (((2 * st + (lane >> 5)) ^ kswz(r)) << 4));
  }
  __device__ __forceinline__ static u32x4 value_chunk(const uint8_t* sv, int st, int db, int lane) {
    const int d = 32 * db + (lane & 31);
    return *reinterpret_cast<const u32x4*>(sv + d * 128 + (((2 * st + (lane >> 5)) ^ vswz(d)) << 4));
  }
};

// one wave's 32 rows: state of their softmax and a block of H x 32 keys into it
template <int HD>
struct Rows32 {
  using L = Tile<HD>;
  u32x4 qf[L::QS];
  f32x16 o[L::NDB];
  float m = -INFINITY, l = 0.f;   // reference (log2 units), this lane's part of the sum

  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int db = 0; db < L::NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  }
  __device__ __forceinline__ void load_q(const bf16_t* q) {
    const int f = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int st = 0; st < L::QS; ++st) qf[st] = *reinterpret_cast<const u32x4*>(q + (2 * st + f) * 8);
  }
  template <int H>
  __device__ __forceinline__ void scores(const u32x4 (&kf)[H][L::QS], f32x16 (&sc)[H]) const {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[h][i] = 0.f;
#pragma unroll
    for (int st = 0; st < L::QS; ++st)
#pragma unroll
      for (int h = 0; h < H; ++h)
        sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[h][st]),
                                                        __builtin_bit_cast(bf16x8, qf[st]), sc[h], 0, 0, 0);
  }
  // scores of keys k0 .. into probabilities (binary16 pairs); keys from lim on are not seen
  template <int H>
  __device__ __forceinline__ void softmax(f32x16 (&sc)[H], int k0, int lim, float scale_log2, u32x4 (&pf)[2 * H]) {
    const int f = (threadIdx.x >> 5) & 1;
    // element i of half h: key 32 h + 16 (i / 8) + 8 f + i % 8
    if (!__all(k0 + 32 * H <= lim)) {
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (k0 + 32 * h + 16 * (i >> 3) + 8 * f + (i & 7) >= lim) sc[h][i] = -INFINITY;
    }
    // With the reference as it is, unless a weight would pass what binary16 holds
    // (or there is none yet): no lane's 16 H weights sum up to more than 2^kMost.
    // Their maximum is only looked for where it may have to move: not if none
    // of them passes 2^kMost / 32.
    float sum = weights(sc, scale_log2, m, pf);
    if (!__all(sum <= float(1 << int(kMost)))) {
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[h][i]);
      top = pair_max(top) * scale_log2;
      const float mn = top > m + (kMost - 5.f) ? top - kFirst : m;
      const float ref = mn == -INFINITY ? 0.f : mn;   // no key seen yet: weights 2^-inf
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < L::NDB; ++db) o[db] *= alpha;
      m = mn;
      sum = weights(sc, scale_log2, ref, pf);
    }
    l += sum;
  }
  // 2^(score - ref) in binary16, and their sum as rounded
  template <int H>
  __device__ __forceinline__ static float weights(const f32x16 (&sc)[H], float scale_log2, float ref, u32x4 (&pf)[2 * H]) {
    typedef _Float16 half2v __attribute__((ext_vector_type(2)));
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const uint32_t xy = pack_f16x2(__builtin_amdgcn_exp2f(fmaf(sc[h][i], scale_log2, -ref)),
                                       __builtin_amdgcn_exp2f(fmaf(sc[h][i + 1], scale_log2, -ref)));
        sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, xy), half2v{1, 1}, sum, false);
        pf[2 * h + (i >> 3)][(i & 7) >> 1] = xy;
      }
    return sum;
  }
  __device__ __forceinline__ void add(int db, u32x4 vf, u32x4 pf) {
    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, vf), __builtin_bit_cast(half8, pf), o[db],
                                                   0, 0, 0);
  }
};

// 128 rows, 32 a wave, over one range of keys; two tiles in LDS, so that two
// workgroups share a CU.  Measured equal (16 x 32 rows, 32 heads, over 30011
// positions: 320 us, 0.79 PFLOP/s): eight waves and 256 rows with three tiles on
// their way, whose copies are half as many a row; the same in two groups that
// take turns at matrix and vector work.  64 rows a wave, alone on its SIMD with
// products and softmax in one stream, took 350.
template <int HD>
struct Wide {
  using L = Tile<HD>;
  using Copier = typename L::Copier;
  static constexpr int SMEM = 2 * L::BYTES;

  __device__ static void run(const Job& j, const Share& w, uint8_t* smem) {
    const PagedAttn& a = j.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, f = lane >> 5;
    const uint32_t lds0 = lds_address(smem);
    const Copier copier(a, w.head, wave, w.k1);

    const RowAt at = row_at(j, min(w.row0 + 32 * wave + fr, w.row_end - 1));
    Rows32<HD> rows;
    rows.load_q(static_cast<const bf16_t*>(a.q.p) + at.b * a.q.seq + at.i * a.q.row +
                (w.head * j.group + at.g) * a.q.head);
    rows.begin();
    const Entry entry = entry_of(a, at.b);
    const int lim_row = limit_of(a, entry, at.i), lim = min(lim_row, w.k1);

    int id[4];
    copier.pages_at(w, w.k0, id);
    if (w.k0 < w.k1) copier.issue(w.k0, id, lds0);
    copier.pages_at(w, w.k0 + kTile, id);
    int slot = 0;
    for (int k0 = w.k0; k0 < w.k1; k0 += kTile, slot ^= 1) {
      wait_vmcnt<0>();
      barrier_lds();   // tile k0 has landed; the other slot has been read
      const uint8_t* sk = smem + slot * L::BYTES;
      uint8_t* sv = smem + slot * L::BYTES + L::KB;
      if (k0 + kTile > w.k1) {
        L::zero_values(sv, tid, kThreads, w.k1 - k0);
        barrier_lds();
      } else if (k0 + kTile < w.k1) {
        copier.issue(k0 + kTile, id, lds0 + (slot ^ 1) * L::BYTES);
        copier.pages_at(w, k0 + 2 * kTile, id);
      }
      // every K fragment is on its way before the first product waits for one,
      // half of the V fragments before the softmax
      u32x4 kf[2][L::QS], vf[2][L::NDB], pf[4];
      f32x16 sc[2];
#pragma unroll
      for (int st = 0; st < L::QS; ++st)
#pragma unroll
        for (int h = 0; h < 2; ++h) kf[h][st] = L::key_chunk(sk, h, st, lane);
      __builtin_amdgcn_sched_barrier(0);
      rows.scores(kf, sc);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) vf[st][db] = L::value_chunk(sv, st, db, lane);
      __builtin_amdgcn_sched_barrier(0);
      rows.softmax(sc, k0, lim, j.scale_log2, pf);
#pragma unroll
      for (int st = 0; st < 4; ++st) {
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) rows.add(db, vf[st & 1][db], pf[st]);
        if (st < 2) {
#pragma unroll
          for (int db = 0; db < L::NDB; ++db) vf[st][db] = L::value_chunk(sv, st + 2, db, lane);
        }
      }
    }
    const float l = pair_sum(rows.l);
    if (w.row0 + 32 * wave + fr >= w.row_end || at.i >= entry.rows) return;
    // element i of block db: dim 32 db + 8 (i / 4) + 4 f + i % 4
    if (j.direct) {
      bf16_t* out = static_cast<bf16_t*>(a.out.p) + at.b * a.out.seq + at.i * a.out.row +
                    (w.head * j.group + at.g) * a.out.head;
      const float inv = 1.f / l;
#pragma unroll
      for (int db = 0; db < L::NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          store_f(out + 32 * db + 8 * (i >> 2) + 4 * f + (i & 3), lim_row > 0 ? rows.o[db][i] * inv : 0.f);
    } else {
      float* rec = record_of(j, w.part, at, w.head, HD);
#pragma unroll
      for (int db = 0; db < L::NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(rec + 32 * db + 2 * i + 4 * f) =
              f32x4{rows.o[db][i], rows.o[db][i + 1], rows.o[db][i + 2], rows.o[db][i + 3]};
      if (f == 0) {
        rec[HD] = rows.m;
        rec[HD + 1] = l;
      }
    }
  }
};

// ---------------------------------------------------------------- pairs

// Two blocks of 32 rows, each of one entry, over the shared prefix and then
// each over its own tail, in one workgroup of 8 waves that writes the output:
// wave w takes block w % 2 and every fourth 32 keys.  A pair of 64-key tiles of
// the prefix is in LDS at a time; waves 0 .. 3 copy and use the first, 4 .. 7 the
// second.  A tail's keys are few and used by one block alone: their fragments
// come straight from memory.  The four states of a block are joined through LDS.
template <int HD>
struct Pairs {
  using L = Tile<HD>;
  static constexpr int kWays = 4;
  static constexpr int kPairThreads = 2 * kWays * kWave;
  static constexpr int kKeys = kWays * 32;             // keys of a step
  static constexpr int RING = 4 * L::BYTES;            // two slots of two tiles
  static constexpr int STATE = 32 + 2;                 // floats a lane hands over at a time
  static constexpr int JOIN = 2 * kWays * STATE * kWave * 4;
  static constexpr int SMEM = RING > JOIN ? RING : JOIN;

  __device__ static void run(const Job& j, int x, uint8_t* smem) {
    const PagedAttn& a = j.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, f = lane >> 5, block = wave & 1, way = wave >> 1, tile = wave >> 2;
    const int per = a.max_rows * j.group, per_blocks = (per + 31) / 32, pairs = (a.n * per_blocks + 1) / 2;
    const Item it = item_of(x, pairs);
    if (it.item >= a.p.n_kv_heads) return;
    const int head = it.item;
    const int rb = min(2 * it.tile + block, a.n * per_blocks - 1);   // an odd last block is taken twice
    const bool own = 2 * it.tile + block < a.n * per_blocks;
    const int b = rb / per_blocks, r0 = rb % per_blocks * 32;

    const int s = shared_of(a);
    const Entry e = entry_of(a, b);
    Share prefix{}, tail{};
    prefix.before = prefix.after = table_row(a, a.prefix_seq);
    const int own_from = __builtin_amdgcn_readfirstlane(stacked_of(e, s, kKeys));
    tail.split = s;
    tail.before = prefix.before;
    tail.after = table_row(a, __builtin_amdgcn_readfirstlane(max(e.seq, 0)));
    const typename L::Copier copier(a, head, wave & 3, s), own_keys(a, head, 0, e.held);
    const int first = kTile * tile;   // of this wave's tile in a step
    const uint32_t lds0 = lds_address(smem) + tile * L::BYTES;
    int id[4];
    copier.pages_at(prefix, first, id);
    if (s > 0) copier.issue(first, id, lds0);
    copier.pages_at(prefix, first + kKeys, id);

    const int row = min(r0 + fr, per - 1), i = row / j.group, g = row % j.group;
    Rows32<HD> rows;
    rows.load_q(static_cast<const bf16_t*>(a.q.p) + b * a.q.seq + i * a.q.row + (head * j.group + g) * a.q.head);
    rows.begin();
    const int limit = limit_of(a, e, i), lim = min(limit, s);

    int slot = 0;
    for (int k0 = 0; k0 < s; k0 += kKeys, slot ^= 1) {
      wait_vmcnt<0>();
      __syncthreads();
      uint8_t* sk = smem + slot * (2 * L::BYTES) + tile * L::BYTES;
      uint8_t* sv = sk + L::KB;
      if (k0 + kKeys > s) {
        L::zero_values(sv, tid & (kThreads - 1), kThreads, s - k0 - first);
        __syncthreads();
      } else if (k0 + kKeys < s) {
        copier.issue(k0 + kKeys + first, id, lds0 + (slot ^ 1) * (2 * L::BYTES));
        copier.pages_at(prefix, k0 + 2 * kKeys + first, id);
      }
      if (k0 >= own_from) continue;   // the entry ends in this step, or before it
      const int h = way & 1, keys = k0 + 32 * way;
      u32x4 kf[1][L::QS], vf[2][L::NDB], pf[2];
      f32x16 sc[1];
#pragma unroll
      for (int st = 0; st < L::QS; ++st) kf[0][st] = L::key_chunk(sk, h, st, lane);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) vf[st][db] = L::value_chunk(sv, 2 * h + st, db, lane);
      __builtin_amdgcn_sched_barrier(0);
      rows.scores(kf, sc);
      rows.softmax(sc, keys, lim, j.scale_log2, pf);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) rows.add(db, vf[st][db], pf[st]);
    }

    // this block's own keys
    const int pmask = a.p.page_len - 1;
    for (int k0 = own_from + 32 * way; k0 < e.held; k0 += kKeys) {
      const int p0 = own_keys.in_pool(tail.page(k0, own_keys.shift, own_keys.last_block));
      const int p1 = own_keys.in_pool(tail.page(k0 + 16, own_keys.shift, own_keys.last_block));
      const int kr = L::key_of(fr);
      const uint8_t* ks = own_keys.K + (kr < 16 ? p0 : p1) * own_keys.page_bytes + ((k0 + kr) & pmask) * L::RB;
      u32x4 kf[1][L::QS], vf[2][L::NDB], pf[2];
      f32x16 sc[1];
#pragma unroll
      for (int st = 0; st < L::QS; ++st) kf[0][st] = *reinterpret_cast<const u32x4*>(ks + (2 * st + f) * 16);
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const uint8_t* vs = own_keys.V + (st ? p1 : p0) * own_keys.page_bytes + ((k0 + 16 * st + 8 * f) & pmask) * 2;
        const int left = e.held - (k0 + 16 * st + 8 * f);
#pragma unroll
        for (int db = 0; db < L::NDB; ++db)
          vf[st][db] = *reinterpret_cast<const u32x4*>(vs + size_t(32 * db + fr) * (a.p.page_len * 2));
        if (k0 + 32 > e.held) {   // values past the last key: whatever they are, times 0
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t keep = left > 2 * c + 1 ? ~0u : left > 2 * c ? 0xffffu : 0u;
#pragma unroll
            for (int db = 0; db < L::NDB; ++db) vf[st][db][c] &= keep;
          }
        }
      }
      rows.scores(kf, sc);
      rows.softmax(sc, k0, limit, j.scale_log2, pf);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) rows.add(db, vf[st][db], pf[st]);
    }

    // join the ways, two dim blocks at a time: way v sums 8 of a lane's 32 elements
    const float lsum = pair_sum(rows.l);
    float* xs = reinterpret_cast<float*>(smem) + block * (kWays * STATE * kWave) + lane;
    bf16_t* out = static_cast<bf16_t*>(a.out.p) + b * a.out.seq + i * a.out.row + (head * j.group + g) * a.out.head;
    const bool live = own && r0 + fr < per && i < e.rows;
#pragma unroll
    for (int d2 = 0; d2 < L::NDB; d2 += 2) {
      __syncthreads();   // the ring, or the last two blocks, have been read
#pragma unroll
      for (int c = 0; c < 32; ++c) xs[(way * STATE + c) * kWave] = rows.o[d2 + (c >> 4)][c & 15];
      xs[(way * STATE + 32) * kWave] = rows.m;
      xs[(way * STATE + 33) * kWave] = lsum;
      __syncthreads();
      float wt[kWays], top = -INFINITY, l = 0.f;
#pragma unroll
      for (int v = 0; v < kWays; ++v) {
        wt[v] = xs[(v * STATE + 32) * kWave];
        top = fmaxf(top, wt[v]);
      }
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int v = 0; v < kWays; ++v) {
        wt[v] = __builtin_amdgcn_exp2f(wt[v] - ref);
        l += xs[(v * STATE + 33) * kWave] * wt[v];
      }
      const float inv = 1.f / l;
#pragma unroll
      for (int c = 0; c < 8; c += 4) {
        const int c0 = 8 * way + c;   // element c0 % 16 of block d2 + c0 / 16
        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kWays; ++v)
#pragma unroll
          for (int u = 0; u < 4; ++u) y[u] += xs[(v * STATE + c0 + u) * kWave] * wt[v];
        if (live) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            store_f(out + 32 * (d2 + (c0 >> 4)) + 2 * (c0 & 15) + 4 * f + u, limit > 0 ? y[u] * inv : 0.f);
        }
      }
    }
  }
};

template <int HD>
__global__ __launch_bounds__(Pairs<HD>::kPairThreads, 2) void pairs_kernel(Job j) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[Pairs<HD>::SMEM];
  Pairs<HD>::run(j, blockIdx.x, smem);
}

// ---------------------------------------------------------------- launch

// how a part's rows are taken: 16 or 32 of them narrow, or 128 wide
enum { ROWS16 = 1, ROWS32 = 2, ROWS128 = 3 };
constexpr int rows_of(int mode) { return mode == ROWS16 ? 16 : mode == ROWS32 ? 32 : 128; }

template <typename T, int HD, int MODE> struct Taker;
template <typename T, int HD> struct Taker<T, HD, ROWS16> : Narrow<T, HD, 1> {};
template <typename T, int HD> struct Taker<T, HD, ROWS32> : Narrow<T, HD, 2> {};
template <int HD> struct Taker<bf16_t, HD, ROWS128> : Wide<HD> {};

// both parts in one launch: prefix workgroups, then the tails'
template <typename T, int HD, int PREFIX, int TAIL>
__global__ __launch_bounds__(kThreads, 2) void attention_kernel(Job j, int prefix_blocks) {
  using P = Taker<T, HD, PREFIX>;
  using U = Taker<T, HD, TAIL>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[P::SMEM > U::SMEM ? P::SMEM : U::SMEM];
  Share w;
  const int x = blockIdx.x;
  if (x < prefix_blocks) {
    if (share_of(j, x, true, rows_of(PREFIX), w)) P::run(j, w, smem);
  } else {
    if (share_of(j, x - prefix_blocks, false, rows_of(TAIL), w)) U::run(j, w, smem);
  }
}

// ---------------------------------------------------------------- merge

// out[row] = sum_r o_r 2^(m_r - m) / sum_r l_r 2^(m_r - m) over the ranges that
// hold positions the row sees; HD / 4 lanes a row and slice, slice c takes the
// ranges c, c + slices, .., and the slices are joined in order.
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void join_kernel(Job j, int slices) {
  constexpr int kLanes = HD / 4;
  __shared__ __attribute__((aligned(16))) float part[kThreads / kLanes][HD + 4];
  const PagedAttn& a = j.a;
  const int group = int(threadIdx.x) / kLanes, c = int(threadIdx.x) % kLanes * 4, slice = group % slices;
  const int rows = kThreads / kLanes / slices, row = blockIdx.x * rows + group / slices;
  const bool in = row < a.n * a.max_rows * a.heads;
  const int h = row % a.heads, t = row / a.heads, b = in ? t / a.max_rows : 0, i = t % a.max_rows;
  const Entry e = entry_of(a, b);
  const bool live = in && i < e.rows;
  const int s = j.stacked ? stacked_of(e, shared_of(a), j.prefix.range) : 0, lim = limit_of(a, e, i);
  const int np = live && j.prefix.ranges ? (min(lim, s) + j.prefix.range - 1) / j.prefix.range : 0;
  const int nt = live && lim > s ? min((lim - s + j.tail.range - 1) / j.tail.range, j.tail.ranges) : 0;
  const size_t stride = size_t(a.n) * a.max_rows * a.heads * record(HD);
  const float* rec = a.part + size_t(row) * record(HD);
  float m = -INFINITY, l = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](float mr, float lr, f32x4 v) {
    const float mn = fmaxf(m, mr), ref = mn == -INFINITY ? 0.f : mn;
    const float w0 = __builtin_amdgcn_exp2f(m - ref), w1 = __builtin_amdgcn_exp2f(mr - ref);
    l = l * w0 + lr * w1;
    o = o * w0 + v * w1;
    m = mn;
  };
  // four records in flight
  for (int r0 = slice; r0 < np + nt; r0 += 4 * slices) {
    float mr[4], lr[4];
    f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = min(r0 + u * slices, np + nt - 1);
      const float* x = rec + (r < np ? r : j.prefix.ranges + r - np) * stride;
      mr[u] = x[HD];
      lr[u] = x[HD + 1];
      v[u] = *reinterpret_cast<const f32x4*>(x + c);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (r0 + u * slices < np + nt) add(mr[u], lr[u], v[u]);
  }
  if (slices > 1) {
    *reinterpret_cast<f32x4*>(&part[group][c]) = o;
    if (c == 0) {
      part[group][HD] = m;
      part[group][HD + 1] = l;
    }
    __syncthreads();
    if (slice) return;
    for (int u = 1; u < slices; ++u)
      add(part[group + u][HD], part[group + u][HD + 1], *reinterpret_cast<const f32x4*>(&part[group + u][c]));
  }
  if (!live) return;
  T* out = static_cast<T*>(a.out.p) + b * a.out.seq + i * a.out.row + h * a.out.head + c;
#pragma unroll
  for (int x = 0; x < 4; ++x) store_f(out + x, lim > 0 ? o[x] / l : 0.f);
}

// ---------------------------------------------------------------- host

constexpr int kCus = 256;
constexpr int kMaxRanges = 64;

// How `groups` sets of stacked rows per key head are taken.  fp32 products
// cost an eighth of the bf16 rate, so there 32 rows, which halve what is
// read, are only taken where 16 fill the chip twice over (1000 positions, 16
// key heads of 64, 16 / 32 rows a workgroup: 8 x 32 rows 21 us / 24, 16 x 64
// 65 / 51, 32 x 32 67 / 53; at 16 x 32, which fill it once, 37 / 29, so there
// the border lies too high).  bf16 takes the wide kernel from 33 rows on
// (narrow / wide, 32 heads of 128: 8 x 40 rows over 1000 positions 39 us / 32,
// 16 x 48 over 2000 140 / 103, 16 x 33 over 1000 69 / 52, but 4 x 64 over 300 12
// / 14 and 4 x 33 over 1000 22 / 24: few rows over few keys lose 2 us to it).
int mode_of(int dtype, int rows, int64_t groups, int kv_heads) {
  if (dtype == DLLM_BF16) return rows > kNarrowRows ? ROWS128 : rows > 16 ? ROWS32 : ROWS16;
  return rows > 16 && cdiv(rows, 16) * groups * kv_heads >= 4 * kCus ? ROWS32 : ROWS16;
}

// most key ranges that a part of `items` workgroups a range is ever given: as
// many as give each CU two wide workgroups or eight narrow ones
int64_t most_ranges(int mode, int64_t items) {
  const int64_t wgs = mode == ROWS128 ? 2 * kCus : 8 * kCus;
  return std::min<int64_t>(kMaxRanges, (wgs + items - 1) / items);
}

// the unit in which plan_part counts: what a narrow workgroup of 16 bf16 rows
// (of heads of 64: 32 too) takes at a time; fp32 and wider ones take a half or a
// quarter of it a step (Narrow::KS)
constexpr int kStep = kWaves * kTile;

// Rows stacked per key head, in `groups` separate sets (entries of a tail).
// Two workgroups fit a CU.  Narrow parts are bound by memory: as many ranges
// as fill the chip, and where they are long ones of 24 tiles, so that batches
// of unlike lengths come out even.  Joining them costs 3 us, so parts of up to
// two kStep are not divided, nor parts of up to six that have a workgroup for
// every CU (single tokens of 8 key heads, whole / divided: 8 over 500 positions
// 11.8 us / 12.6, over 520 13.3 / 13.0, over 1000 19.4 / 13.3; 1 over 1000 18.6 /
// 11.6; 32 over 600 17.0 / 20.5, over 1000 23.1 / 26.9, over 1500 32.0 / 35.7).
// Wide ones take one workgroup a CU, which leaves the other slot to the tails,
// and two where ranges stay long enough for the second to gain more than its
// records cost to join; beside tails that take `beside_us` by themselves, only
// as many as end by then (14 us and 1.2 us a tile: 64 single tokens over 8000
// shared positions and up to 1500 of their own, 16 ranges 58 us, 8 ranges 47, the
// rule's 6 50, 4 ranges 62).
Part plan_part(int mode, int rows, int64_t groups, int kv_heads, int64_t keys, double beside_us = 0.0) {
  Part p;
  p.row_tiles = cdiv(rows, rows_of(mode));
  const int64_t tiles = (keys + kTile - 1) / kTile, items = p.row_tiles * groups * kv_heads;
  auto fill = [&](int64_t wgs) { return (wgs + items - 1) / items; };
  int64_t ranges;
  if (mode == ROWS128) {
    ranges = tiles >= 24 * fill(kCus) ? fill(2 * kCus) : fill(kCus);
    if (beside_us > 16.0) ranges = std::min(ranges, int64_t(1.2 * double(tiles) / (beside_us - 14.0)) + 1);
  } else ranges = keys <= (items >= kCus ? 6 : 2) * kStep ? 1 : std::max(fill(2 * kCus), tiles / 24);
  ranges = std::max<int64_t>(1, std::min<int64_t>({ranges, most_ranges(mode, items), tiles / 4}));
  p.range = int(std::max<int64_t>(1, (tiles + ranges - 1) / ranges)) * kTile;
  p.ranges = int(std::max<int64_t>(1, (keys + p.range - 1) / p.range));
  return p;
}

template <typename T, int HD, int PREFIX, int TAIL>
void launch_parts(const Job& j, hipStream_t s) {
  const int kvh = j.a.p.n_kv_heads;
  const int prefix = j.prefix.ranges ? blocks_of(j.prefix.ranges * kvh, j.prefix.row_tiles) : 0;
  const int tail = blocks_of(j.a.n * j.tail.ranges * kvh, j.tail.row_tiles);
  hipLaunchKernelGGL((attention_kernel<T, HD, PREFIX, TAIL>), dim3(prefix + tail),
                     dim3(kThreads), 0, s, j, prefix);
}

// (a prefix never takes fewer rows than the tails, see divide)
template <typename T, int HD>
void launch_modes(const Job& j, int prefix, int tail, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (tail == ROWS128) return launch_parts<T, HD, ROWS128, ROWS128>(j, s);
    if (prefix == ROWS128)
      return tail == ROWS32 ? launch_parts<T, HD, ROWS128, ROWS32>(j, s) : launch_parts<T, HD, ROWS128, ROWS16>(j, s);
  }
  if (tail == ROWS32) return launch_parts<T, HD, ROWS32, ROWS32>(j, s);
  return prefix == ROWS32 ? launch_parts<T, HD, ROWS32, ROWS16>(j, s) : launch_parts<T, HD, ROWS16, ROWS16>(j, s);
}

template <typename T, int HD>
void launch(const Job& j, int prefix, int tail, hipStream_t s) {
  launch_modes<T, HD>(j, prefix, tail, s);
  if (j.direct) return;
  // rows of many ranges take several groups of lanes each: the records of a
  // row come in turn, four at a time
  constexpr int kGroups = kThreads / (HD / 4);
  const int ranges = j.prefix.ranges + j.tail.ranges;
  const int slices = ranges <= 4 ? 1 : ranges <= 8 ? 2 : ranges <= 16 ? 4 : 8;
  hipLaunchKernelGGL((join_kernel<T, HD>), dim3(cdiv(j.a.n * j.a.max_rows * j.a.heads, kGroups / slices)),
                     dim3(kThreads), 0, s, j, slices);
}

}  // namespace

size_t paged_attention_workspace(const dllm_kv_pages& p, int n, int max_rows, int heads) {
  const int group = heads / p.n_kv_heads;
  auto ranges = [&](int rows, int groups) {
    const int mode = mode_of(p.dtype, rows, groups, p.n_kv_heads);
    return most_ranges(mode, int64_t(cdiv(rows, rows_of(mode))) * groups * p.n_kv_heads);
  };
  const size_t parts = ranges(n * max_rows * group, 1) + ranges(max_rows * group, n);
  return parts * n * max_rows * heads * record(p.head_dim) * sizeof(float);
}

size_t paged_attention_workspace_upto(const dllm_kv_pages& p, int n, int max_rows, int heads) {
  // R rows of all heads in a part of `items` workgroups have at most
  // kMaxRanges records each, and at most (wgs / items + 1) R <= wgs * tile rows + R
  // together
  const int64_t R = int64_t(n) * max_rows * heads;
  const int64_t each = std::max<int64_t>(2 * kCus * rows_of(ROWS128), 8 * kCus * rows_of(ROWS32));
  return size_t(2 * std::min(kMaxRanges * R, each + R)) * record(p.head_dim) * sizeof(float);
}

namespace {

// Three ways to take a batch over a shared prefix: every entry by itself, from
// position 0 on; the prefix and the tails as parts, joined; pairs.  The one of the
// least estimated time is taken (measured, us, heads of 128, entries / parts /
// pairs: 32 heads, 16 x 32 rows over 64 positions 10.5 / 22.4 / 11.3, over 128
// 12.8 / 21.8 / 10.6, over 1024 38 / 31 / 22, over 8000 247 / 98 / 97, over 30000
// 1000 / 313 / 366; 16 x 128 over 1024 53 / 83 / 81; 16 x 40 over 128 15 / 28 /
// 19, over 4096 151 / 87 / 106; 64 x 32 over 64 32 / 61 / 43, over 4096 462 / 200
// / 204; 8 key heads, 32 single tokens over 500 19.6 / 22.4, over 1000 26.2 /
// 20.6; fp32, 16 heads of 64, 7 x 19 over 203 10.3 / 13.8, 7 x 4 over 1000 19.7 /
// 14.4).  Of 92 batches of this kind all but three were within 10% of the best
// of the three, those within 16%.
//
// Estimated times, in us on a whole MI355X:
//   work   of a part where the chip is full of it: keys and values of narrow
//          workgroups at 8.5 TB/s (they come from the caches for the most
//          part), and 4.5 for every round of two workgroups a CU after the
//          first; 2.4 for a wide tile of two workgroups on every CU
//   wait   along one workgroup: 2.7 a narrow step, 1.6 a wide tile
struct Cost {
  double work, wait;
};
Cost cost_of(const PagedAttn& a, int mode, const Part& p, int groups, double keys) {
  const double items = double(p.row_tiles) * groups * a.p.n_kv_heads, range = std::min(double(p.range), keys);
  const int row = a.p.head_dim * (a.p.dtype == DLLM_BF16 ? 2 : 4);
  if (mode == ROWS128) {
    const double u = row / 256.0 / kTile;
    return {2.4 * u * keys * items / (2 * kCus), 1.6 * u * range};
  }
  const int step = kWaves * std::min(64, (mode == ROWS16 && a.p.dtype == DLLM_BF16 ? 16 : 8) * 1024 / row);
  return {items * keys * 2 * row / 8.5e6 + 4.5 * std::max(0.0, items / (2 * kCus) - 1), 2.7 * range / step};
}
// a launch, two parts in it, and the join of a row's records, written and read at 5 TB/s
double parts_us(const PagedAttn& a, int mode, Cost x, Cost y, int records) {
  const double rows = double(a.n) * a.max_rows * a.heads;
  return (mode == ROWS32 ? 7.0 : 6.0) + std::max({x.work + y.work, x.wait, y.wait}) +
         (records > 1 ? 3.0 + rows * records * 2 * record(a.p.head_dim) * sizeof(float) / 5e6 : 0.0);
}
// blocks of 32 rows in pairs (see Pairs), a pair on a CU: steps of 128 keys of
// the prefix, then of the tail
double pairs_us(const PagedAttn& a, int rows, int64_t shared, double tail) {
  const double u = a.p.head_dim / 128.0, all = double(a.n) * cdiv(rows, 32) * a.p.n_kv_heads;
  return std::ceil(all / (2 * kCus)) * (4.8 + u * (3.4 + (1.45 * shared + 3.5 * tail) / Pairs<128>::kKeys));
}

// how a call is taken: pairs, or a prefix (stacked) and tails
struct Division {
  bool pairs, stacked;
  int mode_p, mode_t;
  Part prefix, tail;
  int64_t shared;   // whole pages of the prefix, as far as the caller knows
};
Division divide(const PagedAttn& a) {
  Division d{};
  const int dt = a.p.dtype, kvh = a.p.n_kv_heads, group = a.heads / kvh;
  const int64_t most = int64_t(a.p.max_blocks) * a.p.page_len;
  const int64_t shared = d.shared = std::min<int64_t>(a.shared_len, most) / a.p.page_len * a.p.page_len;
  const int rows_t = a.max_rows * group, rows_p = a.n * rows_t;
  const int64_t keys = std::max<int64_t>(1, std::min<int64_t>(a.max_len, most));
  d.mode_p = d.mode_t = mode_of(dt, rows_t, a.n, kvh);
  // lengths of the tails: the longest, and half of it on average
  const int64_t longest = std::max<int64_t>(1, keys - shared);
  const double mean = std::max<int64_t>(0, keys - shared) / 2.0;
  d.prefix = Part{1, 0, kTile};
  d.tail = plan_part(d.mode_t, rows_t, a.n, kvh, std::max(keys, shared));
  if (shared == 0) return d;
  const Cost none{0, 0};
  const double own = parts_us(a, d.mode_t, cost_of(a, d.mode_t, d.tail, a.n, shared + mean), none, d.tail.ranges);
  const int mode = mode_of(dt, rows_p, 1, kvh);
  const Part tail = plan_part(d.mode_t, rows_t, a.n, kvh, longest);
  // what the tails take by themselves, at 5 TB/s
  const double tail_us =
      double(a.n) * tail.row_tiles * kvh * mean * 2 * a.p.head_dim * (dt == DLLM_BF16 ? 2 : 4) / 5e6;
  const Part prefix = plan_part(mode, rows_p, 1, kvh, shared, tail_us);
  const double parts = parts_us(a, d.mode_t, cost_of(a, mode, prefix, 1, double(shared)),
                                cost_of(a, d.mode_t, tail, a.n, mean), prefix.ranges + tail.ranges);
  // (of fewer rows than half a block most of a pair would be empty; a prefix
  // in 16 rows over tails in 32, which only fp32 could ask for, has at least as
  // many row tiles as the entries by themselves and costs more than they do)
  d.pairs = dt == DLLM_BF16 && rows_t >= 16 && pairs_us(a, rows_t, shared, mean) < std::min(own, parts);
  d.stacked = !d.pairs && parts < own && mode >= d.mode_t;
  if (d.stacked) {
    d.prefix = prefix;
    d.tail = tail;
    d.mode_p = mode;
  }
  return d;
}

}  // namespace

hipError_t paged_attention(const PagedAttn& a, hipStream_t s) {
  Job j{};
  j.a = a;
  j.scale_log2 = a.scale * 1.4426950408889634f;
  j.group = a.heads / a.p.n_kv_heads;
  const Division d = divide(a);
  const int kvh = a.p.n_kv_heads, hd = a.p.head_dim;
  if (d.pairs) {
    j.direct = true;
    const int grid = blocks_of(kvh, cdiv(a.n * cdiv(a.max_rows * j.group, 32), 2));
    if (hd == 128) hipLaunchKernelGGL(pairs_kernel<128>, dim3(grid), dim3(Pairs<128>::kPairThreads), 0, s, j);
    else hipLaunchKernelGGL(pairs_kernel<64>, dim3(grid), dim3(Pairs<64>::kPairThreads), 0, s, j);
    return hipGetLastError();
  }
  j.prefix = d.prefix;
  j.tail = d.tail;
  j.stacked = d.stacked;
  if (d.shared == 0) j.a.shared_len = j.a.prefix_seq = 0;
  j.direct = j.prefix.ranges + j.tail.ranges == 1;
  if (a.p.dtype == DLLM_BF16)
    hd == 128 ? launch<bf16_t, 128>(j, d.mode_p, d.mode_t, s) : launch<bf16_t, 64>(j, d.mode_p, d.mode_t, s);
  else
    hd == 128 ? launch<float, 128>(j, d.mode_p, d.mode_t, s) : launch<float, 64>(j, d.mode_p, d.mode_t, s);
  return hipGetLastError();
}

kv_attention_plan paged_attention_plan(const PagedAttn& a) {
  const Division d = divide(a);
  kv_attention_plan p{};
  p.way = d.pairs ? KV_WAY_PAIRS : d.stacked ? KV_WAY_PARTS : KV_WAY_ENTRIES;
  if (d.pairs) return p;
  if (d.stacked) {
    p.prefix_rows = rows_of(d.mode_p);
    p.prefix_ranges = d.prefix.ranges;
    p.prefix_keys = d.prefix.range;
  }
  p.tail_rows = rows_of(d.mode_t);
  p.tail_ranges = d.tail.ranges;
  p.tail_keys = d.tail.range;
  return p;
}

}  // namespace dllm
