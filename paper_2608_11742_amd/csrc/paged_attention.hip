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
// Four kernels, by the number of stacked rows (MI355X; floors by the rates of
// a large copy, 4.9 TB/s, and a large bf16 product, 1190 TFLOP/s):
//   narrow   up to 32 rows: bound by the keys and values it streams.  The
//            waves share the rows and take the key steps in turn; a step's
//            fragments come straight from memory into registers, K of the
//            next step while the softmax runs, V after it (no LDS, no
//            barrier), and the waves' states are joined through LDS at the
//            end.  Single tokens of 4 sequences up to 120000 long, 8 key heads
//            of 128: 217 us, 5.7 TB/s.
//   wide     128 rows, 32 a wave (bf16).  Tiles of 64 keys go through a
//            two-slot LDS ring, copied one tile ahead, on 32 x 32 MFMAs; a
//            wave issues one copy after each step of the score products (2%
//            faster than all of them before the products).  16 x 32 rows of 32
//            heads over 30011 positions: 299-316 us by device, 0.80-0.85 PFLOP/s,
//            floor 213.  Matrix units are
//            busy 44% of it: products and softmax alone take 177 us, and
//            fragment reads from LDS, the copies and the join of the ranges
//            (15) are covered in part.
//   halves   33 to 64 rows of a tree (bf16): the wide kernel with two waves on
//            each block of 32 rows, which take half the keys of a tile each.
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
// million keys that weigh 2^-25 each are not lost beside one that weighs 1.  Such
// an output is 1.67e-3 off 64 bits (root mean square, the rounding to bf16), with
// weights in 32 bits 1.66e-3; the two differ by 8e-4, where the rounding to bf16
// falls the other way.  The
// sums l and products o are held in 32 bits; wide and pairs sum the weights as
// rounded, narrow before.  fp32 needs no such room above a rounding.  There the
// reference is the largest score itself when it moves, where the exponent of the
// largest weights is near 0 and its own rounding smallest, and stands up to 2^7;
// and every weight is divided by 2^8 times the positions that a sequence can
// have, so that all of a row's weights sum up to less than 1 and no sum of
// products passes the largest value: finite values give a finite output, as a mean
// has to be.  At the other end, products of values below 2^-118 times those
// positions lose bits.
#include <algorithm>
#include <climits>
#include <utility>

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
constexpr float kFirst32 = 0.f, kMost32 = 7.f;   // fp32: before Job::weight
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
  float weight;       // fp32: what every weight is multiplied by, a power of two
  int group;          // query heads per key head
  Part prefix, tail;
  bool stacked;       // the prefix is a part of its own; else each tail starts at position 0
  bool direct;        // one range in all: the output itself
  int slots;          // of a tree's tails (see Slots); 0: each entry has tail.ranges
  int slices;         // groups of lanes that a row of the join has
};
// Kernels take it by value: arguments past 256 bytes cost each launch 0.3 us (24
// single tokens of 32 heads of 64 over 530 positions 11.75 -> 12.06 us)
static_assert(sizeof(Job) <= 256, "arguments of a launch");

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
// positions that all rows of the entry see, from the first on (the rest: its tail's)
template <bool TREE>
__device__ __forceinline__ int common_of(const Entry& e) {
  return TREE ? max(e.held - e.rows, 0) : e.held;
}
// of the `shared` positions, those that the entry takes with the others', which are in steps of `range`
template <bool TREE>
__device__ __forceinline__ int stacked_of(const Entry& e, int shared, int range) {
  const int held = common_of<TREE>(e);
  return held >= shared ? shared : held / range * range;
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
  int row0, row_end, head, k0, k1, split;
  int part;    // of the share's records (see record_of)
  int slots;   // how far a slot of a tree's tails is past its entry's number; 0 without slots
  Entry e;     // of a tail of a tree
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
__host__ __device__ __forceinline__ int blocks_of(int items, int row_tiles) { return (items + 7) / 8 * 8 * row_tiles; }
// workgroups of the prefix
__host__ __device__ __forceinline__ int prefix_blocks(const Job& j) {
  return blocks_of(j.prefix.ranges * j.a.p.n_kv_heads, j.prefix.row_tiles);
}

// v of the lane that `CTRL` moves here (0 where the rows of ROWS do not take part)
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int moved(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
// sums of v over the lanes up to each one
__device__ __forceinline__ int wave_sums(int v) {
  v += moved<0x111>(v);   // the lanes 1, 2, 4, 8 before it in its 16
  v += moved<0x112>(v);
  v += moved<0x114>(v);
  v += moved<0x118>(v);
  v += moved<0x142, 0xa>(v);   // the last of the 16 before, and of the 32
  v += moved<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_sums(v), kWave - 1); }

// The tails of trees are divided by what the entries hold: of the slots that a
// head and row tile have, an entry gets one for every `step` tiles, the least
// step with which all find a slot (and 4 at least).  So one long entry among short
// ones, or a max_len that is far off, leaves no workgroup without work.  Every
// wave works it out from the lengths, a lane for each of up to 64 entries; more
// have even ranges, and more than 32 bf16 rows of each of them one (see plan_tree).
struct Slots {
  Entry e;                   // of this lane
  int count, first, tiles;   // its slots, and the tiles in them
};
template <bool TREE>
__device__ __forceinline__ Slots slots_of(const Job& j, int shared) {
  const int lane = threadIdx.x & 63, all = j.slots;
  Slots s{};
  if (lane < j.a.n) {
    s.e = entry_of(j.a, lane);
    const int from = j.stacked ? stacked_of<TREE>(s.e, shared, j.prefix.range) : 0;
    s.tiles = s.e.rows > 0 ? (s.e.held - from + kTile - 1) / kTile : 0;
  }
  int step = max((wave_total(s.tiles) + all - 1) / all, 4), used;
  // at most a slot too many an entry: the step grows until they fit
  while (s.count = (s.tiles + step - 1) / step, used = wave_total(s.count), used > all)
    step += max(1, int(int64_t(step) * (used - all) / all));
  s.first = wave_sums(s.count) - s.count;
  return s;
}

// False if the share is empty.
template <bool TREE>
__device__ __forceinline__ bool share_of(const Job& j, int x, bool in_prefix, int tile_rows, Share& w) {
  const PagedAttn& a = j.a;
  const int per = a.max_rows * j.group;   // stacked rows of one entry
  const Part& part = in_prefix ? j.prefix : j.tail;
  const Item it = item_of(x, part.row_tiles);
  w.head = it.item % a.p.n_kv_heads;
  const int t = it.item / a.p.n_kv_heads;
  int r = t % part.ranges, b = t / part.ranges;
  const bool by_length = TREE && j.slots && !in_prefix;
  // items are filled up to whole rounds of XCDs
  if (by_length ? t >= j.slots : b >= (in_prefix ? 1 : a.n)) return false;
  const int s = shared_of(a);
  w.slots = 0;
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
  int range = part.range, ranges = part.ranges;
  w.part = j.prefix.ranges + r;
  if (by_length) {
    const Slots z = slots_of<TREE>(j, s);
    // slot t is of the last entry that starts at or before it (one without any starts where the next does)
    b = __popcll(__ballot(int(threadIdx.x & 63) < a.n && z.first <= t)) - 1;
    r = t - __builtin_amdgcn_readlane(z.first, b);
    ranges = __builtin_amdgcn_readlane(z.count, b);
    if (r >= ranges) return false;
    const int tiles = __builtin_amdgcn_readlane(z.tiles, b);
    range = (tiles + ranges - 1) / ranges * kTile;   // even
    w.part = j.prefix.ranges;
    w.slots = t - b;
    w.e = Entry{__builtin_amdgcn_readlane(z.e.seq, b), __builtin_amdgcn_readlane(z.e.held, b),
                __builtin_amdgcn_readlane(z.e.rows, b)};
  } else {
    w.e = entry_of(a, b);
  }
  const Entry& e = w.e;
  w.row0 = b * per + it.tile * tile_rows;
  w.row_end = (b + 1) * per;
  w.k0 = (j.stacked ? stacked_of<TREE>(e, s, j.prefix.range) : 0) + r * range;
  w.k1 = r + 1 == ranges ? e.held : min(w.k0 + range, e.held);
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

// A part has a record for every row of all entries; the slots of a tree's tails,
// with the rows of one entry each, follow one another from their first part on.
__device__ __forceinline__ float* record_of(const Job& j, const Share& w, const RowAt& r, int kvh, int hd) {
  const int64_t row = (int64_t(r.b + w.slots) * j.a.max_rows + r.i) * j.a.heads + kvh * j.group + r.g;
  return j.a.part + (int64_t(w.part) * j.a.n * j.a.max_rows * j.a.heads + row) * record(hd);
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

// ---------------------------------------------------------------- trees
//
// A tree's keys are in the tails alone, a few of the last steps, where a row
// sees what its mask names: its words give the bits of a step's keys.  A value
// that one row must not see is there for the others, and a weight of 0 would not
// cancel it if it is infinite or no number.  Such values, looked for in these
// steps only, are taken out before the product; where there were any, a pass
// over the steps' values at the end brings them to the rows that see them: two
// products with the masks in place of the weights count per row and dim those
// that are +inf or NaN and those that are -inf or NaN.

// the words of row i's mask that hold the tree's keys among k0 .. k0 + 63; `root`:
// the tree's first position, negative where the sequence is shorter than its rows
struct MaskWords {
  uint32_t w[3];
};
__device__ __forceinline__ MaskWords mask_words(const PagedAttn& a, int b, int i, int root, int k0) {
  const int words = (a.max_rows + 31) / 32;
  const uint32_t* row = a.mask + (size_t(b) * a.max_rows + i) * words;
  const int j = max(k0 - root, 0) >> 5;
  MaskWords m;
  // (words past the mask's are read from inside it, so that no load waits behind a branch)
#pragma unroll
  for (int u = 0; u < 3; ++u) {
    const uint32_t w = row[min(j + u, words - 1)];
    m.w[u] = j + u < words ? w : 0u;
  }
  return m;
}
// bits of the keys k0 .. k0 + 63 that the row sees: those before the tree, of the
// tree those in its mask, none from `end` on
__device__ __forceinline__ uint64_t seen_in(const MaskWords& m, int root, int end, int k0) {
  const int t = k0 - root, shift = t & 31;
  const uint64_t w = uint64_t(m.w[1]) << 32 | m.w[0];
  uint64_t bits;
  if (t >= 0) bits = w >> shift | (shift ? uint64_t(m.w[2]) << (64 - shift) : 0);
  else bits = t <= -64 ? ~uint64_t(0) : w << -t | ~(~uint64_t(0) << -t);
  const int left = end - k0;
  return left >= 64 ? bits : left <= 0 ? 0 : bits & ~(~uint64_t(0) << left);
}
__device__ __forceinline__ uint64_t seen_of(const PagedAttn& a, int b, int i, int root, int end, int k0) {
  return seen_in(mask_words(a, b, i, root, k0), root, end, k0);
}

// of a word of values: 1 in the places of those that are +inf or NaN (up), -inf or NaN (down)
struct Wild {
  uint32_t up, down;
};
template <bool kHalf>
__device__ __forceinline__ Wild wild_of(uint32_t w) {
  if constexpr (kHalf) {
    Wild x{0, 0};
#pragma unroll
    for (int s = 0; s < 32; s += 16) {
      const uint32_t v = w >> s & 0xffffu, e = v & 0x7fffu;
      if (e > 0x7c00u || v == 0x7c00u) x.up |= 0x3c00u << s;
      if (e > 0x7c00u || v == 0xfc00u) x.down |= 0x3c00u << s;
    }
    return x;
  } else {
    const uint32_t e = w & 0x7fffffffu;
    return Wild{e > 0x7f800000u || w == 0x7f800000u ? 0x3f800000u : 0u,
                e > 0x7f800000u || w == 0xff800000u ? 0x3f800000u : 0u};
  }
}
// the top bit of each value of a word that is infinite or no number: its
// exponent, all ones, carries into it
template <bool kHalf>
__device__ __forceinline__ uint32_t wild_bits(uint32_t w) {
  return kHalf ? ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u : ((w & 0x7f800000u) + 0x00800000u) & 0x80000000u;
}
// those values as 0
template <bool kHalf>
__device__ __forceinline__ uint32_t tame(uint32_t w) {
  const uint32_t x = wild_bits<kHalf>(w);
  return w & ~(kHalf ? (x >> 15) * 0xffffu : uint32_t(int32_t(x) >> 31));
}
// what counts of `up` and `down` add to an output
__device__ __forceinline__ float wild_sum(bool up, bool down) {
  return (up ? INFINITY : 0.f) + (down ? -INFINITY : 0.f);
}
// the low bits of x as 1s and 0s of a chunk of 8 binary16 or 4 fp32 values
template <bool kHalf>
__device__ __forceinline__ u32x4 ones_of(uint32_t x) {
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    y[i] = kHalf ? (x >> (2 * i) & 1 ? 0x3c00u : 0u) | (x >> (2 * i + 1) & 1 ? 0x3c000000u : 0u)
                 : (x >> i & 1 ? 0x3f800000u : 0u);
  return y;
}

// ---------------------------------------------------------------- narrow

// NQB blocks of 16 rows.  A key step is KS keys in blocks of 16; bf16 keys of
// a 32-key half are gathered so that output element i of lane group g in
// block kk is key 8 g + 4 kk + i: the lane's 8 probabilities of the half are 8
// consecutive keys, one 16-byte chunk of a V^T row.
template <typename T, int HD, int NQB, bool TREE>
struct Narrow {
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr float FIRST = kHalf ? kFirst : kFirst32, MOST = kHalf ? kMost : kMost32;
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
    int root = 0;   // position of the tree's first row
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
      at[qb] = row_at(j, min(w.row0 + 16 * qb + fr, w.row_end - 1));
      const Entry e = TREE ? w.e : entry_of(a, at[qb].b);
      lim[qb] = min(limit_of(a, e, at[qb].i), w.k1);
      rows[qb] = e.rows;
      root = e.held - e.rows;
    }
    // keys up to `end` are in the steps on their way, those of a tree (from its 16-key group on) in others
    int end = w.k1;
    if constexpr (TREE) {
      root = __builtin_amdgcn_readfirstlane(root);
      end = min(max(max(root, 0) & ~15, w.k0), w.k1);
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) lim[qb] = min(lim[qb], end);
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

    // the parts of a step, on the fragments loaded
    typedef f32x4 Scores[NB][NQB];
    auto score = [&](Scores& sc) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          sc[kb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int st = 0; st < QS; ++st) Mfma<T>::run(sc[kb][qb], kf[kb][st], qf[qb][st]);
        }
    };
    auto softmax = [&](Scores& sc) {
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
        const float mn = top > m[qb] + MOST ? top - FIRST : m[qb];
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
            if constexpr (!kHalf) sc[kb][qb][i] *= j.weight;
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
    };
    // values past the last key: whatever they are, times 0
    auto cut_values = [&](int k0) {
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        const int left = end - (k0 + (4 * c + g) * E);   // valid elements of this lane's chunks
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t keep = kHalf ? (left > 2 * x + 1 ? ~0u : left > 2 * x ? 0xffffu : 0u) : (left > x ? ~0u : 0u);
#pragma unroll
          for (int db = 0; db < NDB; ++db) vf[db][c][x] &= keep;
        }
      }
    };
    auto multiply = [&](const Scores& sc) {
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
    };

    int k0 = w.k0 + wave * KS;
    int id[NB];
    if (k0 < end) {
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
    if (k0 < end) load_v(k0, id);
    for (; k0 < end; k0 += kWaves * KS) {
      const int next = k0 + kWaves * KS;
      const bool more = next < end;
      if (more) pages_at(next, id);
      Scores sc;
      score(sc);
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
      softmax(sc);
      if (k0 + KS > end) cut_values(k0);
      multiply(sc);
      if (more) load_v(next, id);
    }

    if constexpr (TREE) {
      // the tree's keys, which few steps hold: the first is the wave's whose turn it would be
      const int steps = (max(end - w.k0, 0) + KS - 1) / KS, first = end + ((wave - steps) & (kWaves - 1)) * KS;
      end = w.k1;
      bool any_wild = false;
      for (k0 = first; k0 < end; k0 += kWaves * KS) {
        pages_at(k0, id);
        load_k(k0, id);
        constexpr bool kLate = !kHalf && NQB == 2;   // K and V together would spill
        if (!kLate) load_v(k0, id);
        uint64_t seen[NQB];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) seen[qb] = seen_of(a, at[qb].b, at[qb].i, root, end, k0);
        Scores sc;
        score(sc);
        if (kLate) load_v(k0, id);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
#pragma unroll
          for (int kb = 0; kb < NB; ++kb) {
            const uint32_t bits = uint32_t(seen[qb] >> key_of(kb, 4 * g));
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!(bits >> i & 1)) sc[kb][qb][i] = -INFINITY;
          }
        }
        softmax(sc);
        if (k0 + KS > end) cut_values(k0);
        uint32_t wild = 0;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
          for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int x = 0; x < 4; ++x) wild |= wild_bits<kHalf>(vf[db][c][x]);
        if (__any(wild)) {
          any_wild = true;
#pragma unroll
          for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                asm volatile("" : "+v"(vf[db][c][x]));   // else what was found above is kept, a register a word
                vf[db][c][x] = tame<kHalf>(vf[db][c][x]);
              }
        }
        multiply(sc);
      }
      for (k0 = any_wild ? first : end; k0 < end; k0 += kWaves * KS) {
        pages_at(k0, id);
        load_v(k0, id);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          const uint64_t seen = seen_of(a, at[qb].b, at[qb].i, root, end, k0);
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            f32x4 up = f32x4{0.f, 0.f, 0.f, 0.f}, down = up;
#pragma unroll
            for (int c = 0; c < NV; ++c) {
              const u32x4 sees = ones_of<kHalf>(uint32_t(seen >> ((4 * c + g) * E)));
              u32x4 wu, wd;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const Wild y = wild_of<kHalf>(vf[db][c][x]);
                wu[x] = y.up;
                wd[x] = y.down;
              }
              if constexpr (kHalf) {
                MfmaF16::run(up, wu, sees);
                MfmaF16::run(down, wd, sees);
              } else {
                Mfma<float>::run(up, wu, sees);
                Mfma<float>::run(down, wd, sees);
              }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) o[db][qb][i] += wild_sum(up[i] > 0.f, down[i] > 0.f);
          }
        }
      }
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
      const bool any = TREE ? sum != 0.f : lim[qb] > 0;   // the row sees a position
      const float inv = any ? 1.f / sum : 0.f;
      T* out = static_cast<T*>(a.out.p) + at[qb].b * a.out.seq + at[qb].i * a.out.row +
               (kvh * j.group + at[qb].g) * a.out.head;
      float* rec = record_of(j, w, at[qb], kvh, HD);
      for (int db = wave; db < NDB; db += kWaves) {
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] += smem[(v * STATE + 4 * db + i) * kWave + lane] * mw[v];
        if (!live) continue;
        if (j.direct) {
#pragma unroll
          for (int i = 0; i < 4; ++i) store_f(out + 16 * db + 4 * g + i, any ? x[i] * inv : 0.f);
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

template <class F, int... I>
__device__ __forceinline__ void static_for_each(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(0) .. f(N - 1), each with a constant
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_each(std::make_integer_sequence<int, N>{}, f);
}

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

  // page ids of a tile's 16-key groups
  struct Ids {
    int a, b, c, d;
    template <int i>
    __device__ __forceinline__ int of() const {
      return i == 0 ? a : i == 1 ? b : i == 2 ? c : d;
    }
  };

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
    __device__ __forceinline__ Ids pages_at(const Share& w, int k0) const {
      return Ids{w.page(k0, shift, last_block), w.page(k0 + 16, shift, last_block), w.page(k0 + 32, shift, last_block),
                 w.page(k0 + 48, shift, last_block)};
    }
    // the i-th of IC copies of keys, and of values
    template <int i>
    __device__ __forceinline__ void issue_keys(int k0, Ids id, uint32_t dst) const {
      const int pmask = page_len - 1, kr = lane / CK;
      const int grp = i * kWaves + wave, r = grp * KROWS + kr;
      // a copy's rows share a 16-key group, one of C over the waves
      constexpr int C = kWaves * KROWS / 16;
      const int u = wave * KROWS / 16, sub = i * C + u;
      const int page = in_pool(u ? id.template of<i * C + C - 1>() : id.template of<i * C>());
      const uint8_t* src = K + page * page_bytes + ((k0 + sub * 16) & pmask) * RB;
      copy16(src + (r & 15) * RB + ((lane % CK) ^ kswz(r)) * 16, dst + grp * 1024);
    }
    template <int i>
    __device__ __forceinline__ void issue_values(int k0, Ids id, uint32_t dst) const {
      const int pmask = page_len - 1, vd = lane >> 3, vc = (lane & 7) ^ vswz(8 * wave + vd);
      const int page = in_pool(vc < 4 ? (vc < 2 ? id.a : id.b) : (vc < 6 ? id.c : id.d));
      const uint8_t* src = V + page * page_bytes + size_t(vd) * (page_len * 2) + ((k0 + 8 * vc) & pmask) * 2;
      const int grp = i * kWaves + wave;
      copy16(src + size_t(grp) * 8 * (page_len * 2), dst + KB + grp * 1024);
    }
    // the c-th of all 2 IC, one after each step over head_dim of the products
    template <int c>
    __device__ __forceinline__ void issue_one(int k0, Ids id, uint32_t dst) const {
      static_assert(2 * IC == QS, "a copy a step");
      if constexpr (c < IC) issue_keys<c>(k0, id, dst);
      else issue_values<c - IC>(k0, id, dst);
      __builtin_amdgcn_sched_barrier(0);
    }
    __device__ __forceinline__ void issue(int k0, Ids id, uint32_t dst) const {
      static_for<IC>([&](auto i) { issue_keys<i>(k0, id, dst); });
      static_for<IC>([&](auto i) { issue_values<i>(k0, id, dst); });
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
  // zero_values, and whether any other of the tile's values is infinite or no
  // number, as this one of kThreads threads finds it
  __device__ __forceinline__ static bool tidy_values(uint8_t* sv, int t, int left) {
    constexpr int N = HD * 8 / kThreads;
    u32x4 x[N];
    auto at = [&](int i) {
      const int c = t + i * kThreads, d = c >> 3;
      return reinterpret_cast<u32x4*>(sv + d * 128 + (((c & 7) ^ vswz(d)) << 4));
    };
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *at(i);
    const int n = left - 8 * (t & 7);   // kThreads is a multiple of 8: all of a thread's chunks are of the same keys
    uint32_t wild = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        x[i][u] &= n > 2 * u + 1 ? ~0u : n > 2 * u ? 0xffffu : 0u;
        wild |= wild_bits<true>(x[i][u]);
      }
    if (n < 8) {
#pragma unroll
      for (int i = 0; i < N; ++i) *at(i) = x[i];
    }
    return wild != 0;
  }
  __device__ __forceinline__ static void tame_values(uint8_t* sv, int t, int threads) {
    for (int c = t; c < HD * 8; c += threads) {
      u32x4* p = reinterpret_cast<u32x4*>(sv + 16 * c);
      u32x4 x = *p;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = tame<true>(x[i]);
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
    scores(kf, sc, [](auto) {});
  }
  // step(st) after the products of step st
  template <int H, class F>
  __device__ __forceinline__ void scores(const u32x4 (&kf)[H][L::QS], f32x16 (&sc)[H], F&& step) const {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[h][i] = 0.f;
    static_for<L::QS>([&](auto st) {
#pragma unroll
      for (int h = 0; h < H; ++h)
        sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[h][st]),
                                                        __builtin_bit_cast(bf16x8, qf[st]), sc[h], 0, 0, 0);
      step(st);
    });
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
  // scores of keys that the row does not see (bit: key of the block)
  template <int H>
  __device__ __forceinline__ static void hide(f32x16 (&sc)[H], uint64_t seen) {
    const int f = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const uint32_t bits = uint32_t(seen >> (32 * h)) >> (8 * f);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(bits >> (16 * (i >> 3) + (i & 7)) & 1)) sc[h][i] = -INFINITY;
    }
  }
  // What the products left out (see trees): infinite values and NaN among keys
  // k0 .., 32 of every `step`, that row i of entry b sees, straight from memory.
  __device__ __forceinline__ void bring_wild(const PagedAttn& a, const typename L::Copier& keys, const Share& w, int b,
                                             int i, int root, int end, int k0, int step) {
    const int fr = threadIdx.x & 31, f = (threadIdx.x >> 5) & 1, pmask = a.p.page_len - 1;
    for (; k0 < w.k1; k0 += step) {
      const uint32_t seen = uint32_t(seen_of(a, b, i, root, end, k0));
#pragma unroll
      for (int db = 0; db < L::NDB; ++db) {
        f32x16 up, down;
#pragma unroll
        for (int e = 0; e < 16; ++e) up[e] = down[e] = 0.f;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const int page = keys.in_pool(w.page(k0 + 16 * st, keys.shift, keys.last_block));
          const u32x4 v = *reinterpret_cast<const u32x4*>(keys.V + page * keys.page_bytes +
                                                          ((k0 + 16 * st + 8 * f) & pmask) * 2 +
                                                          size_t(32 * db + fr) * (a.p.page_len * 2));
          u32x4 wu, wd;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const Wild y = wild_of<true>(v[x]);
            wu[x] = y.up;
            wd[x] = y.down;
          }
          const half8 sees = __builtin_bit_cast(half8, ones_of<true>(seen >> (16 * st + 8 * f)));
          up = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, wu), sees, up, 0, 0, 0);
          down = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, wd), sees, down, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] += wild_sum(up[e] > 0.f, down[e] > 0.f);
      }
    }
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
// positions, as it was then: 320 us, 0.79 PFLOP/s): eight waves and 256 rows with three tiles on
// their way, whose copies are half as many a row; the same in two groups that
// take turns at matrix and vector work.  64 rows a wave, alone on its SIMD with
// products and softmax in one stream, took 350.
template <int HD, bool TREE>
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
    const Entry entry = TREE ? w.e : entry_of(a, at.b);
    const bool idle = w.row0 + 32 * wave >= w.row_end;   // none of the wave's rows is there: it only copies
    const int lim_row = limit_of(a, entry, at.i), lim = min(lim_row, w.k1);
    const int root = TREE ? __builtin_amdgcn_readfirstlane(entry.held - entry.rows) : 0;   // the tree's first position

    typename L::Ids id = copier.pages_at(w, w.k0);
    if (w.k0 < w.k1) copier.issue(w.k0, id, lds0);
    id = copier.pages_at(w, w.k0 + kTile);
    int slot = 0;
    bool any_wild = false;
    for (int k0 = w.k0; k0 < w.k1; k0 += kTile, slot ^= 1) {
      const bool masked = TREE && k0 + kTile > root;
      MaskWords words{};
      if (masked) words = mask_words(a, at.b, at.i, root, k0);
      wait_vmcnt<0>();
      barrier_lds();   // tile k0 has landed; the other slot has been read
      const uint8_t* sk = smem + slot * L::BYTES;
      uint8_t* sv = smem + slot * L::BYTES + L::KB;
      if (masked) {
        if (__syncthreads_or(L::tidy_values(sv, tid, w.k1 - k0))) {
          any_wild = true;
          L::tame_values(sv, tid, kThreads);
          __syncthreads();
        }
      } else if (k0 + kTile > w.k1) {
        L::zero_values(sv, tid, kThreads, w.k1 - k0);
        barrier_lds();
      }
      const bool more = k0 + kTile < w.k1;
      const uint32_t next = lds0 + (slot ^ 1) * L::BYTES;
      const uint64_t seen = masked ? seen_in(words, root, lim, k0) : 0;
      if (idle) {
        if (more) {
          copier.issue(k0 + kTile, id, next);
          id = copier.pages_at(w, k0 + 2 * kTile);
        }
        continue;
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
      if (more) {
        rows.scores(kf, sc, [&](auto st) { copier.template issue_one<st>(k0 + kTile, id, next); });
        id = copier.pages_at(w, k0 + 2 * kTile);
      } else {
        rows.scores(kf, sc);
      }
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) vf[st][db] = L::value_chunk(sv, st, db, lane);
      __builtin_amdgcn_sched_barrier(0);
      if (masked) Rows32<HD>::hide(sc, seen);
      rows.softmax(sc, k0, masked ? INT_MAX : lim, j.scale_log2, pf);
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
    if (TREE && any_wild)   // from the first tile that held keys of the tree
      rows.bring_wild(a, copier, w, at.b, at.i, root, lim, w.k0 + max(root - w.k0, 0) / kTile * kTile, 32);
    const float l = pair_sum(rows.l);
    const bool any = TREE ? l != 0.f : lim_row > 0;   // the row sees a position
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
          store_f(out + 32 * db + 8 * (i >> 2) + 4 * f + (i & 3), any ? rows.o[db][i] * inv : 0.f);
    } else {
      float* rec = record_of(j, w, at, w.head, HD);
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

// ---------------------------------------------------------------- halves

// 33 to 64 rows of a tree over one range of keys: wave w takes block w % 2 of 32
// rows and half w / 2 of every tile's keys, so that no wave is without rows; the
// two states of a block are joined through LDS.  Bound as wide is, by a wave's
// products, softmax and fragment reads in turn: a tile takes 0.95 us alone on a
// CU where wide takes 1.45 (32 heads on 8 key heads of 128, 16 x 16 rows over 100
// to 1500 positions: 25.1 us, 27.2 wide).
template <int HD>
struct Halves {
  using L = Tile<HD>;
  using Copier = typename L::Copier;
  static constexpr int RING = 2 * L::BYTES;
  static constexpr int OWN = L::NDB / 2;            // dim blocks that a wave writes, after it has the other's
  static constexpr int STATE = OWN * 16 + 2;        // floats a lane hands over
  static constexpr int JOIN = kWaves * STATE * kWave * 4;
  static constexpr int SMEM = RING > JOIN ? RING : JOIN;

  __device__ static void run(const Job& j, const Share& w, uint8_t* smem) {
    const PagedAttn& a = j.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, f = lane >> 5, block = wave & 1, half = wave >> 1;
    const uint32_t lds0 = lds_address(smem);
    const Copier copier(a, w.head, wave, w.k1);
    typename L::Ids id = copier.pages_at(w, w.k0);
    if (w.k0 < w.k1) copier.issue(w.k0, id, lds0);
    id = copier.pages_at(w, w.k0 + kTile);

    const RowAt at = row_at(j, min(w.row0 + 32 * block + fr, w.row_end - 1));
    Rows32<HD> rows;
    rows.load_q(static_cast<const bf16_t*>(a.q.p) + at.b * a.q.seq + at.i * a.q.row +
                (w.head * j.group + at.g) * a.q.head);
    rows.begin();
    const int root = w.e.held - w.e.rows;   // the tree's first position

    int slot = 0;
    bool any_wild = false;
    for (int k0 = w.k0; k0 < w.k1; k0 += kTile, slot ^= 1) {
      const int keys = k0 + 32 * half;
      const bool masked = k0 + kTile > root;
      MaskWords words{};
      if (masked) words = mask_words(a, at.b, at.i, root, keys);
      wait_vmcnt<0>();
      barrier_lds();   // tile k0 has landed; the other slot has been read
      const uint8_t* sk = smem + slot * L::BYTES;
      uint8_t* sv = smem + slot * L::BYTES + L::KB;
      if (masked) {
        if (__syncthreads_or(L::tidy_values(sv, tid, w.k1 - k0))) {
          any_wild = true;
          L::tame_values(sv, tid, kThreads);
          __syncthreads();
        }
      } else if (k0 + kTile > w.k1) {
        L::zero_values(sv, tid, kThreads, w.k1 - k0);
        barrier_lds();
      }
      const bool more = k0 + kTile < w.k1;
      const uint32_t next = lds0 + (slot ^ 1) * L::BYTES;
      u32x4 kf[1][L::QS], vf[2][L::NDB], pf[2];
      f32x16 sc[1];
#pragma unroll
      for (int st = 0; st < L::QS; ++st) kf[0][st] = L::key_chunk(sk, half, st, lane);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) vf[st][db] = L::value_chunk(sv, 2 * half + st, db, lane);
      __builtin_amdgcn_sched_barrier(0);
      if (more) {
        rows.scores(kf, sc, [&](auto st) { copier.template issue_one<st>(k0 + kTile, id, next); });
        id = copier.pages_at(w, k0 + 2 * kTile);
      } else {
        rows.scores(kf, sc);
      }
      if (masked) Rows32<HD>::hide(sc, seen_in(words, root, w.k1, keys));
      rows.softmax(sc, keys, masked ? INT_MAX : w.k1, j.scale_log2, pf);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) rows.add(db, vf[st][db], pf[st]);
    }
    if (any_wild)   // from the first tile that held keys of the tree
      rows.bring_wild(a, copier, w, at.b, at.i, root, w.k1, w.k0 + max(root - w.k0, 0) / kTile * kTile + 32 * half, kTile);

    // the other half's state of the dim blocks that this wave writes
    float* xs = reinterpret_cast<float*>(smem) + lane;
    const float lsum = pair_sum(rows.l);
    __syncthreads();   // the ring has been read
    float* mine = xs + wave * (STATE * kWave);
#pragma unroll
    for (int c = 0; c < OWN * 16; ++c)
      mine[c * kWave] = half ? rows.o[c >> 4][c & 15] : rows.o[OWN + (c >> 4)][c & 15];
    mine[(STATE - 2) * kWave] = rows.m;
    mine[(STATE - 1) * kWave] = lsum;
    __syncthreads();
    const float* other = xs + (wave ^ 2) * (STATE * kWave);
    const float m1 = other[(STATE - 2) * kWave], top = fmaxf(rows.m, m1), ref = top == -INFINITY ? 0.f : top;
    const float w0 = __builtin_amdgcn_exp2f(rows.m - ref), w1 = __builtin_amdgcn_exp2f(m1 - ref);
    const float l = lsum * w0 + other[(STATE - 1) * kWave] * w1, inv = 1.f / l;
    if (w.row0 + 32 * block + fr >= w.row_end || at.i >= w.e.rows) return;
    bf16_t* out = static_cast<bf16_t*>(a.out.p) + at.b * a.out.seq + at.i * a.out.row + (w.head * j.group + at.g) * a.out.head;
    float* rec = record_of(j, w, at, w.head, HD);
#pragma unroll
    for (int c = 0; c < OWN * 16; c += 4) {
      f32x4 y;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        y[u] = (half ? rows.o[OWN + (c >> 4)][(c & 15) + u] : rows.o[c >> 4][(c & 15) + u]) * w0 + other[(c + u) * kWave] * w1;
      const int dim = 32 * (half * OWN + (c >> 4)) + 2 * (c & 15) + 4 * f;
      if (j.direct) {
#pragma unroll
        for (int u = 0; u < 4; ++u) store_f(out + dim + u, l != 0.f ? y[u] * inv : 0.f);
      } else {
        *reinterpret_cast<f32x4*>(rec + dim) = y;
      }
    }
    if (!j.direct && half == 0 && f == 0) {
      rec[HD] = top;
      rec[HD + 1] = l;
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
template <int HD, bool TREE>
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
    const int own_from = __builtin_amdgcn_readfirstlane(stacked_of<TREE>(e, s, kKeys));
    tail.split = s;
    tail.before = prefix.before;
    tail.after = table_row(a, __builtin_amdgcn_readfirstlane(max(e.seq, 0)));
    const typename L::Copier copier(a, head, wave & 3, s), own_keys(a, head, 0, e.held);
    const int first = kTile * tile;   // of this wave's tile in a step
    const uint32_t lds0 = lds_address(smem) + tile * L::BYTES;
    typename L::Ids id = copier.pages_at(prefix, first);
    if (s > 0) copier.issue(first, id, lds0);
    id = copier.pages_at(prefix, first + kKeys);

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
        id = copier.pages_at(prefix, k0 + 2 * kKeys + first);
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
    const int root = __builtin_amdgcn_readfirstlane(e.held - e.rows);   // the tree's first position
    bool any_wild = false;
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
      const bool masked = TREE && k0 + 32 > root;
      const uint64_t seen = masked ? seen_of(a, b, i, root, limit, k0) : 0;
      rows.scores(kf, sc);
      if (masked) {
        Rows32<HD>::hide(sc, seen);
        uint32_t wild = 0;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int db = 0; db < L::NDB; ++db)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              wild |= wild_bits<true>(vf[st][db][c]);
              vf[st][db][c] = tame<true>(vf[st][db][c]);
            }
        any_wild = any_wild || __any(wild);
      }
      rows.softmax(sc, k0, masked ? INT_MAX : limit, j.scale_log2, pf);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < L::NDB; ++db) rows.add(db, vf[st][db], pf[st]);
    }
    if (TREE && any_wild) {   // from this way's first step that held keys of the tree
      tail.k1 = e.held;
      const int first_own = own_from + 32 * way, steps = max(root - first_own - 31 + kKeys - 1, 0) / kKeys;
      rows.bring_wild(a, own_keys, tail, b, i, root, limit, first_own + steps * kKeys, kKeys);
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
      const bool any = TREE ? l != 0.f : limit > 0;   // the row sees a position
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
            store_f(out + 32 * (d2 + (c0 >> 4)) + 2 * (c0 & 15) + 4 * f + u, any ? y[u] * inv : 0.f);
        }
      }
    }
  }
};

template <int HD, bool TREE>
__global__ __launch_bounds__((Pairs<HD, TREE>::kPairThreads), 2) void pairs_kernel(Job j) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[Pairs<HD, TREE>::SMEM];
  Pairs<HD, TREE>::run(j, blockIdx.x, smem);
}

// ---------------------------------------------------------------- launch

// how a part's rows are taken: 16 or 32 of them narrow, 64 in halves (tails of trees), or 128 wide
enum { ROWS16 = 1, ROWS32 = 2, ROWS128 = 3, ROWS64 = 4 };
constexpr int rows_of(int mode) { return mode == ROWS16 ? 16 : mode == ROWS32 ? 32 : mode == ROWS64 ? 64 : 128; }

template <typename T, int HD, int MODE, bool TREE> struct Taker;
template <typename T, int HD, bool TREE> struct Taker<T, HD, ROWS16, TREE> : Narrow<T, HD, 1, TREE> {};
template <typename T, int HD, bool TREE> struct Taker<T, HD, ROWS32, TREE> : Narrow<T, HD, 2, TREE> {};
template <int HD, bool TREE> struct Taker<bf16_t, HD, ROWS128, TREE> : Wide<HD, TREE> {};
template <int HD> struct Taker<bf16_t, HD, ROWS64, true> : Halves<HD> {};

// both parts in one launch: prefix workgroups, then the tails' (trees are in those alone)
template <typename T, int HD, int PREFIX, int TAIL, bool TREE>
__global__ __launch_bounds__(kThreads, 2) void attention_kernel(Job j) {
  using P = Taker<T, HD, PREFIX, false>;
  using U = Taker<T, HD, TAIL, TREE>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[P::SMEM > U::SMEM ? P::SMEM : U::SMEM];
  Share w;
  const int x = blockIdx.x, prefix = prefix_blocks(j);
  if (x < prefix) {
    if (share_of<TREE>(j, x, true, rows_of(PREFIX), w)) P::run(j, w, smem);
  } else {
    if (share_of<TREE>(j, x - prefix, false, rows_of(TAIL), w)) U::run(j, w, smem);
  }
}

// ---------------------------------------------------------------- merge

// out[row] = sum_r o_r 2^(m_r - m) / sum_r l_r 2^(m_r - m) over the ranges that
// hold positions the row sees; HD / 4 lanes a row and slice, slice c takes the
// ranges c, c + slices, .., and the slices are joined in order.
template <typename T, int HD, bool TREE>
__global__ __launch_bounds__(kThreads) void join_kernel(Job j) {
  constexpr int kLanes = HD / 4;
  __shared__ __attribute__((aligned(16))) float part[kThreads / kLanes][HD + 4];
  const PagedAttn& a = j.a;
  const int slices = j.slices, group = int(threadIdx.x) / kLanes, c = int(threadIdx.x) % kLanes * 4, slice = group % slices;
  const int rows = kThreads / kLanes / slices, row = blockIdx.x * rows + group / slices;
  const bool in = row < a.n * a.max_rows * a.heads;
  const int h = row % a.heads, t = row / a.heads, b = in ? t / a.max_rows : 0, i = t % a.max_rows;
  const Entry e = entry_of(a, b);
  const bool live = in && i < e.rows;
  const int s = j.stacked ? stacked_of<TREE>(e, shared_of(a), j.prefix.range) : 0, lim = limit_of(a, e, i);
  const int np = live && j.prefix.ranges ? (min(lim, s) + j.prefix.range - 1) / j.prefix.range : 0;
  int nt = live && lim > s ? min((lim - s + j.tail.range - 1) / j.tail.range, j.tail.ranges) : 0;
  const size_t stride = size_t(a.n) * a.max_rows * a.heads * record(HD);
  const float* rec = a.part + size_t(row) * record(HD);
  // the tail's records: one after another like the prefix's, or slots of an entry's rows
  const float* tails = rec + j.prefix.ranges * stride;
  size_t tail_stride = stride;
  if (TREE && j.slots) {
    const Slots z = slots_of<TREE>(j, shared_of(a));
    const int count = __shfl(z.count, b, kWave), first = __shfl(z.first, b, kWave);
    nt = live ? count : 0;
    tail_stride = size_t(a.max_rows) * a.heads * record(HD);
    tails += (int64_t(first) - b) * int64_t(tail_stride);
  }
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
      const float* x = !TREE ? rec + (r < np ? r : j.prefix.ranges + r - np) * stride
                             : r < np ? rec + r * stride : tails + (r - np) * tail_stride;
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
  for (int x = 0; x < 4; ++x) store_f(out + x, (TREE ? l != 0.f : lim > 0) ? o[x] / l : 0.f);
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

template <typename T, int HD, int PREFIX, int TAIL, bool TREE>
void launch_parts(const Job& j, hipStream_t s) {
  const int kvh = j.a.p.n_kv_heads;
  const int tail = blocks_of((j.slots ? j.slots : j.a.n * j.tail.ranges) * kvh, j.tail.row_tiles);
  hipLaunchKernelGGL((attention_kernel<T, HD, PREFIX, TAIL, TREE>), dim3(prefix_blocks(j) + tail), dim3(kThreads), 0, s, j);
}

// (a prefix never takes fewer rows than the tails, see divide)
template <typename T, int HD, bool TREE>
void launch_modes(const Job& j, int prefix, int tail, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if constexpr (TREE) {
      if (tail == ROWS64) return launch_parts<T, HD, ROWS128, ROWS64, TREE>(j, s);
    }
    if (tail == ROWS128) return launch_parts<T, HD, ROWS128, ROWS128, TREE>(j, s);
    if (prefix == ROWS128)
      return tail == ROWS32 ? launch_parts<T, HD, ROWS128, ROWS32, TREE>(j, s) : launch_parts<T, HD, ROWS128, ROWS16, TREE>(j, s);
  }
  if (tail == ROWS32) return launch_parts<T, HD, ROWS32, ROWS32, TREE>(j, s);
  return prefix == ROWS32 ? launch_parts<T, HD, ROWS32, ROWS16, TREE>(j, s) : launch_parts<T, HD, ROWS16, ROWS16, TREE>(j, s);
}

template <typename T, int HD, bool TREE>
void launch(Job& j, int prefix, int tail, hipStream_t s) {
  launch_modes<T, HD, TREE>(j, prefix, tail, s);
  if (j.direct) return;
  // rows of many ranges take several groups of lanes each: the records of a
  // row come in turn, four at a time
  constexpr int kGroups = kThreads / (HD / 4);
  const int ranges = j.prefix.ranges + (j.slots ? cdiv(j.slots, j.a.n) : j.tail.ranges);
  j.slices = ranges <= 4 ? 1 : ranges <= 8 ? 2 : ranges <= 16 ? 4 : 8;
  hipLaunchKernelGGL((join_kernel<T, HD, TREE>), dim3(cdiv(j.a.n * j.a.max_rows * j.a.heads, kGroups / j.slices)),
                     dim3(kThreads), 0, s, j);
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
  return std::ceil(all / (2 * kCus)) * (4.8 + u * (3.4 + (1.45 * shared + 3.5 * tail) / Pairs<128, false>::kKeys));
}

// how a call is taken: pairs, or a prefix (stacked) and tails
struct Division {
  bool pairs, stacked;
  int mode_p, mode_t;
  Part prefix, tail;
  int slots;        // of a tree's tails, as in Job
  int64_t shared;   // whole pages of the prefix, as far as the caller knows
};

// More than 32 rows of a tree over keys of their own: in halves or wide, and in
// how many slots.  Not divided, or as many as give each CU one or two
// workgroups, by the least estimated time: 2.5 us and, for every round of two
// workgroups a CU, 4 and what a tile of 64 keys of heads of 128 takes, 1.45 wide
// and 0.95 in halves alone on a CU, 2.3 and 1.75 where two share it, or what the keys
// take from memory; 4 more and the records at 5 TB/s where they are joined.  (A slot
// is of one entry, so that on average half a slot of each is left out.)  Measured, us, 32 heads, wide not
// divided / one a CU / two / halves not divided: 12 x 43 rows of 8 key heads
// over 480 positions 19.4 / 29.8 / 29.8 / 19.9, 4 x 100 over 3000 69 / 45 / 44 / 49, 1 x
// 64 over 2000 49 / 20.1 / 20.1 / 35 (halves, one a CU: 18.0), 16 x 24 over 1000 to 3500
// 77 / 49 / 44 / 64, 9 x 28 over 6100 130 / 58 / 53 / 89; 32 key heads, 8 x 75 over 990
// 29 / 29 / 38 / 32; 32 heads of 64, 8 x 60 over 1500 23.7 (halves not divided), 26.4 (two a CU);
// 32 key heads, 4 x 64 over 4000 to 8000 in halves 101 (one a CU), 89 (two).
struct TreeTail {
  int mode, slots;
  double us;
};
// (keys: the longest entry's, theirs on average, and all that are read, a shared prefix once)
TreeTail plan_tree(const PagedAttn& a, int rows, double longest, double mean, double once) {
  const int kvh = a.p.n_kv_heads;
  const int64_t most = a.n <= kWave ? a.n * most_ranges(ROWS128, int64_t(cdiv(rows, rows_of(ROWS128))) * a.n * kvh) : a.n;
  const double u = a.p.head_dim == 128 ? 1.0 : 0.55;
  TreeTail best{ROWS128, a.n, 1e30};
  for (int mode : {ROWS64, ROWS128}) {
    const int per_slot = cdiv(rows, rows_of(mode)) * kvh;
    for (int wgs : {0, kCus, 2 * kCus}) {
      const int slots = int(std::min<int64_t>(std::max(a.n, wgs / per_slot), most));
      const bool divided = slots > a.n;
      if (wgs && !divided) continue;
      const double all = double(slots) * per_slot, rounds = std::max(1.0, all / (2 * kCus));
      const double tile = u * (mode == ROWS64 ? (all > kCus ? 1.75 : 0.95) : (all > kCus ? 2.3 : 1.45));
      const double tiles = divided ? std::max(4.0, a.n * mean / kTile / (slots - 0.5 * a.n)) : longest / kTile;
      // (keys and values from memory: 4.5 TB/s with one workgroup a CU, 5.5 with two)
      const double memory = once * kvh * a.p.head_dim * 4 / (all > kCus ? 5.5e6 : 4.5e6);
      const double us = 2.5 + rounds * 4.0 + std::max(rounds * tiles * tile, memory) +
                        (divided ? 4.0 + double(slots) * a.max_rows * a.heads * 2 * record(a.p.head_dim) * sizeof(float) / 5e6 : 0.0);
      if (us < best.us) best = TreeTail{mode, slots, us};
    }
  }
  return best;
}

Division divide(const PagedAttn& a, bool tree) {
  Division d{};
  const int dt = a.p.dtype, kvh = a.p.n_kv_heads, group = a.heads / kvh;
  const int64_t most = int64_t(a.p.max_blocks) * a.p.page_len;
  const int64_t shared = d.shared = std::min<int64_t>(a.shared_len, most) / a.p.page_len * a.p.page_len;
  const int rows_t = a.max_rows * group, rows_p = a.n * rows_t;
  const int64_t keys = std::max<int64_t>(1, std::min<int64_t>(a.max_len, most));
  d.mode_p = d.mode_t = mode_of(dt, rows_t, a.n, kvh);
  // fp32 rows of trees that leave much of the last 32 empty are taken 16 at a time: the
  // products bound them (16 key heads of 64, 26 x 72 rows over 97 positions 31.5 us, 32
  // at a time 36.9; 32 key heads, 12 x 48 over 1100 82.7 and 93.5; 16 x 33 over 1060 54
  // and 55; but 32 x 32 over 400 37.6 and 30.8)
  if (tree && dt == DLLM_F32 && d.mode_t == ROWS32 && cdiv(rows_t, 16) * 16 * 1.1 < cdiv(rows_t, 32) * 32)
    d.mode_p = d.mode_t = ROWS16;
  // lengths of the tails: the longest, and half of it on average
  const int64_t longest = std::max<int64_t>(1, keys - shared);
  const double mean = std::max<int64_t>(0, keys - shared) / 2.0;
  d.prefix = Part{1, 0, kTile};
  d.tail = plan_part(d.mode_t, rows_t, a.n, kvh, std::max(keys, shared));
  // (the slots of entries that are divided evenly)
  auto even = [&] { d.slots = tree && a.n <= kWave && d.tail.ranges > 1 ? a.n * d.tail.ranges : 0; };
  const bool wide_tree = tree && d.mode_t == ROWS128;
  double own = 0.0;
  if (wide_tree) {
    const TreeTail z = plan_tree(a, rows_t, double(std::max(keys, shared)), shared + mean, shared + a.n * mean);
    d.mode_t = z.mode;
    // (slots have lengths of their own)
    d.tail = Part{cdiv(rows_t, rows_of(z.mode)), cdiv(z.slots, a.n),
                  int((std::max(keys, shared) + kTile - 1) / kTile) * kTile};
    d.slots = z.slots > a.n ? z.slots : 0;
    own = z.us;
  } else {
    even();
  }
  if (shared == 0) return d;
  const Cost none{0, 0};
  if (!wide_tree) own = parts_us(a, d.mode_t, cost_of(a, d.mode_t, d.tail, a.n, shared + mean), none, d.tail.ranges);
  const TreeTail alone{d.mode_t, d.slots, own};
  if (wide_tree) d.mode_t = ROWS128;
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
    even();
    if (wide_tree && rows_t <= rows_of(ROWS64)) d.mode_t = ROWS64;
  } else {
    d.mode_t = alone.mode;
  }
  return d;
}

}  // namespace

namespace {

template <bool TREE>
hipError_t attend(const PagedAttn& a, hipStream_t s) {
  Job j{};
  j.a = a;
  j.scale_log2 = a.scale * 1.4426950408889634f;
  // positions of a sequence: up to 2^30
  j.weight = 0x1p-8f;
  for (int64_t most = 1; most < int64_t(a.p.max_blocks) * a.p.page_len; most *= 2) j.weight *= 0.5f;
  j.group = a.heads / a.p.n_kv_heads;
  const Division d = divide(a, TREE);
  const int kvh = a.p.n_kv_heads, hd = a.p.head_dim;
  if (d.pairs) {
    j.direct = true;
    const int grid = blocks_of(kvh, cdiv(a.n * cdiv(a.max_rows * j.group, 32), 2));
    constexpr int kPairThreads = Pairs<128, TREE>::kPairThreads;
    if (hd == 128) hipLaunchKernelGGL((pairs_kernel<128, TREE>), dim3(grid), dim3(kPairThreads), 0, s, j);
    else hipLaunchKernelGGL((pairs_kernel<64, TREE>), dim3(grid), dim3(kPairThreads), 0, s, j);
    return hipGetLastError();
  }
  j.prefix = d.prefix;
  j.tail = d.tail;
  j.stacked = d.stacked;
  if (d.shared == 0) j.a.shared_len = j.a.prefix_seq = 0;
  j.direct = j.prefix.ranges + j.tail.ranges == 1;
  j.slots = d.slots;
  if (a.p.dtype == DLLM_BF16)
    hd == 128 ? launch<bf16_t, 128, TREE>(j, d.mode_p, d.mode_t, s) : launch<bf16_t, 64, TREE>(j, d.mode_p, d.mode_t, s);
  else
    hd == 128 ? launch<float, 128, TREE>(j, d.mode_p, d.mode_t, s) : launch<float, 64, TREE>(j, d.mode_p, d.mode_t, s);
  return hipGetLastError();
}

}  // namespace

hipError_t paged_attention(const PagedAttn& a, hipStream_t s) { return a.mask ? attend<true>(a, s) : attend<false>(a, s); }

kv_attention_plan paged_attention_plan(const PagedAttn& a, bool tree) {
  const Division d = divide(a, tree);
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
  p.tail_keys = d.slots ? 0 : d.tail.range;
  return p;
}

}  // namespace dllm
