// Trees of drafted tokens: from each row's parent, the rows that it sees (itself
// and those it follows) as words of bits, and its position.
//
// A thread takes a row and one word of its mask and walks up the tree until it
// is past the word; the thread of word 0 walks to the root and counts.  Parents
// are in LDS.  Bound by that walk's dependent reads, as many as the tree is deep,
// behind a launch: 64 trees of 200 rows 3.2 us, one of 5 1.6, calls of 3.3 to 4;
// a chain of 64 rows 5.4, of 1024 69, 64 of those 286.
#include "common.h"
#include "kernels.h"

namespace dllm {

namespace {

constexpr int kThreads = 256;

__global__ __launch_bounds__(kThreads) void tree_kernel(dllm_kv_pages p, const int32_t* __restrict__ seqs,
                                                        int max_rows, int words, const int32_t* __restrict__ n_rows,
                                                        const int32_t* __restrict__ parent, uint32_t* __restrict__ mask,
                                                        int32_t* __restrict__ pos) {
  __shared__ int up[KV_TREE_MAX_ROWS];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int rows = n_rows ? min(max(n_rows[b], 0), max_rows) : max_rows;
  if (int(blockIdx.x) * kThreads >= rows * words) return;
  for (int i = tid; i < rows; i += kThreads) up[i] = parent[size_t(b) * max_rows + i];
  const int s = seqs[b];
  const int held = s >= 0 && s < p.max_seqs ? min(max(p.len[s], 0), p.max_blocks * p.page_len) : 0;
  __syncthreads();
  const int t = blockIdx.x * kThreads + tid, row = t / words, word = t % words;
  if (row >= rows) return;
  uint32_t bits = 0;
  int i = row, followed = -1;
  while (i >= 32 * word) {   // ends: each step is to a lower row, or out
    if (i < 32 * word + 32) bits |= 1u << (i & 31);
    ++followed;
    const int next = up[i];
    i = next < i ? next : -1;
  }
  const size_t at = size_t(b) * max_rows + row;
  mask[at * words + word] = bits;
  if (pos && word == 0) pos[at] = held - rows + followed;
}

}  // namespace

hipError_t pages_tree(const dllm_kv_pages& p, const int32_t* seqs, int n, int max_rows, const int32_t* n_rows,
                      const int32_t* parent, uint32_t* mask, int32_t* pos, hipStream_t s) {
  const int words = (max_rows + 31) / 32;
  hipLaunchKernelGGL(tree_kernel, dim3(cdiv(max_rows * words, kThreads), n), dim3(kThreads), 0, s, p, seqs, max_rows,
                     words, n_rows, parent, mask, pos);
  return hipGetLastError();
}

}  // namespace dllm
