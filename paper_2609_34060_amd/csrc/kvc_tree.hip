// Drafted tokens' trees (kvc_tree): the ancestors of every new token of a sequence as bits, and its position.
//
// One workgroup a sequence, one thread a token.  A token's line of parents is walked upwards in LDS, a run of tokens that
// each continue the one before them in one stride, so that a chain costs one stride and a tree as many as its line has turns.
// Ancestors stand before their descendants: words are met from the last to the first, and each is written once.
//
// Latency: 2.5 us for eight tokens, 7.2 us for 256 trees of 33-512 tokens (two loads one after the other, the walk,
// 5 MB written).  A thread a word instead, so that masks were written as they lie in memory, walked every line as often as it
// has words: 17 us.
#include <algorithm>

#include "kvc_drafts.h"

namespace kvc {
namespace {

constexpr int kTreeThreads = 512;

__global__ __launch_bounds__(kTreeThreads) void tree_masks(TreeArgs a) {
  __shared__ int32_t parent[KVC_MAX_TREE];
  __shared__ uint64_t breaks[KVC_MAX_TREE / 64];  // bit j: token j does not continue token j - 1
  // The run that token j ends: its first token, and that one's parent plus one (bits 16 ..; all ones: there is none).
  __shared__ uint32_t runs[KVC_MAX_TREE];
  static_assert(KVC_MAX_TREE < 0xffff, "a parent in 16 bits");
  const int seq = a.seq0 + blockIdx.x;
  const SeqView sq = step_seq(a.step, seq);
  if (!sq.ok) return;
  const int q = sq.q;
  for (int j = threadIdx.x; j < (q + kWave - 1) / kWave * kWave; j += kTreeThreads) {
    const int p = j < q ? a.parents[(int64_t)sq.start + j] : -1;
    if (j < q) parent[j] = p;
    const uint64_t b = __ballot(j == 0 || p != j - 1);
    if (j % kWave == 0) breaks[j / kWave] = b;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < q; j += kTreeThreads) {
    int w = j >> 6;
    uint64_t b = breaks[w] & (~0ull >> (63 - (j & 63)));
    while (b == 0) b = breaks[--w];  // (token 0 is one)
    const int r = 64 * w + 63 - __builtin_clzll(b), p = parent[r];
    runs[j] = (uint32_t)r | (uint32_t)(p >= -1 && p < r ? p + 1 : 0xffff) << 16;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < q; j += kTreeThreads) {
    uint64_t* mask = a.masks + ((int64_t)sq.start + j) * a.words;
    int word = j >> 6, line = 0, v = j;
    for (int w = word + 1; w < a.words; ++w) mask[w] = 0;
    uint64_t bits = 0;
    bool good = true;
    while (v >= 0) {
      const uint32_t run = runs[v];
      const int r = run & 0xffff, up = run >> 16;
      line += v - r + 1;
      int to = v;  // the run's tokens, a word at a time
      while (true) {
        const int w = to >> 6;
        while (word > w) {
          mask[word--] = bits;
          bits = 0;
        }
        const int from = max(r, 64 * w);
        bits |= (~0ull >> (63 - (to & 63))) & (~0ull << (from & 63));
        if (from == r) break;
        to = from - 1;
      }
      good = up != 0xffff;
      v = good ? up - 1 : -1;
    }
    for (; word >= 0; --word) {
      mask[word] = bits;
      bits = 0;
    }
    if (!good)
      for (int w = 0; w < a.words; ++w) mask[w] = 0;
    if (a.positions) a.positions[sq.start + j] = good ? sq.ctx - q + line - 1 : -1;
  }
}

}  // namespace

hipError_t launch_tree(TreeArgs a, hipStream_t stream) {
  constexpr int32_t kMost = 1 << 23;  // (a grid's dimension ends at 2^32 threads)
  for (int32_t first = 0; first < a.step.num_seqs; first += kMost) {
    a.seq0 = first;
    tree_masks<<<std::min(kMost, a.step.num_seqs - first), kTreeThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace kvc
