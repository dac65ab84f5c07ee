// A served step over the paged cache: launch arguments and device helpers of the append, gather and attention kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvc.h"
#include "kvc_device.h"

namespace kvc {

// What kvc_last_hip_error() tells (kvc_api.cpp).
void set_last_hip_error(hipError_t e);

// x / d = (x * mul) >> shift for 0 <= x < 2^31: with 2^(L-1) < d <= 2^L, mul = floor(2^(31+L) / d) + 1 exceeds the
// quotient by at most 1, so that x times that is below 2^(31+L).
struct Divisor {
  uint32_t mul, shift;
};
inline Divisor divisor(int32_t d) {
  uint32_t log = 0;
  while ((int64_t{1} << log) < d) ++log;
  return {static_cast<uint32_t>((uint64_t{1} << (31 + log)) / static_cast<uint32_t>(d) + 1), 31 + log};
}
__device__ __forceinline__ int32_t quotient(int32_t x, const Divisor& d) {
  return (int32_t)(((uint64_t)(uint32_t)x * d.mul) >> d.shift);
}

// Pools of a cache without its layer pointers (those travel beside it).  Strides in bytes.
struct ServePool {
  uint32_t block_bytes, token_bytes;    // of the rows
  uint32_t sblock_bytes, stoken_bytes;  // of an 8-bit cache's scales
  int64_t head_bytes, shead_bytes;
  int32_t block_size, num_blocks, num_kv_heads;
  Divisor block;  // block_size
};

struct StepView {
  int32_t num_seqs, num_rows, max_new, max_context, max_blocks;
  int64_t capacity;  // positions that a sequence's table row (or the pool) holds, at most 2^31 - 1
  const int32_t* starts;
  const int32_t* contexts;
  const int32_t* offsets;
  const int32_t* tables;
};

// Sequence i of a step, checked against the host's bounds (ok = 0: left out).
struct SeqView {
  int32_t start, q, ctx, off;
  int32_t ok;
};
__device__ __forceinline__ SeqView step_check(const StepView& st, int32_t start, int32_t end, int32_t ctx, int32_t off) {
  const int64_t q = (int64_t)end - start;
  SeqView s = {start, (int32_t)q, ctx, off, 0};
  s.ok = start >= 0 && q >= 0 && end <= st.num_rows && q <= st.max_new && ctx >= 0 && ctx <= st.max_context && off >= 0 &&
         (int64_t)off + ctx <= st.capacity;
  return s;
}
// Sequence i, which every lane of the wave asks for.  Left out as well if an earlier start lies above its own, so that a row
// has one sequence at most however the starts run: the starts before it are looked at, the loads of 2048 in flight together.
// Up to 512 sequences that costs nothing that shows; 1024, 4096 (of 64-512 tokens) and 16384 (of 16-100) take 256, 1002 and
// 2160 us, 252, 951 and 1512 without it, 259, 1061 and 3009 with loads of four bytes.
__device__ __forceinline__ SeqView step_seq(const StepView& st, int i) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4), aligned(4)));
  const int lane = threadIdx.x & (kWave - 1);
  constexpr int AHEAD = 8;
  int32_t top = INT32_MIN;
  if (i <= kWave) {
    if (i > 0) top = st.starts[min(lane, i - 1)];
  } else {
    for (int b = 0; b < i; b += AHEAD * 4 * kWave) {
      i32x4 before[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int at = b + j * 4 * kWave;
        before[j] = i32x4{INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN};
        if (at < i) before[j] = *reinterpret_cast<const i32x4*>(st.starts + min(at + 4 * lane, i - 4));
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, before[j][e]);
    }
  }
  SeqView s = step_check(st, st.starts[i], st.starts[i + 1], st.contexts[i], st.offsets ? st.offsets[i] : 0);
  if (__any(top > s.start)) s.ok = 0;
  return s;
}

// The sequence i with first(start, i) <= x < last(start, end, i), for its starts[i] and starts[i + 1], in s (-1: none), left
// out (s.ok = 0) as in step_seq.  `first` ascends with the start and with i, and no sequence that follows without a descent
// has a `first` below an earlier `last`.  Every lane of the wave calls it with the same x; 64 sequences are looked at at a
// time, with all that is to be known of them, so that nothing is loaded once the one is found.  (A start that lets the search
// end, or takes x for a sequence that is then left out, lies above the starts of the sequences behind it that would hold x:
// these are left out too.)
template <class X, class First, class Last>
__device__ __forceinline__ int step_find(const StepView& st, X x, SeqView& s, First first, Last last) {
  const int lane = threadIdx.x & (kWave - 1);
  int32_t top = INT32_MIN;  // the largest start of this lane's sequences so far
  for (int b = 0; b < st.num_seqs; b += kWave) {
    const int i = min(b + lane, st.num_seqs - 1);
    const int start = st.starts[i], end = st.starts[i + 1], ctx = st.contexts[i], off = st.offsets ? st.offsets[i] : 0;
    const X at = first(start, i);
    const uint64_t held = __ballot(at <= x && x < last(start, end, i));
    if (held) {
      const int j = __builtin_ctzll(held);
      s = step_check(st, __builtin_amdgcn_readlane(start, j), __builtin_amdgcn_readlane(end, j),
                     __builtin_amdgcn_readlane(ctx, j), __builtin_amdgcn_readlane(off, j));
      if (__any(max(top, lane < j ? start : INT32_MIN) > s.start)) s.ok = 0;
      return b + j;
    }
    if (__any(at > x)) break;
    top = max(top, start);
  }
  return -1;
}
// The sequence of token row x.
__device__ __forceinline__ int step_find_row(const StepView& st, int32_t x, SeqView& s) {
  return step_find(
      st, x, s, [](int32_t start, int) { return start; }, [](int32_t, int32_t end, int) { return end; });
}

// Table entry of position p of a sequence, unchecked, and the slot in its block.
__device__ __forceinline__ int32_t step_entry(const ServePool& pv, const int32_t* __restrict__ table, int32_t p,
                                              int32_t& slot) {
  const int32_t lb = quotient(p, pv.block);
  slot = p - lb * pv.block_size;
  return table ? table[lb] : lb;
}
// Physical block of position p, or -1 where the entry lies outside the pool.
__device__ __forceinline__ int32_t step_block(const ServePool& pv, const int32_t* __restrict__ table, int32_t p,
                                              int32_t& slot) {
  const int32_t blk = step_entry(pv, table, p, slot);
  return (uint32_t)blk < (uint32_t)pv.num_blocks ? blk : -1;
}

// Byte offset of a slot's rows (scales) in their pool.
__device__ __forceinline__ int64_t slot_bytes(const ServePool& pv, int32_t blk, int32_t slot) {
  return (int64_t)((uint64_t)(uint32_t)blk * pv.block_bytes + (uint64_t)(uint32_t)slot * pv.token_bytes);
}
__device__ __forceinline__ int64_t slot_scale_bytes(const ServePool& pv, int32_t blk, int32_t slot) {
  return (int64_t)((uint64_t)(uint32_t)blk * pv.sblock_bytes + (uint64_t)(uint32_t)slot * pv.stoken_bytes);
}

// kvc_append / kvc_gather (kvc_rows.hip).
constexpr int kRowsLayers = 64;  // layers of one launch
struct RowsArgs {
  ServePool pv;
  StepView step;
  int32_t num_layers;  // of this launch
  int32_t token0;      // its first token
  char* rows[2];       // K, V
  int64_t layer_stride, token_stride, head_stride;  // of the rows, bytes
};
template <int LAYERS>
struct RowsLayers {
  void* pools[2][LAYERS];    // [K/V][layer]
  float* scales[2][LAYERS];  // (8-bit caches)
};
hipError_t launch_rows(const RowsArgs& a, const RowsLayers<kRowsLayers>& layers, kvc_dtype cache, kvc_dtype rows,
                       int head_dim, bool gather, hipStream_t stream);

// kvc_attend (kvc_attend.hip).
constexpr int kAttendTile = 256;  // most rows of a tile
struct AttendArgs {
  ServePool pv;
  StepView step;
  const void* k;
  const void* v;
  const float* ks;          // scales of an 8-bit cache
  const float* vs;
  const char* q;
  char* out;
  float* lse;
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;  // bytes
  int32_t num_heads, group;  // group: query heads of a KV head
  Divisor by_heads, by_group;
  int32_t causal, window;
  float scale_log2;          // scale * log2(e)
  int32_t direct;            // one tile per sequence (max_new * group <= the tile's rows)
  int32_t splits, chunk;     // key ranges of a row tile, and keys of one
  int32_t tile0;             // first row tile of this launch (a grid's third dimension ends at 65535)
  int32_t flat0;             // first row and head of a join (a grid's first dimension ends at 2^32 threads)
  float* part_o;             // [splits][num_rows * num_heads][head_dim]
  float2* part_ml;           // [splits][num_rows * num_heads]: maximum (log2 units), sum
};
struct AttendPlan {
  int32_t tile_rows, direct, tiles, splits, chunk;
  size_t bytes;       // workspace of this plan
  size_t most_bytes;  // no plan of the same step with a span up to max_span needs more
};
// span: the longest key range that a row tile can see, at most max_span.
AttendPlan plan_attend(kvc_dtype cache, int num_seqs, int num_rows, int max_new, int64_t span, int64_t max_span,
                       int num_kv_heads, int group, int head_dim);
hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, kvc_dtype cache, int head_dim, hipStream_t stream);

}  // namespace kvc
