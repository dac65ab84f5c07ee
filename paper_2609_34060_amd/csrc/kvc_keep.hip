// Accepted tokens' rows to their places in the cache (kvc_keep).
//
// A wave moves 16 bytes a lane of a token's rows (of one layer, K or V), one accepted token of the sequence after the other:
// a path ascends, so a token comes from its own place or from behind it, and whatever a lane overwrites, that lane has read
// before.  Moves are latency: lengths, path, table and rows one after the other, eight rows in flight; 3.4 us for one request
// and 6.0 for 64, two rows to move, 32 layers of 8 heads of 128.
#include <algorithm>

#include "kvc_drafts.h"

namespace kvc {
namespace {

constexpr int kKeepThreads = 256;
constexpr int kFewLayers = 4;  // (more pointers in the arguments: a longer launch)

// CACHE: kvc_dtype.  One wave: 64 of the pieces (head, part of a row) of a sequence's rows.
template <int D, int CACHE, int LAYERS>
__global__ __launch_bounds__(kKeepThreads) void keep_rows(KeepArgs a, RowsLayers<LAYERS> at, int pieces) {
  constexpr int ES = CACHE == KVC_I8 ? 1 : CACHE == KVC_BF16 ? 2 : 4;
  constexpr int LPR = D * ES / 16;  // lanes of a row
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & (kWave - 1);
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kKeepThreads / kWave) + threadIdx.x / kWave);
  const int layer = blockIdx.z, kv = blockIdx.y;
  const int seq = a.seq0 + unit / pieces, piece = unit % pieces * kWave + lane;
  if (seq >= a.step.num_seqs) return;
  const int counted = a.counts[seq];
  const SeqView sq = step_seq(a.step, seq);
  if (!sq.ok) return;
  const int head = piece / LPR, part = piece % LPR;
  const bool mine = head < a.pv.num_kv_heads;
  const int count = min(counted, sq.q), base = sq.ctx - sq.q;
  const int32_t* table = a.step.tables ? a.step.tables + (int64_t)seq * a.step.max_blocks : nullptr;
  char* rows = static_cast<char*>(at.pools[kv][layer]) + (mine ? head : 0) * a.pv.head_bytes + part * 16;
  char* scales = nullptr;
  if constexpr (CACHE == KVC_I8)
    scales = reinterpret_cast<char*>(at.scales[kv][layer]) + (mine ? head : 0) * a.pv.shead_bytes;
  int before = -1;  // the path's token before these 64
  for (int d0 = 0; d0 < count; d0 += kWave) {
    const int d = d0 + lane;
    const int come = d < count ? a.path[(int64_t)sq.start + d] : INT32_MAX;
    const int prev = __shfl_up(come, 1, kWave);
    const bool good = d < count && come > (lane ? prev : before) && come < sq.q;
    const uint64_t bad = __ballot(!good);
    const int here = bad ? __builtin_ctzll(bad) : kWave;  // tokens of the path among these
    // this lane's token: where it comes from, and where it goes
    int32_t from_slot = 0, to_slot = 0, from = -1, to = -1;
    if (lane < here && come != d && base + d >= 0) {
      from = step_block(a.pv, table, sq.off + base + come, from_slot);
      to = step_block(a.pv, table, sq.off + base + d, to_slot);
    }
    uint64_t moves = __ballot(from >= 0 && to >= 0);
    while (moves) {
      u32x4 x[AHEAD];
      float s[AHEAD];
      uint64_t left = moves;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (!left) break;
        const int j = __builtin_ctzll(left);
        left &= left - 1;
        const int blk = __builtin_amdgcn_readlane(from, j), slot = __builtin_amdgcn_readlane(from_slot, j);
        if (mine) x[i] = *reinterpret_cast<const u32x4*>(rows + slot_bytes(a.pv, blk, slot));
        if constexpr (CACHE == KVC_I8)
          if (mine && part == 0) s[i] = *reinterpret_cast<const float*>(scales + slot_scale_bytes(a.pv, blk, slot));
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (!moves) break;
        const int j = __builtin_ctzll(moves);
        moves &= moves - 1;
        const int blk = __builtin_amdgcn_readlane(to, j), slot = __builtin_amdgcn_readlane(to_slot, j);
        if (mine) *reinterpret_cast<u32x4*>(rows + slot_bytes(a.pv, blk, slot)) = x[i];
        if constexpr (CACHE == KVC_I8)
          if (mine && part == 0) *reinterpret_cast<float*>(scales + slot_scale_bytes(a.pv, blk, slot)) = s[i];
      }
    }
    if (here < kWave) return;
    before = __builtin_amdgcn_readlane(come, kWave - 1);
  }
}

template <int D, int CACHE>
hipError_t launch(KeepArgs a, const RowsLayers<kRowsLayers>& layers, hipStream_t stream) {
  constexpr int LPR = D * (CACHE == KVC_I8 ? 1 : CACHE == KVC_BF16 ? 2 : 4) / 16, WAVES = kKeepThreads / kWave;
  const int pieces = (a.pv.num_kv_heads * LPR + kWave - 1) / kWave;
  const int32_t most = (1 << 24) / pieces;  // sequences of a launch (a grid's dimension ends at 2^32 threads)
  const bool by_few = a.num_layers <= kFewLayers;
  RowsLayers<kFewLayers> few = {};
  if (by_few) {
    for (int kv = 0; kv < 2; ++kv) {
      for (int l = 0; l < a.num_layers; ++l) {
        few.pools[kv][l] = layers.pools[kv][l];
        few.scales[kv][l] = CACHE == KVC_I8 ? layers.scales[kv][l] : nullptr;
      }
    }
  }
  for (int32_t first = 0; first < a.step.num_seqs; first += most) {
    a.seq0 = first;
    const int64_t units = (int64_t)std::min(most, a.step.num_seqs - first) * pieces;
    const dim3 grid((unsigned)((units + WAVES - 1) / WAVES), 2, a.num_layers);
    if (by_few) keep_rows<D, CACHE, kFewLayers><<<grid, kKeepThreads, 0, stream>>>(a, few, pieces);
    else keep_rows<D, CACHE, kRowsLayers><<<grid, kKeepThreads, 0, stream>>>(a, layers, pieces);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_types(const KeepArgs& a, const RowsLayers<kRowsLayers>& layers, kvc_dtype cache, hipStream_t stream) {
  if (cache == KVC_F32) return launch<D, KVC_F32>(a, layers, stream);
  return cache == KVC_BF16 ? launch<D, KVC_BF16>(a, layers, stream) : launch<D, KVC_I8>(a, layers, stream);
}

}  // namespace

hipError_t launch_keep(const KeepArgs& a, const RowsLayers<kRowsLayers>& layers, kvc_dtype cache, int head_dim,
                       hipStream_t stream) {
  if (a.step.num_rows == 0 || a.num_layers == 0) return hipSuccess;
  return head_dim == 64 ? launch_types<64>(a, layers, cache, stream) : launch_types<128>(a, layers, cache, stream);
}

}  // namespace kvc
