// New tokens' rows into the paged cache (kvc_append) and back (kvc_gather).
//
// A row is one token's key or value of one KV head.  8-bit cache: scale = max|x| / 127, code = rint(x * (127 / max|x|)),
// value = code * scale.  Both directions move each byte once and are bound by HBM.  A lane holds 16 elements of a row (16
// bytes of a row that is only copied), so a token's heads side by side are one or more waves' width, a row's maximum is a
// reduction over head_dim / 16 neighbouring lanes, and a token's place in the cache is the same for the whole wave.  One
// token a wave: the loads in flight come from many waves with few registers.  Two, four and eight tokens a wave, loads
// first, took 309, 321 and 358 us against 299 us for 32 layers x 4096 tokens x 8 heads x 128 written to and read back from
// an 8-bit cache (1.63 GB, 5.4 TB/s), 140, 144 and 161 against 130 us for the reading of 22 K tokens of four layers.
#include <algorithm>

#include "kvc_serve.h"

namespace kvc {
namespace {

constexpr int kRowsThreads = 256;
// The layers' pointers travel in the kernel arguments, and the more of these there are, the longer a launch takes: a small
// call of two layers 5.8 us with room for 64, 5.3 us with room for four, which is what a model's own calls (a layer at a
// time) come with.
constexpr int kFewLayers = 4;

template <bool BF16>
__device__ __forceinline__ void widen(const u32x4& w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = bf16_lo_to_f32(w[i]);
      x[2 * i + 1] = bf16_hi_to_f32(w[i]);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}

// CACHE, ROWS: kvc_dtype.  One wave: 64 of the pieces (head, part of a row) of one token.
template <int D, int CACHE, int ROWS, bool GATHER, int LAYERS>
__global__ __launch_bounds__(kRowsThreads) void serve_rows(RowsArgs a, RowsLayers<LAYERS> at, int pieces) {
  constexpr bool QUANT = CACHE == KVC_I8, RB = ROWS == KVC_BF16;
  constexpr int RE = RB ? 2 : 4;              // bytes of a dense element
  constexpr int CH = QUANT ? 16 : 16 / RE;    // elements of a lane
  constexpr int LPR = D / CH;                 // lanes of a row
  constexpr int NW = CH * RE / 16;            // 16-byte words of a lane's dense elements
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int layer = blockIdx.z, kv = blockIdx.y;
  const int group = blockIdx.x / pieces, piece = (blockIdx.x - group * pieces) * kWave + lane;
  const int head = piece / LPR, part = piece % LPR;
  const int token = a.token0 + group * (kRowsThreads / kWave) + wave;
  if (token >= a.step.num_rows) return;

  SeqView sq;
  const int seq = step_find_row(a.step, token, sq);
  if (seq < 0 || head >= a.pv.num_kv_heads) return;
  const int t = sq.ctx - sq.q + (token - sq.start);
  if (!sq.ok || t < 0) return;
  int32_t slot;
  const int32_t* table = a.step.tables ? a.step.tables + (int64_t)seq * a.step.max_blocks : nullptr;
  const int32_t blk = step_block(a.pv, table, sq.off + t, slot);
  if (blk < 0) return;

  char* row = static_cast<char*>(at.pools[kv][layer]) + slot_bytes(a.pv, blk, slot) + head * a.pv.head_bytes +
              part * (QUANT ? CH : 16);
  char* dense = a.rows[kv] + layer * a.layer_stride + (int64_t)token * a.token_stride + head * a.head_stride +
                part * (CH * RE);
  if constexpr (!QUANT) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(GATHER ? row : dense);
    *reinterpret_cast<u32x4*>(GATHER ? dense : row) = w;
    return;
  }
  float* scale = reinterpret_cast<float*>(reinterpret_cast<char*>(at.scales[kv][layer]) +
                                          slot_scale_bytes(a.pv, blk, slot) + head * a.pv.shead_bytes);
  if constexpr (QUANT && GATHER) {
    const u32x4 c = *reinterpret_cast<const u32x4*>(row);
    const float s = *scale;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      constexpr int E = 16 / RE;  // elements of a word
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int k = E * j + e;
        x[e] = (float)(int8_t)(c[k / 4] >> (8 * (k & 3))) * s;
      }
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (RB) o[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
        else o[e] = __float_as_uint(x[e]);
      }
      *reinterpret_cast<u32x4*>(dense + 16 * j) = o;
    }
  } else if constexpr (QUANT) {
    u32x4 w[NW];
    float x[CH];
#pragma unroll
    for (int j = 0; j < NW; ++j) w[j] = *reinterpret_cast<const u32x4*>(dense + 16 * j);
#pragma unroll
    for (int j = 0; j < NW; ++j) widen<RB>(w[j], x + j * (16 / RE));
    // the magnitudes' bits are ordered as the magnitudes are, with infinity and NaN above every number
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < CH; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
#pragma unroll
    for (int m = 1; m < LPR; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m, kWave));
    const float most = __uint_as_float(top);
    const bool finite = top < 0x7f800000u, kept = finite && most >= 0x1p-100f;
    const float inv = kept ? 127.0f / most : 0.0f;
    u32x4 code;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      code[j] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        code[j] |= ((uint32_t)(int32_t)rintf(kept ? x[4 * j + e] * inv : 0.0f) & 0xffu) << (8 * e);
    }
    *reinterpret_cast<u32x4*>(row) = code;
    if (part == 0) *scale = kept ? most / 127.0f : finite ? 0.0f : __uint_as_float(0x7fc00000u);
  }
}

template <int D, int CACHE, int ROWS, bool GATHER>
hipError_t launch(RowsArgs a, const RowsLayers<kRowsLayers>& layers, hipStream_t stream) {
  constexpr int LPR = D / (CACHE == KVC_I8 ? 16 : ROWS == KVC_BF16 ? 8 : 4), WAVES = kRowsThreads / kWave;
  const int pieces = (a.pv.num_kv_heads * LPR + kWave - 1) / kWave;
  const int64_t groups = ((int64_t)a.step.num_rows + WAVES - 1) / WAVES;
  const int64_t most = (INT64_C(1) << 32) / kRowsThreads / pieces - 1;  // (a grid's dimension ends at 2^32 threads)
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
  for (int64_t first = 0; first < groups; first += most) {
    const dim3 grid((unsigned)(std::min(most, groups - first) * pieces), 2, a.num_layers);
    a.token0 = (int32_t)(first * WAVES);
    if (by_few) serve_rows<D, CACHE, ROWS, GATHER, kFewLayers><<<grid, kRowsThreads, 0, stream>>>(a, few, pieces);
    else serve_rows<D, CACHE, ROWS, GATHER, kRowsLayers><<<grid, kRowsThreads, 0, stream>>>(a, layers, pieces);
  }
  return hipGetLastError();
}

template <int D, bool GATHER>
hipError_t launch_types(const RowsArgs& a, const RowsLayers<kRowsLayers>& layers, kvc_dtype cache, kvc_dtype rows,
                        hipStream_t stream) {
  if (cache == KVC_F32) return launch<D, KVC_F32, KVC_F32, GATHER>(a, layers, stream);
  if (cache == KVC_BF16) return launch<D, KVC_BF16, KVC_BF16, GATHER>(a, layers, stream);
  return rows == KVC_BF16 ? launch<D, KVC_I8, KVC_BF16, GATHER>(a, layers, stream)
                          : launch<D, KVC_I8, KVC_F32, GATHER>(a, layers, stream);
}

}  // namespace

hipError_t launch_rows(const RowsArgs& a, const RowsLayers<kRowsLayers>& layers, kvc_dtype cache, kvc_dtype rows,
                       int head_dim, bool gather, hipStream_t stream) {
  if (a.step.num_rows == 0 || a.num_layers == 0) return hipSuccess;
  if (head_dim == 64)
    return gather ? launch_types<64, true>(a, layers, cache, rows, stream)
                  : launch_types<64, false>(a, layers, cache, rows, stream);
  return gather ? launch_types<128, true>(a, layers, cache, rows, stream)
                : launch_types<128, false>(a, layers, cache, rows, stream);
}

}  // namespace kvc
