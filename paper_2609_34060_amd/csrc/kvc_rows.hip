// New tokens' rows into the paged cache (kvc_append) and back (kvc_gather).
//
// A row is one token's key or value of one KV head.  8-bit cache: scale = max|x| / 127, code = rint(x * (127 / max|x|)),
// value = code * scale.  Both directions move each byte once and are bound by HBM.  A lane handles 16 bytes of a dense
// row (8 bf16 or 4 float32 elements), so a row's maximum is a reduction over head_dim / 8 (/ 4) neighbouring lanes, and
// a wave reads 1 KB at a time; 256 threads take ROUNDS such groups of rows, all loads issued before the first use.
#include "kvc_serve.h"

namespace kvc {
namespace {

constexpr int kRowsThreads = 256;

// Token row -> sequence and cache row.  `seq` is a sequence that starts at or before the token (the walk goes on from
// it); returns the byte offset of head h's row, or -1 where the token has no place, and that of its scale.
__device__ __forceinline__ int64_t token_place(const RowsArgs& a, int& seq, int token, int head, int64_t& scale_at) {
  while (seq + 1 < a.step.num_seqs && a.step.starts[seq + 1] <= token) ++seq;
  scale_at = 0;
  const SeqView s = step_seq(a.step, seq);
  const int t = s.ctx - s.q + (token - s.start);
  if (!s.ok || token >= s.start + s.q || t < 0) return -1;
  int32_t slot;
  const int32_t* table = a.step.tables ? a.step.tables + (int64_t)seq * a.step.max_blocks : nullptr;
  const int32_t blk = step_block(a.pv, table, s.off + t, slot);
  if (blk < 0) return -1;
  scale_at = slot_scale_bytes(a.pv, blk, slot) + head * a.pv.shead_bytes;
  return slot_bytes(a.pv, blk, slot) + head * a.pv.head_bytes;
}

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

// CACHE, ROWS: kvc_dtype.  One thread: the CH = 16 / sizeof(element) elements `part` of a row.
template <int D, int CACHE, int ROWS, bool GATHER, int ROUNDS>
__global__ __launch_bounds__(kRowsThreads) void serve_rows(RowsArgs a) {
  constexpr bool QUANT = CACHE == KVC_I8, RB = ROWS == KVC_BF16;
  constexpr int CH = RB ? 8 : 4;          // elements of a thread
  constexpr int LPR = D / CH;             // threads of a row
  constexpr int GROUP = kRowsThreads / LPR;
  const int tid = threadIdx.x, part = tid % LPR;
  const int layer = blockIdx.z, kv = blockIdx.y;
  const int H = a.pv.num_kv_heads;
  const int total = a.step.num_rows * H;
  const int first = blockIdx.x * (GROUP * ROUNDS);
  char* pool = static_cast<char*>(a.pools[kv][layer]);
  char* scales = QUANT ? reinterpret_cast<char*>(a.scales[kv][layer]) : nullptr;
  char* rows = a.rows[kv] + layer * a.layer_stride;

  // the first row's sequence, then a walk from row to row
  int seq = step_find(a.step, first / H, [](int64_t start, int) { return start; });
  if (seq < 0) return;
  int64_t at[ROUNDS], sat[ROUNDS];
  char* dense[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int r = first + i * GROUP + tid / LPR;
    const int token = r / H, head = r - token * H;
    at[i] = -1;
    if (r < total) at[i] = token_place(a, seq, token, head, sat[i]);
    dense[i] = rows + token * a.token_stride + head * a.head_stride + part * 16;
  }
  if constexpr (!QUANT) {
    u32x4 w[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
      if (at[i] >= 0) w[i] = *reinterpret_cast<const u32x4*>(GATHER ? pool + at[i] + part * 16 : dense[i]);
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
      if (at[i] >= 0) *reinterpret_cast<u32x4*>(GATHER ? dense[i] : pool + at[i] + part * 16) = w[i];
  } else if constexpr (GATHER) {
    uint32_t c[ROUNDS][CH / 4];
    float s[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
      if (at[i] >= 0) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(pool + at[i] + part * CH);
#pragma unroll
        for (int j = 0; j < CH / 4; ++j) c[i][j] = p[j];
        s[i] = *reinterpret_cast<const float*>(scales + sat[i]);
      }
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
      if (at[i] >= 0) {
        float x[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) x[j] = (float)(int8_t)(c[i][j / 4] >> (8 * (j & 3))) * s[i];
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (RB) w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
          else w[j] = __float_as_uint(x[j]);
        }
        *reinterpret_cast<u32x4*>(dense[i]) = w;
      }
  } else {
    u32x4 w[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      w[i] = u32x4{0, 0, 0, 0};
      if (at[i] >= 0) w[i] = *reinterpret_cast<const u32x4*>(dense[i]);
    }
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
      float x[CH];
      widen<RB>(w[i], x);
      // the magnitudes' bits are ordered as the magnitudes are, with infinity and NaN above every number
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < CH; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
#pragma unroll
      for (int m = 1; m < LPR; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m, kWave));
      if (at[i] < 0) continue;
      const float most = __uint_as_float(top);
      const bool finite = top < 0x7f800000u, kept = finite && most >= 0x1p-100f;
      const float inv = kept ? 127.0f / most : 0.0f;
      uint32_t c[CH / 4];
#pragma unroll
      for (int j = 0; j < CH / 4; ++j) {
        c[j] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          c[j] |= ((uint32_t)(int32_t)rintf(kept ? x[4 * j + e] * inv : 0.0f) & 0xffu) << (8 * e);
      }
      uint32_t* p = reinterpret_cast<uint32_t*>(pool + at[i] + part * CH);
#pragma unroll
      for (int j = 0; j < CH / 4; ++j) p[j] = c[j];
      if (part == 0)
        *reinterpret_cast<float*>(scales + sat[i]) = kept ? most / 127.0f : finite ? 0.0f : __uint_as_float(0x7fc00000u);
    }
  }
}

template <int D, int CACHE, int ROWS, bool GATHER>
hipError_t launch(const RowsArgs& a, hipStream_t stream) {
  constexpr int GROUP = kRowsThreads / (D / (ROWS == KVC_BF16 ? 8 : 4));
  const int64_t total = (int64_t)a.step.num_rows * a.pv.num_kv_heads;
  const dim3 small((unsigned)((total + GROUP - 1) / GROUP), 2, a.num_layers);
  // four rows a thread once that leaves every CU two workgroups; fewer rows are spread over the chip
  if ((int64_t)small.x * 2 * a.num_layers >= 4 * 512) {
    const dim3 grid((unsigned)((total + 4 * GROUP - 1) / (4 * GROUP)), 2, a.num_layers);
    serve_rows<D, CACHE, ROWS, GATHER, 4><<<grid, kRowsThreads, 0, stream>>>(a);
  } else {
    serve_rows<D, CACHE, ROWS, GATHER, 1><<<small, kRowsThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <int D, bool GATHER>
hipError_t launch_types(const RowsArgs& a, kvc_dtype cache, kvc_dtype rows, hipStream_t stream) {
  if (cache == KVC_F32) return launch<D, KVC_F32, KVC_F32, GATHER>(a, stream);
  if (cache == KVC_BF16) return launch<D, KVC_BF16, KVC_BF16, GATHER>(a, stream);
  return rows == KVC_BF16 ? launch<D, KVC_I8, KVC_BF16, GATHER>(a, stream)
                          : launch<D, KVC_I8, KVC_F32, GATHER>(a, stream);
}

}  // namespace

hipError_t launch_rows(const RowsArgs& a, kvc_dtype cache, kvc_dtype rows, int head_dim, bool gather,
                       hipStream_t stream) {
  if (a.step.num_rows == 0 || a.num_layers == 0) return hipSuccess;
  if (head_dim == 64)
    return gather ? launch_types<64, true>(a, cache, rows, stream) : launch_types<64, false>(a, cache, rows, stream);
  return gather ? launch_types<128, true>(a, cache, rows, stream) : launch_types<128, false>(a, cache, rows, stream);
}

}  // namespace kvc
