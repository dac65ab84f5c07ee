// Attention of a step's new tokens over the paged cache (kvc_attend):
//
//   out = sum_t exp(s_t - m) V[t] / sum_t exp(s_t - m),   s_t = scale * (q . K[t]),   m = max_t s_t.
//
// One pass over the keys with a running reference m and sum; scores are kept in units of log2 so that the exponentials
// are v_exp_f32.  The g = num_heads / num_kv_heads query heads of a KV head and the new tokens of a sequence form one
// list of rows, row r = token r / g, head r % g, so that a key is read once for all of them.
#include <algorithm>

#include "kvc_serve.h"

namespace kvc {
namespace {

constexpr int kRowTile = 16;     // rows of a workgroup
constexpr int kStepKeys = 32;    // keys of a wave's step
constexpr int kWaves = 4;
constexpr float kRescale = 8.0f; // log2 units by which scores may pass the reference before it moves

constexpr int kTileKeys = 64;    // keys of a shared tile (attend_tiles)

// Where 16-byte chunk c of row r of a shared tile lies in its row.  K is read a chunk of 32 rows at a time, V four chunks
// of four rows: the exclusive or gives each a place of its own in the 256 bytes of the banks.
template <int D>
__device__ __forceinline__ int k_chunk(int r, int c) {
  return D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int v_chunk(int r, int c) {
  return D == 128 ? c ^ (4 * (r & 3)) : c ^ (4 * ((r >> 1) & 1));
}

// 512 bytes of zeros: what a lane reads for a key that is not there.
__device__ const uint32_t g_zeros[128] = {};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
// Device memory as such: a pointer that may be one of two would otherwise be loaded from by flat instructions, which
// wait for LDS as well.
typedef const __attribute__((address_space(1))) char* GlobalPtr;
__device__ __forceinline__ u32x4 load16(GlobalPtr p) {
  return *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(p);
}
__device__ __forceinline__ float load_float(GlobalPtr p) {
  return *reinterpret_cast<const __attribute__((address_space(1))) float*>(p);
}
#define KVC_LDS(T, p) ((__attribute__((address_space(3))) T*)(p))

// Four signed 8-bit codes as bf16 (exact).
__device__ __forceinline__ void widen_codes(uint32_t c, uint32_t& lo, uint32_t& hi) {
  lo = pack_bf16x2((float)(int8_t)c, (float)(int8_t)(c >> 8));
  hi = pack_bf16x2((float)(int8_t)(c >> 16), (float)(int8_t)(c >> 24));
}

// Lane j of each row of R lanes (8 or 4: by an LDS permute) to all of that row.
template <int R>
__device__ __forceinline__ uint32_t row_lane(uint32_t x, int j) {
  if constexpr (R == 16) {
    switch (j) {  // (an instruction's constant)
      case 0: return __builtin_amdgcn_update_dpp(0, x, 0x150, 0xf, 0xf, true);
      case 1: return __builtin_amdgcn_update_dpp(0, x, 0x151, 0xf, 0xf, true);
      case 2: return __builtin_amdgcn_update_dpp(0, x, 0x152, 0xf, 0xf, true);
      default: return __builtin_amdgcn_update_dpp(0, x, 0x153, 0xf, 0xf, true);
    }
  }
  return __shfl((int)x, (int)((threadIdx.x & (kWave - 1)) / R * R + j), kWave);
}

// The bits below n of a word, for any n.
__device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }

// LDS that one wave alone writes and reads: the hardware keeps its order, and so must the compiler.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// 16 bytes of values with zeros in the place of NaN and infinities.
template <bool F32>
__device__ __forceinline__ u32x4 numbers_of(u32x4 w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32) {
      w[i] = (w[i] & 0x7f800000u) == 0x7f800000u ? 0u : w[i];
    } else {
      w[i] &= ((w[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
    }
  }
  return w;
}
// The same in place; whether there was one.
template <bool F32>
__device__ __forceinline__ bool to_numbers(u32x4& w) {
  const u32x4 x = numbers_of<F32>(w), d = x ^ w;
  w = x;
  return (d[0] | d[1] | d[2] | d[3]) != 0;
}

// A range of keys leaves its part of a row (the products with the values, not yet divided) unless its sum is +0: nothing
// that the row sees has a weight there.  Zero weights alone, but a value that is no number among those seen, whose product
// with zero is NaN as it would be in one range: a part under this sum.  So what a row gets does not depend on where its
// ranges end; the weights of a row sum to zero only where all its scores are -inf, and then it gets zeros.
constexpr float kOddRange = -0.0f;
__device__ __forceinline__ bool holds_part(float sum) { return __float_as_uint(sum) != 0u; }

struct Tile {
  SeqView s;
  int seq, row0, rows;  // rows row0 .. of the sequence's q * g
};

// Tiles of BM rows.  direct: tile i is sequence i.  Otherwise sequence i owns the tiles from floor(starts[i] g / BM) + i
// on: at least as many as it needs, and none of another's, without a list of them.
template <int BM>
__device__ __forceinline__ Tile find_tile(const AttendArgs& a, int tile) {
  Tile t;
  t.row0 = 0;
  t.seq = tile;
  const int g = a.group;
  if (a.direct) {
    t.s = step_seq(a.step, t.seq);
  } else {
    // (rows outside the step's are brought to its ends, so that 32 bits do: their sequences are left out)
    auto rows_to = [&a, g](int x) { return (uint32_t)min(max(x, 0), a.step.num_rows) * (uint32_t)g; };
    t.seq = step_find(
        a.step, tile, t.s, [rows_to](int start, int i) { return (int)(rows_to(start) / BM) + i; },
        [rows_to](int start, int end, int i) {
          const uint32_t r = rows_to(start);
          return (int)(r / BM) + i + ((int)(rows_to(end) - r) + BM - 1) / BM;
        });
  }
  if (t.seq < 0) {
    t.rows = 0;
    return t;
  }
  if (!a.direct) t.row0 = (int)(tile - ((int64_t)t.s.start * g / BM + t.seq)) * BM;
  t.rows = t.s.ok ? min(BM, t.s.q * g - t.row0) : 0;
  return t;
}

// Context indices [lo, hi) that new token j of a sequence sees.
__device__ __forceinline__ void visible(const AttendArgs& a, const SeqView& s, int j, int& lo, int& hi) {
  const int pos = s.ctx - s.q + j;
  hi = pos < 0 ? 0 : a.causal ? pos + 1 : s.ctx;
  lo = a.window && pos >= a.window ? pos + 1 - a.window : 0;  // (pos may lie far below 0, and a window near 2^31)
}

// The values of one key that are no numbers (bfloat16 and float32 caches), for the rows that see it: where a step of
// keys is not seen by all rows, the products take zeros in their place, since zero times infinity would reach a row that
// does not see them (attend_rows takes zeros in every step of a bfloat16 cache, for the sake of its weights' two terms).  Lane `part` of the G lanes of a row; add(v) adds v(f) to each of the lane's accumulators.
template <int D, bool F32, int G, class Add>
__device__ __forceinline__ void odd_values(GlobalPtr q, GlobalPtr k, GlobalPtr v, int part, float scale_log2,
                                           float ref, bool sees, Add add) {
  auto value = [](GlobalPtr x, int f) {
    return F32 ? load_float(x + 4 * f)
               : bf16_lo_to_f32(*reinterpret_cast<const __attribute__((address_space(1))) uint16_t*>(x + 2 * f));
  };
  bool odd = false;
  for (int f = threadIdx.x & (kWave - 1); f < D; f += kWave) odd = odd || !(fabsf(value(v, f)) < INFINITY);
  if (!__any(odd)) return;
  float s = 0.0f;
  for (int f = part * (D / G); f < (part + 1) * (D / G); ++f) s += value(q, f) * value(k, f);
#pragma unroll
  for (int x = kWave / G; x < kWave; x *= 2) s += __shfl_xor(s, x, kWave);
  const float p = __builtin_amdgcn_exp2f(s * scale_log2 - ref);
  add([&](int f) {
    const float x = value(v, f);
    return sees && !(fabsf(x) < INFINITY) ? p * x : 0.0f;
  });
}

// Two weights, each as the sum of two bf16, to within 2^-16 of it (one that is a bf16 is the first term).  The values that they
// multiply are finite; a weight over an 8-bit cache may be infinite (of an infinite scale), and is then the first term alone.
template <bool I8>
__device__ __forceinline__ uint2 two_terms(float x, float y) {
  const uint32_t first = pack_bf16x2(x, y);
  float rx = x - __uint_as_float(first << 16), ry = y - __uint_as_float(first & 0xffff0000u);
  if constexpr (I8) {
    rx = rx == rx ? rx : 0.0f;
    ry = ry == ry ? ry : 0.0f;
  }
  return make_uint2(first, pack_bf16x2(rx, ry));
}

// One tile of 16 rows, one KV head, one range of keys.  S^T = K Q^T and O^T = V^T P^T on 16 x 16 tiles, a row of the
// tile being column lane % 16 throughout: the scores of a row are in registers of the four lanes (n, kg) and become the
// operand of the second product where they are.  Waves take the 32-key steps of the range in turn, each on its own, and
// are joined at the end.  K comes from memory in operand layout; V goes through the wave's own LDS (written as loaded,
// read back transposed).
//
// Bound by HBM where there are few rows: each byte of K and V is read once, and the next step's loads are in flight while a
// step is worked on.  64 single tokens of 1K-16K keys, 32 heads on 8: 446 us, 5.8 TB/s of the 6.05 that reads of this
// pattern reach alone (bfloat16); 252 us, 5.3 of 6.0 (8 bits: the vector unit, with the codes' widening, is at 44 %, and a
// fourth wave a SIMD changes nothing).  One token of 32771 keys, 28 heads on 4: 14.8 us.  A call on 1000 keys is five
// memory latencies, 7 us.  Float32 products run on 16 x 16 x 4 tiles.
//
// The matrix unit takes the weights exp(s - m) in bf16.  It has room here, so they go in as the sum of two: 458.0 against
// 458.1 us and 258.8 against 257.3 for the batches above, and the result is off by 0.00166 and 0.00168 of its norm where one
// bf16 gives 0.00211 and 0.00234; rounding the result alone gives 0.00166 and 0.00168.  Values that are no numbers are
// looked for in every step; zeros then take their place (see odd_values).
template <int D, int CACHE>
__global__ __launch_bounds__(kWaves * kWave, CACHE == KVC_I8 ? 3 : 2) void attend_rows(AttendArgs a) {
  constexpr bool F32 = CACHE == KVC_F32, I8 = CACHE == KVC_I8;
  constexpr int ES = F32 ? 4 : I8 ? 1 : 2;
  constexpr int NL = D * ES / 64;        // 16-byte loads of a lane per 16 keys
  constexpr int FT = D / 16;             // feature tiles of O^T
  constexpr int SLOT = 16 * D * ES;      // bytes of 16 keys
  constexpr int WAVE_LDS = 2 * SLOT + (I8 ? 256 : 0);
  constexpr int JOIN = kWaves * 16 * D * 4;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves * WAVE_LDS > JOIN ? kWaves * WAVE_LDS : JOIN];
  __shared__ float join_m[kWaves][16], join_l[kWaves][16];

  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int n = lane & 15, kg = lane >> 4;
  // Consecutive workgroups go to the eight XCDs in turn: with the ranges fastest, an XCD would get the same ranges of
  // every row of the grid wherever their number divides 8 or is a multiple of it, and those with the late ranges, which
  // short sequences lack, would idle.  So the ranges of a row are shifted by one whenever 8 workgroups have come round.
  const int head = blockIdx.y;
  const unsigned grid_row = blockIdx.y + gridDim.y * blockIdx.z;
  const unsigned common = min(gridDim.x & -gridDim.x, 8u);  // with 8
  const int split = (blockIdx.x + grid_row * common / 8) % gridDim.x;
  const Tile tile = find_tile<kRowTile>(a, a.tile0 + blockIdx.z);
  if (tile.rows <= 0) return;
  const SeqView& sq = tile.s;
  const int g = a.group;

  // this lane's row
  const bool has_row = n < tile.rows;
  const int row = tile.row0 + (has_row ? n : 0);
  const int token = quotient(row, a.by_group), qh = head * g + row - token * g;
  int lo = 0, hi = 0;
  if (has_row) visible(a, sq, token, lo, hi);
  // the tile's keys, and those that every row sees
  int t_lo, t_hi, u0, u1;
  visible(a, sq, quotient(tile.row0, a.by_group), t_lo, u1);
  visible(a, sq, quotient(tile.row0 + tile.rows - 1, a.by_group), u0, t_hi);
  const int begin = t_lo + split * a.chunk;
  const int end = min(t_hi, begin + a.chunk);
  if (begin >= end && a.splits > 1) {  // nothing in this range
    if (tid < tile.rows) {
      const int r = tile.row0 + tid;
      const int tok = quotient(r, a.by_group);
      const int64_t flat = (int64_t)(sq.start + tok) * a.num_heads + head * g + r - tok * g;
      a.part_ml[(int64_t)split * a.step.num_rows * a.num_heads + flat] = make_float2(-INFINITY, 0.0f);
    }
    return;
  }

  // Q as the B operand: lane (n, kg) holds the features that the K operand has in lane (m, kg)
  // (read from LDS in every step where 16 or 32 registers more would cost a wave on each SIMD)
  constexpr bool QLDS = F32 && D == 128;
  constexpr int NQ = F32 ? D / 16 : D / 32;
  __shared__ __attribute__((aligned(16))) u32x4 q_lds[QLDS ? NQ * kWave : 1];
  u32x4 q_reg[QLDS ? 1 : NQ];
  const char* qp = a.q + (int64_t)(sq.start + token) * a.q_token_stride + (int64_t)qh * a.q_head_stride;
#pragma unroll
  for (int s = 0; s < NQ; ++s) {
    const int chunk = I8 ? (4 * (s >> 1) + kg) * 2 + (s & 1) : 4 * s + kg;  // of 16 bytes
    if constexpr (!QLDS) q_reg[s] = load16((GlobalPtr)qp + chunk * 16);
    else if (s % kWaves == wave) q_lds[s * kWave + lane] = load16((GlobalPtr)qp + chunk * 16);
  }
  if constexpr (QLDS) __syncthreads();
  auto q_of = [&](int s) -> u32x4 {
    if constexpr (QLDS) return q_lds[s * kWave + lane];
    else return q_reg[s];
  };

  f32x4 o[FT];
#pragma unroll
  for (int i = 0; i < FT; ++i) o[i] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;
  int odd_from = end, odd_to = begin;  // steps between these may have had zeros in the place of values (see odd_values)

  const int32_t* table = a.step.tables ? a.step.tables + (int64_t)tile.seq * a.step.max_blocks : nullptr;
  const GlobalPtr kp = (GlobalPtr)a.k + head * a.pv.head_bytes;
  const GlobalPtr vp = (GlobalPtr)a.v + head * a.pv.head_bytes;
  const GlobalPtr zeros = (GlobalPtr)(const void*)g_zeros;
  const GlobalPtr ksp = (GlobalPtr)a.ks + head * a.pv.shead_bytes;
  const GlobalPtr vsp = (GlobalPtr)a.vs + head * a.pv.shead_bytes;
  unsigned char* slot = lds + wave * WAVE_LDS;
  float* scl = reinterpret_cast<float*>(slot + 2 * SLOT);  // [K/V][32 keys]

  // This lane's key of 16-key half h of a step: its table entry is fetched a step ahead of the loads that it is for, and
  // ahead of that step's own loads in the queue, so that no load waits for the one before it.
  struct Places {
    int entry[2], slot[2];
  };
  auto fetch = [&](int kb) {
    Places f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      f.entry[h] = step_entry(a.pv, table, sq.off + min(kb + 16 * h + n, end - 1), f.slot[h]);
    return f;
  };
  auto resolve = [&](int kb, const Places& f, int* blk) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      blk[h] = kb + 16 * h + n < end && (uint32_t)f.entry[h] < (uint32_t)a.pv.num_blocks ? f.entry[h] : -1;
  };
  u32x4 kr[2][NL], vr[2][NL];
  float scale_r = 0.0f;  // of key lane % 32 of a step: K's in the lower lanes, V's in the upper
  auto load_v = [&](const int* blk, const int* at) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const GlobalPtr p = blk[h] >= 0 ? vp + slot_bytes(a.pv, blk[h], at[h]) : zeros;
#pragma unroll
      for (int s = 0; s < NL; ++s) vr[h][s] = load16(p + (4 * s + kg) * 16);
    }
    if constexpr (I8) {
      const int odd = -(kg & 1), b = blk[0] ^ ((blk[0] ^ blk[1]) & odd), slot_of = at[0] ^ ((at[0] ^ at[1]) & odd);
      scale_r = load_float(b >= 0 ? (lane < 32 ? ksp : vsp) + slot_scale_bytes(a.pv, b, slot_of) : zeros);
    }
  };
  auto load_k = [&](const int* blk, const int* at) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const GlobalPtr p = blk[h] >= 0 ? kp + slot_bytes(a.pv, blk[h], at[h]) : zeros;
#pragma unroll
      for (int s = 0; s < NL; ++s) kr[h][s] = load16(p + (4 * s + kg) * 16);
    }
  };

  constexpr int STRIDE = kWaves * kStepKeys;
  int kb = begin + wave * kStepKeys;
  int blk[2], nblk[2];
  Places next = {};
  if (kb < end) {
    const Places first = fetch(kb);
    next = fetch(kb + STRIDE);
    resolve(kb, first, blk);
    load_v(blk, first.slot);
    load_k(blk, first.slot);
  }

  for (; kb < end; kb += STRIDE) {
    const bool all = kb >= u0 && kb + kStepKeys <= u1;
    bool clean = F32 && !all;
    if constexpr (CACHE == KVC_BF16) {  // (the terms of a weight would meet an infinity as 0 or with two signs)
      uint32_t top = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < NL; ++s)
#pragma unroll
          for (int e = 0; e < 4; ++e) top |= (vr[h][s][e] & 0x7f807f80u) + 0x00800080u;
      clean = __any(top & 0x80008000u);  // (an exponent of ones)
    }
    if (clean) {
      bool odd = false;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < NL; ++s) odd |= to_numbers<F32>(vr[h][s]);
      if (__any(odd)) {
        odd_from = min(odd_from, kb);
        odd_to = kb + kStepKeys;
      }
    }
    // V into LDS as it was loaded: 16 bytes of lane (m, kg), load s, half h at h SLOT + s 1024 + lane 16
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int s = 0; s < NL; ++s) *reinterpret_cast<u32x4*>(slot + h * SLOT + s * 1024 + lane * 16) = vr[h][s];
    if constexpr (I8) scl[lane] = scale_r;
    wave_lds_order();
    // bits 0..31: this step's keys that are there
    uint32_t there = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) there |= (uint32_t)(__ballot(blk[h] >= 0) & 0xffffu) << (16 * h);
    const bool whole = all && there == 0xffffffffu;
    const Places now = next;
    resolve(kb + STRIDE, now, nblk);
    next = fetch(kb + 2 * STRIDE);
    load_v(nblk, now.slot);

    // scores of keys 16 h + 4 kg + i
    float s[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 acc = {0, 0, 0, 0};
      if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < NL; ++j) {
          const u32x4 qx = q_of(j);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[h][j][e]), __uint_as_float(qx[e]), acc, 0, 0,
                                                       0);
        }
      } else if constexpr (I8) {
#pragma unroll
        for (int j = 0; j < NL; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            u32x4 f;
            uint32_t x, y;
            widen_codes(kr[h][j][2 * e], x, y);
            f[0] = x;
            f[1] = y;
            widen_codes(kr[h][j][2 * e + 1], x, y);
            f[2] = x;
            f[3] = y;
            acc = mfma16x16x32(as_bf16x8(f), as_bf16x8(q_of(2 * j + e)), acc);
          }
      } else {
#pragma unroll
        for (int j = 0; j < NL; ++j) acc = mfma16x16x32(as_bf16x8(kr[h][j]), as_bf16x8(q_of(j)), acc);
      }
      f32x4 sk = {1, 1, 1, 1};
      if constexpr (I8) sk = *reinterpret_cast<const f32x4*>(scl + 16 * h + 4 * kg);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[h][i] = acc[i] * (I8 ? a.scale_log2 * sk[i] : a.scale_log2);
    }
    load_k(nblk, now.slot);
    uint32_t seen = 0xffu;  // bit 4 h + i
    if (!whole) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 16 * h + 4 * kg + i;
          const bool sees = kb + k >= lo && kb + k < hi && ((there >> k) & 1);
          s[h][i] = sees ? s[h][i] : -INFINITY;
          seen &= sees ? 0xffu : ~(1u << (4 * h + i));
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) blk[h] = nblk[h];

    // the reference moves only when a score passes it by 2^kRescale: any m serves, as long as nothing overflows
    float mx = s[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[j >> 2][j & 3]);
    if (__any(mx > m + kRescale)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      const bool move = mx > m + kRescale;  // (row by row: no row's bits depend on another's scores)
      const float f = move ? __builtin_amdgcn_exp2f(m - mx) : 1.0f;
      m = move ? mx : m;
      l *= f;
#pragma unroll
      for (int i = 0; i < FT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] *= f;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
    float p[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[h][i] = __builtin_amdgcn_exp2f(s[h][i] - ref);
        l += p[h][i];
      }
    if constexpr (I8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 sv = *reinterpret_cast<const f32x4*>(scl + 32 + 16 * h + 4 * kg);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[h][i] *= sv[i];
      }
      if (!whole) {  // (a scale that is no number belongs to those that see its key)
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j >> 2][j & 3] = (seen >> j) & 1 ? p[j >> 2][j & 3] : 0.0f;
      }
    }

    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) {
          const int h = j >> 2, mrow = 4 * kg + (j & 3), byte = (16 * ft + n) * 4;
          const float v = *reinterpret_cast<const float*>(slot + h * SLOT + (byte / 64) * 1024 +
                                                          ((byte % 64) / 16 * 16 + mrow) * 16 + byte % 16);
          o[ft] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[h][j & 3], o[ft], 0, 0, 0);
        }
    } else {
      u32x4 pf, pl;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint2 w = two_terms<I8>(p[h][2 * i], p[h][2 * i + 1]);
          pf[2 * h + i] = w.x;
          pl[2 * h + i] = w.y;
        }
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        u32x4 vf;
        if constexpr (I8) {
          // 8 keys (rows n / 2) x 16 features; result: this lane's feature, keys 4 kg + 0..3 of both halves
          const int r = n >> 1, byte = 16 * ft;
          const unsigned char* x = slot + (r >> 2) * SLOT + (byte / 64) * 1024 +
                                   ((byte % 64) / 16 * 16 + 4 * kg + (r & 3)) * 16 + 8 * (n & 1);
          const i32x2 c = __builtin_amdgcn_ds_read_tr8_b64_v2i32(KVC_LDS(i32x2, x));
          uint32_t lo2, hi2;
          widen_codes((uint32_t)c[0], lo2, hi2);
          vf[0] = lo2;
          vf[1] = hi2;
          widen_codes((uint32_t)c[1], lo2, hi2);
          vf[2] = lo2;
          vf[3] = hi2;
        } else {
          // 4 keys (rows n / 4) x 16 features of each half
          const int byte = (16 * ft + 4 * (n & 3)) * 2;
          const unsigned char* x =
              slot + (byte / 64) * 1024 + ((byte % 64) / 16 * 16 + 4 * kg + (n >> 2)) * 16 + byte % 16;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint2 c = __builtin_bit_cast(
                uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(KVC_LDS(s16x4, x + h * SLOT)));
            vf[2 * h] = c.x;
            vf[2 * h + 1] = c.y;
          }
        }
        o[ft] = mfma16x16x32(as_bf16x8(vf), as_bf16x8(pf), o[ft]);
        o[ft] = mfma16x16x32(as_bf16x8(vf), as_bf16x8(pl), o[ft]);
        // (reads of all tiles at once would take the registers of a third wave on each SIMD)
        if (ft % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
    wave_lds_order();
  }

  const float last_ref = m == -INFINITY ? 0.0f : m;
  if (!I8 && odd_from < odd_to) {
    for (kb = odd_from; kb < odd_to; kb += STRIDE) {
      if (F32 && kb >= u0 && kb + kStepKeys <= u1) continue;
      for (int key = kb; key < min(kb + kStepKeys, end); ++key) {
        int slot_of;
        const int32_t b = step_block(a.pv, table, sq.off + key, slot_of);
        if (b < 0) continue;
        const int64_t off = slot_bytes(a.pv, b, slot_of);
        odd_values<D, F32, 4>((GlobalPtr)qp, kp + off, vp + off, kg, a.scale_log2, last_ref, key >= lo && key < hi, [&](auto v) {
#pragma unroll
          for (int ft = 0; ft < FT; ++ft)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ft][i] += v(16 * ft + 4 * kg + i);
        });
      }
    }
  }

  // join the four waves
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  __syncthreads();  // every wave is done with its part of lds
  if (kg == 0) {
    join_m[wave][n] = m;
    join_l[wave][n] = l;
  }
  float* join = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) *reinterpret_cast<f32x4*>(join + (wave * 16 + n) * D + 16 * ft + 4 * kg) = o[ft];
  __syncthreads();
  constexpr int PER = D / 16;  // features of a thread
  const int r = tid / 16, f0 = (tid % 16) * PER;
  if (r >= tile.rows) return;
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, join_m[w][r]);
  float sum = 0.0f, x[PER] = {};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = join_m[w][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(join_m[w][r] - top);
    // (a wave without a finite maximum has no sum; a NaN in it must still show)
    sum += join_m[w][r] == -INFINITY ? join_l[w][r] : join_l[w][r] * f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float v = join[(w * 16 + r) * D + f0 + i];
      x[i] += join_m[w][r] == -INFINITY ? v : v * f;
    }
  }
  const int tok = quotient(tile.row0 + r, a.by_group), h = head * g + tile.row0 + r - tok * g;
  const int64_t flat = (int64_t)(sq.start + tok) * a.num_heads + h;
  if (a.splits > 1) {
    const int64_t at_s = (int64_t)split * a.step.num_rows * a.num_heads + flat;
    if (sum == 0.0f) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < PER; ++i) odd = odd || x[i] != 0.0f;
#pragma unroll
      for (int i = 1; i < 16; i *= 2) odd = __shfl_xor((int)odd, i, kWave) || odd;
      if (odd) sum = kOddRange;
    }
    if (f0 == 0) a.part_ml[at_s] = make_float2(top, sum);
    if (holds_part(sum))
#pragma unroll
      for (int i = 0; i < PER; i += 4)
        *reinterpret_cast<f32x4*>(a.part_o + at_s * D + f0 + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
    return;
  }
  const float inv = 1.0f / sum;
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = sum == 0.0f ? 0.0f : x[i] * inv;
  char* op = a.out + (int64_t)(sq.start + tok) * a.out_token_stride + (int64_t)h * a.out_head_stride;
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < PER; ++i) reinterpret_cast<float*>(op)[f0 + i] = x[i];
  } else {
#pragma unroll
    for (int i = 0; i < PER; i += 2)
      reinterpret_cast<uint32_t*>(op)[(f0 + i) / 2] = pack_bf16x2(x[i], x[i + 1]);
  }
  if (a.lse && f0 == 0)
    a.lse[flat] = sum == 0.0f ? -INFINITY : (top == -INFINITY ? 0.0f : top) * 0.69314718055994531f + logf(sum);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The sum to keep of a row of a tile whose weights sum to zero, from its accumulators o (in lanes n and n + 32).
template <int D>
__device__ __forceinline__ float without_weights(const f32x16* o) {
  bool odd = false;
#pragma unroll
  for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
    for (int j = 0; j < 16; ++j) odd = odd || o[ft][j] != 0.0f;
  odd = __shfl_xor((int)odd, 32, kWave) || odd;
  return odd ? kOddRange : 0.0f;
}

// Features 2 j .. 2 j + 15 of a row's 32 in the accumulators o of its two lanes (4 hf + 0..3 and 8 + 4 hf + 0..3 of them in
// lane hf): the lanes trade halves so that each writes eight in a row (4096 tokens: 147 us with stores of 8 bytes, 145 so).
__device__ __forceinline__ void write_features(char* to, int hf, const f32x16* o, int j, float inv) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const auto t = __builtin_amdgcn_permlane32_swap(
        pack_bf16x2((*o)[j + 2 * e] * inv, (*o)[j + 2 * e + 1] * inv),
        pack_bf16x2((*o)[j + 4 + 2 * e] * inv, (*o)[j + 5 + 2 * e] * inv), false, false);
    w[e] = t[0];
    w[2 + e] = t[1];
  }
  *reinterpret_cast<u32x4*>(to + 16 * hf) = w;
}

// Tiles of many rows (chunks of new tokens) over a bfloat16 cache: WAVES x 32 rows of one KV head share 64-key tiles of K
// and V in LDS.  S^T = K Q^T and O^T = V^T P^T on 32 x 32 tiles, a wave's row being column lane % 32: a row's scores are
// in registers of two lanes, and are the second product's operand where they are, under an order of the keys that the
// transposed reads of V follow.
//
// The scores of a tile are formed while the weights of the one before it are taken (matrix and vector unit at once), and
// K comes in a tile ahead of V.  Loads go straight to LDS and take no registers; they land while a step is worked on.
// Where two waves of the workgroup share a SIMD, one is half a step behind, so that one's exponentials meet the other's
// product with V.
//
// 4096 new tokens, 32 heads on 8 (137 GFLOP): 145 us, 948 TFLOP/s (154 on a card that holds less under power).  160 us
// with a step's products and weights one after the other and tiles that came in through registers; 154 with both waves of
// a SIMD in step.  What bounds it is power and the two units together: a step of 64 keys takes 4100 cycles of which the
// matrix unit has 2048, 4840 before, but the clock falls from 2.30 to 2.07 GHz as they are used better.  64 rows a wave,
// one wave a SIMD (half of the LDS reads): 192 us, as a wave alone issues a vector instruction every 5.5 cycles only.
//
// The weights go into the product with V in one bf16, for the matrix unit's sake (the result is off by 0.0022-0.0024 of
// its norm, 0.00165 of which is its own rounding): in two, as attend_rows has them, 4096 new tokens took 201 us, and
// attend_codes' case below 1658.
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, WAVES == 8 ? 1 : 2) void attend_tiles(AttendArgs a) {
  constexpr int BM = WAVES * 32;
  constexpr int RC = D / 8;                // 16-byte chunks of a row in memory
  constexpr int RPL = kWave / RC;          // rows of a wave's load
  constexpr int RW = kTileKeys / WAVES;    // rows of a tile that a wave brings in
  constexpr int NC = RW / RPL;             // its loads, of K and of V
  static_assert(NC <= RC, "lane j of a row's lanes holds the address of load j");
  constexpr int RB = D * 2;                // bytes of a row in LDS
  constexpr int HALF = kTileKeys * RB;     // bytes of a K (V) tile
  constexpr bool TURNS = WAVES == 8;       // the second wave of a SIMD is half a step behind the first
  // (tiles by names of their own: reads of one do not wait for loads into another)
  __shared__ __attribute__((aligned(16))) unsigned char lds_k0[HALF], lds_k1[HALF], lds_v0[HALF], lds_v1[HALF],
      lds_v2[TURNS ? HALF : 16], lds_v3[TURNS ? HALF : 16];
  __shared__ uint32_t lds_there[2][WAVES];  // bit r: row r of the wave's rows of the tile is there
  __shared__ int lds_odd;  // zeros stood for values of a tile that not every row sees all of

  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);  // (what goes by it is in scalar registers)
  const int n = lane & 31, hf = lane >> 5;
  const int head = blockIdx.x, split = blockIdx.y;
  // (later tiles of a sequence see more keys: they go first)
  const Tile tile = find_tile<BM>(a, a.tile0 + gridDim.z - 1 - blockIdx.z);
  if (tile.rows <= 0) return;
  const SeqView& sq = tile.s;
  const int g = a.group;

  int t_lo, t_hi, t_u0, t_u1;  // the keys that any row sees, and those that all of them see
  visible(a, sq, quotient(tile.row0, a.by_group), t_lo, t_u1);
  visible(a, sq, quotient(tile.row0 + tile.rows - 1, a.by_group), t_u0, t_hi);
  const int begin = t_lo + split * a.chunk;
  const int end = min(t_hi, begin + a.chunk);
  const int steps = end > begin ? (end - begin + kTileKeys - 1) / kTileKeys : 0;

  // this wave's rows, the keys that any and that all of them see, and this lane's row
  const int w_rows = min(32, tile.rows - wave * 32), w_row0 = tile.row0 + wave * 32;
  const bool has_row = n < w_rows;
  const int row = w_rows > 0 ? w_row0 + (has_row ? n : 0) : tile.row0;
  const int token = quotient(row, a.by_group), qh = head * g + row - token * g;
  int lo = 0, hi = 0, w_lo = 0, w_hi = 0, u0 = 0, u1 = 0;
  if (has_row) visible(a, sq, token, lo, hi);
  if (w_rows > 0) {
    visible(a, sq, quotient(w_row0, a.by_group), w_lo, u1);
    visible(a, sq, quotient(w_row0 + w_rows - 1, a.by_group), u0, w_hi);
  }

  // Scores are acc * c with c > 0, so that their order is that of the accumulators: a negative scale's sign goes to Q, and
  // with a scale of zero Q is zero.
  const float c_abs = a.scale_log2 == 0.0f ? 1.0f : fabsf(a.scale_log2);
  const uint32_t q_sign = a.scale_log2 < 0.0f ? 0x80008000u : 0u, q_keep = a.scale_log2 == 0.0f ? 0u : ~0u;
  bf16x8 qf[D / 16];
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  const int32_t* table = a.step.tables ? a.step.tables + (int64_t)tile.seq * a.step.max_blocks : nullptr;
  const GlobalPtr kp = (GlobalPtr)a.k + head * a.pv.head_bytes;
  const GlobalPtr vp = (GlobalPtr)a.v + head * a.pv.head_bytes;
  // Load j of a wave brings in rows RW wave + RPL j .. of the tile, RC lanes a row.  A row's address is worked out by one
  // lane: lane j of a row's RC lanes has that of load j (lanes beyond NC repeat it), and passes it to the others.
  const int c_row = lane / RC, c_col = lane % RC;
  const int my_row = RW * wave + RPL * (c_col % NC) + c_row;
  auto tile_k = [&](int buf) { return buf ? lds_k1 : lds_k0; };
  auto tile_v = [&](int buf) { return buf == 0 ? lds_v0 : buf == 1 ? lds_v1 : buf == 2 ? lds_v2 : lds_v3; };
  struct Row {
    int64_t off;  // bytes of the row (one that is not there: of any that is)
    bool ok;
  };
  int entry, at;  // table entry and slot of my_row of the tile after the last one whose Row was taken
  auto fetch = [&](int kb) { entry = step_entry(a.pv, table, sq.off + min(kb + my_row, end - 1), at); };
  auto take = [&](int kb) {
    Row r;
    r.ok = kb + my_row < end && (uint32_t)entry < (uint32_t)a.pv.num_blocks;
    r.off = slot_bytes(a.pv, r.ok ? entry : 0, at);
    return r;
  };
  // bytes of the row that load j brings a part of
  auto row_bytes = [&](const Row& row, int j) {
    if (NC == 1) return row.off;  // (every lane of the row has it)
    const uint32_t lo32 = row_lane<RC>((uint32_t)row.off, j);
    const uint32_t hi32 = row_lane<RC>((uint32_t)((uint64_t)row.off >> 32), j);
    return (int64_t)(((uint64_t)hi32 << 32) | lo32);
  };
  // A wave's load goes straight into LDS, 64 chunks of 16 bytes in the order of its lanes: a lane fetches the chunk whose
  // place that is.
  auto load_lds = [&](GlobalPtr p, const int64_t* off, unsigned char* tile, bool values) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int r0 = RW * wave + RPL * j, r = r0 + c_row;
      const int c = values ? v_chunk<D>(r, c_col) : k_chunk<D>(r, c_col);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + off[j] + c * 16),
                                       KVC_LDS(void, tile + r0 * RB), 16, 0, 0);
    }
  };
  auto mark = [&](int buf, const Row& row) {
    const uint64_t have = __ballot(row.ok);
    uint32_t bits = (1u << RW) - 1;  // bit r: row r of the wave's
    if (have != ~0ull) {
      bits = 0;
#pragma unroll
      for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int r = 0; r < RPL; ++r) bits |= ((uint32_t)(have >> (r * RC + j)) & 1u) << (RPL * j + r);
    }
    if (lane == 0) lds_there[buf][wave] = bits;
  };
  // What was loaded of V, once it is there: zeros for rows that are not, and for values that are no numbers in a tile
  // that not all rows see all of (see odd_values)
  auto mend = [&](unsigned char* tile, const Row& row, int kb) {
    const bool partial = kb < t_u0 || kb + kTileKeys > t_u1;
    if (__ballot(row.ok) == ~0ull && !partial) return;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      u32x4* x = reinterpret_cast<u32x4*>(tile + (RW * wave + RPL * j) * RB + lane * 16);
      u32x4 y = *x;
      const bool ok_j = NC == 1 ? row.ok : row_lane<RC>(row.ok ? 1u : 0u, j) != 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = ok_j ? y[e] : 0u;
      if (partial) odd |= to_numbers<false>(y);
      *x = y;
    }
    if (__any(odd) && lane == 0) lds_odd = 1;
  };
  // (for places that are worked out where they are used: kept, they would take registers that are not there, and what is
  // spilled waits for every load when it comes back)
  auto here = [](int x) {
    asm volatile("" : "+v"(x));
    return x;
  };
  // this lane's K operand (row n, chunk hf) and V operand (row 4 hf + lane % 16 / 4, eight bytes of a 16-feature group);
  // the chunk's number is in bits that the rows' pitch leaves free, so that later chunks are an exclusive or away
  const int k_at = n * RB + k_chunk<D>(n, hf) * 16;
  const int v_row = 4 * hf + ((lane & 15) >> 2);
  const int v_at = v_row * RB + v_chunk<D>(v_row, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + 8 * (lane & 1);

  // element j of s[t]: key 32 t + 8 (j / 4) + 4 hf + j % 4
  auto read_keys = [&](const unsigned char* kt, int k_at, int c, u32x4* kf) {
#pragma unroll
    for (int t = 0; t < 2; ++t) kf[t] = *reinterpret_cast<const u32x4*>(kt + (k_at ^ (32 * c)) + 32 * t * RB);
  };
  auto all_there = [&](int buf) {
    uint32_t every = lds_there[buf][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) every &= lds_there[buf][w];
    return __builtin_amdgcn_readfirstlane(every) == (1u << RW) - 1;
  };
  // scores of keys that this lane's row does not see
  auto hide = [&](int buf, int kb, f32x16* s) {
    uint64_t there = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) there |= (uint64_t)__builtin_amdgcn_readfirstlane(lds_there[buf][w]) << (RW * w);
    const uint64_t see = there & below(hi - kb) & ~below(lo - kb);
    const uint32_t seen[2] = {(uint32_t)see >> (4 * hf), (uint32_t)(see >> 32) >> (4 * hf)};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 16; ++j) s[t][j] = (seen[t] >> (8 * (j / 4) + j % 4)) & 1 ? s[t][j] : -INFINITY;
  };
  auto move_reference = [&](float mx) {
    if (__any(mx > m + kRescale)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      const bool move = mx > m + kRescale;  // (row by row: no row's bits depend on another's scores)
      const float f = move ? __builtin_amdgcn_exp2f(m - mx) : 1.0f;
      m = move ? mx : m;
      l *= f;
#pragma unroll
      for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[ft][j] *= f;
    }
  };
  auto form = [&](const unsigned char* kt, f32x16* s) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 16; ++j) s[t][j] = 0.0f;
    u32x4 kf[2][2];
    read_keys(kt, k_at, 0, kf[0]);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      if (c + 1 < D / 16) read_keys(kt, k_at, c + 1, kf[(c + 1) & 1]);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[c & 1][t]), qf[c], s[t], 0, 0, 0);
      if (c % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto maximum = [&](const f32x16* s) {
    float mx = s[0][0];
#pragma unroll
    for (int j = 1; j < 32; ++j) mx = fmaxf(mx, s[j >> 4][j & 15]);
    return mx * c_abs;
  };
  u32x4 pf[4];
  // The weights of the scores sc of the 64 keys at kb, and beside them the scores sn of the next 64.
  auto weigh = [&](f32x16* sc, f32x16* sn, int kb, int buf) {
    const unsigned char* kt = tile_k(buf ^ 1);
    const float ref = m == -INFINITY ? 0.0f : m;
    constexpr int NK = D / 16, PER = 32 / (2 * NK);  // weights beside a product
    const int ka = here(k_at);
    u32x4 kf[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 16; ++j) sn[t][j] = 0.0f;
    read_keys(kt, ka, 0, kf[0]);
    const bool whole = kb + kTileKeys >= u0 && kb + 2 * kTileKeys <= u1 && all_there(buf ^ 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < NK; ++c) {
      if (c + 1 < NK) read_keys(kt, ka, c + 1, kf[(c + 1) & 1]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sn[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[c & 1][t]), qf[c], sn[t], 0, 0, 0);
#pragma unroll
        for (int e0 = 0; e0 < PER; e0 += 2) {
          const int at = (2 * c + t) * PER + e0, h = at / 16, j = at % 16;
          float p[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            p[e] = __builtin_amdgcn_exp2f(fmaf(sc[h][j + e], c_abs, -ref));
            l += p[e];
          }
          pf[at / 8][at % 8 / 2] = pack_bf16x2(p[0], p[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // (the weights stay beside the products: not sunk to where they are used)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(pf[ks]));
    asm volatile("" : "+v"(l));
    if (!whole) hide(buf ^ 1, kb + kTileKeys, sn);
  };
  // The weights' product with the values, and beside it the maximum of the scores sn, for which the reference then moves.
  auto add_up = [&](f32x16* sn, const unsigned char* vt) {
    const int va = here(v_at);
    constexpr int FT = D / 32, NV = 4 * FT;
    u32x4 vf[3];
    auto read_value = [&](int u) {
      u32x4 v;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // 4 keys x 16 features of each group of 16 lanes
        const unsigned char* x = vt + (va ^ (64 * (u % FT))) + (16 * (u / FT) + 8 * e) * RB;
        const uint2 c = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(KVC_LDS(s16x4, x)));
        v[2 * e] = c.x;
        v[2 * e + 1] = c.y;
      }
      return v;
    };
    __builtin_amdgcn_sched_barrier(0);
    vf[0] = read_value(0);
    vf[1] = read_value(1);
    __builtin_amdgcn_sched_barrier(0);
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (u + 2 < NV) vf[(u + 2) % 3] = read_value(u + 2);
      o[u % FT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[u % 3]), as_bf16x8(pf[u / FT]), o[u % FT], 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 32 / NV; e += 2) {
        const int at = 32 / NV * u + e;
        mx = fmaxf(fmaxf(mx, sn[at / 16][at % 16]), sn[at / 16][at % 16 + 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    move_reference(mx * c_abs);
  };

  int64_t off_k[NC], off_v[NC];  // rows of the next loads
  Row row_k = {}, row_v = {}, row_n = {};
  f32x16 s0[2], s1[2];
  auto landed = [] { __builtin_amdgcn_s_waitcnt(0x0f70); };  // (loads into LDS are counted with the others)
  // the first tiles: everything that does not wait for something else is asked for at once
  int entry0 = 0, at0 = 0, entry1 = 0, at1 = 0;
  if (steps > 0) {
    fetch(begin);
    entry0 = entry, at0 = at;
    fetch(begin + kTileKeys);
    entry1 = entry, at1 = at;
    fetch(begin + 2 * kTileKeys);
  }
  u32x4 qx[D / 16];
  const char* qp = a.q + (int64_t)(sq.start + token) * a.q_token_stride + (int64_t)qh * a.q_head_stride;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) qx[s] = load16((GlobalPtr)qp + (2 * s + hf) * 16);
  if (tid == 0) lds_odd = 0;
  __syncthreads();
  if (steps > 0) {
    const int entry2 = entry, at2 = at;
    entry = entry0, at = at0;
    row_v = take(begin);
    entry = entry1, at = at1;
    row_k = take(begin + kTileKeys);
    entry = entry2, at = at2;
#pragma unroll
    for (int j = 0; j < NC; ++j) off_v[j] = row_bytes(row_v, j);
#pragma unroll
    for (int j = 0; j < NC; ++j) off_k[j] = row_bytes(row_k, j);
    load_lds(kp, off_v, tile_k(0), false);
    load_lds(vp, off_v, tile_v(0), true);
    load_lds(kp, off_k, tile_k(1), false);
    mark(0, row_v);
    mark(1, row_k);
    row_n = take(begin + 2 * kTileKeys);
    fetch(begin + 3 * kTileKeys);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      off_v[j] = off_k[j];
      off_k[j] = row_bytes(row_n, j);
    }
    landed();
    mend(tile_v(0), row_v, begin);
  }
#pragma unroll
  for (int s = 0; s < D / 16; ++s) qf[s] = as_bf16x8((qx[s] ^ q_sign) & q_keep);
  if (steps > 0) {
    __syncthreads();
    if (w_rows > 0) {
      form(tile_k(0), s0);
      if (!(begin >= u0 && begin + kTileKeys <= u1 && all_there(0))) hide(0, begin, s0);
      move_reference(maximum(s0));
    }
    __syncthreads();
  }
  const bool second = TURNS && wave >= 4;
  auto turn = [&](int i, int buf, int vbuf, f32x16* sc, f32x16* sn) {
    constexpr int VB = TURNS ? 4 : 2;
    const int kb = begin + i * kTileKeys;
    // V of the next tile, K of the one after it
    row_v = row_k;
    row_k = row_n;
    load_lds(vp, off_v, tile_v((vbuf + 1) % VB), true);
    load_lds(kp, off_k, tile_k(buf), false);
    row_n = take(kb + 3 * kTileKeys);
    fetch(kb + 4 * kTileKeys);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      off_v[j] = off_k[j];
      off_k[j] = row_bytes(row_n, j);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (second && i > 0 && w_rows > 0 && kb - kTileKeys < w_hi) add_up(sc, tile_v((vbuf + VB - 1) % VB));
    if (w_rows > 0 && kb < w_hi) {
      weigh(sc, sn, kb, buf);
      if (!second) add_up(sn, tile_v(vbuf));
    }
    mark(buf, row_k);
    landed();
    mend(tile_v((vbuf + 1) % VB), row_v, kb + kTileKeys);
    __syncthreads();
  };
  if constexpr (TURNS) {
    for (int i = 0; i < steps; i += 4) {
      turn(i, 0, 0, s0, s1);
      if (i + 1 >= steps) break;
      turn(i + 1, 1, 1, s1, s0);
      if (i + 2 >= steps) break;
      turn(i + 2, 0, 2, s0, s1);
      if (i + 3 >= steps) break;
      turn(i + 3, 1, 3, s1, s0);
    }
    const int last = begin + (steps - 1) * kTileKeys;
    if (second && steps > 0 && w_rows > 0 && last < w_hi) {
      f32x16 sn[2] = {steps & 1 ? s1[0] : s0[0], steps & 1 ? s1[1] : s0[1]};  // (all hidden)
      const int b = (steps - 1) & 3;
      if (b == 0) add_up(sn, lds_v0);
      if (b == 1) add_up(sn, lds_v1);
      if (b == 2) add_up(sn, lds_v2);
      if (b == 3) add_up(sn, lds_v3);
    }
  } else {
    for (int i = 0; i < steps; i += 2) {
      turn(i, 0, 0, s0, s1);
      if (i + 1 >= steps) break;
      turn(i + 1, 1, 1, s1, s0);
    }
  }

  if (w_rows > 0 && lds_odd) {
    const float ref = m == -INFINITY ? 0.0f : m;
    for (int key = max(begin, w_lo); key < min(end, w_hi); ++key) {
      const int kb = begin + (key - begin) / kTileKeys * kTileKeys;
      int slot_of;
      const int32_t b = step_block(a.pv, table, sq.off + key, slot_of);
      // (a tile that all rows of the workgroup see took the values as they are)
      if (b < 0 || (kb >= t_u0 && kb + kTileKeys <= t_u1)) continue;
      const int64_t off = slot_bytes(a.pv, b, slot_of);
      odd_values<D, false, 2>((GlobalPtr)qp, kp + off, vp + off, hf, a.scale_log2, ref, key >= lo && key < hi, [&](auto v) {
#pragma unroll
        for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[ft][j] += v(32 * ft + 8 * (j / 4) + 4 * hf + j % 4);
      });
    }
  }
  l += __shfl_xor(l, 32, kWave);
  if (!has_row) return;
  const int64_t flat = (int64_t)(sq.start + token) * a.num_heads + qh;
  if (l == 0.0f) l = without_weights<D>(o);
  if (a.splits > 1) {
    const int64_t at_s = (int64_t)split * a.step.num_rows * a.num_heads + flat;
    if (hf == 0) a.part_ml[at_s] = make_float2(m, l);
    if (holds_part(l)) {
#pragma unroll
      for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          *reinterpret_cast<f32x4*>(a.part_o + at_s * D + 32 * ft + 2 * j + 4 * hf) =
              f32x4{o[ft][j], o[ft][j + 1], o[ft][j + 2], o[ft][j + 3]};
    }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (l == 0.0f) {
#pragma unroll
    for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[ft][j] = 0.0f;
  }
  char* op = a.out + (int64_t)(sq.start + token) * a.out_token_stride + (int64_t)qh * a.out_head_stride;
#pragma unroll
  for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
    for (int j = 0; j < 16; j += 8) write_features(op + (32 * ft + 2 * j) * 2, hf, &o[ft], j, inv);
  if (a.lse && hf == 0)
    a.lse[flat] = l == 0.0f ? -INFINITY : (m == -INFINITY ? 0.0f : m) * 0.69314718055994531f + logf(l);
}

// The same over an 8-bit cache: codes are widened to bf16 (exactly) on their way through registers into LDS, two tiles of K
// and V of which take turns, and scores and weights are multiplied by the keys' scales.  2048 new tokens at the end of 32768
// keys, 32 heads on 8 (1.07 TFLOP): 1190 us, 900 TFLOP/s, bound by the vector unit (49 %) beside the matrix unit (36 %),
// which a wave uses in turn.  Scores formed a step ahead as above took 1298 us: the scales and the loads in registers leave
// none for a second set of scores.
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, WAVES == 8 ? 1 : 2) void attend_codes(AttendArgs a) {
  constexpr int BM = WAVES * 32;
  constexpr int RC = D / 16;          // 16-byte chunks of a row in memory
  constexpr int RPL = kWave / RC;          // rows of a wave's load
  constexpr int RW = kTileKeys / WAVES;    // rows of a tile that a wave brings in
  constexpr int NC = RW > RPL ? RW / RPL : 1;  // its loads, of K and of V
  constexpr bool SPARE = RPL > RW;         // (a load's lanes beyond the wave's rows idle)
  static_assert(NC <= RC, "lane j of a row's lanes holds the address of load j");
  constexpr int RB = D * 2;                // bytes of a row in LDS
  constexpr int HALF = kTileKeys * RB;     // bytes of a K (V) tile
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][2][HALF];  // [buffer][K, V]
  __shared__ float lds_scale[2][2][kTileKeys];
  __shared__ uint32_t lds_there[2][WAVES];  // bit r: row r of the wave's rows of the tile is there

  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);  // (what goes by it is in scalar registers)
  const int n = lane & 31, hf = lane >> 5;
  const int head = blockIdx.x, split = blockIdx.y;
  // (later tiles of a sequence see more keys: they go first)
  const Tile tile = find_tile<BM>(a, a.tile0 + gridDim.z - 1 - blockIdx.z);
  if (tile.rows <= 0) return;
  const SeqView& sq = tile.s;
  const int g = a.group;

  int t_lo, t_hi, t_u0, t_u1;  // the keys that any row sees, and those that all of them see
  visible(a, sq, quotient(tile.row0, a.by_group), t_lo, t_u1);
  visible(a, sq, quotient(tile.row0 + tile.rows - 1, a.by_group), t_u0, t_hi);
  const int begin = t_lo + split * a.chunk;
  const int end = min(t_hi, begin + a.chunk);
  const int steps = end > begin ? (end - begin + kTileKeys - 1) / kTileKeys : 0;

  // this wave's rows, the keys that any and that all of them see, and this lane's row
  const int w_rows = min(32, tile.rows - wave * 32), w_row0 = tile.row0 + wave * 32;
  const bool has_row = n < w_rows;
  const int row = w_rows > 0 ? w_row0 + (has_row ? n : 0) : tile.row0;
  const int token = quotient(row, a.by_group), qh = head * g + row - token * g;
  int lo = 0, hi = 0, w_lo = 0, w_hi = 0, u0 = 0, u1 = 0;
  if (has_row) visible(a, sq, token, lo, hi);
  if (w_rows > 0) {
    visible(a, sq, quotient(w_row0, a.by_group), w_lo, u1);
    visible(a, sq, quotient(w_row0 + w_rows - 1, a.by_group), u0, w_hi);
  }

  // Scores are acc * c with c > 0, so that their order is that of the accumulators: a negative scale's sign goes to Q, and
  // with a scale of zero Q is zero.
  const float c_abs = a.scale_log2 == 0.0f ? 1.0f : fabsf(a.scale_log2);
  const uint32_t q_sign = a.scale_log2 < 0.0f ? 0x80008000u : 0u, q_keep = a.scale_log2 == 0.0f ? 0u : ~0u;
  bf16x8 qf[D / 16];
  const char* qp = a.q + (int64_t)(sq.start + token) * a.q_token_stride + (int64_t)qh * a.q_head_stride;
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    qf[s] = as_bf16x8((load16((GlobalPtr)qp + (2 * s + hf) * 16) ^ q_sign) & q_keep);
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  const int32_t* table = a.step.tables ? a.step.tables + (int64_t)tile.seq * a.step.max_blocks : nullptr;
  const GlobalPtr kp = (GlobalPtr)a.k + head * a.pv.head_bytes;
  const GlobalPtr vp = (GlobalPtr)a.v + head * a.pv.head_bytes;
  // Load j of a wave brings in rows RW wave + RPL j .. of the tile, RC lanes a row.  A row's address is worked out by one
  // lane: lane j of a row's RC lanes has that of load j (lanes beyond NC repeat it), and passes it to the others.
  const int c_row = lane / RC, c_col = lane % RC;
  const bool lane_on = !SPARE || c_row < RW;
  const int my_row = RW * wave + RPL * (c_col % NC) + (SPARE ? c_row % RW : c_row);
  u32x4 kr[NC], vr[NC];
  int entry, at;        // table entry and slot of my_row of the next tile
  bool ok = false;      // my_row of the tile in the registers is there
  float scale_r = 0.0f;
  auto fetch = [&](int kb) { entry = step_entry(a.pv, table, sq.off + min(kb + my_row, end - 1), at); };
  // loads the tile at kb, and fetches the entries of the one after it first (they are older than the next loads)
  auto load = [&](int kb) {
    ok = kb + my_row < end && (uint32_t)entry < (uint32_t)a.pv.num_blocks;
    const int blk = ok ? entry : 0, slot_of = at;  // (a row that is not there: any, as zeros follow)
    const int64_t off = slot_bytes(a.pv, blk, slot_of);
    fetch(kb + kTileKeys);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const uint32_t lo32 = row_lane<RC>((uint32_t)off, j), hi32 = row_lane<RC>((uint32_t)((uint64_t)off >> 32), j);
      const int64_t at_j = (int64_t)(((uint64_t)hi32 << 32) | lo32) + c_col * 16;
      kr[j] = load16(kp + at_j);
      vr[j] = load16(vp + at_j);
    }
    if (c_col < 2 * NC) {
      const GlobalPtr sp = (GlobalPtr)(c_col < NC ? a.ks : a.vs) + head * a.pv.shead_bytes;
      scale_r = ok ? load_float(sp + slot_scale_bytes(a.pv, blk, slot_of)) : 0.0f;
    }
  };
  auto store = [&](int buf, int kb) {
    const uint64_t have = __ballot(ok);
    uint32_t bits = (1u << RW) - 1;  // bit r: row r of the wave's
    if (have != ~0ull) {
      bits = 0;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
#pragma unroll
        for (int r = 0; r < (SPARE ? RW : RPL); ++r) bits |= ((uint32_t)(have >> (r * RC + j)) & 1u) << (RPL * j + r);
        const bool ok_j = row_lane<RC>(ok ? 1u : 0u, j) != 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) vr[j][e] = ok_j ? vr[j][e] : 0u;
      }
    }
    if (lane == 0) lds_there[buf][wave] = bits;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      if (!lane_on) continue;
      const int r = RW * wave + RPL * j + c_row;
      unsigned char* kd = &lds[buf][0][r * RB];
      unsigned char* vd = &lds[buf][1][r * RB];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4 x, y;
        uint32_t p, q;
        widen_codes(kr[j][2 * e], p, q);
        x[0] = p;
        x[1] = q;
        widen_codes(kr[j][2 * e + 1], p, q);
        x[2] = p;
        x[3] = q;
        widen_codes(vr[j][2 * e], p, q);
        y[0] = p;
        y[1] = q;
        widen_codes(vr[j][2 * e + 1], p, q);
        y[2] = p;
        y[3] = q;
        *reinterpret_cast<u32x4*>(kd + k_chunk<D>(r, 2 * c_col + e) * 16) = x;
        *reinterpret_cast<u32x4*>(vd + v_chunk<D>(r, 2 * c_col + e) * 16) = y;
      }
    }
    if (lane_on && c_col < 2 * NC) lds_scale[buf][c_col < NC ? 0 : 1][my_row] = c_col < NC ? scale_r * c_abs : scale_r;
  };
  // this lane's K operand (row n, chunk hf) and V operand (row 4 hf + lane % 16 / 4, eight bytes of a 16-feature group);
  // the chunk's number is in bits that the rows' pitch leaves free, so that later chunks are an exclusive or away
  const int k_at = n * RB + k_chunk<D>(n, hf) * 16;
  const int v_row = 4 * hf + ((lane & 15) >> 2);
  const int v_at = v_row * RB + v_chunk<D>(v_row, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + 8 * (lane & 1);
  if (steps > 0) {
    fetch(begin);
    load(begin);
    store(0, begin);
  }
  __syncthreads();
  for (int i = 0; i < steps; ++i) {
    const int buf = i & 1, kb = begin + i * kTileKeys;
    const bool busy = w_rows > 0 && kb < w_hi && kb + kTileKeys > w_lo;
    if (!busy && i + 1 < steps) load(kb + kTileKeys);
    if (busy) {
      uint32_t words[WAVES];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) words[w] = lds_there[buf][w];
      const unsigned char* kt = lds[buf][0];
      const unsigned char* vt = lds[buf][1];
      f32x16 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[t][j] = 0.0f;
      f32x4 sk[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) sk[j] = *reinterpret_cast<const f32x4*>(&lds_scale[buf][0][8 * j + 4 * hf]);
      {
        u32x4 kf[2][2];
        auto read_keys = [&](int c) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
            kf[c & 1][t] = *reinterpret_cast<const u32x4*>(kt + (k_at ^ (32 * c)) + 32 * t * RB);
        };
        read_keys(0);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          if (c + 1 < D / 16) read_keys(c + 1);
#pragma unroll
          for (int t = 0; t < 2; ++t)
            s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[c & 1][t]), qf[c], s[t], 0, 0, 0);
          if (c % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < steps) load(kb + kTileKeys);
      uint32_t every = words[0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) every &= words[w];
      const bool whole = kb >= u0 && kb + kTileKeys <= u1 && __builtin_amdgcn_readfirstlane(every) == (1u << RW) - 1;
      // what this lane's row sees of its keys 8 q + 4 hf + i: bits 8 q + i of a word for each half of the tile
      uint32_t seen[2] = {~0u, ~0u};
      if (!whole) {
        uint64_t there = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) there |= (uint64_t)__builtin_amdgcn_readfirstlane(words[w]) << (RW * w);
        const uint64_t see = there & below(hi - kb) & ~below(lo - kb);
        seen[0] = (uint32_t)see >> (4 * hf);
        seen[1] = (uint32_t)(see >> 32) >> (4 * hf);
      }
      // element j of s[t]: key 32 t + 8 (j / 4) + 4 hf + j % 4; from here on, what enters the exponential under the reference
      // so far (one operation a score with its key's scale, where scaling and subtracting apart would be two)
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[t][j] = fmaf(s[t][j], sk[4 * t + j / 4][j % 4], -ref);
#pragma unroll
      for (int j = 0; j < 8; ++j) sk[j] = *reinterpret_cast<const f32x4*>(&lds_scale[buf][1][8 * j + 4 * hf]);
      if (!whole) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            s[t][j] = (seen[t] >> (8 * (j / 4) + j % 4)) & 1 ? s[t][j] : -INFINITY;
          }
      }
      float mx = s[0][0];
#pragma unroll
      for (int j = 1; j < 32; ++j) mx = fmaxf(mx, s[j >> 4][j & 15]);
      const float limit = m == -INFINITY ? -INFINITY : kRescale;
      if (__any(mx > limit)) {
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        const bool move = mx > limit;  // (row by row: no row's bits depend on another's scores)
        const float top = move ? ref + mx : m, by = move ? top - ref : 0.0f;
        const float f = move ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
        m = top;
        l *= f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int j = 0; j < 16; ++j) s[t][j] -= by;
#pragma unroll
        for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[ft][j] *= f;
      }
      u32x4 pf[4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        float p[8];
        const int t = ks >> 1, j0 = 8 * (ks & 1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(s[t][j0 + e]);
          l += p[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] *= sk[2 * ks + e / 4][e % 4];
        if (!whole) {  // (a scale that is no number belongs to those that see its key)
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = (seen[t] >> (16 * (ks & 1) + 8 * (e / 4) + e % 4)) & 1 ? p[e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[ks][e] = pack_bf16x2(p[2 * e], p[2 * e + 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
      {
        u32x4 vf[2][D / 32];
        auto read_values = [&](int ks) {
#pragma unroll
          for (int ft = 0; ft < D / 32; ++ft) {
            u32x4& v = vf[ks & 1][ft];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // 4 keys x 16 features of each group of 16 lanes
              const unsigned char* x = vt + (v_at ^ (64 * ft)) + (16 * ks + 8 * e) * RB;
              const uint2 c =
                  __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(KVC_LDS(s16x4, x)));
              v[2 * e] = c.x;
              v[2 * e + 1] = c.y;
            }
          }
        };
        read_values(0);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          if (ks < 3) read_values(ks + 1);
#pragma unroll
          for (int ft = 0; ft < D / 32; ++ft)
            o[ft] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[ks & 1][ft]), as_bf16x8(pf[ks]), o[ft], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (i + 1 < steps) store(buf ^ 1, kb + kTileKeys);
    __syncthreads();
  }

  l += __shfl_xor(l, 32, kWave);
  if (!has_row) return;
  const int64_t flat = (int64_t)(sq.start + token) * a.num_heads + qh;
  if (l == 0.0f) l = without_weights<D>(o);
  if (a.splits > 1) {
    const int64_t at_s = (int64_t)split * a.step.num_rows * a.num_heads + flat;
    if (hf == 0) a.part_ml[at_s] = make_float2(m, l);
    if (holds_part(l)) {
#pragma unroll
      for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          *reinterpret_cast<f32x4*>(a.part_o + at_s * D + 32 * ft + 2 * j + 4 * hf) =
              f32x4{o[ft][j], o[ft][j + 1], o[ft][j + 2], o[ft][j + 3]};
    }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (l == 0.0f) {
#pragma unroll
    for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[ft][j] = 0.0f;
  }
  char* op = a.out + (int64_t)(sq.start + token) * a.out_token_stride + (int64_t)qh * a.out_head_stride;
#pragma unroll
  for (int ft = 0; ft < D / 32; ++ft)
#pragma unroll
    for (int j = 0; j < 16; j += 8) write_features(op + (32 * ft + 2 * j) * 2, hf, &o[ft], j, inv);
  if (a.lse && hf == 0)
    a.lse[flat] = l == 0.0f ? -INFINITY : (m == -INFINITY ? 0.0f : m) * 0.69314718055994531f + logf(l);
}

// Whether token row `token` belongs to a sequence that was worked on.
__device__ __forceinline__ bool step_has(const AttendArgs& a, int token) {
  SeqView sq;
  return step_find_row(a.step, token, sq) >= 0 && sq.ok;
}

// The result of a row from its sum and its features f0 .. f0 + 3 (first: of the lane that writes the logarithm).
template <bool F32>
__device__ __forceinline__ void write_row(const AttendArgs& a, int flat, int f0, bool first, float top, float sum,
                                          const f32x4& o) {
  const int token = quotient(flat, a.by_heads), h = flat - token * a.num_heads;
  const float inv = 1.0f / sum;
  f32x4 x;
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = sum == 0.0f ? 0.0f : o[j] * inv;
  char* op = a.out + (int64_t)token * a.out_token_stride + (int64_t)h * a.out_head_stride;
  if constexpr (F32) *reinterpret_cast<f32x4*>(op + f0 * 4) = x;
  else *reinterpret_cast<uint2*>(op + f0 * 2) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  if (a.lse && first)
    a.lse[flat] = sum == 0.0f ? -INFINITY : (top == -INFINITY ? 0.0f : top) * 0.69314718055994531f + logf(sum);
}
// Weight of a range that holds a part (one without a maximum holds nothing but what is no number).  It multiplies a part also
// where it is zero, since a NaN is one however far its range lies below the row's maximum.
__device__ __forceinline__ float range_weight(const float2& ml, float top) {
  return ml.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml.x - top);
}

// The ranges' partial results of a row, joined in their order.  Up to FEW ranges: D / 4 lanes a row, four features each,
// every load in flight at once, and beside them those that tell whether the row was worked on (what is read in vain is
// workspace).  3.4 us for 32 rows of eight ranges and 6 us for 2048 of thirteen: launch and latency.
template <int D, bool F32, int FEW>
__global__ __launch_bounds__(256) void attend_join_few(AttendArgs a) {
  constexpr int LANES = D / 4;
  const int rows = a.step.num_rows * a.num_heads;
  const int flat0 = a.flat0 + (int)blockIdx.x * (256 / LANES), lane = threadIdx.x % LANES;
  const int there = min(flat0 + (int)(threadIdx.x / LANES), rows - 1);  // (every lane takes part in the search)
  float2 ml[FEW];
  f32x4 v[FEW];
#pragma unroll
  for (int s = 0; s < FEW; ++s) {
    ml[s] = make_float2(-INFINITY, 0.0f);
    v[s] = f32x4{0, 0, 0, 0};
    if (s < a.splits) {
      const int64_t at = (int64_t)s * rows + there;
      ml[s] = a.part_ml[at];
      v[s] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + lane * 4);
    }
  }
  // (the rows of a wave: at most two tokens apart at one head, and a search serves one)
  bool has = false;
  const int wave_flat = min(flat0 + (int)(threadIdx.x & ~(kWave - 1)) / LANES, rows - 1);
#pragma unroll
  for (int r = 0; r < kWave / LANES; ++r) {
    const int token = quotient(min(wave_flat + r, rows - 1), a.by_heads);
    const bool ok = step_has(a, token);
    if (there == wave_flat + r) has = ok;
  }
  if ((int)(threadIdx.x / LANES) >= rows - flat0 || !has) return;
  float top = -INFINITY;
#pragma unroll
  for (int s = 0; s < FEW; ++s) top = fmaxf(top, ml[s].x);
  float sum = 0.0f;
  f32x4 o = {0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < FEW; ++s) {
    if (holds_part(ml[s].y)) {
      const float f = range_weight(ml[s], top);
      sum += ml[s].y * f;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += v[s][j] * f;
    }
  }
  write_row<F32>(a, there, lane * 4, lane == 0, top, sum, o);
}

// Many ranges: the four waves of a workgroup a row, a quarter of the ranges each.  Each lane reads the maxima of the
// ranges lane, lane + 64, ..; then D / 4 lanes hold four features each, and the 256 / D groups of them in each wave take
// its ranges in turn (their sums are added at the end, in a fixed order).  28 rows of 52 ranges: 3.9 us.
template <int D, bool F32>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a) {
  constexpr int LANES = D / 4, GROUPS = kWave / LANES;
  __shared__ float part[4][D + 4];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int rows = a.step.num_rows * a.num_heads;
  const int flat = a.flat0 + blockIdx.x;
  const int group = lane / LANES, f0 = (lane % LANES) * 4;
  // this wave's ranges [first, last)
  const int each = (a.splits + 3) / 4, first = wave * each, last = min(a.splits, first + each);
  float top = -INFINITY;
  for (int s = lane; s < a.splits; s += kWave) top = fmaxf(top, a.part_ml[(int64_t)s * rows + flat].x);
  const bool has = step_has(a, quotient(flat, a.by_heads));
#pragma unroll
  for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kWave));
  float sum = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  for (int s0 = first; s0 < last; s0 += kWave) {
    const int s = s0 + lane;
    const float2 ml = s < last ? a.part_ml[(int64_t)s * rows + flat] : make_float2(-INFINITY, 0.0f);
    const float f = range_weight(ml, top);
    const uint64_t parts = __ballot(holds_part(ml.y));
    if (holds_part(ml.y)) sum += ml.y * f;
    const int here = min(kWave, last - s0);
    constexpr int AHEAD = 8;
    for (int i0 = 0; i0 < here; i0 += AHEAD * GROUPS) {
      f32x4 v[AHEAD];
      float w[AHEAD];
      bool held[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int at = min(i0 + i * GROUPS + group, here - 1);
        v[i] = *reinterpret_cast<const f32x4*>(a.part_o + ((int64_t)(s0 + at) * rows + flat) * D + f0);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int at = i0 + i * GROUPS + group;
        w[i] = __shfl(f, at & (kWave - 1), kWave);
        held[i] = at < here && ((parts >> (at & (kWave - 1))) & 1);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += held[i] ? w[i] * v[i][j] : 0.0f;
    }
  }
#pragma unroll
  for (int x = 1; x < kWave; x *= 2) sum += __shfl_xor(sum, x, kWave);
#pragma unroll
  for (int x = LANES; x < kWave; x *= 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], x, kWave);
  if (group == 0) *reinterpret_cast<f32x4*>(&part[wave][f0]) = o;
  if (lane == 0) part[wave][D] = sum;
  __syncthreads();
  if (wave != 0 || group != 0 || !has) return;
  o = f32x4{0, 0, 0, 0};
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    o += *reinterpret_cast<const f32x4*>(&part[w][f0]);
    sum += part[w][D];
  }
  write_row<F32>(a, flat, f0, lane == 0, top, sum, o);
}

template <int D, int CACHE>
hipError_t launch(AttendArgs a, const AttendPlan& p, hipStream_t stream) {
  const int H = a.pv.num_kv_heads;
  constexpr int kMostTiles = 65535;  // of a launch
  for (a.tile0 = 0; a.tile0 < p.tiles; a.tile0 += kMostTiles) {
    const int tiles = std::min(kMostTiles, p.tiles - a.tile0);
    bool rows = true;
    if constexpr (CACHE != KVC_F32) {
      if (p.tile_rows > kRowTile) {
        const dim3 grid(H, p.splits, tiles);
        if constexpr (CACHE == KVC_I8) {
          if (p.tile_rows == kAttendTile) attend_codes<D, 8><<<grid, 8 * kWave, 0, stream>>>(a);
          else attend_codes<D, 4><<<grid, 4 * kWave, 0, stream>>>(a);
        } else {
          if (p.tile_rows == kAttendTile) attend_tiles<D, 8><<<grid, 8 * kWave, 0, stream>>>(a);
          else attend_tiles<D, 4><<<grid, 4 * kWave, 0, stream>>>(a);
        }
        rows = false;
      }
    }
    if (rows) attend_rows<D, CACHE><<<dim3(p.splits, H, tiles), kWaves * kWave, 0, stream>>>(a);
  }
  if (p.splits > 1) {
    constexpr bool F32 = CACHE == KVC_F32;
    const int64_t n = (int64_t)a.step.num_rows * a.num_heads;
    const int64_t each = p.splits <= 16 ? 1024 / D : 1;              // rows of a workgroup
    const int64_t most = ((INT64_C(1) << 32) / 256 - 1) * each;  // of a launch
    for (int64_t first = 0; first < n; first += most) {
      const unsigned groups = (unsigned)((std::min(most, n - first) + each - 1) / each);
      a.flat0 = (int32_t)first;
      if (p.splits <= 4) attend_join_few<D, F32, 4><<<groups, 256, 0, stream>>>(a);
      else if (p.splits <= 8) attend_join_few<D, F32, 8><<<groups, 256, 0, stream>>>(a);
      else if (p.splits <= 16) attend_join_few<D, F32, 16><<<groups, 256, 0, stream>>>(a);
      else attend_join<D, F32><<<groups, 256, 0, stream>>>(a);
    }
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_types(const AttendArgs& a, const AttendPlan& p, kvc_dtype cache, hipStream_t stream) {
  if (cache == KVC_F32) return launch<D, KVC_F32>(a, p, stream);
  return cache == KVC_BF16 ? launch<D, KVC_BF16>(a, p, stream) : launch<D, KVC_I8>(a, p, stream);
}

}  // namespace

AttendPlan plan_attend(kvc_dtype cache, int num_seqs, int num_rows, int max_new, int64_t span, int64_t max_span,
                       int num_kv_heads, int group, int head_dim) {
  AttendPlan p = {};
  const int64_t most = (int64_t)max_new * group;
  // Lists of up to one 16-row tile go to attend_rows, taller ones to attend_tiles or attend_codes (64 sequences of 8 new
  // tokens, 4 heads a KV head, 4096 keys: 198 us as 32 rows of a 128-row tile, 357 us as two 16-row tiles, which read the
  // keys twice).  There, 256 rows a workgroup share more of what is brought in (codes that are widened, above all), but one
  // of 128 rows, two of which share a CU, ends sooner, and more of them fill the chip.  So it goes by the turns of 64 keys
  // that there are to make in all, fewer of them where contexts are longer than what is new, so that the workgroups are
  // alike.  256 against 128 rows, one sequence of 32 heads on 8 (us): bf16, all of the context new, 512 tokens (0.5 K turns)
  // 25 and 19, 2048 (8 K) 66 and 59, 3000 (18 K) 101 and 99, 4096 (33 K) 160 and 173; bf16, 64 at 8192 keys (1 K) 32 and
  // 28, 128 at 8192 (2 K) 39 and 40, 300 at 16000 (10 K) 101 and 109; int8, 512 at 512 28 and 25, 1024 at 1024 (2 K) 44 and
  // 47, 2048 at 32768 (131 K) 1313 and 1517.
  const bool tiles = cache != KVC_F32 && most > kRowTile;
  auto tiles_of = [&](int rows) {
    return most <= rows ? (int64_t)num_seqs : (int64_t)num_rows * group / rows + num_seqs;
  };
  const int64_t all_turns = tiles_of(kAttendTile) * num_kv_heads * ((span + kTileKeys - 1) / kTileKeys);
  const int64_t enough = cache == KVC_I8 ? 1500 : span >= 2 * (int64_t)max_new ? 2000 : 20000;
  p.tile_rows = !tiles ? kRowTile : most > kAttendTile / 2 && all_turns >= enough ? kAttendTile : kAttendTile / 2;
  p.direct = most <= p.tile_rows;
  p.tiles = (int)tiles_of(p.tile_rows);
  const int64_t units = std::max<int64_t>(1, (int64_t)p.tiles * num_kv_heads);
  const int64_t step = tiles ? kTileKeys : kWaves * kStepKeys;  // keys of a workgroup's turn
  const int64_t turns = (span + step - 1) / step, most_turns = (max_span + step - 1) / step;
  int64_t per, most_splits;  // turns of a range; ranges that no shorter span has more of
  if (tiles) {
    // As many ranges as give every CU its workgroup, or two of the smaller ones, of at least eight turns (four: 24 against
    // 19 us for the 512 new tokens, 33 against 28 for the 64).
    // (Workgroups beyond those wait for a second round: tiles are counted without the spare ones, half of the sequences'
    // last ones being taken as there.)
    auto ranges = [&](int rows) {
      const int64_t count = ((int64_t)num_rows * group + rows - 1) / rows + (num_seqs - 1) / 2;
      return std::max<int64_t>(1, (rows == kAttendTile ? 256 : 512) / std::max<int64_t>(1, count * num_kv_heads));
    };
    const int64_t splits = ranges(p.tile_rows);
    per = std::max<int64_t>(8, (turns + splits - 1) / splits);
    most_splits = std::min(std::max(ranges(kAttendTile), ranges(kAttendTile / 2)), (most_turns + 7) / 8);
  } else {
    // Up to three turns are not worth a second launch (3 sequences of up to 257 new tokens and keys, float32, 64
    // features: 9.0 against 11.0 us; four turns of bf16 11.1 against 9.4), but float32 ones of 128 features take twice as
    // long (one token, two turns 14.7 against 13.8 us, three 18.6 against 13.9).  Otherwise as many ranges as give up to
    // 256 workgroups (one request of 32771 tokens, 28 heads on 4: 20 us with 52 ranges of five turns, 24 for up to 512
    // workgroups, 26 for 128).  Beyond these, at most ten turns a range where a sequence has up to kCutRows rows, since
    // the lengths of many sequences differ: 64 requests of 1K-16K tokens, bf16, 461 us at ten turns, 476 at eight, 571 at
    // 32; float32, 64 sequences of 8 new tokens 1354 us cut, 1664 whole, two of 64 at 4K and 20K keys 625 and 855.  The
    // parts are then a tenth of the keys and values at most (264 or 520 bytes a row, 1280 keys a range).  A chunk of more
    // rows has workgroups enough and would have a workspace of its rows times its context: float32, 32 heads on 8 of 128,
    // 8 sequences of 20-300 new tokens 2125 us whole, 2446 cut; 512 at 8192 keys 889 and 1191; 4096 at 4096 1907 and 4116
    // (with 273 MB), 4096 at 32768 26.8 and 34.4 ms (with 1.8 GB).
    constexpr int64_t kGroups = 256, kMostTurns = 10, kCutRows = 256;
    const bool cut = most <= kCutRows;
    per = std::max<int64_t>(1, (turns * units + kGroups - 1) / kGroups);
    per = std::min(cut ? kMostTurns : std::max<int64_t>(1, turns), per);
    if (turns <= (cache == KVC_F32 && head_dim == 128 ? 1 : 3)) per = std::max<int64_t>(1, turns);
    // (a range has kMostTurns where it is cut there, or at least turns * units / kGroups)
    most_splits = std::max(cut ? (most_turns + kMostTurns - 1) / kMostTurns : 1,
                           std::min(most_turns, (kGroups + units - 1) / units));
  }
  p.chunk = (int32_t)(per * step);
  p.splits = (int32_t)std::max<int64_t>(1, (turns + per - 1) / per);
  const size_t row_bytes = (size_t)num_rows * group * num_kv_heads * (head_dim * 4 + 8);
  p.bytes = p.splits > 1 ? p.splits * row_bytes : 0;
  p.most_bytes = most_splits > 1 ? most_splits * row_bytes : 0;
  return p;
}

hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, kvc_dtype cache, int head_dim, hipStream_t stream) {
  if (p.tiles == 0) return hipSuccess;
  return head_dim == 64 ? launch_types<64>(a, p, cache, stream) : launch_types<128>(a, p, cache, stream);
}

}  // namespace kvc
