// Query and key rows rotated to their positions (kvc_rotate): with c = factor cos(p f_i), s = factor sin(p f_i),
//
//   (x, y) -> (x c - y s, x s + y c)
//
// for the feature pairs i of every head of a token at position p.  Bound by HBM: each row is read and written once; 16384
// tokens of 32 and 8 bfloat16 heads of 128 (336 MB) 69 us, 4.9 TB/s, the rate of a large copy; 512 tokens 4.5 us, two loads
// one after the other and the sines between them.  Pairs that fill no whole pieces of 16 bytes (bfloat16: no multiple of 8) go
// element by element, the copied features with them, in loads and stores of two bytes: 16384 tokens with 20 of 128 features
// rotated 245 us, with 126 180, and 512 tokens 12.4.  The sines and cosines, which the heads of a token share, are formed once
// a token, by a workgroup a token; rows loaded ahead of them, two pieces a thread, took 117 us.  The angle
// is taken in turns, p * f_i / 2 pi with the frequency in two parts and the whole turns taken off in 64 bits, so that it
// stays right far beyond the positions at which p * f_i itself would lose its fraction in 32.
#include <algorithm>

#include "kvc_drafts.h"

namespace kvc {
namespace {

constexpr int kRotateThreads = 256;

// E elements of a row as floats.
template <int E, bool BF16>
struct Piece {
  float x[E];
  __device__ __forceinline__ void load(const char* p) {
    if constexpr (BF16 && E == 8) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo_to_f32(w[i]);
        x[2 * i + 1] = bf16_hi_to_f32(w[i]);
      }
    } else if constexpr (!BF16 && E == 4) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        x[i] = BF16 ? bf16_lo_to_f32(reinterpret_cast<const uint16_t*>(p)[i]) : reinterpret_cast<const float*>(p)[i];
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    if constexpr (BF16 && E == 8) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      *reinterpret_cast<u32x4*>(p) = w;
    } else if constexpr (!BF16 && E == 4) {
      *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if constexpr (BF16) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_bits(x[i]);
        else reinterpret_cast<float*>(p)[i] = x[i];
      }
    }
  }
};

// One workgroup: one token.  A thread takes E pairs of a head at a time; copies go by E elements.
template <int D, bool BF16, bool HALF, int E>
__global__ __launch_bounds__(kRotateThreads) void rotate_rows(RotateArgs a) {
  constexpr int ES = BF16 ? 2 : 4;
  __shared__ float cs[D / 2], sn[D / 2];
  const int token = a.token0 + blockIdx.x;
  if ((int)threadIdx.x < a.pairs) {
    const int i = threadIdx.x;
    const double p = a.sign * a.positions[token];
    const double t = p * a.turns[i][0], e = fma(p, a.turns[i][0], -t);
    double s, c;
    sincospi(2.0 * ((t - rint(t)) + fma(p, a.turns[i][1], e)), &s, &c);
    cs[i] = (float)(c * a.factor);
    sn[i] = (float)(s * a.factor);
  }
  __syncthreads();
  const int turned = a.pairs / E, copied = a.copy ? (D - 2 * a.pairs) / E : 0, each = turned + copied;
  const int tasks = (a.heads[0] + a.heads[1]) * each;
  for (int task = threadIdx.x; task < tasks; task += kRotateThreads) {
    int head = task / each;
    const int at = task - head * each;
    const int which = head >= a.heads[0];
    head -= which ? a.heads[0] : 0;
    const RotateRows& r = a.rows[which];
    const char* in = r.in + (int64_t)token * r.in_token + (int64_t)head * r.in_head;
    char* out = r.out + (int64_t)token * r.out_token + (int64_t)head * r.out_head;
    Piece<E, BF16> x, y;
    if (at >= turned) {
      const int f = 2 * a.pairs + (at - turned) * E;
      x.load(in + f * ES);
      x.store(out + f * ES);
    } else if (HALF) {
      const int i = at * E;
      x.load(in + i * ES);
      y.load(in + (i + a.pairs) * ES);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float u = x.x[e], v = y.x[e], c = cs[i + e], s = sn[i + e];
        x.x[e] = u * c - v * s;
        y.x[e] = u * s + v * c;
      }
      x.store(out + i * ES);
      y.store(out + (i + a.pairs) * ES);
    } else {
      const int i = at * E;
      x.load(in + 2 * i * ES);
      y.load(in + (2 * i + E) * ES);
      Piece<E, BF16> z[2] = {x, y};
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float& u = z[2 * e / E].x[2 * e % E];
        float& v = z[(2 * e + 1) / E].x[(2 * e + 1) % E];
        const float c = cs[i + e], s = sn[i + e], w = u;
        u = w * c - v * s;
        v = w * s + v * c;
      }
      z[0].store(out + 2 * i * ES);
      z[1].store(out + (2 * i + E) * ES);
    }
  }
}

template <int D, bool BF16, bool HALF>
hipError_t launch(RotateArgs a, hipStream_t stream) {
  constexpr int E = BF16 ? 8 : 4;  // elements of 16 bytes
  constexpr int32_t kMost = 1 << 23;  // (a grid's dimension ends at 2^32 threads)
  for (int32_t first = 0; first < a.num_rows; first += kMost) {
    a.token0 = first;
    const int groups = std::min(kMost, a.num_rows - first);
    // whole 16-byte pieces where the pairs are as many, otherwise an element at a time
    if (a.pairs % E == 0) rotate_rows<D, BF16, HALF, E><<<groups, kRotateThreads, 0, stream>>>(a);
    else rotate_rows<D, BF16, HALF, 1><<<groups, kRotateThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_types(const RotateArgs& a, kvc_dtype dtype, int style, hipStream_t stream) {
  if (style == KVC_ROPE_HALF)
    return dtype == KVC_BF16 ? launch<D, true, true>(a, stream) : launch<D, false, true>(a, stream);
  return dtype == KVC_BF16 ? launch<D, true, false>(a, stream) : launch<D, false, false>(a, stream);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, kvc_dtype dtype, int head_dim, int style, hipStream_t stream) {
  if (a.num_rows == 0 || a.heads[0] + a.heads[1] == 0) return hipSuccess;
  return head_dim == 64 ? launch_types<64>(a, dtype, style, stream) : launch_types<128>(a, dtype, style, stream);
}

}  // namespace kvc
