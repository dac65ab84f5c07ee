// Drafted tokens against the target's probabilities (kvc_verify).
//
// At the last accepted token, with P and Q the target's and the draft's probabilities, multi-round rejection leaves
// r_1 = max(0, P - Q) / T_1, then max(0, r_1 - Q) / T_2, and so on.  Since max(0, max(0, P - a Q) - T Q) =
// max(0, P - (a + T) Q) for T >= 0 and Q >= 0, what is left after any number of rejections is max(0, P - a Q) for one
// number a, up to its sum: nothing but a and that sum T is carried along.  Children stand behind their parents, so one
// ascending pass over a sequence's tokens meets the children of the last accepted one in their order.
//
// Everything is held in 64 bits: the next token is where a running sum of up to millions of probabilities passes a random
// share of the whole, and in 32 bits a rounding, 2^-24 of the sum, is 1/128 of a token's mean share of 131072.  Sums are
// cut into pieces of 2048 probabilities, a wave each, and joined in the pieces' order.
//
//   verify_rounds  (several drawn children a token) walks, with a workgroup a sequence summing P - a Q whenever another
//                  child is to be tried;
//   verify_sums    walks, or takes up where verify_rounds ended, and sums what is left there, all pieces at once;
//   verify_choose  finds the piece and the probability in it that pass the random share.
//
// 64 chains of four drawn tokens over 131072 probabilities (67 MB of the rows where the walks end): 15.4 us, and 6.0 us for
// the choice.  8 trees of 31 drawn tokens, rounds of two sums in the slowest walk: 14.6 us over 50021 probabilities, 22.4
// over 100042, 39.9 over 200000, on one CU a sequence (with one load a lane in flight 15.5, 23.8, 43.2); sums over several
// CUs would each need a launch, or a wait for other workgroups.  Tokens that were not drawn: the 64 chains 11.1 and 6.4 us,
// 8 trees of 31 over 50021 8.6 and 6.5.  There each token looks for an earlier sibling of its kind among all that lie between it
// and its parent, in every workgroup of the sequence: two trees of 1000 tokens, up to 956 of them one token's, over 131072 260 us.
#include <algorithm>

#include "kvc_drafts.h"

namespace kvc {
namespace {

constexpr int kSumThreads = 256, kRoundThreads = 1024;
constexpr int kRoundLoads = 4;  // loads of four of a lane in flight while a round is summed
constexpr int kPieceLoads = kVerifyPiece / (4 * kWave);  // loads of four of a lane

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// A probability as it counts: a positive finite number, or 0.
__device__ __forceinline__ float counting(float x) { return __builtin_amdgcn_classf(x, 0x180) ? x : 0.0f; }
__device__ __forceinline__ double weight(float x) { return (double)counting(x); }
__device__ __forceinline__ double random_number(float u) { return (double)fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f); }
__device__ __forceinline__ double left_over(double p, double a, double q) { return fmax(0.0, fma(-a, q, p)); }

// Four elements of a row of n that hold e .. e + 3, as far as there are any, in one load: from element `at` on, which lies
// before e at the row's end.  Those before e (and, of a row of less than four, those behind its end) do not count.
struct Four {
  f32x4u x;
  int at;
};
__device__ __forceinline__ Four load4(const float* row, int e, int n) {
  if (n >= 4) {
    const int at = min(e, n - 4);
    return {*reinterpret_cast<const f32x4u*>(row + at), at};
  }
  Four f = {{0, 0, 0, 0}, e};
  for (int i = 0; i < n; ++i)
    if (e == 0) f.x[i] = row[i];
  return f;
}
__device__ __forceinline__ double counted(const Four& f, int i, int e) { return f.at + i >= e ? weight(f.x[i]) : 0.0; }

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) x += __shfl_xor(x, m, kWave);
  return x;
}

// A sequence's tokens in LDS: what is asked of each against its parent's row.
struct Tokens {
  int32_t parent[KVC_MAX_TREE], token[KVC_MAX_TREE];
  float p[KVC_MAX_TREE], q[KVC_MAX_TREE], u[KVC_MAX_TREE];
};

template <bool DRAFT>
__device__ __forceinline__ void load_tokens(const VerifyArgs& a, const SeqView& sq, Tokens& t) {
  for (int j = threadIdx.x; j < sq.q; j += blockDim.x) {
    const int64_t row = (int64_t)sq.start + j;
    const int parent = a.parents[row], token = a.tokens[row];
    const bool there = parent >= 0 && parent < j && (uint32_t)token < (uint32_t)a.vocab;
    const int64_t above = sq.start + (there ? parent : 0), x = there ? token : 0;
    t.parent[j] = parent;
    t.token[j] = token;
    t.u[j] = a.uniforms[row];
    t.p[j] = there ? a.target[above * a.target_stride + x] : 0.0f;
    if constexpr (DRAFT) t.q[j] = there ? a.draft[above * a.draft_stride + x] : 0.0f;
  }
  __syncthreads();
  if constexpr (!DRAFT) {  // a token that an earlier sibling has is rejected by then, and nothing is left of it
    for (int j = threadIdx.x; j < sq.q; j += blockDim.x) {
      const int parent = t.parent[j], token = t.token[j];
      for (int b = max(parent, 0) + 1; parent >= 0 && b < j; ++b)
        if (t.parent[b] == parent && t.token[b] == token) t.p[j] = 0.0f;
    }
    __syncthreads();
  }
}

// The walk down a sequence's tree: every lane of the wave takes part.  again(at, a) gives the sum of what is left where
// another child may be tried; write(d, j) notes accepted token j.
struct Walk {
  int at = 0, count = 1, first = 0, last = -1;
  double a = 0.0;
};
template <bool DRAFT, class Again, class Write>
__device__ __forceinline__ Walk walk_tree(const VerifyArgs& v, const SeqView& sq, const Tokens& t, Again again,
                                          Write write) {
  const int lane = threadIdx.x & (kWave - 1);
  Walk w;
  double T = 1.0;
  int tried = 0;
  for (int c = 0; c < sq.q; c += kWave) {
    const int j0 = c + lane;
    const int parent = j0 > 0 && j0 < sq.q ? t.parent[j0] : -1;
    uint64_t open = ~0ull;  // tokens of these 64 that are not behind
    while (true) {
      const uint64_t kids = __ballot(parent == w.at) & open;
      if (!kids || (v.children && tried >= v.children)) break;
      const int i = __builtin_ctzll(kids), j = c + i;
      open = i == 63 ? 0ull : ~0ull << (i + 1);
      if (j <= w.at) continue;
      const double u = random_number(t.u[j]), p = weight(t.p[j]);
      bool yes;
      if constexpr (DRAFT) {
        if (tried > 0) T = again(w.at, w.a);
        const double q = weight(t.q[j]);
        yes = u * T * q < left_over(p, w.a, q);
        if (!yes) w.a += T;
      } else {
        yes = u * fmax(0.0, T) < p;
        if (!yes) T -= p;
      }
      if (yes) {
        write(w.count, j);
        w.at = j;
        ++w.count;
        w.a = 0.0;
        T = 1.0;
        tried = 0;
        w.last = -1;
      } else {
        ++tried;
        w.last = j;
      }
    }
  }
  w.first = w.at + 1;
  return w;
}

// The walk's results of sequence i, as one wave writes them.
__device__ __forceinline__ void write_walk(const VerifyArgs& a, const SeqView& sq, int seq, const Walk& w, bool draft) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int d = w.count + lane; d < sq.q; d += kWave) a.path[(int64_t)sq.start + d] = -1;
  if (lane == 0) {
    a.path[sq.start] = 0;
    a.counts[seq] = w.count;
    VerifyEnd e = {w.a, sq.start + w.at, sq.start + w.first, draft ? -1 : sq.start + w.last, 0};
    if (w.last < 0) e.last = -1;
    a.ends[seq] = e;
  }
}
__device__ __forceinline__ void write_nothing(const VerifyArgs& a, int seq) {
  if ((threadIdx.x & (kWave - 1)) == 0) {
    a.counts[seq] = 0;
    a.chosen[seq] = -1;
    a.ends[seq] = VerifyEnd{0.0, -1, 0, -1, 0};
  }
}

// Drafts drawn several to a token: one workgroup a sequence.
__global__ __launch_bounds__(kRoundThreads) void verify_rounds(VerifyArgs a) {
  __shared__ Tokens t;
  __shared__ double part[2][kRoundThreads / kWave];
  const int seq = a.seq0 + blockIdx.x;
  const SeqView sq = step_seq(a.step, seq);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  if (!sq.ok || sq.q == 0) {
    if (wave == 0) write_nothing(a, seq);
    return;
  }
  load_tokens<true>(a, sq, t);
  int turn = 0;
  // (every wave walks alike, since all of them come by the same numbers)
  const Walk w = walk_tree<true>(
      a, sq, t,
      [&](int at, double by) {
        const float* p = a.target + (int64_t)(sq.start + at) * a.target_stride;
        const float* q = a.draft + (int64_t)(sq.start + at) * a.draft_stride;
        double sum = 0.0;
        int e = 4 * threadIdx.x;
        const int first = 4 * (int)threadIdx.x;
        for (; e - first <= a.vocab - kRoundLoads * 4 * kRoundThreads; e += kRoundLoads * 4 * kRoundThreads) {
          f32x4u x[kRoundLoads], y[kRoundLoads];
#pragma unroll
          for (int i = 0; i < kRoundLoads; ++i) {
            x[i] = *reinterpret_cast<const f32x4u*>(p + e + 4 * kRoundThreads * i);
            y[i] = *reinterpret_cast<const f32x4u*>(q + e + 4 * kRoundThreads * i);
          }
#pragma unroll
          for (int i = 0; i < kRoundLoads; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += left_over(weight(x[i][k]), by, weight(y[i][k]));
        }
        for (; e - first <= a.vocab - 4 * kRoundThreads; e += 4 * kRoundThreads) {
          const f32x4u x = *reinterpret_cast<const f32x4u*>(p + e), y = *reinterpret_cast<const f32x4u*>(q + e);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum += left_over(weight(x[k]), by, weight(y[k]));
        }
        if (e < a.vocab) {
          const Four x = load4(p, e, a.vocab), y = load4(q, e, a.vocab);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum += left_over(counted(x, k, e), by, counted(y, k, e));
        }
        sum = wave_sum(sum);
        turn ^= 1;  // (the other places: those of the last sum may still be read)
        if (lane == 0) part[turn][wave] = sum;
        __syncthreads();
        double T = 0.0;
#pragma unroll
        for (int i = 0; i < kRoundThreads / kWave; ++i) T += part[turn][i];
        return T;
      },
      [&](int d, int j) {
        if (threadIdx.x == 0) a.path[(int64_t)sq.start + d] = j;
      });
  if (wave == 0) write_walk(a, sq, seq, w, true);
}

// Marks the tokens of a piece that rejected children have, one bit each, in the wave's own LDS.
__device__ __forceinline__ void mark_rejected(const VerifyArgs& a, const VerifyEnd& e, int start, int from,
                                              uint32_t* marks) {
  const int lane = threadIdx.x & (kWave - 1);
  marks[lane] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int j = e.first + lane; j <= e.last; j += kWave) {
    const uint32_t x = (uint32_t)(a.tokens[j] - from);
    if (a.parents[j] == e.at - start && x < (uint32_t)kVerifyPiece) atomicOr(&marks[x / 32], 1u << (x % 32));
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What is left of a piece's probabilities, four at a time: visit(i, at, left[4], whole[4]) for those from `at` on (see
// load4; what does not count is 0), and the probabilities themselves.
template <bool DRAFT, class Visit>
__device__ __forceinline__ void visit_piece(const VerifyArgs& a, const VerifyEnd& e, int from, const uint32_t* marks,
                                            Visit visit) {
  const int mine = from + 4 * (threadIdx.x & (kWave - 1));
  const float* p = a.target + (int64_t)e.at * a.target_stride;
  const float* q = DRAFT ? a.draft + (int64_t)e.at * a.draft_stride : nullptr;
  Four x[kPieceLoads], y[kPieceLoads] = {};
#pragma unroll
  for (int i = 0; i < kPieceLoads; ++i) x[i] = load4(p, mine + 4 * kWave * i, a.vocab);
  if (DRAFT && e.a > 0.0) {
#pragma unroll
    for (int i = 0; i < kPieceLoads; ++i) y[i] = load4(q, mine + 4 * kWave * i, a.vocab);
  }
#pragma unroll
  for (int i = 0; i < kPieceLoads; ++i) {
    const int at = x[i].at;
    double left[4], whole[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      whole[k] = counted(x[i], k, mine + 4 * kWave * i);
      if constexpr (DRAFT) {
        left[k] = left_over(whole[k], e.a, weight(y[i].x[k]));
      } else {
        const int bit = max(at + k - from, 0);
        left[k] = (marks[bit / 32] >> (bit % 32)) & 1 ? 0.0 : whole[k];
      }
    }
    visit(i, at, left, whole);
  }
}

// WALK: the walk is this kernel's own (every workgroup of a sequence does it for itself, the first writes its results).
template <bool DRAFT, bool WALK>
__global__ __launch_bounds__(kSumThreads) void verify_sums(VerifyArgs a) {
  __shared__ Tokens t;
  __shared__ VerifyEnd end;
  __shared__ uint32_t marks[kSumThreads / kWave][kWave];
  const int seq = a.seq0 + blockIdx.y;
  const SeqView sq = step_seq(a.step, seq);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  const bool first = blockIdx.x == 0;
  if (!sq.ok || sq.q == 0) {
    if (WALK && first && wave == 0) write_nothing(a, seq);
    return;
  }
  VerifyEnd e;
  if constexpr (WALK) {
    load_tokens<DRAFT>(a, sq, t);
    if (wave == 0) {
      // (one child is tried of drawn tokens: what is left has no part in that)
      const Walk w = walk_tree<DRAFT>(
          a, sq, t, [](int, double) { return 1.0; },
          [&](int d, int j) {
            if (first && lane == 0) a.path[(int64_t)sq.start + d] = j;
          });
      if (first) write_walk(a, sq, seq, w, DRAFT);
      if (lane == 0) end = VerifyEnd{w.a, sq.start + w.at, sq.start + w.first, w.last < 0 ? -1 : sq.start + w.last, 0};
    }
    __syncthreads();
    e = end;
  } else {
    e = a.ends[seq];
  }
  const int piece = blockIdx.x * (kSumThreads / kWave) + wave;
  if (piece >= a.pieces) return;
  const int from = piece * kVerifyPiece;
  if constexpr (!DRAFT) mark_rejected(a, e, sq.start, from, marks[wave]);
  double left = 0.0, whole = 0.0;
  visit_piece<DRAFT>(a, e, from, marks[wave], [&](int, int, const double* l, const double* w) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      left += l[k];
      whole += w[k];
    }
  });
  left = wave_sum(left);
  whole = wave_sum(whole);
  if (lane == 0) a.sums[(int64_t)seq * a.pieces + piece] = make_double2(left, whole);
}

// The running sums over the wave's lanes up to this one, of N numbers side by side.
template <int N>
__device__ __forceinline__ void wave_upto(double* x) {
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) {
    double y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __shfl_up(x[i], m, kWave);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane >= m ? y[i] : 0.0;
  }
}

// One wave a sequence.  Its lanes sum runs of pieces, the first lane whose running sum passes the share has the piece, and
// the same again within the piece: two scans, in which what is independent goes side by side.
template <bool DRAFT>
__global__ __launch_bounds__(kWave) void verify_choose(VerifyArgs a) {
  __shared__ uint32_t marks[kWave];
  const int seq = a.seq0 + blockIdx.x, lane = threadIdx.x;
  const double2* sums = a.sums + (int64_t)seq * a.pieces;
  const int run = (a.pieces + kWave - 1) / kWave;  // pieces of a lane
  // (whatever does not wait for something else is asked for at once: of a sequence that is left out, what lies there)
  double2 mine = {0.0, 0.0};
  for (int s = lane * run; s < min(a.pieces, (lane + 1) * run); ++s) {
    mine.x += sums[s].x;
    mine.y += sums[s].y;
  }
  const double random = random_number(a.last[seq]);
  const int start = a.step.starts[seq];
  VerifyEnd e = a.ends[seq];
  if (e.at < 0) return;
  double upto[2] = {mine.x, mine.y};
  wave_upto<2>(upto);
  const bool none = !(__shfl(upto[0], kWave - 1, kWave) > 0.0);  // nothing is left: the target's own
  const double total = __shfl(none ? upto[1] : upto[0], kWave - 1, kWave);
  if (!(total > 0.0)) {
    if (lane == 0) a.chosen[seq] = -1;
    return;
  }
  if (none) {
    e.a = 0.0;
    e.last = -1;
  }
  const double share = random * total;
  const double here = none ? mine.y : mine.x, up = none ? upto[1] : upto[0];
  // (the last lane that has anything, should rounding leave none whose sum passes)
  const uint64_t past = __ballot(up > share && here > 0.0), some = __ballot(here > 0.0);
  const int j = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
  double before = __shfl(up, j > 0 ? j - 1 : 0, kWave);
  if (j == 0) before = 0.0;
  int piece = j;
  double at_piece = before;
  if (run > 1) {
    for (int s = j * run; s < min(a.pieces, (j + 1) * run); ++s) {
      const double x = none ? sums[s].y : sums[s].x;
      if (x > 0.0) {
        piece = s;
        at_piece = before;
        if (before + x > share) break;
      }
      before += x;
    }
  }
  const int from = piece * kVerifyPiece;
  if constexpr (!DRAFT) mark_rejected(a, e, start, from, marks);
  double l[kPieceLoads][4], sum[kPieceLoads];
  int places[kPieceLoads];
  visit_piece<DRAFT>(a, e, from, marks, [&](int i, int at, const double* left, const double*) {
    places[i] = at;
#pragma unroll
    for (int k = 0; k < 4; ++k) l[i][k] = left[k];
    sum[i] = left[0] + left[1] + left[2] + left[3];
  });
  double end[kPieceLoads];
#pragma unroll
  for (int i = 0; i < kPieceLoads; ++i) end[i] = sum[i];
  wave_upto<kPieceLoads>(end);
  int found = -1, last = -1;
#pragma unroll
  for (int i = 0; i < kPieceLoads; ++i) {
    double x = at_piece + (end[i] - sum[i]);
    int first = -1, any = -1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x += l[i][k];
      if (l[i][k] > 0.0) {
        any = k;
        if (first < 0 && x > share) first = k;
      }
    }
    const uint64_t hits = __ballot(first >= 0), have = __ballot(any >= 0);
    if (hits && found < 0) found = __builtin_amdgcn_readlane(places[i] + first, __builtin_ctzll(hits));
    if (have) last = __builtin_amdgcn_readlane(places[i] + any, 63 - __builtin_clzll(have));
    at_piece += __shfl(end[i], kWave - 1, kWave);
  }
  if (lane == 0) a.chosen[seq] = found >= 0 ? found : last;
}

template <bool DRAFT>
hipError_t launch(VerifyArgs a, hipStream_t stream) {
  constexpr int32_t kMost = 65535;  // sequences of a launch (a grid's second dimension)
  constexpr int WAVES = kSumThreads / kWave;
  const bool rounds = DRAFT && a.children != 1;
  for (int32_t first = 0; first < a.step.num_seqs; first += kMost) {
    a.seq0 = first;
    const int32_t seqs = std::min(kMost, a.step.num_seqs - first);
    const dim3 grid((a.pieces + WAVES - 1) / WAVES, seqs);
    if (rounds) {
      verify_rounds<<<seqs, kRoundThreads, 0, stream>>>(a);
      verify_sums<DRAFT, false><<<grid, kSumThreads, 0, stream>>>(a);
    } else {
      verify_sums<DRAFT, true><<<grid, kSumThreads, 0, stream>>>(a);
    }
    verify_choose<DRAFT><<<seqs, kWave, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(VerifyArgs a, hipStream_t stream) {
  return a.draft ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace kvc
