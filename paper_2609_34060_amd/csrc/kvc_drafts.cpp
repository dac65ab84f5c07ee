// Host entry points of a step of drafted tokens (kvc_rotate, kvc_tree, kvc_verify, kvc_keep): argument checks and dispatch.
// Every check runs before anything is enqueued; on an error nothing is enqueued.
#include "kvc_drafts.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvc.h"
#include "kvc_check.h"

namespace {

using namespace kvc;

constexpr double kMostAngle = 65536.0;     // of a frequency, and of a factor
constexpr int32_t kMostVocab = 1 << 30;
constexpr int32_t kMostRows = 1 << 30;     // tokens that kvc_rotate counts through

kvc_status check_heads(const kvc_heads* h, const kvc_rotary* r) {
  const int64_t es = elem_size(r->dtype);
  if (h->reserved != 0 || h->num_heads < 0 || h->num_heads > 65535) return KVC_ERR_SHAPE;
  if (!in_range(0, h->in_token_stride, h->in_head_stride, h->out_token_stride, h->out_head_stride)) return KVC_ERR_SHAPE;
  if (h->num_heads == 0 || r->num_rows == 0) return KVC_OK;
  if ((r->num_rows > 1 && h->out_token_stride < r->head_dim) || (h->num_heads > 1 && h->out_head_stride < r->head_dim))
    return KVC_ERR_SHAPE;
  if (!h->in || !h->out) return KVC_ERR_NULL_ARG;
  if (!aligned(h->in, 16) || !aligned(h->out, 16) || (h->in_token_stride * es) % 16 || (h->in_head_stride * es) % 16 ||
      (h->out_token_stride * es) % 16 || (h->out_head_stride * es) % 16)
    return KVC_ERR_ALIGN;
  // results lie apart: all heads of a token before the next one's, or all tokens of a head (a < b c as a / b < c: b c may
  // pass 64 bits)
  if (r->num_rows > 1 && h->num_heads > 1 &&
      (h->out_token_stride - r->head_dim) / (h->num_heads - 1) < h->out_head_stride &&
      (h->out_head_stride - r->head_dim) / (r->num_rows - 1) < h->out_token_stride)
    return KVC_ERR_SHAPE;
  if (h->in == h->out && ((r->num_rows > 1 && h->in_token_stride != h->out_token_stride) ||
                          (h->num_heads > 1 && h->in_head_stride != h->out_head_stride)))
    return KVC_ERR_ALIAS;
  return KVC_OK;
}

RotateRows rotate_rows(const kvc_heads& h, int64_t es) {
  return {static_cast<const char*>(h.in), static_cast<char*>(h.out), h.in_token_stride * es, h.in_head_stride * es,
          h.out_token_stride * es,        h.out_head_stride * es};
}

int64_t verify_pieces(int32_t vocab) { return (static_cast<int64_t>(vocab) + kVerifyPiece - 1) / kVerifyPiece; }
size_t verify_ends_bytes(int32_t seqs) { return (seqs * sizeof(VerifyEnd) + 255) / 256 * 256; }

}  // namespace

extern "C" {

kvc_status kvc_rotate(const kvc_rotary* rotary, const kvc_heads* first, const kvc_heads* second, hipStream_t stream) {
  const kvc_rotary* r = rotary;
  if (!r || !first) return KVC_ERR_NULL_ARG;
  if (r->dtype != KVC_F32 && r->dtype != KVC_BF16) return KVC_ERR_DTYPE;
  if (r->head_dim != 64 && r->head_dim != 128) return KVC_ERR_UNSUPPORTED;
  if (r->style != KVC_ROPE_HALF && r->style != KVC_ROPE_PAIRS) return KVC_ERR_UNSUPPORTED;
  if (r->num_rows < 0 || r->num_rows > kMostRows || r->rotary_dim < 2 || r->rotary_dim > r->head_dim ||
      r->rotary_dim % 2 || r->inverse < 0 || r->inverse > 1 || !(std::fabs(r->factor) <= kMostAngle))
    return KVC_ERR_SHAPE;
  if (!r->inv_freq) return KVC_ERR_NULL_ARG;
  RotateArgs a = {};
  a.pairs = r->rotary_dim / 2;
  for (int32_t i = 0; i < a.pairs; ++i) {
    if (!(std::fabs(r->inv_freq[i]) <= kMostAngle)) return KVC_ERR_SHAPE;
    const long double turns = r->inv_freq[i] * 0.159154943091895335768883763372514362L;  // 1 / 2 pi
    a.turns[i][0] = static_cast<double>(turns);
    a.turns[i][1] = static_cast<double>(turns - a.turns[i][0]);
  }
  const int64_t es = elem_size(r->dtype);
  const kvc_heads* both[2] = {first, second};
  for (int i = 0; i < 2; ++i) {
    if (!both[i]) continue;
    const kvc_status s = check_heads(both[i], r);
    if (s != KVC_OK) return s;
    a.rows[i] = rotate_rows(*both[i], es);
    a.heads[i] = both[i]->num_heads;
    if (r->rotary_dim < r->head_dim && both[i]->in != both[i]->out) a.copy = 1;
  }
  if (r->num_rows == 0 || a.heads[0] + a.heads[1] == 0) return KVC_OK;
  if (a.heads[0] > 0 && a.heads[1] > 0 &&
      (first->out == second->out || first->out == second->in || first->in == second->out))
    return KVC_ERR_ALIAS;
  if (!r->positions) return KVC_ERR_NULL_ARG;
  if (!aligned(r->positions, 4)) return KVC_ERR_ALIGN;
  a.num_rows = r->num_rows;
  a.factor = r->factor;
  a.sign = r->inverse ? -1.0 : 1.0;
  a.positions = r->positions;
  return hip_status(launch_rotate(a, r->dtype, r->head_dim, r->style, stream));
}

kvc_status kvc_tree(const kvc_step* step, const int32_t* parents, uint64_t* masks, int32_t words, int32_t* positions,
                    hipStream_t stream) {
  const kvc_status s = check_step(nullptr, step);
  if (s != KVC_OK) return s;
  if (step->max_new > KVC_MAX_TREE) return KVC_ERR_UNSUPPORTED;
  if (words < 1 || words < (step->max_new + 63) / 64) return KVC_ERR_SHAPE;
  if (step->num_rows == 0) return KVC_OK;
  if (!parents || !masks) return KVC_ERR_NULL_ARG;
  if (!aligned(parents, 4) || !aligned(masks, 8) || !aligned(positions, 4)) return KVC_ERR_ALIGN;
  TreeArgs a = {};
  a.step = step_view(nullptr, step);
  a.parents = parents;
  a.masks = masks;
  a.words = words;
  a.positions = positions;
  return hip_status(launch_tree(a, stream));
}

size_t kvc_verify_workspace_bytes(const kvc_step* step, int32_t vocab) {
  if (check_step(nullptr, step) != KVC_OK || vocab < 1 || vocab > kMostVocab) return 0;
  return verify_ends_bytes(step->num_seqs) + static_cast<size_t>(step->num_seqs) * verify_pieces(vocab) * sizeof(double2);
}

kvc_status kvc_verify(const kvc_step* step, const kvc_draft* draft, void* workspace, size_t workspace_bytes,
                      hipStream_t stream) {
  const kvc_status s = check_step(nullptr, step);
  if (s != KVC_OK) return s;
  const kvc_draft* d = draft;
  if (!d) return KVC_ERR_NULL_ARG;
  if (step->max_new > KVC_MAX_TREE) return KVC_ERR_UNSUPPORTED;
  if (d->vocab < 1 || d->vocab > kMostVocab || d->children < 0 || !in_range(d->vocab, d->target_stride) ||
      (d->draft && !in_range(d->vocab, d->draft_stride)))
    return KVC_ERR_SHAPE;
  if (step->num_seqs == 0) return KVC_OK;
  if (!d->counts || !d->chosen || !d->last) return KVC_ERR_NULL_ARG;
  if (step->num_rows > 0 && (!d->parents || !d->tokens || !d->target || !d->uniforms || !d->path)) return KVC_ERR_NULL_ARG;
  for (const void* p : {static_cast<const void*>(d->parents), static_cast<const void*>(d->tokens),
                        static_cast<const void*>(d->target), static_cast<const void*>(d->draft),
                        static_cast<const void*>(d->uniforms), static_cast<const void*>(d->last),
                        static_cast<const void*>(d->path), static_cast<const void*>(d->counts),
                        static_cast<const void*>(d->chosen)})
    if (!aligned(p, 4)) return KVC_ERR_ALIGN;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < kvc_verify_workspace_bytes(step, d->vocab))
    return KVC_ERR_WORKSPACE;
  const void* written[3] = {d->path, d->counts, d->chosen};
  for (int i = 0; i < 3; ++i) {
    if (!written[i]) continue;
    for (int j = 0; j < i; ++j)
      if (written[i] == written[j]) return KVC_ERR_ALIAS;
    for (const void* p : {static_cast<const void*>(d->parents), static_cast<const void*>(d->tokens),
                          static_cast<const void*>(d->target), static_cast<const void*>(d->draft),
                          static_cast<const void*>(d->uniforms), static_cast<const void*>(d->last)})
      if (written[i] == p) return KVC_ERR_ALIAS;
  }
  VerifyArgs a = {};
  a.step = step_view(nullptr, step);
  a.parents = d->parents;
  a.tokens = d->tokens;
  a.target = d->target;
  a.draft = d->draft;
  a.target_stride = d->target_stride;
  a.draft_stride = d->draft_stride;
  a.vocab = d->vocab;
  a.children = d->children;
  a.pieces = static_cast<int32_t>(verify_pieces(d->vocab));
  a.uniforms = d->uniforms;
  a.last = d->last;
  a.path = d->path;
  a.counts = d->counts;
  a.chosen = d->chosen;
  a.ends = static_cast<VerifyEnd*>(workspace);
  a.sums = reinterpret_cast<double2*>(static_cast<char*>(workspace) + verify_ends_bytes(step->num_seqs));
  return hip_status(launch_verify(a, stream));
}

kvc_status kvc_keep(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const int32_t* path,
                    const int32_t* counts, int32_t layer_begin, int32_t layer_end, hipStream_t stream) {
  kvc_status s = check_pools(cache, scales, layer_begin, layer_end);
  if (s != KVC_OK) return s;
  s = check_step(cache, step);
  if (s != KVC_OK) return s;
  if (step->num_rows == 0 || layer_end == layer_begin) return KVC_OK;
  if (!path || !counts) return KVC_ERR_NULL_ARG;
  if (!aligned(path, 4) || !aligned(counts, 4)) return KVC_ERR_ALIGN;
  KeepArgs a = {};
  a.pv = pool_view(cache, scales);
  a.step = step_view(cache, step);
  a.path = path;
  a.counts = counts;
  RowsLayers<kRowsLayers> layers = {};
  for (int32_t l0 = layer_begin; l0 < layer_end; l0 += kRowsLayers) {
    a.num_layers = std::min(kRowsLayers, layer_end - l0);
    for (int32_t l = 0; l < a.num_layers; ++l) {
      layers.pools[0][l] = cache->k_layers[l0 + l];
      layers.pools[1][l] = cache->v_layers[l0 + l];
      if (scales) {
        layers.scales[0][l] = scales->k_layers[l0 + l];
        layers.scales[1][l] = scales->v_layers[l0 + l];
      }
    }
    s = hip_status(launch_keep(a, layers, cache->dtype, cache->head_dim, stream));
    if (s != KVC_OK) return s;
  }
  return KVC_OK;
}

}  // extern "C"
