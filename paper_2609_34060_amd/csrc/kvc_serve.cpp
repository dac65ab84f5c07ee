// Host entry points of a served step (kvc_append, kvc_gather, kvc_attend, kvc_attend_tree): argument checks, launch sizing
// and dispatch.  Every check runs before anything is enqueued; on an error nothing is enqueued.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvc.h"
#include "kvc_check.h"
#include "kvc_serve.h"

namespace {

using namespace kvc;

constexpr float kLog2e = 1.4426950408889634f;

kvc_status move_rows(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const kvc_rows* rows,
                     int32_t lb, int32_t le, bool gather, hipStream_t stream) {
  kvc_status s = check_pools(cache, scales, lb, le);
  if (s != KVC_OK) return s;
  s = check_step(cache, step);
  if (s != KVC_OK) return s;
  if (!rows) return KVC_ERR_NULL_ARG;
  if (rows->reserved != 0) return KVC_ERR_SHAPE;
  if (rows->dtype != KVC_F32 && rows->dtype != KVC_BF16) return KVC_ERR_DTYPE;
  if (cache->dtype != KVC_I8 && rows->dtype != cache->dtype) return KVC_ERR_DTYPE;
  const int64_t es = elem_size(rows->dtype);
  if (!in_range(0, rows->layer_stride, rows->token_stride, rows->head_stride)) return KVC_ERR_SHAPE;
  if (step->num_rows == 0 || le == lb) return KVC_OK;
  if (!rows->k || !rows->v) return KVC_ERR_NULL_ARG;
  if (!aligned(rows->k, 16) || !aligned(rows->v, 16) || (rows->layer_stride * es) % 16 ||
      (rows->token_stride * es) % 16 || (rows->head_stride * es) % 16)
    return KVC_ERR_ALIGN;
  RowsArgs a = {};
  a.pv = pool_view(cache, scales);
  a.step = step_view(cache, step);
  a.layer_stride = rows->layer_stride * es;
  a.token_stride = rows->token_stride * es;
  a.head_stride = rows->head_stride * es;
  RowsLayers<kRowsLayers> layers = {};
  for (int32_t l0 = lb; l0 < le; l0 += kRowsLayers) {
    a.num_layers = std::min(kRowsLayers, le - l0);
    for (int32_t l = 0; l < a.num_layers; ++l) {
      layers.pools[0][l] = cache->k_layers[l0 + l];
      layers.pools[1][l] = cache->v_layers[l0 + l];
      if (scales) {
        layers.scales[0][l] = scales->k_layers[l0 + l];
        layers.scales[1][l] = scales->v_layers[l0 + l];
      }
    }
    a.rows[0] = static_cast<char*>(rows->k) + (l0 - lb) * a.layer_stride;
    a.rows[1] = static_cast<char*>(rows->v) + (l0 - lb) * a.layer_stride;
    s = hip_status(launch_rows(a, layers, cache->dtype, rows->dtype, cache->head_dim, gather, stream));
    if (s != KVC_OK) return s;
  }
  return KVC_OK;
}

struct Masks {
  const uint64_t* at;
  int32_t words;
};

// kvc_attend, or with masks kvc_attend_tree.
kvc_status attend(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const kvc_query* query,
                  const Masks* masks, int32_t layer, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!cache) return KVC_ERR_NULL_ARG;
  if (layer < 0 || layer >= cache->num_layers) return KVC_ERR_SHAPE;
  kvc_status s = check_pools(cache, scales, layer, layer + 1);
  if (s != KVC_OK) return s;
  s = check_step(cache, step);
  if (s != KVC_OK) return s;
  if (!query) return KVC_ERR_NULL_ARG;
  if (query->reserved != 0 || query->causal < 0 || query->causal > 1 || query->window < 0 ||
      !std::isfinite(query->scale * kLog2e))  // (scores are kept in units of log2)
    return KVC_ERR_SHAPE;
  if (query->window > 0 && !query->causal) return KVC_ERR_UNSUPPORTED;
  if (masks) {
    if (!query->causal || masks->words < 1 || masks->words < (step->max_new + INT64_C(63)) / 64) return KVC_ERR_SHAPE;
    if (query->window > 0 && query->window < step->max_new) return KVC_ERR_UNSUPPORTED;
  }
  if (query->dtype != (cache->dtype == KVC_F32 ? KVC_F32 : KVC_BF16)) return KVC_ERR_DTYPE;
  const int32_t H = cache->num_kv_heads;
  if (query->num_heads < 1 || query->num_heads % H ||
      static_cast<int64_t>(step->num_rows) * query->num_heads > INT32_MAX)
    return KVC_ERR_SHAPE;
  if (!in_range(0, query->q_token_stride, query->q_head_stride, query->out_token_stride, query->out_head_stride))
    return KVC_ERR_SHAPE;
  if (step->num_rows == 0) return KVC_OK;
  if (!query->q || !query->out || (masks && !masks->at)) return KVC_ERR_NULL_ARG;
  const int64_t es = elem_size(query->dtype);
  if (!aligned(query->q, 16) || !aligned(query->out, 16) || !aligned(query->lse, 4) ||
      (query->q_token_stride * es) % 16 || (query->q_head_stride * es) % 16 || (query->out_token_stride * es) % 16 ||
      (query->out_head_stride * es) % 16 || (masks && !aligned(masks->at, 8)))
    return KVC_ERR_ALIGN;
  // a window bounds the keys of a tile of rows: its own, and one more for each further token of the tile (under masks, the
  // new tokens beside those of a token before them)
  int64_t span = step->max_context;
  if (query->window)
    span = std::min<int64_t>(span, static_cast<int64_t>(query->window) + (masks ? step->max_new : kAttendTile));
  const int32_t group = query->num_heads / H;
  const AttendPlan p =
      plan_attend(cache->dtype, step->num_seqs, step->num_rows, step->max_new, span, step->max_context, H, group,
                       cache->head_dim, masks != nullptr);
  if (p.bytes > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < p.bytes)) return KVC_ERR_WORKSPACE;
  AttendArgs a = {};
  a.pv = pool_view(cache, scales);
  a.step = step_view(cache, step);
  a.k = cache->k_layers[layer];
  a.v = cache->v_layers[layer];
  if (scales) {
    a.ks = scales->k_layers[layer];
    a.vs = scales->v_layers[layer];
  }
  a.q = static_cast<const char*>(query->q);
  a.out = static_cast<char*>(query->out);
  a.lse = query->lse;
  a.q_token_stride = query->q_token_stride * es;
  a.q_head_stride = query->q_head_stride * es;
  a.out_token_stride = query->out_token_stride * es;
  a.out_head_stride = query->out_head_stride * es;
  a.num_heads = query->num_heads;
  a.group = group;
  a.by_heads = divisor(query->num_heads);
  a.by_group = divisor(group);
  a.causal = masks ? 0 : query->causal;
  a.window = query->window;
  a.scale_log2 = query->scale * kLog2e;
  if (masks) {
    a.masks = masks->at;
    a.words = masks->words;
  }
  a.direct = p.direct;
  a.splits = p.splits;
  a.chunk = p.chunk;
  if (p.splits > 1) {
    // (the parts first: rows of them are a multiple of 256 bytes, and so they stay aligned whatever their number)
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + static_cast<int64_t>(p.splits) * step->num_rows * a.num_heads *
                                                         cache->head_dim);
  }
  return hip_status(launch_attend(a, p, cache->dtype, cache->head_dim, stream));
}

}  // namespace

extern "C" {

kvc_status kvc_append(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const kvc_rows* rows,
                      int32_t layer_begin, int32_t layer_end, hipStream_t stream) {
  return move_rows(cache, scales, step, rows, layer_begin, layer_end, false, stream);
}

kvc_status kvc_gather(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const kvc_rows* rows,
                      int32_t layer_begin, int32_t layer_end, hipStream_t stream) {
  return move_rows(cache, scales, step, rows, layer_begin, layer_end, true, stream);
}

size_t kvc_attend_call_workspace_bytes(const kvc_cache* cache, const kvc_step* step, int32_t num_heads, int32_t tree) {
  if (!cache || !step || cache->num_kv_heads < 1 || num_heads < 1 || num_heads % cache->num_kv_heads) return 0;
  if (cache->head_dim != 64 && cache->head_dim != 128) return 0;
  if (tree < 0 || tree > 1 || check_step(cache, step) != KVC_OK) return 0;
  return plan_attend(cache->dtype, step->num_seqs, step->num_rows, step->max_new, step->max_context, step->max_context,
                     cache->num_kv_heads, num_heads / cache->num_kv_heads, cache->head_dim, tree == 1)
      .most_bytes;
}

size_t kvc_attend_workspace_bytes(const kvc_cache* cache, const kvc_step* step, int32_t num_heads) {
  return std::max(kvc_attend_call_workspace_bytes(cache, step, num_heads, 0),
                  kvc_attend_call_workspace_bytes(cache, step, num_heads, 1));
}

kvc_status kvc_attend(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const kvc_query* query,
                      int32_t layer, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return attend(cache, scales, step, query, nullptr, layer, workspace, workspace_bytes, stream);
}

kvc_status kvc_attend_tree(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step,
                           const kvc_query* query, const uint64_t* masks, int32_t words, int32_t layer,
                           void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const Masks m = {masks, words};
  return attend(cache, scales, step, query, &m, layer, workspace, workspace_bytes, stream);
}

}  // extern "C"
