// Host entry points of a served step (kvc_append, kvc_gather, kvc_attend): argument checks, launch sizing and dispatch.
// Every check runs before anything is enqueued; on an error nothing is enqueued.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvc.h"
#include "kvc_serve.h"

namespace {

constexpr int32_t kMaxSeqs = 1 << 30;
constexpr int32_t kMaxContext = 1 << 30;  // key indices a step ahead of the last one stay within 32 bits

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMostStride = INT64_C(1) << 40;  // elements: more than any memory, and bytes of it fit in 64 bits

// Whether strides lie in [least, kMostStride].
template <class... S>
bool in_range(int64_t least, S... strides) {
  return ((strides >= least && strides <= kMostStride) && ...);
}

kvc_status hip_status(hipError_t e) {
  if (e == hipSuccess) return KVC_OK;
  kvc::set_last_hip_error(e);
  return KVC_ERR_HIP;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int64_t elem_size(int32_t t) { return t == KVC_I8 ? 1 : t == KVC_BF16 ? 2 : 4; }

kvc_status check_pools(const kvc_cache* c, const kvc_scales* sc, int32_t lb, int32_t le) {
  if (!c) return KVC_ERR_NULL_ARG;
  if (c->dtype != KVC_F32 && c->dtype != KVC_BF16 && c->dtype != KVC_I8) return KVC_ERR_DTYPE;
  if (c->head_dim != 64 && c->head_dim != 128) return KVC_ERR_UNSUPPORTED;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_kv_heads > 65535 || c->block_size < 1 || c->num_blocks < 1)
    return KVC_ERR_SHAPE;
  if (lb < 0 || le < lb || le > c->num_layers) return KVC_ERR_SHAPE;
  if (!in_range(1, c->block_stride, c->token_stride, c->head_stride)) return KVC_ERR_SHAPE;
  if (c->head_stride < c->head_dim && c->num_kv_heads > 1) return KVC_ERR_SHAPE;
  const int64_t es = elem_size(c->dtype);
  if ((c->block_stride * es) % 16 || (c->token_stride * es) % 16 || (c->head_stride * es) % 16) return KVC_ERR_ALIGN;
  if (c->block_stride > UINT32_MAX / es || c->token_stride > UINT32_MAX / es) return KVC_ERR_UNSUPPORTED;
  if ((c->dtype == KVC_I8) != (sc != nullptr)) return sc ? KVC_ERR_DTYPE : KVC_ERR_NULL_ARG;
  if (sc && !in_range(1, sc->block_stride, sc->token_stride, sc->head_stride)) return KVC_ERR_SHAPE;
  if (sc && (sc->block_stride > UINT32_MAX / 4 || sc->token_stride > UINT32_MAX / 4)) return KVC_ERR_UNSUPPORTED;
  if (le > lb && (!c->k_layers || !c->v_layers || (sc && (!sc->k_layers || !sc->v_layers)))) return KVC_ERR_NULL_ARG;
  for (int32_t l = lb; l < le; ++l) {
    if (!c->k_layers[l] || !c->v_layers[l]) return KVC_ERR_NULL_ARG;
    if (!aligned(c->k_layers[l], 16) || !aligned(c->v_layers[l], 16)) return KVC_ERR_ALIGN;
    if (!sc) continue;
    if (!sc->k_layers[l] || !sc->v_layers[l]) return KVC_ERR_NULL_ARG;
    if (!aligned(sc->k_layers[l], 4) || !aligned(sc->v_layers[l], 4)) return KVC_ERR_ALIGN;
  }
  return KVC_OK;
}

kvc_status check_step(const kvc_cache* c, const kvc_step* s) {
  if (!s) return KVC_ERR_NULL_ARG;
  if (s->num_seqs < 0 || s->num_seqs > kMaxSeqs || s->num_rows < 0 || s->max_new < 0 || s->max_context < 0 ||
      s->max_context > kMaxContext || s->max_blocks < 0 || s->reserved != 0)
    return KVC_ERR_SHAPE;
  if (s->num_seqs == 0) return s->num_rows == 0 ? KVC_OK : KVC_ERR_SHAPE;
  if (s->max_new > s->num_rows || static_cast<int64_t>(s->num_rows) * c->num_kv_heads > INT32_MAX)
    return KVC_ERR_SHAPE;
  if (!s->starts || !s->contexts) return KVC_ERR_NULL_ARG;
  if (s->tables && s->max_blocks < 1) return KVC_ERR_SHAPE;
  if (!aligned(s->starts, 4) || !aligned(s->contexts, 4) || !aligned(s->offsets, 4) || !aligned(s->tables, 4))
    return KVC_ERR_ALIGN;
  return KVC_OK;
}

kvc::ServePool pool_view(const kvc_cache* c, const kvc_scales* sc) {
  kvc::ServePool p = {};
  const int64_t es = elem_size(c->dtype);
  p.block_bytes = static_cast<uint32_t>(c->block_stride * es);
  p.token_bytes = static_cast<uint32_t>(c->token_stride * es);
  p.head_bytes = c->head_stride * es;
  if (sc) {
    p.sblock_bytes = static_cast<uint32_t>(sc->block_stride * 4);
    p.stoken_bytes = static_cast<uint32_t>(sc->token_stride * 4);
    p.shead_bytes = sc->head_stride * 4;
  }
  p.block_size = c->block_size;
  p.num_blocks = c->num_blocks;
  p.num_kv_heads = c->num_kv_heads;
  p.block = kvc::divisor(c->block_size);
  return p;
}

kvc::StepView step_view(const kvc_cache* c, const kvc_step* s) {
  kvc::StepView v = {};
  v.num_seqs = s->num_seqs;
  v.num_rows = s->num_rows;
  v.max_new = s->max_new;
  v.max_context = s->max_context;
  v.max_blocks = s->max_blocks;
  v.capacity = static_cast<int64_t>(s->tables ? s->max_blocks : c->num_blocks) * c->block_size;
  v.capacity = std::min<int64_t>(v.capacity, INT32_MAX);
  v.starts = s->starts;
  v.contexts = s->contexts;
  v.offsets = s->offsets;
  v.tables = s->tables;
  return v;
}

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
  kvc::RowsArgs a = {};
  a.pv = pool_view(cache, scales);
  a.step = step_view(cache, step);
  a.layer_stride = rows->layer_stride * es;
  a.token_stride = rows->token_stride * es;
  a.head_stride = rows->head_stride * es;
  kvc::RowsLayers<kvc::kRowsLayers> layers = {};
  for (int32_t l0 = lb; l0 < le; l0 += kvc::kRowsLayers) {
    a.num_layers = std::min(kvc::kRowsLayers, le - l0);
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
    s = hip_status(kvc::launch_rows(a, layers, cache->dtype, rows->dtype, cache->head_dim, gather, stream));
    if (s != KVC_OK) return s;
  }
  return KVC_OK;
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

size_t kvc_attend_workspace_bytes(const kvc_cache* cache, const kvc_step* step, int32_t num_heads) {
  if (!cache || !step || cache->num_kv_heads < 1 || num_heads < 1 || num_heads % cache->num_kv_heads) return 0;
  if (cache->head_dim != 64 && cache->head_dim != 128) return 0;
  if (check_step(cache, step) != KVC_OK) return 0;
  return kvc::plan_attend(cache->dtype, step->num_seqs, step->num_rows, step->max_new, step->max_context,
                          step->max_context, cache->num_kv_heads, num_heads / cache->num_kv_heads, cache->head_dim)
      .most_bytes;
}

kvc_status kvc_attend(const kvc_cache* cache, const kvc_scales* scales, const kvc_step* step, const kvc_query* query,
                      int32_t layer, void* workspace, size_t workspace_bytes, hipStream_t stream) {
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
  if (query->dtype != (cache->dtype == KVC_F32 ? KVC_F32 : KVC_BF16)) return KVC_ERR_DTYPE;
  const int32_t H = cache->num_kv_heads;
  if (query->num_heads < 1 || query->num_heads % H ||
      static_cast<int64_t>(step->num_rows) * query->num_heads > INT32_MAX)
    return KVC_ERR_SHAPE;
  if (!in_range(0, query->q_token_stride, query->q_head_stride, query->out_token_stride, query->out_head_stride))
    return KVC_ERR_SHAPE;
  if (step->num_rows == 0) return KVC_OK;
  if (!query->q || !query->out) return KVC_ERR_NULL_ARG;
  const int64_t es = elem_size(query->dtype);
  if (!aligned(query->q, 16) || !aligned(query->out, 16) || !aligned(query->lse, 4) ||
      (query->q_token_stride * es) % 16 || (query->q_head_stride * es) % 16 || (query->out_token_stride * es) % 16 ||
      (query->out_head_stride * es) % 16)
    return KVC_ERR_ALIGN;
  // a window bounds the keys of a tile of rows: its own, and one more for each further token of the tile
  int64_t span = step->max_context;
  if (query->window) span = std::min<int64_t>(span, static_cast<int64_t>(query->window) + kvc::kAttendTile);
  const int32_t group = query->num_heads / H;
  const kvc::AttendPlan p =
      kvc::plan_attend(cache->dtype, step->num_seqs, step->num_rows, step->max_new, span, step->max_context, H, group,
                       cache->head_dim);
  if (p.bytes > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < p.bytes)) return KVC_ERR_WORKSPACE;
  kvc::AttendArgs a = {};
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
  a.by_heads = kvc::divisor(query->num_heads);
  a.by_group = kvc::divisor(group);
  a.causal = query->causal;
  a.window = query->window;
  a.scale_log2 = query->scale * kLog2e;
  a.direct = p.direct;
  a.splits = p.splits;
  a.chunk = p.chunk;
  if (p.splits > 1) {
    // (the parts first: rows of them are a multiple of 256 bytes, and so they stay aligned whatever their number)
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + static_cast<int64_t>(p.splits) * step->num_rows * a.num_heads *
                                                         cache->head_dim);
  }
  return hip_status(kvc::launch_attend(a, p, cache->dtype, cache->head_dim, stream));
}

}  // extern "C"
