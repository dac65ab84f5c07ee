// Host checks and views that the served step's entry points share.
#pragma once

#include <algorithm>
#include <cstdint>

#include "kvc.h"
#include "kvc_serve.h"

namespace kvc {

constexpr int32_t kMaxSeqs = 1 << 30;
constexpr int32_t kMaxContext = 1 << 30;  // key indices a step ahead of the last one stay within 32 bits

constexpr int64_t kMostStride = INT64_C(1) << 40;  // elements: more than any memory, and bytes of it fit in 64 bits

// Whether strides lie in [least, kMostStride].
template <class... S>
bool in_range(int64_t least, S... strides) {
  return ((strides >= least && strides <= kMostStride) && ...);
}

inline kvc_status hip_status(hipError_t e) {
  if (e == hipSuccess) return KVC_OK;
  set_last_hip_error(e);
  return KVC_ERR_HIP;
}

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline int64_t elem_size(int32_t t) { return t == KVC_I8 ? 1 : t == KVC_BF16 ? 2 : 4; }

inline kvc_status check_pools(const kvc_cache* c, const kvc_scales* sc, int32_t lb, int32_t le) {
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

// c: the cache that the step belongs to, or null where a call reads none.
inline kvc_status check_step(const kvc_cache* c, const kvc_step* s) {
  if (!s) return KVC_ERR_NULL_ARG;
  if (s->num_seqs < 0 || s->num_seqs > kMaxSeqs || s->num_rows < 0 || s->max_new < 0 || s->max_context < 0 ||
      s->max_context > kMaxContext || s->max_blocks < 0 || s->reserved != 0)
    return KVC_ERR_SHAPE;
  if (s->num_seqs == 0) return s->num_rows == 0 ? KVC_OK : KVC_ERR_SHAPE;
  if (s->max_new > s->num_rows || (c && static_cast<int64_t>(s->num_rows) * c->num_kv_heads > INT32_MAX))
    return KVC_ERR_SHAPE;
  if (!s->starts || !s->contexts) return KVC_ERR_NULL_ARG;
  if (s->tables && s->max_blocks < 1) return KVC_ERR_SHAPE;
  if (!aligned(s->starts, 4) || !aligned(s->contexts, 4) || !aligned(s->offsets, 4) || !aligned(s->tables, 4))
    return KVC_ERR_ALIGN;
  return KVC_OK;
}

inline ServePool pool_view(const kvc_cache* c, const kvc_scales* sc) {
  ServePool p = {};
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
  p.block = divisor(c->block_size);
  return p;
}

inline StepView step_view(const kvc_cache* c, const kvc_step* s) {
  StepView v = {};
  v.num_seqs = s->num_seqs;
  v.num_rows = s->num_rows;
  v.max_new = s->max_new;
  v.max_context = s->max_context;
  v.max_blocks = s->max_blocks;
  v.capacity = INT32_MAX;
  if (c) v.capacity = std::min<int64_t>(v.capacity, static_cast<int64_t>(s->tables ? s->max_blocks : c->num_blocks) * c->block_size);
  v.starts = s->starts;
  v.contexts = s->contexts;
  v.offsets = s->offsets;
  v.tables = s->tables;
  return v;
}

}  // namespace kvc
