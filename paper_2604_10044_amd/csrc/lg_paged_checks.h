// lg_paged_checks.h -- host-side checks that the entry points on a paged cache share (lg_paged.h, lg_fp4.h).
#pragma once

#include "lg_fp4.h"
#include "lg_paged_internal.h"

namespace lg {

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

// A grid holds fewer than 2^32 threads; the launches that grow with the step have at most 512 a workgroup.
constexpr long kMaxGrid = (1 << 23) - 1;

inline lg_status check_map(const lg_page_map* m) {
  if (m == nullptr || !m->table || !m->pos || !m->len || !m->ref) return LG_ERR_NULL;
  if (misaligned(m->ref)) return LG_ERR_ALIGN;
  if (m->batch <= 0 || m->max_pages <= 0 || m->n_pages <= 0) return LG_ERR_SHAPE;
  if (m->batch > 65535 || m->n_pages > 1 << 28) return LG_ERR_SHAPE;
  if (m->page_size < 16 || m->page_size > 256 || (m->page_size & (m->page_size - 1)) != 0)
    return LG_ERR_UNSUPPORTED;
  if ((int64_t)m->max_pages * m->page_size > 1 << 30) return LG_ERR_SHAPE;
  if ((int64_t)m->batch * m->max_pages > INT32_MAX) return LG_ERR_SHAPE;
  return LG_OK;
}

// fp4: whether the call takes 4-bit layers too.
inline lg_status check_paged_layer(const lg_paged_layer* l, const lg_page_map& m, bool fp4 = false) {
  if (l == nullptr || !l->k || !l->v) return LG_ERR_NULL;
  if (misaligned(l->k) || misaligned(l->v)) return LG_ERR_ALIGN;
  if (l->n_pages != m.n_pages || l->page_size != m.page_size) return LG_ERR_SHAPE;
  if (l->n_q_heads <= 0 || l->n_kv_heads <= 0 || l->n_kv_heads > 65535) return LG_ERR_SHAPE;
  if (l->n_q_heads % l->n_kv_heads != 0) return LG_ERR_SHAPE;
  if (l->n_q_heads / l->n_kv_heads > kMaxGroup) return LG_ERR_UNSUPPORTED;
  if (l->head_dim != 64 && l->head_dim != 128) return LG_ERR_UNSUPPORTED;
  if (l->dtype != LG_F32 && l->dtype != LG_BF16 && !(fp4 && l->dtype == LG_FP4)) return LG_ERR_UNSUPPORTED;
  // lg_page_compact numbers the pool's slots in 32 bits; wider slots reach no such number in memory
  if (l->dtype == LG_FP4 && (int64_t)m.n_pages * m.page_size >= UINT32_MAX) return LG_ERR_SHAPE;
  return LG_OK;
}

inline lg_status check_layers(int32_t n, const lg_paged_layer* layers, const lg_page_map& m) {
  if (n < 0) return LG_ERR_SHAPE;
  if (n > 0 && layers == nullptr) return LG_ERR_NULL;
  for (int i = 0; i < n; ++i) {
    const lg_status s = check_paged_layer(&layers[i], m, true);
    if (s != LG_OK) return s;
    if (layers[i].n_kv_heads != layers[0].n_kv_heads || layers[i].head_dim != layers[0].head_dim ||
        layers[i].dtype != layers[0].dtype)
      return LG_ERR_SHAPE;
  }
  return LG_OK;
}

inline lg_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (ws == nullptr) return LG_ERR_NULL;
  if (misaligned(ws)) return LG_ERR_ALIGN;
  return bytes < need ? LG_ERR_WORKSPACE : LG_OK;
}

inline lg_status done(hipError_t e) { return e == hipSuccess ? LG_OK : LG_ERR_HIP; }

}  // namespace lg
