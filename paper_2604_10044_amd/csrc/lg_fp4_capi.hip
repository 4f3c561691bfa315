// lg_fp4_capi.hip -- the extern "C" entry points of lg_fp4.h: host-side validation and launch. Nothing here
// allocates, frees or synchronises.
#include "lg_paged_checks.h"

namespace lg {
hipError_t launch_append_axes(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, const void* q,
                              int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              const float* inv_freq, int rot, bool interleaved, float scale, const int32_t* axis,
                              const int32_t* coord, int64_t coord_stride, int n_axes, void* q_out,
                              const int32_t* q_start, const int32_t* base, int total, hipStream_t st);
hipError_t launch_unpack(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, void* k, void* v,
                         const int32_t* q_start, const int32_t* base, int total, hipStream_t st);
size_t fp4_attend_bytes(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, int total, int max_chunk);
size_t fp4_attend_need(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, int total, int max_chunk,
                       int window, int n_sink);
long fp4_attend_grid(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, int total, int max_chunk);
hipError_t launch_fp4_attend(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, const void* q, void* out,
                             const int32_t* q_start, const int32_t* base, int total, int max_chunk, int window,
                             int n_sink, const int32_t* suffix_w, float* lse, float* suffix, float* conf, void* ws,
                             hipStream_t st);

constexpr int kMaxAxes = 8;

static bool is_number(lg_dtype t) { return t == LG_F32 || t == LG_BF16; }

static lg_status check_fp4_layer(const lg_paged_layer* layer, const lg_page_map* map, lg_dtype dtype) {
  lg_status s = check_map(map);
  if (s == LG_OK) s = check_paged_layer(layer, *map, true);
  if (s == LG_OK && (layer->dtype != LG_FP4 || !is_number(dtype))) s = LG_ERR_UNSUPPORTED;
  return s;
}

static lg_status check_fp4_sizes(const lg_paged_layer* layer, const lg_page_map* map, lg_dtype dtype, int32_t total,
                                 int32_t max_chunk) {
  const lg_status s = check_fp4_layer(layer, map, dtype);
  if (s != LG_OK) return s;
  if (total < 0 || max_chunk < 0) return LG_ERR_SHAPE;
  if ((int64_t)total * layer->n_q_heads > INT32_MAX) return LG_ERR_SHAPE;
  if (fp4_attend_grid(*layer, *map, dtype, total, max_chunk) > kMaxGrid) return LG_ERR_SHAPE;
  return LG_OK;
}

}  // namespace lg

using namespace lg;

extern "C" {

lg_status lg_rope_axes(int32_t n_axes, const int32_t* sections, int32_t order, int32_t* axis) {
  if (sections == nullptr || axis == nullptr) return LG_ERR_NULL;
  if (n_axes < 1 || n_axes > kMaxAxes || (order != LG_AXES_BLOCKS && order != LG_AXES_TURNS)) return LG_ERR_PARAM;
  int32_t left[kMaxAxes], pairs = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (sections[a] < 0 || sections[a] > 64) return LG_ERR_PARAM;
    left[a] = sections[a];
    pairs += sections[a];
  }
  if (pairs < 1 || pairs > 64) return LG_ERR_PARAM;
  for (int j = 0, a = 0; j < pairs; ++j) {
    while (left[a] == 0) a = (a + 1) % n_axes;
    --left[a];
    axis[j] = a;
    if (order == LG_AXES_TURNS) a = (a + 1) % n_axes;
  }
  return LG_OK;
}

lg_status lg_rope_append_axes(const lg_paged_layer* layer, const lg_page_map* map, lg_dtype dtype, const void* q,
                              int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              const float* inv_freq, int32_t rot_dim, int32_t interleaved, float scale,
                              const int32_t* axis, const int32_t* coord, int64_t coord_stride, int32_t n_axes,
                              void* q_out, const int32_t* q_start, const int32_t* base, int32_t total,
                              hipStream_t stream) {
  lg_status s = check_map(map);
  if (s == LG_OK) s = check_paged_layer(layer, *map, true);
  if (s != LG_OK) return s;
  if (!is_number(dtype) || (layer->dtype != LG_FP4 && layer->dtype != dtype)) return LG_ERR_UNSUPPORTED;
  if (total == 0) return LG_OK;
  if (!q_start || !base || (k == nullptr) != (v == nullptr) || (q == nullptr) != (q_out == nullptr) || (!q && !k))
    return LG_ERR_NULL;
  if (rot_dim < 0 || rot_dim > layer->head_dim || rot_dim % 2 != 0) return LG_ERR_PARAM;
  if (rot_dim > 0 && !inv_freq) return LG_ERR_NULL;
  if (n_axes < 0 || n_axes > kMaxAxes || (n_axes == 0 && (axis != nullptr || coord != nullptr))) return LG_ERR_PARAM;
  if (n_axes > 0 && rot_dim > 0 && (!axis || !coord)) return LG_ERR_NULL;
  if (total < 0 || total > kMaxGrid) return LG_ERR_SHAPE;
  const int64_t wq = (int64_t)layer->n_q_heads * layer->head_dim;
  const int64_t wk = (int64_t)layer->n_kv_heads * layer->head_dim;
  const int64_t most = (int64_t)1 << 40;
  if (q != nullptr && (q_stride < wq || q_stride > most)) return LG_ERR_SHAPE;
  if (k != nullptr && (k_stride < wk || v_stride < wk || k_stride > most || v_stride > most)) return LG_ERR_SHAPE;
  if (n_axes > 1 && (coord_stride < total || coord_stride > most)) return LG_ERR_SHAPE;
  if (q != nullptr && q_out == q && total > 1 && q_stride != wq) return LG_ERR_PARAM;  // rows would be read after others' are written
  const int64_t e = dtype == LG_BF16 ? 2 : 4;
  if (misaligned(q) || misaligned(q_out) || misaligned(k) || misaligned(v)) return LG_ERR_ALIGN;
  if (q != nullptr && q_stride * e % 16 != 0) return LG_ERR_ALIGN;
  if (k != nullptr && (k_stride * e % 16 != 0 || v_stride * e % 16 != 0)) return LG_ERR_ALIGN;
  return done(launch_append_axes(*layer, *map, dtype, q, q_stride, k, k_stride, v, v_stride, inv_freq, rot_dim,
                                 interleaved != 0, scale, axis, coord, coord_stride, n_axes, q_out, q_start, base, total,
                                 stream));
}

lg_status lg_page_unpack_fp4(const lg_paged_layer* layer, const lg_page_map* map, lg_dtype dtype, void* k_out,
                             void* v_out, const int32_t* q_start, const int32_t* base, int32_t total,
                             hipStream_t stream) {
  const lg_status s = check_fp4_layer(layer, map, dtype);
  if (s != LG_OK || total == 0) return s;
  if ((!k_out && !v_out) || !q_start || !base) return LG_ERR_NULL;
  if (total < 0 || total > kMaxGrid) return LG_ERR_SHAPE;
  if (k_out == v_out) return LG_ERR_PARAM;
  if (misaligned(k_out) || misaligned(v_out)) return LG_ERR_ALIGN;
  return done(launch_unpack(*layer, *map, dtype, k_out, v_out, q_start, base, total, stream));
}

size_t lg_paged_attend_fp4_workspace(const lg_paged_layer* layer, const lg_page_map* map, lg_dtype dtype,
                                     int32_t total, int32_t max_chunk) {
  if (check_fp4_sizes(layer, map, dtype, total, max_chunk) != LG_OK) return 0;
  return fp4_attend_bytes(*layer, *map, dtype, total, max_chunk);
}

lg_status lg_paged_attend_fp4(const lg_paged_layer* layer, const lg_page_map* map, lg_dtype dtype, const void* q,
                              void* out, const int32_t* q_start, const int32_t* base, int32_t total,
                              int32_t max_chunk, int32_t window, int32_t n_sink, const int32_t* suffix_w,
                              float* lse, float* suffix_mass, float* conf, void* workspace,
                              size_t workspace_bytes, hipStream_t stream) {
  lg_status s = check_fp4_sizes(layer, map, dtype, total, max_chunk);
  if (s != LG_OK || total == 0) return s;
  if (!q || !out || !q_start || !base || !lse) return LG_ERR_NULL;
  if (suffix_w == nullptr && (suffix_mass != nullptr || conf != nullptr)) return LG_ERR_NULL;
  if (window < 0 || n_sink < 0 || out == q) return LG_ERR_PARAM;
  if (misaligned(q) || misaligned(out)) return LG_ERR_ALIGN;
  s = check_workspace(workspace, workspace_bytes,
                      fp4_attend_need(*layer, *map, dtype, total, max_chunk, window, n_sink));
  if (s != LG_OK) return s;
  return done(launch_fp4_attend(*layer, *map, dtype, q, out, q_start, base, total, max_chunk, window, n_sink, suffix_w,
                                lse, suffix_mass, conf, workspace, stream));
}

}  // extern "C"
