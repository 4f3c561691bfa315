// lg_paged_capi.hip -- the extern "C" entry points of the paged cache (lg_paged.h): host-side
// validation and launch. Nothing here allocates, frees or synchronises.
#include <math.h>

#include "lg_paged_checks.h"

namespace lg {
size_t page_workspace_bytes(const lg_page_map& m);
hipError_t launch_reserve(const lg_page_map& map, int n_layers, const lg_paged_layer* layers,
                          const int32_t* q_start, const int32_t* t, int32_t* base, void* ws,
                          hipStream_t st);
hipError_t launch_fork(const lg_page_map& map, const int32_t* parent, void* ws, hipStream_t st);
hipError_t launch_page_compact(const lg_page_map& map, int n_layers, const lg_paged_layer* layers,
                               const int32_t* keep_idx, const int32_t* new_len, int32_t* moved,
                               void* ws, hipStream_t st);
hipError_t launch_rope(const lg_paged_layer& l, const lg_page_map& m, const void* q, int64_t q_stride,
                       const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                       const float* inv_freq, int rot, bool interleaved, float scale, void* q_out,
                       const int32_t* q_start, const int32_t* base, int total, hipStream_t st);
size_t paged_attend_bytes(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk);
size_t paged_attend_need(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk, int window,
                         int n_sink);
long paged_attend_grid(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk);
hipError_t launch_paged_attend(const lg_paged_layer& l, const lg_page_map& m, const void* q, void* out,
                               const int32_t* q_start, const int32_t* base, int total, int max_chunk,
                               int window, int n_sink, const int32_t* suffix_w, float* lse, float* suffix,
                               float* conf, void* ws, hipStream_t st);

static lg_status check_attend_sizes(const lg_paged_layer* layer, const lg_page_map* map, int32_t total,
                                    int32_t max_chunk) {
  lg_status s = check_map(map);
  if (s != LG_OK) return s;
  s = check_paged_layer(layer, *map);
  if (s != LG_OK) return s;
  if (total < 0 || max_chunk < 0) return LG_ERR_SHAPE;
  if ((int64_t)total * layer->n_q_heads > INT32_MAX) return LG_ERR_SHAPE;
  if (paged_attend_grid(*layer, *map, total, max_chunk) > kMaxGrid) return LG_ERR_SHAPE;
  return LG_OK;
}

}  // namespace lg

using namespace lg;

extern "C" {

size_t lg_page_workspace(const lg_page_map* map) {
  return check_map(map) == LG_OK ? page_workspace_bytes(*map) : 0;
}

lg_status lg_page_reserve(const lg_page_map* map, int32_t n_layers, const lg_paged_layer* layers,
                          const int32_t* q_start, const int32_t* t, int32_t* base, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  lg_status s = check_map(map);
  if (s == LG_OK) s = check_layers(n_layers, layers, *map);
  if (s != LG_OK) return s;
  if (!q_start || !t || !base) return LG_ERR_NULL;
  s = check_workspace(workspace, workspace_bytes, page_workspace_bytes(*map));
  if (s != LG_OK) return s;
  return done(launch_reserve(*map, n_layers, layers, q_start, t, base, workspace, stream));
}

lg_status lg_page_fork(const lg_page_map* map, const int32_t* parent, void* workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  lg_status s = check_map(map);
  if (s != LG_OK) return s;
  if (!parent) return LG_ERR_NULL;
  s = check_workspace(workspace, workspace_bytes, page_workspace_bytes(*map));
  if (s != LG_OK) return s;
  return done(launch_fork(*map, parent, workspace, stream));
}

lg_status lg_page_compact(const lg_page_map* map, int32_t n_layers, const lg_paged_layer* layers,
                          const int32_t* keep_idx, const int32_t* new_len, int32_t* moved,
                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
  lg_status s = check_map(map);
  if (s == LG_OK) s = check_layers(n_layers, layers, *map);
  if (s != LG_OK) return s;
  if (!keep_idx || !new_len || !moved) return LG_ERR_NULL;
  s = check_workspace(workspace, workspace_bytes, page_workspace_bytes(*map));
  if (s != LG_OK) return s;
  return done(launch_page_compact(*map, n_layers, layers, keep_idx, new_len, moved, workspace, stream));
}

lg_status lg_rope_frequencies(const lg_rope_params* p, float* inv_freq, float* scale) {
  if (p == nullptr || inv_freq == nullptr || scale == nullptr) return LG_ERR_NULL;
  const int d = p->rot_dim, half = d / 2;
  const bool regions = p->kind == LG_ROPE_RAMP || p->kind == LG_ROPE_BANDS;
  if (p->kind < LG_ROPE_PLAIN || p->kind > LG_ROPE_BANDS) return LG_ERR_PARAM;
  if (d < 2 || d > 128 || d % 2 != 0 || !(p->theta > 1.) || !(isfinite(p->theta))) return LG_ERR_PARAM;
  if (p->kind != LG_ROPE_PLAIN && !(p->factor >= 1. && isfinite(p->factor))) return LG_ERR_PARAM;
  if (p->kind == LG_ROPE_BASE && d < 4) return LG_ERR_PARAM;
  if (regions && !(p->original_context >= 1. && isfinite(p->original_context) && p->slow > 0. &&
                   p->slow < p->fast && isfinite(p->fast)))
    return LG_ERR_PARAM;
  const double two_pi = 6.283185307179586477;
  const double theta = p->kind == LG_ROPE_BASE ? p->theta * pow(p->factor, d / (d - 2.)) : p->theta;
  double lo = 0., hi = 0.;
  if (p->kind == LG_ROPE_RAMP) {
    // index whose frequency turns n times in the original context: theta^(-2 i / d) context = 2 pi n
    auto index = [&](double n) { return d * log(p->original_context / (two_pi * n)) / (2. * log(theta)); };
    lo = fmin(fmax(floor(index(p->fast)), 0.), d - 1.);
    hi = fmin(fmax(ceil(index(p->slow)), 0.), d - 1.);
  }
  for (int i = 0; i < half; ++i) {
    const double f = pow(theta, -2. * i / d);
    double kept = 1.;  // share of the frequency that is not divided
    if (p->kind == LG_ROPE_LINEAR) kept = 0.;
    if (p->kind == LG_ROPE_RAMP) kept = 1. - fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.), 1.);
    if (p->kind == LG_ROPE_BANDS)
      kept = fmin(fmax((p->original_context * f / two_pi - p->slow) / (p->fast - p->slow), 0.), 1.);
    const bool divides = p->kind == LG_ROPE_LINEAR || regions;
    inv_freq[i] = (float)(divides ? kept * f + (1. - kept) * f / p->factor : f);
  }
  *scale = p->kind == LG_ROPE_RAMP ? (float)(1. + 0.1 * log(p->factor)) : 1.f;
  return LG_OK;
}

lg_status lg_rope_append(const lg_paged_layer* layer, const lg_page_map* map, const void* q,
                         int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, const float* inv_freq, int32_t rot_dim,
                         int32_t interleaved, float scale, void* q_out, const int32_t* q_start,
                         const int32_t* base, int32_t total, hipStream_t stream) {
  lg_status s = check_map(map);
  if (s == LG_OK) s = check_paged_layer(layer, *map);
  if (s != LG_OK) return s;
  if (total == 0) return LG_OK;
  if (!q || !q_out || !q_start || !base || (k == nullptr) != (v == nullptr)) return LG_ERR_NULL;
  if (rot_dim < 0 || rot_dim > layer->head_dim || rot_dim % 2 != 0) return LG_ERR_PARAM;
  if (rot_dim > 0 && !inv_freq) return LG_ERR_NULL;
  const int64_t wq = (int64_t)layer->n_q_heads * layer->head_dim;
  const int64_t wk = (int64_t)layer->n_kv_heads * layer->head_dim;
  if (q_stride < wq || (k != nullptr && (k_stride < wk || v_stride < wk))) return LG_ERR_SHAPE;
  if (q_stride > (int64_t)1 << 40 || k_stride > (int64_t)1 << 40 || v_stride > (int64_t)1 << 40) return LG_ERR_SHAPE;
  if (total < 0 || total > kMaxGrid) return LG_ERR_SHAPE;
  if (q_out == q && total > 1 && q_stride != wq) return LG_ERR_PARAM;  // rows would be read after others' are written
  const int64_t e = layer->dtype == LG_BF16 ? 2 : 4;
  if (misaligned(q) || misaligned(q_out) || misaligned(k) || misaligned(v)) return LG_ERR_ALIGN;
  if (q_stride * e % 16 != 0 || (k != nullptr && (k_stride * e % 16 != 0 || v_stride * e % 16 != 0)))
    return LG_ERR_ALIGN;
  return done(launch_rope(*layer, *map, q, q_stride, k, k_stride, v, v_stride, inv_freq, rot_dim,
                          interleaved != 0, scale, q_out, q_start, base, total, stream));
}

size_t lg_paged_attend_workspace(const lg_paged_layer* layer, const lg_page_map* map, int32_t total,
                                 int32_t max_chunk) {
  if (check_attend_sizes(layer, map, total, max_chunk) != LG_OK) return 0;
  return paged_attend_bytes(*layer, *map, total, max_chunk);
}

lg_status lg_paged_attend(const lg_paged_layer* layer, const lg_page_map* map, const void* q,
                          void* out, const int32_t* q_start, const int32_t* base, int32_t total,
                          int32_t max_chunk, int32_t window, int32_t n_sink,
                          const int32_t* suffix_w, float* lse, float* suffix_mass, float* conf,
                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
  lg_status s = check_attend_sizes(layer, map, total, max_chunk);
  if (s != LG_OK || total == 0) return s;
  if (!q || !out || !q_start || !base || !lse) return LG_ERR_NULL;
  if (suffix_w == nullptr && (suffix_mass != nullptr || conf != nullptr)) return LG_ERR_NULL;
  if (window < 0 || n_sink < 0 || out == q) return LG_ERR_PARAM;
  if (misaligned(q) || misaligned(out)) return LG_ERR_ALIGN;
  s = check_workspace(workspace, workspace_bytes, paged_attend_need(*layer, *map, total, max_chunk, window, n_sink));
  if (s != LG_OK) return s;
  return done(launch_paged_attend(*layer, *map, q, out, q_start, base, total, max_chunk, window, n_sink,
                                  suffix_w, lse, suffix_mass, conf, workspace, stream));
}

}  // extern "C"
