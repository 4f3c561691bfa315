// lg_fp4_attend.hip -- attention of a step's new tokens over 4-bit pages (lg_paged_attend_fp4).
//
// A wave a query row (a token's query head): 64 slots at a time, a lane forms the score of one, then the lanes hold
// D / 64 values of the output each and add up the 64 weighted values, with the running maximum and sum of a softmax.
#include "lg_fp4.h"
#include "lg_paged_internal.h"

namespace lg {

struct Fp4AttendArgs {
  const void* q;
  const char *k, *v;
  void* out;
  const int32_t *q_start, *base, *suffix_w;
  float *lse, *suffix, *conf;
  MapArgs map;
  int32_t Hq, Hkv, G, D, total, max_chunk, window, n_sink;
  float scale_log2;
};

constexpr int kRowThreads = 64;
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float wave_max(float x) {
  for (int o = 1; o < 64; o <<= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o, 64);
  return x;
}

template <typename T, int D>
__global__ __launch_bounds__(kRowThreads) void fp4_attend(Fp4AttendArgs a) {
  __shared__ float q[D];
  const int lane = threadIdx.x, r = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, h = hq / a.G;
  const int b = seq_of_row(a.q_start, a.map.B, r);
  if (b >= a.map.B) return;
  const Chunk c = chunk_of(a.q_start, b, a.total);
  if (r < c.first || r >= c.first + c.n) return;
  const int base = a.base[b];
  if (base < 0 || c.n > a.max_chunk || base > a.map.cap - c.n) {
    if (a.conf != nullptr && lane == 0) a.conf[b] = NAN;
    return;
  }
  const MapArgs& m = a.map;
  const int slot_q = base + r - c.first;
  const int32_t* pos = m.pos + (size_t)b * m.cap;
  const int p_q = pos[slot_q];
  const int win = a.window > 0 ? (int)max((long long)p_q - a.window, (long long)INT32_MIN) : INT32_MIN;
  const int suf = (int)max((long long)p_q - (a.suffix_w != nullptr ? max(a.suffix_w[b], 0) : 0), (long long)INT32_MIN);
  const size_t row = (size_t)r * a.Hq + hq;
  for (int d = lane; d < D; d += 64) q[d] = (float)((const T*)a.q)[row * D + d];
  __syncthreads();
  const size_t block = fp4_block(D, m.shift);
  const int ps = 1 << m.shift;
  float mx = -INFINITY, l = 0.f, sfx = 0.f, o[2] = {0.f, 0.f};
  for (int s0 = 0; s0 <= slot_q; s0 += 64) {
    const int s = s0 + lane;
    int page = -1;
    float sc = -INFINITY;
    bool see = false, near = false;
    if (s <= slot_q) {
      page = m.table[(size_t)b * m.P + (s >> m.shift)];
      see = is_page(m, page) && (a.window == 0 || pos[s] > win || pos[s] < a.n_sink);
      near = pos[s] > suf;
    }
    if (see) {
      const char* at = a.k + ((size_t)page * a.Hkv + h) * block;
      const uint32_t* codes = (const uint32_t*)(at + (s & (ps - 1)) * (D / 2));
      sc = 0.f;
      for (int w = 0; w < D / 8; ++w) {
        const float u = fp4_unit(*(const uint8_t*)(at + ps * (D / 2) + (s & (ps - 1)) * (D / 32) + w / 4));
        const f32x2 x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], u, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], u, 1);
        const f32x2 x2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], u, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[w], u, 3);
        sc += x0[0] * q[8 * w] + x0[1] * q[8 * w + 1] + x1[0] * q[8 * w + 2] + x1[1] * q[8 * w + 3] + x2[0] * q[8 * w + 4] +
              x2[1] * q[8 * w + 5] + x3[0] * q[8 * w + 6] + x3[1] * q[8 * w + 7];
      }
      sc *= a.scale_log2;
    }
    const float top = fmaxf(mx, wave_max(sc)), ms = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(mx - ms), p = see ? __builtin_amdgcn_exp2f(sc - ms) : 0.f;
    mx = top;
    l = l * f + wave_sum(p);
    sfx = sfx * f + wave_sum(near ? p : 0.f);
    o[0] *= f;
    o[1] *= f;
    unsigned long long seen = __ballot(see);
    while (seen != 0) {
      const int j = __builtin_ctzll(seen);
      seen &= seen - 1;
      const float pj = __shfl(p, j, 64);
      const int pg = __shfl(page, j, 64), in = (s0 + j) & (ps - 1), d = lane * (D / 64);
      const char* at = a.v + ((size_t)pg * a.Hkv + h) * block;
      const float u = fp4_unit(*(const uint8_t*)(at + ps * (D / 2) + in * (D / 32) + d / 32));
      const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)*(const uint8_t*)(at + in * (D / 2) + d / 2), u, 0);
      if constexpr (D == 128) {
        o[0] += pj * x[0];
        o[1] += pj * x[1];
      } else {
        o[0] += pj * x[d & 1];
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int i = 0; i < D / 64; ++i) ((T*)a.out)[row * D + lane * (D / 64) + i] = (T)(l == 0.f ? 0.f : o[i] * inv);
  if (lane == 0) {
    const float mass = l == 0.f ? 0.f : sfx * inv;
    a.lse[row] = l == 0.f ? -INFINITY : kLn2 * (mx + __builtin_amdgcn_logf(l));
    if (a.suffix != nullptr) a.suffix[row] = mass;
    if (a.conf != nullptr && r == c.first + c.n - 1) atomicMax((int*)a.conf + b, mass != mass ? 0x7fc00000 : __float_as_int(mass));
  }
}

long fp4_attend_grid(const lg_paged_layer& l, const lg_page_map&, lg_dtype, int total, int) { return (long)total * l.n_q_heads / 8; }
size_t fp4_attend_need(const lg_paged_layer&, const lg_page_map&, lg_dtype, int, int, int, int) { return 0; }
size_t fp4_attend_bytes(const lg_paged_layer&, const lg_page_map&, lg_dtype, int, int) { return 16; }

hipError_t launch_fp4_attend(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, const void* q, void* out,
                             const int32_t* q_start, const int32_t* base, int total, int max_chunk, int window,
                             int n_sink, const int32_t* suffix_w, float* lse, float* suffix, float* conf, void* ws,
                             hipStream_t st) {
  Fp4AttendArgs a = {};
  a.q = q;
  a.k = (const char*)l.k;
  a.v = (const char*)l.v;
  a.out = out;
  a.q_start = q_start;
  a.base = base;
  a.suffix_w = suffix_w;
  a.lse = lse;
  a.suffix = suffix;
  a.conf = conf;
  a.map = map_args(m);
  a.Hq = l.n_q_heads;
  a.Hkv = l.n_kv_heads;
  a.G = l.n_q_heads / l.n_kv_heads;
  a.D = l.head_dim;
  a.total = total;
  a.max_chunk = max_chunk;
  a.window = window;
  a.n_sink = n_sink;
  a.scale_log2 = kLog2e / sqrtf((float)l.head_dim);
  const dim3 grid((unsigned)total * l.n_q_heads), block(kRowThreads);
  if (dtype == LG_BF16) {
    if (l.head_dim == 128) hipLaunchKernelGGL((fp4_attend<__bf16, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((fp4_attend<__bf16, 64>), grid, block, 0, st, a);
  } else {
    if (l.head_dim == 128) hipLaunchKernelGGL((fp4_attend<float, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((fp4_attend<float, 64>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace lg
