// lg_rope.hip -- rotary positions of a step's queries and keys with the append of its keys and
// values to their pages (lg_rope_append).
//
// One workgroup per token: its slot, page and position are found once, the cosines and sines of its
// rot_dim / 2 angles are formed once in LDS for all heads (one thread each), and the threads walk the
// token's heads in 16-byte pieces. Every value is read once and written once, so memory bounds the
// kernel at long chunks and launch latency at one token a sequence. Measured: 403 MB (two bf16 prompts
// of 8192 tokens, 32 + 8 heads of 128) in 70.5 us, 5.7 TB/s; one token of 32 sequences in 3.8 us. Rotated parts that
// are no whole pieces (kRopeAny) go value by value: the two prompts with 100 rotated values 168 us, 177 interleaved.
//
// An angle p * f is reduced in double to a fraction of a turn in [-1/2, 1/2] (positions reach 2^30: a
// float32 product would keep no digit of the fraction), and only the fraction is rounded to float32.
#include "lg_paged_internal.h"

namespace lg {

struct RopeArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  void *q_out, *pk, *pv;
  const float* inv_freq;
  const int32_t *q_start, *base;
  MapArgs map;
  int32_t Hq, Hkv, D, rot, total;
  float scale;
};

constexpr int kRopeThreads = 256;

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Elem<__bf16> {
  static __device__ __forceinline__ float get(__bf16 x) { return (float)x; }
  static __device__ __forceinline__ __bf16 put(float x) { return (__bf16)x; }  // to nearest, ties to even
};

template <typename T>
union Piece {  // 16 bytes of a head
  u32x4_t u;
  T e[16 / sizeof(T)];
};

enum { kRopeHalf = 0, kRopePairs = 1, kRopeAny = 2 };

// One unit of work on a head: M = kRopeHalf: the pieces at 16 u bytes of both halves of the rotated part,
// or a piece behind it; kRopePairs: a piece; kRopeAny (rotated parts that are no whole pieces): a pair of
// values, or a value behind the rotated part. A pair is read and written by one thread, so dst may be src.
template <typename T, int M, bool ILV>
__device__ __forceinline__ void rope_unit(const T* src, T* dst, int u, int rot, const float* cs) {
  constexpr int E = 16 / sizeof(T);
  const int half = rot / 2;
  const float* sn = cs + 64;
  if constexpr (M == kRopeHalf) {
    Piece<T> x, y;
    if (u * E < half) {
      x.u = *(const u32x4_t*)(src + u * E);
      y.u = *(const u32x4_t*)(src + half + u * E);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float a = Elem<T>::get(x.e[e]), b = Elem<T>::get(y.e[e]);
        const float c = cs[u * E + e], s = sn[u * E + e];
        x.e[e] = Elem<T>::put(a * c - b * s);
        y.e[e] = Elem<T>::put(b * c + a * s);
      }
      *(u32x4_t*)(dst + u * E) = x.u;
      *(u32x4_t*)(dst + half + u * E) = y.u;
    } else {
      *(u32x4_t*)(dst + half + u * E) = *(const u32x4_t*)(src + half + u * E);
    }
  } else if constexpr (M == kRopePairs) {
    Piece<T> x;
    x.u = *(const u32x4_t*)(src + u * E);
    if (u * E < rot) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float a = Elem<T>::get(x.e[e]), b = Elem<T>::get(x.e[e + 1]);
        const float c = cs[(u * E + e) / 2], s = sn[(u * E + e) / 2];
        x.e[e] = Elem<T>::put(a * c - b * s);
        x.e[e + 1] = Elem<T>::put(b * c + a * s);
      }
    }
    *(u32x4_t*)(dst + u * E) = x.u;
  } else if (u < half) {
    const int i = ILV ? 2 * u : u, j = ILV ? 2 * u + 1 : u + half;
    const float a = Elem<T>::get(src[i]), b = Elem<T>::get(src[j]);
    dst[i] = Elem<T>::put(a * cs[u] - b * sn[u]);
    dst[j] = Elem<T>::put(b * cs[u] + a * sn[u]);
  } else {
    dst[half + u] = src[half + u];
  }
}

template <typename T, int M, bool ILV>
__global__ __launch_bounds__(kRopeThreads) void rope_append(RopeArgs a) {
  __shared__ float cs[128];  // cosines, then sines from 64
  constexpr int E = 16 / sizeof(T);
  const int r = blockIdx.x, tid = threadIdx.x;
  const int b = seq_of_row(a.q_start, a.map.B, r);
  if (b >= a.map.B) return;
  const Chunk c = chunk_of(a.q_start, b, a.total);
  const int base = a.base[b];
  if (base < 0 || r < c.first || r >= c.first + c.n || base >= a.map.cap - (r - c.first)) return;
  const int slot = base + r - c.first;
  const int page = a.map.table[(size_t)b * a.map.P + (slot >> a.map.shift)];
  if (!is_page(a.map, page)) return;
  const int half = a.rot / 2;
  if (tid < half) {
    const double turns = (double)a.map.pos[(size_t)b * a.map.cap + slot] * (double)a.inv_freq[tid] *
                         0.15915494309189533577;  // 1 / (2 pi)
    float s, co;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
    cs[tid] = a.scale * co;
    cs[64 + tid] = a.scale * s;
  }
  __syncthreads();
  // units of a rotated head and of a value head
  const int ur = M == kRopeHalf ? (a.D - half) / E : M == kRopePairs ? a.D / E : a.D - half;
  const int uv = a.D / E;
  const int nq = a.Hq * ur, nk = a.k != nullptr ? a.Hkv * ur : 0, nv = a.k != nullptr ? a.Hkv * uv : 0;
  const size_t head_rows = (size_t)1 << a.map.shift;
  const size_t row0 = (size_t)page * a.Hkv * head_rows + (slot & (head_rows - 1));
  for (int i = tid; i < nq + nk + nv; i += kRopeThreads) {
    if (i < nq) {
      const int h = i / ur;
      rope_unit<T, M, ILV>((const T*)a.q + r * a.q_stride + h * a.D,
                           (T*)a.q_out + ((size_t)r * a.Hq + h) * a.D, i - h * ur, a.rot, cs);
    } else if (i < nq + nk) {
      const int h = (i - nq) / ur;
      rope_unit<T, M, ILV>((const T*)a.k + r * a.k_stride + h * a.D,
                           (T*)a.pk + (row0 + h * head_rows) * a.D, i - nq - h * ur, a.rot, cs);
    } else {
      const int h = (i - nq - nk) / uv, u = i - nq - nk - h * uv;
      *(u32x4_t*)((T*)a.pv + (row0 + h * head_rows) * a.D + u * E) =
          *(const u32x4_t*)((const T*)a.v + r * a.v_stride + h * a.D + u * E);
    }
  }
}

template <typename T>
static void launch_typed(const RopeArgs& a, bool interleaved, hipStream_t st) {
  constexpr int E = 16 / sizeof(T);
  const dim3 grid(a.total), block(kRopeThreads);
  if (interleaved && a.rot % E == 0)
    hipLaunchKernelGGL((rope_append<T, kRopePairs, true>), grid, block, 0, st, a);
  else if (!interleaved && a.rot / 2 % E == 0)
    hipLaunchKernelGGL((rope_append<T, kRopeHalf, false>), grid, block, 0, st, a);
  else if (interleaved)
    hipLaunchKernelGGL((rope_append<T, kRopeAny, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((rope_append<T, kRopeAny, false>), grid, block, 0, st, a);
}

hipError_t launch_rope(const lg_paged_layer& l, const lg_page_map& m, const void* q, int64_t q_stride,
                       const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                       const float* inv_freq, int rot, bool interleaved, float scale, void* q_out,
                       const int32_t* q_start, const int32_t* base, int total, hipStream_t st) {
  RopeArgs a = {};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out = q_out;
  a.pk = l.k;
  a.pv = l.v;
  a.inv_freq = inv_freq;
  a.q_start = q_start;
  a.base = base;
  a.map = map_args(m);
  a.Hq = l.n_q_heads;
  a.Hkv = l.n_kv_heads;
  a.D = l.head_dim;
  a.rot = rot;
  a.total = total;
  a.scale = scale;
  if (l.dtype == LG_BF16)
    launch_typed<__bf16>(a, interleaved, st);
  else
    launch_typed<float>(a, interleaved, st);
  return hipGetLastError();
}

}  // namespace lg
