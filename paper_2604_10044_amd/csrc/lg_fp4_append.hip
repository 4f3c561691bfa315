// lg_fp4_append.hip -- rotary positions on several axes with the append to pages of any type
// (lg_rope_append_axes), and 4-bit rows read back as values (lg_page_unpack_fp4).
//
// A group of 32 values x_i becomes codes c_i and an exponent: with m = max |x_i| the unit u is the smallest power of
// two that has m <= 6 u, and c_i is x_i / u to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (the conversion instruction's
// rounding: ties to the even code, a tie being the same as the definition's in every unit). A lane holds 8 values, so
// a group is four lanes of a row of 16 and m two exchanges between neighbours.
//
// Memory bounds long chunks: two prompts of 8192 tokens of 32 / 8 heads of 128 in bfloat16 on three axes, 354 MB, 71 us, 5.0 TB/s (a
// copy reaches 5.13). A decode step's append is a chain of dependent reads and one launch: 3.9 us for 32 sequences.
#include "lg_fp4.h"
#include "lg_rope.h"

namespace lg {

struct AxesArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, coord_stride;
  void *q_out, *pk, *pv;
  const float* inv_freq;
  const int32_t *axis, *coord, *q_start, *base;
  MapArgs map;
  int32_t Hq, Hkv, D, rot, total, n_axes;
  float scale;
};

constexpr int kAxesThreads = 256;

// 8 values of a head as float32
struct Values {
  float x[8];
};
template <typename T>
__device__ __forceinline__ Values load_values(const T* src) {
  Values y;
  constexpr int E = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < 8 / E; ++i) {
    Piece<T> p;
    p.u = *(const u32x4_t*)(src + i * E);
#pragma unroll
    for (int e = 0; e < E; ++e) y.x[i * E + e] = Elem<T>::get(p.e[e]);
  }
  return y;
}

// The largest of x over groups of four lanes.
__device__ __forceinline__ uint32_t max_of_four(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));  // quad_perm 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));  // quad_perm 2 3 0 1
}

// The codes of a lane's 8 values and the exponent byte of the group that four lanes hold. With the bits of m as
// exponent and fraction, m <= 1.5 2^(x - 127) exactly when the fraction is at most 0x400000: the sum below carries
// otherwise, and u is 2^-2 of that power.
__device__ __forceinline__ uint32_t encode(const Values& y, uint32_t* exponent) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(y.x[i]) & 0x7fffffffu);
  m = max_of_four(m);
  if (m >= 0x7f800000u) {
    *exponent = 255;
    return 0;
  }
  const int x = min(max((int)((m + 0x3fffffu) >> 23) - 2, 2), 252);
  *exponent = x;
  const float u = __uint_as_float((uint32_t)x << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y.x[0], y.x[1], u, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y.x[2], y.x[3], u, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y.x[4], y.x[5], u, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y.x[6], y.x[7], u, 3);
}

// Values 8 u .. 8 u + 7 of a rotated head. The products and sums are rounded one by one, as a program that multiplies and
// adds would: a value next to the middle of two codes then falls to the same side.
template <typename T, int M, bool ILV>
__device__ __forceinline__ Values rotated_eight(const T* src, int u, int rot, const float* cs) {
#pragma clang fp contract(off)
  const int half = rot / 2, i0 = 8 * u;
  const float* sn = cs + 64;
  Values y = load_values(src + i0);
  if constexpr (M == kRopePairs) {
    if (i0 < rot) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float a = y.x[e], b = y.x[e + 1], c = cs[(i0 + e) / 2], s = sn[(i0 + e) / 2];
        const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
        y.x[e] = ac - bs;
        y.x[e + 1] = bc + as;
      }
    }
  } else if constexpr (M == kRopeHalf) {
    if (i0 < rot) {
      const bool low = i0 < half;
      const int j = low ? i0 : i0 - half;
      const Values z = load_values(src + (low ? i0 + half : j));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = cs[j + e], s = sn[j + e];
        const float yc = y.x[e] * c, zs = z.x[e] * s;
        y.x[e] = low ? yc - zs : yc + zs;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + e;
      if (i < rot) {
        const bool low = ILV ? (i & 1) == 0 : i < half;
        const int j = ILV ? i / 2 : low ? i : i - half;
        const float z = Elem<T>::get(src[ILV ? i ^ 1 : low ? i + half : j]);
        const float yc = y.x[e] * cs[j], zs = z * sn[j];
        y.x[e] = low ? yc - zs : yc + zs;
      }
    }
  }
  return y;
}

// The fraction of a turn, at most half a turn in size, of the angle p f: within 2^-53 of a turn at any p. The product has up to
// 55 bits and its whole turns up to 31, so it is carried as two doubles, as is 1 / (2 pi); the whole turns leave in a fused
// step (with one double each, the angle at 2^30 is off by 2e-7, 3.5 units of a float32 sine).
__device__ __forceinline__ double fraction_of_turn(int p, float f) {
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;  // together 1 / (2 pi)
  const double x = (double)p * (double)f, rest = fma((double)p, (double)f, -x);
  return fma(x, kTurn, -rint(x * kTurn)) + fma(x, kTurnRest, rest * kTurn);
}

// A workgroup a token. Its rot_dim / 2 angles are formed once, in double (positions and coordinates reach 2^31, and what
// is rounded to 4 bits shall not depend on the last bits of a sine): a thread each. The
// threads then walk the token's keys and values (8 values each, so that four lanes are a group) and its queries.
template <typename T, bool FP4, int M, bool ILV>
__global__ __launch_bounds__(kAxesThreads) void append_axes(AxesArgs a) {
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
    const int p = a.n_axes > 0 ? a.coord[min(max(a.axis[tid], 0), a.n_axes - 1) * a.coord_stride + r]
                               : a.map.pos[(size_t)b * a.map.cap + slot];
    double s, co;
    sincospi(2. * fraction_of_turn(p, a.inv_freq[tid]), &s, &co);
    cs[tid] = (float)((double)a.scale * co);
    cs[64 + tid] = (float)((double)a.scale * s);
  }
  __syncthreads();
  const int ur = M == kRopeHalf ? (a.D - half) / E : M == kRopePairs ? a.D / E : a.D - half;  // units of a rotated head
  const size_t head_rows = (size_t)1 << a.map.shift;
  const size_t in_page = slot & (head_rows - 1);
  const int nq = a.q != nullptr ? a.Hq * ur : 0;
  if constexpr (FP4) {
    const int ue = a.D / 8, nk = a.k != nullptr ? a.Hkv * ue : 0;
    const size_t block = fp4_block(a.D, a.map.shift);
    for (int i = tid; i < 2 * nk + nq; i += kAxesThreads) {
      if (i < 2 * nk) {  // a group's four lanes are here together: nk is a multiple of 8
        const bool is_k = i < nk;
        const int x = is_k ? i : i - nk, h = x / ue, u = x - h * ue;
        const T* src = is_k ? (const T*)a.k + r * a.k_stride + h * a.D : (const T*)a.v + r * a.v_stride + h * a.D;
        const Values y = is_k ? rotated_eight<T, M, ILV>(src, u, a.rot, cs) : load_values(src + 8 * u);
        uint32_t exponent;
        const uint32_t codes = encode(y, &exponent);
        char* at = (char*)(is_k ? a.pk : a.pv) + ((size_t)page * a.Hkv + h) * block;
        *(uint32_t*)(at + in_page * fp4_row(a.D) + 4 * u) = codes;
        if ((u & 3) == 0)
          *(uint8_t*)(at + head_rows * fp4_row(a.D) + in_page * fp4_exps(a.D) + u / 4) = (uint8_t)exponent;
      } else {
        const int h = (i - 2 * nk) / ur;
        rope_unit<T, M, ILV>((const T*)a.q + r * a.q_stride + h * a.D, (T*)a.q_out + ((size_t)r * a.Hq + h) * a.D,
                             i - 2 * nk - h * ur, a.rot, cs);
      }
    }
  } else {
    const int uv = a.D / E, nk = a.k != nullptr ? a.Hkv * ur : 0, nv = a.k != nullptr ? a.Hkv * uv : 0;
    const size_t row0 = (size_t)page * a.Hkv * head_rows + in_page;
    for (int i = tid; i < nq + nk + nv; i += kAxesThreads) {
      if (i < nq) {
        const int h = i / ur;
        rope_unit<T, M, ILV>((const T*)a.q + r * a.q_stride + h * a.D, (T*)a.q_out + ((size_t)r * a.Hq + h) * a.D,
                             i - h * ur, a.rot, cs);
      } else if (i < nq + nk) {
        const int h = (i - nq) / ur;
        rope_unit<T, M, ILV>((const T*)a.k + r * a.k_stride + h * a.D, (T*)a.pk + (row0 + h * head_rows) * a.D,
                             i - nq - h * ur, a.rot, cs);
      } else {
        const int h = (i - nq - nk) / uv, u = i - nq - nk - h * uv;
        *(u32x4_t*)((T*)a.pv + (row0 + h * head_rows) * a.D + u * E) =
            *(const u32x4_t*)((const T*)a.v + r * a.v_stride + h * a.D + u * E);
      }
    }
  }
}

template <typename T, bool FP4>
static void launch_axes_typed(const AxesArgs& a, bool interleaved, hipStream_t st) {
  constexpr int E = FP4 ? 8 : 16 / sizeof(T);  // values that a lane takes of one head's half at least
  const dim3 grid(a.total), block(kAxesThreads);
  if (interleaved && a.rot % E == 0)
    hipLaunchKernelGGL((append_axes<T, FP4, kRopePairs, true>), grid, block, 0, st, a);
  else if (!interleaved && a.rot / 2 % E == 0)
    hipLaunchKernelGGL((append_axes<T, FP4, kRopeHalf, false>), grid, block, 0, st, a);
  else if (interleaved)
    hipLaunchKernelGGL((append_axes<T, FP4, kRopeAny, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((append_axes<T, FP4, kRopeAny, false>), grid, block, 0, st, a);
}

hipError_t launch_append_axes(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, const void* q,
                              int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              const float* inv_freq, int rot, bool interleaved, float scale, const int32_t* axis,
                              const int32_t* coord, int64_t coord_stride, int n_axes, void* q_out,
                              const int32_t* q_start, const int32_t* base, int total, hipStream_t st) {
  AxesArgs a = {};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.coord_stride = coord_stride;
  a.q_out = q_out;
  a.pk = l.k;
  a.pv = l.v;
  a.inv_freq = inv_freq;
  a.axis = axis;
  a.coord = coord;
  a.q_start = q_start;
  a.base = base;
  a.map = map_args(m);
  a.Hq = l.n_q_heads;
  a.Hkv = l.n_kv_heads;
  a.D = l.head_dim;
  a.rot = rot;
  a.total = total;
  a.n_axes = n_axes;
  a.scale = scale;
  if (l.dtype == LG_FP4) {
    if (dtype == LG_BF16) launch_axes_typed<__bf16, true>(a, interleaved, st);
    else launch_axes_typed<float, true>(a, interleaved, st);
  } else {
    if (dtype == LG_BF16) launch_axes_typed<__bf16, false>(a, interleaved, st);
    else launch_axes_typed<float, false>(a, interleaved, st);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// Reading back
// ------------------------------------------------------------------------------------------
struct UnpackArgs {
  const char *pk, *pv;
  void *k, *v;
  const int32_t *q_start, *base;
  MapArgs map;
  int32_t Hkv, D, total;
  int32_t log_rows;  // slots of a workgroup
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void store_values(__bf16* dst, uint32_t codes, float unit) {
  const bf16x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3)};
  u32x4_t x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(uint32_t, y[i]);
  *(u32x4_t*)dst = x;
}
__device__ __forceinline__ void store_values(float* dst, uint32_t codes, float unit) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  *(f32x4*)dst = f32x4{a[0], a[1], b[0], b[1]};
  *(f32x4*)(dst + 4) = f32x4{c[0], c[1], d[0], d[1]};
}

// A workgroup takes up to 16 slots that follow each other: their rows of a head, 1 KB in a page, are read by one CU (a
// workgroup a slot reads lines that another one reads too, and finds its sequence for 256 pieces alone: a batch of 23700 slots of
// 8 heads of 128, 123 MB, took 37 us, 28 so). A thread reads 4 bytes of a row with their exponent and writes 8 values. Memory
// bounds it.
constexpr int kUnpackRows = 16;

template <typename T>
__global__ __launch_bounds__(kAxesThreads) void page_unpack(UnpackArgs a) {
  __shared__ int2 place[kUnpackRows];  // page (-1: nothing to read) and row in it
  const int rows = 1 << a.log_rows, r0 = blockIdx.x * rows, tid = threadIdx.x;
  if (tid < 64) {
    const int r = r0 + min(tid, rows - 1);
    const int b = seq_behind(a.q_start, a.map.B, seq_of_row(a.q_start, a.map.B, r0), r);  // rows ascend, as sequences do
    int page = -1, slot = 0;
    if (b < a.map.B && r < a.total) {
      const Chunk c = chunk_of(a.q_start, b, a.total);
      const int base = a.base[b], i = r - c.first;
      if (base >= 0 && i >= 0 && i < c.n && base < a.map.cap - i) {
        slot = base + i;
        page = a.map.table[(size_t)b * a.map.P + (slot >> a.map.shift)];
        if (!is_page(a.map, page)) page = -1;
      }
    }
    if (tid < rows) place[tid] = int2{page, slot & ((1 << a.map.shift) - 1)};
  }
  __syncthreads();
  const int log_pieces = a.D == 128 ? 4 : 3, n = a.Hkv << (log_pieces + a.log_rows);
  const size_t exps = (size_t)fp4_row(a.D) << a.map.shift, block = fp4_block(a.D, a.map.shift);
  for (int i = tid; i < 2 * n; i += kAxesThreads) {
    const bool is_k = i < n;
    const int x = is_k ? i : i - n, u = x & ((1 << log_pieces) - 1), in = x >> log_pieces & (rows - 1), h = x >> (log_pieces + a.log_rows);
    T* dst = (T*)(is_k ? a.k : a.v);
    const int2 at = place[in];
    if (dst == nullptr || at.x < 0) continue;
    const char* from = (is_k ? a.pk : a.pv) + ((size_t)at.x * a.Hkv + h) * block;
    const uint32_t codes = *(const uint32_t*)(from + at.y * fp4_row(a.D) + 4 * u);
    const uint32_t e = *(const uint8_t*)(from + exps + at.y * fp4_exps(a.D) + u / 4);
    store_values(dst + ((size_t)(r0 + in) * a.Hkv + h) * a.D + 8 * u, codes, fp4_unit(e));
  }
}

hipError_t launch_unpack(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, void* k, void* v,
                         const int32_t* q_start, const int32_t* base, int total, hipStream_t st) {
  UnpackArgs a = {};
  a.pk = (const char*)l.k;
  a.pv = (const char*)l.v;
  a.k = k;
  a.v = v;
  a.q_start = q_start;
  a.base = base;
  a.map = map_args(m);
  a.Hkv = l.n_kv_heads;
  a.D = l.head_dim;
  a.total = total;
  a.log_rows = 0;  // as many as leave a thousand workgroups
  while (2 << a.log_rows <= kUnpackRows && (total >> (a.log_rows + 1)) >= 1024) ++a.log_rows;
  const dim3 grid((unsigned)((total + (1 << a.log_rows) - 1) >> a.log_rows));
  if (dtype == LG_BF16)
    hipLaunchKernelGGL(page_unpack<__bf16>, grid, dim3(kAxesThreads), 0, st, a);
  else
    hipLaunchKernelGGL(page_unpack<float>, grid, dim3(kAxesThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace lg
