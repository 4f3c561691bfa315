// lg_paged_attend.hip -- attention of a step's new tokens over the pages of their sequences
// (lg_paged_attend).
//
// The query rows of one KV head of one sequence are its tokens' G query heads, token by token: row
// R = i G + g. A wave takes 32 of them and walks the slots in tiles with the running maximum m, sum l
// and output O of a softmax, all float32:
//   S^T = K Q^T    (keys x rows)   A = K from LDS, B = Q from registers
//   m' = max(m, max S), P = 2^(S - m'), l = l 2^(m - m') + sum P, and the suffix sum likewise
//   O^T = O^T 2^(m - m') + V^T P^T   A = V^T read transposed from LDS, B = P^T
// With S transposed a lane holds 16 keys of ONE row (the accumulator of v_mfma_f32_32x32: column =
// lane % 32, rows 8 i + 4 (lane / 32) + j), so the maximum and the sums are in the lane but for one exchange
// with lane ^ 32, and the rounded P is the B operand of the second product as it lies in the registers:
// V^T is read in the same order of keys. Scores are in units of log 2 (exp2).
//
// Two shapes of workgroup in one launch (template KW, waves along the keys):
//   KW = 1  sequences with more than 32 query rows: 128 rows, four waves of 32, which share every tile.
//   KW = 4  the others (a decode step: G rows): the four waves take every fourth tile of the sequence, each
//           with LDS of its own and no barrier, and their (m, l, O) are joined at the end.
// When these workgroups are fewer than the CUs hold, the slots of a row are split over several and a second
// launch joins them.
//
// A tile whose slots every row of the wave sees needs no comparison. In the others (the end of the
// causal triangle, the edges of the window and of the suffix) visibility is decided slot by slot from its
// number and position. There a value that some row does not see could still reach it as 0 x inf = NaN
// through the matrix product: when such a tile holds a value that is not finite, its product is
// formed term by term for the rows that see it.
#include "lg_paged_internal.h"

namespace lg {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kWaveRows = 32;
constexpr int kManyRows = 128;   // rows of a KW = 1 workgroup
constexpr int kPagedThreads = 256;
// Workgroups a launch aims for by splitting slots: two a CU.
constexpr long kPagedTarget = 512;
constexpr int kMinSplitSlots = 256;  // slots of a split at least (by capacity)
constexpr int kHidden = 0x7fffffff;  // position of a slot whose page is missing

struct PagedAttendArgs {
  const void *q, *k, *v;
  void* out;
  const int32_t *q_start, *base, *suffix_w;
  float *lse, *suffix, *conf;
  float *po, *pml;  // split partials: [ns][total Hq][D]; [ns][total Hq][4] (m, l, suffix sum)
  MapArgs map;
  int32_t Hq, Hkv, G, total, max_chunk, window, n_sink, ns, many_tiles;
  float scale_log2;
};

template <typename T, int D>
struct Tile {
  static constexpr bool kF32 = sizeof(T) == 4;
  static constexpr int kRowBytes = D * (int)sizeof(T);
  // Row strides in LDS: the 16-byte pieces of K that a read takes from 16 rows, and the 32-byte pieces
  // (4 lanes x 8 bytes) of V that a transposed read takes from 8 rows, fall into different banks.
  static constexpr int kStrideK = kRowBytes + 16;
  static constexpr int kStrideV = kRowBytes + (kF32 ? 32 : 64);
};

// Sizes of the team that shares a tile: the workgroup (KW = 1) or a wave (KW = 4).
template <typename T, int D, int KW>
struct Team : Tile<T, D> {
  using B = Tile<T, D>;
  static constexpr int kKeys = B::kF32 || KW > 1 ? 32 : 64;  // slots of a tile
  static constexpr int kThreads = KW > 1 ? 64 : kPagedThreads;
  static constexpr int kPieces = kKeys * B::kRowBytes / 16 / kThreads;  // 16-byte pieces a thread, of K and of V
  static constexpr int kRowsStep = kThreads * 16 / B::kRowBytes;         // rows between a thread's pieces
  static constexpr int kLdsK = kKeys * B::kStrideK, kLdsV = kKeys * B::kStrideV;
  static constexpr int kLds = kLdsK + kLdsV + 4 * kKeys;
  // the join of KW = 4: a wave's O as [row][D + 4] and its m, l, suffix sums
  static constexpr int kLdsJoin = KW > 1 ? kWaveRows * (D + 4) * 4 + 3 * kWaveRows * 4 : 0;
  static constexpr int kLdsTeam = (kLds > kLdsJoin ? kLds : kLdsJoin) + 15 & ~15;
};

template <typename T, int D>
constexpr int paged_lds() {
  return Team<T, D, 1>::kLdsTeam > 4 * Team<T, D, 4>::kLdsTeam ? Team<T, D, 1>::kLdsTeam
                                                               : 4 * Team<T, D, 4>::kLdsTeam;
}

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // to nearest, ties to even
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

__device__ __forceinline__ bool odd_bits(uint32_t x, bool f32) {  // an infinity or NaN in a word
  return f32 ? (x & 0x7f800000u) == 0x7f800000u
             : (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
}

// conf[b] = max(conf[b], mass): masses are not negative, so their order is that of their bits; a NaN (of
// whatever sign) makes it NaN.
__device__ __forceinline__ void raise_conf(float* conf, float mass) {
  atomicMax((int*)conf, mass != mass ? 0x7fc00000 : __float_as_int(mass));
}

// What a workgroup attends with: its rows, and the slots that any of them may see.
struct Job {
  int b, h;         // sequence, KV head
  int first;        // row of the sequence's first token in q
  int rows;         // query rows of the sequence (tokens x G)
  int row0;         // first query row of the workgroup
  int base;         // slot of the first token
  int sink_tiles;   // tiles from slot 0 for the first tokens that stay visible
  int tile0;        // first tile of the rest
  int t_begin, t_end;  // this split's share of the sink_tiles + rest tiles
  int split;
};

template <typename T, int D, int KW>
__device__ __forceinline__ void paged_body(const PagedAttendArgs& a, const Job& job, char* lds) {
  using C = Team<T, D, KW>;
  constexpr bool F32 = C::kF32;
  constexpr int NK = C::kKeys, NB = NK / 32, ND = D / 32, NP = C::kPieces;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
  const int ttid = KW > 1 ? lane : tid;  // thread of the team
  char* const my = KW > 1 ? lds + wave * C::kLdsTeam : lds;
  char* const ldsk = my;
  char* const ldsv = my + C::kLdsK;
  int* const ldsp = (int*)(my + C::kLdsK + C::kLdsV);
  const MapArgs& m = a.map;
  const int32_t* const table = m.table + (size_t)job.b * m.P;
  const int32_t* const pos = m.pos + (size_t)job.b * m.cap;

  // The lane's query row.
  const int wrow0 = job.row0 + (KW > 1 ? 0 : wave * kWaveRows);
  const int R = wrow0 + col;
  const bool live = R < job.rows;
  const int Rc = live ? R : job.rows - 1;  // rows behind the last repeat it; they are not written
  const int tok = Rc / a.G, g = Rc - tok * a.G;
  const size_t qrow = (size_t)(job.first + tok) * a.Hq + job.h * a.G + g;
  const int slot_q = job.base + tok;
  const int p_q = pos[slot_q];
  const int sw = a.suffix_w != nullptr ? a.suffix_w[job.b] : 0;
  // the row sees pos > win and, of these, counts pos > suf as its suffix
  const int win = a.window > 0 ? (int)max((long long)p_q - a.window, (long long)INT32_MIN) : INT32_MIN;
  const int suf = (int)max((long long)p_q - max(sw, 0), (long long)INT32_MIN);
  // bounds over the wave's rows (tokens ascend with the row, positions with the token)
  const int slot_lo = __builtin_amdgcn_readlane(slot_q, 0), slot_hi = __builtin_amdgcn_readlane(slot_q, 31);
  const int win_hi = __builtin_amdgcn_readlane(win, 31);
  const int suf_lo = __builtin_amdgcn_readlane(suf, 0), suf_hi = __builtin_amdgcn_readlane(suf, 31);
  const bool idle = wrow0 >= job.rows;  // KW = 1: a wave without rows only loads

  // Q as the B operand: bf16: values 16 kk + 8 half ..; float32: values half D / 2 + 4 u ..
  u32x4_t qf[F32 ? D / 8 : D / 16];
  {
    const char* src = (const char*)a.q + qrow * C::kRowBytes;
#pragma unroll
    for (int i = 0; i < (F32 ? D / 8 : D / 16); ++i)
      qf[i] = *(const u32x4_t*)(src + (F32 ? half * (D / 2) * 4 + 16 * i : 32 * i + 16 * half));
  }

  f32x16 O[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[d][i] = 0.f;
  float mx = -INFINITY, l = 0.f, sfx = 0.f;  // l and sfx: the lane's half of the keys

  const int n_all = job.t_end;
  const int t_first = KW > 1 ? job.t_begin + wave : job.t_begin;
  const int end_slot = min(job.base + (min(job.row0 + (KW > 1 ? kWaveRows : kManyRows), job.rows) - 1) / a.G + 1,
                           m.cap);  // slots from here on no row of the workgroup sees

  u32x4_t kr[NP], vr[NP];
  int pr = 0;
  auto slot_of = [&](int t) { return (t < job.sink_tiles ? t : t - job.sink_tiles + job.tile0) * NK; };
  // Loads of a tile into registers: rows behind end_slot and rows of missing pages become zero.
  auto load = [&](int t) {
    const int s0 = slot_of(t);
    const int r0 = ttid / (C::kRowBytes / 16), piece = ttid % (C::kRowBytes / 16);
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int s = s0 + r0 + u * C::kRowsStep;
      const int page = s < end_slot ? table[s >> m.shift] : -1;
      if (is_page(m, page)) {
        const size_t at = ((((size_t)page * a.Hkv + job.h) << m.shift) + (s & ((1 << m.shift) - 1))) * C::kRowBytes + 16 * piece;
        kr[u] = *(const u32x4_t*)((const char*)a.k + at);
        vr[u] = *(const u32x4_t*)((const char*)a.v + at);
      } else {
        kr[u] = u32x4_t{};
        vr[u] = u32x4_t{};
      }
    }
    if (ttid < NK) {
      const int s = s0 + ttid;
      pr = s < end_slot && is_page(m, table[s >> m.shift]) ? pos[s] : kHidden;
    }
  };
  auto store = [&]() {
    const int r0 = ttid / (C::kRowBytes / 16), piece = ttid % (C::kRowBytes / 16);
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int r = r0 + u * C::kRowsStep;
      *(u32x4_t*)(ldsk + r * C::kStrideK + 16 * piece) = kr[u];
      *(u32x4_t*)(ldsv + r * C::kStrideV + 16 * piece) = vr[u];
    }
    if (ttid < NK) ldsp[ttid] = pr;
  };
  auto team_sync = [&]() {
    if constexpr (KW > 1) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      __syncthreads();
    }
  };

  if (t_first < n_all) load(t_first);
  for (int t = t_first; t < n_all; t += KW) {
    team_sync();  // the tile before is read
    store();
    team_sync();
    if (t + KW < n_all) load(t + KW);
    const int s0 = slot_of(t);
    if (idle || s0 > slot_hi) continue;

    // S^T, one 32 x 32 block per 32 keys
    f32x16 S[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) S[nb][i] = 0.f;
      const char* row = ldsk + (32 * nb + col) * C::kStrideK;
      if constexpr (F32) {
#pragma unroll
        for (int u = 0; u < D / 8; ++u) {
          const u32x4_t kx = *(const u32x4_t*)(row + half * (D / 2) * 4 + 16 * u);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            S[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kx[e]), __uint_as_float(qf[u][e]),
                                                         S[nb], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          S[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8, *(const u32x4_t*)(row + 32 * kk + 16 * half)),
              __builtin_bit_cast(bf16x8, qf[kk]), S[nb], 0, 0, 0);
      }
    }

    // What the tile needs compared, the same in all lanes.
    const int tp = ldsp[lane & (NK - 1)];
    const int p_first = __builtin_amdgcn_readlane(tp, 0), p_last = __builtin_amdgcn_readlane(tp, NK - 1);
    const bool hidden = __ballot(tp == kHidden) != 0;
    const bool masked = hidden || s0 + NK - 1 > slot_lo ||
                        (a.window > 0 && p_first <= win_hi && p_last >= a.n_sink);
    // suffix: 0 none of the tile, 1 all of it, 2 compare
    const int suf_how = a.suffix == nullptr && a.conf == nullptr ? 0
                        : masked ? 2 : p_last <= suf_lo ? 0 : p_first > suf_hi ? 1 : 2;

    float tmax = -INFINITY;
    if (masked) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 32 * nb + 8 * (i >> 2) + 4 * half + (i & 3);
          const int pj = ldsp[key];
          const bool see = s0 + key <= slot_q && pj != kHidden && (pj > win || a.window == 0 || pj < a.n_sink);
          S[nb][i] = see ? S[nb][i] * a.scale_log2 : -INFINITY;
          tmax = fmaxf(tmax, S[nb][i]);
        }
    } else {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          S[nb][i] *= a.scale_log2;
          tmax = fmaxf(tmax, S[nb][i]);
        }
    }
    tmax = fmaxf(tmax, other_half(tmax));
    const float m_new = fmaxf(mx, tmax);
    const float ms = m_new == -INFINITY ? 0.f : m_new;  // a row that has seen nothing yet
    if (__any(m_new > mx)) {
      const float f = __builtin_amdgcn_exp2f(mx - ms);  // 0 from -inf
      l *= f;
      sfx *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[d][i] *= f;
      mx = m_new;
    }
    float sum = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        S[nb][i] = __builtin_amdgcn_exp2f(S[nb][i] - ms);
        sum += S[nb][i];
      }
    l += sum;
    if (suf_how == 1) {
      sfx += sum;
    } else if (suf_how == 2) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 32 * nb + 8 * (i >> 2) + 4 * half + (i & 3);
          sfx += ldsp[key] > suf ? S[nb][i] : 0.f;
        }
    }

    bool odd = false;
    if (masked) {
      for (int i = lane; i < NK * (C::kRowBytes / 16); i += 64) {
        const u32x4_t x = *(const u32x4_t*)(ldsv + i / (C::kRowBytes / 16) * C::kStrideV + i % (C::kRowBytes / 16) * 16);
        odd |= odd_bits(x[0], F32) || odd_bits(x[1], F32) || odd_bits(x[2], F32) || odd_bits(x[3], F32);
      }
      odd = __any(odd);
    }
    if (!odd) {
      // O^T += V^T P^T
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const char* row = ldsv + (8 * (i >> 2) + 4 * half + (i & 3)) * C::kStrideV + 4 * col;
#pragma unroll
          for (int d = 0; d < ND; ++d)
            O[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*(const float*)(row + 128 * d), S[0][i], O[d], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            u32x4_t p;  // the weights as bfloat16: the matrix product's type
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = pack_bf16(S[nb][8 * s + 2 * e], S[nb][8 * s + 2 * e + 1]);
            // a 16-lane group reads 4 keys x 16 values and gets them transposed: lane = value
            const char* row = ldsv + (32 * nb + 16 * s + 4 * half + ((lane & 15) >> 2)) * C::kStrideV +
                              32 * ((lane >> 4) & 1) + 8 * (lane & 3);
#pragma unroll
            for (int d = 0; d < ND; ++d) {
              const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) i16x4*)(row + 64 * d));
              const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) i16x4*)(row + 64 * d + 8 * C::kStrideV));
              const u32x2_t x = __builtin_bit_cast(u32x2_t, lo), y = __builtin_bit_cast(u32x2_t, hi);
              O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  __builtin_bit_cast(bf16x8, u32x4_t{x[0], x[1], y[0], y[1]}), __builtin_bit_cast(bf16x8, p),
                  O[d], 0, 0, 0);
            }
          }
      }
    } else {
      // A value that is not finite in a tile that not every row sees: term by term, seen slots only.
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const int key = 32 * nb + 8 * (i >> 2) + 4 * hh + (i & 3);
            const float p = __shfl(S[nb][i], 32 * hh + col, 64);
            const int pj = ldsp[key];
            const bool see = s0 + key <= slot_q && pj != kHidden && (pj > win || a.window == 0 || pj < a.n_sink);
            if (see) {
#pragma unroll
              for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const int dd = 32 * d + 8 * (e >> 2) + 4 * half + (e & 3);
                  const float x = F32 ? *(const float*)(ldsv + key * C::kStrideV + 4 * dd)
                                      : __uint_as_float((uint32_t)*(const uint16_t*)(ldsv + key * C::kStrideV + 2 * dd) << 16);
                  O[d][e] += p * x;
                }
            }
          }
    }
  }

  l += other_half(l);
  sfx += other_half(sfx);

  if constexpr (KW == 1) {
    if (idle || !live) return;
    if (a.ns > 1) {
      const size_t at = (size_t)job.split * a.total * a.Hq + qrow;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(a.po + at * D + 32 * d + 8 * i + 4 * half) =
              f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
      if (half == 0) *(f32x4*)(a.pml + at * 4) = f32x4{mx, l, sfx, 0.f};
      return;
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;  // no slot seen: 0
    T* dst = (T*)a.out + qrow * D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 32 * d + 8 * i + 4 * half;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : O[d][4 * i + e] * inv;
        if constexpr (F32)
          *(f32x4*)(dst + at) = f32x4{x[0], x[1], x[2], x[3]};
        else
          *(u32x2_t*)(dst + at) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
      }
    if (half == 0) {
      a.lse[qrow] = l == 0.f ? -INFINITY : kLn2 * (mx + __builtin_amdgcn_logf(l));
      const float mass = l == 0.f ? 0.f : sfx * inv;
      if (a.suffix != nullptr) a.suffix[qrow] = mass;
      if (a.conf != nullptr && tok == job.rows / a.G - 1)
        raise_conf(a.conf + job.b, mass);
    }
  } else {
    // Join the four waves: their numerators and statistics through LDS, 8 threads a row.
    float* const num = (float*)my;
    float* const st = num + kWaveRows * (D + 4);
    team_sync();
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(num + col * (D + 4) + 32 * d + 8 * i + 4 * half) =
            f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
    if (half == 0) {
      st[col] = mx;
      st[kWaveRows + col] = l;
      st[2 * kWaveRows + col] = sfx;
    }
    __syncthreads();
    const int r = tid >> 3, part = tid & 7;
    if (job.row0 + r >= job.rows) return;
    constexpr int kStatAt = kWaveRows * (D + 4);
    float wm[4], M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      wm[w] = ((const float*)(lds + w * C::kLdsTeam))[kStatAt + r];
      M = fmaxf(M, wm[w]);
    }
    const float Ms = M == -INFINITY ? 0.f : M;
    float L = 0.f, SF = 0.f, x[D / 8] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float* src = (const float*)(lds + w * C::kLdsTeam);
      const float f = __builtin_amdgcn_exp2f(wm[w] - Ms);
      L += f * src[kStatAt + kWaveRows + r];
      SF += f * src[kStatAt + 2 * kWaveRows + r];
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const f32x4 y = *(const f32x4*)(src + r * (D + 4) + 32 * i + 4 * part);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] += f * y[e];
      }
    }
    const int tk = (job.row0 + r) / a.G, gg = job.row0 + r - tk * a.G;
    const size_t row = (size_t)(job.first + tk) * a.Hq + job.h * a.G + gg;
    if (a.ns > 1) {
      const size_t at = (size_t)job.split * a.total * a.Hq + row;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        *(f32x4*)(a.po + at * D + 32 * i + 4 * part) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
      if (part == 0) *(f32x4*)(a.pml + at * 4) = f32x4{M, L, SF, 0.f};
      return;
    }
    const float inv = 1.f / L;
    T* dst = (T*)a.out + row * D;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = L == 0.f ? 0.f : x[4 * i + e] * inv;
      if constexpr (F32)
        *(f32x4*)(dst + 32 * i + 4 * part) = f32x4{y[0], y[1], y[2], y[3]};
      else
        *(u32x2_t*)(dst + 32 * i + 4 * part) = u32x2_t{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    }
    if (part == 0) {
      a.lse[row] = L == 0.f ? -INFINITY : kLn2 * (M + __builtin_amdgcn_logf(L));
      const float mass = L == 0.f ? 0.f : SF * inv;
      if (a.suffix != nullptr) a.suffix[row] = mass;
      if (a.conf != nullptr && tk == job.rows / a.G - 1)
        raise_conf(a.conf + job.b, mass);
    }
  }
}

// The slots that the workgroup's rows may see, in tiles, and this split's share of them. A window's first
// slot is at least (slot - window + 1): positions ascend by at least one a slot; slots below n_sink
// likewise hold the positions below n_sink. Holes make the true range shorter: compared slot by slot.
template <int NK>
__device__ __forceinline__ void job_tiles(const PagedAttendArgs& a, Job& job, int rows_of_wg, int split) {
  const int tok_lo = job.row0 / a.G;
  const int tok_hi = (min(job.row0 + rows_of_wg, job.rows) - 1) / a.G;
  const int end = min(job.base + tok_hi + 1, a.map.cap);
  const int tiles = (end + NK - 1) / NK;
  job.sink_tiles = 0;
  job.tile0 = 0;
  if (a.window > 0) {
    const long long begin = (long long)job.base + tok_lo - a.window + 1;
    job.tile0 = begin > 0 ? (int)(begin / NK) : 0;
    job.sink_tiles = min((min(a.n_sink, end) + NK - 1) / NK, job.tile0);
  }
  const int n = job.sink_tiles + tiles - job.tile0;
  job.split = split;
  job.t_begin = (int)((long long)n * split / a.ns);
  job.t_end = (int)((long long)n * (split + 1) / a.ns);
}

// Grid: (Hkv, ns, many_tiles + B), flattened with the KV head fastest: the workgroups of one head of one
// sequence are Hkv apart, so with 8 heads (the XCDs are dealt workgroups in turn) they share an L2. The
// tiles of many rows come first, the last of a sequence (the longest) before the others.
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_attend(PagedAttendArgs a) {
  __shared__ __align__(16) char lds[paged_lds<T, D>()];
  const int per = a.Hkv * a.ns;
  const int unit = blockIdx.x / per, rest = blockIdx.x % per;
  Job job;
  job.h = rest % a.Hkv;
  const int split = rest / a.Hkv;
  const int lane = threadIdx.x & 63;
  if (unit < a.many_tiles) {
    // the sequence of this tile: tiles of sequences with more than 32 rows, counted 64 sequences at a time
    int left = unit, b = -1, tiles = 0;
    for (int b0 = 0; b0 < a.map.B; b0 += 64) {
      int n = 0;
      if (b0 + lane < a.map.B) {
        const Chunk c = chunk_of(a.q_start, b0 + lane, a.total);
        if (c.n <= a.max_chunk && (long long)c.n * a.G > kWaveRows) n = (int)(((long long)c.n * a.G + kManyRows - 1) / kManyRows);
      }
      int inc = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(inc, o, 64);
        if (lane >= o) inc += y;
      }
      const unsigned long long over = __ballot(inc > left);
      if (over != 0) {
        const int k = __builtin_ctzll(over);
        tiles = __builtin_amdgcn_readlane(n, k);
        left -= __builtin_amdgcn_readlane(inc, k) - tiles;
        b = b0 + k;
        break;
      }
      left -= __builtin_amdgcn_readlane(inc, 63);
    }
    if (b < 0) return;
    const Chunk c = chunk_of(a.q_start, b, a.total);
    job.b = b;
    job.first = c.first;
    job.rows = c.n * a.G;
    job.row0 = (tiles - 1 - left) * kManyRows;
    job.base = a.base[b];
    if (job.base < 0 || job.base > a.map.cap - c.n) return;
    job_tiles<Team<T, D, 1>::kKeys>(a, job, kManyRows, split);
    paged_body<T, D, 1>(a, job, lds);
    return;
  }
  const int b = unit - a.many_tiles;
  const Chunk c = chunk_of(a.q_start, b, a.total);
  job.base = a.base[b];
  if (c.n == 0) return;
  if (job.base < 0 || c.n > a.max_chunk || job.base > a.map.cap - c.n) {  // refused
    if (a.conf != nullptr && rest == 0 && threadIdx.x == 0) a.conf[b] = NAN;
    return;
  }
  if ((long long)c.n * a.G > kWaveRows) return;
  job.b = b;
  job.first = c.first;
  job.rows = c.n * a.G;
  job.row0 = 0;
  job_tiles<Team<T, D, 4>::kKeys>(a, job, kWaveRows, split);
  paged_body<T, D, 4>(a, job, lds);
}

// Joins the splits of a row: a wave per query row of a token.
constexpr int kJoinRows = kPagedThreads / 64;

template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_join(PagedAttendArgs a) {
  const long long row = (long long)blockIdx.x * kJoinRows + (threadIdx.x >> 6);
  const long long rows = (long long)a.total * a.Hq;
  if (row >= rows) return;
  const int r = (int)(row / a.Hq), lane = threadIdx.x & 63;
  const int b = seq_of_row(a.q_start, a.map.B, r);
  if (b >= a.map.B) return;
  const Chunk c = chunk_of(a.q_start, b, a.total);
  const int base = a.base[b];
  if (r < c.first || r >= c.first + c.n || c.n > a.max_chunk || base < 0 || base > a.map.cap - c.n) return;
  float M = -INFINITY;
  for (int s = 0; s < a.ns; ++s) M = fmaxf(M, a.pml[(s * rows + row) * 4]);
  const float Ms = M == -INFINITY ? 0.f : M;
  float L = 0.f, SF = 0.f, x[D / 64] = {};
  for (int s = 0; s < a.ns; ++s) {
    const f32x4 st = *(const f32x4*)(a.pml + (s * rows + row) * 4);
    const float f = __builtin_amdgcn_exp2f(st[0] - Ms);
    L += f * st[1];
    SF += f * st[2];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) x[e] += f * a.po[(s * rows + row) * D + lane * (D / 64) + e];
  }
  const float inv = 1.f / L;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) ((T*)a.out)[row * D + lane * (D / 64) + e] = (T)(L == 0.f ? 0.f : x[e] * inv);
  if (lane == 0) {
    a.lse[row] = L == 0.f ? -INFINITY : kLn2 * (M + __builtin_amdgcn_logf(L));
    const float mass = L == 0.f ? 0.f : SF * inv;
    if (a.suffix != nullptr) a.suffix[row] = mass;
    if (a.conf != nullptr && r == c.first + c.n - 1) raise_conf(a.conf + b, mass);
  }
}

// ------------------------------------------------------------------------------------------
// Plan and launch
// ------------------------------------------------------------------------------------------
struct PagedPlan {
  long many_tiles;  // upper bound over the chunks that `total` rows can be
  int ns;
};

static PagedPlan paged_plan(const lg_paged_layer& l, const lg_page_map& m, long total, long max_chunk) {
  const long G = l.n_q_heads / l.n_kv_heads;
  PagedPlan p;
  p.many_tiles = 0;
  if (max_chunk * G > kWaveRows && total * G > kWaveRows) {
    // a sequence of n rows has at most n / 128 + 1 tiles, and more than 32 rows
    p.many_tiles = total * G / kManyRows;
    const long seqs = total * G / (kWaveRows + 1);
    p.many_tiles += seqs < m.batch ? seqs : m.batch;
  }
  const long units = (p.many_tiles + m.batch) * l.n_kv_heads;
  const long cap = (long)m.max_pages * m.page_size;
  long ns = (kPagedTarget + units - 1) / units;
  const long most = (cap + kMinSplitSlots - 1) / kMinSplitSlots;
  if (ns > most) ns = most;
  p.ns = (int)(ns < 1 ? 1 : ns);
  return p;
}

static size_t paged_need(const lg_paged_layer& l, const PagedPlan& p, long total) {
  return p.ns > 1 ? (size_t)p.ns * total * l.n_q_heads * (l.head_dim + 4) * 4 : 0;
}

// Workgroups of the launch (a grid holds fewer than 2^32 threads).
long paged_attend_grid(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk) {
  const PagedPlan p = paged_plan(l, m, total, max_chunk);
  return (p.many_tiles + m.batch) * l.n_kv_heads * p.ns;
}

size_t paged_attend_need(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk) {
  return paged_need(l, paged_plan(l, m, total, max_chunk), total);
}

// The largest need of any total up to this one and any max_chunk up to this one: for a given number of
// splits the need grows with total, and the number falls as total grows, so the ends of its steps count.
size_t paged_attend_bytes(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk) {
  size_t most = 16;
  for (int form = 0; form < 2; ++form) {
    const long chunk = form == 0 ? 1 : max_chunk;
    long t = total;
    while (t > 0) {
      const PagedPlan p = paged_plan(l, m, t, chunk);
      const size_t need = paged_need(l, p, t);
      if (need > most) most = need;
      long lo = 0, hi = t;  // the largest smaller total with more splits
      while (hi - lo > 1) {
        const long mid = (lo + hi) / 2;
        if (paged_plan(l, m, mid, chunk).ns > p.ns) lo = mid; else hi = mid;
      }
      t = lo;
    }
  }
  return align_up(most, 16);
}

hipError_t launch_paged_attend(const lg_paged_layer& l, const lg_page_map& m, const void* q, void* out,
                               const int32_t* q_start, const int32_t* base, int total, int max_chunk,
                               int window, int n_sink, const int32_t* suffix_w, float* lse, float* suffix,
                               float* conf, void* ws, hipStream_t st) {
  const PagedPlan p = paged_plan(l, m, total, max_chunk);
  PagedAttendArgs a = {};
  a.q = q;
  a.k = l.k;
  a.v = l.v;
  a.out = out;
  a.q_start = q_start;
  a.base = base;
  a.suffix_w = suffix_w;
  a.lse = lse;
  a.suffix = suffix;
  a.conf = conf;
  a.po = (float*)ws;
  a.pml = (float*)ws + (size_t)p.ns * total * l.n_q_heads * l.head_dim;
  a.map = map_args(m);
  a.Hq = l.n_q_heads;
  a.Hkv = l.n_kv_heads;
  a.G = l.n_q_heads / l.n_kv_heads;
  a.total = total;
  a.max_chunk = max_chunk;
  a.window = window;
  a.n_sink = n_sink;
  a.ns = p.ns;
  a.many_tiles = (int)p.many_tiles;
  a.scale_log2 = kLog2e / sqrtf((float)l.head_dim);
  const dim3 grid((unsigned)((p.many_tiles + m.batch) * l.n_kv_heads * p.ns));
  const dim3 join((unsigned)(((long)total * l.n_q_heads + kJoinRows - 1) / kJoinRows));
  auto go = [&](auto kernel, auto joined) {
    hipLaunchKernelGGL(kernel, grid, dim3(kPagedThreads), 0, st, a);
    if (p.ns > 1) hipLaunchKernelGGL(joined, join, dim3(kPagedThreads), 0, st, a);
  };
  if (l.dtype == LG_BF16) {
    if (l.head_dim == 128) go(paged_attend<__bf16, 128>, paged_join<__bf16, 128>);
    else go(paged_attend<__bf16, 64>, paged_join<__bf16, 64>);
  } else {
    if (l.head_dim == 128) go(paged_attend<float, 128>, paged_join<float, 128>);
    else go(paged_attend<float, 64>, paged_join<float, 64>);
  }
  return hipGetLastError();
}

}  // namespace lg
