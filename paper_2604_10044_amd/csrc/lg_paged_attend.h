// lg_paged_attend.h -- what the attention kernels over pages share (lg_paged_attend.hip, lg_fp4_attend.hip): their
// arguments, the rows and slots of a workgroup, the statistics of a row.
#pragma once

#include <algorithm>
#include <type_traits>

#include "lg_paged_internal.h"

namespace lg {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));


constexpr int kWaveRows = 32;
constexpr int kManyRows = 128;   // rows of a KW = 1 workgroup
constexpr int kPagedThreads = 256;
constexpr float kSlack = 8.f;  // see paged_body
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

// The value of lane ^ 16 (rows of 16 lanes change places in pairs).
__device__ __forceinline__ float other_row(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 16) != 0 ? r[0] : r[1]);
}

// The value of lane ^ 32.
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) != 0 ? r[0] : r[1]);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // to nearest, ties to even
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// Two values that are not negative as bfloat16, each the largest below it, and what is left, rounded: the sum of
// both is within 2^-16 of the value, and neither is 0 unless the value is (0 x inf would be NaN).
struct TwoTerms {
  uint32_t most, rest;
};
__device__ __forceinline__ TwoTerms split_bf16(float a, float b) {
  const uint32_t x = bf16_below(a), y = bf16_below(b);
  return {x >> 16 | y, pack_bf16(a - __uint_as_float(x), b - __uint_as_float(y))};
}

// conf[b] = max(conf[b], mass): masses are not negative, so their order is that of their bits; a NaN (of
// whatever sign) makes it NaN.
__device__ __forceinline__ int conf_bits(float mass) { return mass != mass ? 0x7fc00000 : __float_as_int(mass); }

// For the lanes of a wave that are `mine`, of one sequence. The confidences of a batch lie in a few cache lines, where
// atomics wait for each other: with one a row a decode step of 16 x 48 heads of 64 took 20.6 us, with one a wave, or a
// workgroup and token in paged_join, 12.0.
__device__ __forceinline__ void raise_conf(float* conf, float mass, bool mine) {
  if (__ballot(mine) == 0) return;
  int x = mine ? conf_bits(mass) : 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = max(x, __shfl_xor(x, o, 64));
  if ((threadIdx.x & 63) == 0) atomicMax((int*)conf, x);
}

template <int N>
using Num = std::integral_constant<int, N>;

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
  int end;  // slots that any of its rows may see lie below
  int d0;  // first of the DV values of V
};

// This split's share of a workgroup's tiles: those for the first tokens, and those from tile0 to the last.
__device__ __forceinline__ void share_tiles(const PagedAttendArgs& a, Job& job, int nk, int end, int tile0) {
  job.tile0 = tile0;
  job.sink_tiles = a.window > 0 ? min((min(a.n_sink, end) + nk - 1) / nk, tile0) : 0;
  const int n = job.sink_tiles + (end + nk - 1) / nk - tile0;
  // n <= 2^25 + 2 tiles, at most 64 splits: below 2^32
  job.t_begin = (int)((unsigned)n * (unsigned)job.split / (unsigned)a.ns);
  job.t_end = (int)((unsigned)n * (unsigned)(job.split + 1) / (unsigned)a.ns);
}

// The slots that the workgroup's rows may see, in tiles. A window's first slot is at least (slot - window + 1):
// positions ascend by at least one a slot; slots below n_sink likewise hold the positions below n_sink.
// Where the guard has pruned, the window holds fewer slots: skip_hidden.
template <int NK>
__device__ __forceinline__ void job_tiles(const PagedAttendArgs& a, Job& job, int rows_of_wg, int split) {
  const int tok_lo = job.row0 / a.G;
  const int tok_hi = (min(job.row0 + rows_of_wg, job.rows) - 1) / a.G;
  const long long begin = a.window > 0 ? (long long)job.base + tok_lo - a.window + 1 : 0;
  job.split = split;
  job.end = min(job.base + tok_hi + 1, a.map.cap);
  share_tiles(a, job, NK, job.end, begin > 0 ? (int)(begin / NK) : 0);
}

// Tiles behind the first tokens' that no row sees, by the window of the workgroup's first one: the first tile whose last
// slot it sees, found by search, 64 probes a round. True if the share has changed. Without holes one read that the
// first tile's lookup overlaps (no difference for the mixed step above). 32 sequences of 8192 slots
// that decode with a window of 4096 over a history thinned out four to one: 58 us, 100 without.
template <int NK>
__device__ __forceinline__ bool skip_hidden(const PagedAttendArgs& a, Job& job, const int32_t* pos) {
  // No window, or one of at least as many positions as the cache holds slots: nothing is looked for, and slots that
  // holes in the positions put out of such a window are compared and masked.
  if (job.tile0 == 0) return false;
  const int slot = job.base + job.row0 / a.G, lane = threadIdx.x & 63;
  const int w = (int)max((long long)pos[slot] - a.window, (long long)INT32_MIN);
  int lo = job.tile0, hi = slot / NK;  // the tile of the token's own slot is seen
  if (lo >= hi || pos[lo * NK + NK - 1] > w) return false;
  while (lo < hi) {
    const int step = (hi - lo + 63) >> 6;
    const long long first = (long long)lo + (long long)lane * step;
    const int at = (int)min(first + step - 1, (long long)hi - 1);
    const int cnt = __popcll(__ballot(first < hi && pos[at * NK + NK - 1] <= w));
    lo = (int)min((long long)lo + (long long)cnt * step, (long long)hi);
    hi = step == 1 ? lo : (int)min((long long)lo + step - 1, (long long)hi);
  }
  share_tiles(a, job, NK, job.end, lo);
  return true;
}

// A sequence of at most 32 query rows: false if it has none, more, or is refused.
__device__ __forceinline__ bool few_job(const PagedAttendArgs& a, Job& job, int b, bool first) {
  const Chunk c = chunk_of(a.q_start, b, a.total);
  job.base = a.base[b];
  if (c.n == 0) return false;
  if (job.base < 0 || c.n > a.max_chunk || job.base > a.map.cap - c.n) {  // refused
    if (a.conf != nullptr && first && threadIdx.x == 0) a.conf[b] = NAN;
    return false;
  }
  if ((long long)c.n * a.G > kWaveRows) return false;
  job.b = b;
  job.first = c.first;
  job.rows = c.n * a.G;
  job.row0 = 0;
  return true;
}

// The 128 rows of tile `unit` of a launch's sequences with more than 32 rows: false if there is none or its sequence is
// refused.
__device__ __forceinline__ bool many_job(const PagedAttendArgs& a, Job& job, int unit) {
  const int lane = threadIdx.x & 63;
  // the sequence of this tile: tiles of sequences with more than 32 rows, counted 64 sequences at a time
  int left = unit, tiles = 0, k = 0, b0 = 0, base = -1;
  Chunk c = {0, 0};
  for (;; b0 += 64) {
    if (b0 >= a.map.B) return false;
    int n = 0;
    if (b0 + lane < a.map.B) {
      c = chunk_of(a.q_start, b0 + lane, a.total);
      base = a.base[b0 + lane];
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
      k = __builtin_ctzll(over);
      tiles = __builtin_amdgcn_readlane(n, k);
      left -= __builtin_amdgcn_readlane(inc, k) - tiles;
      break;
    }
    left -= __builtin_amdgcn_readlane(inc, 63);
  }
  const int n = __builtin_amdgcn_readlane(c.n, k);
  job.b = b0 + k;
  job.first = __builtin_amdgcn_readlane(c.first, k);
  job.rows = n * a.G;
  job.row0 = (tiles - 1 - left) * kManyRows;
  job.base = __builtin_amdgcn_readlane(base, k);
  return job.base >= 0 && job.base <= a.map.cap - n;
}

inline long whole_reach(const lg_page_map& m) { return (long)m.max_pages * m.page_size; }
inline long window_reach(const lg_page_map& m, long max_chunk, long window, long n_sink) {
  return window > 0 ? std::min(whole_reach(m), window + n_sink + max_chunk) : whole_reach(m);
}

}  // namespace lg
