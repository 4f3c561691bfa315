// lg_paged_internal.h -- what the kernels of the paged cache share: the map as device arguments, and
// the sequence that a row of a step's token arrays belongs to.
#pragma once

#include "lg_internal.h"
#include "lg_paged.h"

namespace lg {

constexpr int kMaxLayersPaged = 64;  // layers of one launch

struct MapArgs {
  int32_t *table, *pos, *len, *ref;
  int32_t B, P, n_pages, shift;  // page_size = 1 << shift
  int32_t cap;                   // P << shift
};

inline MapArgs map_args(const lg_page_map& m) {
  MapArgs a;
  a.table = m.table;
  a.pos = m.pos;
  a.len = m.len;
  a.ref = m.ref;
  a.B = m.batch;
  a.P = m.max_pages;
  a.n_pages = m.n_pages;
  a.shift = __builtin_ctz((unsigned)m.page_size);
  a.cap = m.max_pages << a.shift;
  return a;
}

__device__ __forceinline__ bool is_page(const MapArgs& m, int p) { return (unsigned)p < (unsigned)m.n_pages; }

// New tokens of sequence b: its rows of the step's token arrays, [first, first + n). Values that do
// not ascend or pass `total` give n = 0 or end at total.
struct Chunk {
  int first, n;
};
__device__ __forceinline__ Chunk chunk_of(const int32_t* q_start, int b, int total) {
  const int first = min(max(q_start[b], 0), total);
  const int end = min(max(q_start[b + 1], 0), total);
  return {first, max(end - first, 0)};
}

// The sequence of row r, found by a wave (r the same in its lanes): the entries of q_start[1 .. B]
// that are at most r, counted 64 at a time. B when the row lies behind the last sequence.
__device__ __forceinline__ int seq_of_row(const int32_t* q_start, int B, int r) {
  const int lane = threadIdx.x & 63;
  int b = 0;
  for (int i0 = 1; i0 <= B; i0 += 64) {
    const bool below = i0 + lane <= B && q_start[i0 + lane] <= r;
    const int c = __popcll(__ballot(below));
    b += c;
    if (c < 64) break;
  }
  return b;
}

// The sequence of a row at or behind those of sequence b, each lane for itself: steps that double, then halves, since
// thousands of sequences without rows may lie between.
__device__ __forceinline__ int seq_behind(const int32_t* q_start, int B, int b, int r) {
  int lo = b, step = 1;  // the answer is lo or more
  while (lo < B && q_start[min(lo + step, B)] <= r) {
    lo = min(lo + step, B);
    step *= 2;
  }
  for (int hi = min(lo + step - 1, B); lo < hi;) {
    const int mid = (lo + hi) >> 1;
    if (q_start[mid + 1] <= r) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// 4-bit layers (lg_fp4.h): bytes of a row's values, of its exponents, and of the block of a page and a head.
constexpr int kFp4Group = 32;  // values of one exponent
__host__ __device__ __forceinline__ constexpr int fp4_row(int D) { return D / 2; }
__host__ __device__ __forceinline__ constexpr int fp4_exps(int D) { return D / kFp4Group; }
__host__ __device__ __forceinline__ size_t fp4_block(int D, int shift) { return (size_t)(fp4_row(D) + fp4_exps(D)) << shift; }

// The unit 2^(x - 127) of an exponent byte as the conversion instructions take it: NaN above 252.
__device__ __forceinline__ float fp4_unit(uint32_t x) { return __uint_as_float((x > 252 ? 255u : x) << 23); }

}  // namespace lg
