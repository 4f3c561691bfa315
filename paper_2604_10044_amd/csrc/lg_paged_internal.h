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

}  // namespace lg
