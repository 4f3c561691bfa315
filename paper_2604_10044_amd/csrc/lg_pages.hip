// lg_pages.hip -- the map of a paged cache: reserving, forking, compacting and freeing pages
// (lg_page_reserve, lg_page_fork, lg_page_compact).
//
// What a sequence needs depends on the lengths, reference counts and free pages of the moment, all on
// the device, so one workgroup decides for the whole batch: needs (a thread or wave per sequence), their
// prefix sums, then the lowest free pages in order of their number. A free page is a zero in ref, found
// by a scan that ends as soon as the needs are covered and is left out when nothing is needed. Every
// decision reads ref as it was before the call and every change is an integer sum, so results do not
// depend on the order in which waves run. A second launch moves rows.
#include "lg_keepset.h"
#include "lg_paged_internal.h"

namespace lg {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kMapThreads = 1024;
constexpr int kMapWaves = kMapThreads / 64;

// Workspace of the lg_page_* calls, in int32 words: per-sequence fields first.
struct PageWs {
  int32_t* count;   // [16]; [0]: sequences in `list`
  int32_t* need;    // [B] pages
  int32_t* before;  // [B] pages that the sequences before need
  int32_t* first;   // [B] compact: first column that changes; reserve: rows to copy
  int32_t* list;    // [B] sequences whose rows a second launch moves
  int32_t* src;     // [B] reserve: the page copied from; fork: len
  int32_t* dst;     // [B] reserve: the page copied to
  int32_t* table;   // [B][P] fork, compact: columns before the call
  int32_t* fresh;   // [B][P] reserve, compact: free pages in ascending order; fork: [B][cap] pos
};

static size_t ws_words(const lg_page_map& m) {
  const size_t B = m.batch, P = m.max_pages;
  return 16 + 6 * B + B * P + B * P * (size_t)m.page_size;
}
size_t page_workspace_bytes(const lg_page_map& m) { return align_up(4 * ws_words(m), 16); }

static PageWs page_ws(const lg_page_map& m, void* ws) {
  const size_t B = m.batch, P = m.max_pages;
  PageWs w;
  w.count = (int32_t*)ws;
  w.need = w.count + 16;
  w.before = w.need + B;
  w.first = w.before + B;
  w.list = w.first + B;
  w.src = w.list + B;
  w.dst = w.src + B;
  w.table = w.dst + B;
  w.fresh = w.table + B * P;
  return w;
}

// Prefix sums of need[] into before[], the lowest free pages into fresh[]; returns how many were
// found (at least the sum of the needs, or all there are). Ends with a barrier.
__device__ __forceinline__ long long find_pages(const MapArgs& m, const PageWs& w, int* red) {
  const int tid = threadIdx.x;
  long long want = 0;  // batch * max_pages < 2^31
  for (int b0 = 0; b0 < m.B; b0 += kMapThreads) {
    const int b = b0 + tid;
    int total;
    const int ex = block_exclusive_scan<kMapThreads>(b < m.B ? w.need[b] : 0, &total, red);
    if (b < m.B) w.before[b] = (int)(want + ex);
    want += total;
    __syncthreads();
  }
  long long found = 0;
  // Four pages a thread, 4096 a round, in page order across the workgroup. The rounds follow each other, and the lowest
  // pages are taken first, so a running pool is searched past what it holds: 32 new pages behind 0 / 16000 / 64000 /
  // 100000 / 400000 held ones make lg_page_reserve 5.8 / 10 / 23 / 33 / 113 us, 1.1 us a round.
  for (long long p0 = 0; found < want && p0 < m.n_pages; p0 += kMapThreads * 4) {
    const int p = (int)p0 + tid * 4;
    int free4 = 0;
    if (p + 3 < m.n_pages) {
      const u32x4_t r = *(const u32x4_t*)(m.ref + p);
      free4 = (r[0] == 0) | (r[1] == 0) << 1 | (r[2] == 0) << 2 | (r[3] == 0) << 3;
    } else {
      for (int i = 0; i < 4; ++i)
        if (p + i < m.n_pages && m.ref[p + i] == 0) free4 |= 1 << i;
    }
    int total;
    long long at = found + block_exclusive_scan<kMapThreads>(__popc(free4), &total, red);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free4 >> i & 1) {
        if (at < want) w.fresh[at] = p + i;
        ++at;
      }
    found += total;
    __syncthreads();
  }
  __syncthreads();
  return found;
}

__device__ __forceinline__ bool granted(const PageWs& w, int b, long long found) {
  return w.need[b] == 0 || (long long)w.before[b] + w.need[b] <= found;
}

// ------------------------------------------------------------------------------------------
// Reserve
// ------------------------------------------------------------------------------------------
struct ReserveArgs {
  MapArgs map;
  PageWs ws;
  const int32_t *q_start, *t;
  int32_t* base;
};

// Pages a sequence needs = ceil((len + n) / ps) - ceil(len / ps), and one more where its last page holds live
// slots that others share. A few integers a sequence: the chain of dependent reads (len, table, ref, then the
// scan of ref, then table) bounds it, not their bytes, so everything is one launch of one workgroup. Measured:
// 5.8 us for 32 sequences of one token and one round of the search (see find_pages for larger pools).
__global__ __launch_bounds__(kMapThreads) void reserve_map(ReserveArgs a) {
  __shared__ int red[kMapWaves];
  __shared__ int copies;
  const MapArgs& m = a.map;
  const PageWs& w = a.ws;
  const int tid = threadIdx.x, lane = tid & 63, ps = 1 << m.shift;
  if (tid == 0) copies = 0;
  for (int b = tid; b < m.B; b += kMapThreads) {
    const int old = min(max(m.len[b], 0), m.cap);
    const long long n = max((long long)a.q_start[b + 1] - a.q_start[b], 0ll);
    int need = 0, rows = 0, page = -1;
    bool able = n <= m.cap - old;
    if (able && n > 0) {
      const int col = old >> m.shift;
      if (old & (ps - 1)) {
        page = m.table[(size_t)b * m.P + col];
        if (!is_page(m, page))
          able = false;
        else if (m.ref[page] > 1)
          rows = old & (ps - 1);
      }
      need = ((old + (int)n + ps - 1) >> m.shift) - ((old + ps - 1) >> m.shift) + (rows > 0);
    }
    w.need[b] = able ? need : 0;
    w.first[b] = rows;
    w.src[b] = able ? page : -2;  // -2: refused whatever is free
  }
  __syncthreads();
  const long long found = find_pages(m, w, red);
  for (int b = tid >> 6; b < m.B; b += kMapWaves) {  // a wave per sequence
    const int old = min(max(m.len[b], 0), m.cap);
    const bool ok = w.src[b] != -2 && granted(w, b, found);
    if (!ok) {
      if (lane == 0) a.base[b] = -1;
      continue;
    }
    const int n = max(a.q_start[b + 1] - a.q_start[b], 0);
    const int need = w.need[b], rows = w.first[b];
    const int32_t* fresh = w.fresh + w.before[b];
    int32_t* table = m.table + (size_t)b * m.P;
    const int col0 = rows > 0 ? old >> m.shift : (old + ps - 1) >> m.shift;
    for (int i = lane; i < need; i += 64) {
      const int p = fresh[i];
      table[col0 + i] = p;
      m.ref[p] = 1;
    }
    int32_t* pos = m.pos + (size_t)b * m.cap;
    const int p0 = (int)((unsigned)a.t[b] - (unsigned)n + 1u);
    for (int i = lane; i < n; i += 64) pos[old + i] = (int)((unsigned)p0 + (unsigned)i);
    if (lane == 0) {
      a.base[b] = old;
      m.len[b] = old + n;
      if (rows > 0) {
        atomicSub(m.ref + w.src[b], 1);
        w.dst[b] = fresh[0];
        w.list[atomicAdd(&copies, 1)] = b;  // in any order: the copies do not meet
      }
    }
  }
  __syncthreads();
  if (tid == 0) w.count[0] = copies;
}

struct LayerPtrs {
  void* k[kMaxLayersPaged];
  void* v[kMaxLayersPaged];
};

struct CopyArgs {
  LayerPtrs layer;
  PageWs ws;
  int32_t n_layers, Hkv, shift, row_bytes;
};

constexpr int kCopyThreads = 256;
constexpr int kCopyWorkgroups = 1024;

// The live rows of replaced last pages: an item is one layer's K or V of one head, contiguous rows, at most
// page_size * row_bytes = 128 KB, that one workgroup copies in 16-byte pieces. How many there are is known on
// the device only, so the grid is fixed and walks the items. Measured: 2.0 us with nothing to copy, 7.4 us for
// eight forks of one prompt over 32 layers.
__global__ __launch_bounds__(kCopyThreads) void copy_rows(CopyArgs a) {
  const int copies = a.ws.count[0];
  const int per = 2 * a.n_layers * a.Hkv;
  const long long items = (long long)copies * per;
  const size_t head = (size_t)a.row_bytes << a.shift;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int b = a.ws.list[it / per], x = (int)(it % per);
    const int h = x % a.Hkv, l = x / a.Hkv % a.n_layers;
    char* pages = (char*)(x < a.n_layers * a.Hkv ? a.layer.k[l] : a.layer.v[l]);
    const u32x4_t* src = (const u32x4_t*)(pages + ((size_t)a.ws.src[b] * a.Hkv + h) * head);
    u32x4_t* dst = (u32x4_t*)(pages + ((size_t)a.ws.dst[b] * a.Hkv + h) * head);
    const int n = a.ws.first[b] * (a.row_bytes / 16);
    for (int i = threadIdx.x; i < n; i += kCopyThreads) dst[i] = src[i];
  }
}

// ------------------------------------------------------------------------------------------
// Fork
// ------------------------------------------------------------------------------------------
struct ForkArgs {
  MapArgs map;
  PageWs ws;
  const int32_t* parent;
};

constexpr int kForkThreads = 256;
constexpr int kForkSlots = 1024;  // of capacity for a workgroup ...
constexpr int kForkSpread = 64;   // ... up to this many a sequence
// One workgroup takes both steps of small maps: up to kForkSmallBatch sequences, of which it works on four at once, each
// round a chain of dependent reads, and kForkSmall slots of capacity in all. Sequences x slots in a graph / a call, in two
// launches behind the stroke (a call's second launch costs the host 4 us):
//   4 x 256 3.5 / 4.7 us | 5.4 / 7.2    8 x 512 5.3 / 5.0 | 5.5 / 7.0    8 x 1024 6.9 / 6.5 | 6.3 / 7.1
//   8 x 2048 9.2 / 8.9 | 6.2 / 7.3      16 x 256 8.8 / 8.4 | 5.5 / 7.1   32 x 256 15.4 / 15.1 | 5.7 / 7.0
//   64 x 128 32.6 / 32.4 | 5.6 / 7.0    512 x 16 281 / 280 | 5.8 / 7.3
constexpr int kForkSmallBatch = 8;
constexpr long kForkSmall = 8192;

__device__ __forceinline__ bool fork_changes(const ForkArgs& a, int b, int* parent) {
  const int p = a.parent[b];
  *parent = p;
  return p != b && p >= -1 && p < a.map.B;
}

// First step: what each changed sequence becomes goes to the workspace (its parent may change too), and the
// pages it will share are counted. Second step: the references it held are given back, and it becomes what the
// workspace holds. A page is never seen at zero in between. A thread of the second step reads only what the
// first one wrote and the one entry that it replaces itself, so a sequence's row can be split freely.
// t: one of the `step` threads that work on b.
__device__ __forceinline__ void fork_read_one(const ForkArgs& a, int b, int t, int step) {
  const MapArgs& m = a.map;
  int p;
  if (!fork_changes(a, b, &p) || p < 0) return;
  const int n = min(max(m.len[p], 0), m.cap);
  for (int c = t; c < m.P; c += step) {
    const int page = m.table[(size_t)p * m.P + c];
    a.ws.table[(size_t)b * m.P + c] = page;
    if (is_page(m, page)) atomicAdd(m.ref + page, 1);
  }
  for (int j = t; j < n; j += step) a.ws.fresh[(size_t)b * m.cap + j] = m.pos[(size_t)p * m.cap + j];
  if (t == 0) a.ws.src[b] = n;
}

__device__ __forceinline__ void fork_write_one(const ForkArgs& a, int b, int t, int step) {
  const MapArgs& m = a.map;
  int p;
  if (!fork_changes(a, b, &p)) return;
  const int n = p < 0 ? 0 : a.ws.src[b];
  for (int c = t; c < m.P; c += step) {
    const size_t at = (size_t)b * m.P + c;
    const int page = m.table[at];
    if (is_page(m, page)) atomicSub(m.ref + page, 1);
    m.table[at] = p < 0 ? -1 : a.ws.table[at];
  }
  for (int j = t; j < n; j += step) m.pos[(size_t)b * m.cap + j] = a.ws.fresh[(size_t)b * m.cap + j];
  if (t == 0) m.len[b] = n;
}

// A launch a step; a workgroup takes kForkSlots slots of a sequence's capacity. The bytes (a few hundred KB) are
// nothing; what bounds it is two launches and one dependent read each. Measured in a graph, both launches: 6.4 us
// for 8 x 1024 slots, 6.5 for 32 x 2048, 7.1 for 4 x 16384; with one workgroup a sequence 6.4, 8.0 and 29.6.
__global__ __launch_bounds__(kForkThreads) void fork_read(ForkArgs a) {
  fork_read_one(a, blockIdx.x, blockIdx.y * kForkThreads + threadIdx.x, gridDim.y * kForkThreads);
}
__global__ __launch_bounds__(kForkThreads) void fork_write(ForkArgs a) {
  fork_write_one(a, blockIdx.x, blockIdx.y * kForkThreads + threadIdx.x, gridDim.y * kForkThreads);
}

// Both steps of a small map in one workgroup and launch.
__global__ __launch_bounds__(kMapThreads) void fork_small(ForkArgs a) {
  const int t = threadIdx.x % kForkThreads, step = kMapThreads / kForkThreads;
  for (int b = threadIdx.x / kForkThreads; b < a.map.B; b += step) fork_read_one(a, b, t, kForkThreads);
  __syncthreads();
  for (int b = threadIdx.x / kForkThreads; b < a.map.B; b += step) fork_write_one(a, b, t, kForkThreads);
}

// ------------------------------------------------------------------------------------------
// Compact
// ------------------------------------------------------------------------------------------
struct CompactMapArgs {
  MapArgs map;
  PageWs ws;
  const int32_t *keep_idx, *new_len;
  int32_t* moved;
};

constexpr int kSharedMark = 1 << 29;  // beside a page number (< 2^28) in the workspace's columns

// Leading rows with keep[r] == r, of n: keep[r] - r does not fall, so one wave finds the end by search,
// 64 probes a round (see wave_lower_bound).
__device__ __forceinline__ int rows_in_place(const int32_t* keep, int n) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo + 63) >> 6;
    const long long first = (long long)lo + (long long)lane * step;
    const int at = (int)min(first + step - 1, (long long)hi - 1);
    const bool still = first < hi && keep[at] <= at;
    const int cnt = __popcll(__ballot(still));
    const int seg = (int)min((long long)lo + (long long)cnt * step, (long long)hi);
    hi = step == 1 ? seg : (int)min((long long)seg + step, (long long)hi);
    lo = seg;
    if (step == 1) break;
  }
  return lo;
}

// Which columns change (from the first row that moves), which of those are shared and need a page, and the
// references given back. Like reserve_map a chain of dependent reads: 5.2 us for one flagged sequence of
// 32, 13.3 us for eight long ones that share their pages.
__global__ __launch_bounds__(kMapThreads) void compact_map(CompactMapArgs a) {
  __shared__ int red[kMapWaves];
  __shared__ int moves;
  const MapArgs& m = a.map;
  const PageWs& w = a.ws;
  const int tid = threadIdx.x, lane = tid & 63, ps = 1 << m.shift;
  if (tid == 0) moves = 0;
  // Nothing flagged, the usual step: one look at new_len.
  int mine = 0;
  for (int b = tid; b < m.B; b += kMapThreads) {
    const bool f = a.new_len[b] >= 0;
    mine |= f;
    if (!f) a.moved[b] = 0;
    w.need[b] = 0;
  }
  if (!__syncthreads_or(mine)) {
    if (tid == 0) w.count[0] = 0;
    return;
  }
  for (int b = tid >> 6; b < m.B; b += kMapWaves) {
    const int nl = min(a.new_len[b], m.cap);
    if (nl < 0) continue;
    const int still = rows_in_place(a.keep_idx + (size_t)b * m.cap, nl);
    const int cols = (nl + ps - 1) >> m.shift;
    const int first = still < nl ? still >> m.shift : cols;
    int need = 0;
    for (int c0 = first; c0 < m.P; c0 += 64) {
      const int c = c0 + lane;
      int page = c < m.P ? m.table[(size_t)b * m.P + c] : -1;
      if (!is_page(m, page)) page = -1;
      const bool shared = c < cols && page >= 0 && m.ref[page] > 1;
      if (c < m.P) w.table[(size_t)b * m.P + c] = shared ? page | kSharedMark : page;
      need += __popcll(__ballot(shared));
    }
    if (lane == 0) {
      w.need[b] = need;
      w.first[b] = first;
    }
  }
  __syncthreads();
  const long long found = find_pages(m, w, red);
  for (int b = tid >> 6; b < m.B; b += kMapWaves) {
    const int nl = min(a.new_len[b], m.cap);
    if (nl < 0) continue;
    const bool ok = granted(w, b, found);
    if (lane == 0) a.moved[b] = ok ? 1 : -1;
    if (!ok) continue;
    const int cols = (nl + ps - 1) >> m.shift, first = w.first[b];
    const int32_t* fresh = w.fresh + w.before[b];
    for (int c0 = first; c0 < m.P; c0 += 64) {
      const int c = c0 + lane;
      const int old = c < m.P ? w.table[(size_t)b * m.P + c] : -1;
      const bool shared = old >= 0 && (old & kSharedMark);
      const unsigned long long mask = __ballot(shared);
      if (shared) {
        const int p = fresh[__popcll(mask & ((1ull << lane) - 1))];
        m.ref[p] = 1;
        m.table[(size_t)b * m.P + c] = p;
        atomicSub(m.ref + (old & ~kSharedMark), 1);
      } else if (c >= cols && c < m.P) {
        m.table[(size_t)b * m.P + c] = -1;
        if (old >= 0) atomicSub(m.ref + old, 1);
      }
      fresh += __popcll(mask);
    }
    if (lane == 0 && first < cols) w.list[atomicAdd(&moves, 1)] = b;  // in any order: no rows in common
  }
  __syncthreads();
  if (tid == 0) w.count[0] = moves;
}

struct MoveArgs {
  LayerPtrs layer;
  PageWs ws;
  MapArgs map;
  const int32_t *keep_idx, *new_len;
  int32_t n_layers, Hkv, row_bytes;
  int32_t n_col;  // 128-byte columns of a K row and a V row together
};

// Threads x rows in flight a thread, for one sequence of 28 layers (166 MB, read and written) / eight of 16 (3.0 GB),
// in a graph with the map's restoring copies: 512 x 4 51.9 / 552 us, 512 x 6 51.7 / 629, 512 x 8 49.2 / 578,
// 256 x 8 47.9 / 550, 1024 x 4 47.7 / 533.
constexpr int kMoveThreads = 1024;
constexpr int kMoveUnroll = 4;  // rows in flight per thread
constexpr int kColBytes = 128;
constexpr int kColLanes = kColBytes / 16;
constexpr int kPassRows = kMoveThreads / kColLanes;
constexpr int kRowsPerPass = kPassRows * kMoveUnroll;
constexpr int kSegmentRows = 2048;  // rows whose places are looked up at once
constexpr int kMoveWorkgroups = 1024;
constexpr uint32_t kStays = 0xffffffffu;

// A workgroup moves one 128-byte column of one head's K or V rows of one sequence, in passes of ascending rows
// whose loads complete before their stores (as the contiguous compaction does: sources lie at or above
// the rows they fill, so what a pass writes in place no later pass reads, and fresh pages are nobody's
// source). Where a row comes from and goes to takes two dependent loads (keep_idx, then the columns of both
// ends), so a segment's rows look them up together and the passes find them in LDS, as slots of the pool (page x
// page_size + row: below 2^32, since a slot has 128 bytes at least).
// Memory bounds it: 3.0 GB in 534 us, 5.6 TB/s, where a copy of 1 GiB runs at 5.2.
struct Moves {
  u32x4_t x[kMoveUnroll];
};

__device__ __forceinline__ size_t pool_row(const MapArgs& m, uint32_t slot, int Hkv, int h) {
  return (((size_t)(slot >> m.shift) * Hkv + h) << m.shift) + (slot & ((1u << m.shift) - 1));
}

__device__ __forceinline__ void move_load(const MoveArgs& a, Moves& v, int r0, int n, int h, const uint32_t* src,
                                          const char* col) {
#pragma unroll
  for (int u = 0; u < kMoveUnroll; ++u) {
    const int r = r0 + u * kPassRows + (int)threadIdx.x / kColLanes;
    const uint32_t s = r < n ? src[r] : kStays;
    if (s != kStays)
      v.x[u] = __builtin_nontemporal_load((const u32x4_t*)(col + pool_row(a.map, s, a.Hkv, h) * a.row_bytes));
  }
}

__device__ __forceinline__ void move_store(const MoveArgs& a, const Moves& v, int r0, int n, int h, const uint32_t* src,
                                           const uint32_t* dst, char* col) {
#pragma unroll
  for (int u = 0; u < kMoveUnroll; ++u) {
    const int r = r0 + u * kPassRows + (int)threadIdx.x / kColLanes;
    if (r < n && src[r] != kStays)
      __builtin_nontemporal_store(v.x[u], (u32x4_t*)(col + pool_row(a.map, dst[r], a.Hkv, h) * a.row_bytes));
  }
}

__global__ __launch_bounds__(kMoveThreads) void move_rows(MoveArgs a) {
  __shared__ uint32_t src[kSegmentRows], dst[kSegmentRows];
  const MapArgs& m = a.map;
  const int per = a.n_layers * a.Hkv * a.n_col, mask = (1 << m.shift) - 1;
  const long long items = (long long)a.ws.count[0] * per;
  int last = -1;  // the sequence whose places LDS holds, if all of them
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int b = a.ws.list[it / per], x = (int)(it % per);
    const int l = x % a.n_layers, y = x / a.n_layers;
    const int c = y % a.n_col, h = y / a.n_col, half = a.n_col / 2;
    char* col = (char*)(c < half ? a.layer.k[l] : a.layer.v[l]) + (c % half) * kColBytes +
                16 * (threadIdx.x % kColLanes);
    const int nl = min(a.new_len[b], m.cap);
    const int32_t* keep = a.keep_idx + (size_t)b * m.cap;
    const int32_t *from = a.ws.table + (size_t)b * m.P, *to = m.table + (size_t)b * m.P;
    const int begin = a.ws.first[b] << m.shift;
    for (int g0 = begin; g0 < nl; g0 += kSegmentRows) {
      const int n = min(nl - g0, kSegmentRows);
      if (b != last) {
        __syncthreads();  // the segment before is done
        for (int i = threadIdx.x; i < n; i += kMoveThreads) {
          const int r = g0 + i, k = keep[r];
          uint32_t s = kStays, d = 0;
          if (k >= r && k < m.cap) {
            const int sp = from[k >> m.shift], dp = to[r >> m.shift];
            if (sp >= 0 && is_page(m, dp)) {
              s = ((uint32_t)(sp & ~kSharedMark) << m.shift) + (k & mask);
              d = ((uint32_t)dp << m.shift) + (r & mask);
              if (s == d) s = kStays;
            }
          }
          src[i] = s;
          dst[i] = d;
        }
        __syncthreads();
      }
      Moves cur, nxt;
      move_load(a, cur, 0, n, h, src, col);
      for (int r0 = 0; r0 < n; r0 += kRowsPerPass) {
        __syncthreads();  // every thread holds this pass's rows
        const bool more = r0 + kRowsPerPass < n;
        if (more) move_load(a, nxt, r0 + kRowsPerPass, n, h, src, col);
        move_store(a, cur, r0, n, h, src, dst, col);
        if (more) cur = nxt;
      }
    }
    last = nl - begin <= kSegmentRows ? b : -1;
  }
}

// ------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------
static void layer_ptrs(LayerPtrs* p, const lg_paged_layer* layers, int n) {
  for (int i = 0; i < n; ++i) {
    p->k[i] = layers[i].k;
    p->v[i] = layers[i].v;
  }
}

static int row_bytes_of(const lg_paged_layer& l) { return l.head_dim * (l.dtype == LG_BF16 ? 2 : 4); }

hipError_t launch_reserve(const lg_page_map& map, int n_layers, const lg_paged_layer* layers,
                          const int32_t* q_start, const int32_t* t, int32_t* base, void* ws,
                          hipStream_t st) {
  ReserveArgs a;
  a.map = map_args(map);
  a.ws = page_ws(map, ws);
  a.q_start = q_start;
  a.t = t;
  a.base = base;
  hipLaunchKernelGGL(reserve_map, dim3(1), dim3(kMapThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  for (int l0 = 0; l0 < n_layers && e == hipSuccess; l0 += kMaxLayersPaged) {
    CopyArgs c;
    c.n_layers = min(kMaxLayersPaged, n_layers - l0);
    layer_ptrs(&c.layer, layers + l0, c.n_layers);
    c.ws = a.ws;
    c.Hkv = layers[0].n_kv_heads;
    c.shift = a.map.shift;
    c.row_bytes = row_bytes_of(layers[0]);
    const long long items = 2ll * c.n_layers * c.Hkv * map.batch;
    hipLaunchKernelGGL(copy_rows, dim3((unsigned)min(items, (long long)kCopyWorkgroups)),
                       dim3(kCopyThreads), 0, st, c);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_fork(const lg_page_map& map, const int32_t* parent, void* ws, hipStream_t st) {
  ForkArgs a;
  a.map = map_args(map);
  a.ws = page_ws(map, ws);
  a.parent = parent;
  if (map.batch <= kForkSmallBatch && (long)map.batch * a.map.cap <= kForkSmall) {
    hipLaunchKernelGGL(fork_small, dim3(1), dim3(kMapThreads), 0, st, a);
    return hipGetLastError();
  }
  const dim3 grid(map.batch, (unsigned)min((a.map.cap - 1) / kForkSlots + 1, kForkSpread));
  hipLaunchKernelGGL(fork_read, grid, dim3(kForkThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fork_write, grid, dim3(kForkThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_compact(const lg_page_map& map, int n_layers, const lg_paged_layer* layers,
                               const int32_t* keep_idx, const int32_t* new_len, int32_t* moved,
                               void* ws, hipStream_t st) {
  CompactMapArgs a;
  a.map = map_args(map);
  a.ws = page_ws(map, ws);
  a.keep_idx = keep_idx;
  a.new_len = new_len;
  a.moved = moved;
  hipLaunchKernelGGL(compact_map, dim3(1), dim3(kMapThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  for (int l0 = 0; l0 < n_layers && e == hipSuccess; l0 += kMaxLayersPaged) {
    MoveArgs c;
    c.n_layers = min(kMaxLayersPaged, n_layers - l0);
    layer_ptrs(&c.layer, layers + l0, c.n_layers);
    c.ws = a.ws;
    c.map = a.map;
    c.keep_idx = keep_idx;
    c.new_len = new_len;
    c.Hkv = layers[0].n_kv_heads;
    c.row_bytes = row_bytes_of(layers[0]);
    c.n_col = 2 * c.row_bytes / kColBytes;
    const long long items = (long long)c.n_layers * c.Hkv * c.n_col * map.batch;
    hipLaunchKernelGGL(move_rows, dim3((unsigned)min(items, (long long)kMoveWorkgroups)),
                       dim3(kMoveThreads), 0, st, c);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace lg
