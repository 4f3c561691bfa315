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
// with lane ^ 32, and P in bfloat16 is the B operand of the second product as it lies in the registers:
// V^T is read in the same order of keys. Scores are in units of log 2 (exp2).
//
// Workgroups (template KW, waves along the keys):
//   KW = 1  sequences with more than 32 query rows: 128 rows, four waves of 32, which share every tile of 64
//           slots (32 in float32), two buffers, one barrier a tile, two workgroups a CU. A row's share of K and
//           V then comes from LDS four times as often as from the L2.
//   KW > 1  the others (a decode step: G rows): the waves take every KW-th tile of 32 slots, each with LDS of its
//           own and no barrier, and their (m, l, O) are joined at the end. paged_few is the launch for steps that
//           have no others, 8 waves a workgroup; beside long chunks (paged_attend) see side_waves.
// When these workgroups are fewer than the CUs hold, the slots of a row are split over several and a second
// launch joins them (paged_plan).
//
// A tile whose slots every row of the wave sees needs no comparison. In the others (the end of the
// causal triangle, the edges of the window) visibility is decided slot by slot. There a value that some
// row does not see could still reach it as 0 x inf = NaN through the matrix product: such a tile's values that
// are not finite count as 0 in it, and reach the rows that see them in a pass behind the loop.
//
// What bounds it, measured on MI355X (a copy reaches 5.2 TB/s, a bfloat16 matrix product of 8192^3 1100
// TFLOP/s): a decode step of 32 sequences of 28 / 4 heads and 1280 to 2047 slots, 112 MB, 23.7 us in a graph, 4.7
// TB/s: the memory. 4096 tokens of 32 / 8 heads behind 4096, 412 GFLOP, 421 to 474 us by card, 870 to 980
// TFLOP/s: of a wave's time a third is matrix instructions and as much the exponentials with their maxima, sums
// and roundings, which the other wave of its SIMD covers in part; the rest is issuing loads and scalar code.
// float32 runs at 133 of the 154 TFLOP/s of a float32 product. 128 tokens each of four sequences with a window
// of 2048 beside 12 decoding ones, 147 MB: 54 to 58 us: a workgroup's chain (4 us to its first tile, 17 tiles of 1.7 us
// and 1.4 more for each of the two or three that are masked) and the launch that joins two splits.
//
// Tried and left: 8 waves sharing the tiles of 256 rows, one workgroup a CU (422 against 440 us for the 4096
// tokens, but 85 against 54 for the mixed step and 177 against 163 for chunks of 512 at head_dim 64); tiles of 32
// slots four deep with counted waits (510 us); the scores of the next tile beside this one's exponentials (539
// us: registers spill).
#include "lg_paged_attend.h"

namespace lg {

// Workgroups a launch with long chunks aims for by splitting slots: two a CU. The mixed step above at 256 / 512 /
// 768 / 1024: 66.3 / 54.9 / 54.8 / 59.7 us, 256 tokens behind 16128 slots 109 / 101 at 256 / 512, 2048 behind 6144
// 245 / 270 at 512 / 768.
constexpr long kPagedTarget = 512;
// Slots of a split at least, and in bfloat16 one more for every 32 query rows of the launch: the partials of a split
// are written and read by row, what it saves goes by its slots (in float32 by 8 times as much). 8 sequences of 128
// tokens, 32 / 8 heads, windows of 256 / 512 / 1024: 22.3 / 28.4 / 40.5 us, 38.7 / 41.7 / 49.5 without the second term;
// half of it 22.6 / 28.9 / 51.7.
constexpr int kMinSplitSlots = 256;
constexpr long kSplitRows = 32;
// Sizes of the team that shares a tile: the workgroup (KW = 1) or a wave (KW = 2, 4, 8).
//
// A row of K or V in LDS is its 16-byte pieces in the order piece ^ f(row): the 16 rows whose pieces one read
// of K takes, and the 4 rows (of 64 bytes) that a transposed read of V takes, then lie in different banks,
// without padding. The rows a lane reads differ from its first one by multiples that leave f as it is, so the
// exchange is one xor with a constant on its first address (tiles lie at multiples of 1024 bytes).
//
// DV: the values of V that the workgroup forms outputs of, D or (KW = 8) half of them. RW: rows of a matrix
// instruction, 32 or (float32, KW > 1) 16.
template <typename T, int D, int KW, int DV = D, int RW = 32>
struct Team {
  static constexpr bool kF32 = sizeof(T) == 4;
  static constexpr int kRowBytes = D * (int)sizeof(T), kRowBytesV = DV * (int)sizeof(T);
  static constexpr int kRowPieces = kRowBytes / 16, kRowPiecesV = kRowBytesV / 16;
  static constexpr int kKeys = kF32 || KW > 1 ? 32 : 64;  // slots of a tile
  static constexpr int kThreads = KW > 1 ? 64 : kPagedThreads;
  static constexpr int kPieces = kKeys * kRowPieces / kThreads;  // 16-byte pieces a thread, of K ...
  static constexpr int kPiecesV = kKeys * kRowPiecesV / kThreads;  // ... and of V
  static constexpr int kLoadRows = 64 / kRowPieces, kLoadRowsV = 64 / kRowPiecesV;  // rows that a wave loads at once
  static constexpr int kWaveLoad = kKeys / (KW > 1 ? 1 : 4);      // rows of a tile that a wave loads
  static constexpr int kGroups = kWaveLoad > 16 ? kWaveLoad / 16 : 1;  // of 16 rows, each inside one page
  static constexpr int kTile = kKeys * kRowBytes, kTileV = kKeys * kRowBytesV;
  static constexpr int kBuffer = kTile + kTileV;
  // the join of KW > 1: a wave's O as [row][DV + 4] and its m, l, suffix sums
  static constexpr int kJoin = KW > 1 ? kWaveRows * (DV + 4) * 4 + 3 * kWaveRows * 4 : 0;
  static constexpr int kTiles = kBuffer * (KW > 1 ? 1 : 2);
  static constexpr int kLds = kTiles > kJoin ? kTiles : (kJoin + 511) & ~511;
  static __device__ __forceinline__ int fk(int row) { return kF32 || D == 128 ? row & 15 : (row >> 1) & 7; }
  static __device__ __forceinline__ int fv(int row) {
    return kF32 && RW == 16 ? 4 * ((row >> 2) & 3) : kF32 ? 8 * ((row >> 2) & 1) : DV == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
  }
};

// Tiles whose table entries and positions (64 of each) a wave holds at once.
constexpr int kRing = 3 * 512;

// Waves for a sequence of few rows beside long chunks; the other waves of the workgroup end at once (a barrier waits for
// those that are left). Two in float32 with rows of 512 bytes: a workgroup then has 70 KB of LDS, and two of them on a CU
// carry long chunks faster than one with 134 KB: 256 tokens each of 4 sequences of 4096 slots, 32 / 8 heads, 459 us
// against 506, 16 sequences of which 4 bring 128 tokens to a window of 1024 116 against 138; steps whose decoding
// sequences weigh most lose (8 sequences of 2048 slots, two bring 64 tokens: 99 against 92).
template <typename T, int D>
constexpr int side_waves() { return sizeof(T) == 4 && D == 128 ? 2 : 4; }

template <typename T, int D>
constexpr int paged_lds() {
  constexpr int many = Team<T, D, 1>::kLds + 4 * kRing, few = side_waves<T, D>() * (Team<T, D, side_waves<T, D>()>::kLds + kRing);
  return (many > few ? many : few) + 4 * 4;  // and the flags of make_finite
}

template <typename T, int D, int KW, int DV>
constexpr int few_lds() {
  return KW * (Team<T, D, KW, DV>::kLds + kRing) + 4 * KW;
}

// 16 bytes a lane from global memory straight into LDS: lane i's go to lds + 16 i. lds is the same in all
// lanes.
__device__ __forceinline__ void load_lds(const char* base, unsigned off, char* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + off),
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

__device__ __forceinline__ void load_lds4(const int32_t* from, int32_t* lds) {  // 4 bytes a lane, likewise
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)lds, 4, 0, 0);
}

// Waits until at most N of the wave's loads are on their way, and keeps reads of LDS behind that.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);  // vmcnt(N)
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  __builtin_amdgcn_sched_barrier(0);
}

// The wave's reads of LDS have returned, and what it asks for next stays behind them.
__device__ __forceinline__ void reads_done() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ bool odd_bits(uint32_t x, bool f32) {  // an infinity or NaN in a word
  return f32 ? (x & 0x7f800000u) == 0x7f800000u
             : (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
}

// Order for the scheduler: the scores of 64 keys' 16 reads of LDS and 16 matrix instructions, the reads 8
// ahead (left to itself it reads 2 ahead; 462 us for a chunk of 4096 tokens behind 4096, 455 with this).
__device__ __forceinline__ void schedule_scores() {
  __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);  // reads of LDS
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix instructions
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
}

// flags: in LDS, one a team (see make_finite).
//
// RW = 16 (float32, at most 16 rows): the same walk with v_mfma_f32_16x16x4. A lane holds 8 of 32 keys, 4 of every 16, and
// the four lanes of a row are 16 apart. The float32 products bound a decode step: with 32 rows of which a few live they
// cost twice as much. 8 sequences of 4096 / 16 of 8192 slots of capacity, 32 / 8 heads: 44.8 / 179 us, 52.2 / 248 with 32
// rows; 16 tokens of a tiny layer 8.6, 10.6. (bfloat16 has no need: its decode steps are bound by memory.)
//
// The lane's values of S and O lie in fours: S at keys kFour i + 4 part, O at values RW d + kFour i + 4 part.
template <typename T, int D, int KW, int DV, int RW = 32>
__device__ __forceinline__ void paged_body(const PagedAttendArgs& a, Job job, char* lds, int32_t* flags) {
  using C = Team<T, D, KW, DV, RW>;
  static_assert(RW == 32 || (C::kF32 && KW > 1), "16 rows: float32, few rows");
  constexpr bool F32 = C::kF32;
  // How bfloat16 weights enter the product with V. Few rows: as two terms, within 2^-16, as in lg_decode_attend; memory
  // bounds these steps (32 sequences of 28 / 4 heads above: 23.7 us, 22.8 with one term; 64 sequences of 32 / 8 heads
  // and 1024 slots 40.6 and 39.7; most where few tiles a wave leave the chain to show: 16 of 28 / 4 and 2048 slots 18.7
  // and 17.1). Chunks of more than 32 rows: rounded once, since their matrix instructions bound them: with two terms 4096
  // tokens behind 4096 take 577 us (429), at head_dim 64 372 (280), 8 x 128 tokens of a window of 1024 51 (43). An
  // output then lies within 2^-8 sum alpha |v|; against 64 bits, over all outputs of a mixed step, 1.71e-3 where the
  // outputs' own rounding is 1.67e-3.
  constexpr bool kTwoTerms = !F32 && KW > 1;
  constexpr int NK = C::kKeys, NB = NK / 32, ND = DV / RW, RB = C::kRowBytes, RBV = C::kRowBytesV;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = lane / RW, col = lane % RW;
  constexpr int kParts4 = 64 / RW, kFour = 4 * kParts4;  // lanes of a row; keys (values) between a lane's fours
  constexpr int NS = RW / 2, NI = NS / 4;                // the lane's weights of 32 keys
  constexpr int NO = RW * RW / 64, NOI = NO / 4;         // ... and values of an accumulator of O
  using Weights = std::conditional_t<RW == 32, f32x16, f32x8>;
  using Acc = std::conditional_t<RW == 32, f32x16, f32x4>;
  char* const my = KW > 1 ? lds + wave * (C::kLds + kRing) : lds;
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
  const bool idle = wrow0 >= job.rows;  // KW = 1: a wave without rows only loads

  Acc O[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < NO; ++i) O[d][i] = 0.f;
  float mx = -INFINITY, l = 0.f, sfx = 0.f;  // l and sfx: the lane's share of the keys

  int t_end = job.t_end, t_first = KW > 1 ? job.t_begin + wave : job.t_begin;
  const int last_slot =  // the last one that any row of the workgroup sees
      job.base + (min(job.row0 + (KW > 1 ? kWaveRows : kManyRows), job.rows) - 1) / a.G;
  auto slot_of = [&](int t) __attribute__((always_inline)) { return (t < job.sink_tiles ? t : t - job.sink_tiles + job.tile0) * NK; };

  // A tile comes in two steps: its columns of the table and its positions (a lane per slot), then its rows,
  // both straight into LDS, with no registers in between. A load instruction of a wave fills LDS in the
  // order of its lanes, so the exchange of a row's pieces is made on the global side: the lane at position
  // p of a row loads piece p ^ f(row). Slots behind last_slot read as last_slot and slots of missing pages
  // as page 0: no row sees them.
  int32_t* const ring = (int32_t*)(my + C::kLds + (KW > 1 ? 0 : wave * kRing));
  int32_t* const odd = flags + (KW > 1 ? wave : 0);
  auto look = [&](int t, int32_t* __restrict__ to) __attribute__((always_inline)) {
    const int s = min(slot_of(min(t, t_end - 1)) + (lane & (NK - 1)), last_slot);
    load_lds4(table + (s >> m.shift), to);
    load_lds4(pos + s, to + 64);
  };
  // What depends on the sequence alone is asked for together: the first tile's lookup, the queries, positions.
  if (t_first < t_end) look(t_first, ring);
  // Q as the B operand: bf16: values 16 kk + 8 part ..; float32: values part D / kParts4 + 4 u ..
  constexpr int NQ = F32 ? D / (4 * kParts4) : D / 16;
  u32x4_t qf[NQ];
  {
    const char* src = (const char*)a.q + qrow * RB;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
      qf[i] = *(const u32x4_t*)(src + (F32 ? part * (RB / kParts4) + 16 * i : 32 * i + 16 * part));
  }

  const int p_q = pos[slot_q];
  if (skip_hidden<NK>(a, job, pos)) {
    t_end = job.t_end;
    t_first = KW > 1 ? job.t_begin + wave : job.t_begin;
    wait_loads<0>();  // the first lookup has landed
    if (t_first < t_end) look(t_first, ring);
  }
  const int sw = a.suffix_w != nullptr ? a.suffix_w[job.b] : 0;
  // the row sees pos > win and, of these, counts pos > suf as its suffix
  const int win = a.window > 0 ? (int)max((long long)p_q - a.window, (long long)INT32_MIN) : INT32_MIN;
  const int suf = (int)max((long long)p_q - max(sw, 0), (long long)INT32_MIN);
  // bounds over the wave's rows (tokens ascend with the row, positions with the token)
  const int slot_lo = __builtin_amdgcn_readlane(slot_q, 0), slot_hi = __builtin_amdgcn_readlane(slot_q, 31);
  const int win_hi = __builtin_amdgcn_readlane(win, 31);
  // and over the workgroup's (KW = 1)
  const int slot_lo_all = job.base + job.row0 / a.G;
  const int win_hi_all = KW == 1 && a.window > 0 ? (int)max((long long)pos[last_slot] - a.window, (long long)INT32_MIN) : INT32_MIN;
  const int suf_lo = __builtin_amdgcn_readlane(suf, 0), suf_hi = __builtin_amdgcn_readlane(suf, 31);
  // The position of the lane's slot, kHidden without a page.
  auto place = [&](const int32_t* at) __attribute__((always_inline)) { return is_page(m, at[lane]) ? at[64 + lane] : kHidden; };
  const int load0 = KW > 1 ? 0 : wave * C::kWaveLoad;  // the wave's first row of a tile
  struct Groups {
    size_t at[C::kGroups];  // bytes of the group's first row in k and v
    int most[C::kGroups];   // rows of the group from here on repeat it
  };
  auto groups = [&](int t, const int32_t* at) __attribute__((always_inline)) {
    const int tv = at[lane];
    Groups gr;
#pragma unroll
    for (int i = 0; i < C::kGroups; ++i) {
      const int r0 = (load0 & ~15) + 16 * i;
      int page = __builtin_amdgcn_readlane(tv, r0);  // of slot min(s0 + r0, last_slot)
      page = is_page(m, page) ? page : 0;
      const int s = min(slot_of(t) + r0, last_slot & ~15);
      gr.at[i] = ((((size_t)page * a.Hkv + job.h) << m.shift) + (s & ((1 << m.shift) - 1))) * RB;
      gr.most[i] = last_slot - s;
    }
    return gr;
  };
  // Rows of a tile's K or V to LDS at `to` + off. A group with all its rows (all but the last of a sequence)
  // needs one offset a lane; the rest is in the instruction and an exclusive or.
  auto load_part = [&](const Groups& gr, const char* pages, char* to, int off, auto pieces, auto n, auto stride,
                       auto f) __attribute__((always_inline)) {
    constexpr int kRow = decltype(pieces)::value, kN = decltype(n)::value, kStep = 64 / kRow;
    const int lrow = lane / kRow, piece = lane % kRow;
    const int first = lrow * RB + 16 * (piece ^ f(load0 | lrow));
#pragma unroll
    for (int i = 0; i < C::kGroups; ++i) {
      const char* base = pages + gr.at[i];
      const bool whole = gr.most[i] >= 15;
#pragma unroll
      for (int u = i * kN / C::kGroups; u < (i + 1) * kN / C::kGroups; ++u) {
        const int up = u * kStep, row = (load0 + up) | lrow;
        unsigned at = (first ^ (16 * f(up))) + ((load0 + up) & 15) * RB;
        if (!whole) at = (unsigned)(min(row & 15, gr.most[i]) * RB + 16 * (piece ^ f(row)));
        load_lds(base, at, to + off + (load0 + up) * decltype(stride)::value);
      }
    }
  };
  auto load_k = [&](const Groups& gr, char* to, int off) __attribute__((always_inline)) {
    load_part(gr, (const char*)a.k, to, off, Num<C::kRowPieces>{}, Num<C::kPieces>{}, Num<RB>{},
              [](int row) { return C::fk(row); });
  };
  auto load_v = [&](const Groups& gr, char* to, int off) __attribute__((always_inline)) {
    load_part(gr, (const char*)a.v + job.d0 * sizeof(T), to, off, Num<C::kRowPiecesV>{}, Num<C::kPiecesV>{}, Num<RBV>{},
              [](int row) { return C::fv(row); });
  };

  // The lane's first addresses in a tile (see Team).
  const int kx = col * RB + 16 * ((F32 ? part * (C::kRowPieces / kParts4) : part) ^ C::fk(col));
  const int vx = F32 ? 4 * part * RBV + 16 * ((col >> 2) ^ C::fv(4 * part)) + 4 * (col & 3)
                     : (4 * part + ((lane & 15) >> 2)) * RBV +
                           16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ C::fv((lane & 15) >> 2)) +
                           8 * (lane & 1);

  // S^T of 32 keys of a tile
  auto scores = [&](const char* from, int k, Weights& S) __attribute__((always_inline)) {
    if constexpr (RW == 16) {
      f32x4 s0 = {}, s1 = {};
#pragma unroll
      for (int u = 0; u < NQ; ++u) {
        const u32x4_t x = *(const u32x4_t*)(from + ((k + kx) ^ (16 * u)));
        const u32x4_t y = *(const u32x4_t*)(from + ((k + kx) ^ (16 * u)) + 16 * RB);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[e]), __uint_as_float(qf[u][e]), s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(y[e]), __uint_as_float(qf[u][e]), s1, 0, 0, 0);
        }
      }
      S = Weights{s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
      for (int u = 0; u < NQ; ++u) {
        const u32x4_t x = *(const u32x4_t*)(from + ((k + kx) ^ (F32 ? 16 * u : 32 * u)));
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            S = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(qf[u][e]), S, 0, 0, 0);
        } else {
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, qf[u]),
                                                      S, 0, 0, 0);
        }
      }
    }
  };
  // Maximum of the lane's row over the block, in all its lanes
  auto top = [&](const Weights& S) __attribute__((always_inline)) {
    float t4[4] = {S[0], S[1], S[2], S[3]};
#pragma unroll
    for (int i = 4; i < NS; ++i) t4[i & 3] = fmaxf(t4[i & 3], S[i]);
    float x = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
    if constexpr (RW == 16) x = fmaxf(x, other_row(x));
    return fmaxf(x, other_half(x));
  };

  // What a tile needs compared, the same in all lanes. tp: its positions, a lane per slot; at: the wave's table
  // entries and positions of it in LDS. In a masked tile the entries, not needed any more, become the slots' own
  // bounds: a row sees slot j if bound_j > win and the slot is none behind its own. Both are read four slots
  // at a time, as they lie in the accumulators' rows.
  int s0, tp;
  int32_t* at;
  // for rows whose first one is at slot lo and whose last one sees positions above hi
  auto is_masked = [&](int lo, int hi) __attribute__((always_inline)) {
    const int p_first = __builtin_amdgcn_readlane(tp, 0), p_last = __builtin_amdgcn_readlane(tp, NK - 1);
    return __ballot(tp == kHidden) != 0 || s0 + NK - 1 > lo || (a.window > 0 && p_first <= hi && p_last >= a.n_sink);
  };
  auto four = [&](const int32_t* x, int nb, int i) __attribute__((always_inline)) {
    return *(const i32x4*)(x + 32 * nb + kFour * i + 4 * part);
  };
  auto set_bounds = [&]() __attribute__((always_inline)) {
    at[lane] = tp == kHidden ? INT32_MIN : a.window == 0 || tp < a.n_sink ? INT32_MAX : tp;
  };
  auto mask = [&](Weights& S, int nb) __attribute__((always_inline)) {
    const int last = slot_q - s0 - 32 * nb - 4 * part;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const i32x4 bound = four(at, nb, i);
#pragma unroll
      for (int j = 0; j < 4; ++j) S[4 * i + j] = bound[j] > win && kFour * i + j <= last ? S[4 * i + j] : -INFINITY;
    }
  };
  // The running maximum follows only when a score passes it by kSlack: weights are then at most 2^kSlack,
  // which costs no precision, and most tiles leave O as it is. A row goes by its own scores alone.
  auto raise_max = [&](float most) __attribute__((always_inline)) {
    const float tmax = most * a.scale_log2;
    const bool raise = tmax > mx + kSlack;
    if (__any(raise)) {
      const float f = raise ? __builtin_amdgcn_exp2f(mx - tmax) : 1.f;  // 0 where nothing was seen before
      mx = raise ? tmax : mx;
      l *= f;
      sfx *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < NO; ++i) O[d][i] *= f;
    }
  };
  // The suffix's share of a tile: none, all, or slot by slot (slots that are not seen have weight 0)
  enum { kNone, kAll, kSome };
  auto suffix_of = [&]() __attribute__((always_inline)) {
    if (a.suffix == nullptr && a.conf == nullptr) return (int)kNone;
    const int p_first = __builtin_amdgcn_readlane(tp, 0), p_last = __builtin_amdgcn_readlane(tp, NK - 1);
    // kHidden in front says nothing about the slots behind it
    return p_last <= suf_lo ? (int)kNone : p_first > suf_hi && p_first != kHidden ? (int)kAll : (int)kSome;
  };
  auto add_suffix = [&](const Weights& P, int nb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const i32x4 p = four(at + 64, nb, i);
#pragma unroll
      for (int j = 0; j < 4; ++j) sfx += p[j] > suf ? P[4 * i + j] : 0.f;
    }
  };
  // S becomes the weights; returns their sum over the lane's share.
  auto weights = [&](Weights& S) __attribute__((always_inline)) {
    float s4[4];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      S[i] = __builtin_amdgcn_exp2f(fmaf(S[i], a.scale_log2, mx == -INFINITY ? 0.f : -mx));
      s4[i & 3] = i < 4 ? S[i] : s4[i & 3] + S[i];
    }
    return (s4[0] + s4[1]) + (s4[2] + s4[3]);
  };
  // Puts 0 in the place of what is not finite in V of a tile (in LDS), and says so in *odd. With KW = 1 the waves
  // share the tile, so each that reads it does this first when any of them has to, all with the same result:
  // what a wave then reads does not depend on the others' pace.
  auto make_finite = [&](char* v) __attribute__((always_inline)) {
    // Is there any? An exponent of ones and one more carries into the bit above it.
    constexpr uint32_t kExp = F32 ? 0x7f800000u : 0x7f807f80u, kOne = F32 ? 0x00800000u : 0x00800080u;
    uint32_t carry = 0;
#pragma unroll
    for (int i = 0; i < C::kTileV / 1024; ++i) {
      const u32x4_t x = *(const u32x4_t*)(v + 1024 * i + 16 * lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) carry |= (x[e] & kExp) + kOne;
    }
    if (!__any((carry & (kExp + kOne)) != 0)) return;
    for (int i = lane; i < C::kTileV / 16; i += 64) {
      u32x4_t x = *(const u32x4_t*)(v + 16 * i);
      if (odd_bits(x[0], F32) || odd_bits(x[1], F32) || odd_bits(x[2], F32) || odd_bits(x[3], F32)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (F32) {
            if (odd_bits(x[e], true)) x[e] = 0;
          } else {
            if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
            if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
          }
        }
        *(u32x4_t*)(v + 16 * i) = x;
        *odd = 1;
      }
    }
  };

  // O^T += V^T P^T over 32 keys
  auto product = [&](const char* from, int v, const Weights& P) __attribute__((always_inline)) {
    if constexpr (RW == 16) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const float x = *(const float*)(from + ((v + vx) ^ (64 * d)) + (kFour * (i >> 2) + (i & 3)) * RBV);
          O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, P[i], O[d], 0, 0, 0);
        }
    } else if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const float x = *(const float*)(from + ((v + vx) ^ (128 * d)) + (8 * (i >> 2) + (i & 3)) * RBV);
          O[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, P[i], O[d], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4_t p, rest;  // the weights as bfloat16, the matrix product's type
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = P[8 * s + 2 * e], y = P[8 * s + 2 * e + 1];
          if constexpr (kTwoTerms) {
            const TwoTerms two = split_bf16(x, y);
            p[e] = two.most;
            rest[e] = two.rest;
          } else {
            p[e] = pack_bf16(x, y);
          }
        }
        // a 16-lane group reads 4 keys x 16 values and gets them transposed: lane = value
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const char* at = from + ((v + vx) ^ (64 * d)) + 16 * s * RBV;
          const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at);
          const i16x4 hi =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(at + 8 * RBV));
          const u32x2_t x = __builtin_bit_cast(u32x2_t, lo), y = __builtin_bit_cast(u32x2_t, hi);
          const u32x4_t z = {x[0], x[1], y[0], y[1]};
          O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, z), __builtin_bit_cast(bf16x8, p),
                                                         O[d], 0, 0, 0);
          if constexpr (kTwoTerms)
            O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, z),
                                                           __builtin_bit_cast(bf16x8, rest), O[d], 0, 0, 0);
        }
      }
    }
  };
  constexpr int kBlock = 32 * RB, kBlockV = 32 * RBV;  // bytes of 32 keys

  // KW = 1: two buffers and one barrier a tile: a wave's loads have landed before it, so all have behind it, and
  // what the loads behind it fill has been read. KW > 1: one buffer; K of the next tile is asked for when the
  // scores are formed, V when the product is, and the waits count the loads that may be on their way behind
  // those needed (loads land in order; others among them only make a wait longer). The tile functions take
  // what they fill and what they read as pointers that do not alias: the compiler would make every read wait for
  // every load.
  const int step = KW;
  if (KW > 1 || tid == 0) *odd = 0;
  if constexpr (KW == 1) __syncthreads();
  if (t_first < t_end) {
    wait_loads<0>();
    const Groups gr = groups(t_first, ring);
    load_k(gr, my, 0);
    look(t_first + step, ring + 128);
    load_v(gr, my, C::kTile);
  }
  if constexpr (KW == 1) {
    auto tile = [&](int t, int here, const char* __restrict__ from, char* __restrict__ to, const Groups& gr,
                    int32_t* __restrict__ ring_to) __attribute__((always_inline)) {
      const int other = C::kBuffer - here;
      if (t + 1 < t_end) {
        load_k(gr, to, other);
        load_v(gr, to, other + C::kTile);
      }
      look(t + 2, ring_to);
      if (idle || s0 > slot_hi) return;
      Weights S, S1;
      scores(from, here, S);
      if constexpr (NB > 1) {
        scores(from, here + kBlock, S1);
        schedule_scores();
      }
      const int how = suffix_of();
      if (is_masked(slot_lo_all, win_hi_all)) {
        make_finite(const_cast<char*>(from) + here + C::kTile);
        if (is_masked(slot_lo, win_hi)) {
          set_bounds();
          mask(S, 0);
          if constexpr (NB > 1) mask(S1, 1);
        }
      }
      raise_max(NB > 1 ? fmaxf(top(S), top(S1)) : top(S));
      // Without a branch up to the sums: the second block's exponentials beside the first one's product.
      float sum = weights(S);
      product(from, here + C::kTile, S);
      if constexpr (NB > 1) {
        sum += weights(S1);
        product(from, here + C::kTile + kBlockV, S1);
      }
      l += sum;
      sfx += how == kAll ? sum : 0.f;
      if (how == kSome) {
        add_suffix(S, 0);
        if constexpr (NB > 1) add_suffix(S1, 1);
      }
    };
    for (int t = t_first, n = 0; t < t_end; ++t, n = n == 2 ? 0 : n + 1) {
      wait_loads<0>();
      __syncthreads();
      const int n1 = n == 2 ? 0 : n + 1, n2 = n1 == 2 ? 0 : n1 + 1;
      const Groups gr = groups(t + 1, ring + 128 * n1);
      at = ring + 128 * n;
      tp = place(at);
      s0 = slot_of(t);
      tile(t, ((t - t_first) & 1) * C::kBuffer, my, my, gr, ring + 128 * n2);
    }
  } else {
    auto behind_scores = [&](int t, bool more, const Groups& gr, Weights& S, const char* __restrict__ from,
                             char* __restrict__ to, int32_t* __restrict__ ring_to) __attribute__((always_inline)) {
      if (more) load_k(gr, to, 0);
      look(t + 2 * KW, ring_to);
      const bool masked = is_masked(slot_lo, win_hi);
      const int how = suffix_of();
      if (masked) {
        set_bounds();
        mask(S, 0);
      }
      raise_max(top(S));
      const float sum = weights(S);
      l += sum;
      sfx += how == kAll ? sum : 0.f;
      if (how == kSome) add_suffix(S, 0);
      if (more)
        wait_loads<C::kPieces>();  // V is here; K of the next tile may be on its way
      else
        wait_loads<0>();
      if (masked) make_finite(const_cast<char*>(from) + C::kTile);
      product(from, C::kTile, S);
    };
    for (int t = t_first, n = 0; t < t_end; t += KW, n = n == 2 ? 0 : n + 1) {
      const bool more = t + KW < t_end;
      wait_loads<C::kPiecesV>();  // K is here; V may be on its way
      const int n1 = n == 2 ? 0 : n + 1, n2 = n1 == 2 ? 0 : n1 + 1;
      const Groups gr = groups(t + KW, ring + 128 * n1);
      at = ring + 128 * n;
      tp = place(at);
      s0 = slot_of(t);
      Weights S;
      scores(my, 0, S);
      reads_done();
      behind_scores(t, more, gr, S, my, my, ring + 128 * n2);
      reads_done();
      if (more) load_v(gr, my, C::kTile);
    }
    wait_loads<0>();
  }

  // Values that are not finite in tiles that not every row sees counted as 0 so far. To a row that sees one with a
  // weight above 0 it is what it is, whatever that weight: added here, slot by slot (again where a
  // product has it already, which changes nothing).
  if constexpr (KW == 1) __syncthreads();
  if (*odd != 0) {
    for (int t = t_first; t < t_end; t += KW) {
      s0 = slot_of(t);
      if (idle || s0 > slot_hi) continue;
      for (int key = 0; key < NK; ++key) {
        const int j = min(s0 + key, last_slot);
        const int page = table[j >> m.shift];
        if (!is_page(m, page) || s0 + key > slot_q || (a.window > 0 && pos[j] <= win && pos[j] >= a.n_sink)) continue;
        const T* row = (const T*)a.v +
                       ((((size_t)page * a.Hkv + job.h) << m.shift) + (j & ((1 << m.shift) - 1))) * D +
                       job.d0 + 4 * part;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int e = 0; e < NO; ++e) {
            const float x = (float)row[RW * d + kFour * (e >> 2) + (e & 3)];
            O[d][e] += odd_bits(__float_as_uint(x), true) ? x : 0.f;
          }
      }
    }
  }

  if constexpr (RW == 16) {
    l += other_row(l);
    sfx += other_row(sfx);
  }
  l += other_half(l);
  sfx += other_half(sfx);

  if constexpr (KW == 1) {
    if (idle) return;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;  // no slot seen: 0
    const float mass = l == 0.f ? 0.f : sfx * inv;
    if (a.ns == 1 && a.conf != nullptr) raise_conf(a.conf + job.b, mass, tok == job.rows / a.G - 1);
    if (!live) return;
    if (a.ns > 1) {
      const size_t at = (size_t)job.split * a.total * a.Hq + qrow;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(a.po + at * D + 32 * d + 8 * i + 4 * part) =
              f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
      if (part == 0) *(f32x4*)(a.pml + at * 4) = f32x4{mx, l, sfx, 0.f};
      return;
    }
    T* dst = (T*)a.out + qrow * D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 32 * d + 8 * i + 4 * part;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : O[d][4 * i + e] * inv;
        if constexpr (F32)
          *(f32x4*)(dst + at) = f32x4{x[0], x[1], x[2], x[3]};
        else
          *(u32x2_t*)(dst + at) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
      }
    if (part == 0) {
      a.lse[qrow] = l == 0.f ? -INFINITY : kLn2 * (mx + __builtin_amdgcn_logf(l));
      if (a.suffix != nullptr) a.suffix[qrow] = mass;
    }
  } else {
    // Join the waves: their numerators and statistics through LDS, 2 KW threads a row.
    constexpr int kStat = kWaveRows * (DV + 4), kParts = 2 * KW, kChunks = DV / (4 * kParts);
    float* const num = (float*)my;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < NOI; ++i)
        *(f32x4*)(num + col * (DV + 4) + RW * d + kFour * i + 4 * part) =
            f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
    if (part == 0) {
      num[kStat + col] = mx;
      num[kStat + kWaveRows + col] = l;
      num[kStat + 2 * kWaveRows + col] = sfx;
    }
    __syncthreads();
    auto row_of = [&](int r) __attribute__((always_inline)) {
      const int tk = r / a.G;
      return (size_t)(job.first + tk) * a.Hq + job.h * a.G + (r - tk * a.G);
    };
    const size_t split0 = (size_t)job.split * a.total * a.Hq;
    if (wave == KW - 1 && job.d0 == 0) {  // the statistics, a lane a row
      const int r = min(col, job.rows - 1);
      float M = -INFINITY, L = 0.f, SF = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) M = fmaxf(M, ((const float*)(lds + w * (C::kLds + kRing)))[kStat + r]);
      const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float* src = (const float*)(lds + w * (C::kLds + kRing)) + kStat + r;
        const float f = __builtin_amdgcn_exp2f(src[0] - Ms);
        L += f * src[kWaveRows];
        SF += f * src[2 * kWaveRows];
      }
      const bool own = lane < job.rows;
      const size_t row = row_of(r);
      if (a.ns > 1) {
        if (own) *(f32x4*)(a.pml + (split0 + row) * 4) = f32x4{M, L, SF, 0.f};
      } else {
        const float mass = L == 0.f ? 0.f : SF * (1.f / L);
        if (own) {
          a.lse[row] = L == 0.f ? -INFINITY : kLn2 * (M + __builtin_amdgcn_logf(L));
          if (a.suffix != nullptr) a.suffix[row] = mass;
        }
        if (a.conf != nullptr) raise_conf(a.conf + job.b, mass, r / a.G == job.rows / a.G - 1);
      }
    }
    const int r = tid / kParts, share = tid % kParts;
    if (r >= job.rows) return;
    float wm[KW], M = -INFINITY;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      wm[w] = ((const float*)(lds + w * (C::kLds + kRing)))[kStat + r];
      M = fmaxf(M, wm[w]);
    }
    const float Ms = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    f32x4 x[kChunks] = {};
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float* src = (const float*)(lds + w * (C::kLds + kRing));
      const float f = __builtin_amdgcn_exp2f(wm[w] - Ms);
      L += f * src[kStat + kWaveRows + r];
#pragma unroll
      for (int i = 0; i < kChunks; ++i) x[i] += f * *(const f32x4*)(src + r * (DV + 4) + 4 * (kParts * i + share));
    }
    const size_t row = row_of(r);
    if (a.ns > 1) {
#pragma unroll
      for (int i = 0; i < kChunks; ++i)
        *(f32x4*)(a.po + (split0 + row) * D + job.d0 + 4 * (kParts * i + share)) = x[i];
      return;
    }
    const float inv = 1.f / L;
    T* dst = (T*)a.out + row * D + job.d0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = L == 0.f ? 0.f : x[i][e] * inv;
      if constexpr (F32)
        *(f32x4*)(dst + 4 * (kParts * i + share)) = y;
      else
        *(u32x2_t*)(dst + 4 * (kParts * i + share)) = u32x2_t{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    }
  }
}

// Grid: (Hkv, ns, many_tiles + B), flattened with the KV head fastest: the workgroups of one head of one
// sequence are Hkv apart, so with 8 heads (the XCDs are dealt workgroups in turn) they share an L2. The
// tiles of many rows come first, the last of a sequence (the longest) before the others.
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_attend(PagedAttendArgs a) {
  __shared__ __align__(512) char lds[paged_lds<T, D>()];
  int32_t* const flags = (int32_t*)(lds + paged_lds<T, D>() - 16);
  const int per = a.Hkv * a.ns;
  const int unit = blockIdx.x / per, rest = blockIdx.x % per;
  Job job;
  job.h = rest % a.Hkv;
  const int split = rest / a.Hkv;
  if (unit < a.many_tiles) {
    if (!many_job(a, job, unit)) return;
    job_tiles<Team<T, D, 1>::kKeys>(a, job, kManyRows, split);
    job.d0 = 0;
    paged_body<T, D, 1, D>(a, job, lds, flags);
    return;
  }
  constexpr int KW = side_waves<T, D>();
  if (few_job(a, job, unit - a.many_tiles, rest == 0) && threadIdx.x < 64 * KW) {
    job_tiles<Team<T, D, KW>::kKeys>(a, job, kWaveRows, split);
    job.d0 = 0;
    if constexpr (sizeof(T) == 4) {
      if (job.rows <= 16) {
        paged_body<T, D, KW, D, 16>(a, job, lds, flags);
        return;
      }
    }
    paged_body<T, D, KW, D>(a, job, lds, flags);
  }
}

// A step without sequences of more than 32 query rows. KW waves a workgroup (8 where LDS holds their tiles), so
// a sequence's slots are swept by as many loads as the memory needs on their way with one workgroup a CU.
// DV < D: two workgroups a KV head, each with all of K and half of V, in place of a split of the slots: no
// second launch to join them, and K comes to the second from the L2 of their XCD (they are 8 workgroups apart).
// For the 128 pairs of the decode step above 26.4 us a call, 34.4 with four-wave workgroups, four splits and the
// launch that joins them (24 and 8 us).
// Grid: (Hkv, ns, B) flattened into units; with two halves, groups of 8 units' first halves, then their second.
template <typename T, int D, int KW, int DV, int RW>
__global__ __launch_bounds__(64 * KW) void paged_few(PagedAttendArgs a) {
  __shared__ __align__(512) char lds[few_lds<T, D, KW, DV>()];
  const unsigned per = (unsigned)(a.Hkv * a.ns);
  unsigned unit = blockIdx.x;
  Job job;
  job.d0 = 0;
  if constexpr (DV < D) {
    const unsigned group = unit / 16 * 8, in = unit % 16, size = min(8u, per * a.map.B - group);
    unit = group + in % size;
    job.d0 = in / size * DV;
  }
  const unsigned b = unit / per, x = unit % per;
  job.h = x % a.Hkv;
  if (!few_job(a, job, b, x == 0 && job.d0 == 0)) return;
  job_tiles<32>(a, job, kWaveRows, x / a.Hkv);
  paged_body<T, D, KW, DV, RW>(a, job, lds, (int32_t*)(lds + few_lds<T, D, KW, DV>() - 4 * KW));
}

// Joins the splits of a row: D / 4 lanes a query row of a token, four values each. What it reads of the partials
// does not depend on the sequence (rows of no sequence hold anything), so its first loads are on their way while
// the sequence is found.
constexpr int kMaxNs = 64;
constexpr int kJoinAhead = 8;  // splits that are loaded together

template <int D>
constexpr int join_rows() { return kPagedThreads / (D / 4); }

template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_join(PagedAttendArgs a) {
  __shared__ int best[join_rows<D>()];  // of the tokens that the workgroup has rows of
  const long long rows = (long long)a.total * a.Hq;
  const long long first = (long long)blockIdx.x * join_rows<D>();
  if (threadIdx.x < join_rows<D>()) best[threadIdx.x] = -1;
  const long long row = min(first + threadIdx.x / (D / 4), rows - 1);
  const int d = threadIdx.x % (D / 4) * 4;
  f32x4 st[kJoinAhead], y[kJoinAhead];
  auto load = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      const long long at = min(s0 + i, a.ns - 1) * rows + row;
      st[i] = *(const f32x4*)(a.pml + at * 4);
      y[i] = *(const f32x4*)(a.po + at * D + d);
    }
  };
  load(0);
  // the sequences of the workgroup's first row, and from there on those that end before this row
  const int r = (int)(row / a.Hq);
  int b = seq_of_row(a.q_start, a.map.B, (int)(first / a.Hq));
  while (b < a.map.B && a.q_start[b + 1] <= r) ++b;
  const bool some = b < a.map.B;
  const Chunk c = some ? chunk_of(a.q_start, b, a.total) : Chunk{0, 0};
  const int base = some ? a.base[b] : -1;
  float M = -INFINITY, L = 0.f, SF = 0.f;
  f32x4 x = {};
  for (int s0 = 0; s0 < a.ns; s0 += kJoinAhead) {
    if (s0 > 0) load(s0);
    float top = M;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i)
      if (s0 + i < a.ns) top = fmaxf(top, st[i][0]);
    const float ms = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(M - ms);
    L *= f0;
    SF *= f0;
    x *= f0;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i)
      if (s0 + i < a.ns) {
        const float f = __builtin_amdgcn_exp2f(st[i][0] - ms);
        L += f * st[i][1];
        SF += f * st[i][2];
        x += f * y[i];
      }
    M = top;
  }
  const bool live = first + threadIdx.x / (D / 4) < rows && r >= c.first && r < c.first + c.n && c.n <= a.max_chunk &&
                    base >= 0 && base <= a.map.cap - c.n;
  const float inv = 1.f / L;
  const float mass = L == 0.f ? 0.f : SF * inv;
  if (a.conf != nullptr) {
    const int at = r - (int)(first / a.Hq);  // below join_rows: a token has a row at least
    const bool newest = live && r == c.first + c.n - 1;
    __syncthreads();
    if (d == 0 && newest) atomicMax(best + at, conf_bits(mass));
    __syncthreads();
    // the first thread of the token's first row here
    const bool begins = row == first || row % a.Hq == 0;
    if (d == 0 && newest && begins) atomicMax((int*)a.conf + b, best[at]);
  }
  if (!live) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = L == 0.f ? 0.f : x[e] * inv;
  T* dst = (T*)a.out + row * D + d;
  if constexpr (sizeof(T) == 4)
    *(f32x4*)dst = x;
  else
    *(u32x2_t*)dst = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  if (d == 0) {
    a.lse[row] = L == 0.f ? -INFINITY : kLn2 * (M + __builtin_amdgcn_logf(L));
    if (a.suffix != nullptr) a.suffix[row] = mass;
  }
}

// ------------------------------------------------------------------------------------------
// Plan and launch
// ------------------------------------------------------------------------------------------
struct PagedPlan {
  long many_tiles;  // upper bound over the chunks that `total` rows can be
  int ns;           // splits of a row's slots
  int halves;       // workgroups that share a row's output values (paged_few)
  bool few;         // paged_few
};

// Workgroups for the split of a launch without long chunks: one a CU.
constexpr long kFewTarget = 256;
// Three or four splits (64 pairs of a sequence and a KV head on) take more than two halves without a join up to this many
// slots (bfloat16, head_dim 128: in float32 the scores, which both halves form, bound it). Decode steps of 16 / 20
// sequences, 28 / 4 heads, 1024 slots 12.6 / 13.0 us, split 12.5 / 13.9; 2048 slots 19.1 / 19.5, split 18.3 / 21.0; 3008 slots
// 23.5 / 25.6, split 22.6 / 25.5; 4096 slots 29.5 / 31.0, split 25.5 / 30.3. With fewer pairs the two are within half a
// microsecond at 1024 slots and splits ahead behind that.
constexpr long kHalvesReach = 2560, kHalvesPairs = 64;
// Slots of a split at most, whatever the number of workgroups: what one long sequence among many short ones
// may hold up the launch by. Decode steps of 32 / 8 heads over 65536 slots of capacity, at 8192 / 16384 / 32768
// slots a split / no such bound: 63 sequences of 1000 slots and one of 60000 182 / 219 / 335 / 571 us, 64 sequences
// of 1000 slots 103 / 76 / 65.5 / 48.6 (the capacity is all the host knows).
constexpr long kMaxSplitSlotsPaged = 32768;

// Rows (of a token and a query head) that a launch joins at most: its 256 threads a workgroup must stay below the 2^32 of
// a grid, 8 rows a workgroup at head_dim 128. A larger step has a million workgroups and is not split.
constexpr long kMaxJoinRows = (1l << 27) - 8;

// reach: slots that a token may see, by the capacity and the window.
static PagedPlan paged_plan(const lg_paged_layer& l, const lg_page_map& m, long total, long max_chunk, long reach) {
  const long G = l.n_q_heads / l.n_kv_heads;
  PagedPlan p;
  p.many_tiles = 0;
  p.halves = 1;
  p.few = max_chunk * G <= kWaveRows;
  long ns, slots = kMinSplitSlots;
  if (p.few) {
    const long units = (long)m.batch * l.n_kv_heads;
    ns = kFewTarget / units;  // more than one a CU would run in two rounds
    if (ns > 2 && units >= kHalvesPairs && reach <= kHalvesReach && l.dtype == LG_BF16 && l.head_dim == 128) ns = 2;
  } else {
    if (total * G > kWaveRows) {
      // a sequence of n rows has at most n / 128 + 1 tiles, and more than 32 rows
      p.many_tiles = total * G / kManyRows;
      const long seqs = total * G / (kWaveRows + 1);
      p.many_tiles += seqs < m.batch ? seqs : m.batch;
    }
    const long units = (p.many_tiles + m.batch) * l.n_kv_heads;
    ns = (kPagedTarget + units - 1) / units;
    if (l.dtype == LG_BF16) slots += total * l.n_q_heads / kSplitRows;
  }
  ns = std::min({ns, (reach + slots - 1) / slots, (long)kMaxNs});
  const long least = std::min(reach / kMaxSplitSlotsPaged, (long)kMaxNs);
  if (p.few && ns == 2 && least < 2 && l.head_dim == 128) {
    ns = 1;
    p.halves = 2;
  }
  p.ns = (int)std::max({ns, least, 1l});
  if (total * l.n_q_heads > kMaxJoinRows) p.ns = 1;
  return p;
}

static size_t paged_need(const lg_paged_layer& l, const PagedPlan& p, long total) {
  return p.ns > 1 ? (size_t)p.ns * total * l.n_q_heads * (l.head_dim + 4) * 4 : 0;
}

// Workgroups of the launch (a grid holds fewer than 2^32 threads).
long paged_attend_grid(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk) {
  const PagedPlan p = paged_plan(l, m, total, max_chunk, whole_reach(m));
  return (p.many_tiles + m.batch) * l.n_kv_heads * p.ns * p.halves;
}

size_t paged_attend_need(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk, int window,
                         int n_sink) {
  return paged_need(l, paged_plan(l, m, total, max_chunk, window_reach(m, max_chunk, window, n_sink)), total);
}

// The largest need of any total up to this one and any max_chunk up to this one, with any window (a shorter reach
// has no more splits). For a given number of splits the need grows with total, and the number falls as total
// grows, so the ends of its steps count.
size_t paged_attend_bytes(const lg_paged_layer& l, const lg_page_map& m, int total, int max_chunk) {
  size_t most = 16;
  for (int form = 0; form < 2; ++form) {
    const long chunk = form == 0 ? 1 : max_chunk;
    long t = total;
    while (t > 0) {
      const PagedPlan p = paged_plan(l, m, t, chunk, whole_reach(m));
      const size_t need = paged_need(l, p, t);
      if (need > most) most = need;
      long lo = 0, hi = t;  // the largest smaller total with more splits
      while (hi - lo > 1) {
        const long mid = (lo + hi) / 2;
        if (paged_plan(l, m, mid, chunk, whole_reach(m)).ns > p.ns) lo = mid; else hi = mid;
      }
      t = lo;
    }
  }
  return align_up(most, 16);
}

template <typename T, int D, int KW, int RW>
static void launch_few(const PagedAttendArgs& a, const PagedPlan& p, dim3 grid, hipStream_t st) {
  if (p.halves == 1)
    hipLaunchKernelGGL((paged_few<T, D, KW, D, RW>), grid, dim3(64 * KW), 0, st, a);
  else if constexpr (D == 128)
    hipLaunchKernelGGL((paged_few<T, D, KW, D / 2, RW>), grid, dim3(64 * KW), 0, st, a);
}

template <typename T, int D>
static void launch_typed(const PagedAttendArgs& a, const PagedPlan& p, dim3 grid, hipStream_t st) {
  constexpr int KW = sizeof(T) == 4 && D == 128 ? 4 : 8;
  if (!p.few) {
    hipLaunchKernelGGL((paged_attend<T, D>), grid, dim3(kPagedThreads), 0, st, a);
  } else if (sizeof(T) == 4 && (long)a.max_chunk * a.G <= 16) {
    launch_few<T, D, KW, sizeof(T) == 4 ? 16 : 32>(a, p, grid, st);
  } else {
    launch_few<T, D, KW, 32>(a, p, grid, st);
  }
  const long rows = (long)a.total * a.Hq;
  if (p.ns > 1)
    hipLaunchKernelGGL((paged_join<T, D>), dim3((unsigned)((rows + join_rows<D>() - 1) / join_rows<D>())), dim3(kPagedThreads), 0,
                       st, a);
}

hipError_t launch_paged_attend(const lg_paged_layer& l, const lg_page_map& m, const void* q, void* out,
                               const int32_t* q_start, const int32_t* base, int total, int max_chunk,
                               int window, int n_sink, const int32_t* suffix_w, float* lse, float* suffix,
                               float* conf, void* ws, hipStream_t st) {
  const PagedPlan p = paged_plan(l, m, total, max_chunk, window_reach(m, max_chunk, window, n_sink));
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
  const dim3 grid((unsigned)((p.many_tiles + m.batch) * l.n_kv_heads * p.ns * p.halves));
  if (l.dtype == LG_BF16) {
    if (l.head_dim == 128) launch_typed<__bf16, 128>(a, p, grid, st);
    else launch_typed<__bf16, 64>(a, p, grid, st);
  } else {
    if (l.head_dim == 128) launch_typed<float, 128>(a, p, grid, st);
    else launch_typed<float, 64>(a, p, grid, st);
  }
  return hipGetLastError();
}

}  // namespace lg
