// lg_fp4_attend.hip -- attention of a step's new tokens over 4-bit pages (lg_paged_attend_fp4).
//
// The mathematics, the workgroups' rows and slots and the running maximum are those of lg_paged_attend.hip: a wave takes
// query rows of one KV head of one sequence and walks tiles of slots with
//   S^T = K Q^T,  m' = max(m, max S),  P = 2^(S - m'),  l = l 2^(m - m') + sum P,  O^T = O^T 2^(m - m') + V^T P^T.
// A 4-bit number times its power of two is a bfloat16 number exactly, and one instruction makes two of them. So K
// and V become bfloat16 in registers, and both products are bfloat16 matrix instructions whose products are exact. float32
// queries and weights enter as three bfloat16 terms each (8 + 8 + 8 bits, exact), three times the instructions, still
// a fifth of what float32 ones would take.
//
// What bounds it, measured on MI355X (a copy reaches 5.13 TB/s, plain reads 6.3 and non-temporal ones 7.0, a bfloat16 matrix product
// of 8192^3 1122 TFLOP/s), in a graph: 64 sequences of 5120 to 8192 slots, 32 / 8 heads of 128, 471 MB, 97 us, 4.85 TB/s: loads
// on their way, it seems, since neither the memory is at its reads' rate nor the vector instructions (49% of the cycles) or the
// matrix ones (21%) are busy. A decode step of 32 sequences of 28 / 4
// heads and 1280 to 2047 slots, 30 MB, 13.5 us: its chain and its instructions. The sequence is known after 0.9 us, the first
// rows are asked for after 2.0, the first tile of 32 slots is done after 4.2, and each further one takes a wave 1.2 us beside
// the others of its SIMD (230 vector and 16 matrix instructions, 100 scalar ones); the bytes alone would take 6. 4096 tokens of
// 32 / 8 heads behind 4096, 412 GFLOP, 419 us, 984 TFLOP/s: matrix instructions (42% of the cycles), with the conversions and
// exponentials beside them in part (vector instructions 54%); at head_dim 64 267 us, 771 TFLOP/s, and the vector instructions
// are first (70%, matrix ones 33%); in float32 1075 us, 384 TFLOP/s of exact products. Four sequences of 128 tokens with a window of
// 2048 beside 12 that decode, 44 us: a workgroup's chain, 17 tiles of 2 us with one wave on a SIMD, and the launch that joins two splits.
// 32 sequences of 5 tokens, 35 rows a KV head, 34 us: tiles of 128 rows, of which the last two waves have none.
//
// Tried and left (us, the decode step of 32 sequences / 64 sequences of 8192 slots unless said): tiles two to four ahead in
// registers (16.7 to 17.6 against 15.8 / 103 to 109 against 97: the copies of their registers wait for all of them); the
// exponents of a row in one load, spread by permutes (18.4 / 139); tiles of 64 slots (15.7 against 16.0 / 103 against 101); 4 waves
// a workgroup (18.3 against 16.0). Chunks: the scores of both blocks of 32 keys side by side, or the next tile's conversion among
// them (4096 tokens 510 to 640: registers); two teams of four waves a workgroup that share out the tiles (8 sequences of 128 tokens,
// window 1024, 28.5 against 31.4, the mixed step 51 against 46: one barrier keeps the teams in step); a higher priority for a wave
// in its matrix instructions (4096 tokens 422 to 426 against 425, in float32 1105 to 1153 against 1084) or in its exponentials (432); all
// exponentials before the second product (433); a maximum for each 32 keys, so that the second scores run beside the first
// exponentials (445 against 434, with the scheduler's order forced 452 to 463).
#include "lg_fp4.h"
#include "lg_paged_attend.h"

namespace lg {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------------
// Terms
// ------------------------------------------------------------------------------------------
// Terms of a query, and of a weight in steps of few rows and in chunks (see lg_paged_attend.hip for bfloat16 calls' one
// and two).
template <typename T> constexpr int q_terms() { return sizeof(T) == 4 ? 3 : 1; }
template <typename T, bool FEW> constexpr int p_terms() { return sizeof(T) == 4 ? 3 : FEW ? 2 : 1; }

// Two weights as N bfloat16 terms, each what the ones before leave, to nearest: with two within 2^-16, with three exact.
template <int N>
__device__ __forceinline__ void weight_terms(float x, float y, uint32_t (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    t[i] = pack_bf16(x, y);
    if (i + 1 < N) {
      x -= __uint_as_float(t[i] << 16);
      y -= __uint_as_float(t[i] & 0xffff0000u);
    }
  }
}

// 8 values of a query as they lie, and as N terms. float32: cut off after 8 and 16 bits, so that no term is larger than the
// value; one that is not finite is its first term alone.
template <typename T>
struct Eight {
  u32x4_t x[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T* src) {
  Eight<T> y;
  y.x[0] = *(const u32x4_t*)src;
  if constexpr (sizeof(T) == 4) y.x[1] = *(const u32x4_t*)(src + 4);
  return y;
}
template <typename T, int N>
__device__ __forceinline__ void query_terms(const Eight<T>& q, u32x4_t (&t)[N]) {
  if constexpr (N == 1) {
    t[0] = q.x[0];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[N] = {};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float y = __uint_as_float(q.x[i / 2][2 * (i % 2) + e]);
        const bool finite = (__float_as_uint(y) & 0x7f800000u) != 0x7f800000u;
        if (!finite) {
          w[0] |= (pack_bf16(y, y) & 0xffffu) << (16 * e);
        } else {
#pragma unroll
          for (int n = 0; n < N; ++n) {
            const uint32_t top = __float_as_uint(y) & 0xffff0000u;
            w[n] |= e == 0 ? top >> 16 : top;
            y -= __uint_as_float(top);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < N; ++n) t[n][i] = w[n];
    }
  }
}

// 8 values of a word of codes as bfloat16.
__device__ __forceinline__ u32x4_t decode(uint32_t codes, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3);
  return u32x4_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                 __builtin_bit_cast(uint32_t, d)};
}

__device__ __forceinline__ f32x4 mfma16(u32x4_t a, u32x4_t b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(u32x4_t a, u32x4_t b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 4 keys x 16 values of bfloat16 in LDS, a lane 4 values of a key; each lane gets one value of 4 keys.
__device__ __forceinline__ u32x2_t read_turned(const char* at) {
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
}

// The larger one, NaN if one is (a row with such a score is NaN whatever its maximum), which takes no instruction to make
// its operands canonical.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// ------------------------------------------------------------------------------------------
// Tiles
// ------------------------------------------------------------------------------------------
// A value at an offset of at most 32 bits in bytes: the base stays in scalar registers.
template <typename X>
__device__ __forceinline__ X at32(const X* base, unsigned off) { return *(const X*)((const char*)base + off); }

struct Look {
  int page, pos;
};

// An entry, by way of the scalar cache, of an array that nothing writes while the kernel reads it.
__device__ __forceinline__ int of_all(const int32_t* x, int at) {
  return ((const __attribute__((address_space(4))) int32_t*)x)[__builtin_amdgcn_readfirstlane(at)];
}

// The slots of a workgroup's rows in tiles of NK.
template <int NK>
struct Walk {
  const PagedAttendArgs& a;
  const Job& job;
  const int32_t *table, *pos;
  int last_slot;  // the last one that any of the rows sees; what is read of slots behind it is read of this one

  __device__ __forceinline__ int slot_of(int t) const { return (t < job.sink_tiles ? t : t - job.sink_tiles + job.tile0) * NK; }
  // The page of a slot that all lanes ask for: scalar loads are counted apart from the rows', which return in order, so it
  // is there before the rows that were asked for first.
  __device__ __forceinline__ int page_of(int slot) const { return of_all(table, min(slot, last_slot) >> a.map.shift); }
  // Page and position of the lane's slot of a tile.
  __device__ __forceinline__ Look look(int t) const {
    const unsigned s = min(slot_of(min(t, job.t_end - 1)) + ((int)threadIdx.x & (NK - 1)), last_slot);  // below 2^30
    return {at32(table, 4 * (s >> a.map.shift)), at32(pos, 4 * s)};
  }
  __device__ __forceinline__ int pos_of_lane(int s0) const {  // slots are below 2^30
    return at32(pos, 4u * (unsigned)min(s0 + ((int)threadIdx.x & (NK - 1)), last_slot));
  }
};

// Where a page of the workgroup's KV head lies in K or V (a page that is none: page 0). Blocks have at least 544 bytes, so
// their numbers stay below 2^32 in any memory.
template <int D>
__device__ __forceinline__ size_t block_at(const PagedAttendArgs& a, const Job& job, int page) {
  const unsigned n = (unsigned)(is_page(a.map, page) ? page : 0) * (unsigned)a.Hkv + (unsigned)job.h;
  return (size_t)n * (unsigned)fp4_block(D, a.map.shift);
}

// What a row of the wave sees: slots up to its own, at positions above win or below n_sink; it counts those above
// suf as its suffix.
struct Sight {
  int slot, win, suf;
};
__device__ __forceinline__ Sight sight_of(const PagedAttendArgs& a, int slot, int p, int sw) {
  Sight s;
  s.slot = slot;
  s.win = a.window > 0 ? (int)max((long long)p - a.window, (long long)INT32_MIN) : INT32_MIN;
  s.suf = (int)max((long long)p - max(sw, 0), (long long)INT32_MIN);
  return s;
}

__device__ __forceinline__ bool sees(const PagedAttendArgs& a, const Sight& s, int slot, int p) {
  return slot <= s.slot && p != kHidden && (a.window == 0 || p > s.win || p < a.n_sink);
}

// How a tile of NK slots from s0 on, with the lane's slot at position tp, is to be compared: whether some row may not
// see a slot (lo, hi: the first and the last row), and what it has of the suffix.
enum { kNone, kAll, kSome };
struct Compare {
  bool masked;
  int suffix;
};
template <int NK>
__device__ __forceinline__ Compare compare_of(const PagedAttendArgs& a, int tp, int s0, const Sight& lo, const Sight& hi) {
  const int p_first = __builtin_amdgcn_readlane(tp, 0), p_last = __builtin_amdgcn_readlane(tp, NK - 1);
  Compare c;
  c.masked = __ballot(tp == kHidden) != 0 || s0 + NK - 1 > lo.slot || (a.window > 0 && p_first <= hi.win && p_last >= a.n_sink);
  // kHidden in front says nothing about the slots behind it
  c.suffix = p_last <= lo.suf ? kNone : p_first > hi.suf && p_first != kHidden ? kAll : kSome;
  if (a.suffix == nullptr && a.conf == nullptr) c.suffix = kNone;
  return c;
}

// LDS of a wave beside its tiles: 64 bounds (a row sees slot j if bound_j > win and the slot is none behind its own), 64
// positions.
constexpr int kNotes = 512;
__device__ __forceinline__ void note(const PagedAttendArgs& a, int32_t* notes, int tp) {
  const int lane = threadIdx.x & 63;
  notes[lane] = tp == kHidden ? INT32_MIN : a.window == 0 || tp < a.n_sink ? INT32_MAX : tp;
  notes[64 + lane] = tp;
}

// ------------------------------------------------------------------------------------------
// Few rows
// ------------------------------------------------------------------------------------------
// At most 16 NR query rows of a sequence (a decode step: G rows), KW waves that take every KW-th tile of 32 slots each,
// with no barrier until their (m, l, O) are joined. Matrix instructions of 16 rows: a lane holds 4 of every 16 keys of ONE
// row, the four lanes of a row are 16 apart. K comes from memory as the first product's operand: the order of the
// dimensions in a product is free, so a lane takes a quarter of its key's row as it lies (with 128 dimensions, one
// group). V passes through LDS as bfloat16 and is read transposed.
constexpr int kFewKeys = 32;

template <int DV, int NR>
struct Few {
  static constexpr int kTile = kFewKeys * DV * 2;
  static constexpr int kStat = 16 * NR * (DV + 4);  // floats of a wave's O, [row][DV + 4], before its m, l, suffix sums
  static constexpr int kJoin = (kStat + 3 * 16 * NR) * 4;
  static constexpr int kLds = ((kTile + kNotes > kJoin ? kTile + kNotes : kJoin) + 255) & ~255;
  // 16-byte pieces of a row of V lie in the order piece ^ turn(row): the 4 rows that 16 lanes write and the 8 rows of 32
  // bytes that 32 lanes read then lie in different banks.
  static __device__ __forceinline__ int turn(int row) {
    return DV == 128 ? 2 * (row & 7) | ((row >> 1) & 1) : 2 * ((row >> 1) & 3) | ((row >> 2) & 1);
  }
};

template <typename T, int D, int KW, int DV, int NR>
__device__ __forceinline__ void few_body(const PagedAttendArgs& a, Job job, char* lds) {
  using C = Few<DV, NR>;
  constexpr int NK = kFewKeys;
  constexpr int QT = q_terms<T>(), PT = p_terms<T, true>();
  constexpr int NJ = NK / 16, NKK = D / 32, ND = DV / 16;
  constexpr int RB = D / 2, EB = D / 32;    // bytes of a row and of its exponents
  constexpr int VP = DV / 32, VU = NK * VP / 64;  // groups of a row of V, and of them a lane's
  constexpr int RBV = 2 * DV;
  using KRow = std::conditional_t<D == 128, u32x4_t, u32x2_t>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = lane >> 4, col = lane & 15;
  char* const my = lds + wave * C::kLds;
  int32_t* const notes = (int32_t*)(my + C::kTile);
  const int ps = 1 << a.map.shift;
  const Walk<NK> walk = {a, job, a.map.table + (size_t)job.b * a.map.P, a.map.pos + (size_t)job.b * a.map.cap,
                         job.base + (job.rows - 1) / a.G};
  const int32_t* const pos = walk.pos;
  const int last_slot = walk.last_slot;

  // What the first rows need comes first; everything else is asked for behind it and used when they are on their way.
  skip_hidden<NK>(a, job, pos);
  const int t_first = job.t_begin + wave;
  const bool some = t_first < job.t_end;
  f32x4 O[NR][ND];
  float mx[NR], l[NR], sfx[NR];  // l and sfx: the lane's share of the keys
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int d = 0; d < ND; ++d) O[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    mx[n] = -INFINITY;
    l[n] = sfx[n] = 0.f;
  }

  // The pages of a tile: of its first 16 slots, and where a page is 16 slots of the others.
  struct Pages {
    int first, second;
  };
  const bool short_pages = ps == 16;
  auto pages_of = [&](int t) __attribute__((always_inline)) {
    const int s0 = walk.slot_of(min(t, job.t_end - 1));
    Pages p = {walk.page_of(s0), 0};
    if (short_pages) p.second = walk.page_of(s0 + 16);
    return p;
  };
  // A tile as it lies in memory, the lane's pieces with their exponents.
  struct Raw {
    KRow k[NJ];
    u32x4_t v[VU];
    uint32_t ke[NJ], ve[VU];
    int pos;
    Pages pages;
  };
  // Rows behind last_slot are read as that one.
  auto load = [&](int t, const Pages& p) __attribute__((always_inline)) {
    Raw raw;
    const int s0 = walk.slot_of(t), most = last_slot - s0;
    // Rows from 16 on lie in the second page where a page is 16 slots.
    const bool two = short_pages && most >= 16;
    const size_t first = block_at<D>(a, job, p.first), second = two ? block_at<D>(a, job, p.second) : first;
    const int row0 = s0 & (ps - 1), row1 = two ? -16 : row0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const unsigned row = min(16 * j + col, most) + (j == 0 ? row0 : row1);
      const char* at = (const char*)a.k + (j == 0 ? first : second);
      raw.k[j] = at32((const KRow*)at, row * RB + part * (RB / 4));
      raw.ke[j] = at32((const uint8_t*)at, ps * RB + row * EB + (D == 128 ? part : part >> 1));
    }
#pragma unroll
    for (int u = 0; u < VU; ++u) {
      const bool later = VP == 4 ? u == 1 : lane >= 32;
      const unsigned row = min(lane / VP + u * (64 / VP), most) + (later ? row1 : row0);
      const char* at = (const char*)a.v + (later ? second : first);
      raw.v[u] = at32((const u32x4_t*)at, row * RB + job.d0 / 2 + lane % VP * 16);
      raw.ve[u] = at32((const uint8_t*)at, ps * RB + row * EB + job.d0 / 32 + lane % VP);
    }
    raw.pos = walk.pos_of_lane(s0);
    raw.pages = p;
    return raw;
  };
  Pages next = {};
  Raw raw = {};
  if (some) next = pages_of(t_first);
  Eight<T> query[NR][NKK];
  int slot_q[NR], p_q[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int R = min(16 * n + col, job.rows - 1), tok = R / a.G;  // rows behind the last repeat it; they are not written
    const T* src = (const T*)a.q + ((size_t)(job.first + tok) * a.Hq + job.h * a.G + R - tok * a.G) * D + part * (D / 4);
#pragma unroll
    for (int k = 0; k < NKK; ++k) query[n][k] = load_eight(src + 8 * k);
    slot_q[n] = job.base + tok;
    p_q[n] = pos[slot_q[n]];
  }
  const int p_lo = of_all(pos, job.base), p_hi = of_all(pos, last_slot);
  const int sw = of_all(a.suffix_w != nullptr ? a.suffix_w : a.base, job.b);  // without suffix_w nothing goes by it
  if (some) {
    raw = load(t_first, next);
    if (t_first + KW < job.t_end) next = pages_of(t_first + KW);
  }
  u32x4_t qf[NR][NKK][QT];
  Sight sight[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int k = 0; k < NKK; ++k) query_terms<T, QT>(query[n][k], qf[n][k]);
    sight[n] = sight_of(a, slot_q[n], p_q[n], sw);
  }
  // the first and the last row's
  const Sight lo = sight_of(a, job.base, p_lo, sw), hi = sight_of(a, last_slot, p_hi, sw);

  const int v_row = lane / VP, v_write = v_row * RBV, v_turn = C::turn(v_row);
  const int k_row = 4 * part + (col >> 2);
  const char* const v_read = my + k_row * RBV + 16 * (((col & 3) >> 1) ^ C::turn(k_row)) + 8 * (col & 1);

  // A tile up to its scores, which is when its rows are not needed any more.
  f32x4 S[NR][NJ];
  int s0, tp;
  auto begin = [&](int t, const Raw& raw) __attribute__((always_inline)) {
    s0 = walk.slot_of(t);
    tp = is_page(a.map, short_pages && (lane & 16) != 0 ? raw.pages.second : raw.pages.first) ? raw.pos : kHidden;
    // V as bfloat16
#pragma unroll
    for (int u = 0; u < VU; ++u) {
      u32x4_t codes = raw.v[u];
      const bool nan = raw.ve[u] > 252;
      if (__any(nan)) {
        // Groups that stand for NaN: 0 in the product, and NaN in their 32 values of the rows that see the slot.
        if (nan) codes = u32x4_t{0, 0, 0, 0};
        for (unsigned long long left = __ballot(nan); left != 0; left &= left - 1) {
          const int bit = __builtin_ctzll(left), key = bit / VP + u * (64 / VP), g = bit % VP;
          const int p = __builtin_amdgcn_readlane(tp, key);
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const bool see = sees(a, sight[n], s0 + key, p);
#pragma unroll
            for (int d = 0; d < ND; ++d)
              if (d / 2 == g && see) O[n][d] = f32x4{NAN, NAN, NAN, NAN};
          }
        }
      }
      const float unit = fp4_unit(nan ? 127 : raw.ve[u]);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        *(u32x4_t*)(my + u * (64 / VP) * RBV + v_write + 16 * ((4 * (lane % VP) + w) ^ v_turn)) = decode(codes[w], unit);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float unit = fp4_unit(raw.ke[j]);
#pragma unroll
      for (int n = 0; n < NR; ++n) S[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < NKK; ++k) {
        const u32x4_t x = decode(raw.k[j][k], unit);
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int i = 0; i < QT; ++i) S[n][j] = mfma16(x, qf[n][k][i], S[n][j]);
      }
    }
  };
  auto finish = [&]() __attribute__((always_inline)) {
    const Compare is = compare_of<NK>(a, tp, s0, lo, hi);
    if (is.masked || is.suffix == kSome) note(a, notes, tp);
    if (is.masked) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const i32x4 bound = *(const i32x4*)(notes + 16 * j + 4 * part);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const int last = sight[n].slot - s0 - 16 * j - 4 * part;
#pragma unroll
          for (int i = 0; i < 4; ++i) S[n][j][i] = bound[i] > sight[n].win && i <= last ? S[n][j][i] : -INFINITY;
        }
      }
    }
    uint32_t P[NR][NK / 32][4][PT];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float top = larger(larger(S[n][0][0], S[n][0][1]), larger(S[n][0][2], S[n][0][3]));
#pragma unroll
      for (int j = 1; j < NJ; ++j) top = larger(larger(top, S[n][j][0]), larger(larger(S[n][j][1], S[n][j][2]), S[n][j][3]));
      top = larger(top, other_row(top));
      top = larger(top, other_half(top)) * a.scale_log2;
      // The running maximum follows only when a score passes it by kSlack (weights are then at most 2^kSlack).
      const bool raise = top > mx[n] + kSlack;
      if (__any(raise)) {
        const float f = raise ? __builtin_amdgcn_exp2f(mx[n] - top) : 1.f;  // 0 where nothing was seen before
        mx[n] = raise ? top : mx[n];
        l[n] *= f;
        sfx[n] *= f;
#pragma unroll
        for (int d = 0; d < ND; ++d) O[n][d] *= f;
      }
      const float off = mx[n] == -INFINITY ? 0.f : -mx[n];
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) S[n][j][i] = __builtin_amdgcn_exp2f(fmaf(S[n][j][i], a.scale_log2, off));
        sum += (S[n][j][0] + S[n][j][1]) + (S[n][j][2] + S[n][j][3]);
#pragma unroll
        for (int i = 0; i < 2; ++i) weight_terms<PT>(S[n][j][2 * i], S[n][j][2 * i + 1], P[n][j / 2][2 * (j & 1) + i]);
      }
      l[n] += sum;
      sfx[n] += is.suffix == kAll ? sum : 0.f;
      if (is.suffix == kSome) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const i32x4 p = *(const i32x4*)(notes + 64 + 16 * j + 4 * part);
#pragma unroll
          for (int i = 0; i < 4; ++i) sfx[n] += p[i] > sight[n].suf ? S[n][j][i] : 0.f;
        }
      }
    }
    // O^T += V^T P^T: the lane's keys of a product are 4 part .. and 16 + 4 part ..
#pragma unroll
    for (int s = 0; s < NK / 32; ++s)
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const char* at = my + (((int)(v_read - my) + 32 * s * RBV) ^ (32 * d));
        const u32x2_t x = read_turned(at), y = read_turned(at + 16 * RBV);
        const u32x4_t z = {x[0], x[1], y[0], y[1]};
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int i = 0; i < PT; ++i)
            O[n][d] = mfma16(z, u32x4_t{P[n][s][0][i], P[n][s][1][i], P[n][s][2][i], P[n][s][3][i]}, O[n][d]);
      }
  };

  for (int t = t_first; t < job.t_end; t += KW) {
    begin(t, raw);
    if (t + KW < job.t_end) raw = load(t + KW, next);
    if (t + 2 * KW < job.t_end) next = pages_of(t + 2 * KW);
    finish();
  }

  // Join the waves: their numerators and statistics through LDS.
  constexpr int kRows = 16 * NR, kShare = 64 * KW / kRows, kParts = kShare < DV / 2 ? kShare : DV / 2;  // threads a row
  constexpr int kPairs = DV / (2 * kParts);
  float* const num = (float*)my;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    l[n] += other_row(l[n]);
    l[n] += other_half(l[n]);
    sfx[n] += other_row(sfx[n]);
    sfx[n] += other_half(sfx[n]);
#pragma unroll
    for (int d = 0; d < ND; ++d) *(f32x4*)(num + (16 * n + col) * (DV + 4) + 16 * d + 4 * part) = O[n][d];
    if (part == 0) {
      num[C::kStat + 16 * n + col] = mx[n];
      num[C::kStat + kRows + 16 * n + col] = l[n];
      num[C::kStat + 2 * kRows + 16 * n + col] = sfx[n];
    }
  }
  __syncthreads();
  auto row_of = [&](int r) __attribute__((always_inline)) {
    const int tk = r / a.G;
    return (size_t)(job.first + tk) * a.Hq + job.h * a.G + (r - tk * a.G);
  };
  const size_t split0 = (size_t)job.split * a.total * a.Hq;
  if (wave == KW - 1 && job.d0 == 0) {  // the statistics, a lane a row
    const int r = min(lane, job.rows - 1);
    float M = -INFINITY, L = 0.f, SF = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) M = fmaxf(M, ((const float*)(lds + w * C::kLds))[C::kStat + r]);
    const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float* src = (const float*)(lds + w * C::kLds) + C::kStat + r;
      const float f = __builtin_amdgcn_exp2f(src[0] - Ms);
      L += f * src[kRows];
      SF += f * src[2 * kRows];
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
    wm[w] = ((const float*)(lds + w * C::kLds))[C::kStat + r];
    M = fmaxf(M, wm[w]);
  }
  const float Ms = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  f32x2 x[kPairs] = {};
#pragma unroll
  for (int w = 0; w < KW; ++w) {
    const float* src = (const float*)(lds + w * C::kLds);
    const float f = __builtin_amdgcn_exp2f(wm[w] - Ms);
    L += f * src[C::kStat + kRows + r];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) x[i] += f * *(const f32x2*)(src + r * (DV + 4) + 2 * (kParts * i + share));
  }
  const size_t row = row_of(r);
  if (a.ns > 1) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) *(f32x2*)(a.po + (split0 + row) * D + job.d0 + 2 * (kParts * i + share)) = x[i];
    return;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;  // without weight x is 0, or NaN by a group that stands for it
  T* dst = (T*)a.out + row * D + job.d0;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const float y0 = x[i][0] * inv, y1 = x[i][1] * inv;
    if constexpr (sizeof(T) == 4)
      *(f32x2*)(dst + 2 * (kParts * i + share)) = f32x2{y0, y1};
    else
      *(uint32_t*)(dst + 2 * (kParts * i + share)) = pack_bf16(y0, y1);
  }
}

// ------------------------------------------------------------------------------------------
// Many rows
// ------------------------------------------------------------------------------------------
// 128 query rows of a sequence, four waves of 32, which share every tile of 64 slots: a thread brings a quarter of a row of
// K and of V as bfloat16 to LDS, while the tile before is multiplied (two buffers, one barrier a tile). From there on it is
// the bfloat16 kernel's walk, in its layout but for V's turn.
constexpr int kManyKeys = 64;

template <int D>
struct Many {
  static constexpr int kRow = 2 * D, kTile = kManyKeys * kRow, kBuffer = 2 * kTile;
  static constexpr int kFlags = 2 * kBuffer;  // a byte a quarter of a row of V, two buffers: it stands for NaN
  static constexpr int kOwnNotes = kFlags + 2 * 256;
  static constexpr int kLds = kOwnNotes + 4 * kNotes;
  // 16-byte pieces of a row lie in the order piece ^ turn(row): K for the 16 rows of a read, V for the 4 rows (of 64 bytes)
  // of a transposed one, both also for the 4 rows that 16 lanes write.
  static __device__ __forceinline__ int turn_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
  static __device__ __forceinline__ int turn_v(int row) { return 5 * (D == 128 ? row & 3 : (row >> 1) & 1); }
};

// Order for the scheduler: the 8 reads of LDS and 8 matrix instructions of a tile's scores at head_dim 64, the reads 4 ahead
// (4096 tokens behind 4096, 32 / 8 heads: 298 us left to itself, 280 so; at head_dim 128 431 and 435, in float32 1081 and
// 1123).
__device__ __forceinline__ void schedule_scores_64() {
  __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);  // reads of LDS
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix instructions
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
}

template <typename T, int D>
__device__ __forceinline__ void many_body(const PagedAttendArgs& a, Job job, char* lds) {
  using C = Many<D>;
  constexpr int QT = q_terms<T>(), PT = p_terms<T, false>();
  constexpr int NK = kManyKeys, ND = D / 32, RB = D / 2, EB = D / 32, RBV = C::kRow;
  using Quarter = std::conditional_t<D == 128, u32x4_t, u32x2_t>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = lane >> 5, col = lane & 31;
  int32_t* const notes = (int32_t*)(lds + C::kOwnNotes + wave * kNotes);
  const int ps = 1 << a.map.shift;
  const Walk<NK> walk = {a, job, a.map.table + (size_t)job.b * a.map.P, a.map.pos + (size_t)job.b * a.map.cap,
                         job.base + (min(job.row0 + kManyRows, job.rows) - 1) / a.G};
  const int32_t* const pos = walk.pos;
  const int last_slot = walk.last_slot;

  const int wrow0 = job.row0 + wave * kWaveRows;
  const int R = wrow0 + col;
  const bool live = R < job.rows, idle = wrow0 >= job.rows;  // a wave without rows only loads
  const int Rc = live ? R : job.rows - 1, tok = Rc / a.G;    // rows behind the last repeat it; they are not written
  const size_t qrow = (size_t)(job.first + tok) * a.Hq + job.h * a.G + Rc - tok * a.G;
  u32x4_t qf[D / 16][QT];
#pragma unroll
  for (int k = 0; k < D / 16; ++k) query_terms<T, QT>(load_eight((const T*)a.q + qrow * D + 16 * k + 8 * part), qf[k]);
  const Sight sight = sight_of(a, job.base + tok, pos[job.base + tok], a.suffix_w != nullptr ? a.suffix_w[job.b] : 0);
  skip_hidden<NK>(a, job, pos);
  // bounds over the wave's rows (tokens ascend with the row, positions with the token)
  const auto row_of = [&](int lane_of) __attribute__((always_inline)) {
    return Sight{__builtin_amdgcn_readlane(sight.slot, lane_of), __builtin_amdgcn_readlane(sight.win, lane_of),
                 __builtin_amdgcn_readlane(sight.suf, lane_of)};
  };
  const Sight lo = row_of(0), hi = row_of(31);

  f32x16 O[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[d][i] = 0.f;
  float mx = -INFINITY, l = 0.f, sfx = 0.f;

  // The thread's quarter of a row: wave w brings rows 16 w .. of one page.
  struct Raw {
    Quarter k, v;
    uint32_t ke, ve;
  };
  const int in = lane >> 2, quarter = lane & 3;
  auto load = [&](int t, const Look& lk) __attribute__((always_inline)) {
    const int s0 = min(walk.slot_of(t) + 16 * wave, last_slot & ~15);  // rows behind last_slot repeat it
    const size_t at = block_at<D>(a, job, __builtin_amdgcn_readlane(lk.page, 16 * wave));
    const unsigned row = (s0 & (ps - 1)) + min(in, last_slot - s0);
    const unsigned off = row * RB + quarter * (RB / 4), ea = ps * RB + row * EB + (D == 128 ? quarter : quarter >> 1);
    const char *k = (const char*)a.k + at, *v = (const char*)a.v + at;
    return Raw{at32((const Quarter*)k, off), at32((const Quarter*)v, off), at32((const uint8_t*)k, ea), at32((const uint8_t*)v, ea)};
  };
  const int w_row = 16 * wave + in, w_at = w_row * RBV;
  auto store = [&](const Raw& raw, int buffer, char* __restrict__ to) __attribute__((always_inline)) {
    const float uk = fp4_unit(raw.ke);
    const bool odd = raw.ve > 252;  // counts as 0 in the product; see below
    const float uv = fp4_unit(odd ? 127 : raw.ve);
    char* const base = to + buffer * C::kBuffer + w_at;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      const int piece = D / 32 * quarter + w;
      *(u32x4_t*)(base + 16 * (piece ^ C::turn_k(w_row))) = decode(raw.k[w], uk);
      *(u32x4_t*)(base + C::kTile + 16 * (piece ^ C::turn_v(w_row))) = decode(odd ? 0 : raw.v[w], uv);
    }
    to[C::kFlags + 256 * buffer + 4 * w_row + quarter] = odd;
  };

  // The lane's first addresses in a tile.
  const int kx = col * RBV + 16 * (part ^ C::turn_k(col));
  const int v_row = 4 * part + ((lane & 15) >> 2);
  const int vx = v_row * RBV + 16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ C::turn_v(v_row)) + 8 * (lane & 1);

  auto scores = [&](const char* from, int k, f32x16& S) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
    for (int u = 0; u < D / 16; ++u) {
      const u32x4_t x = *(const u32x4_t*)(from + ((k + kx) ^ (32 * u)));
#pragma unroll
      for (int i = 0; i < QT; ++i) S = mfma32(x, qf[u][i], S);
    }
  };
  auto top = [&](const f32x16& S) __attribute__((always_inline)) {
    float t4[4] = {S[0], S[1], S[2], S[3]};
#pragma unroll
    for (int i = 4; i < 16; ++i) t4[i & 3] = larger(t4[i & 3], S[i]);
    const float x = larger(larger(t4[0], t4[1]), larger(t4[2], t4[3]));
    return larger(x, other_half(x));
  };
  auto mask = [&](f32x16& S, int s0, int nb) __attribute__((always_inline)) {
    const int last = sight.slot - s0 - 32 * nb - 4 * part;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const i32x4 bound = *(const i32x4*)(notes + 32 * nb + 8 * i + 4 * part);
#pragma unroll
      for (int j = 0; j < 4; ++j) S[4 * i + j] = bound[j] > sight.win && 8 * i + j <= last ? S[4 * i + j] : -INFINITY;
    }
  };
  auto raise_max = [&](float most) __attribute__((always_inline)) {
    const float tmax = most * a.scale_log2;
    const bool raise = tmax > mx + kSlack;
    if (__any(raise)) {
      const float f = raise ? __builtin_amdgcn_exp2f(mx - tmax) : 1.f;
      mx = raise ? tmax : mx;
      l *= f;
      sfx *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[d][i] *= f;
    }
  };
  auto weights = [&](f32x16& S) __attribute__((always_inline)) {
    float s4[4];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      S[i] = __builtin_amdgcn_exp2f(fmaf(S[i], a.scale_log2, mx == -INFINITY ? 0.f : -mx));
      s4[i & 3] = i < 4 ? S[i] : s4[i & 3] + S[i];
    }
    return (s4[0] + s4[1]) + (s4[2] + s4[3]);
  };
  auto add_suffix = [&](const f32x16& P, int nb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const i32x4 p = *(const i32x4*)(notes + 64 + 32 * nb + 8 * i + 4 * part);
#pragma unroll
      for (int j = 0; j < 4; ++j) sfx += p[j] > sight.suf ? P[4 * i + j] : 0.f;
    }
  };
  auto product = [&](const char* from, int v, const f32x16& P) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint32_t p[4][PT];
#pragma unroll
      for (int e = 0; e < 4; ++e) weight_terms<PT>(P[8 * s + 2 * e], P[8 * s + 2 * e + 1], p[e]);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const char* at = from + ((v + vx) ^ (64 * d)) + 16 * s * RBV;
        const u32x2_t x = read_turned(at), y = read_turned(at + 8 * RBV);
        const u32x4_t z = {x[0], x[1], y[0], y[1]};
#pragma unroll
        for (int i = 0; i < PT; ++i) O[d] = mfma32(z, u32x4_t{p[0][i], p[1][i], p[2][i], p[3][i]}, O[d]);
      }
    }
  };
  // Tile t from its buffer, while the next one's rows go to the other buffer. The two are pointers that do not alias: the
  // reads need not wait for the writes.
  auto tile = [&](int t, int buffer, int tp, const Raw& raw, const char* __restrict__ from, char* __restrict__ to) __attribute__((always_inline)) {
    const uint32_t flags = *(const uint32_t*)(from + C::kFlags + 256 * buffer + 4 * lane);
    if (t + 1 < job.t_end) store(raw, buffer ^ 1, to);
    const int s0 = walk.slot_of(t);
    if (idle || s0 > hi.slot) return;
    const int here = buffer * C::kBuffer;
    constexpr int kBlock = 32 * RBV;
    const Compare is = compare_of<NK>(a, tp, s0, lo, hi);
    if (is.masked || is.suffix == kSome) note(a, notes, tp);
    unsigned long long odd = __ballot(flags != 0);
    for (; odd != 0; odd &= odd - 1) {  // values that stand for NaN: in their 32 values of the rows that see the slot
      const int key = __builtin_ctzll(odd);
      const uint32_t f = __builtin_amdgcn_readlane(flags, key);
      if (sees(a, sight, s0 + key, __builtin_amdgcn_readlane(tp, key))) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
          if (D == 128 ? f >> (8 * d) & 1 : f >> (16 * d) & 1) {
#pragma unroll
            for (int i = 0; i < 16; ++i) O[d][i] = NAN;
          }
      }
    }
    f32x16 S, S1;
    scores(from, here, S);
    scores(from, here + kBlock, S1);
    if constexpr (D == 64 && QT == 1) schedule_scores_64();
    if (is.masked) {
      mask(S, s0, 0);
      mask(S1, s0, 1);
    }
    raise_max(larger(top(S), top(S1)));
    float sum = weights(S);
    product(from, here + C::kTile, S);
    sum += weights(S1);
    product(from, here + C::kTile + kBlock, S1);
    l += sum;
    sfx += is.suffix == kAll ? sum : 0.f;
    if (is.suffix == kSome) {
      add_suffix(S, 0);
      add_suffix(S1, 1);
    }
  };
  if (job.t_begin < job.t_end) {
    Look l0 = walk.look(job.t_begin), l1 = walk.look(job.t_begin + 1);
    Raw raw = load(job.t_begin, l0);
    store(raw, 0, lds);
    raw = load(min(job.t_begin + 1, job.t_end - 1), l1);
    Look l2 = walk.look(job.t_begin + 2);
    for (int t = job.t_begin; t < job.t_end; ++t) {
      __syncthreads();  // every wave has written this tile, and has read the one before
      const Raw now = raw;
      if (t + 2 < job.t_end) raw = load(t + 2, l2);
      const Look l3 = walk.look(t + 3);
      tile(t, (t - job.t_begin) & 1, is_page(a.map, l0.page) ? l0.pos : kHidden, now, lds, lds);
      l0 = l1;
      l1 = l2;
      l2 = l3;
    }
  }
  if (idle) return;
  l += other_half(l);
  sfx += other_half(sfx);
  const float inv = l == 0.f ? 0.f : 1.f / l;  // without weight O is 0, or NaN by a group that stands for it
  const float mass = sfx * inv;
  if (a.ns == 1 && a.conf != nullptr) raise_conf(a.conf + job.b, mass, tok == job.rows / a.G - 1);
  if (!live) return;
  if (a.ns > 1) {
    const size_t at = (size_t)job.split * a.total * a.Hq + qrow;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(a.po + at * D + 32 * d + 8 * i + 4 * part) = f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
    if (part == 0) *(f32x4*)(a.pml + at * 4) = f32x4{mx, l, sfx, 0.f};
    return;
  }
  T* dst = (T*)a.out + qrow * D;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = O[d][4 * i + e] * inv;
      if constexpr (sizeof(T) == 4)
        *(f32x4*)(dst + 32 * d + 8 * i + 4 * part) = f32x4{x[0], x[1], x[2], x[3]};
      else
        *(u32x2_t*)(dst + 32 * d + 8 * i + 4 * part) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    }
  if (part == 0) {
    a.lse[qrow] = l == 0.f ? -INFINITY : kLn2 * (mx + __builtin_amdgcn_logf(l));
    if (a.suffix != nullptr) a.suffix[qrow] = mass;
  }
}

// ------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------
constexpr int kSideWaves = 4;  // waves for a sequence of few rows beside long chunks

template <int D>
constexpr int attend_lds() {
  constexpr int few = kSideWaves * Few<D, 2>::kLds;
  return Many<D>::kLds > few ? Many<D>::kLds : few;
}

// Grid: (Hkv, ns, many_tiles + B), flattened with the KV head fastest, the tiles of many rows first.
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads, sizeof(T) == 4 ? 1 : 2) void fp4_attend(PagedAttendArgs a) {
  __shared__ __align__(512) char lds[attend_lds<D>()];
  const int per = a.Hkv * a.ns;
  const int unit = blockIdx.x / per, rest = blockIdx.x % per;
  Job job;
  job.h = rest % a.Hkv;
  job.d0 = 0;
  const int split = rest / a.Hkv;
  if (unit < a.many_tiles) {
    if (!many_job(a, job, unit)) return;
    job_tiles<kManyKeys>(a, job, kManyRows, split);
    many_body<T, D>(a, job, lds);
    return;
  }
  if (!few_job(a, job, unit - a.many_tiles, rest == 0)) return;
  job_tiles<kFewKeys>(a, job, kWaveRows, split);
  if (job.rows <= 16)
    few_body<T, D, kSideWaves, D, 1>(a, job, lds);
  else
    few_body<T, D, kSideWaves, D, 2>(a, job, lds);
}

// A step without sequences of more than 32 query rows. DV < D: two workgroups a KV head, each with all of K and half of V,
// in place of a split of the slots and the launch that joins it.
// Grid: (Hkv, ns, B) flattened into units; with two halves, groups of 8 units' first halves, then their second.
template <typename T, int D, int KW, int DV, int NR>
__global__ __launch_bounds__(64 * KW) void fp4_few(PagedAttendArgs a) {
  __shared__ __align__(512) char lds[KW * Few<DV, NR>::kLds];
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
  job_tiles<kFewKeys>(a, job, kWaveRows, x / a.Hkv);
  few_body<T, D, KW, DV, NR>(a, job, lds);
}

// Joins the splits of a row: D / 4 lanes for four values each, GS of them a split apart, which take every GS-th split, NB at
// a time, and are added up through LDS. With few rows many lanes a row: the loads of all splits are on their way at once (32
// splits of 32 rows 4.0 us with 8 lanes, 6.6 with one; two splits of 16800 rows 6.7 with two at a time, 8.6 with eight).
template <typename T, int D, int GS, int NB>
__global__ __launch_bounds__(kPagedThreads) void fp4_join(PagedAttendArgs a) {
  constexpr int kLanes = D / 4, kRows = kPagedThreads / (kLanes * GS);
  __shared__ f32x4 part_x[GS > 1 ? kPagedThreads : 1];
  __shared__ f32x4 part_s[GS > 1 ? kRows * GS : 1];
  __shared__ int best[kRows];  // of the tokens that the workgroup has rows of
  const long long rows = (long long)a.total * a.Hq, first = (long long)blockIdx.x * kRows;
  const int tid = threadIdx.x, lane = tid % kLanes, g = tid / kLanes % GS, in = tid / (kLanes * GS);
  if (tid < kRows) best[tid] = -1;
  const long long row = min(first + in, rows - 1);
  const int r = (int)(row / a.Hq);
  f32x4 st[NB], y[NB];
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const long long at = min(s0 + GS * i, a.ns - 1) * rows + row;
      st[i] = *(const f32x4*)(a.pml + at * 4);
      y[i] = *(const f32x4*)(a.po + at * D + 4 * lane);
    }
  };
  load(g);
  // the sequences of the workgroup's first row, and from there on those that end before this row
  const int b = seq_behind(a.q_start, a.map.B, seq_of_row(a.q_start, a.map.B, (int)(first / a.Hq)), r);
  const bool some = b < a.map.B;
  const Chunk c = some ? chunk_of(a.q_start, b, a.total) : Chunk{0, 0};
  const int base = some ? a.base[b] : -1;
  float M = -INFINITY, L = 0.f, SF = 0.f;
  f32x4 x = {};
  auto add = [&](const f32x4& s, const f32x4& v) __attribute__((always_inline)) {  // s: m, l, suffix sum of a share v
    const float top = fmaxf(M, s[0]), ms = top == -INFINITY ? 0.f : top;
    const float f0 = __builtin_amdgcn_exp2f(M - ms), f = __builtin_amdgcn_exp2f(s[0] - ms);
    L = f0 * L + f * s[1];
    SF = f0 * SF + f * s[2];
    x = f0 * x + f * v;
    M = top;
  };
  for (int s0 = g; s0 < a.ns; s0 += GS * NB) {
    if (s0 > g) load(s0);
#pragma unroll
    for (int i = 0; i < NB; ++i)
      if (s0 + GS * i < a.ns) add(st[i], y[i]);
  }
  if constexpr (GS > 1) {
    part_x[tid] = x;
    if (lane == 0) part_s[in * GS + g] = f32x4{M, L, SF, 0.f};
    __syncthreads();
    if (g == 0) {
#pragma unroll
      for (int i = 1; i < GS; ++i) add(part_s[in * GS + i], part_x[tid + i * kLanes]);
    }
  }
  const bool live = g == 0 && first + in < rows && r >= c.first && r < c.first + c.n && c.n <= a.max_chunk && base >= 0 &&
                    base <= a.map.cap - c.n;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const float mass = SF * inv;
  if (a.conf != nullptr) {  // one atomic a workgroup and token
    const int at = r - (int)(first / a.Hq);  // below kRows: a token has a row at least
    const bool newest = live && r == c.first + c.n - 1;
    __syncthreads();
    if (lane == 0 && newest) atomicMax(best + at, conf_bits(mass));
    __syncthreads();
    const bool begins = row == first || row % a.Hq == 0;  // the token's first row here
    if (lane == 0 && newest && begins) atomicMax((int*)a.conf + b, best[at]);
  }
  if (!live) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= inv;
  T* dst = (T*)a.out + row * D + 4 * lane;
  if constexpr (sizeof(T) == 4)
    *(f32x4*)dst = x;
  else
    *(u32x2_t*)dst = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  if (lane == 0) {
    a.lse[row] = L == 0.f ? -INFINITY : kLn2 * (M + __builtin_amdgcn_logf(L));
    if (a.suffix != nullptr) a.suffix[row] = mass;
  }
}

template <typename T, int D, int GS, int NB>
static void launch_join_as(const PagedAttendArgs& a, hipStream_t st) {
  constexpr long kRows = kPagedThreads / (D / 4 * GS);
  const long rows = (long)a.total * a.Hq;
  hipLaunchKernelGGL((fp4_join<T, D, GS, NB>), dim3((unsigned)((rows + kRows - 1) / kRows)), dim3(kPagedThreads), 0, st, a);
}
template <typename T, int D>
static void launch_join(const PagedAttendArgs& a, hipStream_t st) {
  if (a.ns <= 2) launch_join_as<T, D, 1, 2>(a, st);
  else if (a.ns <= 4) launch_join_as<T, D, 1, 4>(a, st);
  else if (a.ns <= 16) launch_join_as<T, D, 4, 4>(a, st);
  else if (a.ns <= 32) launch_join_as<T, D, 8, 4>(a, st);
  else launch_join_as<T, D, 8, 8>(a, st);
}

// ------------------------------------------------------------------------------------------
// Plan
// ------------------------------------------------------------------------------------------
struct Fp4Plan {
  long many_tiles;  // upper bound over the chunks that `total` rows can be
  int ns;           // splits of a row's slots
  int halves;       // workgroups that share a row's output values (fp4_few)
  int waves;        // of a workgroup of fp4_few: 8, or 16; 0: fp4_attend
};

// Decode steps (us in a graph, 28 / 4 or 32 / 8 heads of 128, bfloat16, at capacities of 1024 / 2048 / 4096 / 16384 slots,
// 640 to 1024, ... live). A CU holds one workgroup of 16 waves or two of 8 (of at most 16 rows).
//   up to 64 pairs of a sequence and a KV head: one workgroup a CU by splits. 32 pairs in 1 / 4 / 8 splits 9.8 15.9 26.0 85.1 /
//     9.2 11.0 13.3 29.1 / 9.6 10.4 12.8 20.7; 8 pairs and 4096 slots in 4 / 8 / 16 / 32 splits 12.2 11.1 9.8 9.7.
//   up to 128: one launch without a split is ahead on short caches: at 128 values two halves of 16 waves, up to 2560 slots
//     (128 pairs, halves / four splits 10.7 14.5 21.5 69.3 / 12.8 15.8 20.6 56.6), at 64 values 16 waves, up to 1536 (9.6 13.2 19.8
//     58.5 / 10.8 12.9 16.1 36.5). Behind that two workgroups a CU by splits.
//   up to 256: 16 waves, no split (192 pairs 12.0 16.5 25.3 79.8, 8 waves 12.5 18.2 29.8 95.7, in two splits 15.4 19.8 28.0 83.6).
//   more: 8 waves, no split (512 pairs of up to 8192 slots 97; with 16 waves 99).
// float32 at 128 values has registers for 8 waves alone, one workgroup a CU, and halves win up to 1024 slots (128 pairs, halves /
// two splits 14.5 20.2 31.6 / 15.0 18.8 25.9); so have steps of 17 to 32 rows (128 pairs of 28 rows 14.7 33.9 / 15.9 27.6 at
// 1024 / 4096).
constexpr long kFewCUs = 256, kFewUnsplit = 64, kFewWhole = 128;
constexpr long kFewSlots = 256;  // of a split at least: the launch that joins takes 1.3 us more than it saves a cache of 256 slots
// Workgroups that a launch with long chunks aims for by splitting slots. The mixed step (4 sequences of 128 tokens, 12 that decode,
// a window of 2048) unsplit / in 2 / 3 / 4 splits: 63.8 / 46.1 / 49.4 / 52.9 us; 256 tokens behind 16128 slots in 4 / 6 / 8 / 16: 106 / 109 /
// 91 / 103; 64 behind 8128 in 8 / 16 / 32: 33.9 / 27.0 / 30.9; 2048 behind 6144 unsplit / in 2: 249 / 259.
constexpr long kManyTarget = 512;
// Slots of a split there: 256, and one for every 32 query rows of the launch, whose partials are written and read.
constexpr long kManySlots = 256, kRowsPerSlot = 32;
// A split for each whole 32768 slots at least (so one holds fewer than twice as many), whatever the number of workgroups: the
// capacity is all that the host knows, and one long sequence among many short ones shall not hold up the launch. Beside a long
// chunk a shorter one does: the splits go by the launch's workgroups, and a chunk of 4096 tokens behind 4096 with 8 sequences that
// decode behind 32767 slots takes 667 us, in two calls 432 and 59.
constexpr long kMaxSlots = 32768;
constexpr long kMaxSplits = 64;
// Rows that a launch joins at most: its 256 threads a workgroup of one row at least must stay below the 2^32 of a grid.
constexpr long kMaxJoined = (1l << 24) - 1;

// reach: slots that a token may see, by the capacity and the window.
static Fp4Plan fp4_plan(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, long total, long max_chunk, long reach) {
  const long G = l.n_q_heads / l.n_kv_heads;
  const bool wide = l.head_dim == 128;
  Fp4Plan p = {0, 1, 1, 0};
  long ns = 1, slots = kFewSlots;
  if (max_chunk * G <= kWaveRows) {
    const bool two = max_chunk * G <= 16 && !(dtype == LG_F32 && wide);  // two workgroups of 8 waves fit a CU, or one of 16
    const long units = (long)m.batch * l.n_kv_heads;
    const long whole = !wide ? 1536 : dtype == LG_F32 ? 1024 : 2560;
    p.waves = 8;
    if (units <= kFewUnsplit) {
      ns = kFewCUs / units;
    } else if (units <= kFewWhole) {
      if (reach > whole) {
        ns = (two ? 2 : 1) * kFewCUs / units;
      } else {
        p.halves = wide ? 2 : 1;
        p.waves = two ? 16 : 8;
      }
    } else if (units <= kFewCUs) {
      p.waves = two ? 16 : 8;
    }
  } else {
    if (total * G > kWaveRows) {
      // a sequence of n rows has at most n / 128 + 1 tiles, and more than 32 rows
      p.many_tiles = total * G / kManyRows;
      p.many_tiles += std::min(total * G / (kWaveRows + 1), (long)m.batch);
    }
    const long units = (p.many_tiles + m.batch) * l.n_kv_heads;
    ns = (kManyTarget + units - 1) / units;
    slots = kManySlots + total * l.n_q_heads / kRowsPerSlot;
  }
  ns = std::min({ns, (reach + slots - 1) / slots, kMaxSplits});
  p.ns = (int)std::max({ns, std::min(reach / kMaxSlots, kMaxSplits), 1l});
  if (total * l.n_q_heads > kMaxJoined) p.ns = 1;
  return p;
}

static size_t fp4_need(const lg_paged_layer& l, const Fp4Plan& p, long total) {
  return p.ns > 1 ? (size_t)p.ns * total * l.n_q_heads * (l.head_dim + 4) * 4 : 0;
}

// Workgroups of the launch (a grid holds fewer than 2^32 threads).
long fp4_attend_grid(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, int total, int max_chunk) {
  const Fp4Plan p = fp4_plan(l, m, dtype, total, max_chunk, whole_reach(m));
  return (p.many_tiles + m.batch) * l.n_kv_heads * p.ns * p.halves;
}

size_t fp4_attend_need(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, int total, int max_chunk, int window,
                       int n_sink) {
  return fp4_need(l, fp4_plan(l, m, dtype, total, max_chunk, window_reach(m, max_chunk, window, n_sink)), total);
}

// The largest need of any total up to this one and any max_chunk up to this one, with any window (a shorter reach
// has no more splits). For a given number of splits the need grows with total, and the number falls as total
// grows, so the ends of its steps count.
size_t fp4_attend_bytes(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, int total, int max_chunk) {
  size_t most = 16;
  for (int form = 0; form < 2; ++form) {
    const long chunk = form == 0 ? 1 : max_chunk;
    long t = total;
    while (t > 0) {
      const Fp4Plan p = fp4_plan(l, m, dtype, t, chunk, whole_reach(m));
      most = std::max(most, fp4_need(l, p, t));
      long lo = 0, hi = t;  // the largest smaller total with more splits
      while (hi - lo > 1) {
        const long mid = (lo + hi) / 2;
        if (fp4_plan(l, m, dtype, mid, chunk, whole_reach(m)).ns > p.ns) lo = mid; else hi = mid;
      }
      t = lo;
    }
  }
  return align_up(most, 16);
}

template <typename T, int D, int KW, int NR>
static void launch_few(const PagedAttendArgs& a, const Fp4Plan& p, dim3 grid, hipStream_t st) {
  if (p.halves == 1)
    hipLaunchKernelGGL((fp4_few<T, D, KW, D, NR>), grid, dim3(64 * KW), 0, st, a);
  else if constexpr (D == 128)
    hipLaunchKernelGGL((fp4_few<T, D, KW, D / 2, NR>), grid, dim3(64 * KW), 0, st, a);
}

template <typename T, int D>
static void launch_typed(const PagedAttendArgs& a, const Fp4Plan& p, dim3 grid, hipStream_t st) {
  if (p.waves == 0) {
    hipLaunchKernelGGL((fp4_attend<T, D>), grid, dim3(kPagedThreads), 0, st, a);
  } else if ((long)a.max_chunk * a.G > 16) {
    launch_few<T, D, 8, 2>(a, p, grid, st);
  } else if (p.waves == 8) {
    launch_few<T, D, 8, 1>(a, p, grid, st);
  } else if constexpr (sizeof(T) == 2 || D == 64) {
    launch_few<T, D, 16, 1>(a, p, grid, st);
  }
  if (p.ns > 1) launch_join<T, D>(a, st);
}

hipError_t launch_fp4_attend(const lg_paged_layer& l, const lg_page_map& m, lg_dtype dtype, const void* q, void* out,
                             const int32_t* q_start, const int32_t* base, int total, int max_chunk, int window,
                             int n_sink, const int32_t* suffix_w, float* lse, float* suffix, float* conf, void* ws,
                             hipStream_t st) {
  const Fp4Plan p = fp4_plan(l, m, dtype, total, max_chunk, window_reach(m, max_chunk, window, n_sink));
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
  if (dtype == LG_BF16) {
    if (l.head_dim == 128) launch_typed<__bf16, 128>(a, p, grid, st);
    else launch_typed<__bf16, 64>(a, p, grid, st);
  } else {
    if (l.head_dim == 128) launch_typed<float, 128>(a, p, grid, st);
    else launch_typed<float, 64>(a, p, grid, st);
  }
  return hipGetLastError();
}

}  // namespace lg
