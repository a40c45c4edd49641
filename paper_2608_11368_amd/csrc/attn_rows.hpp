// Attention of a few new tokens per request (decoding, drafted tokens): all
// rows of a key/value head -- a row is one query head of one token -- fit one
// or two tiles of 16, and the time goes into reading the cache once.
//
// Layout.  A wave takes 32 keys at a time from memory into registers, whole rows
// at a time; keys then pass through the wave's own LDS, values do not.
//   scores   S^T = K Q^T: a key row is 16-byte pieces of the A operand, and lane
//            (x, g) ends up with row x's scores of keys 4 g + i and 16 + 4 g + i;
//   weights  exactly those are its eight entries of the B operand of
//   output   O^T += V^T P^T once the product's k index is taken in that order:
//            only V has to be transposed, and a lane that loads eight dims of
//            its eight keys does it with one byte permute per dword.
// The rows' running maximum is raised (and the sums rescaled) only when a score
// exceeds it by 2^8, so most steps need no exchange between lanes.
//
// Work split.  The keys of all requests form one line of units of kUnit keys; it
// is cut into equal runs whatever the lengths (the lengths are scanned by every
// workgroup: they are a few cached kilobytes), and a run has one workgroup for
// each key head.  Those walk it side by side, so that the heads of a slot, which
// lie together in memory, are read at about the same time.  A request that is
// cut leaves partial sums that a second launch joins.  The waves of a workgroup
// (four; eight in calls of a few short requests, which are not cut) take the
// 32-key blocks in turn and are joined through LDS.
//
// Bound by the cache's bytes.  Measured: one token for each of 256 requests of
// 4000 keys on average, 8 heads of width 128, 4.1 GB: 649 us and 8 us for the
// joins, 6.3 TB/s (a read of the same bytes with no work on them runs at 7.0);
// five drafted tokens of 2 requests of 131,000 keys, 1.07 GB: 176 us, 6.1 TB/s.
// What was measured on the first of these and decides the layout: K in 64-byte
// pieces of a row straight into the products' operands 5.7 TB/s at any
// occupancy or order, whole rows past the caches and through LDS 6.3; the heads
// of a run on one XCD 5.5 instead of side by side.
//
// Over a cache in 8 or 4 bits (add_codes) the first of these is 2.16 GB, 326 us and 7
// for the joins, 6.6 TB/s, and 1.12 GB, 183 and 7, 6.1 TB/s: as fast as the same loads
// with nothing done to what they bring but a store to LDS (331 and 183 in all).
// What is left are the ends of requests, where a workgroup starts anew (64 requests
// of 16,000 keys take 12 us less in 4 bits than 256 of 4000).
#pragma once

#include "attn.hpp"

namespace pair {

namespace rows {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kBlock = 32;                  // keys of a wave's step
constexpr int kUnit = kBlock * kWaves;      // keys of a workgroup's step
constexpr int kWideWaves = 2 * kWaves;      // of a workgroup that has a compute unit for itself
// Requests whose lengths a workgroup scans; more of them fill the card with
// one workgroup per request and head, whole, unless one is far longer than the rest
// (8 heads of 128: 2100 uneven ones of 400 keys 582 us so, cut 627; 4000 of 1000
// 2640 and 2675; but one of 60,000 beside 2100 of 100 836 and 279).
constexpr int kMostScanned = 2048;
constexpr int kMostRuns = 1024;
constexpr float kLazy = 8.0f;
constexpr uint32_t kXcds = 8;

struct RowArgs {
  AttnCall a;
  FastDiv page, group;
  float scale_log2;
  int32_t runs;         // most runs; 0: one workgroup per request and head
  int32_t* starts;      // [n + 1] units before each request (workspace)
  float* part_o;        // [2 runs][kv_heads][rows][dim]
  float* part_ml;       // [2 runs][kv_heads][rows][2]
};

__device__ __forceinline__ int units_of(const RowArgs& s, int64_t r, int32_t* bad) {
  Request q;
  if (!attention_request(s.a, s.page.d, r, &q, bad)) return 0;
  if (q.tokens == 0 || (int64_t)q.tokens * s.group.d > kRowsMost) return 0;
  return q.len <= kUnit ? 1 : (q.len + kUnit - 1) / kUnit;
}

// No more runs than there are units, so that none of those between two of a
// request is empty.
__device__ __forceinline__ int64_t runs_of(const RowArgs& s, int64_t units) {
  return units < s.runs ? units : s.runs;
}

// a / b for 0 <= a < 2^42 and 0 < b < 2^31 with a / b < 2^31: the exact quotient is
// an integer or further than 1 / b from the next one, which the rounding of the
// double's (2^-53 of it) does not reach.  A division of 64-bit integers takes
// some hundred instructions.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (int64_t)((double)a / (double)b);
}

// First unit of run w of `runs` on a line of `units`.
__device__ __forceinline__ int64_t run_start(int64_t units, int64_t runs, int64_t w) {
  return quotient(units * w, runs);
}

// One wave's running softmax over its keys: row x = lane & 15 of each tile.
template <int DIM, int NT>
struct State {
  float m[NT], l[NT];                // l: this lane's keys only
  f32x4_t acc[NT][DIM / 16];         // O^T: dims (4 g + i) * (DIM / 16) + j of row x
};

// A lane's sixteenth of a key or value row.  Each is read once: the loads are
// non-temporal, and each instruction covers whole cache lines.
template <int DIM>
struct Piece {
  uint32_t w[DIM / 32];
  __device__ __forceinline__ void load(const unsigned char* p) {
    if (DIM == 128) {
      const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
#pragma unroll
      for (int i = 0; i < DIM / 32; ++i) w[i] = v[i];
    } else {
      const u32x2_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p));
#pragma unroll
      for (int i = 0; i < DIM / 32; ++i) w[i] = v[i];
    }
  }
  __device__ __forceinline__ void store(unsigned char* p) const {
#pragma unroll
    for (int i = 0; i < DIM / 32; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
  }
};

// Byte `b` of LDS row `row` of a block's keys: 16-byte pieces permuted by the
// row, so that neither 16 lanes on one row nor 16 rows at one place meet in a
// bank.
template <int DIM>
__device__ __forceinline__ int key_place(int row, int b) {
  return row * (DIM * 2) + ((((b >> 4) ^ row) & (DIM / 8 - 1)) << 4) + (b & 15);
}

// LDS of one wave: a block's keys (in 8 and 4 bits its keys' and values' codes), the
// values and weights of an odd one, or the wave's sums.
template <int BITS, int DIM, int NT>
struct WaveLds {
  static constexpr int kRowBytes = DIM * BITS / 8;
  union {
    float sum[16][DIM + 4];
    unsigned char key[kBlock * DIM * 2];
    unsigned char codes[BITS == 16 ? 16 : 2 * kBlock * kRowBytes];
    uint16_t value[kBlock][DIM];
  };
  uint32_t weight[NT][16][kBlock / 2];
  union {
    float stat[16][2];
    uint32_t scale[BITS == 16 ? 1 : 2 * kBlock];   // of a block's keys and values: each row's bytes
  };

  // Piece `c` of 16 bytes of key `y`: permuted by the row so that eight rows'
  // pieces at one place lie in different banks.
  static __device__ __forceinline__ int key_at(int y, int c) {
    const int turn = kRowBytes == 128 ? y & 7 : kRowBytes == 64 ? (y >> 2) & 3 : 0;
    return y * kRowBytes + ((c ^ turn) << 4);
  }
  // Value `y`: rows 4 g + i of a tile, of which an instruction reads one i, side by side.
  static __device__ __forceinline__ int value_at(int y) {
    return (kBlock + (y & 16) + (y & 3) * 4 + ((y >> 2) & 3)) * kRowBytes;
  }
};

// A block whose values are not all finite and not all seen by every row: each
// row adds the values that it sees, one key at a time, and the values are
// cleared so that the matrix product adds nothing.
template <int BITS, bool BF16, int DIM, int NT>
__device__ __forceinline__ void add_odd_block(WaveLds<BITS, DIM, NT>* lds, const u32x4_t (&pf)[NT],
                                              int kb, const int (&limit)[NT],
                                              Piece<DIM> (*vr)[8], State<DIM, NT>* st) {
  constexpr int ND = DIM / 16;
  const int lane = threadIdx.x & (kWave - 1);
  const int x = lane & 15, g = lane >> 4;
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int w = 0; w < ND / 2; ++w) {
      uint32_t* to = reinterpret_cast<uint32_t*>(lds->value[16 * (e >> 2) + 4 * g + (e & 3)]);
      to[x * (ND / 2) + w] = (*vr)[e].w[w];
      (*vr)[e].w[w] = 0u;
    }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int w = 0; w < 4; ++w) lds->weight[nt][x][8 * (w >> 1) + 2 * g + (w & 1)] = pf[nt][w];
  wave_lds_order();
#pragma unroll 1
  for (int k = 0; k < kBlock; ++k) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float p = half_value<BF16>((lds->weight[nt][x][k >> 1] >> (16 * (k & 1))) & 0xffffu);
      if (kb + k > limit[nt]) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < ND; ++j)
          st->acc[nt][j][i] = __builtin_fmaf(
              p, half_value<BF16>(lds->value[k][(4 * g + i) * ND + j]), st->acc[nt][j][i]);
    }
  }
  wave_lds_order();
}

// A block's scores of this lane's rows (keys 16 t + 4 g + i) and its values, piece
// x of eight rows: their share of the sums.  `tiles` of rows are in use: a launch that
// serves chunks as well is built for two (eight chunks beside 64 single tokens over
// 2500 keys in 8 bits: 156 us for both tiles, 151 for those that there are).
template <int BITS, bool BF16, int DIM, int NT>
__device__ __forceinline__ void weigh_block(const RowArgs& s, const f32x4_t (&sc)[NT][2],
                                            const int (&limit)[NT], int first_limit, int len,
                                            int kb, Piece<DIM> (&vr)[8], int tiles,
                                            WaveLds<BITS, DIM, NT>* lds, State<DIM, NT>* st) {
  constexpr int ND = DIM / 16;       // dims of a lane's piece of a value row
  const int g = (threadIdx.x & (kWave - 1)) >> 4;
  float p[NT][8];
  const bool masked = kb + kBlock - 1 > first_limit;   // some row does not see some key
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (nt >= tiles) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[nt][e] = sc[nt][e >> 2][e & 3] * s.scale_log2;
    if (masked) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (kb + 16 * (e >> 2) + 4 * g + (e & 3) > limit[nt]) p[nt][e] = -INFINITY;
    }
    float top = p[nt][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, p[nt][e]);
    if (__any(top > st->m[nt] + kLazy)) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float mn = fmaxf(st->m[nt], top);
      const float keep = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st->m[nt] - mn);
      st->m[nt] = mn;
      st->l[nt] *= keep;
#pragma unroll
      for (int j = 0; j < ND; ++j) st->acc[nt][j] *= keep;
    }
    const float base = (st->m[nt] == -INFINITY ? 0.0f : st->m[nt]) - kLift<BF16>;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[nt][e] = __builtin_amdgcn_exp2f(p[nt][e] - base);
      st->l[nt] += p[nt][e];
    }
  }

  u32x4_t pf[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int w = 0; w < 4; ++w)
      pf[nt][w] = nt < tiles ? pack2<BF16>(p[nt][2 * w], p[nt][2 * w + 1]) : 0u;
  // Values that some row must not see: past the end they are no values at
  // all, and within the chunk a weight of zero does not hide a NaN or an
  // infinity from the matrix product.
  if (masked) {
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = kb + 16 * (e >> 2) + 4 * g + (e & 3);
#pragma unroll
      for (int w = 0; w < ND / 2; ++w) {
        if (key >= len) vr[e].w[w] = 0u;
        bad |= not_finite<BF16>(vr[e].w[w]) ? 1u : 0u;
      }
    }
    if (__any(bad != 0u)) add_odd_block<BITS, BF16, DIM, NT>(lds, pf, kb, limit, &vr, st);
  }

#pragma unroll
  for (int j = 0; j < ND; ++j) {
    u32x4_t vt;                                   // dim j of this lane's eight keys
#pragma unroll
    for (int w = 0; w < 4; ++w)
      vt[w] = __builtin_amdgcn_perm(vr[2 * w + 1].w[j >> 1], vr[2 * w].w[j >> 1],
                                    (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (nt < tiles) st->acc[nt][j] = mma16<BF16>(vt, pf[nt], st->acc[nt][j]);
  }
}

// A block's keys and values, piece x of eight rows: its scores, and its share of
// the sums.
template <bool BF16, int DIM, int NT>
__device__ __forceinline__ void add_block(const RowArgs& s, const u32x4_t (&qf)[NT][DIM / 32],
                                          const int (&limit)[NT], int first_limit, int len, int kb,
                                          const Piece<DIM> (&kr)[8], Piece<DIM> (&vr)[8],
                                          WaveLds<16, DIM, NT>* lds, State<DIM, NT>* st) {
  constexpr int NC = DIM / 32;       // 32-dim pieces of a key row
  const int lane = threadIdx.x & (kWave - 1);
  const int x = lane & 15, g = lane >> 4;

  // keys through LDS: whole rows come from memory, the product wants a row's
  // piece from every lane
  wave_lds_order();
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int y = 16 * (e >> 2) + 4 * g + (e & 3);
    kr[e].store(lds->key + key_place<DIM>(y, x * (DIM / 8)));
  }
  wave_lds_order();
  f32x4_t sc[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int t = 0; t < 2; ++t) sc[nt][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4_t kf = *reinterpret_cast<const u32x4_t*>(
          lds->key + key_place<DIM>(16 * t + x, 64 * c + 16 * g));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][t] = mma16<BF16>(kf, qf[nt][c], sc[nt][t]);
    }
  weigh_block<16, BF16, DIM, NT>(s, sc, limit, first_limit, len, kb, vr, NT, lds, st);
}

template <bool BF16, int DIM, int NT, bool ALIGNED, int WAVES>
__device__ __forceinline__ void add_keys(const RowArgs& s, const u32x4_t (&qf)[NT][DIM / 32],
                                         const int (&limit)[NT], int first_limit, int64_t r,
                                         int64_t kvh, int len, int k0, int k1,
                                         WaveLds<16, DIM, NT>* lds, State<DIM, NT>* st) {
  const int lane = threadIdx.x & (kWave - 1);
  const int x = lane & 15, g = lane >> 4;
  const int64_t head = kvh * s.a.cache.head_stride * 2;
  const unsigned char* kbase = static_cast<const unsigned char*>(s.a.k_cache) + head;
  const unsigned char* vbase = static_cast<const unsigned char*>(s.a.v_cache) + head;
  const int64_t slot_bytes = s.a.cache.slot_stride * 2, page_bytes = s.a.cache.page_stride * 2;
  const int32_t* row = s.a.table + r * s.a.ldt;
  const int64_t lane_off = x * (DIM / 8) + (ALIGNED ? 4 * g * slot_bytes : 0);

  // A lane reads piece x of eight rows, the same of keys and values.  Pages are
  // looked up a step before: one per tile of 16 keys where pages are multiples
  // of 16 (by scalar loads), else one per row.
  constexpr int kIds = ALIGNED ? 2 : 8;
  int32_t id[kIds];
  int32_t bad_page = 0;
  auto key_of = [&](int kb, int n) {
    if (ALIGNED) {                       // a tile past the end repeats the last
      const int key = kb + 16 * n;
      return uniform(key < len ? key : (len - 1) & ~15);
    }
    const int key = kb + 16 * (n >> 2) + 4 * g + (n & 3);
    return key < len ? key : len - 1;
  };
  auto lookup = [&](int kb) {
#pragma unroll
    for (int n = 0; n < kIds; ++n) {
      const uint32_t pg = div_by((uint32_t)key_of(kb, n), s.page);
      id[n] = ALIGNED ? table_entry(row, pg) : row[pg];
    }
  };
  if (k0 < k1) lookup(k0);
  for (int kb = k0; kb < k1; kb += kBlock * WAVES) {
    Piece<DIM> kr[8], vr[8];
    int64_t at[kIds];
#pragma unroll
    for (int n = 0; n < kIds; ++n) {
      const uint32_t key = (uint32_t)key_of(kb, n);
      at[n] = checked_page(s.a, id[n], &bad_page) * page_bytes +
              (int64_t)(key - div_by(key, s.page) * s.page.d) * slot_bytes + lane_off;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      kr[e].load(kbase + at[ALIGNED ? e >> 2 : e] + (ALIGNED ? (e & 3) * slot_bytes : 0));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      vr[e].load(vbase + at[ALIGNED ? e >> 2 : e] + (ALIGNED ? (e & 3) * slot_bytes : 0));
    if (kb + kBlock * WAVES < k1) lookup(kb + kBlock * WAVES);
    add_block<BF16, DIM, NT>(s, qf, limit, first_limit, len, kb, kr, vr, lds, st);
  }
  if (bad_page) raise_status(s.a.d_status, bad_page);
}

// The same as add_keys over a cache in 8 or 4 bits.  A wave's loads are contiguous,
// 16 bytes a lane; codes pass through the wave's LDS and are converted when they are
// read from it.  The products' k index takes a key's elements in the order in which
// a lane has those of one block (with the queries alike), so that it needs one scale.
// The next block is on its way while one is used: a block has a half or a quarter of
// the bytes, too few in flight otherwise (4 bits: 226 us without, 203 with one ahead,
// 203 with two; 256 requests of 4000 keys, 8 heads of 128).
//
// The matrix instructions that take codes and scales as they are were measured and
// not taken: their sums are not those of 32 bits (off by up to 2^-12 of the largest
// product, 2^-19 of the sum of magnitudes in the mean square).
template <int BITS, bool BF16, int DIM, int NT, bool ALIGNED, int WAVES>
__device__ __forceinline__ void add_codes(const RowArgs& s,
                                          const u32x4_t (&qf)[NT][DIM / 32],
                                          const int (&limit)[NT], int first_limit, int64_t r,
                                          int64_t kvh, int len, int k0, int k1, int tiles,
                                          WaveLds<BITS, DIM, NT>* lds, State<DIM, NT>* st) {
  using Lds = WaveLds<BITS, DIM, NT>;
  constexpr int W = DIM * BITS / 8;                        // bytes of a row
  constexpr int kLoads = kBlock * W / 1024;                // of keys, and of values
  constexpr int kRowLanes = W / 16;
  constexpr int kStep = kBlock * WAVES;
  // Not beside two tiles of rows, which leave no registers for it (five drafted tokens
  // of 2 requests of 131,000 keys, 32 query heads on 8, in 8 bits: 128 us with
  // registers spilled, 97 without).
  constexpr bool kAhead = NT == 1;
  const int lane = threadIdx.x & (kWave - 1);
  const int x = lane & 15, g = lane >> 4;
  const int64_t head = kvh * s.a.cache.head_stride;
  const unsigned char* kbase = static_cast<const unsigned char*>(s.a.k_cache) + head;
  const unsigned char* vbase = static_cast<const unsigned char*>(s.a.v_cache) + head;
  const unsigned char* sbase =                             // those of a key, or of its value
      (lane < kBlock ? s.a.scales.k : s.a.scales.v) + kvh * s.a.scales.head;
  const int64_t slot_bytes = s.a.cache.slot_stride, page_bytes = s.a.cache.page_stride;
  const int32_t* row = s.a.table + r * s.a.ldt;
  const int my_row = lane / kRowLanes, my_piece = lane % kRowLanes;   // of a load
  const int s_row = lane & (kBlock - 1);
  const int v_turn = (8 * (x * (DIM / 16) / kMxBlock) + 9) & 31;

  // Pages of a block's tiles, or (pages not of a multiple of 16) of this lane's
  // rows, the last for its scales; looked up a step before.
  constexpr int kIds = ALIGNED ? 2 : kLoads + 1;
  int32_t id[kIds];
  int32_t bad_page = 0;
  auto key_of = [&](int kb, int n) {
    if (ALIGNED) {                       // a tile past the end repeats the last
      const int key = kb + 16 * n;
      return uniform(key < len ? key : (len - 1) & ~15);
    }
    const int key = kb + (n < kLoads ? n * (kWave / kRowLanes) + my_row : s_row);
    return key < len ? key : len - 1;
  };
  auto lookup = [&](int kb) {
#pragma unroll
    for (int n = 0; n < kIds; ++n) {
      const uint32_t pg = div_by((uint32_t)key_of(kb, n), s.page);
      id[n] = ALIGNED ? table_entry(row, pg) : row[pg];
    }
  };
  struct Ahead {
    u32x4_t k[kLoads], v[kLoads];
    uint32_t scales;
  };
  Ahead ahead;
  // ALIGNED: a tile's place is scalar, a lane's place in it the same for every tile.
  const int64_t lane_at = (ALIGNED ? (my_row & 15) * slot_bytes : 0) + my_piece * 16;
  const unsigned char* s_at = sbase + (ALIGNED ? (s_row & 15) * s.a.scales.slot : 0);
  auto fetch = [&](int kb) {
    int64_t place[kIds], scale_place[kIds];
#pragma unroll
    for (int n = 0; n < kIds; ++n) {
      const uint32_t key = (uint32_t)key_of(kb, n);
      const int64_t pg = checked_page(s.a, id[n], &bad_page);
      const int64_t y = key - div_by(key, s.page) * s.page.d;          // slot in the page
      place[n] = pg * page_bytes + y * slot_bytes;
      scale_place[n] = pg * s.a.scales.page + y * s.a.scales.slot;
    }
    const unsigned char* scales =
        s_at + (ALIGNED && (s_row & 16) == 0 ? scale_place[0] : scale_place[kIds - 1]);
    ahead.scales = DIM == 128 ? *reinterpret_cast<const uint32_t*>(scales)
                               : *reinterpret_cast<const uint16_t*>(scales);
    int64_t at[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      int64_t from = place[ALIGNED ? j * (kWave / kRowLanes) / 16 : j];
      if (ALIGNED && kLoads == 1 && my_row >= 16) from = place[kIds - 1];
      if (ALIGNED && kLoads > 2 && j % 2 == 1) from += 8 * slot_bytes;  // half a tile a load
      at[j] = from + lane_at;
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      ahead.k[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(kbase + at[j]));
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      ahead.v[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(vbase + at[j]));
  };
  auto use = [&](int kb) {
    wave_lds_order();
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int y = j * (kWave / kRowLanes) + my_row;
      *reinterpret_cast<u32x4_t*>(lds->codes + Lds::key_at(y, my_piece)) = ahead.k[j];
      *reinterpret_cast<u32x4_t*>(lds->codes + Lds::value_at(y) + my_piece * 16) = ahead.v[j];
    }
    lds->scale[lane] = ahead.scales;
    wave_lds_order();
    const int next = kb + kStep;
    if (kAhead && next < k1) {
      fetch(next);
      if (next + kStep < k1) lookup(next + kStep);
    }
    f32x4_t sc[NT][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int y = 16 * t + x;
      Codes<BITS, DIM / 4> c;            // elements DIM / 4 * g .. of key x of the tile
      if constexpr (Lds::kRowBytes == 32) {
        c.load(lds->codes + Lds::key_at(y, g >> 1) + (g & 1) * 8);
      } else {
        constexpr int kOwn = W / 64;     // pieces
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(
              lds->codes + Lds::key_at(y, kOwn * g + j));
#pragma unroll
          for (int w = 0; w < 4; ++w) c.w[4 * j + w] = v[w];
        }
      }
      uint32_t kf[DIM / 8];
      c.template values<BF16>(mx_scale(reinterpret_cast<const unsigned char*>(
                                  &lds->scale[y])[g * (DIM / 4) / kMxBlock]), kf);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        sc[nt][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < DIM / 32; ++j) {
          const u32x4_t eight = {kf[4 * j], kf[4 * j + 1], kf[4 * j + 2], kf[4 * j + 3]};
          if (nt < tiles) sc[nt][t] = mma16<BF16>(eight, qf[nt][j], sc[nt][t]);
        }
      }
    }
    Piece<DIM> vr[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4_t four = *reinterpret_cast<const u32x4_t*>(&lds->scale[kBlock + 16 * t + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {      // the block's byte where a float's exponent is
        Codes<BITS, DIM / 16> c;
        c.load(lds->codes + Lds::value_at(16 * t + 4 * g + i) + x * (W / 16));
        c.template values<BF16>(
            __uint_as_float(__builtin_amdgcn_alignbit(four[i], four[i], v_turn)), vr[4 * t + i].w);
      }
    }
    weigh_block<BITS, BF16, DIM, NT>(s, sc, limit, first_limit, len, kb, vr, tiles, lds, st);
  };
  if (k0 < k1) lookup(k0);
  if (kAhead && k0 < k1) {
    fetch(k0);
    if (k0 + kStep < k1) lookup(k0 + kStep);
  }
  for (int kb = k0; kb < k1; kb += kStep) {
    if (!kAhead) {
      fetch(kb);
      if (kb + kStep < k1) lookup(kb + kStep);
    }
    use(kb);
  }
  if (bad_page) raise_status(s.a.d_status, bad_page);
}

// Keys [k0, k1) of one request and head (k0 a multiple of kUnit): the waves'
// sums, joined, either as results (slot < 0) or as partial sums.
template <int BITS, bool BF16, int DIM, int NT, bool ALIGNED, int WAVES>
__device__ __forceinline__ void attend(const RowArgs& s, int64_t r, int kvh, int k0, int k1,
                                       int64_t slot, WaveLds<BITS, DIM, NT>* lds) {
  constexpr int ND = DIM / 16;
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int x = lane & 15, g = lane >> 4;
  Request q;
  int32_t bad = 0;
  if (!attention_request(s.a, s.page.d, r, &q, &bad)) return;   // seen good by the scan
  const int rows = q.tokens * (int)s.group.d;
  u32x4_t qf[NT][DIM / 32];
  int limit[NT];
  State<DIM, NT> st;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int i = 16 * nt + x;
    const int tok = (int)div_by((uint32_t)i, s.group);
    limit[nt] = i < rows ? limit_of(q, tok) : -1;
    st.m[nt] = -INFINITY;
    st.l[nt] = 0.0f;
#pragma unroll
    for (int j = 0; j < ND; ++j) st.acc[nt][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < DIM / 32; ++c) qf[nt][c] = u32x4_t{0u, 0u, 0u, 0u};
    if (i < rows) {
      // elements 32 c + 8 g .., as the products take a key's; add_codes' order
      constexpr int kLane = BITS == 16 ? 8 : DIM / 4, kNext = BITS == 16 ? 32 : 8;
      const uint16_t* p = static_cast<const uint16_t*>(s.a.q) + (q.q0 + tok) * s.a.q_token +
                          (kvh * (int)s.group.d + i - tok * (int)s.group.d) * s.a.q_head + g * kLane;
#pragma unroll
      for (int c = 0; c < DIM / 32; ++c)
        qf[nt][c] = *reinterpret_cast<const u32x4_t*>(p + c * kNext);
    }
  }
  // unused rows see nothing, so every block counts as masked for them only if
  // it does for the first token
  const int end = k1 < q.len ? k1 : q.len;
  if constexpr (BITS == 16)
    add_keys<BF16, DIM, NT, ALIGNED, WAVES>(s, qf, limit, q.len - q.tokens, r, kvh, q.len,
                                            k0 + kBlock * wave, end, lds + wave, &st);
  else
    add_codes<BITS, BF16, DIM, NT, ALIGNED, WAVES>(s, qf, limit, q.len - q.tokens, r, kvh, q.len,
                                                   k0 + kBlock * wave, end,
                                                   NT == 1 || rows <= 16 ? 1 : 2, lds + wave, &st);

#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float l = st.l[nt];
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (g == 0) {
      lds[wave].stat[x][0] = st.m[nt];
      lds[wave].stat[x][1] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < ND; ++j) lds[wave].sum[x][(4 * g + i) * ND + j] = st.acc[nt][j][i];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * DIM / 8; e += WAVES * kWave) {
      const int y = e / (DIM / 8), d = (e - y * (DIM / 8)) * 8;
      const int i = 16 * nt + y;
      if (i < rows) {
        float m = lds[0].stat[y][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, lds[w].stat[y][0]);
        const float base = m == -INFINITY ? 0.0f : m;
        float tot = 0.0f, o[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const float mw = lds[w].stat[y][0], lw = lds[w].stat[y][1];
          if (mw == -INFINITY && lw == 0.0f) continue;   // saw no key
          const float f = __builtin_amdgcn_exp2f(mw - base);
          tot = __builtin_fmaf(f, lw, tot);
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = __builtin_fmaf(f, lds[w].sum[y][d + k], o[k]);
        }
        if (slot >= 0) {
          float* to = s.part_o + (slot * (16 * NT) + i) * DIM + d;
          *reinterpret_cast<f32x4_t*>(to) = f32x4_t{o[0], o[1], o[2], o[3]};
          *reinterpret_cast<f32x4_t*>(to + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
          if (d == 0) {
            s.part_ml[(slot * (16 * NT) + i) * 2] = m;
            s.part_ml[(slot * (16 * NT) + i) * 2 + 1] = tot;
          }
        } else {
          const int tok = (int)div_by((uint32_t)i, s.group);
          const int h = kvh * (int)s.group.d + i - tok * (int)s.group.d;
          const bool none = limit_of(q, tok) < 0;
          const float inv = none ? 0.0f : 1.0f / tot;
          u32x4_t w;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            w[k] = none ? 0u : pack2<BF16>(o[2 * k] * inv, o[2 * k + 1] * inv);
          *reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(s.a.out) +
                                      (q.q0 + tok) * s.a.out_token + h * s.a.out_head + d) = w;
          if (s.a.lse != nullptr && d == 0)
            s.a.lse[(q.q0 + tok) * s.a.q_heads + h] =
                none ? -INFINITY : log_sum<BF16>(m, tot);
        }
      }
    }
    __syncthreads();
  }
}

// Units before each request, in every workgroup; the first leaves them to the
// launch that joins.
__device__ __forceinline__ void scan_units(const RowArgs& s, uint32_t block, int32_t* start,
                                           int32_t* wave_sums) {
  const int n = (int)s.a.n, lane = threadIdx.x & (kWave - 1);
  const int per = (n + kThreads - 1) / kThreads;
  const int r0 = (int)threadIdx.x * per, r1 = r0 + per < n ? r0 + per : n;
  int32_t bad = 0, mine = 0;
  for (int r = r0; r < r1; ++r) {
    const int u = units_of(s, r, &bad);
    start[r + 1] = u;
    mine += u;
  }
  if (bad && block == 0) raise_status(s.a.d_status, bad);
  int32_t scan = mine;
#pragma unroll
  for (int by = 1; by < kWave; by <<= 1) {
    const int32_t v = __shfl_up(scan, by, kWave);
    if (lane >= by) scan += v;
  }
  if (lane == kWave - 1) wave_sums[threadIdx.x / kWave] = scan;
  if (threadIdx.x == 0) start[0] = 0;
  __syncthreads();
  int32_t at = scan - mine;
  for (int w = 0; w < (int)threadIdx.x / kWave; ++w) at += wave_sums[w];
  for (int r = r0; r < r1; ++r) {
    at += start[r + 1];
    start[r + 1] = at;
  }
  __syncthreads();
  if (block == 0)
    for (int r = threadIdx.x; r <= n; r += kThreads) s.starts[r] = start[r];
}

// One workgroup's share of a call, `block` its number.  Only workgroups of kWaves
// waves serve cut calls, and need `start` (kMostScanned + 1) and `sums` (kWaves).
template <int BITS, bool BF16, int DIM, int NT, bool ALIGNED, int WAVES>
__device__ __forceinline__ void serve(const RowArgs& s, uint32_t block,
                                      WaveLds<BITS, DIM, NT>* lds, int32_t* start, int32_t* sums) {
  const int64_t heads = s.a.kv_heads;
  const bool direct = WAVES != kWaves || s.runs == 0;   // one workgroup per request and head
  int64_t run = block / (uint32_t)s.a.kv_heads;         // or the request
  int h = (int)(block - run * heads);
  if (BITS != 16) {
    // Workgroups go to the XCDs in turn: a run's heads to one of them, because rows
    // and scales of several heads may lie in a cache line of 128 bytes (codes of a
    // head side by side: 340 us, this 330 in 8 bits, 199 and 193 in 4; heads side by
    // side in 4 bits 387 and 277).
    const uint32_t of_runs = s.runs != 0 ? (uint32_t)s.runs : (uint32_t)s.a.n;
    if (block < of_runs / kXcds * kXcds * (uint32_t)heads) {
      const uint32_t i = block / kXcds, turn = i / (uint32_t)heads;
      run = turn * kXcds + block % kXcds;
      h = (int)(i - turn * (uint32_t)heads);
    }
  }
  const int n = (int)s.a.n;
  int64_t u = 0, end = 0;
  if (direct) {
    int32_t bad = 0;
    const int units = units_of(s, run, &bad);
    if (bad && threadIdx.x == 0) raise_status(s.a.d_status, bad);
    end = uniform(units);
  } else {
    scan_units(s, block, start, sums);
    const int64_t units = start[n];
    const int64_t runs = runs_of(s, units);
    if (run >= runs) return;
    u = uniform64(run_start(units, runs, run));
    end = uniform64(run_start(units, runs, run + 1));
  }
  int64_t part = 2 * run;
  while (u < end) {
    int64_t r = run;
    int c0 = 0, c1 = (int)end;
    bool whole = true;
    if (!direct) {
      int lo = 0, hi = n - 1;               // the request of unit u
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (uniform(start[mid + 1]) > u)
          hi = mid;
        else
          lo = mid + 1;
      }
      r = lo;
      const int first = uniform(start[lo]), count = uniform(start[lo + 1]) - first;
      c0 = (int)u - first;
      c1 = count - c0 < end - u ? count : c0 + (int)(end - u);
      whole = c0 == 0 && c1 == count;
    }
    attend<BITS, BF16, DIM, NT, ALIGNED, WAVES>(s, r, h, c0 * kUnit, c1 * kUnit,
                                                whole ? -1 : part * heads + h, lds);
    part = 2 * run + 1;
    u += c1 - c0;
  }
}

// How a call's requests of few rows are cut.
struct Plan {
  int tiles;            // of 16 rows
  int rows;             // bound on a request's rows
  int32_t runs;
  size_t starts, ml, total;   // workspace: bytes of the parts
};

Plan plan_of(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t bits,
             int32_t max_q, int32_t max_len);

// Workgroups of one tile of rows that fit a compute unit.  Rows of 32 bytes (64
// elements in 4 bits) leave room for three, which read a cache of 256 requests of
// 4000 keys, 8 heads, in 133 us, two in 161; rows of 64 bytes gain nothing (8 bits
// of 64 186 us both, 4 of 128 198 and 199), wider ones have no room.
constexpr int groups_per_cu(int bits, int dim) { return bits * dim == 256 ? 3 : 2; }
RowArgs args_of(const AttnCall& a, const Plan& p, void* workspace);

// Workgroups of a call: one for each run and head, or request and head.
inline int64_t groups_of(const AttnCall& a, const Plan& p) {
  return (p.runs != 0 ? p.runs : a.n) * a.kv_heads;
}

// The launch that joins cut requests, if any may be.
int join_rows(const RowArgs& s, const Plan& p, hipStream_t stream);

template <int BITS, bool BF16, int DIM, int NT, bool ALIGNED, int WAVES>
__global__ __launch_bounds__(WAVES * kWave,
                             NT == 1 && WAVES == kWaves ? groups_per_cu(BITS, DIM) : 2)
void attention_rows_kernel(RowArgs s) {
  __shared__ WaveLds<BITS, DIM, NT> lds[WAVES];
  __shared__ int32_t start[WAVES == kWaves ? kMostScanned + 1 : 1];
  __shared__ int32_t sums[kWaves];
  serve<BITS, BF16, DIM, NT, ALIGNED, WAVES>(s, blockIdx.x, lds, start, sums);
}

template <int BITS, bool BF16, int DIM>
int launch(const RowArgs& s, const Plan& p, hipStream_t stream) {
  const int64_t grid = groups_of(s.a, p);
  const bool aligned = s.page.d % 16 == 0;
  // Uncut workgroups that have a compute unit each: eight waves instead of four
  // (4 requests of 400 keys, 8 heads of 128: 6.8 us instead of 7.8, of 1000: 9.3
  // instead of 11.3; 32 requests, a workgroup for every unit: 22.1 both).
  const bool wide = p.runs == 0 && grid <= device_cu_count();
#define PAIR_ROWS(NT, AL, W)                                                                     \
  hipLaunchKernelGGL((attention_rows_kernel<BITS, BF16, DIM, NT, AL, W>),                         \
                     dim3((unsigned)grid), dim3(W * kWave), 0, stream, s)
#define PAIR_ROWS_OF(NT, AL)                                                                     \
  do {                                                                                           \
    if (wide) PAIR_ROWS(NT, AL, kWideWaves); else PAIR_ROWS(NT, AL, kWaves);                      \
  } while (0)
  if (p.tiles == 1) {
    if (aligned) PAIR_ROWS_OF(1, true); else PAIR_ROWS_OF(1, false);
  } else {
    if (aligned) PAIR_ROWS_OF(2, true); else PAIR_ROWS_OF(2, false);
  }
#undef PAIR_ROWS_OF
#undef PAIR_ROWS
  if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
  return join_rows(s, p, stream);
}

template <int BITS>
int launch_of(const RowArgs& s, const Plan& p, hipStream_t stream) {
  if (s.a.dim == 64)
    return s.a.bf16 ? launch<BITS, true, 64>(s, p, stream) : launch<BITS, false, 64>(s, p, stream);
  return s.a.bf16 ? launch<BITS, true, 128>(s, p, stream) : launch<BITS, false, 128>(s, p, stream);
}

// launch_of for caches of 8 and 4 bits (a file each).
int launch_mx8(const RowArgs& s, const Plan& p, hipStream_t stream);
int launch_mx4(const RowArgs& s, const Plan& p, hipStream_t stream);

}  // namespace rows

}  // namespace pair
