// Attention of a chunk of new tokens (prompts, chunks of prompts): tiles of 128
// rows -- a row is one query head of one token, and all rows of a tile share a
// key/value head -- against steps of 64 keys.  Bound by the matrix cores.
//
// A workgroup's four waves own 32 rows each.  Keys and values of a step go
// through LDS, two steps deep: while one is multiplied, the next is on its way
// from memory in registers, and one barrier a step suffices.
//   scores   S^T = K Q^T, so that a lane holds scores of one row only (keys
//            8 b + 4 h + e of a tile of 32, lane = row + 32 h): the row's maximum
//            and sum need one exchange between two lanes, and
//   weights  are, rounded, already the lane's entries of the B operand of
//   output   O^T += V^T P^T with the product's k index in that order.  The A
//            operand, four keys of one dim twice, is what the transposing LDS
//            read returns.
// LDS rows are stored with their 16-byte pieces permuted by the row number, so
// that neither the reads of K (32 rows at one place) nor those of V (four rows
// at two neighbouring places) meet in a bank.
// The maximum is raised only when a score exceeds it by 2^8 (attn_rows.hpp does
// the same), and steps that every row of a wave sees whole skip the masks.
//
// When the tiles are too few for the card, each tile's keys are split and a
// second launch joins the parts.
//
// Measured, in 4 * rows * keys * width operations that the masks leave, 32 query
// heads on 8 unless said: at width 128 one prompt of 16,384 tokens 980 TFLOP/s, 8
// chunks of 2048 after 8192 keys 980, three uneven ones after 4000 to 8000 keys 950,
// 8 prompts of 4096 (16 on 4) 870, 16 chunks of 64 over 4000 keys 690; at width 64
// the first two 875 and 860, 8 prompts of 301 to 4096 tokens (16 on 4) 710.  A
// product of two 8192^2 matrices by the library runs at 1250.  At width 128 the
// products and their LDS reads are what is left: a wave's 32 rows use each 1 KiB
// fragment once, and four SIMDs taking one every 32 cycles ask for all of LDS's 128
// bytes a cycle; left alone (no weights, no loads) they take 80% of the time, at
// clocks that the power limit sets.  At width 64 the exponentials (one per 256
// operations instead of 512) take the larger part.  Eight waves in two groups that
// alternate between products and weights, one workgroup a compute unit, reached 1050
// to 1100 on the longest chunks and lost 20 to 40% on 16 x 64 tokens and on single
// prompts, for which four stay.
#include <type_traits>

#include "attn_rows.hpp"

namespace pair {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRows = 32 * kWaves;          // of a tile
constexpr int kKeys = 64;                   // of a step
constexpr float kLazy = 8.0f;
constexpr int kClasses = 8;                 // of work, in the order of the tiles
// Requests that a workgroup orders itself.  Beyond 64 of them a lane holds four, and
// counting the tiles in a launch before is as fast or faster (16 on 4 heads, 30 to
// 128 tokens after 300, at width 64 and 128: 65 requests 26.6 and 49.5 us ordered,
// 27.6 and 48.4 counted; 130 requests 47.7 and 83, 45.7 and 76; 256 requests 83 and
// 158, 75 and 147).
constexpr int kInline = 256;

// kinds of instructions in a scheduling group
constexpr int kMfma = 0x8, kDsRead = 0x100;

typedef short s16x4_t __attribute__((ext_vector_type(4)));

struct TileArgs {
  AttnCall a;
  FastDiv page, group;
  float scale_log2;
  int32_t least;        // requests of fewer rows are left to the other kernel
  int32_t splits;
  int32_t* starts;      // [n + 1] tiles before each request, if n > kInline
  float* part_o;        // [tokens][q_heads][splits][dim]
  float* part_ml;       // [tokens][q_heads][splits][2]
};

__device__ __forceinline__ int tiles_of(const TileArgs& s, int64_t r, int32_t* bad) {
  Request q;
  if (!attention_request(s.a, s.page.d, r, &q, bad)) return 0;
  const int64_t rows = (int64_t)q.tokens * s.group.d;
  return rows < s.least ? 0 : (int)((rows + kRows - 1) / kRows);
}

// Tiles before each request, for the calls of many requests.
__global__ __launch_bounds__(1024) void tile_starts_kernel(TileArgs s) {
  __shared__ int32_t ends[1024 / kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int32_t carry = 0, bad = 0;
  for (int64_t r0 = 0; r0 < s.a.n; r0 += 1024) {
    const int64_t r = r0 + threadIdx.x;
    int32_t scan = r < s.a.n ? tiles_of(s, r, &bad) : 0;
#pragma unroll
    for (int by = 1; by < kWave; by <<= 1) {
      const int32_t v = __shfl_up(scan, by, kWave);
      if (lane >= by) scan += v;
    }
    if (lane == kWave - 1) ends[wave] = scan;
    __syncthreads();
    int32_t all = 0;
#pragma unroll
    for (int w = 0; w < 1024 / kWave; ++w) {
      if (w < wave) scan += ends[w];
      all += ends[w];
    }
    if (r < s.a.n) s.starts[r + 1] = carry + scan;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) s.starts[0] = 0;
  if (bad) raise_status(s.a.d_status, bad);
}

__device__ __forceinline__ int wave_sum_i(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) +
         __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
}

__device__ __forceinline__ int wave_scan_i(int v) {   // inclusive
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Tile `at` of the call: the request, and the tile's number in it; false past the
// last.  Every wave holds the requests in its lanes, SETS each.  The order is by
// falling work, so that the last workgroups to start are the shortest, but only
// in kClasses classes of the keys seen: within a class request by request, so
// that the workgroups that run at one time share a request's keys in their
// caches.  (8 prompts of 300 to 4096 tokens at width 64: 157 us in the order of
// the requests, 147 us strictly by work, 151 us so.  8 chunks of 2048 tokens over
// 8192 keys, 16 heads of width 128: 1441 us strictly by work, 1300 us so; 4 or 16
// classes differ from 8 by 1 to 3% either way.)  A request's tiles of a class are
// counted in closed form.  A workgroup takes 2 us for this beside others' work.
template <int SETS>
__device__ __forceinline__ bool find_ordered(const TileArgs& s, int64_t at, Request* q,
                                             int64_t* request, int* tile) {
  const int n = (int)s.a.n, lane = threadIdx.x & (kWave - 1);
  Request own[SETS];
  int tiles[SETS];
  int32_t bad = 0;
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    const int r = i * kWave + lane;
    own[i] = Request{0, 0, 0};
    tiles[i] = 0;
    if (r < n && attention_request(s.a, s.page.d, r, &own[i], &bad)) {
      const int rows = own[i].tokens * (int)s.group.d;
      if (rows >= s.least) tiles[i] = (rows + kRows - 1) / kRows;
    }
  }
  if (bad && at == 0 && threadIdx.x < kWave) raise_status(s.a.d_status, bad);
  const int steps = (s.a.max_len + kKeys - 1) / kKeys;
  const int each = (steps + kClasses - 1) / kClasses;
  // tiles of set i's request of class c or a longer one (class 0: of any length)
  auto from_class = [&](int i, int c) {
    int token = c * each * kKeys - (own[i].len - own[i].tokens);   // first that sees more
    if (token < 0 || c == 0) token = 0;
    const int before = (token < own[i].tokens ? token : own[i].tokens) * (int)s.group.d / kRows;
    return token < own[i].tokens ? tiles[i] - before : 0;
  };
  int totals[kClasses + 1];                 // side by side: each is a chain of lane exchanges
#pragma unroll
  for (int c = 0; c < kClasses; ++c) {
    int v = 0;
#pragma unroll
    for (int i = 0; i < SETS; ++i) v += tiles[i] > 0 ? from_class(i, c) : 0;
    totals[c] = wave_sum_i(v);
  }
  totals[kClasses] = 0;
  if (at >= totals[0]) return false;
  int cls = 0, ahead = totals[1];           // tiles of longer classes
#pragma unroll
  for (int c = 1; c < kClasses; ++c)
    if (at < totals[c]) {
      cls = c;
      ahead = totals[c + 1];
    }
  int left = (int)at - ahead;
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    const int longer = tiles[i] > 0 && cls + 1 < kClasses ? from_class(i, cls + 1) : 0;
    const int mine = tiles[i] > 0 ? from_class(i, cls) - longer : 0;
    const int scan = wave_scan_i(mine);
    const int all = __builtin_amdgcn_readlane(scan, kWave - 1);
    if (left >= all) {
      left -= all;
      continue;
    }
    const int x = uniform(__popcll(__ballot(scan <= left)));
    *request = i * kWave + x;
    *tile = __builtin_amdgcn_readlane(tiles[i] - longer - 1 + scan - mine, x) - left;
    q->tokens = __builtin_amdgcn_readlane(own[i].tokens, x);
    q->len = __builtin_amdgcn_readlane(own[i].len, x);
    q->q0 = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane(
                           (int)(uint32_t)((uint64_t)own[i].q0 >> 32), x) << 32) |
                      (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)own[i].q0, x));
    return true;
  }
  return false;
}

// The same for more requests, from the tiles counted before each, and only in
// the order of the last tile first: with so many of them the ends even out.
__device__ __forceinline__ bool find_counted(const TileArgs& s, int64_t back, Request* q,
                                             int64_t* request, int* tile) {
  const int n = (int)s.a.n;
  const int64_t t = (int64_t)s.starts[n] - 1 - back;
  if (t < 0) return false;
  int lo = 0, hi = n;                       // starts[lo] <= t < starts[hi]
  while (hi - lo > 1) {
    const int step = (hi - lo + kThreads - 1) / kThreads;
    const int at = lo + ((int)threadIdx.x + 1) * step;
    const int below = __syncthreads_count(at < hi && s.starts[at] <= t);
    const int top = lo + (below + 1) * step;
    lo += below * step;
    hi = top < hi ? top : hi;
  }
  *request = uniform(lo);
  *tile = uniform((int)(t - s.starts[lo]));
  int32_t bad = 0;
  return attention_request(s.a, s.page.d, lo, q, &bad);
}

// 16-byte piece `c` of LDS row `row` of a step's keys, and of its values.
template <int DIM>
__device__ __forceinline__ int key_piece(int row, int c) {
  const int f = DIM == 128 ? row & 15 : (row >> 1) & 7;   // two rows of 64 fill the banks
  return row * (DIM * 2) + ((c ^ f) << 4);
}
template <int DIM>
__device__ __forceinline__ int value_piece(int row, int c) {
  const int f = DIM == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
  return row * (DIM * 2) + ((c ^ f) << 4);
}

// A step whose values are not all finite, and not all seen by every row: a
// weight of zero would not keep a NaN or an infinity out of the matrix
// product.  The weights go through LDS (over the keys, which are done with)
// and each row adds the values that it sees, one key at a time.
template <bool BF16, int DIM>
__device__ __forceinline__ void add_odd_step(unsigned char* keys, unsigned char* values,
                                             const u32x4_t (&pf)[4], int kb, int limit,
                                             f32x16_t (*acc)[DIM / 32]) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int x = lane & 31, h = lane >> 5;
  uint32_t* weights = reinterpret_cast<uint32_t*>(keys) + (wave * 32 + x) * (kKeys / 2);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int w = 0; w < 4; ++w) weights[8 * u + 4 * (w >> 1) + 2 * h + (w & 1)] = pf[u][w];
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < kKeys; ++k) {
    const float p = half_value<BF16>((weights[k >> 1] >> (16 * (k & 1))) & 0xffffu);
    const bool seen = kb + k <= limit;
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const u32x2_t v = *reinterpret_cast<const u32x2_t*>(
            values + value_piece<DIM>(k, 4 * d + b) + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (seen)
            (*acc)[d][4 * b + e] = __builtin_fmaf(
                p, half_value<BF16>((v[e >> 1] >> (16 * (e & 1))) & 0xffffu), (*acc)[d][4 * b + e]);
      }
  }
  __syncthreads();
  for (int b = threadIdx.x * 16; b < kKeys * DIM * 2; b += kThreads * 16)
    *reinterpret_cast<u32x4_t*>(values + b) = u32x4_t{0u, 0u, 0u, 0u};
  __syncthreads();
}

// One workgroup's tile, `block` its place in the order.
template <bool BF16, int DIM, bool ALIGNED>
__device__ __forceinline__ void attend_tile(const TileArgs& s, uint32_t block,
                                            unsigned char (&kt)[2][kKeys * DIM * 2],
                                            unsigned char (&vt)[2][kKeys * DIM * 2]) {
  constexpr int NC = DIM / 16;              // k pieces of a score product
  constexpr int ND = DIM / 32;              // dim tiles of the output
  constexpr int kPer = DIM / 8;             // 16-byte pieces of a row
  constexpr int kStage = kKeys * kPer / kThreads;   // pieces of a lane per step
  constexpr int kStep = kThreads / kPer;    // rows between a lane's pieces
  // add_odd_step lays 16 KiB of weights over both key steps
  static_assert(kRows * kKeys * 2 <= 2 * kKeys * DIM * 2, "weights of a step");

  // heads fastest: consecutive workgroups go to the XCDs in turn, so that with
  // 8 (4, 2) key heads each XCD's cache holds one (two, four) of them
  const uint32_t heads = (uint32_t)s.a.kv_heads, splits = (uint32_t)s.splits;
  const uint32_t of_heads = block / heads;   // 32 bits: a long division takes 0.3 us
  const int kvh = (int)(block - of_heads * heads);
  const int split = (int)(of_heads % splits);
  int64_t r;
  int tile;
  Request q;
  __builtin_amdgcn_s_setprio(2);            // until it takes its share of the work
  const int64_t place_in_order = of_heads / splits;
  if (s.a.n <= kWave) {
    if (!find_ordered<1>(s, place_in_order, &q, &r, &tile)) return;
  } else if (s.a.n <= kInline) {
    if (!find_ordered<kInline / kWave>(s, place_in_order, &q, &r, &tile)) return;
  } else if (!find_counted(s, place_in_order, &q, &r, &tile)) {
    return;
  }
  const int rows = q.tokens * (int)s.group.d;
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int x = lane & 31, h = lane >> 5;

  // this lane's row, and the keys that the wave and the tile see
  const int i = tile * kRows + wave * 32 + x;
  const int tok = (int)div_by((uint32_t)i, s.group);
  const int qh = kvh * (int)s.group.d + i - tok * (int)s.group.d;
  const int limit = i < rows ? limit_of(q, tok) : -1;
  const int i_first = tile * kRows + wave * 32;
  const int first_limit = limit_of(q, (int)div_by((uint32_t)i_first, s.group));
  int i_last = tile * kRows + kRows - 1;
  if (i_last >= rows) i_last = rows - 1;
  int keys = limit_of(q, (int)div_by((uint32_t)i_last, s.group)) + 1;
  if (keys < 0) keys = 0;
  int k0 = 0, k1 = keys;
  if (s.splits > 1) {
    const int part = ((keys + s.splits - 1) / s.splits + kKeys - 1) / kKeys * kKeys;
    k0 = split * part < keys ? split * part : keys;
    k1 = k0 + part < keys ? k0 + part : keys;
  }

  u32x4_t qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) qf[c] = u32x4_t{0u, 0u, 0u, 0u};
  if (i < rows) {
    const uint16_t* p = static_cast<const uint16_t*>(s.a.q) + (q.q0 + tok) * s.a.q_token +
                        qh * s.a.q_head + h * 8;
#pragma unroll
    for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const u32x4_t*>(p + c * 16);
  }
  f32x16_t acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;            // l: this lane's keys only

  const int64_t head = kvh * s.a.cache.head_stride * 2;
  const unsigned char* kbase = static_cast<const unsigned char*>(s.a.k_cache) + head;
  const unsigned char* vbase = static_cast<const unsigned char*>(s.a.v_cache) + head;
  const int64_t slot_bytes = s.a.cache.slot_stride * 2, page_bytes = s.a.cache.page_stride * 2;
  const int32_t* table = s.a.table + r * s.a.ldt;
  const int my_row = (int)threadIdx.x / kPer, my_piece = (int)threadIdx.x % kPer;
  constexpr int kWaveRows = kWave / kPer;   // rows of a wave's load: within 16 aligned ones
  int32_t bad_page = 0;
  auto place = [&](int key, int32_t id) {   // byte offset of a key
    const uint32_t pg = div_by((uint32_t)key, s.page);
    return checked_page(s.a, id, &bad_page) * page_bytes +
           (int64_t)((uint32_t)key - pg * s.page.d) * slot_bytes;
  };

  // Where the keys lie.  ALIGNED (pages of a multiple of 16 keys): 16 aligned
  // keys share a page, and lane x of the wave holds the place of 16-key group x
  // of a window of 1024 keys; a fetch reads it from the lane, and the loads take
  // a scalar base.  The next window's pages are loaded a window ahead.  Else
  // each lane looks its rows up a step ahead.
  constexpr int kWindow = 16 * kWave;
  u32x4_t ks[kStage], vs[kStage];
  int32_t id[ALIGNED ? 1 : kStage];
  int64_t group_at = 0;
  int window = k0;
  const uint32_t lane_off =
      my_piece * 16 + (ALIGNED ? (uint32_t)((my_row & 15) * slot_bytes) : 0u);
  auto row_key = [&](int kb, int p) {       // one past the end repeats the last
    const int key = ALIGNED ? kb + 16 * lane : kb + p * kStep + my_row;
    return key < q.len ? key : (ALIGNED ? (q.len - 1) & ~15 : q.len - 1);
  };
  auto lookup = [&](int kb) {
#pragma unroll
    for (int p = 0; p < (ALIGNED ? 1 : kStage); ++p)
      id[p] = table[div_by((uint32_t)row_key(kb, p), s.page)];
  };
  auto fetch = [&](int kb) {
    if (ALIGNED && kb - window == kWindow) {
      window = kb;
      group_at = place(row_key(kb, 0), id[0]);
      lookup(kb + kWindow);
    }
#pragma unroll
    for (int p = 0; p < kStage; ++p) {
      int64_t at;
      if (ALIGNED) {
        const int x16 = ((kb - window) >> 4) + ((p * kStep + wave * kWaveRows) >> 4);
        const uint32_t lo =
            (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)group_at, x16);
        const uint32_t hi =
            (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)group_at >> 32), x16);
        at = (int64_t)(((uint64_t)hi << 32) | lo);
      } else {
        at = place(row_key(kb, p), id[ALIGNED ? 0 : p]);
      }
      ks[p] = *reinterpret_cast<const u32x4_t*>(kbase + at + lane_off);
      vs[p] = *reinterpret_cast<const u32x4_t*>(vbase + at + lane_off);
    }
    if (!ALIGNED) lookup(kb + kKeys);
  };

  // Offsets in LDS; a step's buffer and the rows' higher parts are constants.
  int k_in, v_in, k_out[NC], v_out[ND];
  k_in = key_piece<DIM>(my_row, my_piece);
  v_in = value_piece<DIM>(my_row, my_piece);
#pragma unroll
  for (int c = 0; c < NC; ++c) k_out[c] = key_piece<DIM>(x, 2 * c + h);
#pragma unroll
  for (int d = 0; d < ND; ++d)
    v_out[d] = value_piece<DIM>(4 * h + ((lane & 15) >> 2),
                                4 * d + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) +
               (lane & 1) * 8;

  const int tile_limit = limit_of(q, (int)div_by((uint32_t)(tile * kRows), s.group));
  auto step = [&](int kb, auto buffer) {
    constexpr int buf = decltype(buffer)::value;
    // Into LDS, and a barrier.  `odd`: a step that some row of the tile does not
    // see whole holds a value that is not finite.
    const bool edge = kb + kKeys - 1 > tile_limit;
    bool odd = false;
    if (edge) {
      uint32_t bad = 0;
#pragma unroll
      for (int p = 0; p < kStage; ++p) {
        if (kb + p * kStep + my_row >= q.len) vs[p] = u32x4_t{0u, 0u, 0u, 0u};   // no value at all
#pragma unroll
        for (int w = 0; w < 4; ++w) bad |= not_finite<BF16>(vs[p][w]) ? 1u : 0u;
      }
      odd = __syncthreads_or((int)bad) != 0;
    }
#pragma unroll
    for (int p = 0; p < kStage; ++p) {
      *reinterpret_cast<u32x4_t*>(kt[buf] + p * kStep * DIM * 2 + k_in) = ks[p];
      *reinterpret_cast<u32x4_t*>(vt[buf] + p * kStep * DIM * 2 + v_in) = vs[p];
    }
    __syncthreads();
    if (kb + kKeys < k1) fetch(kb + kKeys);

    f32x16_t sc[2];
    __builtin_amdgcn_s_setprio(1);          // over a wave that is at its softmax
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[t][e] = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4_t kf =
            *reinterpret_cast<const u32x4_t*>(kt[buf] + 32 * t * DIM * 2 + k_out[c]);
        sc[t] = mma32<BF16>(kf, qf[c], sc[t]);
      }
    // four reads ahead of the products
    __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
#pragma unroll
    for (int i = 0; i < 2 * NC - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMfma, 4, 0);
    __builtin_amdgcn_s_setprio(0);
    if (kb + kKeys - 1 > first_limit) {
      const int last = limit - kb - 4 * h;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sc[t][e] = 32 * t + 8 * (e >> 2) + (e & 3) > last ? -INFINITY : sc[t][e];
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[t][e]);
    top *= s.scale_log2;
    if (__any(top > m + kLazy)) {
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float mn = fmaxf(m, top);
      const float keep = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= keep;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] *= keep;
    }
    const float base = (m == -INFINITY ? 0.0f : m) - kLift<BF16>;
    u32x4_t pf[4];
    float part = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const float a =
            __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][2 * w], s.scale_log2, -base));
        const float b =
            __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][2 * w + 1], s.scale_log2, -base));
        part += a + b;
        pf[2 * t + (w >> 2)][w & 3] = pack2<BF16>(a, b);
      }
    l += part;
    if (odd) add_odd_step<BF16, DIM>(kt[0], vt[buf], pf, kb, limit, &acc);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < 4; ++u)             // 16 keys at a time
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        u32x4_t vf;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4_t*)(vt[buf] +
                                                            (16 * u + 8 * half) * DIM * 2 +
                                                            v_out[d]));
          const u32x2_t b = __builtin_bit_cast(u32x2_t, v);
          vf[2 * half] = b[0];
          vf[2 * half + 1] = b[1];
        }
        acc[d] = mma32<BF16>(vf, pf[u], acc[d]);
      }
    __builtin_amdgcn_sched_group_barrier(kDsRead, 8, 0);
#pragma unroll
    for (int i = 0; i < 4 * ND - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMfma, 4, 0);
    __builtin_amdgcn_s_setprio(0);
  };

  if (k0 < k1) {
    lookup(k0);
    if (ALIGNED) {
      group_at = place(row_key(k0, 0), id[0]);
      lookup(k0 + kWindow);
    }
    fetch(k0);
  }
  __builtin_amdgcn_s_setprio(0);
  for (int kb = k0; kb < k1; kb += 2 * kKeys) {
    step(kb, std::integral_constant<int, 0>());
    if (kb + kKeys < k1) step(kb + kKeys, std::integral_constant<int, 1>());
  }

  if (bad_page) raise_status(s.a.d_status, bad_page);
  l += __shfl_xor(l, 32, kWave);
  if (i >= rows) return;
  const int64_t row = (q.q0 + tok) * s.a.q_heads + qh;
  if (s.splits > 1) {
    const int64_t at = row * s.splits + split;
    if (h == 0) {
      s.part_ml[2 * at] = m;
      s.part_ml[2 * at + 1] = l;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<f32x4_t*>(s.part_o + at * DIM + 32 * d + 8 * b + 4 * h) =
            f32x4_t{acc[d][4 * b], acc[d][4 * b + 1], acc[d][4 * b + 2], acc[d][4 * b + 3]};
    return;
  }
  const bool none = limit < 0;
  const float inv = 1.0f / l;
  uint16_t* o = static_cast<uint16_t*>(s.a.out) + (q.q0 + tok) * s.a.out_token + qh * s.a.out_head;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      u32x2_t w;
      w[0] = none ? 0u : pack2<BF16>(acc[d][4 * b] * inv, acc[d][4 * b + 1] * inv);
      w[1] = none ? 0u : pack2<BF16>(acc[d][4 * b + 2] * inv, acc[d][4 * b + 3] * inv);
      *reinterpret_cast<u32x2_t*>(o + 32 * d + 8 * b + 4 * h) = w;
    }
  if (s.a.lse != nullptr && h == 0)
    s.a.lse[row] = none ? -INFINITY : log_sum<BF16>(m, l);
}

template <bool BF16, int DIM, bool ALIGNED>
__global__ __launch_bounds__(kThreads, DIM == 64 ? 3 : 2) void attention_tiles_kernel(TileArgs s) {
  __shared__ __align__(16) unsigned char kt[2][kKeys * DIM * 2];   // a step's keys, twice
  __shared__ __align__(16) unsigned char vt[2][kKeys * DIM * 2];
  attend_tile<BF16, DIM, ALIGNED>(s, blockIdx.x, kt, vt);
}

// What a call's requests of few rows add to the arguments.
struct FewArgs {
  int32_t runs;
  int32_t* starts;
  float* part_o;
  float* part_ml;
};

// A call that may hold requests of few rows, too: `few` workgroups for those and
// `tiles` for the others, the first kDealt of each in turn, so that the reading of
// a long cache and the products run on a compute unit at the same time.
constexpr uint32_t kDealt = 256;

template <bool BF16, int DIM, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void attention_mixed_kernel(TileArgs s, FewArgs w,
                                                                      uint32_t few, uint32_t tiles) {
  struct FewLds {
    rows::WaveLds<DIM, 2> wave[rows::kWaves];
    int32_t start[rows::kMostScanned + 1];
    int32_t sums[rows::kWaves];
  };
  struct StepLds {
    unsigned char k[2][kKeys * DIM * 2], v[2][kKeys * DIM * 2];
  };
  __shared__ __align__(16) union {
    FewLds few;
    StepLds step;
  } lds;
  const uint32_t b = blockIdx.x;
  const uint32_t few_first = few < kDealt ? few : kDealt;
  const uint32_t first = few_first + (tiles < kDealt ? tiles : kDealt);
  if (b >= few_first && (b < first || b >= first + few - few_first)) {
    attend_tile<BF16, DIM, ALIGNED>(s, b < first ? b - few_first : b - few, lds.step.k,
                                    lds.step.v);
  } else {
    rows::RowArgs f;
    f.a = s.a;
    f.page = s.page;
    f.group = s.group;
    f.scale_log2 = s.scale_log2;
    f.runs = w.runs;
    f.starts = w.starts;
    f.part_o = w.part_o;
    f.part_ml = w.part_ml;
    rows::serve<BF16, DIM, 2, ALIGNED, rows::kWaves>(
        f, b < few_first ? b : b - first + few_first, lds.few.wave, lds.few.start, lds.few.sums);
  }
}

// Joins a row's parts: one wave a row.
template <bool BF16, int DIM>
__global__ __launch_bounds__(kThreads) void join_tiles_kernel(TileArgs s) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t row = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x / kWave);
  const int64_t t = (uint32_t)row / (uint32_t)s.a.q_heads;   // rows: below 2^31
  const int qh = (int)(row - t * s.a.q_heads);
  if (t >= s.a.tokens) return;
  int64_t lo = 0, hi = s.a.n - 1;           // the token's request
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (s.a.q_offsets[mid + 1] > t)
      hi = mid;
    else
      lo = mid + 1;
  }
  Request q;
  int32_t bad = 0;
  if (!attention_request(s.a, s.page.d, lo, &q, &bad)) return;
  if (t < q.q0 || t >= q.q0 + q.tokens || (int64_t)q.tokens * s.group.d < s.least) return;
  constexpr int PER = DIM / kWave;
  const int64_t at = row * s.splits;
  float m = -INFINITY;
  for (int p = 0; p < s.splits; ++p) m = fmaxf(m, s.part_ml[2 * (at + p)]);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.0f;
  for (int p = 0; p < s.splits; ++p) {
    const float mp = s.part_ml[2 * (at + p)], lp = s.part_ml[2 * (at + p) + 1];
    if (mp == -INFINITY && lp == 0.0f) continue;          // saw no key
    const float f = __builtin_amdgcn_exp2f(mp - base);
    l = __builtin_fmaf(lp, f, l);
#pragma unroll
    for (int e = 0; e < PER; ++e)
      o[e] = __builtin_fmaf(s.part_o[(at + p) * DIM + lane * PER + e], f, o[e]);
  }
  const bool none = limit_of(q, (int)(t - q.q0)) < 0;
  const float inv = 1.0f / l;
  uint16_t* to = static_cast<uint16_t*>(s.a.out) + t * s.a.out_token + qh * s.a.out_head;
  if (PER == 2) {
    *reinterpret_cast<uint32_t*>(to + 2 * lane) =
        none ? 0u : pack2<BF16>(o[0] * inv, o[PER - 1] * inv);
  } else {
    to[lane] = none ? (uint16_t)0 : (uint16_t)pack2<BF16>(o[0] * inv, 0.0f);
  }
  if (s.a.lse != nullptr && lane == 0)
    s.a.lse[row] = none ? -INFINITY : log_sum<BF16>(m, l);
}

struct Plan {
  int64_t tiles;        // bound on the tiles of one head
  int32_t splits;
  size_t starts, ml, total;
};

Plan plan_tiles(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim,
                int32_t max_len) {
  Plan p;
  p.tiles = tokens * (q_heads / kv_heads) / kRows + (n < tokens ? n : tokens);
  // Two workgroups fit a compute unit.  Fewer tiles than that are split along
  // the keys, down to eight steps a part.
  const int64_t slots = 2 * (int64_t)device_cu_count();
  int64_t split = slots / (p.tiles * kv_heads > 0 ? p.tiles * kv_heads : 1);
  const int64_t most = ((int64_t)max_len + 8 * kKeys - 1) / (8 * kKeys);
  if (split > most) split = most;
  if (split > 32) split = 32;
  p.splits = (int32_t)(split < 1 ? 1 : split);
  p.starts = n > kInline ? ((size_t)(n + 1) * 4 + 255) / 256 * 256 : 0;
  const size_t parts = p.splits > 1 ? (size_t)tokens * q_heads * p.splits : 0;
  p.ml = (parts * 8 + 255) / 256 * 256;
  p.total = p.starts + p.ml + parts * dim * 4 + 256;
  return p;
}

// `w` (or null): the requests of few rows, served by the same launch.
template <bool BF16, int DIM>
int launch(const TileArgs& s, const Plan& p, const rows::RowArgs* w, const rows::Plan* wp,
           hipStream_t stream) {
  const int64_t grid = p.tiles * s.a.kv_heads * p.splits;
  const int64_t few = w != nullptr ? rows::groups_of(s.a, *wp) : 0;
  if (s.a.n > kInline) {
    hipLaunchKernelGGL(tile_starts_kernel, dim3(1), dim3(1024), 0, stream, s);
    if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
  }
  // 16 slots within 32 bits of offset: any sensible layout
  const bool aligned = s.page.d % 16 == 0 && s.a.cache.slot_stride < ((int64_t)1 << 26);
#define PAIR_TILES(AL)                                                                           \
  do {                                                                                           \
    if (w != nullptr)                                                                            \
      hipLaunchKernelGGL((attention_mixed_kernel<BF16, DIM, AL>), dim3((unsigned)(grid + few)),   \
                         dim3(kThreads), 0, stream, s,                                            \
                         (FewArgs{w->runs, w->starts, w->part_o, w->part_ml}), (uint32_t)few,    \
                         (uint32_t)grid);                                                        \
    else                                                                                         \
      hipLaunchKernelGGL((attention_tiles_kernel<BF16, DIM, AL>), dim3((unsigned)grid),           \
                         dim3(kThreads), 0, stream, s);                                          \
  } while (0)
  if (aligned) PAIR_TILES(true); else PAIR_TILES(false);
#undef PAIR_TILES
  if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
  if (w != nullptr) {
    const int rc = rows::join_rows(*w, *wp, stream);
    if (rc != PAIR_OK) return rc;
  }
  if (p.splits > 1) {
    const int64_t rows = s.a.tokens * s.a.q_heads;
    hipLaunchKernelGGL((join_tiles_kernel<BF16, DIM>), dim3((unsigned)((rows + kWaves - 1) / kWaves)),
                       dim3(kThreads), 0, stream, s);
  }
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace

size_t attention_tiles_workspace(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                                 int32_t dim, int32_t max_len) {
  return plan_tiles(n, tokens, q_heads, kv_heads, dim, max_len).total;
}

int64_t attention_tiles_groups(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                               int32_t dim, int32_t max_len) {
  const Plan p = plan_tiles(n, tokens, q_heads, kv_heads, dim, max_len);
  const int64_t grid = p.tiles * kv_heads * p.splits;
  const int64_t joins = p.splits > 1 ? (tokens * q_heads + kWaves - 1) / kWaves : 0;
  return grid > joins ? grid : joins;
}

int launch_attention_tiles(const AttnCall& a, int32_t least_rows, void* few_workspace,
                           void* workspace, hipStream_t stream) {
  const Plan p = plan_tiles(a.n, a.tokens, a.q_heads, a.kv_heads, a.dim, a.max_len);
  TileArgs s;
  s.a = a;
  s.page = fast_div((uint32_t)a.cache.page);
  s.group = fast_div((uint32_t)(a.q_heads / a.kv_heads));
  s.scale_log2 = a.scale * 1.44269504089f;
  s.least = least_rows;
  s.splits = p.splits;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  s.starts = reinterpret_cast<int32_t*>(ws);
  s.part_ml = reinterpret_cast<float*>(ws + p.starts);
  s.part_o = reinterpret_cast<float*>(ws + p.starts + p.ml);
  rows::RowArgs w;
  rows::Plan wp;
  if (few_workspace != nullptr) {
    wp = rows::plan_of(a.n, a.q_heads, a.kv_heads, a.dim, a.max_q, a.max_len);
    w = rows::args_of(a, wp, few_workspace);
  }
  const rows::RowArgs* few = few_workspace != nullptr ? &w : nullptr;
  if (a.dim == 64)
    return a.bf16 ? launch<true, 64>(s, p, few, &wp, stream)
                  : launch<false, 64>(s, p, few, &wp, stream);
  return a.bf16 ? launch<true, 128>(s, p, few, &wp, stream)
                : launch<false, 128>(s, p, few, &wp, stream);
}

}  // namespace pair
