// Paged key/value cache: one step's block tables, slot map and page pool from
// request lengths (pair_page_plan), and the new keys and values into their
// slots (pair_cache_store).
#include "paged.hpp"

namespace pair {

namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------- plan --
// Three exclusive scans over the requests (new tokens, pages taken, pages
// given back) settle everything; each output element then finds its request
// by bisection of the scans' ends.  Bound by launches and by loads that wait for
// each other, not by bytes: 64 requests 4.4 us; 16,896 requests with half of
// them released, 1.1M tokens, 4 + 6 + 13 us (of 16 MB: 3 us at the rate of a
// copy).  Sums saturate at 2^31 - 1, beyond every capacity; saturating addition
// of counts is associative, so the scans may be split anywhere.
struct PlanArgs {
  int64_t n;
  const int32_t* cached;
  const int32_t* fresh;
  const uint8_t* mask;
  FastDiv page;
  int32_t* table;
  int64_t ldt;
  int32_t capacity;
  const int32_t* free_pages;
  const int64_t* free_count;
  int32_t max_tokens;
  int64_t* q_offsets;
  int32_t* lens;
  int64_t* slots;
  int32_t* positions;
  int32_t* free_out;
  int64_t* free_count_out;
  int32_t* d_status;
};

struct Counts {
  uint32_t tokens, taken, given;
};

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) {
  const uint32_t s = a + b;                     // both at most 2^31 - 1
  return s < 0x7fffffffu ? s : 0x7fffffffu;
}

__device__ __forceinline__ Counts operator+(const Counts& a, const Counts& b) {
  return Counts{sat_add(a.tokens, b.tokens), sat_add(a.taken, b.taken),
                sat_add(a.given, b.given)};
}

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, const FastDiv& page) {
  return tokens == 0 ? 0u : div_by(tokens - 1, page) + 1;
}

// What a request takes and gives, and its length after the step in *len (no
// branches: the loads before it are then in flight together).
__device__ __forceinline__ Counts counts_of(const PlanArgs& a, int32_t c, int32_t f, bool live,
                                            int32_t* len, int32_t* bad) {
  const bool sane = (c | f) >= 0 && (uint32_t)c + (uint32_t)f <= 0x7fffffffu;
  const uint32_t cached = sane ? (uint32_t)c : 0u, fresh = sane ? (uint32_t)f : 0u;
  const uint32_t held = pages_of(cached, a.page);
  const uint32_t all = live ? pages_of(cached + fresh, a.page) : held;
  const bool fits = (int64_t)all <= a.ldt;
  *bad |= sane ? (fits ? 0 : PAIR_ST_PAGES) : PAIR_ST_LENGTH;
  const bool goes = sane && fits && live;
  *len = goes ? (int32_t)(cached + fresh) : 0;
  return Counts{goes ? fresh : 0u, goes ? all - held : 0u, sane && fits && !live ? held : 0u};
}

__device__ __forceinline__ Counts request(const PlanArgs& a, int64_t r, int32_t* len,
                                          int32_t* bad) {
  return counts_of(a, a.cached[r], a.fresh[r], a.mask == nullptr || a.mask[r] != 0, len, bad);
}

__device__ __forceinline__ Counts shfl_up(const Counts& v, int by) {
  return Counts{(uint32_t)__shfl_up((int)v.tokens, by, kWave),
                (uint32_t)__shfl_up((int)v.taken, by, kWave),
                (uint32_t)__shfl_up((int)v.given, by, kWave)};
}

// Inclusive scan over a workgroup of NT threads; *total the sum of all.
template <int NT>
__device__ __forceinline__ Counts group_scan(Counts v, Counts* total) {
  __shared__ Counts ends[NT / kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
  for (int by = 1; by < kWave; by <<= 1) {
    const Counts u = shfl_up(v, by);
    if (lane >= by) v = v + u;
  }
  if (lane == kWave - 1) ends[wave] = v;
  __syncthreads();
  Counts before = {0u, 0u, 0u}, all = {0u, 0u, 0u};
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) {
    if (w < wave) before = before + ends[w];
    all = all + ends[w];
  }
  __syncthreads();
  *total = all;
  return before + v;
}

// The scans' ends (inclusive sums), in LDS or in the workspace.
struct Ends {
  const uint32_t* tokens;
  const uint32_t* taken;
  const uint32_t* given;
};

// First request of [lo, hi] whose end is beyond x (hi if none before it is).
__device__ __forceinline__ int owner(const uint32_t* ends, uint32_t x, int lo, int hi) {
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > x)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// The same for two numbers by a whole wave, 64 probes of each at a time.
__device__ __forceinline__ void wave_owners(const uint32_t* ends, uint32_t x, uint32_t y, int last,
                                            int32_t* out) {
  const int lane = threadIdx.x & (kWave - 1);
  int lo[2] = {0, 0}, hi[2] = {last, last};
  const uint32_t want[2] = {x, y};
  while (lo[0] < hi[0] || lo[1] < hi[1]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int step = (hi[k] - lo[k] + kWave - 1) / kWave;
      const int i = lo[k] + lane * step;
      const int below = __popcll(__ballot(i < hi[k] && ends[i < hi[k] ? i : 0] <= want[k]));
      if (below == 0) {
        hi[k] = lo[k];
      } else {
        const int top = lo[k] + below * step;
        lo[k] += (below - 1) * step + 1;
        hi[k] = top < hi[k] ? top : hi[k];
      }
    }
  }
  if (lane < 2) out[lane] = lane == 0 ? lo[0] : lo[1];
}

__device__ __forceinline__ uint32_t free_pages_of(const PlanArgs& a) {
  const int64_t f = *a.free_count;
  return f < 0 ? 0u : (f > a.capacity ? (uint32_t)a.capacity : (uint32_t)f);
}

constexpr int kOwn = 4;               // outputs of a thread: searched and loaded side by side
constexpr int kTile = kOwn * kThreads;
constexpr int kNear = 512;            // requests that a tile keeps in LDS

// A scan's ends over the requests [lo, hi] that a tile needs: in LDS where they
// fit, else where they were.
struct Near {
  const uint32_t* ends;
  int lo, hi;        // requests
  int base;          // request of ends[0]
  uint32_t before;   // end of request lo - 1
};

// Requests of several outputs, and where each request's outputs start: the number
// of ends at or below x, halving all ranges together.
template <int K>
__device__ __forceinline__ void find(const Near& n, const uint32_t (&x)[K], int (&r)[K],
                                     uint32_t (&start)[K]) {
  int at[K];
#pragma unroll
  for (int k = 0; k < K; ++k) at[k] = n.lo - n.base;
  for (int rest = n.hi - n.lo; rest > 0;) {
    const int half = (rest + 1) >> 1;
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] += n.ends[at[k] + half - 1] <= x[k] ? half : 0;
    rest -= half;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    r[k] = at[k] + n.base;
    start[k] = r[k] > n.lo ? n.ends[at[k] - 1] : n.before;
  }
}

// Outputs [tile * kTile, ...) of the tokens, then of the pages (the taken ones
// into the table, the rest into the new list).  NARROW: the ends are in memory;
// the tile's first and last owners are found first, by a wave each, and what
// lies between them is fetched at one go, so that an output costs two loads in
// turn and not one for every halving.
template <bool NARROW>
__device__ __forceinline__ void plan_outputs(const PlanArgs& a, const Ends& e,
                                             const Counts& total, int64_t tile,
                                             int64_t token_tiles) {
  __shared__ int32_t bound[6];
  __shared__ uint32_t near[3][NARROW ? kNear : 1];
  const int last = (int)a.n - 1;
  const int wave = uniform(threadIdx.x / kWave);
  const uint32_t free = free_pages_of(a);
  const uint32_t avail = sat_add(free, total.given);
  auto locate = [&](int i, const uint32_t* ends, uint32_t x, uint32_t y) {
    if (NARROW && wave == i) wave_owners(ends, x, y, last, bound + 2 * i);
  };
  auto stage = [&](int i, const uint32_t* ends) {          // after the bounds are known
    Near n = {ends, 0, last, 0, 0u};
    if (!NARROW) return n;
    n.lo = bound[2 * i];
    n.hi = bound[2 * i + 1];
    n.before = n.lo > 0 ? ends[n.lo - 1] : 0u;
    if (n.hi - n.lo < kNear) {
      for (int k = threadIdx.x; k <= n.hi - n.lo; k += kThreads) near[i][k] = ends[n.lo + k];
      n.ends = near[i];
      n.base = n.lo;
    }
    return n;
  };
  // Entry j of the pool: the free list, then the released pages.  Those of the
  // list are loaded at once; the others take a search first.
  auto pool_entries = [&](const Near& given, const bool (&wanted)[kOwn],
                          const int32_t* (&from)[kOwn], const uint32_t (&j)[kOwn],
                          int32_t (&id)[kOwn]) {
    bool search = false;
#pragma unroll
    for (int s = 0; s < kOwn; ++s) {
      const bool listed = wanted[s] && from[s] == nullptr && j[s] < free;
      const bool released = wanted[s] && from[s] == nullptr && j[s] >= free && j[s] < avail;
      search |= released;
      if (listed) from[s] = a.free_pages + j[s];
    }
#pragma unroll
    for (int s = 0; s < kOwn; ++s) id[s] = from[s] != nullptr ? *from[s] : -1;
    if (!search) return;
    uint32_t x[kOwn], start[kOwn];
    int r[kOwn];
#pragma unroll
    for (int s = 0; s < kOwn; ++s) x[s] = j[s] >= free ? j[s] - free : 0u;
    find(given, x, r, start);
#pragma unroll
    for (int s = 0; s < kOwn; ++s)
      if (wanted[s] && from[s] == nullptr && j[s] >= free && j[s] < avail)
        id[s] = a.table[(int64_t)r[s] * a.ldt + (x[s] - start[s])];
  };
  if (tile < token_tiles) {
    const int64_t t0 = tile * kTile;
    locate(0, e.tokens, (uint32_t)t0, (uint32_t)(t0 + kTile - 1));
    if (NARROW) __syncthreads();
    const Near owners = stage(0, e.tokens);
    const bool staged = NARROW && owners.ends == near[0];
    if (staged) {
      for (int k = threadIdx.x; k <= owners.hi - owners.lo; k += kThreads) {
        const int r = owners.lo + k;
        near[1][k] = (uint32_t)a.cached[r];
        near[2][k] = r > 0 ? e.taken[r - 1] : 0u;
      }
    }
    if (NARROW) __syncthreads();
    const Near anyone = {e.given, 0, last, 0, 0u};
    uint32_t t[kOwn], start[kOwn], off[kOwn], j[kOwn];
    int r[kOwn];
    int32_t pos[kOwn], id[kOwn];
    bool live[kOwn];
    const int32_t* from[kOwn];
#pragma unroll
    for (int s = 0; s < kOwn; ++s) t[s] = (uint32_t)t0 + s * kThreads + threadIdx.x;
    find(owners, t, r, start);
#pragma unroll
    for (int s = 0; s < kOwn; ++s) {
      live[s] = t[s] < total.tokens && t[s] < (uint32_t)a.max_tokens;
      pos[s] = -1;
      off[s] = j[s] = 0;
      from[s] = nullptr;
      if (live[s]) {
        const uint32_t c = staged ? near[1][r[s] - owners.lo] : (uint32_t)a.cached[r[s]];
        const uint32_t x = c + t[s] - start[s];
        const uint32_t held = pages_of(c, a.page);
        const uint32_t pg = div_by(x, a.page);
        pos[s] = (int32_t)x;
        off[s] = x - pg * a.page.d;
        if (pg < held) {
          from[s] = a.table + (int64_t)r[s] * a.ldt + pg;
        } else {
          const uint32_t first =
              staged ? near[2][r[s] - owners.lo] : (r[s] > 0 ? e.taken[r[s] - 1] : 0u);
          j[s] = first + (pg - held);
        }
      }
    }
    pool_entries(anyone, live, from, j, id);
#pragma unroll
    for (int s = 0; s < kOwn; ++s) {
      if (t[s] >= (uint32_t)a.max_tokens) break;
      a.slots[t[s]] = id[s] >= 0 ? (int64_t)id[s] * a.page.d + off[s] : -1;
      if (a.positions != nullptr) a.positions[t[s]] = pos[s];
    }
    return;
  }
  const int64_t j0 = (tile - token_tiles) * kTile;
  const uint32_t used = total.taken < avail ? total.taken : avail;
  const uint32_t first = (uint32_t)j0, final = (uint32_t)j0 + kTile - 1;
  auto released = [&](uint32_t j) { return j > free ? j - free : 0u; };
  locate(0, e.taken, first, final);
  locate(1, e.given, released(first), released(final));
  locate(2, e.given, released(used + first), released(used + final));
  if (NARROW) __syncthreads();
  const Near takers = stage(0, e.taken), givers = stage(1, e.given), later = stage(2, e.given);
  if (NARROW) __syncthreads();
  uint32_t j[kOwn], left[kOwn], start[kOwn];
  int r[kOwn];
  int32_t id[kOwn];
  bool inside[kOwn], taken[kOwn];
  const int32_t* from[kOwn];
#pragma unroll
  for (int s = 0; s < kOwn; ++s) {
    j[s] = (uint32_t)j0 + s * kThreads + threadIdx.x;
    inside[s] = j[s] < (uint32_t)a.capacity;
    taken[s] = inside[s] && j[s] < used;
    left[s] = used + j[s];
    from[s] = nullptr;
  }
  pool_entries(later, inside, from, left, id);
#pragma unroll
  for (int s = 0; s < kOwn; ++s)
    if (inside[s]) a.free_out[j[s]] = id[s];
  // A negative entry among those of the pool (a list or a released row that holds
  // one) is no page.
  bool hole = false;
#pragma unroll
  for (int s = 0; s < kOwn; ++s) hole |= inside[s] && left[s] < avail && id[s] < 0;
  if (hole) raise_status(a.d_status, PAIR_ST_PAGES);
  if (first >= used) return;
  find(takers, j, r, start);
#pragma unroll
  for (int s = 0; s < kOwn; ++s) from[s] = nullptr;
  pool_entries(givers, taken, from, j, id);
  hole = false;
#pragma unroll
  for (int s = 0; s < kOwn; ++s) hole |= taken[s] && id[s] < 0;
  if (hole) raise_status(a.d_status, PAIR_ST_PAGES);
#pragma unroll
  for (int s = 0; s < kOwn; ++s)
    if (taken[s])
      a.table[(int64_t)r[s] * a.ldt + pages_of((uint32_t)a.cached[r[s]], a.page) +
              (j[s] - start[s])] = id[s];
}

// Pages that requests take beyond the list's length go into the table here (the
// tiles of pages are as many as the list has: released pages may be more).  Table
// entries that the pool has no page for become -1, their requests' lengths
// end with the pages that they got, and what does not fit is reported; by the
// threads of one workgroup, after the lengths are written.
__device__ void plan_totals(const PlanArgs& a, const Ends& e, const Counts& total) {
  const uint32_t free = free_pages_of(a);
  const uint32_t avail = sat_add(free, total.given);
  const uint32_t used = total.taken < avail ? total.taken : avail;
  if (threadIdx.x == 0) {
    const uint32_t left = avail - used;
    *a.free_count_out = left < (uint32_t)a.capacity ? left : (uint32_t)a.capacity;
    const int64_t counted = *a.free_count;
    if (total.taken > avail || left > (uint32_t)a.capacity || counted < 0 || counted > a.capacity)
      raise_status(a.d_status, PAIR_ST_PAGES);
    if (total.tokens > (uint32_t)a.max_tokens) raise_status(a.d_status, PAIR_ST_LENGTH);
  }
  const int last = (int)a.n - 1;
  for (uint32_t j = (uint32_t)a.capacity + threadIdx.x; j < used; j += blockDim.x) {
    const uint32_t x = j - free;              // free is at most the capacity
    const int from = owner(e.given, x, 0, last), to = owner(e.taken, j, 0, last);
    const int32_t id = a.table[(int64_t)from * a.ldt + (x - (from > 0 ? e.given[from - 1] : 0u))];
    a.table[(int64_t)to * a.ldt + pages_of((uint32_t)a.cached[to], a.page) +
            (j - (to > 0 ? e.taken[to - 1] : 0u))] = id;
    if (id < 0) raise_status(a.d_status, PAIR_ST_PAGES);
  }
  if (total.taken > used) {
    for (uint32_t j = used + threadIdx.x; j < total.taken; j += blockDim.x) {
      const int r = owner(e.taken, j, 0, last);
      const uint32_t held = pages_of((uint32_t)a.cached[r], a.page);
      const uint32_t start = r > 0 ? e.taken[r - 1] : 0u;
      a.table[(int64_t)r * a.ldt + held + j - start] = -1;
      // The request's first entry without a page: the ones before it are full.
      // A length beyond them would count the -1 as pages when it is released.
      if (j == used || j == start) a.lens[r] = (int32_t)((held + j - start) * a.page.d);
    }
  }
}

// Up to kFused requests: every workgroup scans them all (their lengths come
// from the caches) and writes one tile of the outputs, in one launch.
constexpr int kFused = 2048;

__global__ __launch_bounds__(kThreads) void plan_fused_kernel(PlanArgs a, int64_t token_tiles) {
  __shared__ uint32_t ends[3][kFused];
  const int n = (int)a.n;
  const int per = (n + kThreads - 1) / kThreads;
  const int r0 = (int)threadIdx.x * per;
  const int r1 = r0 + per < n ? r0 + per : n;
  int32_t bad = 0, len;
  Counts sum = {0u, 0u, 0u};
  for (int r = r0; r < r1; ++r) sum = sum + request(a, r, &len, &bad);
  Counts total;
  const Counts end = group_scan<kThreads>(sum, &total);
  // walk back from the inclusive end: saturated sums are past every capacity
  Counts at = {0u, 0u, 0u};
  {
    __shared__ Counts prev[kThreads];
    prev[threadIdx.x] = end;
    __syncthreads();
    if (threadIdx.x > 0) at = prev[threadIdx.x - 1];
  }
  const bool first = blockIdx.x == 0;
  for (int r = r0; r < r1; ++r) {
    if (first) a.q_offsets[r] = at.tokens;
    at = at + request(a, r, &len, &bad);
    ends[0][r] = at.tokens;
    ends[1][r] = at.taken;
    ends[2][r] = at.given;
    if (first) a.lens[r] = len;
  }
  __syncthreads();
  const Ends e = {ends[0], ends[1], ends[2]};
  if (first) {
    if (threadIdx.x == 0) a.q_offsets[n] = total.tokens;
    if (bad) raise_status(a.d_status, bad);
    plan_totals(a, e, total);
  }
  plan_outputs<false>(a, e, total, blockIdx.x, token_tiles);
}

// More requests: a first launch writes the scans' ends to the workspace.  Each
// of its workgroups owns kScan requests and sums the ones before them itself,
// or, beyond kSelfSummed requests, takes the sums that a launch before it left.
// (A call of 4,096 requests 16.2 us by itself, 18.7 us with that launch; 16,384:
// 19.8 and 20.7; 32,768: 25.2 and 23.8; 65,536: 33.1 and 22.8; 2^20: 550 and 52.)
constexpr int kScan = 1024;
constexpr int64_t kSelfSummed = 1 << 14;

__global__ __launch_bounds__(kScan) void plan_sums_kernel(PlanArgs a, Counts* sums) {
  const int64_t r = (int64_t)blockIdx.x * kScan + threadIdx.x;
  int32_t other = 0, len;
  Counts mine = {0u, 0u, 0u}, total;
  if (r < a.n) mine = request(a, r, &len, &other);
  group_scan<kScan>(mine, &total);
  if (threadIdx.x == 0) sums[blockIdx.x] = total;
}

__global__ __launch_bounds__(kScan) void plan_scan_kernel(PlanArgs a, uint32_t* ends,
                                                          const Counts* sums) {
  const int64_t r0 = (int64_t)blockIdx.x * kScan;
  int32_t bad = 0, other = 0, len;
  Counts sum = {0u, 0u, 0u};
  if (sums != nullptr) {
    for (int64_t b = threadIdx.x; b < blockIdx.x; b += kScan) sum = sum + sums[b];
  } else {
    // r0 is a multiple of kScan: four requests of a lane at a time
    for (int64_t r = 4 * threadIdx.x; r < r0; r += 4 * kScan) {
      typedef u32x4_t u32x4_a4 __attribute__((aligned(4)));
      typedef uint32_t u32_a1 __attribute__((aligned(1)));
      const u32x4_t cached = *reinterpret_cast<const u32x4_a4*>(a.cached + r);
      const u32x4_t fresh = *reinterpret_cast<const u32x4_a4*>(a.fresh + r);
      const uint32_t live =
          a.mask != nullptr ? *reinterpret_cast<const u32_a1*>(a.mask + r) : 0x01010101u;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sum = sum + counts_of(a, (int32_t)cached[i], (int32_t)fresh[i],
                              ((live >> (8 * i)) & 0xffu) != 0, &len, &other);
    }
  }
  Counts before, total;
  group_scan<kScan>(sum, &before);
  const int64_t r = r0 + threadIdx.x;
  Counts mine = {0u, 0u, 0u};
  if (r < a.n) mine = request(a, r, &len, &bad);
  const Counts end = before + group_scan<kScan>(mine, &total);
  if (r < a.n) {
    ends[r] = end.tokens;
    ends[a.n + r] = end.taken;
    ends[2 * a.n + r] = end.given;
    a.q_offsets[r + 1] = end.tokens;
    a.lens[r] = len;
    if (r == 0) a.q_offsets[0] = 0;
  }
  if (bad) raise_status(a.d_status, bad);
}

__global__ __launch_bounds__(kThreads) void plan_write_kernel(PlanArgs a, const uint32_t* ends,
                                                              int64_t token_tiles) {
  const Ends e = {ends, ends + a.n, ends + 2 * a.n};
  const Counts total = {e.tokens[a.n - 1], e.taken[a.n - 1], e.given[a.n - 1]};
  if (blockIdx.x == 0) plan_totals(a, e, total);
  plan_outputs<true>(a, e, total, blockIdx.x, token_tiles);
}

// ------------------------------------------------------------------ store --
// A copy of 16-byte pieces: piece i of the call is piece i % per_token of
// token i / per_token, the keys' pieces before the values'.  HBM-bound: 32,467
// tokens of 8 heads of 128 (266 MB read and written) 50 us, 5.3 TB/s, as fast as
// a large copy; 64 tokens 4 us.
constexpr int kStorePieces = 4;   // in flight per lane

struct StoreArgs {
  const unsigned char* src[2];
  unsigned char* dst[2];
  int64_t token_bytes, head_in_bytes;
  int64_t page_bytes, slot_bytes, head_bytes;
  FastDiv page, per_token, per_head;
  uint32_t half;              // pieces of a token's keys
  int64_t slots_total;
  const int64_t* slots;
  int64_t tokens;
  int32_t* d_status;
};

__global__ __launch_bounds__(kThreads) void cache_store_kernel(StoreArgs a, int tokens_per_group) {
  const int64_t t0 = (int64_t)blockIdx.x * tokens_per_group;
  const int64_t left = a.tokens - t0;
  const uint32_t n =
      (uint32_t)(left < tokens_per_group ? left : tokens_per_group) * a.per_token.d;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kThreads * kStorePieces) {
    u32x4_t v[kStorePieces];
    unsigned char* to[kStorePieces];
#pragma unroll
    for (int s = 0; s < kStorePieces; ++s) {
      const uint32_t i = i0 + s * kThreads;
      to[s] = nullptr;
      if (i < n) {
        const uint32_t tok = div_by(i, a.per_token);
        uint32_t c = i - tok * a.per_token.d;
        const int64_t slot = a.slots[t0 + tok];
        const bool value = c >= a.half;
        if (value) c -= a.half;
        const uint32_t h = div_by(c, a.per_head);
        const uint32_t d = (c - h * a.per_head.d) * 16u;
        if (slot >= a.slots_total) {
          raise_status(a.d_status, PAIR_ST_PAGES);
        } else if (slot >= 0) {
          const uint32_t pg = div_by((uint32_t)slot, a.page);
          const uint32_t at = (uint32_t)slot - pg * a.page.d;
          to[s] = (value ? a.dst[1] : a.dst[0]) + pg * a.page_bytes + at * a.slot_bytes +
                  h * a.head_bytes + d;
          v[s] = *reinterpret_cast<const u32x4_t*>((value ? a.src[1] : a.src[0]) +
                                                   (t0 + tok) * a.token_bytes +
                                                   h * a.head_in_bytes + d);
        }
      }
    }
#pragma unroll
    for (int s = 0; s < kStorePieces; ++s)
      if (to[s] != nullptr) *reinterpret_cast<u32x4_t*>(to[s]) = v[s];
  }
}

}  // namespace

size_t page_plan_workspace_bytes(int64_t n) {
  return (((size_t)n * 3 * sizeof(uint32_t) + (size_t)(n + kScan - 1) / kScan * sizeof(Counts)) +
          255) / 256 * 256;
}

int launch_page_plan(int64_t n, const int32_t* cached, const int32_t* fresh, const uint8_t* mask,
                     int32_t page, int32_t* table, int64_t ldt, int64_t capacity,
                     const int32_t* free_pages, const int64_t* free_count, int64_t max_tokens,
                     int64_t* q_offsets, int32_t* lens, int64_t* slots, int32_t* positions,
                     int32_t* free_out, int64_t* free_count_out, void* workspace,
                     int32_t* d_status, hipStream_t stream) {
  const PlanArgs a = {n,         cached,     fresh,          mask,       fast_div((uint32_t)page),
                      table,     ldt,        (int32_t)capacity, free_pages, free_count,
                      (int32_t)max_tokens, q_offsets, lens,   slots,      positions,
                      free_out,  free_count_out, d_status};
  const int64_t token_tiles = (max_tokens + kTile - 1) / kTile;
  const int64_t tiles = token_tiles + (capacity + kTile - 1) / kTile;
  const unsigned grid = (unsigned)(tiles > 0 ? tiles : 1);
  if (n <= kFused) {
    hipLaunchKernelGGL(plan_fused_kernel, dim3(grid), dim3(kThreads), 0, stream, a, token_tiles);
  } else {
    uint32_t* ends = static_cast<uint32_t*>(workspace);
    const dim3 groups((unsigned)((n + kScan - 1) / kScan));
    Counts* sums = n > kSelfSummed ? reinterpret_cast<Counts*>(ends + 3 * n) : nullptr;
    if (sums != nullptr) {
      hipLaunchKernelGGL(plan_sums_kernel, groups, dim3(kScan), 0, stream, a, sums);
      if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
    }
    hipLaunchKernelGGL(plan_scan_kernel, groups, dim3(kScan), 0, stream, a, ends,
                       (const Counts*)sums);
    if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
    hipLaunchKernelGGL(plan_write_kernel, dim3(grid), dim3(kThreads), 0, stream, a, ends,
                       token_tiles);
  }
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

int launch_cache_store(int64_t tokens, int32_t kv_heads, int32_t dim, const void* k, const void* v,
                       int64_t token_stride, int64_t new_head_stride, void* k_cache,
                       void* v_cache, const PagedCache& cache, const int64_t* slots,
                       int32_t* d_status, hipStream_t stream) {
  StoreArgs a;
  a.src[0] = static_cast<const unsigned char*>(k);
  a.src[1] = static_cast<const unsigned char*>(v);
  a.dst[0] = static_cast<unsigned char*>(k_cache);
  a.dst[1] = static_cast<unsigned char*>(v_cache);
  a.token_bytes = token_stride * 2;
  a.head_in_bytes = new_head_stride * 2;
  a.page_bytes = cache.page_stride * 2;
  a.slot_bytes = cache.slot_stride * 2;
  a.head_bytes = cache.head_stride * 2;
  a.page = fast_div((uint32_t)cache.page);
  const uint32_t per_head = (uint32_t)dim / 8;
  a.per_head = fast_div(per_head);
  a.half = (uint32_t)kv_heads * per_head;
  a.per_token = fast_div(2 * a.half);
  a.slots_total = cache.n_pages * cache.page;
  a.slots = slots;
  a.tokens = tokens;
  a.d_status = d_status;
  // About four pieces a lane, at least one token a workgroup, and no more of them
  // than a launch can have (below 2^32 threads).
  int per_group = (int)(kThreads * kStorePieces / a.per_token.d);
  const int least = (int)((tokens + (1 << 23) - 1) >> 23);
  if (per_group < least) per_group = least;
  const int64_t grid = (tokens + per_group - 1) / per_group;
  hipLaunchKernelGGL(cache_store_kernel, dim3((unsigned)grid), dim3(kThreads), 0, stream, a,
                     per_group);
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace pair
