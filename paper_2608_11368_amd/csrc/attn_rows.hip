// Attention of a few new tokens per request (decoding, drafted tokens): all
// rows of a key/value head -- a row is one query head of one token -- fit one
// or two tiles of 16, and the time goes into reading the cache once.
//
// Layout.  A wave takes 32 keys at a time straight from memory into registers;
// nothing goes through LDS in the loop.
//   scores   S^T = K Q^T: a key row is 16-byte pieces of the A operand, and lane
//            (x, g) ends up with row x's scores of keys 4 g + i and 16 + 4 g + i;
//   weights  exactly those are its eight entries of the B operand of
//   output   O^T += V^T P^T once the product's k index is taken in that order:
//            only V has to be transposed, and a lane that loads eight dims of
//            its eight keys does it with one byte permute per dword.
// The rows' running maximum is raised (and the sums rescaled) only when a score
// exceeds it by 2^8, so most steps need no exchange between lanes.
//
// Work split.  The keys of all requests and heads form one line of units of
// kUnit keys; it is cut into equal runs, one per workgroup, whatever the
// lengths (the lengths are scanned by every workgroup: they are a few cached
// kilobytes).  A head whose run is cut leaves partial sums that a second launch
// joins.  The four waves of a workgroup take the 32-key blocks in turn and are
// joined through LDS.
#include "attn.hpp"

namespace pair {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kBlock = 32;                  // keys of a wave's step
constexpr int kUnit = kBlock * kWaves;      // keys of a workgroup's step
// Requests whose lengths a workgroup scans; more of them fill the card with
// one workgroup per request and head.
constexpr int kMostScanned = 4096;
constexpr float kLazy = 8.0f;

struct RowArgs {
  AttnCall a;
  FastDiv page, group;
  float scale_log2;
  int32_t groups;       // workgroups; 0: one per request and head
  int32_t* starts;      // [n + 1] units before each request (workspace)
  float* part_o;        // [2 groups][rows][dim]
  float* part_ml;       // [2 groups][rows][2]
};

__device__ __forceinline__ int units_of(const RowArgs& s, int64_t r, int32_t* bad) {
  Request q;
  if (!attention_request(s.a, s.page.d, r, &q, bad)) return 0;
  if (q.tokens == 0 || (int64_t)q.tokens * s.group.d > kRowsMost) return 0;
  return q.len <= kUnit ? 1 : (q.len + kUnit - 1) / kUnit;
}

// Workgroups that get a run: no more than there are units, so that none of
// those between two of a head is without one.
__device__ __forceinline__ int64_t runs_of(const RowArgs& s, int64_t units) {
  return units < s.groups ? units : s.groups;
}

// First unit of run w of `runs` on a line of `units`.
__device__ __forceinline__ int64_t run_start(int64_t units, int64_t runs, int64_t w) {
  return units * w / runs;
}

// One wave's running softmax over its keys: row x = lane & 15 of each tile.
template <int DIM, int NT>
struct State {
  float m[NT], l[NT];                // l: this lane's keys only
  f32x4_t acc[NT][DIM / 16];         // O^T: dims (4 g + i) * (DIM / 16) + j of row x
};

template <bool BF16, int DIM, int NT, bool ALIGNED>
__device__ __forceinline__ void add_keys(const RowArgs& s, const u32x4_t (&qf)[NT][DIM / 32],
                                         const int (&limit)[NT], int first_limit, int64_t r,
                                         int64_t kvh, int len, int k0, int k1,
                                         State<DIM, NT>* st) {
  constexpr int NC = DIM / 32;       // 32-dim pieces of a key row
  constexpr int ND = DIM / 16;       // dims of a lane's piece of a value row
  const int lane = threadIdx.x & (kWave - 1);
  const int x = lane & 15, g = lane >> 4;
  const int64_t head = kvh * s.a.cache.head_stride * 2;
  const unsigned char* kbase = static_cast<const unsigned char*>(s.a.k_cache) + head;
  const unsigned char* vbase = static_cast<const unsigned char*>(s.a.v_cache) + head;
  const int64_t slot_bytes = s.a.cache.slot_stride * 2, page_bytes = s.a.cache.page_stride * 2;
  const int32_t* row = s.a.table + r * s.a.ldt;
  const int64_t koff = x * slot_bytes + g * 16;
  const int64_t voff = 4 * g * slot_bytes + x * (DIM / 8);

  int32_t bad_page = 0;
  for (int kb = k0; kb < k1; kb += kUnit) {
    // where the keys lie
    u32x4_t kf[2][NC];
    uint32_t vr[8][ND / 2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (ALIGNED) {
        // a tile of 16 keys lies in one page; one past the end repeats the last
        int key = kb + 16 * t;
        if (key >= len) key = (len - 1) & ~15;
        const uint32_t pg = div_by((uint32_t)key, s.page);
        const int64_t at = checked_page(s.a, table_entry(row, pg), &bad_page) * page_bytes +
                           (int64_t)((uint32_t)key - pg * s.page.d) * slot_bytes;
        const unsigned char* kp = kbase + at + koff;
#pragma unroll
        for (int c = 0; c < NC; ++c) kf[t][c] = *reinterpret_cast<const u32x4_t*>(kp + c * 64);
        const unsigned char* vp = vbase + at + voff;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (DIM == 128) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t*>(vp + i * slot_bytes);
#pragma unroll
            for (int e = 0; e < ND / 2; ++e) vr[4 * t + i][e] = w[e];
          } else {
            const u32x2_t w = *reinterpret_cast<const u32x2_t*>(vp + i * slot_bytes);
#pragma unroll
            for (int e = 0; e < ND / 2; ++e) vr[4 * t + i][e] = w[e];
          }
        }
      } else {
#pragma unroll
        for (int i = -1; i < 4; ++i) {     // the key row, then four value rows
          int key = kb + 16 * t + (i < 0 ? x : 4 * g + i);
          if (key >= len) key = len - 1;
          const uint32_t pg = div_by((uint32_t)key, s.page);
          const int64_t at = checked_page(s.a, row[pg], &bad_page) * page_bytes +
                             (int64_t)((uint32_t)key - pg * s.page.d) * slot_bytes;
          if (i < 0) {
            const unsigned char* kp = kbase + at + g * 16;
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[t][c] = *reinterpret_cast<const u32x4_t*>(kp + c * 64);
          } else {
            const unsigned char* vp = vbase + at + x * (DIM / 8);
            const int e0 = 4 * t + (i < 0 ? 0 : i);
            if (DIM == 128) {
              const u32x4_t w = *reinterpret_cast<const u32x4_t*>(vp);
#pragma unroll
              for (int e = 0; e < ND / 2; ++e) vr[e0][e] = w[e];
            } else {
              const u32x2_t w = *reinterpret_cast<const u32x2_t*>(vp);
#pragma unroll
              for (int e = 0; e < ND / 2; ++e) vr[e0][e] = w[e];
            }
          }
        }
      }
    }

    float p[NT][8];
    const bool masked = kb + kBlock - 1 > first_limit;   // some row does not see some key
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      f32x4_t sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < NC; ++c) sc[t] = mma16<BF16>(kf[t][c], qf[nt][c], sc[t]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) p[nt][e] = sc[e >> 2][e & 3] * s.scale_log2;
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
      const float base = st->m[nt] == -INFINITY ? 0.0f : st->m[nt];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[nt][e] = __builtin_amdgcn_exp2f(p[nt][e] - base);
        st->l[nt] += p[nt][e];
      }
    }

    // Values that some row must not see: past the end they are no values at
    // all, and within the chunk a weight of zero does not hide a NaN or an
    // infinity from the matrix product.  Those are taken out of it here and
    // added below, one by one, to the rows that see them.
    uint64_t odd = 0;
    if (masked) {
      uint32_t bad = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = kb + 16 * (e >> 2) + 4 * g + (e & 3);
#pragma unroll
        for (int w = 0; w < ND / 2; ++w) {
          if (key >= len) vr[e][w] = 0u;
          bad |= not_finite<BF16>(vr[e][w]) ? 1u : 0u;
        }
      }
      odd = __ballot(bad != 0u);
    }
    if (odd != 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int j = 0; j < ND; ++j) {
          const uint32_t bits = (vr[e][j >> 1] >> (16 * (j & 1))) & 0xffffu;
          uint64_t where = __ballot(not_finite<BF16>(bits));
          if (not_finite<BF16>(bits)) vr[e][j >> 1] &= (j & 1) ? 0x0000ffffu : 0xffff0000u;
          while (where != 0) {
            const int src = __ffsll((unsigned long long)where) - 1;
            where &= where - 1;
            const float v = half_value<BF16>((uint32_t)__builtin_amdgcn_readlane((int)bits, src));
            const int key = kb + 16 * (e >> 2) + 4 * (src >> 4) + (e & 3);
            const int m = src & 15;                 // dim m * ND + j
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const float pv = __shfl(p[nt][e], x + 16 * (src >> 4), kWave);
              if (key <= limit[nt] && g == (m >> 2)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (i == (m & 3)) st->acc[nt][j][i] = __builtin_fmaf(pv, v, st->acc[nt][j][i]);
              }
            }
          }
        }
      }
    }

    u32x4_t pf[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int w = 0; w < 4; ++w) pf[nt][w] = pack2<BF16>(p[nt][2 * w], p[nt][2 * w + 1]);
#pragma unroll
    for (int j = 0; j < ND; ++j) {
      u32x4_t vt;                                   // dim j of this lane's eight keys
#pragma unroll
      for (int w = 0; w < 4; ++w)
        vt[w] = __builtin_amdgcn_perm(vr[2 * w + 1][j >> 1], vr[2 * w][j >> 1],
                                      (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) st->acc[nt][j] = mma16<BF16>(vt, pf[nt], st->acc[nt][j]);
    }
  }
  if (bad_page) raise_status(s.a.d_status, bad_page);
}

// Keys [k0, k1) of one request and head (k0 a multiple of kUnit): the waves'
// sums, joined, either as results (slot < 0) or as partial sums.
template <bool BF16, int DIM, int NT, bool ALIGNED>
__device__ __forceinline__ void attend(const RowArgs& s, int64_t r, int kvh, int k0, int k1,
                                       int64_t slot) {
  constexpr int ND = DIM / 16;
  constexpr int kRow = DIM + 4;
  __shared__ float sum[kWaves][16][kRow];
  __shared__ float stat[kWaves][16][2];
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
      const uint16_t* p = static_cast<const uint16_t*>(s.a.q) + (q.q0 + tok) * s.a.q_token +
                          (kvh * (int)s.group.d + i - tok * (int)s.group.d) * s.a.q_head + g * 8;
#pragma unroll
      for (int c = 0; c < DIM / 32; ++c) qf[nt][c] = *reinterpret_cast<const u32x4_t*>(p + c * 32);
    }
  }
  // unused rows see nothing, so every block counts as masked for them only if
  // it does for the first token
  const int end = k1 < q.len ? k1 : q.len;
  add_keys<BF16, DIM, NT, ALIGNED>(s, qf, limit, q.len - q.tokens, r, kvh, q.len,
                                   k0 + kBlock * wave, end, &st);

#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float l = st.l[nt];
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (g == 0) {
      stat[wave][x][0] = st.m[nt];
      stat[wave][x][1] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < ND; ++j) sum[wave][x][(4 * g + i) * ND + j] = st.acc[nt][j][i];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * DIM / 8; e += kThreads) {
      const int y = e / (DIM / 8), d = (e - y * (DIM / 8)) * 8;
      const int i = 16 * nt + y;
      if (i < rows) {
        float m = stat[0][y][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, stat[w][y][0]);
        const float base = m == -INFINITY ? 0.0f : m;
        float tot = 0.0f, o[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(stat[w][y][0] - base);
          if (stat[w][y][0] == -INFINITY && stat[w][y][1] == 0.0f) continue;   // saw no key
          tot = __builtin_fmaf(f, stat[w][y][1], tot);
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = __builtin_fmaf(f, sum[w][y][d + k], o[k]);
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
                none ? -INFINITY : (m + __builtin_amdgcn_logf(tot)) * 0.69314718056f;
        }
      }
    }
    __syncthreads();
  }
}

template <bool BF16, int DIM, int NT, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void attention_rows_kernel(RowArgs s) {
  const int64_t heads = s.a.kv_heads;
  if (s.groups == 0) {
    const int64_t r = blockIdx.x / heads;
    int32_t bad = 0;
    const int units = units_of(s, r, &bad);
    if (bad && threadIdx.x == 0) raise_status(s.a.d_status, bad);
    if (units == 0) return;
    attend<BF16, DIM, NT, ALIGNED>(s, r, (int)(blockIdx.x - r * heads), 0, units * kUnit, -1);
    return;
  }
  // units before each request, in every workgroup
  __shared__ int32_t start[kMostScanned + 1];
  __shared__ int32_t wave_sum_of[kWaves];
  const int n = (int)s.a.n, lane = threadIdx.x & (kWave - 1);
  const int per = (n + kThreads - 1) / kThreads;
  const int r0 = (int)threadIdx.x * per, r1 = r0 + per < n ? r0 + per : n;
  int32_t bad = 0, mine = 0;
  for (int r = r0; r < r1; ++r) {
    const int u = units_of(s, r, &bad);
    start[r + 1] = u;
    mine += u;
  }
  if (bad && blockIdx.x == 0) raise_status(s.a.d_status, bad);
  int32_t scan = mine;
#pragma unroll
  for (int by = 1; by < kWave; by <<= 1) {
    const int32_t v = __shfl_up(scan, by, kWave);
    if (lane >= by) scan += v;
  }
  if (lane == kWave - 1) wave_sum_of[threadIdx.x / kWave] = scan;
  if (threadIdx.x == 0) start[0] = 0;
  __syncthreads();
  int32_t at = scan - mine;
  for (int w = 0; w < (int)threadIdx.x / kWave; ++w) at += wave_sum_of[w];
  for (int r = r0; r < r1; ++r) {
    at += start[r + 1];
    start[r + 1] = at;
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int r = threadIdx.x; r <= n; r += kThreads) s.starts[r] = start[r];
  const int64_t units = start[n] * heads;
  const int64_t runs = runs_of(s, units);
  if (blockIdx.x >= runs) return;
  int64_t u = uniform64(run_start(units, runs, blockIdx.x));
  const int64_t end = uniform64(run_start(units, runs, blockIdx.x + 1));
  int64_t slot = 2 * (int64_t)blockIdx.x;
  while (u < end) {
    int lo = 0, hi = n - 1;                         // the request of unit u
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (uniform(start[mid + 1]) * heads > u)
        hi = mid;
      else
        lo = mid + 1;
    }
    const int first = uniform(start[lo]), count = uniform(start[lo + 1]) - first;
    const int x = (int)(u - first * heads);
    const int h = x / count, c0 = x - h * count;
    const int c1 = count - c0 < end - u ? count : c0 + (int)(end - u);
    const bool whole = c0 == 0 && c1 == count;
    attend<BF16, DIM, NT, ALIGNED>(s, lo, h, c0 * kUnit, c1 * kUnit, whole ? -1 : slot);
    slot = 2 * (int64_t)blockIdx.x + 1;
    u += c1 - c0;
  }
}

// Joins the partial sums of the heads that were cut: one workgroup per request,
// head and row, its waves taking the parts in turn.
template <bool BF16, int DIM>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(RowArgs s, int rows_slot) {
  const int64_t heads = s.a.kv_heads;
  const int64_t r = blockIdx.x / heads;
  const int kvh = (int)(blockIdx.x - r * heads);
  const int i = blockIdx.y;
  const int64_t first = s.starts[r] * heads, count = s.starts[r + 1] - s.starts[r];
  if (count == 0) return;
  const int64_t units = s.starts[s.a.n] * heads;
  const int64_t u0 = first + kvh * count, u1 = u0 + count;
  // workgroup of unit u: the last whose run starts at or before it
  const int64_t runs = runs_of(s, units);
  const int64_t w0 = ((u0 + 1) * runs - 1) / units, w1 = (u1 * runs - 1) / units;
  if (w0 == w1) return;
  Request q;
  int32_t bad = 0;
  if (!attention_request(s.a, s.page.d, r, &q, &bad)) return;
  if (i >= q.tokens * (int)s.group.d) return;
  const int tok = (int)div_by((uint32_t)i, s.group);
  const int h = kvh * (int)s.group.d + i - tok * (int)s.group.d;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  constexpr int PER = DIM / kWave;
  float m = -INFINITY, l = 0.0f, o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.0f;
  for (int64_t w = w0 + wave; w <= w1; w += kWaves) {
    // a head that starts inside a workgroup's run is in its second slot
    const int64_t slot = 2 * w + (w == w0 && run_start(units, runs, w) != u0 ? 1 : 0);
    const int64_t at = slot * rows_slot + i;
    const float mw = s.part_ml[at * 2], lw = s.part_ml[at * 2 + 1];
    float ow[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) ow[e] = s.part_o[at * DIM + e * kWave + lane];
    if (mw == -INFINITY && lw == 0.0f) continue;
    const float mn = fmaxf(m, mw);
    const float base = mn == -INFINITY ? 0.0f : mn;
    const float a = __builtin_amdgcn_exp2f(m - base), b = __builtin_amdgcn_exp2f(mw - base);
    l = l * a + lw * b;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = o[e] * a + ow[e] * b;
    m = mn;
  }
  __shared__ float sum[kWaves][DIM], stat[kWaves][2];
#pragma unroll
  for (int e = 0; e < PER; ++e) sum[wave][e * kWave + lane] = o[e];
  if (lane == 0) {
    stat[wave][0] = m;
    stat[wave][1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= DIM / 2) return;
  m = stat[0][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, stat[w][0]);
  const float base = m == -INFINITY ? 0.0f : m;
  l = 0.0f;
  float a = 0.0f, b = 0.0f;
  const int d = threadIdx.x * 2;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (stat[w][0] == -INFINITY && stat[w][1] == 0.0f) continue;
    const float f = __builtin_amdgcn_exp2f(stat[w][0] - base);
    l += stat[w][1] * f;
    a += sum[w][d] * f;
    b += sum[w][d + 1] * f;
  }
  const bool none = limit_of(q, tok) < 0;
  const float inv = 1.0f / l;
  *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(s.a.out) + (q.q0 + tok) * s.a.out_token +
                               h * s.a.out_head + d) = none ? 0u : pack2<BF16>(a * inv, b * inv);
  if (s.a.lse != nullptr && threadIdx.x == 0)
    s.a.lse[(q.q0 + tok) * s.a.q_heads + h] =
        none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718056f;
}

struct Plan {
  int tiles;            // of 16 rows
  int rows;             // bound on a request's rows
  int32_t groups;
  size_t starts, ml, total;   // workspace: bytes of the parts
};

Plan plan_rows(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t max_q,
               int32_t max_len) {
  Plan p;
  const int64_t rows = (int64_t)max_q * (q_heads / kv_heads);
  p.rows = (int)(rows < kRowsMost ? rows : kRowsMost);
  p.tiles = p.rows <= 16 ? 1 : 2;
  // Cut into equal runs unless every head is a step or two anyway, or the
  // requests are so many that they fill the card by themselves.
  const int64_t most = n * kv_heads * ((max_len + kUnit - 1) / kUnit);
  const int64_t slots = 2 * (int64_t)device_cu_count();
  p.groups = n > kMostScanned || max_len <= 2 * kUnit ? 0 : (int32_t)(most < slots ? most : slots);
  const size_t parts = 2 * (size_t)p.groups * 16 * p.tiles;
  p.starts = ((size_t)(n + 1) * 4 + 255) / 256 * 256;
  p.ml = (parts * 8 + 255) / 256 * 256;
  p.total = p.groups == 0 ? 256 : p.starts + p.ml + parts * dim * 4;
  return p;
}

template <bool BF16, int DIM>
int launch(const RowArgs& s, const Plan& p, hipStream_t stream) {
  const int64_t grid = p.groups != 0 ? p.groups : s.a.n * s.a.kv_heads;
  if (grid > 0x7fffffffLL || s.a.n * s.a.kv_heads > 0x7fffffffLL) return PAIR_ERANGE;
  const bool aligned = s.page.d % 16 == 0;
#define PAIR_ROWS(NT, AL)                                                                        \
  hipLaunchKernelGGL((attention_rows_kernel<BF16, DIM, NT, AL>), dim3((unsigned)grid),            \
                     dim3(kThreads), 0, stream, s)
  if (p.tiles == 1) {
    if (aligned) PAIR_ROWS(1, true); else PAIR_ROWS(1, false);
  } else {
    if (aligned) PAIR_ROWS(2, true); else PAIR_ROWS(2, false);
  }
#undef PAIR_ROWS
  if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
  if (p.groups != 0)
    hipLaunchKernelGGL((join_rows_kernel<BF16, DIM>),
                       dim3((unsigned)(s.a.n * s.a.kv_heads), (unsigned)p.rows), dim3(kThreads), 0,
                       stream, s, 16 * p.tiles);
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace

size_t attention_rows_workspace(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                                int32_t max_q, int32_t max_len) {
  return plan_rows(n, q_heads, kv_heads, dim, max_q, max_len).total;
}

int launch_attention_rows(const AttnCall& a, void* workspace, hipStream_t stream) {
  const Plan p = plan_rows(a.n, a.q_heads, a.kv_heads, a.dim, a.max_q, a.max_len);
  RowArgs s;
  s.a = a;
  s.page = fast_div((uint32_t)a.cache.page);
  s.group = fast_div((uint32_t)(a.q_heads / a.kv_heads));
  s.scale_log2 = a.scale * 1.44269504089f;
  s.groups = p.groups;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  s.starts = reinterpret_cast<int32_t*>(ws);
  s.part_ml = reinterpret_cast<float*>(ws + p.starts);
  s.part_o = reinterpret_cast<float*>(ws + p.starts + p.ml);
  if (a.dim == 64) return a.bf16 ? launch<true, 64>(s, p, stream) : launch<false, 64>(s, p, stream);
  return a.bf16 ? launch<true, 128>(s, p, stream) : launch<false, 128>(s, p, stream);
}

}  // namespace pair
