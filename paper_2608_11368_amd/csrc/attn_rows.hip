// Attention of a few new tokens per request: the launches, and the joining of
// requests that were cut (attn_rows.hpp has the kernel's body).
#include <type_traits>

#include "attn_rows.hpp"

namespace pair {

using namespace rows;

namespace {

// Rows that a workgroup joins side by side where it has several.
constexpr int kJoined = kWaves;

// Joins the partial sums of the requests that were cut: a workgroup per request and
// head, or several that take its rows in turn, one or kJoined at a time.  First a row's
// parts' maxima and weights, a wave for each row, a lane for each part, then the parts'
// sums with several loads in flight.
template <bool BF16, int DIM>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(RowArgs s, int rows_slot,
                                                             int rows_turn) {
  const int64_t heads = s.a.kv_heads;
  const int64_t r = blockIdx.x / (uint32_t)s.a.kv_heads;
  const int kvh = (int)(blockIdx.x - r * heads);
  const int64_t u0 = s.starts[r], u1 = s.starts[r + 1];
  if (u0 == u1) return;
  const int64_t units = s.starts[s.a.n], runs = runs_of(s, units);
  // run of unit u: the last that starts at or before it
  const int64_t w0 = quotient((u0 + 1) * runs - 1, units), w1 = quotient(u1 * runs - 1, units);
  if (w0 == w1) return;
  Request q;
  int32_t bad = 0;
  if (!attention_request(s.a, s.page.d, r, &q, &bad)) return;
  const int rows = q.tokens * (int)s.group.d;
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  constexpr int PER = DIM / kWave;
  __shared__ float weight[kMostRuns][kJoined], sum[kWaves][kJoined][DIM], stat[kJoined][2];
  const int parts = (int)(w1 - w0) + 1;
  // a request that starts inside a run is in the run's second part
  const int64_t first = 2 * w0 + (run_start(units, runs, w0) != u0 ? 1 : 0);
  for (int i0 = blockIdx.y * rows_turn; i0 < rows; i0 += gridDim.y * rows_turn) {
    const int count = rows - i0 < rows_turn ? rows - i0 : rows_turn;
    auto place = [&](int p) {            // of row i0
      return ((p == 0 ? first : 2 * (w0 + p)) * heads + kvh) * rows_slot + i0;
    };
    if (wave < count) {
      float m = -INFINITY;
      for (int p = lane; p < parts; p += kWave) m = fmaxf(m, s.part_ml[(place(p) + wave) * 2]);
#pragma unroll
      for (int by = 1; by < kWave; by <<= 1) m = fmaxf(m, __shfl_xor(m, by, kWave));
      const float base = m == -INFINITY ? 0.0f : m;
      float l = 0.0f;
      for (int p = lane; p < parts; p += kWave) {
        const int64_t at = (place(p) + wave) * 2;
        const float mp = s.part_ml[at], lp = s.part_ml[at + 1];
        const bool none = mp == -INFINITY && lp == 0.0f;       // saw no key
        const float f = none ? 0.0f : __builtin_amdgcn_exp2f(mp - base);
        l += none ? 0.0f : lp * f;
        weight[p][wave] = f;
      }
      l = wave_sum(l);
      if (lane == 0) {
        stat[wave][0] = m;
        stat[wave][1] = l;
      }
    }
    __syncthreads();
    auto add = [&](auto rows_now) {      // a wave's share of the parts
      constexpr int N = decltype(rows_now)::value;
      float o[N][PER];
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int e = 0; e < PER; ++e) o[k][e] = 0.0f;
#pragma unroll 4
      for (int p = wave; p < parts; p += kWaves) {
        const float* from = s.part_o + place(p) * DIM;
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
          for (int e = 0; e < PER; ++e)
            o[k][e] = __builtin_fmaf(from[k * DIM + e * kWave + lane], weight[p][k], o[k][e]);
      }
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int e = 0; e < PER; ++e) sum[wave][k][e * kWave + lane] = o[k][e];
    };
    static_assert(kJoined == 4, "the cases");
    if (count == 1)
      add(std::integral_constant<int, 1>());
    else if (count == 2)
      add(std::integral_constant<int, 2>());
    else if (count == 3)
      add(std::integral_constant<int, 3>());
    else
      add(std::integral_constant<int, 4>());
    __syncthreads();
    const int k = (int)threadIdx.x / (DIM / 2);
    if (k < count) {
      const int d = ((int)threadIdx.x - k * (DIM / 2)) * 2;
      const int tok = (int)div_by((uint32_t)(i0 + k), s.group);
      const int h = kvh * (int)s.group.d + i0 + k - tok * (int)s.group.d;
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        a += sum[w][k][d];
        b += sum[w][k][d + 1];
      }
      const bool none = limit_of(q, tok) < 0;
      const float m = stat[k][0], l = stat[k][1];
      const float inv = 1.0f / l;
      *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(s.a.out) + (q.q0 + tok) * s.a.out_token +
                                   h * s.a.out_head + d) =
          none ? 0u : pack2<BF16>(a * inv, b * inv);
      if (s.a.lse != nullptr && d == 0)
        s.a.lse[(q.q0 + tok) * s.a.q_heads + h] = none ? -INFINITY : log_sum<BF16>(m, l);
    }
    __syncthreads();                     // the next rows' weights and sums
  }
}

}  // namespace

Plan rows::plan_of(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t bits,
                   int32_t max_q, int32_t max_len) {
  Plan p;
  const int64_t rows = (int64_t)max_q * (q_heads / kv_heads);
  p.rows = (int)(rows < kRowsMost ? rows : kRowsMost);
  p.tiles = p.rows <= 16 ? 1 : 2;
  // Cut into equal runs (units are counted in 31 bits) unless the longest head is
  // eight steps, which take less than the second launch would (4 requests of 700
  // keys: 8.0 us uncut, 9.5 us cut; of 1000: 9.3 and 9.9; of 2000: 21 and 11; 32
  // requests of 1000: 22 and 27), or the requests are so many that they fill the
  // card by themselves.
  // In 8 and 4 bits 16 steps, with the next block on its way: in 8 bits, 8 heads of
  // 128, uncut and cut, 16 requests of 1500 keys 16.5 and 21 us, 64 36 and 42, 128 68 and
  // 76, 256 of 300 41 and 52; five tokens of 64 43 and 63.  (32 steps: 256 of 1000, up to
  // 4000, 97 and 100, of two heads 41 and 37.)  But 12 where at most 32 workgroups leave
  // the card idle and a step is long: rows of 128 bytes (of 1640 to 2048 keys, a token of 2
  // requests 17.0 and 12.4, of 4 16.8 and 14.0; of 920 to 1150 12.1 and 13.0), or two tiles
  // of rows, whose next block is not on its way (eight tokens of 2 22.9 and 15.5, of 4 23.7
  // and 20.3; in 4 bits 22.0 and 17.2, 22.0 and 20.6; 3 tokens beside a chunk of 500 over
  // 2000 keys 46 and 38).  Else the second launch takes what the cut gains (one tile of 4
  // requests in 4 bits 15.7 and 15.3, of 64 elements 13.5 and 14.9; eight tokens of 64
  // requests, one head, 25 and 30).
  int whole = 8;
  if (bits != 16)
    whole = n * kv_heads <= 32 && (p.tiles == 2 || bits * dim == 1024) ? 12 : 16;
  const int64_t most = n * ((max_len + kUnit - 1) / kUnit);
  const int per_cu = p.tiles == 1 ? groups_per_cu(bits, dim) : 2;
  int64_t runs = per_cu * (int64_t)device_cu_count() / kv_heads;
  if (runs > most) runs = most;
  if (runs > kMostRuns) runs = kMostRuns;
  if (runs < 1) runs = 1;
  p.runs = n > kMostScanned || max_len <= whole * kUnit || most > 0x7fffffff ? 0 : (int32_t)runs;
  const size_t parts = 2 * (size_t)p.runs * kv_heads * 16 * p.tiles;
  p.starts = ((size_t)(n + 1) * 4 + 255) / 256 * 256;
  p.ml = (parts * 8 + 255) / 256 * 256;
  p.total = p.runs == 0 ? 256 : p.starts + p.ml + parts * dim * 4;
  return p;
}

RowArgs rows::args_of(const AttnCall& a, const Plan& p, void* workspace) {
  RowArgs s;
  s.a = a;
  s.page = fast_div((uint32_t)a.cache.page);
  s.group = fast_div((uint32_t)(a.q_heads / a.kv_heads));
  s.scale_log2 = a.scale * 1.44269504089f;
  s.runs = p.runs;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  s.starts = reinterpret_cast<int32_t*>(ws);
  s.part_ml = reinterpret_cast<float*>(ws + p.starts);
  s.part_o = reinterpret_cast<float*>(ws + p.starts + p.ml);
  return s;
}

int rows::join_rows(const RowArgs& s, const Plan& p, hipStream_t stream) {
  if (p.runs == 0) return PAIR_OK;
  // A workgroup for each row while those are at most 16 a compute unit.  Beyond, most
  // find their request uncut, and each takes a chain of loads and divisions for that:
  // about 16 a compute unit, for kJoined rows at a time.  2000 requests, one of 60,000
  // keys among those of 100, with 32 rows each on a key head of 64: 74 us with a workgroup
  // for each row, 149 with one for all, row by row, 59 so; 256 on 8 heads of 128, 146,
  // 196 and 130; 2000 of 1200 keys on 8 heads of 64, 1284 and 1065.  (72 requests of which
  // 64 have two rows and none over 32, 8 heads: the joins take 14 us with a workgroup for
  // each of 32 rows, 5 so.)
  const int64_t each = s.a.n * s.a.kv_heads, most = 16 * (int64_t)device_cu_count();
  const int rows_turn = each * p.rows <= most ? 1 : kJoined;
  int64_t turns = most / each;
  const int all = (p.rows + rows_turn - 1) / rows_turn;
  if (turns > all) turns = all;
  const dim3 grid((unsigned)each, (unsigned)(turns < 1 ? 1 : turns));
#define PAIR_JOIN(BF16, DIM)                                                                     \
  hipLaunchKernelGGL((join_rows_kernel<BF16, DIM>), grid, dim3(kThreads), 0, stream, s, 16 * p.tiles, \
                     rows_turn)
  if (s.a.dim == 64) {
    if (s.a.bf16) PAIR_JOIN(true, 64); else PAIR_JOIN(false, 64);
  } else {
    if (s.a.bf16) PAIR_JOIN(true, 128); else PAIR_JOIN(false, 128);
  }
#undef PAIR_JOIN
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

size_t attention_rows_workspace(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                                int32_t bits, int32_t max_q, int32_t max_len) {
  return plan_of(n, q_heads, kv_heads, dim, bits, max_q, max_len).total;
}

int64_t attention_rows_groups(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                              int32_t bits, int32_t max_q, int32_t max_len) {
  const Plan p = plan_of(n, q_heads, kv_heads, dim, bits, max_q, max_len);
  return (p.runs > n ? p.runs : n) * kv_heads;       // the joins: one for a request and head
}

int launch_attention_rows(const AttnCall& a, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(a.n, a.q_heads, a.kv_heads, a.dim, a.bits, a.max_q, a.max_len);
  const RowArgs s = args_of(a, p, workspace);
  if (a.bits == 8) return launch_mx8(s, p, stream);
  if (a.bits == 4) return launch_mx4(s, p, stream);
  return launch_of<16>(s, p, stream);
}

}  // namespace pair
