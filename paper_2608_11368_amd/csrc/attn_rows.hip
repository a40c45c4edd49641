// Attention of a few new tokens per request: the launches, and the joining of
// requests that were cut (attn_rows.hpp has the kernel's body).
#include "attn_rows.hpp"

namespace pair {

using namespace rows;

namespace {

template <bool BF16, int DIM, int NT, bool ALIGNED, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, 2) void attention_rows_kernel(RowArgs s) {
  __shared__ WaveLds<DIM, NT> lds[WAVES];
  __shared__ int32_t start[WAVES == kWaves ? kMostScanned + 1 : 1];
  __shared__ int32_t sums[kWaves];
  serve<BF16, DIM, NT, ALIGNED, WAVES>(s, blockIdx.x, lds, start, sums);
}

// Joins the partial sums of the requests that were cut: one workgroup per
// request, head and row.  The parts' maxima first, a lane each, then their sums
// with several parts' loads in flight.
template <bool BF16, int DIM>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(RowArgs s, int rows_slot) {
  const int64_t heads = s.a.kv_heads;
  const int64_t r = blockIdx.x / (uint32_t)s.a.kv_heads;
  const int kvh = (int)(blockIdx.x - r * heads);
  const int i = blockIdx.y;
  const int64_t u0 = s.starts[r], u1 = s.starts[r + 1];
  if (u0 == u1) return;
  const int64_t units = s.starts[s.a.n], runs = runs_of(s, units);
  // run of unit u: the last that starts at or before it
  const int64_t w0 = quotient((u0 + 1) * runs - 1, units), w1 = quotient(u1 * runs - 1, units);
  if (w0 == w1) return;
  Request q;
  int32_t bad = 0;
  if (!attention_request(s.a, s.page.d, r, &q, &bad)) return;
  if (i >= q.tokens * (int)s.group.d) return;
  const int tok = (int)div_by((uint32_t)i, s.group);
  const int h = kvh * (int)s.group.d + i - tok * (int)s.group.d;
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  constexpr int PER = DIM / kWave;
  __shared__ float weight[kMostRuns], sum[kWaves][DIM];
  const int parts = (int)(w1 - w0) + 1;
  // a request that starts inside a run is in the run's second part
  const int64_t first = 2 * w0 + (run_start(units, runs, w0) != u0 ? 1 : 0);
  auto place = [&](int p) {
    return ((p == 0 ? first : 2 * (w0 + p)) * heads + kvh) * rows_slot + i;
  };
  float m = -INFINITY;
  for (int p = lane; p < parts; p += kWave) m = fmaxf(m, s.part_ml[place(p) * 2]);
#pragma unroll
  for (int by = 1; by < kWave; by <<= 1) m = fmaxf(m, __shfl_xor(m, by, kWave));
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  for (int p = lane; p < parts; p += kWave) {
    const float mp = s.part_ml[place(p) * 2], lp = s.part_ml[place(p) * 2 + 1];
    const bool none = mp == -INFINITY && lp == 0.0f;       // saw no key
    const float f = none ? 0.0f : __builtin_amdgcn_exp2f(mp - base);
    l += none ? 0.0f : lp * f;
    if (wave == 0) weight[p] = f;
  }
  l = wave_sum(l);
  __syncthreads();
  float o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.0f;
#pragma unroll 4
  for (int p = wave; p < parts; p += kWaves) {
    const float f = weight[p];
    const float* from = s.part_o + place(p) * DIM;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = __builtin_fmaf(from[e * kWave + lane], f, o[e]);
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) sum[wave][e * kWave + lane] = o[e];
  __syncthreads();
  if (threadIdx.x >= DIM / 2) return;
  const int d = threadIdx.x * 2;
  float a = 0.0f, b = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    a += sum[w][d];
    b += sum[w][d + 1];
  }
  const bool none = limit_of(q, tok) < 0;
  const float inv = 1.0f / l;
  *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(s.a.out) + (q.q0 + tok) * s.a.out_token +
                               h * s.a.out_head + d) = none ? 0u : pack2<BF16>(a * inv, b * inv);
  if (s.a.lse != nullptr && threadIdx.x == 0)
    s.a.lse[(q.q0 + tok) * s.a.q_heads + h] =
        none ? -INFINITY : log_sum<BF16>(m, l);
}

template <bool BF16, int DIM>
int launch(const RowArgs& s, const Plan& p, hipStream_t stream) {
  const int64_t grid = groups_of(s.a, p);
  const bool aligned = s.page.d % 16 == 0;
  // Uncut workgroups that have a compute unit each: eight waves instead of four
  // (4 requests of 400 keys, 8 heads of 128: 6.8 us instead of 7.8, of 1000: 9.3
  // instead of 11.3; 32 requests, a workgroup for every unit: 22.1 both).
  const bool wide = p.runs == 0 && grid <= device_cu_count();
#define PAIR_ROWS(NT, AL, W)                                                                     \
  hipLaunchKernelGGL((attention_rows_kernel<BF16, DIM, NT, AL, W>), dim3((unsigned)grid),         \
                     dim3(W * kWave), 0, stream, s)
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

}  // namespace

Plan rows::plan_of(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t max_q,
                   int32_t max_len) {
  Plan p;
  const int64_t rows = (int64_t)max_q * (q_heads / kv_heads);
  p.rows = (int)(rows < kRowsMost ? rows : kRowsMost);
  p.tiles = p.rows <= 16 ? 1 : 2;
  // Cut into equal runs (units are counted in 31 bits) unless the longest head is
  // eight steps, which take less than the second launch would (4 requests of 700
  // keys: 8.0 us uncut, 9.5 us cut; of 1000: 9.3 and 9.9; of 2000: 21 and 11; 32
  // requests of 1000: 22 and 27), or the requests are so many that they fill the
  // card by themselves.
  const int64_t most = n * ((max_len + kUnit - 1) / kUnit);
  int64_t runs = 2 * (int64_t)device_cu_count() / kv_heads;   // two workgroups fit a compute unit
  if (runs > most) runs = most;
  if (runs > kMostRuns) runs = kMostRuns;
  if (runs < 1) runs = 1;
  p.runs = n > kMostScanned || max_len <= 8 * kUnit || most > 0x7fffffff ? 0 : (int32_t)runs;
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
  const dim3 grid((unsigned)(s.a.n * s.a.kv_heads), (unsigned)p.rows);
#define PAIR_JOIN(BF16, DIM)                                                                     \
  hipLaunchKernelGGL((join_rows_kernel<BF16, DIM>), grid, dim3(kThreads), 0, stream, s, 16 * p.tiles)
  if (s.a.dim == 64) {
    if (s.a.bf16) PAIR_JOIN(true, 64); else PAIR_JOIN(false, 64);
  } else {
    if (s.a.bf16) PAIR_JOIN(true, 128); else PAIR_JOIN(false, 128);
  }
#undef PAIR_JOIN
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

size_t attention_rows_workspace(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                                int32_t max_q, int32_t max_len) {
  return plan_of(n, q_heads, kv_heads, dim, max_q, max_len).total;
}

int64_t attention_rows_groups(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                              int32_t max_q, int32_t max_len) {
  const Plan p = plan_of(n, q_heads, kv_heads, dim, max_q, max_len);
  return (p.runs > n ? p.runs : n) * kv_heads;       // the joins: one for a request and head
}

int launch_attention_rows(const AttnCall& a, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(a.n, a.q_heads, a.kv_heads, a.dim, a.max_q, a.max_len);
  const RowArgs s = args_of(a, p, workspace);
  if (a.dim == 64) return a.bf16 ? launch<true, 64>(s, p, stream) : launch<false, 64>(s, p, stream);
  return a.bf16 ? launch<true, 128>(s, p, stream) : launch<false, 128>(s, p, stream);
}

}  // namespace pair
