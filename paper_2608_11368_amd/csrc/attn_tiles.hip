// Attention of chunks of new tokens: the launches, and what surrounds the tiles
// (attn_tiles.hpp has the kernels' body).
#include "attn_tiles.hpp"

namespace pair {

using namespace tiles;

namespace {

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

}  // namespace

Plan tiles::plan_tiles(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim,
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

int tiles::count_tiles(const TileArgs& s, hipStream_t stream) {
  hipLaunchKernelGGL(tile_starts_kernel, dim3(1), dim3(1024), 0, stream, s);
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

int tiles::join_tiles(const TileArgs& s, hipStream_t stream) {
  const int64_t rows = s.a.tokens * s.a.q_heads;
  const dim3 grid((unsigned)((rows + kWaves - 1) / kWaves));
#define PAIR_JOIN(BF16, DIM)                                                                     \
  hipLaunchKernelGGL((join_tiles_kernel<BF16, DIM>), grid, dim3(kThreads), 0, stream, s)
  if (s.a.dim == 64) {
    if (s.a.bf16) PAIR_JOIN(true, 64); else PAIR_JOIN(false, 64);
  } else {
    if (s.a.bf16) PAIR_JOIN(true, 128); else PAIR_JOIN(false, 128);
  }
#undef PAIR_JOIN
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

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
    wp = rows::plan_of(a.n, a.q_heads, a.kv_heads, a.dim, a.bits, a.max_q, a.max_len);
    w = rows::args_of(a, wp, few_workspace);
  }
  const rows::RowArgs* few = few_workspace != nullptr ? &w : nullptr;
  if (a.bits == 8) return launch_mx8(s, p, few, &wp, stream);
  if (a.bits == 4) return launch_mx4(s, p, few, &wp, stream);
  return launch_of<16>(s, p, few, &wp, stream);
}

}  // namespace pair
