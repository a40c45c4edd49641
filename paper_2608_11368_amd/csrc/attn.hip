// Causal attention of each request's new tokens over its pages of a key/value
// cache:
//     s_j = scale <q, k_j>,  l = sum_j exp(s_j),  out = sum_j exp(s_j) v_j / l
// over the keys j <= len - Q + i of token i, with the running maximum and sum
// of the softmax, so that scores are never stored.
//
// One wave per token and query head: the lanes take 64 keys at a time, one
// score each, then add the 64 value rows with a lane for every second element.
#include "attn.hpp"

namespace pair {

namespace {

template <bool BF16>
__device__ __forceinline__ float to_f32(uint16_t b) {
  return BF16 ? __uint_as_float((uint32_t)b << 16) : (float)__builtin_bit_cast(_Float16, b);
}

template <bool BF16>
__device__ __forceinline__ uint16_t from_f32(float v) {
  if (BF16) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40u);
    return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
  }
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}

template <bool BF16, int DIM>
__global__ __launch_bounds__(kWave) void attention_row_kernel(AttnCall a, FastDiv page) {
  __shared__ float qs[DIM];
  const int lane = threadIdx.x;
  const int64_t t = blockIdx.x;
  const int h = blockIdx.y;
  // the request of this token
  int64_t lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (a.q_offsets[mid + 1] > t)
      hi = mid;
    else
      lo = mid + 1;
  }
  const int64_t r = lo, q0 = a.q_offsets[r], q1 = a.q_offsets[r + 1];
  if (q0 > t || q1 <= t || q1 > a.tokens || q0 < 0) {
    if (lane == 0) raise_status(a.d_status, PAIR_ST_BAD_GROUP);
    return;
  }
  int64_t len = a.lens[r];
  if (len < 0 || len > a.max_len || len > a.ldt * page.d || q1 - q0 > a.max_q) {
    if (lane == 0) raise_status(a.d_status, PAIR_ST_LENGTH);
    len = len < 0 ? 0 : (len > a.ldt * page.d ? a.ldt * page.d : len);
  }
  const int64_t seen0 = len - (q1 - q0) + (t - q0) + 1;
  const int seen = (int)(seen0 < 0 ? 0 : (seen0 < len ? seen0 : len));
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + t * a.q_token + h * a.q_head;
  for (int d = lane; d < DIM; d += kWave) qs[d] = to_f32<BF16>(q[d]);
  __syncthreads();
  const int64_t kvh = h / (a.q_heads / a.kv_heads);
  float m = -INFINITY, l = 0.0f, acc[DIM / kWave];
  for (int e = 0; e < DIM / kWave; ++e) acc[e] = 0.0f;
  for (int j0 = 0; j0 < seen; j0 += kWave) {
    const int j = j0 + lane;
    float s = -INFINITY;
    int64_t at = 0;
    if (j < seen) {
      const uint32_t pg = div_by((uint32_t)j, page);
      int64_t id = a.table[r * a.ldt + pg];
      if (id < 0 || id >= a.cache.n_pages) {
        raise_status(a.d_status, PAIR_ST_PAGES);
        id = 0;
      }
      at = id * a.cache.page_stride + (int64_t)(j - pg * page.d) * a.cache.slot_stride +
           kvh * a.cache.head_stride;
      const uint16_t* k = static_cast<const uint16_t*>(a.k_cache) + at;
      float x = 0.0f;
      for (int d = 0; d < DIM; ++d) x = __builtin_fmaf(qs[d], to_f32<BF16>(k[d]), x);
      s = x * a.scale;
    }
    float top = s;
    for (int w = 1; w < kWave; w <<= 1) top = fmaxf(top, __shfl_xor(top, w, kWave));
    const float mn = fmaxf(m, top);
    const float base = mn == -INFINITY ? 0.0f : mn;
    const float p = j < seen ? __expf(s - base) : 0.0f;
    const float keep = __expf(m - base);
    l = l * keep + wave_sum(p);
    for (int e = 0; e < DIM / kWave; ++e) acc[e] *= keep;
    const int n = seen - j0 < kWave ? seen - j0 : kWave;
    for (int w = 0; w < n; ++w) {
      const float pw = __shfl(p, w, kWave);
      const int64_t aw = __shfl(at, w, kWave);
      const uint16_t* v = static_cast<const uint16_t*>(a.v_cache) + aw;
      for (int e = 0; e < DIM / kWave; ++e)
        acc[e] = __builtin_fmaf(pw, to_f32<BF16>(v[e * kWave + lane]), acc[e]);
    }
    m = mn;
  }
  uint16_t* o = static_cast<uint16_t*>(a.out) + t * a.out_token + h * a.out_head;
  for (int e = 0; e < DIM / kWave; ++e)
    o[e * kWave + lane] = from_f32<BF16>(seen > 0 ? acc[e] / l : 0.0f);
  if (a.lse != nullptr && lane == 0)
    a.lse[t * a.q_heads + h] = seen > 0 ? m + __logf(l) : -INFINITY;
}

}  // namespace

size_t attention_workspace_bytes(int64_t n, int64_t, int32_t q_heads, int32_t kv_heads,
                                 int32_t dim, int32_t max_q, int32_t max_len) {
  return attention_rows_workspace(n, q_heads, kv_heads, dim, max_q, max_len);
}

int launch_attention(const AttnCall& a, void* workspace, hipStream_t stream) {
  if ((int64_t)a.max_q * (a.q_heads / a.kv_heads) <= kRowsMost)
    return launch_attention_rows(a, workspace, stream);
  const FastDiv page = fast_div((uint32_t)a.cache.page);
  const dim3 grid((unsigned)a.tokens, (unsigned)a.q_heads);
#define PAIR_ATTN(BF, D_) \
  hipLaunchKernelGGL((attention_row_kernel<BF, D_>), grid, dim3(kWave), 0, stream, a, page)
  if (a.bf16) {
    if (a.dim == 64) PAIR_ATTN(true, 64); else PAIR_ATTN(true, 128);
  } else {
    if (a.dim == 64) PAIR_ATTN(false, 64); else PAIR_ATTN(false, 128);
  }
#undef PAIR_ATTN
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace pair
