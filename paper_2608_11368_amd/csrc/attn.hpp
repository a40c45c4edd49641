// Shared by the attention kernels: matrix instructions on 16-bit operands held
// as raw dwords, the checks of a request, and the page lookups.
#pragma once

#include <math.h>

#include "paged.hpp"

namespace pair {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// D[m][n] += sum_k A[m][k] B[k][n] over one wave.  16x16x32: lane (x = lane & 15,
// g = lane >> 4) holds A[x][8 g ..], B[8 g ..][x] and D[4 g + i][x], i < 4.
template <bool BF16>
__device__ __forceinline__ f32x4_t mma16(u32x4_t a, u32x4_t b, f32x4_t c) {
  if (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                   __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a),
                                                __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// 32x32x16: lane (x = lane & 31, h = lane >> 5) holds A[x][8 h ..], B[8 h ..][x]
// and D[8 (i / 4) + 4 h + i % 4][x], i < 16.
template <bool BF16>
__device__ __forceinline__ f32x16_t mma32(u32x4_t a, u32x4_t b, f32x16_t c) {
  if (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                   __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a),
                                                __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// Two values rounded to nearest even, the first in the low half.
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if (BF16) {
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
  }
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}

// The matrix cores take the softmax's weights in the type of the values, so they
// are rounded to it (their sum l is of the unrounded ones, in fp32): relative to
// 64 bits that makes outputs 1.4 times as far off as rounding them alone does.
// fp16 has no room for small weights below the running maximum's 1: from 2^-14
// they lose bits and below 2^-25 they would vanish from the output while l still
// counts them.  The maximum may lag by 2^8 and fp16 ends at 2^16, so all weights
// are lifted by 2^7, l with them: they keep their bits down to 2^-21 and an
// error of 2^-32 below.
template <bool BF16>
constexpr float kLift = BF16 ? 0.0f : 7.0f;   // log2

// log of the sum of exp(score) from the running maximum and the lifted sum, both
// of powers of two.
template <bool BF16>
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m - kLift<BF16> + __builtin_amdgcn_logf(l)) * 0.69314718056f;
}

template <bool BF16>
__device__ __forceinline__ float half_value(uint32_t bits) {   // of the low 16 bits
  return BF16 ? __uint_as_float(bits << 16)
              : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// Whether either half of a dword has all exponent bits set (NaN or infinity).
template <bool BF16>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  const uint32_t e = BF16 ? 0x7f80u : 0x7c00u;
  return (w & e) == e || ((w >> 16) & e) == e;
}

// A request as the kernels see it; false (with status bits) if its offsets or
// lengths do not fit the call, and nothing of it is then read or written.
struct Request {
  int64_t q0;       // first row of q
  int32_t tokens;   // new tokens
  int32_t len;      // keys
};

__device__ __forceinline__ bool attention_request(const AttnCall& a, uint32_t page, int64_t r,
                                                  Request* q, int32_t* bad) {
  const int64_t q0 = a.q_offsets[r], q1 = a.q_offsets[r + 1];
  const int32_t len = a.lens[r];
  if (q0 < 0 || q1 < q0 || q1 > a.tokens || (r == 0 && q0 != 0)) {
    *bad |= PAIR_ST_BAD_GROUP;
    return false;
  }
  if (len < 0 || len > a.max_len || len > a.ldt * page || q1 - q0 > a.max_q) {
    *bad |= PAIR_ST_LENGTH;
    return false;
  }
  q->q0 = q0;
  q->tokens = (int32_t)(q1 - q0);
  q->len = len;
  return true;
}

// Last key that token i of the request sees (below 0: none).
__device__ __forceinline__ int limit_of(const Request& q, int token) {
  return q.len - q.tokens + token;
}

// Entry `i` (wave-uniform) of a table row, by a scalar load: nothing that runs
// beside the attention writes the table.
__device__ __forceinline__ int32_t table_entry(const int32_t* row, uint32_t i) {
  typedef const __attribute__((address_space(4))) int32_t* scalar_ptr;
  return ((scalar_ptr)(uintptr_t)row)[i];
}

// A page id that may be used as an index: one outside the cache is counted in
// *bad and replaced by page 0 (the request's results are then unspecified).
__device__ __forceinline__ int32_t checked_page(const AttnCall& a, int32_t id, int32_t* bad) {
  const bool ok = (uint32_t)id < (uint32_t)a.cache.n_pages;
  *bad |= ok ? 0 : PAIR_ST_PAGES;
  return ok ? id : 0;
}

// The launches of attn_rows.hip (requests of at most kRowsMost rows, a row being
// a query head of a token) and attn_tiles.hip (those of at least `least_rows`;
// with a workspace for the others, both).  32 rows of 8 heads of 128, by the first
// and by the second: 2 requests of 131,000 keys 187 and 207 us, 256 of 1000 200 and
// 215, 32 of 4000 112 and 104.  Of 40 and 64 rows, for which only tiles are built:
// 209 and 231, 222 and 233, 105 and 109.
constexpr int kRowsMost = 32;

size_t attention_rows_workspace(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                                int32_t max_q, int32_t max_len);
int64_t attention_rows_groups(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t dim,
                              int32_t max_q, int32_t max_len);
int launch_attention_rows(const AttnCall& a, void* workspace, hipStream_t stream);
size_t attention_tiles_workspace(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                                 int32_t dim, int32_t max_len);
int64_t attention_tiles_groups(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                               int32_t dim, int32_t max_len);
int launch_attention_tiles(const AttnCall& a, int32_t least_rows, void* few_workspace,
                           void* workspace, hipStream_t stream);

}  // namespace pair
