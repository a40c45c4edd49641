// The paged cache in 8 and 4 bits: new keys and values quantised into their slots
// (pair_cache_store_mx), and cached ones read back (pair_cache_load_mx).
#include "mx.hpp"

namespace pair {

namespace {

constexpr int kThreads = 256;
// Pieces of a lane at a time.  HBM-bound (a copy of 2 GiB runs at 4.9 TB/s of reads and
// writes): 32,467 fp16 tokens of 8 heads of 128 into 8 bits, 202 MB, 42 us and 4.8
// TB/s with one, 44 with two, 48 with four; 60,000 of 4 heads of 128 out of 8 bits
// 32.5, 32.0 and 41 us.  Pieces of 8 elements stored in 48 us.
constexpr int kStored = 1, kLoaded = 2;

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

// A piece is 16 elements of a row: piece i of a call is piece i % per_token of token
// i / per_token, the keys' pieces before the values'.  Two neighbouring lanes have a
// block.
constexpr int kPiece = 16;

struct MoveArgs {
  unsigned char* rows[2];             // 16-bit rows: keys, values
  unsigned char* codes[2];
  unsigned char* scales[2];
  int64_t token_bytes, head_row_bytes;
  int64_t page_bytes, slot_bytes, head_bytes;
  int64_t scale_page, scale_slot, scale_head;
  FastDiv page, per_token, per_head;
  uint32_t half;                      // pieces of a token's keys
  int64_t slots_total;
  const int64_t* slots;
  int64_t tokens;
  int32_t* d_status;
};

// Where a piece lies.
struct Place {
  unsigned char* row;
  unsigned char* code;
  unsigned char* scale;               // of its block
  bool stored;                        // false: the token has no slot
};

template <int BITS>
__device__ __forceinline__ Place place_of(const MoveArgs& a, int64_t t0, uint32_t i) {
  const uint32_t tok = div_by(i, a.per_token);
  uint32_t c = i - tok * a.per_token.d;
  const int64_t slot = a.slots[t0 + tok];
  const bool value = c >= a.half;
  if (value) c -= a.half;
  const uint32_t h = div_by(c, a.per_head);
  const uint32_t d = c - h * a.per_head.d;
  Place p;
  p.row = (value ? a.rows[1] : a.rows[0]) + (t0 + tok) * a.token_bytes + h * a.head_row_bytes +
          d * (uint32_t)(2 * kPiece);
  if (slot >= a.slots_total) raise_status(a.d_status, PAIR_ST_PAGES);
  p.stored = slot >= 0 && slot < a.slots_total;
  const uint32_t y = p.stored ? (uint32_t)slot : 0u;
  const uint32_t pg = div_by(y, a.page), at = y - pg * a.page.d;
  p.code = (value ? a.codes[1] : a.codes[0]) + pg * a.page_bytes + at * a.slot_bytes +
           h * a.head_bytes + d * (uint32_t)(kPiece * BITS / 8);
  p.scale = (value ? a.scales[1] : a.scales[0]) + pg * a.scale_page + at * a.scale_slot +
            h * a.scale_head + d / (uint32_t)(kMxBlock / kPiece);
  return p;
}

__device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a),
                                                                __builtin_bit_cast(u16x2_t, b)));
}

__device__ __forceinline__ uint32_t min16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2_t, a),
                                                                __builtin_bit_cast(u16x2_t, b)));
}

// Byte of the smallest scale, from 2^-100 on, under which a block's largest
// magnitude is at most the largest code (448 = 1.75 * 2^8, 6 = 1.5 * 2^2), so that
// no element is off by more than half a step.
template <int BITS>
__device__ __forceinline__ uint32_t scale_byte(float most) {
  const uint32_t bits = __float_as_uint(most);
  const int e = (int)(bits >> 23) - (BITS == 8 ? 8 : 2) +
                ((bits & 0x7fffffu) > (BITS == 8 ? 0x600000u : 0x400000u) ? 1 : 0);
  return (uint32_t)(e < 27 ? 27 : e);
}

// Two values with their signs as codes: bytes 2 (I % 2) .. of `old` (8 bits), byte I
// of it (4 bits).
template <bool BF16, int BITS, int I>
__device__ __forceinline__ uint32_t mx_code(uint32_t old, uint32_t two, float scale) {
  if (BITS == 8) {
    const mx_s16x2_t o = __builtin_bit_cast(mx_s16x2_t, old);
    if (BF16)
      return __builtin_bit_cast(uint32_t,
                                __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
                                    o, __builtin_bit_cast(mx_bf16x2_t, two), scale, (I & 1) != 0));
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(
                                  o, __builtin_bit_cast(mx_f16x2_t, two), scale, (I & 1) != 0));
  }
  if (BF16)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(mx_bf16x2_t, two),
                                                     scale, I & 3);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(mx_f16x2_t, two), scale,
                                                  I & 3);
}

// 16 elements, half a block.  Magnitudes are compared as the integers that their
// bits are; the two lanes of a block exchange their largest.  A block that holds a
// NaN or an infinity becomes NaN.
template <bool BF16, int BITS>
__device__ __forceinline__ Codes<BITS, kPiece> quantise(const u32x4_t (&v)[2], uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max16x2(top, v[i >> 2][i & 3] & 0x7fff7fffu);
  uint32_t most = (top & 0xffffu) > (top >> 16) ? top & 0xffffu : top >> 16;
  const uint32_t other =
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xf, 0xf, false);
  most = most > other ? most : other;
  const bool odd = most >= (BF16 ? 0x7f80u : 0x7c00u);
  // The last numbers of the 16-bit type would be rounded past its range: the
  // largest that stays within is 1.875 (1.5 in 4 bits) times its last power of two.
  constexpr uint32_t kTop = BF16 ? (BITS == 8 ? 0x7f70u : 0x7f40u) : (BITS == 8 ? 0x7b80u : 0x7a00u);
  if (most > kTop) most = kTop;
  const float m = BF16 ? __uint_as_float(most << 16)
                       : (float)__builtin_bit_cast(_Float16, (uint16_t)most);
  *byte = odd ? 255u : scale_byte<BITS>(m);
  const float scale = mx_scale(*byte);
  Codes<BITS, kPiece> c;
#pragma unroll
  for (int w = 0; w < Codes<BITS, kPiece>::kWords; ++w) c.w[w] = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t in = v[i >> 2][i & 3];
    const uint32_t two = min16x2(in & 0x7fff7fffu, kTop | kTop << 16) | (in & 0x80008000u);
    uint32_t* w = &c.w[i / (16 / BITS)];
    const int at = i % (16 / BITS);
    *w = at == 0   ? mx_code<BF16, BITS, 0>(*w, two, scale)
         : at == 1 ? mx_code<BF16, BITS, 1>(*w, two, scale)
         : at == 2 ? mx_code<BF16, BITS, 2>(*w, two, scale)
                   : mx_code<BF16, BITS, 3>(*w, two, scale);
  }
#pragma unroll
  for (int w = 0; w < Codes<BITS, kPiece>::kWords; ++w)
    if (odd) c.w[w] = 0;
  return c;
}

template <bool BF16, int BITS>
__global__ __launch_bounds__(kThreads) void mx_store_kernel(MoveArgs a, int tokens_per_group) {
  const int64_t t0 = (int64_t)blockIdx.x * tokens_per_group;
  const int64_t left = a.tokens - t0;
  const uint32_t n =
      (uint32_t)(left < tokens_per_group ? left : tokens_per_group) * a.per_token.d;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kThreads * kStored) {
    u32x4_t v[kStored][2];
    Place p[kStored];
#pragma unroll
    for (int s = 0; s < kStored; ++s) {
      const uint32_t i = i0 + s * kThreads;
      p[s].stored = false;
      if (i < n) {
        p[s] = place_of<BITS>(a, t0, i);
        if (p[s].stored) {
          v[s][0] = *reinterpret_cast<const u32x4_t*>(p[s].row);
          v[s][1] = *reinterpret_cast<const u32x4_t*>(p[s].row + 16);
        }
      }
    }
    bool odd = false;
#pragma unroll
    for (int s = 0; s < kStored; ++s) {
      if (!p[s].stored) continue;               // the same for the lanes of a block
      uint32_t byte;
      const Codes<BITS, kPiece> c = quantise<BF16, BITS>(v[s], &byte);
      c.store(p[s].code);
      if ((threadIdx.x & 1) == 0) *p[s].scale = (unsigned char)byte;
      odd |= byte == 255u;
    }
    if (odd) raise_status(a.d_status, PAIR_ST_NONFINITE);
  }
}

template <bool BF16, int BITS>
__global__ __launch_bounds__(kThreads) void mx_load_kernel(MoveArgs a, int tokens_per_group) {
  const int64_t t0 = (int64_t)blockIdx.x * tokens_per_group;
  const int64_t left = a.tokens - t0;
  const uint32_t n =
      (uint32_t)(left < tokens_per_group ? left : tokens_per_group) * a.per_token.d;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kThreads * kLoaded) {
    Codes<BITS, kPiece> c[kLoaded];
    uint32_t byte[kLoaded];
    unsigned char* to[kLoaded];
#pragma unroll
    for (int s = 0; s < kLoaded; ++s) {
      const uint32_t i = i0 + s * kThreads;
      to[s] = nullptr;
      byte[s] = 0;
#pragma unroll
      for (int w = 0; w < Codes<BITS, kPiece>::kWords; ++w) c[s].w[w] = 0;
      if (i < n) {
        const Place p = place_of<BITS>(a, t0, i);
        to[s] = p.row;
        if (p.stored) {
          c[s].load(p.code);
          byte[s] = *p.scale;
        }
      }
    }
#pragma unroll
    for (int s = 0; s < kLoaded; ++s) {
      if (to[s] == nullptr) continue;
      uint32_t v[kPiece / 2];
      c[s].template values<BF16>(mx_scale(byte[s]), v);
      *reinterpret_cast<u32x4_t*>(to[s]) = u32x4_t{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<u32x4_t*>(to[s] + 16) = u32x4_t{v[4], v[5], v[6], v[7]};
    }
  }
}

}  // namespace

int launch_mx_move(bool store, const MxCache& cache, int64_t tokens, bool bf16, void* k, void* v,
                   int64_t token_stride, int64_t row_head_stride, const int64_t* slots,
                   int32_t* d_status, hipStream_t stream) {
  MoveArgs a;
  a.rows[0] = static_cast<unsigned char*>(k);
  a.rows[1] = static_cast<unsigned char*>(v);
  a.codes[0] = static_cast<unsigned char*>(cache.k);
  a.codes[1] = static_cast<unsigned char*>(cache.v);
  a.scales[0] = static_cast<unsigned char*>(cache.k_scale);
  a.scales[1] = static_cast<unsigned char*>(cache.v_scale);
  a.token_bytes = token_stride * 2;
  a.head_row_bytes = row_head_stride * 2;
  a.page_bytes = cache.page_stride;
  a.slot_bytes = cache.slot_stride;
  a.head_bytes = cache.head_stride;
  a.scale_page = cache.scale_page;
  a.scale_slot = cache.scale_slot;
  a.scale_head = cache.scale_head;
  a.page = fast_div((uint32_t)cache.page);
  const uint32_t per_head = (uint32_t)cache.dim / kPiece;
  a.per_head = fast_div(per_head);
  a.half = (uint32_t)cache.kv_heads * per_head;
  a.per_token = fast_div(2 * a.half);
  a.slots_total = cache.n_pages * cache.page;
  a.slots = slots;
  a.tokens = tokens;
  a.d_status = d_status;
  // About the lanes' pieces, at least one token a workgroup, and no more of them
  // than a launch can have (below 2^32 threads).
  int per_group = (int)(kThreads * (store ? kStored : kLoaded) / a.per_token.d);
  const int least = (int)((tokens + (1 << 23) - 1) >> 23);
  if (per_group < least) per_group = least;
  const dim3 grid((unsigned)((tokens + per_group - 1) / per_group));
#define PAIR_MOVE(KERNEL)                                                                        \
  do {                                                                                           \
    if (cache.bits == 8) {                                                                       \
      if (bf16)                                                                                  \
        hipLaunchKernelGGL((KERNEL<true, 8>), grid, dim3(kThreads), 0, stream, a, per_group);     \
      else                                                                                       \
        hipLaunchKernelGGL((KERNEL<false, 8>), grid, dim3(kThreads), 0, stream, a, per_group);    \
    } else {                                                                                     \
      if (bf16)                                                                                  \
        hipLaunchKernelGGL((KERNEL<true, 4>), grid, dim3(kThreads), 0, stream, a, per_group);     \
      else                                                                                       \
        hipLaunchKernelGGL((KERNEL<false, 4>), grid, dim3(kThreads), 0, stream, a, per_group);    \
    }                                                                                            \
  } while (0)
  if (store) PAIR_MOVE(mx_store_kernel); else PAIR_MOVE(mx_load_kernel);
#undef PAIR_MOVE
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace pair
