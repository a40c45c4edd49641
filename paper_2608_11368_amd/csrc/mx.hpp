// Codes of the paged cache in 8 and 4 bits (MXFP8 E4M3 and MXFP4 E2M1): blocks of
// 32 elements share a scale 2^(b - 127), b its byte (255: the block is NaN).
//
// The conversion instructions take the scale as an operand of which they use the
// exponent, and a code has at most 4 significant bits, so in the 16-bit types the
// values are exact (within the type's range); a scale of exponent 255 gives NaN.
// All 256 codes under all 256 scales were compared with the formats' definition.
#pragma once

#include "paged.hpp"

namespace pair {

typedef __bf16 mx_bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 mx_f16x2_t __attribute__((ext_vector_type(2)));
typedef short mx_s16x2_t __attribute__((ext_vector_type(2)));

constexpr int kMxBlock = 32;

__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Elements 2 i and 2 i + 1 of a dword of codes, as a pair of 16-bit values.
template <bool BF16, int BITS, int I>
__device__ __forceinline__ uint32_t mx_pair(uint32_t codes, float scale) {
  if (BITS == 8) {
    if (BF16)
      return __builtin_bit_cast(uint32_t,
                                __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, (I & 1) != 0));
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, (I & 1) != 0));
  }
  if (BF16)
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, I & 3));
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, I & 3));
}

// N elements of a row as they lie in a cache of BITS bits an element.
template <int BITS, int N>
struct Codes {
  static constexpr int kBytes = N * BITS / 8;
  static constexpr int kWords = kBytes >= 4 ? kBytes / 4 : 1;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const unsigned char* p) {
    if constexpr (kBytes == 16) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else if constexpr (kBytes == 8) {
      const u32x2_t v = *reinterpret_cast<const u32x2_t*>(p);
      w[0] = v[0];
      w[1] = v[1];
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }

  __device__ __forceinline__ void store(unsigned char* p) const {
    static_assert(kBytes == 16 || kBytes == 8, "wide stores");
    if constexpr (kBytes == 16)
      *reinterpret_cast<u32x4_t*>(p) = u32x4_t{w[0], w[1], w[2], w[3]};
    else
      *reinterpret_cast<u32x2_t*>(p) = u32x2_t{w[0], w[1]};
  }

  // The elements' values, two to a dword: all of one block.
  template <bool BF16>
  __device__ __forceinline__ void values(float scale, uint32_t (&to)[N / 2]) const {
    constexpr int kPairs = 16 / BITS;               // of a dword
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const uint32_t c = w[i / kPairs];
      const int at = i % kPairs;
      to[i] = at == 0   ? mx_pair<BF16, BITS, 0>(c, scale)
              : at == 1 ? mx_pair<BF16, BITS, 1>(c, scale)
              : at == 2 ? mx_pair<BF16, BITS, 2>(c, scale)
                        : mx_pair<BF16, BITS, 3>(c, scale);
    }
  }
};

}  // namespace pair
