// Helpers of the matrix-core attention kernels that gather codewords as rows of
// 4 dims from a binary16 table in LDS (gfx950, wave64).
#ifndef FIBQ_ATTN_ROWS4_H
#define FIBQ_ATTN_ROWS4_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fibq {
namespace dev {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

// maximum over the wavefront of v >= 0, in registers
__device__ __forceinline__ float wave_max_dpp(float v) {
  float x = v;
#define FIBQ_ROR(n) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + n, 0xf, 0xf, false)));
  FIBQ_ROR(8) FIBQ_ROR(4) FIBQ_ROR(2) FIBQ_ROR(1)
#undef FIBQ_ROR
  const int i = __float_as_int(x);
  return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(i, 0)), __int_as_float(__builtin_amdgcn_readlane(i, 16))),
               fmaxf(__int_as_float(__builtin_amdgcn_readlane(i, 32)), __int_as_float(__builtin_amdgcn_readlane(i, 48))));
}

// Transposing LDS read: in each 16-lane row, lane 4 a + e receives element e of
// the 4-element rows addressed by lanes a, a + 4, a + 8, a + 12.
__device__ __forceinline__ h4 tr_read(const unsigned char* lds_byte_addr) {
  s4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s4*)(lds_byte_addr));
  return __builtin_bit_cast(h4, r);
}

__device__ __forceinline__ float xmax(float v, int mask) {
  return fmaxf(v, __shfl_xor(v, mask, 64));
}
__device__ __forceinline__ float xsum(float v, int mask) { return v + __shfl_xor(v, mask, 64); }

// LDS byte offset of the 4-dim row b of a quarter: index b / KB of the quarter
// (w-bit indices, little-endian), row b % KB of its codeword.
template <int QW, int W, int KB>
__device__ __forceinline__ uint32_t qrow(const uint32_t (&qq)[QW], int b, int w) {
  if constexpr (W == 8 && KB == 1) {
    return ((qq[b >> 2] >> (8 * (b & 3))) & 0xFFu) * 8u;
  } else if constexpr (W == 12 && KB == 1) {  // bits 12 b .. 12 b + 11 of the quarter
    const int bit = 12 * b, wd = bit >> 5, sh = bit & 31;
    uint32_t v = qq[wd] >> sh;
    if (sh > 20) v |= qq[wd + 1] << (32 - sh);
    return (v & 0xFFFu) * 8u;
  } else {  // the quarter starts at bit 0 of qq
    const int i = b / KB;
    uint32_t v;
    if constexpr (QW == 1) {
      v = qq[0] >> (i * w);
    } else {
      const uint64_t u = (uint64_t)qq[0] | ((uint64_t)qq[1] << 32);
      v = (uint32_t)(u >> (i * w));
    }
    return (v & ((1u << w) - 1u)) * (8u * KB) + 8u * (b % KB);
  }
}

}  // namespace dev
}  // namespace fibq

#endif
