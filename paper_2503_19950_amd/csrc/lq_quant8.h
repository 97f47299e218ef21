// What the kernels of the 8-bit cache share: loads, and the quantizer, on the 16-bit patterns of pairs of values.
#pragma once
#include "lq_device.h"

namespace lq {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {   // reads beyond it: zeros
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t rs, int off) { return __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0); }

// Magnitudes of a pair of values of T order like their 15 low bits as integers.
__device__ __forceinline__ uint32_t max_pair(uint32_t m, uint32_t x) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const u16x2 a = __builtin_bit_cast(u16x2, m), b = __builtin_bit_cast(u16x2, x & 0x7FFF7FFFu);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, b));
}

// The largest value of T that four significant bits carry no further: 1.875 * 2^127, 1.875 * 2^15.
template <bool BF16>
__device__ __forceinline__ constexpr uint32_t cut_bits() { return BF16 ? 0x7F70u : 0x7B80u; }

// Exponent of a block's scale from the bits of its largest magnitude.  448 = 1.75 * 2^8: the addition carries into the
// exponent exactly where the significand is above 1.75.
template <bool BF16>
__device__ __forceinline__ int scale_exponent(uint32_t top) {
  const uint32_t f = __float_as_uint(t2f<BF16>((uint16_t)(top < cut_bits<BF16>() ? top : cut_bits<BF16>())));
  const int e = (int)((f + 0x1FFFFFu) >> 23) - 127 - 8;
  return e < -126 ? -126 : e;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four codes from two pairs of values.  The products are exact; the bound matters to values beyond the cut only.
template <bool BF16>
__device__ __forceinline__ uint32_t codes4(uint32_t a, uint32_t b, float inv, float most) {
  auto scaled = [&](uint32_t u) { return __builtin_amdgcn_fmed3f(t2f<BF16>((uint16_t)u) * inv, most, -most); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(a & 0xFFFF), scaled(a >> 16), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled(b & 0xFFFF), scaled(b >> 16), w, true);
}

}  // namespace lq
