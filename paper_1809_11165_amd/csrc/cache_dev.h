// Device pieces shared by the cache's kernels: 8-bit rows, pages.
//
// E4M3 rows hold x / 2^e in blocks of 32 features; a power of two leaves a value's bits alone, so the block's rounding is that of the format itself
// (half a step, 2^-4 of a value), and values come back exact in fp32 and bf16.
#pragma once

#include "attend_dev.h"
#include "bbmm_cache.h"

namespace att {

__device__ __forceinline__ uint32_t over(uint32_t n, const Div& d) { return (uint32_t)(((uint64_t)n * d.m) >> d.s); }

constexpr int kExpLow = -117;                              // the smallest value, 2^-9 units, is a normal number of fp32 still

// The exponent of a block whose largest finite magnitude is `top`: 448 = 1.75 2^8.
__device__ __forceinline__ int block_exp(float top) {
  unsigned u = __float_as_uint(top);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return top == 0.f ? 0 : max(e, kExpLow);
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }   // -126 .. 127
// Scale of block n from the four bytes of a row's exponents.
__device__ __forceinline__ float block_scale(unsigned bytes, int n) { return __uint_as_float(((bytes >> (8 * n)) & 0xffu) << 23); }

// Two values (bytes 2 HI, 2 HI + 1 of `q`) times a power of two.
template <typename T> struct Wide;
template <> struct Wide<__bf16> {
  typedef __bf16 two __attribute__((ext_vector_type(2)));
  template <bool HI> static __device__ __forceinline__ two get(unsigned q, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, HI); }
};
template <> struct Wide<_Float16> {
  typedef _Float16 two __attribute__((ext_vector_type(2)));
  template <bool HI> static __device__ __forceinline__ two get(unsigned q, float scale) {
    return __builtin_bit_cast(two, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(q, scale, HI));
  }
};
template <> struct Wide<float> {
  typedef float two __attribute__((ext_vector_type(2)));
  template <bool HI> static __device__ __forceinline__ two get(unsigned q, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q, scale, HI); }
};

// The page of row `at` of sequence b, or -1.
__device__ __forceinline__ int page_of(const CacheArgs& c, int b, uint32_t index) {
  int p = c.table[(int64_t)b * c.max_pages + index];
  return (unsigned)p < (unsigned)c.pages ? p : -1;
}

}  // namespace att
