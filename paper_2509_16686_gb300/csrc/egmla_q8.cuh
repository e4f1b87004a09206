// egmla_q8.cuh - the latent in 8 bits: e4m3 codes and one power-of-two scale per token.
//
// For a row c with a = max |c_f|: scale s = 2^e, e the least integer with a <= 448 2^e,
// kept between -100 and 119; code_f = e4m3(c_f / s) to the nearest, ties to even.  A
// power of two costs a floating format nothing but its smallest numbers (15 of e4m3's
// powers of two remain below the largest value), and makes division, product and the way
// back exact: s code_f has four significant bits and an exponent of bf16's normal range.
// A row with an infinity or a NaN has s = NaN, and reads back as NaN.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cstdint>

#include "../../include/egmla.h"

namespace egmla {

// shapes of the calls on the cache in 8 bits; EG_MLA_OK or the error code
int q8_check_dims(const eg_mla_dims* d);

// scale and 1 / scale for a row whose largest magnitude has the fp32 bits `most`; least: of
// the scale's exponent, at least -126 (both are normal numbers)
__device__ __forceinline__ void q8_scale(uint32_t most, float& scale, float& inverse, int least = -100) {
  // 448 = 1.75 2^8; (a subnormal `most` counts as 2^-127 and is far below the least scale)
  int e = static_cast<int>(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = min(max(e, least), 119);
  scale = __int_as_float((e + 127) << 23);
  inverse = __int_as_float((127 - e) << 23);
  if (most >= 0x7f800000u) scale = inverse = __int_as_float(0x7fffffff);
}

// two codes, the first in the low byte (a magnitude above 448 gives 448)
__device__ __forceinline__ uint32_t q8_encode2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

// four codes as fp32 values
__device__ __forceinline__ void q8_decode4(uint32_t w, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * i)), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// Codes of one row as bf16 values, exactly.  e4m3's sign, exponent and significand are put
// where bf16 has them, which gives the value times 2^-120, subnormal codes as subnormal
// numbers; one product with 2^120 s puts that right and applies the scale (above s = 2^7
// the rest of it takes a second).
struct Q8Widen {
  uint32_t mult, more;   // the factors, twice each
  __device__ __forceinline__ void set(float scale) {
    const uint32_t bits = __float_as_uint(scale);
    const int e = static_cast<int>(bits >> 23) - 127;
    mult = min(e + 120, 127) + 127;
    more = max(e - 7, 0) + 127;
    mult = mult << 7 | mult << 23;
    more = more << 7 | more << 23;
    if (bits >= 0x7f800000u) mult = 0x7fff7fffu, more = 0x3f803f80u;   // (a NaN; its sign bit is clear)
  }
  static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b) {
    const __nv_bfloat162 z = __hmul2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&z);
  }
  // codes in the bytes of w, the first in the low one, as two pairs: the low nibble of a code
  // is the second nibble of its bf16 value's low byte, the high nibble makes the high byte
  __device__ __forceinline__ void four(uint32_t w, uint32_t& lo, uint32_t& hi) const {
    const uint32_t a = (w << 4) & 0xf0f0f0f0u, b = ((w >> 4) & 0x07070707u) | (w & 0x80808080u);
    lo = mul(__byte_perm(a, b, 0x5140), mult);
    hi = mul(__byte_perm(a, b, 0x7362), mult);
  }
  // eight codes as a 16-byte unit
  __device__ __forceinline__ uint4 unit(uint32_t w0, uint32_t w1) const {
    uint4 z;
    four(w0, z.x, z.y);
    four(w1, z.z, z.w);
    return z;
  }
  // whether values need the second factor (apart, so that rows that do not pay nothing for it)
  __device__ __forceinline__ bool unfinished() const { return more != 0x3f803f80u; }
  __device__ __forceinline__ void finish(uint4& z) const {
    z = make_uint4(mul(z.x, more), mul(z.y, more), mul(z.z, more), mul(z.w, more));
  }
};

}  // namespace egmla
