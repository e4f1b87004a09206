// egmla_rows.cuh - rows of the latent cache spread over a warp's lanes: 16-byte units as
// pairs of fp32 values, and the sums of a few rows reduced together.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace egmla {

// 16 bytes of a row as pairs of fp32 values
template <typename T>
struct Unit;
template <>
struct Unit<__nv_bfloat16> {
  static constexpr int kPairs = 4;
  static __device__ __forceinline__ void widen(const uint4& w, float2 (&x)[4]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
  }
  // x = c (*) g, exact: bf16 factors, an fp32 product
  static __device__ __forceinline__ void mul(const uint4& c, const uint4& g, float2 (&x)[4]) {
    const uint32_t a[4] = {c.x, c.y, c.z, c.w}, b[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("{\n\t.reg .b16 al, ah, bl, bh;\n\t"
          "mov.b32 {al, ah}, %2;\n\tmov.b32 {bl, bh}, %3;\n\t"
          "fma.rn.f32.bf16 %0, al, bl, %4;\n\tfma.rn.f32.bf16 %1, ah, bh, %4;\n\t}"
          : "=f"(x[i].x), "=f"(x[i].y)
          : "r"(a[i]), "r"(b[i]), "f"(-0.f));
  }
};
template <>
struct Unit<float> {
  static constexpr int kPairs = 2;
  static __device__ __forceinline__ void widen(const uint4& w, float2 (&x)[2]) {
    x[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    x[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
  }
  static __device__ __forceinline__ void mul(const uint4& c, const uint4& g, float2 (&x)[2]) {
    float2 t[2];
    widen(c, x);
    widen(g, t);
    x[0] = __fmul2_rn(x[0], t[0]);
    x[1] = __fmul2_rn(x[1], t[1]);
  }
};

// v[r] summed over the warp's lanes, for every lane
__device__ __forceinline__ void warp_sums(float (&v)[2], int lane) {
  const bool h16 = lane & 16;
  float c = (h16 ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, h16 ? v[0] : v[1], 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
#pragma unroll
  for (int r = 0; r < 2; ++r) v[r] = __shfl_sync(0xffffffffu, c, 16 * r);
}
__device__ __forceinline__ void warp_sums(float (&v)[4], int lane) {
  const bool h16 = lane & 16, h8 = lane & 8;
  const float a = (h16 ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, h16 ? v[0] : v[2], 16);
  const float b = (h16 ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, h16 ? v[1] : v[3], 16);
  float c = (h8 ? b : a) + __shfl_xor_sync(0xffffffffu, h8 ? a : b, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = __shfl_sync(0xffffffffu, c, 16 * (r >> 1) + 8 * (r & 1));
}

}  // namespace egmla
