// Codes in few bits: int8 with a step per row, and blocks of 32 values that share a power of two (8-bit e4m3 and
// 4-bit e2m1 elements, the scale an exponent byte).  Device helpers of norm_quantize.hip, quantize_mx.hip and
// linear_mx.hip, and their launch declarations.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "ssdi8.h"

namespace ssdi8 {

constexpr int kMxBlock = 32;

__host__ __device__ __forceinline__ int64_t mx_blocks(int64_t k) { return (k + kMxBlock - 1) / kMxBlock; }

// Magnitudes are compared as integers: they order as the values do, an infinity above them and a NaN above that.
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// The largest of 64 lanes, and of 4 neighbours, in every one of them.
template <int kCtrl> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xf, 0xf, true);
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t quad_max(uint32_t v) { return dpp_max<0x4E>(dpp_max<0xB1>(v)); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = dpp_max<0x140>(dpp_max<0x141>(quad_max(v)));
  for (int d = 16; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
    v = v > o ? v : o;
  }
  return v;
}

// The scale of a block whose largest magnitude is `big`: floor(log2(big)) less the exponent of the format's largest
// element (8 for e4m3, 2 for e2m1), as the byte e + 127, at least 0; 255 (NaN) for an infinity or a NaN.
template <int kFormat> __device__ __forceinline__ uint32_t mx_scale(uint32_t big) {
  const int e = (int)(big >> 23);
  constexpr int kMost = kFormat == SSDI8_FMT_MXFP8 ? 8 : 2;
  return e == 255 ? 255u : (uint32_t)(e > kMost ? e - kMost : 0);
}
// 2^-e for that byte; 0 for the NaN, whose block has codes of 0.
__device__ __forceinline__ float mx_inverse(uint32_t byte) {
  return byte == 255u ? 0.0f : __builtin_bit_cast(float, (254u - byte) << 23);
}
// Eight values times `inv`, rounded to the nearest element (ties to even), above the largest one to that.  A NaN
// scale gives 0 times a value or 0 times an infinity; the latter is made 0 here.
__device__ __forceinline__ float mx_clean(float v, float inv) {
  return inv == 0.0f ? 0.0f : v * inv;
}
__device__ __forceinline__ uint2 mx_e4m3(const float (&v)[kVec], float inv) {
  float c[kVec];
#pragma unroll
  for (int e = 0; e < kVec; ++e) c[e] = __builtin_amdgcn_fmed3f(mx_clean(v[e], inv), -448.0f, 448.0f);
  uint2 r;
  r.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
  r.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], (int)r.x, true);
  r.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[4], c[5], 0, false);
  r.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[6], c[7], (int)r.y, true);
  return r;
}
__device__ __forceinline__ uint32_t mx_e2m1(const float (&v)[kVec], float inv) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, mx_clean(v[0], inv), mx_clean(v[1], inv), 1.0f, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, mx_clean(v[2], inv), mx_clean(v[3], inv), 1.0f, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, mx_clean(v[4], inv), mx_clean(v[5], inv), 1.0f, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, mx_clean(v[6], inv), mx_clean(v[7], inv), 1.0f, 3);
  return r;
}

// Eight values of a block's quarter (the block is that of four neighbouring lanes) as codes at byte o of a row of
// codes, and the block's scale, written by its first lane.
template <int kFormat>
__device__ __forceinline__ void mx_put(const float (&v)[kVec], uint8_t* codes, uint8_t* scale, bool write) {
  uint32_t big = 0;
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    const uint32_t m = magnitude(v[e]);
    big = big > m ? big : m;
  }
  const uint32_t byte = mx_scale<kFormat>(quad_max(big));
  const float inv = mx_inverse(byte);
  if (!write) return;
  if constexpr (kFormat == SSDI8_FMT_MXFP8) {
    const uint2 c = mx_e4m3(v, inv);
    __builtin_memcpy(codes, &c, 8);
  } else {
    const uint32_t c = mx_e2m1(v, inv);
    __builtin_memcpy(codes, &c, 4);
  }
  if ((threadIdx.x & 3) == 0) *scale = (uint8_t)byte;
}

// ---------------------------------------------------------------------------- launches
struct NormQuant {
  int dtype = 0, format = 0, before = 0;
  int64_t rows = 0, channels = 0, groups = 0;
  const void *x = nullptr, *z = nullptr, *residual = nullptr;
  int64_t x_row = 0, z_row = 0;
  const float* weight = nullptr;
  float eps = 0;
  void *codes = nullptr, *scales = nullptr, *y = nullptr, *residual_out = nullptr;
};
hipError_t launch_norm_quantize(const NormQuant& a, hipStream_t st);

hipError_t launch_quantize_mx(int dtype, int format, int64_t rows, int64_t k, const void* x, int64_t x_row,
                              void* codes, void* scales, hipStream_t st);

struct LinearMx {
  int format = 0, act = 0, out_dtype = 0;   // format of x; weights are e2m1
  int64_t m = 0, n = 0, blocks = 0;         // blocks of 32 along k
  const uint8_t *x = nullptr, *xs = nullptr, *w = nullptr, *ws = nullptr;
  const float* bias = nullptr;
  const void* residual = nullptr;
  int64_t residual_row = 0;
  void* y = nullptr;
  int64_t y_row = 0;
};
hipError_t launch_linear_mx(const LinearMx& a, hipStream_t st);

}  // namespace ssdi8
