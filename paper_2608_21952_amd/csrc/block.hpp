// Device helpers of the operators around the SSD layer (conv, selective scan, gated norm, linear) and
// their launch declarations.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace ssdi8 {

typedef __bf16 bf16;

// kVec consecutive elements move as one access (two for fp32): 16 bytes of a 16-bit type.  The
// address need only be aligned to the element: rows cut out of wider ones start anywhere, and the
// memory path takes unaligned vectors.
constexpr int kVec = 8;

template <typename T> struct RawVec {
  T v[kVec];
};

// The first n of kVec elements at p as fp32, the others 0 and not read.
template <typename T> __device__ __forceinline__ void load_vec(const T* p, int n, float (&out)[kVec]) {
  if (n >= kVec) {
    RawVec<T> r;
    __builtin_memcpy(&r, p, sizeof(r));
#pragma unroll
    for (int i = 0; i < kVec; ++i) out[i] = (float)r.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) out[i] = i < n ? (float)p[i] : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store_vec(T* p, int n, const float (&in)[kVec]) {
  if (n >= kVec) {
    RawVec<T> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.v[i] = (T)in[i];
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < n) p[i] = (T)in[i];
  }
}

// exp in the hardware's base 2: one instruction of 1 ulp; log2(e) and the product with it are rounded, so that
// the result is within (2 |v| + 2) 2^-24 of its size.  Results below the normal range are 0.
constexpr float kLog2eF = 1.44269504088896341f;
__device__ __forceinline__ float fast_exp(float v) {
  return __builtin_amdgcn_exp2f(v * kLog2eF);
}
// v / (1 + exp(-v)).  exp overflows to inf for v < -88, whose reciprocal is 0: the result is -0, the
// limit; -inf gives -inf * 0 = NaN in the plain formula and here.
__device__ __forceinline__ float silu(float v) {
  return v * __builtin_amdgcn_rcpf(1.0f + fast_exp(-v));
}
// log(1 + exp(v)) in fp32 (v itself above 17: what is added there is below half an ulp).  With z = exp(-|v|)
// and u = fl(1 + z), log(u) + (z - (u - 1)) takes back the rounding of u: the exact term is
// (z - (u - 1)) / u, and what the missing division leaves is z (z - (u - 1)), below an ulp of the result.
__device__ __forceinline__ float softplus_fast(float v) {
  const float z = fast_exp(-__builtin_fabsf(v));
  const float u = 1.0f + z;
  const float l1p = __builtin_fmaf(0.693147180559945309f, __builtin_amdgcn_logf(u), z - (u - 1.0f));
  return __builtin_fmaxf(v, 0.0f) + l1p;   // a NaN stays one through z
}

// Sums over kLanes neighbouring lanes (a power of two) of kCount values, in every one of the lanes.
template <int kCtrl> __device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl,
                                                                   0xf, 0xf, true));
}
template <int kLanes, int kCount> __device__ __forceinline__ void lane_sums(float (&v)[kCount]) {
  auto each = [&](auto step) {
#pragma unroll
    for (int j = 0; j < kCount; ++j) v[j] = step(v[j]);
  };
  if constexpr (kLanes >= 2) each([](float x) { return dpp_add<0xB1>(x); });    // quad: 1 0 3 2
  if constexpr (kLanes >= 4) each([](float x) { return dpp_add<0x4E>(x); });    // quad: 2 3 0 1
  if constexpr (kLanes >= 8) each([](float x) { return dpp_add<0x141>(x); });   // half-row mirror
  if constexpr (kLanes >= 16) each([](float x) { return dpp_add<0x140>(x); });  // row mirror
  if constexpr (kLanes >= 32) each([](float x) { return x + __shfl_xor(x, 16); });
  if constexpr (kLanes >= 64) each([](float x) { return x + __shfl_xor(x, 32); });
}
template <int kLanes> __device__ __forceinline__ float lane_sum(float v) {
  float one[1] = {v};
  lane_sums<kLanes, 1>(one);
  return one[0];
}

// ---------------------------------------------------------------------------- launches
// A launch has fewer than 2^32 threads: more workgroups are given to several, f(first, count) each of them.
template <typename F> hipError_t in_parts(int64_t workgroups, int threads, F f) {
  const int64_t most = ((int64_t)1 << 31) / threads;
  for (int64_t first = 0; first < workgroups; first += most) {
    f(first, dim3((unsigned)(workgroups - first < most ? workgroups - first : most)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Element offsets between batch elements and tokens of a [b, l, d] tensor whose d is dense.
struct Rows {
  int64_t batch = 0, token = 0;
};

// Up to three dense outputs that share the columns of a row: [0, end0), [end0, end1), [end1, D).
struct ConvOut {
  void* y[3];
  int end[3];
  int vec_end[3];   // the same in vectors of kVec columns, each output's last one begun anew (set by launch)
};
hipError_t launch_conv(int dtype, int width, int64_t batch, int64_t seqlen, int64_t channels,
                       const void* x, Rows xr, const float* weight, const float* bias, int silu,
                       const void* init, const int* lengths, const ConvOut& out, void* final_state,
                       hipStream_t st);
hipError_t launch_conv_step(int dtype, int width, int64_t batch, int64_t channels, const void* x,
                            int64_t x_row, const float* weight, const float* bias, int silu,
                            void* state, const ConvOut& out, hipStream_t st);

hipError_t launch_gated_norm(int dtype, int64_t rows, int64_t channels, int64_t groups, const void* x,
                             int64_t x_row, const void* z, int64_t z_row, const void* residual,
                             const float* weight, float eps, int norm_before_gate, void* y,
                             void* residual_out, hipStream_t st);

struct SelScan {
  int dtype = 0, dt_dtype = 0, tied = 0, dt_softplus = 0;
  int64_t batch = 0, seqlen = 0, nheads = 0, headdim = 0, ngroups = 0, dstate = 0;
  const void *u = nullptr, *dt = nullptr, *B = nullptr, *C = nullptr, *z = nullptr;
  Rows ur, dtr, Br, Cr, zr;
  const float *A = nullptr, *D = nullptr, *dt_bias = nullptr, *init = nullptr;
  const int* lengths = nullptr;
  void* y = nullptr;
  float* final_state = nullptr;
  float* workspace = nullptr;
};
// Spans that a scan of these sizes is cut into, and the workspace of one (floats).
int sel_scan_spans(int64_t batch, int64_t seqlen, int64_t channels, int64_t groups, int64_t dstate);
int64_t sel_scan_workspace(int64_t batch, int64_t seqlen, int64_t channels, int64_t groups,
                           int64_t dstate);
hipError_t launch_sel_scan(const SelScan& a, hipStream_t st);
hipError_t launch_sel_scan_step(const SelScan& a, float* state, hipStream_t st);

struct LinearArgs {
  int dtype = 0, act = 0, out_dtype = 0;
  int64_t m = 0, n = 0, k = 0;
  const void *x = nullptr, *w = nullptr;
  int64_t x_row = 0, w_row = 0;
  const float *x_scale = nullptr, *w_scale = nullptr, *bias = nullptr;
  const void* residual = nullptr;
  int64_t residual_row = 0;
  void* y = nullptr;
  int64_t y_row = 0;
};
hipError_t launch_linear(const LinearArgs& a, hipStream_t st);

}  // namespace ssdi8
