// RMS norm over groups of channels with an optional gate and an optional residual in front:
//   s = x + residual (written when a residual is given),  g = z / (1 + exp(-z)) (1 without z)
//   gate first:  v = s g,  y = v rsqrt(mean_group(v^2) + eps) w
//   norm first:  y = s rsqrt(mean_group(s^2) + eps) w g
// Sums in fp32; the norm is of the unrounded s, which is rounded only where it is stored.
//
// What bounds it: the bytes of x, z, residual and y, each read or written once: a group's values
// stay in registers between the sum and the scaling, up to kMost vectors per thread.  A wave takes a
// group of up to 2048 channels, so that no barrier stands between the loads and the stores; wider
// groups take 256 or 1024 threads.  A thread reads what it writes and nothing else: y may be x, and
// the sum may be written over the residual.
#include <type_traits>

#include "block.hpp"

namespace ssdi8 {

namespace {

constexpr int kMost = 4;

struct NormArgs {
  const void *x, *z, *residual;
  const float* w;
  void *y, *residual_out;
  int64_t rows, x_row, z_row;
  int D, groups, width;   // width = D / groups
  float eps, inv;
};

// The value whose square is summed, and the gate for afterwards, of one vector.
template <typename T, bool kZ, bool kR, bool kBefore>
__device__ __forceinline__ void norm_load(const NormArgs& a, int64_t row, int c, int n,
                                          float (&v)[kVec], float (&g)[kVec]) {
  float r[kVec];
  load_vec<T>(static_cast<const T*>(a.x) + row * a.x_row + c, n, v);
  if constexpr (kR) load_vec<T>(static_cast<const T*>(a.residual) + row * a.D + c, n, r);
  if constexpr (kZ) load_vec<T>(static_cast<const T*>(a.z) + row * a.z_row + c, n, g);
  if constexpr (kR) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] += r[e];
    store_vec<T>(static_cast<T*>(a.residual_out) + row * a.D + c, n, v);
  }
  if constexpr (kZ) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      g[e] = silu(g[e]);
      if constexpr (!kBefore) v[e] *= g[e];
    }
  }
}

template <typename T, bool kZ, bool kR, bool kBefore>
__device__ __forceinline__ void norm_store(const NormArgs& a, int64_t row, int c, int n, float scale,
                                           const float (&v)[kVec], const float (&g)[kVec]) {
  float w[kVec], y[kVec];
  load_vec<float>(a.w + c, n, w);
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    y[e] = v[e] * scale * w[e];
    if constexpr (kZ && kBefore) y[e] *= g[e];
  }
  store_vec<T>(static_cast<T*>(a.y) + row * a.D + c, n, y);
}

// kThreads threads take a group: 64 (four groups per workgroup), 256 or 1024.
template <typename T, bool kZ, bool kR, bool kBefore, int kThreads>
__global__ __launch_bounds__(kThreads < 256 ? 256 : kThreads) void norm_kernel(NormArgs a) {
  constexpr int kItems = kThreads < 256 ? 256 / kThreads : 1;
  __shared__ float part[kThreads / 64];
  const int t = threadIdx.x % kThreads;
  const int64_t item = (int64_t)blockIdx.x * kItems + threadIdx.x / kThreads;
  if (item >= a.rows * a.groups) return;   // whole waves, and none where a barrier follows
  const int64_t row = item / a.groups;
  const int base = (int)(item % a.groups) * a.width;
  constexpr int kStep = kThreads * kVec;

  float v[kMost][kVec], g[kMost][kVec];
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int o = i * kStep + t * kVec;
    if (o < a.width)
      norm_load<T, kZ, kR, kBefore>(a, row, base + o, a.width - o, v[i], g[i]);
  }
#pragma unroll
  for (int i = 0; i < kMost; ++i)
    if (i * kStep + t * kVec < a.width)
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum = __builtin_fmaf(v[i][e], v[i][e], sum);
  sum = lane_sum<64>(sum);
  if constexpr (kThreads > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) sum += part[i];
  }
  const float scale = 1.0f / __builtin_sqrtf(sum * a.inv + a.eps);
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int o = i * kStep + t * kVec;
    if (o < a.width)
      norm_store<T, kZ, kR, kBefore>(a, row, base + o, a.width - o, scale, v[i], g[i]);
  }
}

template <typename T> hipError_t run(const NormArgs& a, int before, hipStream_t st) {
  const int64_t items = a.rows * a.groups;
  auto go = [&](auto z, auto r, auto b) {
    constexpr bool kZ = decltype(z)::value, kR = decltype(r)::value, kB = decltype(b)::value;
    if (a.width <= kMost * 64 * kVec)
      norm_kernel<T, kZ, kR, kB, 64><<<dim3((unsigned)((items + 3) / 4)), 256, 0, st>>>(a);
    else if (a.width <= kMost * 256 * kVec)
      norm_kernel<T, kZ, kR, kB, 256><<<dim3((unsigned)items), 256, 0, st>>>(a);
    else
      norm_kernel<T, kZ, kR, kB, 1024><<<dim3((unsigned)items), 1024, 0, st>>>(a);
    return hipGetLastError();
  };
  auto by_r = [&](auto z, auto b) {
    return a.residual ? go(z, std::true_type(), b) : go(z, std::false_type(), b);
  };
  if (!a.z) return by_r(std::false_type(), std::false_type());
  return before ? by_r(std::true_type(), std::true_type())
                : by_r(std::true_type(), std::false_type());
}

}  // namespace

hipError_t launch_gated_norm(int dtype, int64_t rows, int64_t channels, int64_t groups, const void* x,
                             int64_t x_row, const void* z, int64_t z_row, const void* residual,
                             const float* weight, float eps, int norm_before_gate, void* y,
                             void* residual_out, hipStream_t st) {
  NormArgs a;
  a.x = x;
  a.z = z;
  a.residual = residual;
  a.w = weight;
  a.y = y;
  a.residual_out = residual_out;
  a.rows = rows;
  a.x_row = x_row;
  a.z_row = z_row;
  a.D = (int)channels;
  a.groups = (int)groups;
  a.width = (int)(channels / groups);
  a.eps = eps;
  a.inv = 1.0f / (float)a.width;
  switch (dtype) {
    case 0: return run<float>(a, norm_before_gate, st);
    case 1: return run<_Float16>(a, norm_before_gate, st);
    default: return run<bf16>(a, norm_before_gate, st);
  }
}

}  // namespace ssdi8
