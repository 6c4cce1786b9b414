// RMS norm over groups of channels with an optional gate and an optional residual in front:
//   s = x + residual (written when a residual is given),  g = z / (1 + exp(-z)) (1 without z)
//   gate first:  v = s g,  y = v rsqrt(mean_group(v^2) + eps) w
//   norm first:  y = s rsqrt(mean_group(s^2) + eps) w g
// Sums in fp32; the norm is of the unrounded s, which is rounded only where it is stored.
//
// What bounds it: the bytes of x, z, residual and y, each read or written once: a group's values
// stay in registers between the sum and the scaling.  A wave takes a group of up to 1024 channels, so
// that no barrier stands between the loads and the stores; wider groups take a workgroup of as many waves
// as they need.  What a thread writes no other one reads for its results: y may
// be x, and the sum may be written over the residual.  16384 x 5120 fp16 with gate: 105 us a pass among
// others, 4.8 TB/s (110 in a kernel trace, which counts each one's start and end; an addition of the same rows 91).
#include <type_traits>

#include "block.hpp"

namespace ssdi8 {

namespace {

struct NormArgs {
  const void *x, *z, *residual;
  const float* w;
  void *y, *residual_out;
  int64_t rows, x_row, z_row;
  int D, groups, width;   // width = D / groups
  float eps, inv;
};

// kMost vectors of every thread of a group.  kWave: a wave takes a group (blockDim = 256 for four), else the
// workgroup does.  A group's last vector is moved back to end with it (its first `shift` values belong to
// the vector before: not summed, not stored); kPart: groups of fewer than kVec channels.
//
// The threads walk `walk` rows of the same group, with its weights in registers (read for every row they
// were, at twice the width of 16-bit activations, as many bytes from the cache again as the rest from
// memory), and the next row's values on their way during a row's arithmetic.
template <typename T, bool kZ, bool kR, bool kBefore, bool kWave, int kMost, bool kPart, int kThreads>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a, int walk) {
  __shared__ float part[2][16];
  const int t = kWave ? threadIdx.x & 63 : threadIdx.x;
  const int threads = kWave ? 64 : blockDim.x;
  const int64_t item = kWave ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int64_t row0 = item / a.groups * walk;
  if (row0 >= a.rows) return;   // whole waves, and none where a barrier follows
  const int64_t row1 = row0 + walk < a.rows ? row0 + walk : a.rows;
  const int base = (int)(item % a.groups) * a.width;

  int at[kMost], shift[kMost];   // of a vector's first value; kVec: none of the vector's values is the group's
  float w[kMost][kVec];
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    int o = (i * threads + t) * kVec;
    shift[i] = 0;
    if (o >= a.width) {
      shift[i] = kVec;
      o = 0;
    } else if (!kPart && o + kVec > a.width) {
      shift[i] = o + kVec - a.width;
      o = a.width - kVec;
    }
    at[i] = base + o;
    load_vec<float>(a.w + at[i], kPart ? a.width : kVec, w[i]);
  }
  const int n = kPart ? a.width : kVec;
  RawVec<T> x[kMost], z[kMost], r[kMost];
  auto request = [&](RawVec<T>& v, const void* p, int64_t off) {
    if (kPart) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v.v[e] = e < n ? static_cast<const T*>(p)[off + e] : (T)0.0f;
    } else {
      __builtin_memcpy(&v, static_cast<const T*>(p) + off, sizeof(v));
    }
  };
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (shift[i] == kVec) continue;
      request(x[i], a.x, row * a.x_row + at[i]);
      if constexpr (kZ) request(z[i], a.z, row * a.z_row + at[i]);
      if constexpr (kR) request(r[i], a.residual, row * a.D + at[i]);
    }
  };
  auto store = [&](void* p, int64_t row, int i, const RawVec<T>& v) {
    T* q = static_cast<T*>(p) + row * a.D + at[i];
    if (!kPart && shift[i] == 0) {
      __builtin_memcpy(q, &v, sizeof(v));
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (e >= shift[i] && e < n) q[e] = v.v[e];
    }
  };
  // A row's results are stored behind the next row's loads: loads and stores count down in one order, and
  // the wait for the loads, had it the stores before it, would be for those too.
  RawVec<T> y[kMost], s[kMost];
  auto put = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (shift[i] == kVec) continue;
      if constexpr (kR) store(a.residual_out, row, i, s[i]);
      store(a.y, row, i, y[i]);
    }
  };
  fetch(row0);
  for (int64_t row = row0; row < row1; ++row) {
    float v[kMost][kVec], g[kMost][kVec];
    float sum = 0.0f;
    // every value of this row is here: said for all lanes, those without a vector too
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (shift[i] == kVec) continue;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        v[i][e] = (float)x[i].v[e];
        if constexpr (kR) v[i][e] += (float)r[i].v[e];
      }
      if constexpr (kZ) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) g[i][e] = silu((float)z[i].v[e]);
      }
    }
    if (row > row0) put(row - 1);
    if (row + 1 < row1) fetch(row + 1);
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (shift[i] == kVec) continue;
      if constexpr (kR) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) s[i].v[e] = (T)v[i][e];
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (kZ && !kBefore) v[i][e] *= g[i][e];
        const bool own = kPart ? e < n : e >= shift[i];
        sum = own ? __builtin_fmaf(v[i][e], v[i][e], sum) : sum;
      }
    }
    sum = lane_sum<64>(sum);
    if constexpr (!kWave) {
      float* p = part[(row - row0) & 1];   // a wave may be a row behind another, not two
      if ((t & 63) == 0) p[t >> 6] = sum;
      __syncthreads();
      sum = 0.0f;
      for (int i = 0; i < threads / 64; ++i) sum += p[i];
    }
    const float scale = 1.0f / __builtin_sqrtf(sum * a.inv + a.eps);
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (shift[i] == kVec) continue;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float u = v[i][e] * scale * w[i][e];
        if constexpr (kZ && kBefore) u *= g[i][e];
        y[i].v[e] = (T)u;
      }
    }
  }
  put(row1 - 1);
}

// Groups of more than 8192 channels: 1024 threads, a row each, up to four vectors per thread, the weights read
// when they are used (in registers beside the rest they spilled).
template <typename T, bool kZ, bool kR, bool kBefore>
__global__ __launch_bounds__(1024) void norm_wide_kernel(NormArgs a) {
  constexpr int kMost = 4, kStep = 1024 * kVec;
  __shared__ float part[16];
  const int64_t row = blockIdx.x / a.groups;
  const int base = (int)(blockIdx.x % a.groups) * a.width, t = threadIdx.x;
  float v[kMost][kVec], g[kMost][kVec];
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int o = i * kStep + t * kVec, c = base + o, n = a.width - o;
    if (n <= 0) continue;
    load_vec<T>(static_cast<const T*>(a.x) + row * a.x_row + c, n, v[i]);
    if constexpr (kZ) load_vec<T>(static_cast<const T*>(a.z) + row * a.z_row + c, n, g[i]);
    if constexpr (kR) {
      float r[kVec];
      load_vec<T>(static_cast<const T*>(a.residual) + row * a.D + c, n, r);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[i][e] += r[e];
      store_vec<T>(static_cast<T*>(a.residual_out) + row * a.D + c, n, v[i]);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {   // 0 behind the group's end
      if constexpr (kZ) g[i][e] = silu(g[i][e]);
      if constexpr (kZ && !kBefore) v[i][e] *= g[i][e];
      sum = __builtin_fmaf(v[i][e], v[i][e], sum);
    }
  }
  sum = lane_sum<64>(sum);
  if ((t & 63) == 0) part[t >> 6] = sum;
  __syncthreads();
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += part[i];
  const float scale = 1.0f / __builtin_sqrtf(sum * a.inv + a.eps);
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int o = i * kStep + t * kVec, c = base + o, n = a.width - o;
    if (n <= 0) continue;
    float w[kVec], y[kVec];
    load_vec<float>(a.w + c, n, w);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      y[e] = v[i][e] * scale * w[e];
      if constexpr (kZ && kBefore) y[e] *= g[i][e];
    }
    store_vec<T>(static_cast<T*>(a.y) + row * a.D + c, n, y);
  }
}

template <typename T> hipError_t run(const NormArgs& a, int before, hipStream_t st) {
  const int64_t items = a.rows * a.groups;
  auto go = [&](auto z, auto r, auto b) {
    constexpr bool kZ = decltype(z)::value, kR = decltype(r)::value, kB = decltype(b)::value;
    const int vecs = (a.width + kVec - 1) / kVec;
    auto launch = [&](auto wave, auto most, auto part, auto limit, int threads) {
      constexpr bool kWave = decltype(wave)::value;
      constexpr int kItems = kWave ? 4 : 1;
      // rows of a walk: as many as leave every CU eight workgroups, four at most (16384 x
      // 5120 with gate: 146 us at one, with the weights read for every row; 105 at four, 108 at eight)
      int walk = 1;
      while (walk < 4 && items / (2 * walk) >= 2048 * kItems) walk *= 2;
      const int64_t count = (a.rows + walk - 1) / walk * a.groups;
      norm_kernel<T, kZ, kR, kB, kWave, decltype(most)::value, decltype(part)::value,
                  decltype(limit)::value>
          <<<dim3((unsigned)((count + kItems - 1) / kItems)), threads, 0, st>>>(a, walk);
    };
    using std::integral_constant;
    using std::true_type;
    using std::false_type;
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    if (a.width < kVec) launch(true_type(), One(), true_type(), integral_constant<int, 256>(), 256);
    else if (vecs <= 64) launch(true_type(), One(), false_type(), integral_constant<int, 256>(), 256);
    else if (vecs <= 128) launch(true_type(), Two(), false_type(), integral_constant<int, 256>(), 256);
    else if (vecs <= 1024)
      launch(false_type(), Two(), false_type(), integral_constant<int, 512>(), (vecs + 127) / 128 * 64);
    else
      norm_wide_kernel<T, kZ, kR, kB><<<dim3((unsigned)items), 1024, 0, st>>>(a);
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
