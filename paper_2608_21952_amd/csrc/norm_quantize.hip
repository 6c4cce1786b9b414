// RMS norm of rows with an optional residual in front, an optional gate and groups of channels (the formulas of
// norm.hip), its output in few bits:
//   int8           step = max |y| / 127 of the row (1 where all are 0), code = rne(y (1 / step))
//   e4m3, e2m1     blocks of 32 channels with a power of two each (mx.hpp)
// The codes are those of the unrounded y; y itself, rounded, is written too where it is wanted.  A row (int8) or a
// block with an infinity or a NaN has a scale of NaN and codes of 0.
//
// What bounds it: the bytes of x, z, residual and the codes, each read or written once: a row's values stay in
// registers from the sums to the codes.  A wave takes a row of up to 1024 channels, wider rows a workgroup; the
// threads walk rows with their weights in registers and the next row's values on their way.  A thread holds vectors
// of eight channels, so that a block of 32 is that of four neighbouring lanes.  With several groups the sums of
// vectors meet in LDS and a wave adds up each group's, in one order.  Rows of more than 8192 channels, and groups whose
// width is no multiple of eight, have their values in LDS instead of registers, a row at a time.
// 16384 x 5120 fp16 with gate to e4m3 97 us (4.3 TB/s), to int8 118, as the workgroup meets once more for a row; 16384 x 2560
// bf16 with residual and its sum 57 (5.2 TB/s), 58.  In LDS: 16384 x 5121 fp16 with gate 177, int8 235 (2.4 and 1.8 TB/s),
// 8192 x 10240 144, 187.
#include "mx.hpp"

namespace ssdi8 {

namespace {

struct Args {
  const void *x, *z, *residual;
  const float* w;
  uint8_t *codes, *scales;
  void *y, *residual_out;
  int64_t rows, x_row, z_row;
  int D, groups, width, format, before, blocks;   // width = D / groups, blocks of 32 in a row
  float eps, inv;
};

__device__ __forceinline__ void int8_codes(const float (&v)[kVec], float inv, uint8_t (&c)[kVec]) {
#pragma unroll
  for (int e = 0; e < kVec; ++e)
    c[e] = (uint8_t)(int8_t)(int)__builtin_amdgcn_fmed3f(__builtin_rintf(mx_clean(v[e], inv)), -127.0f, 127.0f);
}
// The codes of a vector of y, n values of it, at channel `at` of a row: int8 with the row's step.
__device__ __forceinline__ void put_int8(const Args& a, int64_t row, int at, int n, const float (&v)[kVec], float inv) {
  uint8_t c[kVec];
  int8_codes(v, inv, c);
  uint8_t* p = a.codes + row * a.D + at;
  if (n == kVec) {
    __builtin_memcpy(p, c, kVec);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) p[e] = c[e];
  }
}
// A row's int8 step from its largest magnitude, and its inverse: at least the smallest normal number, whose inverse
// there is; 1 for a row of zeros, NaN and 0 where a value is no number.
__device__ __forceinline__ float int8_step(uint32_t big, float& inv) {
  const bool fine = big < 0x7f800000u;
  const float step = !fine ? __builtin_nanf("")
                     : big ? __builtin_fmaxf(__builtin_bit_cast(float, big) / 127.0f, 1.17549435e-38f) : 1.0f;
  inv = fine ? 1.0f / step : 0.0f;
  return step;
}
// Blocks of a vector (mx_put), by the row's format.
__device__ __forceinline__ void put_blocks(const Args& a, int64_t row, int at, const float (&v)[kVec]) {
  const int row_vecs = a.blocks * (kMxBlock / kVec);
  const bool write = at < row_vecs * kVec;
  const int64_t o = row * row_vecs + at / kVec;
  if (a.format == SSDI8_FMT_MXFP8) mx_put<SSDI8_FMT_MXFP8>(v, a.codes + o * kVec, a.scales + o / 4, write);
  else mx_put<SSDI8_FMT_MXFP4>(v, a.codes + o * (kVec / 2), a.scales + o / 4, write);
}
__device__ __forceinline__ uint32_t biggest_of(const float (&v)[kVec], uint32_t big) {
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    const uint32_t m = magnitude(v[e]);
    big = big > m ? big : m;
  }
  return big;
}

// kGroups: several groups of a width that is a multiple of eight.  kMost vectors of every thread, all whole.
template <typename T, bool kWave, int kMost, int kThreads, bool kGroups, bool kZ, bool kR>
__global__ __launch_bounds__(kThreads) void norm_quantize_kernel(Args a, int walk, int64_t first) {
  extern __shared__ float terms_all[];
  __shared__ float part[2][16];
  __shared__ uint32_t biggest[2][16];
  const int t = kWave ? threadIdx.x & 63 : threadIdx.x;
  const int threads = kWave ? 64 : blockDim.x;
  const int64_t item = kWave ? (first + blockIdx.x) * 4 + (threadIdx.x >> 6) : first + blockIdx.x;
  const int64_t row0 = item * walk;
  if (row0 >= a.rows) return;   // whole waves, and none where a barrier follows
  const int64_t row1 = row0 + walk < a.rows ? row0 + walk : a.rows;
  float* terms = terms_all + (kWave ? (threadIdx.x >> 6) * (a.D / kVec) : 0);   // a sum of squares per vector
  auto meet = [&] {
    if (kWave) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    else __syncthreads();
  };

  int at[kMost];   // a vector's first channel
  float w[kMost][kVec];
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    at[i] = (i * threads + t) * kVec;
    if (at[i] < a.D) load_vec<float>(a.w + at[i], kVec, w[i]);
  }
  RawVec<T> x[kMost], z[kMost], r[kMost];
  auto request = [&](RawVec<T>& v, const void* p, int64_t off) { __builtin_memcpy(&v, static_cast<const T*>(p) + off, sizeof(v)); };
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (at[i] >= a.D) continue;
      request(x[i], a.x, row * a.x_row + at[i]);
      if constexpr (kZ) request(z[i], a.z, row * a.z_row + at[i]);
      if constexpr (kR) request(r[i], a.residual, row * a.D + at[i]);
    }
  };
  // A row's results are stored behind the next row's loads: loads and stores count down in one order, and the wait for
  // the loads, had it the stores before it, would be for those too.
  const int row_vecs = a.blocks * (kMxBlock / kVec);
  RawVec<T> sums[kMost];
  uint2 codes[kMost];
  uint32_t scales[kMost];
  float step = 0.0f;
  auto put = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (kR && at[i] < a.D) __builtin_memcpy(static_cast<T*>(a.residual_out) + row * a.D + at[i], &sums[i], sizeof(sums[i]));
      if (a.format == SSDI8_FMT_I8) {
        if (at[i] < a.D) __builtin_memcpy(a.codes + row * a.D + at[i], &codes[i], 8);
      } else if (at[i] < row_vecs * kVec) {
        const int64_t o = row * row_vecs + at[i] / kVec;
        if (a.format == SSDI8_FMT_MXFP8) __builtin_memcpy(a.codes + o * kVec, &codes[i], 8);
        else __builtin_memcpy(a.codes + o * (kVec / 2), &codes[i], 4);
        if ((t & 3) == 0) a.scales[o / 4] = (uint8_t)scales[i];
      }
    }
    if (a.format == SSDI8_FMT_I8 && t == 0) reinterpret_cast<float*>(a.scales)[row] = step;
  };
  fetch(row0);
  for (int64_t row = row0; row < row1; ++row) {
    const int turn = (int)(row - row0) & 1;   // a wave may be a row behind another, not two
    float v[kMost][kVec], g[kMost][kVec];
    float sum = 0.0f;
    // every value of this row is here: said for all lanes, those without a vector too
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (at[i] >= a.D) continue;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        v[i][e] = (float)x[i].v[e];
        if constexpr (kR) v[i][e] += (float)r[i].v[e];
        if constexpr (kZ) g[i][e] = silu((float)z[i].v[e]);
      }
    }
    if (row > row0) put(row - 1);
    if (row + 1 < row1) fetch(row + 1);
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (at[i] >= a.D) continue;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (kR) sums[i].v[e] = (T)v[i][e];
        if constexpr (kZ) v[i][e] = a.before ? v[i][e] : v[i][e] * g[i][e];
      }
    }
    if constexpr (!kGroups) {
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (at[i] >= a.D) continue;
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum = __builtin_fmaf(v[i][e], v[i][e], sum);
      }
      sum = lane_sum<64>(sum);
      if constexpr (!kWave) {
        if ((t & 63) == 0) part[turn][t >> 6] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int i = 0; i < threads / 64; ++i) sum += part[turn][i];
      }
      sum = 1.0f / __builtin_sqrtf(sum * a.inv + a.eps);
    } else {
      if (row > row0) meet();   // the last row's scales are read
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (at[i] >= a.D) continue;
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) s = __builtin_fmaf(v[i][e], v[i][e], s);
        terms[at[i] / kVec] = s;
      }
      meet();
      // a group's scale takes the place of its first term
      const int per = a.width / kVec;
      for (int q = kWave ? 0 : t >> 6; q < a.groups; q += kWave ? 1 : threads / 64) {
        float s = 0.0f;
        for (int c = t & 63; c < per; c += 64) s += terms[q * per + c];
        s = lane_sum<64>(s);
        if ((t & 63) == 0) terms[q * per] = 1.0f / __builtin_sqrtf(s * a.inv + a.eps);
      }
      meet();
    }
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const bool own = at[i] < a.D;
      const float scale = kGroups ? terms[own ? at[i] / a.width * (a.width / kVec) : 0] : sum;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float u = v[i][e] * scale * w[i][e];
        if constexpr (kZ) u = a.before ? u * g[i][e] : u;
        v[i][e] = own ? u : 0.0f;   // behind the row's end, up to a whole block: 0
      }
      big = biggest_of(v[i], big);
      if (a.y && own) store_vec<T>(static_cast<T*>(a.y) + row * a.D + at[i], kVec, v[i]);
    }
    if (a.format == SSDI8_FMT_I8) {
      big = wave_max(big);
      if constexpr (!kWave) {
        if ((t & 63) == 0) biggest[turn][t >> 6] = big;
        __syncthreads();
        big = 0;
        for (int i = 0; i < threads / 64; ++i) big = big > biggest[turn][i] ? big : biggest[turn][i];
      }
      float inv;
      step = int8_step(big, inv);
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        uint8_t c[kVec];
        int8_codes(v[i], inv, c);
        __builtin_memcpy(&codes[i], c, kVec);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const uint32_t block = quad_max(biggest_of(v[i], 0));
        if (a.format == SSDI8_FMT_MXFP8) {
          scales[i] = mx_scale<SSDI8_FMT_MXFP8>(block);
          codes[i] = mx_e4m3(v[i], mx_inverse(scales[i]));
        } else {
          scales[i] = mx_scale<SSDI8_FMT_MXFP4>(block);
          codes[i].x = mx_e2m1(v[i], mx_inverse(scales[i]));
        }
      }
    }
  }
  put(row1 - 1);
}

// A row's values in LDS, a workgroup for each row.
template <typename T> __global__ __launch_bounds__(1024) void norm_quantize_lds_kernel(Args a, int64_t first) {
  extern __shared__ float values[];
  __shared__ float part[16];
  __shared__ uint32_t biggest[16];
  const int t = threadIdx.x, threads = blockDim.x, waves = threads / 64;
  const int64_t row = first + blockIdx.x;
  const int ends = a.blocks * kMxBlock;   // whole blocks
  auto load = [&](const void* p, int64_t off, int n, float (&v)[kVec]) {
    load_vec<T>(static_cast<const T*>(p) + off, n, v);
  };
  auto of_row = [&](int o) { return a.D - o < kVec ? a.D - o : kVec; };
  float sum = 0.0f;
  for (int o = t * kVec; o < a.D; o += threads * kVec) {
    const int n = of_row(o);
    float v[kVec];
    load(a.x, row * a.x_row + o, n, v);
    if (a.residual) {
      float r[kVec];
      load(a.residual, row * a.D + o, n, r);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] += r[e];
      store_vec<T>(static_cast<T*>(a.residual_out) + row * a.D + o, n, v);
    }
    if (a.z && !a.before) {
      float z[kVec];
      load(a.z, row * a.z_row + o, n, z);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] *= silu(z[e]);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) {
        values[o + e] = v[e];
        sum = __builtin_fmaf(v[e], v[e], sum);
      }
  }
  float scale = 1.0f;
  if (a.groups == 1) {
    sum = lane_sum<64>(sum);
    if ((t & 63) == 0) part[t >> 6] = sum;
    __syncthreads();
    sum = 0.0f;
    for (int i = 0; i < waves; ++i) sum += part[i];
    scale = 1.0f / __builtin_sqrtf(sum * a.inv + a.eps);
  } else {
    __syncthreads();
    for (int q = t >> 6; q < a.groups; q += waves) {
      float* of = values + q * a.width;
      float s = 0.0f;
      for (int c = t & 63; c < a.width; c += 64) s = __builtin_fmaf(of[c], of[c], s);
      s = 1.0f / __builtin_sqrtf(lane_sum<64>(s) * a.inv + a.eps);
      for (int c = t & 63; c < a.width; c += 64) of[c] *= s;
    }
    __syncthreads();
  }
  uint32_t big = 0;
  // whole waves walk together: four neighbouring lanes have a block
  for (int base = 0; base < ends; base += threads * kVec) {
    const int o = base + t * kVec, n = of_row(o);
    float v[kVec] = {};
    if (n > 0) {
      float w[kVec], z[kVec];
      load_vec<float>(a.w + o, n, w);
      if (a.z && a.before) load(a.z, row * a.z_row + o, n, z);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (e < n) {
          v[e] = values[o + e] * scale * w[e];
          if (a.z && a.before) v[e] *= silu(z[e]);
        }
      if (a.y) store_vec<T>(static_cast<T*>(a.y) + row * a.D + o, n, v);
      if (a.format == SSDI8_FMT_I8) {   // read again by this thread alone
        big = biggest_of(v, big);
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (e < n) values[o + e] = v[e];
      }
    }
    if (a.format != SSDI8_FMT_I8) put_blocks(a, row, o, v);
  }
  if (a.format != SSDI8_FMT_I8) return;
  big = wave_max(big);
  if ((t & 63) == 0) biggest[t >> 6] = big;
  __syncthreads();
  big = 0;
  for (int i = 0; i < waves; ++i) big = big > biggest[i] ? big : biggest[i];
  float inv;
  const float step = int8_step(big, inv);
  for (int o = t * kVec; o < a.D; o += threads * kVec) {
    const int n = of_row(o);
    float v[kVec] = {};
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) v[e] = values[o + e];
    put_int8(a, row, o, n, v, inv);
  }
  if (t == 0) reinterpret_cast<float*>(a.scales)[row] = step;
}

template <typename T> hipError_t run(const Args& a, hipStream_t st) {
  // Threads for the row's whole blocks, too.
  const int vecs = a.blocks * (kMxBlock / kVec);
  if (vecs > 1024 || a.D % kVec != 0 || a.width % kVec != 0) {
    const int threads = vecs < 1024 ? (vecs + 63) / 64 * 64 : 1024;
    const size_t lds = sizeof(float) * a.D;
    if (lds > 64 * 1024) {   // more than a kernel may have unasked
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(norm_quantize_lds_kernel<T>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, 32768 * 4);
      if (e != hipSuccess) return e;
    }
    return in_parts(a.rows, threads, [&](int64_t first, dim3 grid) {
      norm_quantize_lds_kernel<T><<<grid, threads, lds, st>>>(a, first);
    });
  }
  auto launch = [&](auto wave, auto most, auto limit, auto groups, int threads) {
    constexpr bool kWave = decltype(wave)::value, kGroups = decltype(groups)::value;
    constexpr int kItems = kWave ? 4 : 1;
    // rows of a walk: as many as leave every CU eight workgroups, four at most (us at one, two, four, eight: 16384 x 5120
    // with gate 113, 101, 97, 98; 16384 x 2560 with residual 60, 54, 57, 63)
    int walk = 1;
    while (walk < 4 && a.rows / (2 * walk) >= 2048 * kItems) walk *= 2;
    const int64_t count = (a.rows + walk - 1) / walk;
    const size_t lds = kGroups ? sizeof(float) * kItems * (a.D / kVec) : 0;
    auto go = [&](auto z, auto r) {
      return in_parts((count + kItems - 1) / kItems, threads, [&](int64_t first, dim3 grid) {
        norm_quantize_kernel<T, kWave, decltype(most)::value, decltype(limit)::value, kGroups, decltype(z)::value,
                             decltype(r)::value><<<grid, threads, lds, st>>>(a, walk, first);
      });
    };
    if (a.residual) return a.z ? go(std::true_type(), std::true_type()) : go(std::false_type(), std::true_type());
    return a.z ? go(std::true_type(), std::false_type()) : go(std::false_type(), std::false_type());
  };
  using std::integral_constant;
  auto by_width = [&](auto groups) {
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    using W = integral_constant<int, 256>;
    if (vecs <= 64) return launch(std::true_type(), One(), W(), groups, 256);
    if (vecs <= 128) return launch(std::true_type(), Two(), W(), groups, 256);
    // A vector per thread: two of them left half as many waves (16384 x 5120 with gate 111 us, 97 with one).
    return launch(std::false_type(), One(), integral_constant<int, 1024>(), groups, (vecs + 63) / 64 * 64);
  };
  return a.groups == 1 ? by_width(std::false_type()) : by_width(std::true_type());
}

}  // namespace

hipError_t launch_norm_quantize(const NormQuant& q, hipStream_t st) {
  Args a;
  a.x = q.x;
  a.z = q.z;
  a.residual = q.residual;
  a.w = q.weight;
  a.codes = static_cast<uint8_t*>(q.codes);
  a.scales = static_cast<uint8_t*>(q.scales);
  a.y = q.y;
  a.residual_out = q.residual_out;
  a.rows = q.rows;
  a.x_row = q.x_row;
  a.z_row = q.z_row;
  a.D = (int)q.channels;
  a.groups = (int)q.groups;
  a.width = (int)(q.channels / q.groups);
  a.format = q.format;
  a.before = q.before;
  a.blocks = (int)mx_blocks(q.channels);
  a.eps = q.eps;
  a.inv = 1.0f / (float)a.width;
  switch (q.dtype) {
    case SSDI8_F32: return run<float>(a, st);
    case SSDI8_F16: return run<_Float16>(a, st);
    default: return run<bf16>(a, st);
  }
}

}  // namespace ssdi8
