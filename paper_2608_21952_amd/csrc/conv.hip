// Short causal convolution of every channel with its own W weights, bias and SiLU, over prompts and
// for single tokens:
//   y[b, t, d] = act(bias[d] + sum_{j < W} w[d, j] x[b, t - (W-1) + j, d])
// where x before the first token comes from the state [b, W-1, d] (its last W-1 inputs, oldest first).
//
// What bounds it: the bytes of x and y; a weight is read once per thread.  A thread holds kVec
// channels, its weights and the last W-1 rows in registers and walks kTokens tokens, so a row is read
// once except for the W-1 rows in front of each walk (from the L2 cache).  64 lanes lie along the
// channels: 1 KB of a row per access.
#include <type_traits>

#include "block.hpp"

namespace ssdi8 {

namespace {

constexpr int kTokens = 16;   // of one thread's walk
constexpr int kWaves = 4;     // walks of a workgroup, one behind the other

// One vector of columns [c, c + kVec) of row `row` into the outputs that hold them.
template <typename T>
__device__ __forceinline__ void store_split(const ConvOut& o, int64_t row, int c, int D,
                                            const float (&v)[kVec]) {
  int begin = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int end = o.end[i];
    if (c >= begin && c < end) {
      const int n = end - c < kVec ? end - c : kVec;
      T* dst = static_cast<T*>(o.y[i]) + row * (end - begin) + (c - begin);
      if (n == kVec) {
        store_vec<T>(dst, kVec, v);
      } else {
        for (int e = 0; e < kVec; ++e) {   // the columns that run past this output
          const int col = c + e;
          if (col >= D) break;
          const int k = col < o.end[0] ? 0 : (col < o.end[1] ? 1 : 2);
          const int lo = k == 0 ? 0 : o.end[k - 1];
          static_cast<T*>(o.y[k])[row * (o.end[k] - lo) + (col - lo)] = (T)v[e];
        }
      }
    }
    begin = end;
  }
}

template <int W>
__device__ __forceinline__ void load_weights(const float* w, const float* bias, int c, int n,
                                             float (&wv)[W][kVec], float (&bv)[kVec]) {
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    bv[e] = bias && e < n ? bias[c + e] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) wv[j][e] = e < n ? w[(int64_t)(c + e) * W + j] : 0.0f;
  }
}

template <typename T, int W, bool kSilu>
__global__ __launch_bounds__(64 * kWaves) void conv_kernel(
    const T* __restrict__ x, Rows xr, const float* __restrict__ w, const float* __restrict__ bias,
    const T* init, const int* __restrict__ lengths, ConvOut out, T* final_state, int64_t L, int D,
    int nctile, int64_t nttile) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t bid = blockIdx.x;
  const int ct = (int)(bid % nctile);
  const int64_t tt = (bid / nctile) % nttile;
  const int64_t b = bid / nctile / nttile;
  const int c = (ct * 64 + lane) * kVec;
  if (c >= D) return;
  const int n = D - c < kVec ? D - c : kVec;
  const int64_t t0 = (tt * kWaves + wave) * kTokens;
  int64_t len = L;
  if (lengths) len = lengths[b] < 0 ? 0 : (lengths[b] < L ? lengths[b] : L);
  const T* xb = x + b * xr.batch + c;
  const bool first = t0 == 0;
  if (t0 >= L && !first) return;

  float wv[W][kVec], bv[kVec], win[W][kVec];
  load_weights<W>(w, bias, c, n, wv, bv);
  // rows t0 - (W-1) .. t0 - 1; those before the sequence from the initial state
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t t = t0 - (W - 1) + j;
    if (t >= 0) {
      if (t < len) {
        load_vec<T>(xb + t * xr.token, n, win[j]);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) win[j][e] = 0.0f;
      }
    } else if (init) {
      load_vec<T>(init + (b * (W - 1) + (W - 1 + t)) * D + c, n, win[j]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) win[j][e] = 0.0f;
    }
  }
  // the walk at token 0 also writes the final state: the only reader of the initial state, so that
  // both may be the same memory
  if (first && final_state) {
    float last[W - 1][kVec];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int64_t t = len - (W - 1) + j;
      if (t >= 0) {
        load_vec<T>(xb + t * xr.token, n, last[j]);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) last[j][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < W - 1; ++i)   // t = i - (W - 1): row i of the window
          if (t == i - (W - 1))
#pragma unroll
            for (int e = 0; e < kVec; ++e) last[j][e] = win[i][e];
      }
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
      store_vec<T>(final_state + (b * (W - 1) + j) * D + c, n, last[j]);
  }
#pragma unroll 4
  for (int i = 0; i < kTokens; ++i) {
    const int64_t t = t0 + i;
    if (t >= L) break;
    float y[kVec];
    if (t < len) {
      load_vec<T>(xb + t * xr.token, n, win[W - 1]);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float v = bv[e];
#pragma unroll
        for (int j = 0; j < W; ++j) v = __builtin_fmaf(wv[j][e], win[j][e], v);
        y[e] = kSilu ? silu(v) : v;
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) win[j][e] = win[j + 1][e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) y[e] = 0.0f;
    }
    store_split<T>(out, b * L + t, c, D, y);
  }
}

template <typename T, int W, bool kSilu>
__global__ __launch_bounds__(64) void conv_step_kernel(const T* __restrict__ x, int64_t x_row,
                                                       const float* __restrict__ w,
                                                       const float* __restrict__ bias, T* state,
                                                       ConvOut out, int D, int nctile) {
  const int64_t b = blockIdx.x / nctile;
  const int c = ((int)(blockIdx.x % nctile) * 64 + (int)threadIdx.x) * kVec;
  if (c >= D) return;
  const int n = D - c < kVec ? D - c : kVec;
  float wv[W][kVec], bv[kVec], win[W][kVec], y[kVec];
  T* sb = state + b * (W - 1) * D + c;
  load_vec<T>(x + b * x_row + c, n, win[W - 1]);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) load_vec<T>(sb + (int64_t)j * D, n, win[j]);
  load_weights<W>(w, bias, c, n, wv, bv);
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    float v = bv[e];
#pragma unroll
    for (int j = 0; j < W; ++j) v = __builtin_fmaf(wv[j][e], win[j][e], v);
    y[e] = kSilu ? silu(v) : v;
  }
#pragma unroll
  for (int j = 0; j < W - 1; ++j) store_vec<T>(sb + (int64_t)j * D, n, win[j + 1]);
  store_split<T>(out, b, c, D, y);
}

template <typename F> hipError_t for_type(int dtype, int width, int silu, F&& f) {
  auto by_silu = [&](auto t, auto w) {
    return silu ? f(t, w, std::true_type()) : f(t, w, std::false_type());
  };
  auto by_width = [&](auto t) {
    switch (width) {
      case 2: return by_silu(t, std::integral_constant<int, 2>());
      case 3: return by_silu(t, std::integral_constant<int, 3>());
      default: return by_silu(t, std::integral_constant<int, 4>());
    }
  };
  switch (dtype) {
    case 0: return by_width((float)0);
    case 1: return by_width((_Float16)0);
    default: return by_width((bf16)0);
  }
}

}  // namespace

hipError_t launch_conv(int dtype, int width, int64_t batch, int64_t seqlen, int64_t channels,
                       const void* x, Rows xr, const float* weight, const float* bias, int silu,
                       const void* init, const int* lengths, const ConvOut& out, void* final_state,
                       hipStream_t st) {
  const int nctile = (int)((channels + 64 * kVec - 1) / (64 * kVec));
  int64_t nttile = (seqlen + kTokens * kWaves - 1) / (kTokens * kWaves);
  if (nttile == 0) nttile = 1;   // no tokens: the states alone
  const int64_t grid = nctile * nttile * batch;
  return for_type(dtype, width, silu, [&](auto t, auto w, auto s) {
    using T = decltype(t);
    conv_kernel<T, decltype(w)::value, decltype(s)::value>
        <<<dim3((unsigned)grid), 64 * kWaves, 0, st>>>(
            static_cast<const T*>(x), xr, weight, bias, static_cast<const T*>(init), lengths, out,
            static_cast<T*>(final_state), seqlen, (int)channels, nctile, nttile);
    return hipGetLastError();
  });
}

hipError_t launch_conv_step(int dtype, int width, int64_t batch, int64_t channels, const void* x,
                            int64_t x_row, const float* weight, const float* bias, int silu,
                            void* state, const ConvOut& out, hipStream_t st) {
  const int nctile = (int)((channels + 64 * kVec - 1) / (64 * kVec));
  return for_type(dtype, width, silu, [&](auto t, auto w, auto s) {
    using T = decltype(t);
    conv_step_kernel<T, decltype(w)::value, decltype(s)::value>
        <<<dim3((unsigned)(nctile * batch)), 64, 0, st>>>(static_cast<const T*>(x), x_row, weight,
                                                          bias, static_cast<T*>(state), out,
                                                          (int)channels, nctile);
    return hipGetLastError();
  });
}

}  // namespace ssdi8
