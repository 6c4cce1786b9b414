// Short causal convolution of every channel with its own W weights, bias and SiLU, over prompts and
// for single tokens:
//   y[b, t, d] = act(bias[d] + sum_{j < W} w[d, j] x[b, t - (W-1) + j, d])
// where x before the first token comes from the state [b, W-1, d] (its last W-1 inputs, oldest first).
//
// What bounds it: the bytes of x and y; a weight is read once per thread.  A thread holds kVec
// channels, its weights and the last W-1 rows in registers and walks kTokens tokens, so a row is read
// once except for the W-1 rows in front of each walk (from the L2 cache).  64 lanes lie along the
// channels: 1 KB of a row per access.  4 x 4096 x 5376 fp16, columns of rows twice as wide into three
// outputs: 83 us, 4.3 TB/s (78 on inputs that stay the same; a copy of the same rows 64).  A token of 8
// sequences: 4 us, a launch and one chain of loads.
#include <type_traits>

#include "block.hpp"
#include "common.hpp"

namespace ssdi8 {

namespace {

constexpr int kWaves = 4;     // walks of a workgroup, one behind the other

// A thread's channels: vector `vec` of the columns, which never lies in two outputs.  The last vector of an
// output is moved back to end with it, so that it is whole: the first `shift` of its channels are computed
// twice, to the same values.  An output of fewer than kVec columns has one vector of n.
template <typename T> struct Columns {
  int c, n, shift;
  T* y;           // its first column in the output
  int64_t cols;   // of the output
  __device__ __forceinline__ bool init(const ConvOut& o, int vec) {
    if (vec >= o.vec_end[2]) return false;
    // selects of values: of the arguments' addresses they would put the arguments into scratch memory
    void *y0 = o.y[0], *y1 = o.y[1], *y2 = o.y[2];
    asm("" : "+s"(y0), "+s"(y1), "+s"(y2));
    int begin = 0, end = o.end[0], first = 0;
    void* p = y0;
    if (vec >= o.vec_end[0]) begin = o.end[0], end = o.end[1], first = o.vec_end[0], p = y1;
    if (vec >= o.vec_end[1]) begin = o.end[1], end = o.end[2], first = o.vec_end[1], p = y2;
    c = begin + (vec - first) * kVec;
    n = kVec;
    shift = 0;
    if (c + kVec > end) {
      if (end - begin >= kVec) {
        shift = c + kVec - end;
        c = end - kVec;
      } else {
        n = end - c;
      }
    }
    cols = end - begin;
    y = static_cast<T*>(p) + (c - begin);
    return true;
  }
  // to a state that is read too: its own channels alone
  __device__ __forceinline__ void store_own(T* p, const float (&v)[kVec]) const {
    if (n == kVec && shift == 0) {
      store_vec<T>(p, kVec, v);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (e >= shift && e < n) p[e] = (T)v[e];
    }
  }
};

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

// The last W-1 rows before `len`, those before the sequence from the initial state (which may be the same
// memory: all are read before the first is written, by the channels' one owner).
template <typename T, int W>
__device__ __forceinline__ void write_final(const Columns<T>& col, const T* xb, int64_t token, const T* init,
                                            T* final_state, int64_t len, int64_t D) {
  float last[W - 1][kVec];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t t = len - (W - 1) + j;
#pragma unroll
    for (int e = 0; e < kVec; ++e) last[j][e] = 0.0f;
    if (t >= 0) load_vec<T>(xb + t * token, col.n, last[j]);
    else if (init) load_vec<T>(init + (W - 1 + t) * D, col.n, last[j]);
  }
#pragma unroll
  for (int j = 0; j < W - 1; ++j) col.store_own(final_state + j * D, last[j]);
}

__device__ __forceinline__ int64_t length_of(const int* lengths, int64_t b, int64_t L) {
  if (!lengths) return L;
  return lengths[b] < 0 ? 0 : (lengths[b] < L ? lengths[b] : L);
}

template <typename T, int W, bool kSilu, int kTokens>
__global__ __launch_bounds__(64 * kWaves) void conv_kernel(
    const T* __restrict__ x, Rows xr, const float* __restrict__ w, const float* __restrict__ bias,
    const T* __restrict__ init, const int* __restrict__ lengths, ConvOut out, T* __restrict__ final_state,
    int64_t L, int D, int nctile, int64_t nttile) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // Short walks behind one another on one XCD: the rows that they share come from its L2 (3 x 5000 x 1793 fp16
  // 26.1 -> 23.7 us).  The longest share too little for it, and 65536 x 1024 fp32 went from 116 to 141 us.
  const int64_t bid = kTokens < 64 ? xcd_remap(blockIdx.x, gridDim.x) : (int)blockIdx.x;
  const int ct = (int)(bid % nctile);
  const int64_t tt = (bid / nctile) % nttile;
  const int64_t b = bid / nctile / nttile;
  Columns<T> col;
  if (!col.init(out, ct * 64 + lane)) return;
  const int c = col.c, n = col.n;
  const int64_t t0 = (tt * kWaves + wave) * kTokens;
  if (t0 >= L && t0 > 0) return;
  const int64_t len = length_of(lengths, b, L);
  const T* xb = x + b * xr.batch + c;
  const T* ib = init ? init + b * (W - 1) * D + c : nullptr;
  if (t0 == 0 && final_state)
    write_final<T, W>(col, xb, xr.token, ib, final_state + b * (W - 1) * D + c, len, D);
  if (L == 0) return;

  float wv[W][kVec], bv[kVec], win[W][kVec];
  load_weights<W>(w, bias, c, n, wv, bv);
#pragma unroll
  for (int e = 0; e < kVec; ++e) win[W - 1][e] = 0.0f;
  // rows t0 - (W-1) .. t0 - 1; those before the sequence from the initial state
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t t = t0 - (W - 1) + j;
#pragma unroll
    for (int e = 0; e < kVec; ++e) win[j][e] = 0.0f;
    if (t >= 0) {
      if (t < len) load_vec<T>(xb + t * xr.token, n, win[j]);
    } else if (ib) {
      load_vec<T>(ib + (W - 1 + t) * D, n, win[j]);
    }
  }
  T* dst = col.y + (b * L + t0) * col.cols;
  auto token = [&](float (&y)[kVec]) {   // of the row in win[W - 1]
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      float v = bv[e];
#pragma unroll
      for (int j = 0; j < W; ++j) v = __builtin_fmaf(wv[j][e], win[j][e], v);
      y[e] = kSilu ? silu(v) : v;
#pragma unroll
      for (int j = 0; j + 1 < W; ++j) win[j][e] = win[j + 1][e];
    }
  };
  if (n == kVec && t0 + kTokens <= len) {
    // kAhead tokens' rows on their way during the arithmetic of those before them
    constexpr int kAhead = 4;
    RawVec<T> raw[2][kAhead];
    const T* row = xb + t0 * xr.token;
    auto request = [&](RawVec<T> (&r)[kAhead]) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        __builtin_memcpy(&r[i], row, sizeof(r[i]));
        row += xr.token;
      }
    };
    request(raw[0]);
#pragma unroll
    for (int i0 = 0; i0 < kTokens / kAhead; ++i0) {
      if (i0 + 1 < kTokens / kAhead) request(raw[(i0 + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) win[W - 1][e] = (float)raw[i0 & 1][i].v[e];
        float y[kVec];
        token(y);
        store_vec<T>(dst, kVec, y);
        dst += col.cols;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
    for (int i = 0; i < kTokens && t0 + i < L; ++i) {
      const bool in = t0 + i < len;
      if (in) load_vec<T>(xb + (t0 + i) * xr.token, n, win[W - 1]);
      float y[kVec];
      token(y);
#pragma unroll
      for (int e = 0; e < kVec; ++e) y[e] = in ? y[e] : 0.0f;
      store_vec<T>(dst + i * col.cols, n, y);
    }
  }
}

// The final states alone, where they are written over the initial ones that the kernel above reads.
template <typename T, int W>
__global__ __launch_bounds__(64) void conv_final_kernel(const T* __restrict__ x, Rows xr,
                                                        const int* __restrict__ lengths, ConvOut out,
                                                        T* state, int64_t L, int D, int nctile) {
  const int64_t b = blockIdx.x / nctile;
  Columns<T> col;
  if (!col.init(out, (int)(blockIdx.x % nctile) * 64 + (int)threadIdx.x)) return;
  T* sb = state + b * (W - 1) * D + col.c;
  write_final<T, W>(col, x + b * xr.batch + col.c, xr.token, sb, sb, length_of(lengths, b, L), D);
}

template <typename T, int W, bool kSilu>
__global__ __launch_bounds__(64) void conv_step_kernel(const T* __restrict__ x, int64_t x_row,
                                                       const float* __restrict__ w,
                                                       const float* __restrict__ bias, T* state,
                                                       ConvOut out, int D, int nctile) {
  const int64_t b = blockIdx.x / nctile;
  Columns<T> col;
  if (!col.init(out, (int)(blockIdx.x % nctile) * 64 + (int)threadIdx.x)) return;
  const int c = col.c, n = col.n;
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
  for (int j = 0; j < W - 1; ++j) col.store_own(sb + (int64_t)j * D, win[j + 1]);
  col.store_own(col.y + b * col.cols, y);
}

// Sets the outputs' vectors; the waves that hold them all.
int count_vectors(ConvOut& o) {
  int vecs = 0, begin = 0;
  for (int i = 0; i < 3; ++i) {
    vecs += (o.end[i] - begin + kVec - 1) / kVec;
    o.vec_end[i] = vecs;
    begin = o.end[i];
  }
  return (vecs + 63) / 64;
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
                       const void* init, const int* lengths, const ConvOut& outputs, void* final_state,
                       hipStream_t st) {
  ConvOut out = outputs;
  const int nctile = count_vectors(out);
  // Tokens of a walk: 64 where that leaves every CU two workgroups (4 x 4096 x 5376 fp16: 78 us, 86 with 32, 89
  // with 16), 32 where that leaves it one, else 8 (2048 x 1792: 8.7 us, 14.2 with 32).
  auto count = [&](int64_t tokens) {
    const int64_t n = (seqlen + tokens * kWaves - 1) / (tokens * kWaves);
    return n > 0 ? n : 1;   // no tokens: the states alone
  };
  const int64_t lines = nctile * batch;
  const int tokens = lines * count(64) >= 512 ? 64 : lines * count(32) >= 256 ? 32 : 8;
  const int64_t nttile = count(tokens);
  const int64_t grid = nctile * nttile * batch;
  return for_type(dtype, width, silu, [&](auto t, auto w, auto s) {
    using T = decltype(t);
    constexpr int W = decltype(w)::value;
    const bool over = final_state && final_state == init;
    auto go = [&](auto tokens) {
      conv_kernel<T, W, decltype(s)::value, decltype(tokens)::value>
          <<<dim3((unsigned)grid), 64 * kWaves, 0, st>>>(
              static_cast<const T*>(x), xr, weight, bias, static_cast<const T*>(init), lengths, out,
              over ? nullptr : static_cast<T*>(final_state), seqlen, (int)channels, nctile, nttile);
    };
    if (tokens == 64) go(std::integral_constant<int, 64>());
    else if (tokens == 32) go(std::integral_constant<int, 32>());
    else go(std::integral_constant<int, 8>());
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !over) return e;
    conv_final_kernel<T, W><<<dim3((unsigned)(nctile * batch)), 64, 0, st>>>(
        static_cast<const T*>(x), xr, lengths, out, static_cast<T*>(final_state), seqlen, (int)channels,
        nctile);
    return hipGetLastError();
  });
}

hipError_t launch_conv_step(int dtype, int width, int64_t batch, int64_t channels, const void* x,
                            int64_t x_row, const float* weight, const float* bias, int silu,
                            void* state, const ConvOut& outputs, hipStream_t st) {
  ConvOut out = outputs;
  const int nctile = count_vectors(out);
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
