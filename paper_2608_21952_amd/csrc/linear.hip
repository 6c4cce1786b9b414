// Matrix product with its epilogue:  y[m, n] = act(s[m, n] sum_k x[m, k] w[n, k] + bias[n]) + residual[m, n]
// for fp16, bf16 (fp32 sums, s = 1) and int8 (int32 sums, s = x_scale[m] w_scale[n]).  x and w lie with k
// dense, as activations and a projection's weights do, so a fragment of either matrix instruction operand
// is 16 consecutive bytes of a row for every type: the kernels count k in bytes and differ by type only in
// the instruction.
//
// Many rows (linear_tile): a workgroup forms a kBM x kBN tile of y from k-tiles of 128 bytes per row,
// brought straight into LDS, two buffers deep: the loads of a k-tile are issued behind the barrier that
// frees its buffer and have a whole tile's products to arrive.  LDS holds 16-byte chunk c of row r at slot
// c ^ (r % 8), so that the 64 lanes of a fragment read touch every bank alike; the loads write LDS lane by
// lane, so the exchange is made on the global address.  w is the first operand: a lane then holds four
// consecutive columns of a row, and the tile leaves through LDS in whole lines.
// Few rows (linear_rows): bound by the bytes of w.  A workgroup takes 16 rows of w, its waves share k by
// lines of 128 bytes, each straight from memory into the matrix instruction's registers, and their sums
// meet in LDS.
// A row's end inside a k-tile, and rows that do not start at multiples of 16 bytes, go through registers,
// where what lies behind the end becomes 0 in both operands.
#include <type_traits>

#include "block.hpp"
#include "common.hpp"
#include "ssdi8.h"

namespace ssdi8 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16 v8b __attribute__((ext_vector_type(8)));

struct F16 {
  typedef _Float16 T;
  typedef _Float16 Out;
  typedef v16f Acc32;
  typedef v4f Acc16;
  static __device__ __forceinline__ v16f mma32(uint4 a, uint4 b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a),
                                                  __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ v4f mma16(uint4 a, uint4 b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a),
                                                  __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
};
struct BF16 {
  typedef bf16 T;
  typedef bf16 Out;
  typedef v16f Acc32;
  typedef v4f Acc16;
  static __device__ __forceinline__ v16f mma32(uint4 a, uint4 b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a),
                                                   __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ v4f mma16(uint4 a, uint4 b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a),
                                                   __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  }
};
struct I8 {
  typedef int8_t T;
  typedef _Float16 Out;
  typedef v16i Acc32;
  typedef v4i Acc16;
  static __device__ __forceinline__ v16i mma32(uint4 a, uint4 b, v16i c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(v4i, a),
                                                 __builtin_bit_cast(v4i, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ v4i mma16(uint4 a, uint4 b, v4i c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, a),
                                                 __builtin_bit_cast(v4i, b), c, 0, 0, 0);
  }
};

constexpr int kLine = 128;   // bytes of k per k-tile

// Bytes [at, at + 16) of a row of `bytes`, 0 behind its end; at any alignment of an element.
template <typename T> __device__ __forceinline__ uint4 load_chunk(const char* row, int64_t at, int64_t bytes) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (at + 16 <= bytes) {
    __builtin_memcpy(&v, row + at, 16);
  } else {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; i += (int)sizeof(T))
      if (at + i < bytes) {
        const uint32_t e = sizeof(T) == 2 ? *reinterpret_cast<const uint16_t*>(row + at + i)
                                          : *reinterpret_cast<const uint8_t*>(row + at + i);
        w[i / 4] |= e << (8 * (i % 4));
      }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}

__device__ __forceinline__ float activate(float v, int act) {
  switch (act) {
    case SSDI8_ACT_SILU: return silu(v);
    case SSDI8_ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.707106781186547524f));
    case SSDI8_ACT_SOFTPLUS: return softplus_fast(v);
    default: return v;
  }
}

template <typename Out>
__device__ __forceinline__ void finish_vec(const LinearArgs& a, int64_t m, int64_t c, int n,
                                           float (&v)[kVec]) {
  if (a.residual) {
    float r[kVec];
    if (a.out_dtype == SSDI8_F32)
      load_vec<float>(static_cast<const float*>(a.residual) + m * a.residual_row + c, n, r);
    else
      load_vec<Out>(static_cast<const Out*>(a.residual) + m * a.residual_row + c, n, r);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] += r[e];
  }
  if (a.out_dtype == SSDI8_F32)
    store_vec<float>(static_cast<float*>(a.y) + m * a.y_row + c, n, v);
  else
    store_vec<Out>(static_cast<Out*>(a.y) + m * a.y_row + c, n, v);
}

typedef __attribute__((address_space(3))) void* LdsPtr;
typedef const __attribute__((address_space(1))) void* GlobalPtr;

// kWM x kWN waves, each a (kBM / kWM) x (kBN / kWN) part of the tile.
template <typename K, int kBM, int kBN, int kWM, int kWN>
__global__ __launch_bounds__(64 * kWM * kWN) void linear_tile(LinearArgs a, int mtiles, int ntiles,
                                                               int direct) {
  constexpr int kThreads = 64 * kWM * kWN;
  constexpr int kTM = kBM / kWM / 32, kTN = kBN / kWN / 32;
  constexpr int kBuf = (kBM + kBN) * kLine;
  constexpr int kOutRow = kTN * 32 + 4;   // floats of an LDS row on the way out
  __shared__ __attribute__((aligned(16))) char lds[2 * kBuf];
  static_assert(32 * kOutRow * 4 * kWM * kWN <= 2 * kBuf, "the way out fits");
  typedef typename K::T T;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / kWN, wn = wave % kWN;
  // tiles of one XCD lie together: bands of eight rows of tiles, column by column
  const int id = xcd_remap(blockIdx.x, mtiles * ntiles);
  constexpr int kBand = 8;
  const int band = id / (kBand * ntiles), in = id % (kBand * ntiles);
  const int rows = mtiles - band * kBand < kBand ? mtiles - band * kBand : kBand;
  const int64_t m0 = (int64_t)(band * kBand + in % rows) * kBM;
  const int64_t n0 = (int64_t)(in / rows) * kBN;

  const int64_t kbytes = a.k * (int64_t)sizeof(T);
  const int ktiles = (int)((kbytes + kLine - 1) / kLine);
  const char* xp = static_cast<const char*>(a.x);
  const char* wp = static_cast<const char*>(a.w);

  // this thread's part of a k-tile: chunk `slot` of LDS row r = i * kThreads / 8 + tid / 8 holds chunk
  // slot ^ (r % 8) of that row
  constexpr int kA = kBM * 8 / kThreads, kB = kBN * 8 / kThreads;
  static_assert(kThreads % 64 == 0 && kBM * 8 % kThreads == 0 && kBN * 8 % kThreads == 0, "tile");
  const int lrow = tid >> 3, chunk = (tid & 7) ^ (lrow & 7);
  const char *ap[kA], *bp[kB];
#pragma unroll
  for (int i = 0; i < kA; ++i) {
    int64_t r = m0 + i * (kThreads / 8) + lrow;
    r = r < a.m ? r : a.m - 1;   // rows behind the last: their results are not stored
    ap[i] = xp + r * a.x_row * (int64_t)sizeof(T);
  }
#pragma unroll
  for (int i = 0; i < kB; ++i) {
    int64_t r = n0 + i * (kThreads / 8) + lrow;
    r = r < a.n ? r : a.n - 1;
    bp[i] = wp + r * a.w_row * (int64_t)sizeof(T);
  }
  auto fetch = [&](int kt) {
    char* buf = lds + (kt & 1) * kBuf;
    const int64_t at = (int64_t)kt * kLine + chunk * 16;
    if (direct && (int64_t)(kt + 1) * kLine <= kbytes) {
#pragma unroll
      for (int i = 0; i < kA; ++i)
        __builtin_amdgcn_global_load_lds((GlobalPtr)(ap[i] + at),
                                         (LdsPtr)(buf + (i * kThreads + wave * 64) * 16), 16, 0, 0);
#pragma unroll
      for (int i = 0; i < kB; ++i)
        __builtin_amdgcn_global_load_lds(
            (GlobalPtr)(bp[i] + at), (LdsPtr)(buf + kBM * kLine + (i * kThreads + wave * 64) * 16), 16,
            0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < kA; ++i)
        *reinterpret_cast<uint4*>(buf + (i * kThreads + tid) * 16) = load_chunk<T>(ap[i], at, kbytes);
#pragma unroll
      for (int i = 0; i < kB; ++i)
        *reinterpret_cast<uint4*>(buf + kBM * kLine + (i * kThreads + tid) * 16) =
            load_chunk<T>(bp[i], at, kbytes);
    }
  };

  typename K::Acc32 acc[kTN][kTM] = {};
  const int fr = lane & 31, fk = lane >> 5;
  const int arow = (wm * kTM * 32 + fr) * kLine, brow = kBM * kLine + (wn * kTN * 32 + fr) * kLine;
  fetch(0);
  for (int kt = 0; kt < ktiles; ++kt) {
    // this wave's loads have arrived, every wave has read the other buffer
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (kt + 1 < ktiles) fetch(kt + 1);
    const char* buf = lds + (kt & 1) * kBuf;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const int off = ((2 * ks + fk) ^ (fr & 7)) * 16;
      uint4 av[kTM], bv[kTN];
#pragma unroll
      for (int i = 0; i < kTM; ++i)
        av[i] = *reinterpret_cast<const uint4*>(buf + arow + i * 32 * kLine + off);
#pragma unroll
      for (int i = 0; i < kTN; ++i)
        bv[i] = *reinterpret_cast<const uint4*>(buf + brow + i * 32 * kLine + off);
#pragma unroll
      for (int j = 0; j < kTN; ++j)
#pragma unroll
        for (int i = 0; i < kTM; ++i) acc[j][i] = K::mma32(bv[j], av[i], acc[j][i]);
    }
  }
  __syncthreads();

  // a lane holds row fr of the 32 x 32 block, columns 8 q + 4 fk + (0..3)
  float* out = reinterpret_cast<float*>(lds) + wave * 32 * kOutRow;
  const int64_t wm0 = m0 + wm * kTM * 32, wn0 = n0 + wn * kTN * 32;
  constexpr int kPer = kTN * 32 / kVec;    // lanes of a row on the way out
  constexpr int kRows = 64 / kPer;
#pragma unroll
  for (int i = 0; i < kTM; ++i) {
    const int64_t m = wm0 + i * 32 + fr;
    float sx = 1.0f;
    if constexpr (std::is_same_v<K, I8>) sx = a.x_scale[m < a.m ? m : a.m - 1];
#pragma unroll
    for (int j = 0; j < kTN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t n = wn0 + j * 32 + 8 * q + 4 * fk + e;
          const int64_t nn = n < a.n ? n : a.n - 1;
          v[e] = (float)acc[j][i][4 * q + e];
          if constexpr (std::is_same_v<K, I8>) v[e] *= sx * a.w_scale[nn];
          if (a.bias) v[e] += a.bias[nn];
          if (a.act) v[e] = activate(v[e], a.act);
        }
        *reinterpret_cast<float4*>(out + fr * kOutRow + j * 32 + 8 * q + 4 * fk) =
            make_float4(v[0], v[1], v[2], v[3]);
      }
    // the wave's own rows: no other wave reads or writes them
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += kRows) {
      const int r = r0 + lane / kPer, c = (lane % kPer) * kVec;
      const int64_t mm = wm0 + i * 32 + r, cc = wn0 + c;
      float v[kVec];
      const float4 lo = *reinterpret_cast<const float4*>(out + r * kOutRow + c);
      const float4 hi = *reinterpret_cast<const float4*>(out + r * kOutRow + c + 4);
      v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
      v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
      if (mm < a.m && cc < a.n)
        finish_vec<typename K::Out>(a, mm, cc, a.n - cc < kVec ? (int)(a.n - cc) : kVec, v);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// 16 rows of w by kMT x 16 rows of x per workgroup of kWaves waves.
template <typename K, int kMT, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void linear_rows(LinearArgs a) {
  typedef typename K::T T;
  typedef std::conditional_t<std::is_same_v<K, I8>, int, float> Sum;
  __shared__ Sum part[kWaves][kMT][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * kMT);
  const int64_t kbytes = a.k * (int64_t)sizeof(T);
  const int lines = (int)((kbytes + kLine - 1) / kLine);
  const int fr = lane & 15, fk = lane >> 4;
  const int64_t wr = n0 + fr < a.n ? n0 + fr : a.n - 1;
  const char* wrow = static_cast<const char*>(a.w) + wr * a.w_row * (int64_t)sizeof(T);
  const char* xrow[kMT];
#pragma unroll
  for (int i = 0; i < kMT; ++i) {
    const int64_t m = m0 + i * 16 + fr < a.m ? m0 + i * 16 + fr : a.m - 1;
    xrow[i] = static_cast<const char*>(a.x) + m * a.x_row * (int64_t)sizeof(T);
  }
  typename K::Acc16 acc[kMT] = {};
#pragma unroll 4
  for (int l = wave; l < lines; l += kWaves) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int64_t at = (int64_t)l * kLine + s * 64 + fk * 16;
      const uint4 wv = load_chunk<T>(wrow, at, kbytes);
#pragma unroll
      for (int i = 0; i < kMT; ++i)
        acc[i] = K::mma16(wv, load_chunk<T>(xrow[i], at, kbytes), acc[i]);
    }
  }
  // a lane holds row fr of x, columns 4 fk + (0..3)
#pragma unroll
  for (int i = 0; i < kMT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][i][fr * 16 + fk * 4 + e] = acc[i][e];
  __syncthreads();
  for (int o = tid; o < kMT * 256; o += 64 * kWaves) {
    const int i = o >> 8, r = (o >> 4) & 15, c = o & 15;
    const int64_t m = m0 + i * 16 + r, n = n0 + c;
    Sum sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += part[w][i][o & 255];
    if (m >= a.m || n >= a.n) continue;
    float v = (float)sum;
    if constexpr (std::is_same_v<K, I8>) v *= a.x_scale[m] * a.w_scale[n];
    if (a.bias) v += a.bias[n];
    if (a.act) v = activate(v, a.act);
    typedef typename K::Out Out;
    if (a.out_dtype == SSDI8_F32) {
      if (a.residual) v += static_cast<const float*>(a.residual)[m * a.residual_row + n];
      static_cast<float*>(a.y)[m * a.y_row + n] = v;
    } else {
      if (a.residual) v += (float)static_cast<const Out*>(a.residual)[m * a.residual_row + n];
      static_cast<Out*>(a.y)[m * a.y_row + n] = (Out)v;
    }
  }
}

template <typename K, int kBM, int kBN, int kWM, int kWN>
hipError_t run_tile(const LinearArgs& a, int direct, hipStream_t st) {
  const int64_t mt = (a.m + kBM - 1) / kBM, nt = (a.n + kBN - 1) / kBN;
  linear_tile<K, kBM, kBN, kWM, kWN>
      <<<dim3((unsigned)(mt * nt)), 64 * kWM * kWN, 0, st>>>(a, (int)mt, (int)nt, direct);
  return hipGetLastError();
}

template <typename K> hipError_t run(const LinearArgs& a, hipStream_t st) {
  if (a.m <= 64) {
    const unsigned nt = (unsigned)((a.n + 15) / 16);
    if (a.m <= 16) linear_rows<K, 1, 8><<<dim3(nt, 1), 512, 0, st>>>(a);
    else if (a.m <= 32) linear_rows<K, 2, 8><<<dim3(nt, 1), 512, 0, st>>>(a);
    else linear_rows<K, 4, 8><<<dim3(nt, 1), 512, 0, st>>>(a);
    return hipGetLastError();
  }
  constexpr int64_t es = sizeof(typename K::T);
  const int direct = ((uintptr_t)a.x % 16 == 0 && (uintptr_t)a.w % 16 == 0 &&
                      a.x_row * es % 16 == 0 && a.w_row * es % 16 == 0);
  auto tiles = [&](int64_t bm, int64_t bn) { return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn); };
  if (tiles(256, 256) >= 256) return run_tile<K, 256, 256, 2, 4>(a, direct, st);
  if (tiles(128, 128) >= 128) return run_tile<K, 128, 128, 2, 2>(a, direct, st);
  return run_tile<K, 64, 64, 2, 2>(a, direct, st);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, hipStream_t st) {
  switch (a.dtype) {
    case SSDI8_F16: return run<F16>(a, st);
    case SSDI8_BF16: return run<BF16>(a, st);
    default: return run<I8>(a, st);
  }
}

}  // namespace ssdi8
