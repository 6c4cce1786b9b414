// Matrix product with its epilogue:  y[m, n] = act(s[m, n] sum_k x[m, k] w[n, k] + bias[n]) + residual[m, n]
// for fp16, bf16 (fp32 sums, s = 1) and int8 (int32 sums, s = x_scale[m] w_scale[n]).  x and w lie with k
// dense, as activations and a projection's weights do, so a fragment of either matrix instruction operand
// is 16 consecutive bytes of a row for every type: the kernels count k in bytes and differ by type only in
// the instruction.
//
// Many rows (linear_tile): a workgroup forms a kBM x kBN tile of y from k-tiles of 128 bytes per row in two
// LDS buffers, a third k-tile on its way in registers.  LDS holds 16-byte chunk c of row r at slot
// c ^ (r / 2 % 8), so that the 16 lanes that a fragment read serves at a time touch every bank once.  w is
// the first operand: a lane then holds four consecutive columns of a row, and the tile leaves through LDS
// in whole lines.
// What bounds it: the matrix unit and the way of the operands into it, which do not overlap in full: taken
// apart (8192^3 bf16, loads straight to LDS at that time, 1070 us in all) the products with their fragment
// reads took 703 us, the loads with the reads 802.  int8 16384 x 10496 x 2560 472 us (1.87 Pop/s; the vendor's
// library 472 without the epilogue), fp16 16384 x 768 x 1536 with residual 52 us (0.74 PFLOP/s; 42 without it; 61
// where neither inputs nor outputs are in the cache), fp16 16384 x 10496 x 2560 830 us (779).
// Few rows (linear_rows): bound by the bytes of w.  A workgroup takes 16 or 32 rows of w, its waves share k
// by lines of 128 bytes, each straight from memory into the matrix instruction's registers, and their sums
// meet in LDS.  8 x 10496 x 2560 bf16: 13.0 us, 4.1 TB/s, near the time that the first loads take to arrive.
// What lies behind a row's end in its last k-tile or line becomes 0 in both operands; rows may start at any
// element.
#include <type_traits>

#include "block.hpp"
#include "common.hpp"
#include "epilogue.hpp"
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

constexpr int kLine = 128;    // bytes of k per k-tile
constexpr int kChunks = kLine / 16;

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

// The exchange of chunks in LDS row r (see above).
__device__ __forceinline__ int slot_key(int r) { return (r >> 1) & 7; }

// kWM x kWN waves, each a (kBM / kWM) x (kBN / kWN) part of the tile; kSplit such sets of waves share k, each
// with buffers of its own, and the first adds up the others' sums.
template <typename K, int kBM, int kBN, int kWM, int kWN, int kSplit>
__global__ __launch_bounds__(64 * kWM * kWN * kSplit) void linear_tile(LinearArgs a, int mtiles, int ntiles) {
  constexpr int kThreads = 64 * kWM * kWN;   // of a set
  constexpr int kTM = kBM / kWM / 32, kTN = kBN / kWN / 32;
  constexpr int kBuf = (kBM + kBN) * kLine;
  constexpr int kOutRow = kTN * 32 + 4;   // floats of an LDS row on the way out
  __shared__ __attribute__((aligned(16))) char all_lds[kSplit * 2 * kBuf];
  static_assert(32 * kOutRow * 4 * kWM * kWN <= 2 * kBuf, "the way out fits");
  typedef typename K::T T;

  const int set = kSplit > 1 ? threadIdx.x / kThreads : 0;
  const int tid = kSplit > 1 ? threadIdx.x % kThreads : threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / kWN, wn = wave % kWN;
  char* lds = all_lds + set * 2 * kBuf;
  // tiles of one XCD lie together: bands of four rows of tiles, column by column
  const int id = xcd_remap(blockIdx.x, mtiles * ntiles);
  constexpr int kBand = 4;
  const int band = id / (kBand * ntiles), in = id % (kBand * ntiles);
  const int rows = mtiles - band * kBand < kBand ? mtiles - band * kBand : kBand;
  const int64_t m0 = (int64_t)(band * kBand + in % rows) * kBM;
  const int64_t n0 = (int64_t)(in / rows) * kBN;

  const int64_t kbytes = a.k * (int64_t)sizeof(T);
  // the k-tiles of this set: as many for every set (they meet at the same barriers), zeros behind the last
  const int all = (int)((kbytes + kLine - 1) / kLine), ktiles = (all + kSplit - 1) / kSplit;
  const int64_t k0 = (int64_t)set * ktiles * kLine;
  int whole = (int)((kbytes - k0) / kLine);
  whole = kbytes < k0 ? 0 : (whole < ktiles ? whole : ktiles);
  // this thread's part of a k-tile: slot tid % kChunks of LDS row r = i * kThreads / kChunks + tid / kChunks
  // holds chunk slot ^ key(r) of that row
  constexpr int kLoadRows = kThreads / kChunks;
  constexpr int kA = kBM / kLoadRows, kB = kBN / kLoadRows;
  static_assert(kLoadRows % 16 == 0 && kBM % kLoadRows == 0 && kBN % kLoadRows == 0, "tile");
  const int lrow = tid / kChunks, chunk = (tid % kChunks) ^ slot_key(lrow);
  // rows behind the last are taken for it: their results are not stored.  32-bit offsets from the tile's
  // first row (the host refuses rows too far apart for them)
  uint32_t offset[kA + kB];
#pragma unroll
  for (int i = 0; i < kA + kB; ++i) {
    const int64_t left = i < kA ? a.m - m0 : a.n - n0;
    int64_t r = (i < kA ? i : i - kA) * kLoadRows + lrow;
    r = r < left ? r : left - 1;
    offset[i] = (uint32_t)(r * (i < kA ? a.x_row : a.w_row) * (int64_t)sizeof(T)) + chunk * 16;
  }
  const char* xp = static_cast<const char*>(a.x) + m0 * a.x_row * (int64_t)sizeof(T) + k0;
  const char* wp = static_cast<const char*>(a.w) + n0 * a.w_row * (int64_t)sizeof(T) + k0;

  typename K::Acc32 acc[kTN][kTM] = {};
  const int fr = lane & 31, fk = lane >> 5;
  const int arow = (wm * kTM * 32 + fr) * kLine, brow = kBM * kLine + (wn * kTN * 32 + fr) * kLine;
  struct Frags {
    uint4 x[kTM], w[kTN];
  };
  auto read = [&](int kt, int ks, Frags& f) {
    const char* buf = lds + kt % 2 * kBuf;
    const int off = ((2 * ks + fk) ^ slot_key(fr)) * 16;
#pragma unroll
    for (int i = 0; i < kTM; ++i)
      f.x[i] = *reinterpret_cast<const uint4*>(buf + arow + i * 32 * kLine + off);
#pragma unroll
    for (int i = 0; i < kTN; ++i)
      f.w[i] = *reinterpret_cast<const uint4*>(buf + brow + i * 32 * kLine + off);
  };
  // One 16-byte load per lane of a k-tile on its way, and its place in LDS.
  constexpr int kParts = kA + kB;
  uint4 part[kParts];
  auto request = [&](int kt, int i, auto inside) {   // inside: a whole k-tile
    const char* p = (i < kA ? xp : wp) + (int64_t)kt * kLine + offset[i];
    if constexpr (decltype(inside)::value) __builtin_memcpy(&part[i], p, 16);
    else part[i] = load_chunk<T>(p, 0, kbytes - k0 - (int64_t)kt * kLine - chunk * 16);
  };
  auto put = [&](int kt, int i) {
    char* buf = lds + (kt & 1) * kBuf + (i < kA ? 0 : kBM * kLine) + tid * 16;
    *reinterpret_cast<uint4*>(buf + (i < kA ? i : i - kA) * kThreads * 16) = part[i];
  };
  // Step ks of k-tile kt forms the products of 32 bytes.  Meanwhile the next step's fragments are read,
  // over the k-tiles' borders too, and the next k-tile moves from registers to the other buffer, a part
  // per step, each part's registers taking the k-tile after it: a load has four steps to arrive, and no
  // step waits for the address unit, which takes as long for a k-tile's 64 KB as two steps' products.
  constexpr int kSteps = kLine / 32, kPerStep = (kParts + kSteps - 2) / (kSteps - 1);
  Frags f[2];
  auto begin = [&](auto inside) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) request(0, i, inside);
#pragma unroll
    for (int i = 0; i < kParts; ++i) put(0, i);
    if (decltype(inside)::value || ktiles > 1)
#pragma unroll
      for (int i = 0; i < kParts; ++i) request(1, i, inside);
    __syncthreads();
    read(0, 0, f[0]);
  };
  auto k_tile = [&](int kt, auto inside) {   // inside: k-tiles kt + 1 and kt + 2 are there and whole
    constexpr bool kInside = decltype(inside)::value;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) {
      if (ks + 1 < kSteps) {
        read(kt, ks + 1, f[(ks + 1) & 1]);
      } else if (kInside || kt + 1 < ktiles) {
        __syncthreads();   // the next buffer is written, this one read
        read(kt + 1, 0, f[0]);
      }
#pragma unroll
      for (int j = 0; j < kTN; ++j) {
#pragma unroll
        for (int i = 0; i < kTM; ++i)
          acc[j][i] = K::mma32(f[ks & 1].w[j], f[ks & 1].x[i], acc[j][i]);
        // the compiler would otherwise gather the loads at the end of the k-tile
        __builtin_amdgcn_sched_barrier(0);
        if (j == 0 && ks + 1 < kSteps && (kInside || kt + 1 < ktiles)) {
#pragma unroll
          for (int e = 0; e < kPerStep; ++e) {
            const int i = ks * kPerStep + e;
            if (i < kParts) {
              put(kt + 1, i);
              if (kInside || kt + 2 < ktiles) request(kt + 2, i, inside);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  int kt = 0;
  if (whole > 2) {
    begin(std::true_type());
    for (; kt + 2 < whole; ++kt) k_tile(kt, std::true_type());
  } else {
    begin(std::false_type());
  }
  for (; kt < ktiles; ++kt) k_tile(kt, std::false_type());
  __syncthreads();
  if constexpr (kSplit > 1) {
    typedef std::conditional_t<std::is_same_v<K, I8>, int4, float4> Four;
    static_assert(kThreads * kTN * kTM * 64 <= 2 * kBuf, "a set's sums fit its buffers");
    auto place = [&](char* at, int j, int i, int q) {
      return reinterpret_cast<Four*>(at) + ((((j * kTM + i) * 4 + q) * (kThreads / 64) + wave) * 64 + lane);
    };
    if (set > 0) {
#pragma unroll
      for (int j = 0; j < kTN; ++j)
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            Four v;
            v.x = acc[j][i][4 * q], v.y = acc[j][i][4 * q + 1], v.z = acc[j][i][4 * q + 2], v.w = acc[j][i][4 * q + 3];
            *place(lds, j, i, q) = v;
          }
    }
    __syncthreads();
    if (set > 0) return;
    for (int k = 1; k < kSplit; ++k)
#pragma unroll
      for (int j = 0; j < kTN; ++j)
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const Four v = *place(all_lds + k * 2 * kBuf, j, i, q);
            acc[j][i][4 * q] += v.x, acc[j][i][4 * q + 1] += v.y;
            acc[j][i][4 * q + 2] += v.z, acc[j][i][4 * q + 3] += v.w;
          }
  }

  // a lane holds row fr of the 32 x 32 block, columns 8 q + 4 fk + (0..3); on the way out it has eight
  // columns, the same ones of every row
  float* out = reinterpret_cast<float*>(lds) + wave * 32 * kOutRow;
  const int64_t wm0 = m0 + wm * kTM * 32, wn0 = n0 + wn * kTN * 32;
  constexpr int kPer = kTN * 32 / kVec;    // vectors of a row on the way out
  constexpr bool kSame = 64 % kPer == 0;   // a lane has the same columns in every row
  static_assert(32 * kPer % 64 == 0, "whole waves on the way out");
  float bias[kVec] = {}, ws[kVec] = {};
  auto columns = [&](int64_t c, int n) {
    if (n <= 0) return;
    if (a.bias) load_vec<float>(a.bias + c, n, bias);
    if constexpr (std::is_same_v<K, I8>) load_vec<float>(a.w_scale + c, n, ws);
  };
  if (kSame) columns(wn0 + lane % kPer * kVec, (int)(a.n - wn0 - lane % kPer * kVec < kVec
                                                        ? a.n - wn0 - lane % kPer * kVec : kVec));
#pragma unroll
  for (int i = 0; i < kTM; ++i) {
#pragma unroll
    for (int j = 0; j < kTN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(out + fr * kOutRow + j * 32 + 8 * q + 4 * fk) =
            make_float4((float)acc[j][i][4 * q], (float)acc[j][i][4 * q + 1],
                        (float)acc[j][i][4 * q + 2], (float)acc[j][i][4 * q + 3]);
    // the wave's own rows: no other wave reads or writes them
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 32 * kPer / 64; ++k) {
      const int r = (k * 64 + lane) / kPer, oc = (k * 64 + lane) % kPer * kVec;
      const int64_t mm = wm0 + i * 32 + r, cc = wn0 + oc;
      const int cn = cc >= a.n ? 0 : (a.n - cc < kVec ? (int)(a.n - cc) : kVec);
      if (!kSame) columns(cc, cn);
      float v[kVec];
      const float4 lo = *reinterpret_cast<const float4*>(out + r * kOutRow + oc);
      const float4 hi = *reinterpret_cast<const float4*>(out + r * kOutRow + oc + 4);
      v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
      v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
      if (mm < a.m && cn > 0) {
        if constexpr (std::is_same_v<K, I8>) {
          const float sx = a.x_scale[mm];
#pragma unroll
          for (int e = 0; e < kVec; ++e) v[e] *= sx * ws[e];
        }
        if (a.bias)
#pragma unroll
          for (int e = 0; e < kVec; ++e) v[e] += bias[e];
        if (a.act)
#pragma unroll
          for (int e = 0; e < kVec; ++e) v[e] = activate(v[e], a.act);
        finish_vec<typename K::Out>(a, mm, cc, cn, v);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

constexpr int kRowLine = 128;

// kNT x 16 rows of w by kMT x 16 rows of x per workgroup of kWaves waves.
template <typename K, int kNT, int kMT, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void linear_rows(LinearArgs a) {
  typedef typename K::T T;
  typedef std::conditional_t<std::is_same_v<K, I8>, int, float> Sum;
  __shared__ Sum part[kWaves][kNT * kMT][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * kNT);
  const int64_t kbytes = a.k * (int64_t)sizeof(T);
  const int whole = (int)(kbytes / kRowLine), lines = (int)((kbytes + kRowLine - 1) / kRowLine);
  const int fr = lane & 15, fk = lane >> 4;
  const char *wrow[kNT], *xrow[kMT];
#pragma unroll
  for (int j = 0; j < kNT; ++j) {
    const int64_t n = n0 + j * 16 + fr < a.n ? n0 + j * 16 + fr : a.n - 1;
    wrow[j] = static_cast<const char*>(a.w) + n * a.w_row * (int64_t)sizeof(T) + fk * 16;
  }
#pragma unroll
  for (int i = 0; i < kMT; ++i) {
    const int64_t m = i * 16 + fr < a.m ? i * 16 + fr : a.m - 1;
    xrow[i] = static_cast<const char*>(a.x) + m * a.x_row * (int64_t)sizeof(T) + fk * 16;
  }
  typename K::Acc16 acc[kNT][kMT] = {};
  auto line = [&](int l, auto inside) {
    constexpr bool kInside = decltype(inside)::value;   // the line ends before the row does
    uint4 wv[2][kNT], xv[2][kMT];
    auto get = [&](const char* row, int s) {
      const int64_t at = (int64_t)l * kRowLine + s * 64;
      uint4 v;
      if constexpr (kInside) __builtin_memcpy(&v, row + at, 16);
      else v = load_chunk<T>(row + at, 0, kbytes - at - fk * 16);
      return v;
    };
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int j = 0; j < kNT; ++j) wv[s][j] = get(wrow[j], s);
#pragma unroll
      for (int i = 0; i < kMT; ++i) xv[s][i] = get(xrow[i], s);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < kNT; ++j)
#pragma unroll
        for (int i = 0; i < kMT; ++i) acc[j][i] = K::mma16(wv[s][j], xv[s][i], acc[j][i]);
  };
  int l = wave;
  constexpr int kUnroll = 8 / (kNT + kMT) > 1 ? 8 / (kNT + kMT) : 1;
#pragma unroll kUnroll
  for (; l < whole; l += kWaves) line(l, std::true_type());
  if (l < lines) line(l, std::false_type());
  // a lane holds row fr of x, columns 4 fk + (0..3)
#pragma unroll
  for (int j = 0; j < kNT; ++j)
#pragma unroll
    for (int i = 0; i < kMT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][j * kMT + i][fr * 16 + fk * 4 + e] = acc[j][i][e];
  __syncthreads();
  for (int o = tid; o < kNT * kMT * 256; o += 64 * kWaves) {
    const int tile = o >> 8, r = (o >> 4) & 15, c = o & 15;
    const int64_t m = tile % kMT * 16 + r, n = n0 + tile / kMT * 16 + c;
    Sum sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += part[w][tile][o & 255];
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

template <typename K, int kBM, int kBN, int kWM, int kWN, int kSplit = 1>
hipError_t run_tile(const LinearArgs& a, hipStream_t st) {
  const int64_t mt = (a.m + kBM - 1) / kBM, nt = (a.n + kBN - 1) / kBN;
  linear_tile<K, kBM, kBN, kWM, kWN, kSplit>
      <<<dim3((unsigned)(mt * nt)), 64 * kWM * kWN * kSplit, 0, st>>>(a, (int)mt, (int)nt);
  return hipGetLastError();
}

template <typename K> hipError_t run(const LinearArgs& a, hipStream_t st) {
  // Few rows.  Up to 16, one matrix tile of x: 8 x 10496 x 2560 bf16 13.1 us with 16 rows of w per workgroup,
  // 15.2 with 32 (8 x 2560 x 5120 9.2 / 14.6).  Up to 32, twice the rows of w where they still fill the card:
  // 24 x 5120 x 2560 int8 8.0 / 6.9.  Up to 64, while one round of workgroups does and the rows of x, which every
  // workgroup reads, are short (33 x 2560 x 2560 fp16 10.6 us, tiles 10.9; 64 x 768 x 640 5.2, 5.6; 64 x 2560 x 5120
  // 25.9, 20.2), or two rounds over a short k (48 x 6400 x 320 int8 4.6, 6.2; 33 x 8000 x 2560 fp16 19.2, 12.4).
  auto rows = [&](auto most, auto tiles) {
    constexpr int kMT = decltype(most)::value, kNT = decltype(tiles)::value;
    linear_rows<K, kNT, kMT, 8><<<dim3((unsigned)((a.n + 16 * kNT - 1) / (16 * kNT))), 512, 0, st>>>(a);
    return hipGetLastError();
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  if (a.m <= 16) return rows(One(), One());
  if (a.m <= 32) return a.n >= 4096 ? rows(Two(), Two()) : rows(Two(), One());
  const int64_t kbytes = a.k * (int64_t)sizeof(typename K::T);
  if (a.m <= 64 && (a.n <= 256 * 16 ? a.m * kbytes <= 200000 : a.n < 2 * 256 * 16 && kbytes < 10 * kLine))
    return rows(std::integral_constant<int, 4>(), One());
  // The tile whose rounds over the card's 256 CUs cost least: rounds * area / rate, the rates (of the
  // largest tile's) as 8192^3 in bf16 measured them: 898 us with 256 x 256, 986 with 256 x 192, 1030 with
  // 256 x 128, 1108 with 128 x 128, 1700 with 64 x 64.  Where another than the largest wins: 16384 x 768 x
  // 1536 49.7 / 47.2 us with 256 x 192, 2048 x 2560 x 5120 104 / 68.7 with 256 x 128, 512 x 5120 x 2560
  // 55.4 / 24.0 with 128 x 128, 128 x 5120 x 2560 54.2 / 16.5 with 64 x 64.
  auto count = [&](int64_t bm, int64_t bn) { return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn); };
  auto cost = [&](int64_t bm, int64_t bn, double rate) {
    return (double)((count(bm, bn) + 255) / 256) * (double)(bm * bn) / rate;
  };
  const double costs[] = {cost(256, 256, 1.0), cost(256, 192, 0.9), cost(256, 128, 0.87),
                          cost(128, 128, 0.81), cost(64, 64, 0.53)};
  int best = 0;
  for (int i = 1; i < 5; ++i)
    if (costs[i] < costs[best]) best = i;
  switch (best) {
    case 0: return run_tile<K, 256, 256, 2, 4>(a, st);
    case 1: return run_tile<K, 256, 192, 4, 2>(a, st);
    case 2: return run_tile<K, 256, 128, 4, 2>(a, st);
    case 3: return run_tile<K, 128, 128, 2, 2>(a, st);
    default: break;
  }
  // Small tiles that leave CUs without a second one, over a long k: four sets of waves share it (128 x 5120 x
  // 2560 fp16 16.3 -> 12.3 us, 200 x 2000 x 2000 12.1 -> 10.5, 100 x 768 x 1536 8.8 -> 7.8; over a short one their
  // ends cost more: 300 x 1111 x 1600 int8 8.7 -> 13.2).
  const bool split = count(64, 64) <= 256 && kbytes >= 24 * kLine;
  return split ? run_tile<K, 64, 64, 2, 2, 4>(a, st) : run_tile<K, 64, 64, 2, 2>(a, st);
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
