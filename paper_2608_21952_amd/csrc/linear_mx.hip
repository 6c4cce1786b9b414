// Matrix product of microscaled operands with its epilogue:
//   y[m, n] = act(sum_b 2^(ex[m, b] + ew[n, b]) sum_{k in block b} x[m, k] w[n, k] + bias[n]) + residual[m, n]
// w in e2m1 (two values to a byte), x in e2m1 or e4m3, blocks of 32 along k with a power of two each, sums in fp32:
// the scaled matrix instructions take both scales beside the operands.
//
// The 32 x 32 x 64 instruction takes two blocks of a row: e2m1 lanes hold 32 values (16 bytes) of one block, e4m3
// lanes 16 values of each of the two; the scale of block h comes from the lanes of half h.  Which two blocks meet in
// an instruction is free.  A k-tile is eight blocks: half h takes blocks 4 h + s in step s, so that a lane's four
// scales are the four bytes of one word.
//
// Many rows (mx_tile): a workgroup forms a kBM x kBN tile of y from k-tiles in two LDS buffers, a third one on its way
// in registers.  LDS holds 16-byte chunk c of a line (128 bytes) of row r at slot c ^ (r / 2 % 8), so that the
// 16 lanes that a fragment read serves at a time touch every bank once.
// What bounds it: the way of the operands into LDS (a tile of 128 x 128 needs 32 KB for 512 cycles of a SIMD's products)
// and the way out; 16384 x 10496 x 2560 382 us (2.3 PFLOP/s, the vendor's library 402; products from registers alone
// reach 5.7), with e4m3 x 524 (library, both operands e4m3, 678).  Tiles of 256 x 256 did not fit the registers.
// Few rows (mx_rows): bound by the bytes of w.  A workgroup takes 16 rows of w, its waves share k by lines of 128
// bytes, each straight from memory into the matrix instruction's registers, and their sums meet in LDS.
#include "common.hpp"
#include "epilogue.hpp"
#include "mx.hpp"

namespace ssdi8 {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kLine = 128;           // bytes of a row of w per k-tile
constexpr int kTileBlocks = 8;       // blocks per k-tile
constexpr int kE4m3 = 0, kE2m1 = 4;  // the instruction's names of the types

// A lane's part of an operand: 16 bytes (e2m1) or 32 (e4m3).
template <int kX> struct Part {
  uint4 v[kX == kE4m3 ? 2 : 1];
};
template <int kX> __device__ __forceinline__ v8i operand(const Part<kX>& p) {
  const uint4 hi = kX == kE4m3 ? p.v[kX == kE4m3 ? 1 : 0] : make_uint4(0, 0, 0, 0);
  return v8i{(int)p.v[0].x, (int)p.v[0].y, (int)p.v[0].z, (int)p.v[0].w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}
template <int kX, int kByte>
__device__ __forceinline__ v16f mma32(const Part<kE2m1>& w, uint32_t ws, const Part<kX>& x, uint32_t xs, v16f c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand<kE2m1>(w), operand<kX>(x), c, kE2m1, kX, kByte,
                                                         (int)ws, kByte, (int)xs);
}
template <int kX, int kByte>
__device__ __forceinline__ v4f mma16(const Part<kE2m1>& w, uint32_t ws, const Part<kX>& x, uint32_t xs, v4f c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand<kE2m1>(w), operand<kX>(x), c, kE2m1, kX, kByte,
                                                          (int)ws, kByte, (int)xs);
}

// kBytes scale bytes of a row from block b on, 0 behind its last block (where the codes are 0, too).
template <int kBytes> __device__ __forceinline__ uint32_t scale_word(const uint8_t* row, int64_t b, int64_t blocks) {
  uint32_t v = 0;
  if (b + kBytes <= blocks) {
    __builtin_memcpy(&v, row + b, kBytes);
  } else {
#pragma unroll
    for (int i = 0; i < kBytes; ++i)
      if (b + i < blocks) v |= (uint32_t)row[b + i] << (8 * i);
  }
  return v;
}

template <typename Out>
__device__ __forceinline__ void finish_row(const LinearMx& a, int64_t m, int64_t c, int n, float (&v)[kVec]) {
  if (a.residual) {
    float r[kVec];
    load_vec<Out>(static_cast<const Out*>(a.residual) + m * a.residual_row + c, n, r);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] += r[e];
  }
  store_vec<Out>(static_cast<Out*>(a.y) + m * a.y_row + c, n, v);
}
__device__ __forceinline__ void finish(const LinearMx& a, int64_t m, int64_t c, int n, float (&v)[kVec]) {
  switch (a.out_dtype) {
    case SSDI8_F32: return finish_row<float>(a, m, c, n, v);
    case SSDI8_F16: return finish_row<_Float16>(a, m, c, n, v);
    default: return finish_row<bf16>(a, m, c, n, v);
  }
}

__device__ __forceinline__ int slot_key(int r) { return (r >> 1) & 7; }

// kWM x kWN waves, each a (kBM / kWM) x (kBN / kWN) part of the tile.
template <int kX, int kBM, int kBN, int kWM, int kWN>
__global__ __launch_bounds__(64 * kWM * kWN) void mx_tile(LinearMx a, int mtiles, int ntiles, int first) {
  constexpr int kThreads = 64 * kWM * kWN;
  constexpr int kXL = kX == kE4m3 ? 2 : 1;   // lines of a row of x per k-tile
  constexpr int kTM = kBM / kWM / 32, kTN = kBN / kWN / 32;
  constexpr int kXBytes = kBM * kXL * kLine, kBuf = kXBytes + kBN * kLine;
  constexpr int kOutRow = kTN * 32 + 4;   // floats of an LDS row on the way out
  __shared__ __attribute__((aligned(16))) char lds[2 * kBuf];
  static_assert(32 * kOutRow * 4 * kWM * kWN <= 2 * kBuf, "the way out fits");

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / kWN, wn = wave % kWN;
  // tiles of one XCD lie together: bands of four rows of tiles, column by column
  const int id = first + xcd_remap(blockIdx.x, gridDim.x);
  constexpr int kBand = 4;
  const int band = id / (kBand * ntiles), in = id % (kBand * ntiles);
  const int rows = mtiles - band * kBand < kBand ? mtiles - band * kBand : kBand;
  const int64_t m0 = (int64_t)(band * kBand + in % rows) * kBM;
  const int64_t n0 = (int64_t)(in / rows) * kBN;
  const int64_t x_row = a.blocks * (16 * kXL), w_row = a.blocks * 16;   // bytes
  const int ktiles = (int)((a.blocks + kTileBlocks - 1) / kTileBlocks);

  // this thread's part of a k-tile: slot tid % 8 of LDS lines i * kThreads / 8 + tid / 8, which holds chunk slot ^
  // key of a row's line.  Lines of x: all rows' first lines, then their second ones.
  constexpr int kLoadLines = kThreads / 8;
  constexpr int kA = kBM * kXL / kLoadLines, kB = kBN / kLoadLines, kParts = kA + kB;
  static_assert(kLoadLines % 16 == 0 && kBM % kLoadLines == 0 && kBN % kLoadLines == 0, "tile");
  const int lrow = tid / 8, chunk = (tid % 8) ^ slot_key(lrow);
  // One offset for all loads, the rest in scalar registers; rows behind the last give 0, as what lies at kNowhere does.
  constexpr uint32_t kNowhere = 0xfffffff0u;
  auto tile_of = [](const uint8_t* p, int64_t row, int64_t rows, int64_t row_bytes) {
    const int64_t bytes = (rows - row) * row_bytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p + row * row_bytes), 0,
                                             (int)(uint32_t)(bytes < 0xffff0000ll ? bytes : 0xffff0000ll), 0x00027000);
  };
  const auto x_tile = tile_of(a.x, m0, a.m, x_row), w_tile = tile_of(a.w, n0, a.n, w_row);
  const uint32_t x_off = (uint32_t)(lrow * x_row) + chunk * 16, w_off = (uint32_t)(lrow * w_row) + chunk * 16;

  const int fr = lane & 31, fh = lane >> 5;
  v16f acc[kTN][kTM] = {};
  // A lane's scales of a k-tile: the bytes of blocks 4 fh .. 4 fh + 3, one load for each 32 rows.  Rows behind the last
  // give 0.
  const int xs0 = wm * kTM * 32, ws0 = wn * kTN * 32;
  auto rows_of = [](const uint8_t* p, int64_t row, int64_t rows, int64_t blocks) {
    const int64_t bytes = row < rows ? (rows - row) * blocks : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p + row * blocks), 0,
                                             (int)(bytes < 0x40000000 ? bytes : 0x40000000), 0x00027000);
  };
  const auto xs_rows = rows_of(a.xs, m0 + xs0, a.m, a.blocks), ws_rows = rows_of(a.ws, n0 + ws0, a.n, a.blocks);
  const int blocks = (int)a.blocks, s_off = fr * blocks + 4 * fh;
  struct Scales {
    uint32_t x[kTM], w[kTN];
  };
  auto read_scales = [&](int kt, Scales& s) {
    const int at = s_off + kt * kTileBlocks;
#pragma unroll
    for (int i = 0; i < kTM; ++i) s.x[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(xs_rows, at, i * 32 * blocks, 0);
#pragma unroll
    for (int j = 0; j < kTN; ++j) s.w[j] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ws_rows, at, j * 32 * blocks, 0);
  };
  // In a row's last k-tile: what lies behind its end is another row's, and may be a NaN; its codes are 0.  Where a word
  // would end behind the last row's end it is not read: byte by byte.
  auto cut_scales = [&](int kt, Scales& s) {
    const int left = blocks - kt * kTileBlocks - 4 * fh;
    auto word = [&](auto rows, int row) {
      uint32_t v = 0;
      for (int e = 0; e < 4 && e < left; ++e)
        v |= (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rows, s_off + kt * kTileBlocks + e, row * blocks, 0) << (8 * e);
      return v;
    };
#pragma unroll
    for (int i = 0; i < kTM; ++i) s.x[i] = word(xs_rows, i * 32);
#pragma unroll
    for (int j = 0; j < kTN; ++j) s.w[j] = word(ws_rows, j * 32);
  };

  struct Frags {
    Part<kX> x[kTM];
    Part<kE2m1> w[kTN];
  };
  auto read = [&](int kt, int s, Frags& f) {
    const char* buf = lds + (kt & 1) * kBuf;
    const int w_at = ((4 * fh + s) ^ slot_key(fr)) * 16, x_at = kX == kE4m3 ? ((2 * s + fh) ^ slot_key(fr)) * 16 : w_at;
#pragma unroll
    for (int i = 0; i < kTM; ++i) {
      const char* row = buf + (xs0 + i * 32 + fr) * kLine + x_at;
      f.x[i].v[0] = *reinterpret_cast<const uint4*>(row);
      if constexpr (kX == kE4m3) f.x[i].v[1] = *reinterpret_cast<const uint4*>(row + kBM * kLine);
    }
#pragma unroll
    for (int j = 0; j < kTN; ++j)
      f.w[j].v[0] = *reinterpret_cast<const uint4*>(buf + kXBytes + (ws0 + j * 32 + fr) * kLine + w_at);
  };
  // One 16-byte load per lane of a k-tile on its way, and its place in LDS.
  uint4 part[kParts];
  auto request = [&](int kt, int i, auto inside) {   // inside: a whole k-tile
    const bool is_x = i < kA;
    // rows, and for x lines, from the tile's first on
    const uint32_t line = is_x ? (uint32_t)(i * kLoadLines / kBM * kLine) : 0u;
    const uint32_t row = is_x ? (uint32_t)(i * kLoadLines % kBM) * (uint32_t)x_row : (uint32_t)((i - kA) * kLoadLines) * (uint32_t)w_row;
    const uint32_t at = (uint32_t)kt * (uint32_t)(is_x ? kXL * kLine : kLine) + line;
    uint32_t off = is_x ? x_off : w_off;
    if constexpr (!decltype(inside)::value) off = at + chunk * 16 < (uint32_t)(is_x ? x_row : w_row) ? off : kNowhere;
    part[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(is_x ? x_tile : w_tile, (int)off, (int)(row + at), 0));
  };
  auto put = [&](int kt, int i) {
    char* buf = lds + (kt & 1) * kBuf + tid * 16;
    *reinterpret_cast<uint4*>(buf + (i < kA ? 0 : kXBytes) + (i < kA ? i : i - kA) * kThreads * 16) = part[i];
  };
  // Step s of k-tile kt forms the products of 64 values.  Meanwhile the next step's fragments are read, over the
  // k-tiles' borders too, and the next k-tile moves from registers to the other buffer, a part per step, each part's
  // registers taking the k-tile after it.
  constexpr int kSteps = 4, kPerStep = (kParts + kSteps - 2) / (kSteps - 1);
  Frags f[2];
  Scales sc[2];
  auto begin = [&](auto inside) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) request(0, i, inside);
    read_scales(0, sc[0]);
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
    const Scales now = sc[0];
    auto step = [&](auto s_) {
      constexpr int s = decltype(s_)::value;
      if (s + 1 < kSteps) {
        read(kt, s + 1, f[(s + 1) & 1]);
      } else if (kInside || kt + 1 < ktiles) {
        __syncthreads();   // the next buffer is written, this one read
        read(kt + 1, 0, f[0]);
      }
      if (s == 0 && (kInside || kt + 1 < ktiles)) read_scales(kt + 1, sc[0]);
#pragma unroll
      for (int j = 0; j < kTN; ++j) {
#pragma unroll
        for (int i = 0; i < kTM; ++i)
          acc[j][i] = mma32<kX, s>(f[s & 1].w[j], now.w[j], f[s & 1].x[i], now.x[i], acc[j][i]);
        // the compiler would otherwise gather the loads at the end of the k-tile
        __builtin_amdgcn_sched_barrier(0);
        if (j == 0 && s + 1 < kSteps && (kInside || kt + 1 < ktiles)) {
#pragma unroll
          for (int e = 0; e < kPerStep; ++e) {
            const int i = s * kPerStep + e;
            if (i < kParts) {
              put(kt + 1, i);
              if (kInside || kt + 2 < ktiles) request(kt + 2, i, inside);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    step(std::integral_constant<int, 0>());
    step(std::integral_constant<int, 1>());
    step(std::integral_constant<int, 2>());
    step(std::integral_constant<int, 3>());
  };
  const int whole = (int)(a.blocks / kTileBlocks);   // k-tiles
  int kt = 0;
  if (whole > 2) {
    begin(std::true_type());
    for (; kt + 2 < whole; ++kt) k_tile(kt, std::true_type());
  } else {
    begin(std::false_type());
  }
  for (; kt < ktiles; ++kt) {
    if (kt >= whole) cut_scales(kt, sc[0]);
    k_tile(kt, std::false_type());
  }
  __syncthreads();

  // a lane holds row fr of the 32 x 32 block, columns 8 q + 4 fh + (0..3); on the way out it has eight columns
  float* out = reinterpret_cast<float*>(lds) + wave * 32 * kOutRow;
  const int64_t wm0 = m0 + wm * kTM * 32, wn0 = n0 + wn * kTN * 32;
  constexpr int kPer = kTN * 32 / kVec;    // vectors of a row on the way out
  static_assert(64 % kPer == 0, "a lane has the same columns in every row");
  const int oc = lane % kPer * kVec;
  const int64_t cc = wn0 + oc;
  const int cn = cc >= a.n ? 0 : (a.n - cc < kVec ? (int)(a.n - cc) : kVec);
  float bias[kVec] = {};
  if (a.bias && cn > 0) load_vec<float>(a.bias + cc, cn, bias);
#pragma unroll
  for (int i = 0; i < kTM; ++i) {
#pragma unroll
    for (int j = 0; j < kTN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(out + fr * kOutRow + j * 32 + 8 * q + 4 * fh) =
            make_float4(acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]);
    // the wave's own rows: no other wave reads or writes them
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int k = 0; k < 32 * kPer / 64; ++k) {
      const int r = (k * 64 + lane) / kPer;
      const int64_t mm = wm0 + i * 32 + r;
      float v[kVec];
      const float4 lo = *reinterpret_cast<const float4*>(out + r * kOutRow + oc);
      const float4 hi = *reinterpret_cast<const float4*>(out + r * kOutRow + oc + 4);
      v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
      v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
      if (mm < a.m && cn > 0) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = activate(v[e] + bias[e], a.act);
        finish(a, mm, cc, cn, v);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// 16 rows of w by kMT x 16 rows of x per workgroup of kWaves waves.
template <int kX, int kMT, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void mx_rows(LinearMx a, int64_t first) {
  constexpr int kXL = kX == kE4m3 ? 2 : 1;
  __shared__ float part[kWaves][kMT][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t n0 = (first + blockIdx.x) * 16;
  const int lines = (int)((a.blocks + kTileBlocks - 1) / kTileBlocks);
  const int fr = lane & 15, fg = lane >> 4;
  const int64_t n = n0 + fr < a.n ? n0 + fr : a.n - 1;
  const uint8_t *wrow = a.w + n * a.blocks * 16, *wsrow = a.ws + n * a.blocks;
  const uint8_t *xrow[kMT], *xsrow[kMT];
#pragma unroll
  for (int i = 0; i < kMT; ++i) {
    const int64_t m = i * 16 + fr < a.m ? i * 16 + fr : a.m - 1;
    xrow[i] = a.x + m * a.blocks * (16 * kXL);
    xsrow[i] = a.xs + m * a.blocks;
  }
  v4f acc[kMT] = {};
  // In step s lane group g has block 2 g + s of the line; of e4m3 it holds half g % 2 of blocks 2 (g / 2) + s and
  // 2 (2 + g / 2) + s.
  auto line = [&](int l, auto inside) {
    constexpr bool kInside = decltype(inside)::value;   // eight whole blocks
    const int64_t b0 = (int64_t)l * kTileBlocks;
    auto get = [&](const uint8_t* row, int64_t block, int bytes, int half) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (kInside || block < a.blocks) __builtin_memcpy(&v, row + block * bytes + half * 16, 16);
      return v;
    };
    Part<kE2m1> w[2];
    Part<kX> x[2][kMT];
    uint32_t ws, xs[kMT];
#pragma unroll
    for (int s = 0; s < 2; ++s) w[s].v[0] = get(wrow, b0 + 2 * fg + s, 16, 0);
    if constexpr (kInside) {
      uint16_t t;
      __builtin_memcpy(&t, wsrow + b0 + 2 * fg, 2);
      ws = t;
    } else {
      ws = scale_word<2>(wsrow, b0 + 2 * fg, a.blocks);
    }
#pragma unroll
    for (int i = 0; i < kMT; ++i) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if constexpr (kX == kE4m3) {
          x[s][i].v[0] = get(xrow[i], b0 + 2 * (fg / 2) + s, 32, fg & 1);
          x[s][i].v[1] = get(xrow[i], b0 + 2 * (2 + fg / 2) + s, 32, fg & 1);
        } else {
          x[s][i].v[0] = get(xrow[i], b0 + 2 * fg + s, 16, 0);
        }
      }
      xs[i] = scale_word<2>(xsrow[i], b0 + 2 * fg, a.blocks);
    }
#pragma unroll
    for (int i = 0; i < kMT; ++i) {
      acc[i] = mma16<kX, 0>(w[0], ws, x[0][i], xs[i], acc[i]);
      acc[i] = mma16<kX, 1>(w[1], ws, x[1][i], xs[i], acc[i]);
    }
  };
  const int whole = (int)(a.blocks / kTileBlocks);
  int l = wave;
  for (; l < whole; l += kWaves) line(l, std::true_type());
  if (l < lines) line(l, std::false_type());
  // a lane holds row fr of x, columns 4 fg + (0..3)
#pragma unroll
  for (int i = 0; i < kMT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][i][fr * 16 + fg * 4 + e] = acc[i][e];
  __syncthreads();
  for (int o = tid; o < kMT * 256; o += 64 * kWaves) {
    const int tile = o >> 8, r = (o >> 4) & 15, c = o & 15;
    const int64_t m = tile * 16 + r, nn = n0 + c;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += part[w][tile][o & 255];
    if (m >= a.m || nn >= a.n) continue;
    if (a.bias) v += a.bias[nn];
    v = activate(v, a.act);
    auto put = [&](auto zero) {
      typedef decltype(zero) Out;
      if (a.residual) v += (float)static_cast<const Out*>(a.residual)[m * a.residual_row + nn];
      static_cast<Out*>(a.y)[m * a.y_row + nn] = (Out)v;
    };
    switch (a.out_dtype) {
      case SSDI8_F32: put(0.0f); break;
      case SSDI8_F16: put((_Float16)0.0f); break;
      default: put((bf16)0.0f);
    }
  }
}

template <int kX, int kBM, int kBN, int kWM, int kWN> hipError_t run_tile(const LinearMx& a, hipStream_t st) {
  const int64_t mt = (a.m + kBM - 1) / kBM, nt = (a.n + kBN - 1) / kBN;
  return in_parts(mt * nt, 64 * kWM * kWN, [&](int64_t first, dim3 grid) {
    mx_tile<kX, kBM, kBN, kWM, kWN><<<grid, 64 * kWM * kWN, 0, st>>>(a, (int)mt, (int)nt, (int)first);
  });
}

template <int kX> hipError_t by_tiles(const LinearMx& a, hipStream_t st) {
  auto count = [&](int64_t bm, int64_t bn) { return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn); };
  // Small tiles where large ones leave CUs without work: us with 64 x 64 / 128 x 128 e2m1 512 x 5120 x 2560 12.4 / 12.6,
  // 1000 x 2900 x 992 11.1 / 11.9, 2048 x 2560 x 5120 43.5 / 39.4; e4m3 with 128 x 256 15.0 / 22.6, 12.1 / 17.6, 50.3 / 43.8.
  if constexpr (kX == kE4m3) {
    if (count(128, 256) < 128) return run_tile<kX, 64, 64, 2, 2>(a, st);
    return run_tile<kX, 128, 256, 2, 4>(a, st);
  } else {
    if (count(128, 128) < 256) return run_tile<kX, 64, 64, 2, 2>(a, st);
    // Eight waves where a tile's way out is much of its time, four (more products per value read from LDS) over a long k.
    // us with eight / four: 16384 x 768 of k 1024 22 / 25, 2560 32 / 36, 3584 42 / 44, 4096 54 / 48, 5120 68 / 56; 16384 x 2560
    // of 1024 55 / 60, 2560 95 / 98, 3584 130 / 123, 4096 165 / 141, 8192 318 / 261; 4096 x 4096 of 3584 54 / 55, 4096 71 / 62;
    // 16384 x 10496 x 2560 382 / 372.
    if (a.blocks >= 128) return run_tile<kX, 128, 128, 2, 2>(a, st);
    return run_tile<kX, 128, 128, 2, 4>(a, st);
  }
}

template <int kX> hipError_t run(const LinearMx& a, hipStream_t st) {
  // us up to 32 rows, with mx_rows / 64 x 64 tiles, e4m3 x: 16 x 10496 x 2560 8.0 / 7.6, 16 x 2560 x 5120 6.7 / 11.7, 32 x
  // 1024 x 8192 13.6 / 17.1, 32 x 768 x 1536 4.3 / 6.3; against it, many outputs: 32 x 10496 x 2560 12.0 / 8.1.
  if (a.m > 32) return by_tiles<kX>(a, st);
  return in_parts((a.n + 15) / 16, 512, [&](int64_t first, dim3 grid) {
    if (a.m <= 16) mx_rows<kX, 1, 8><<<grid, 512, 0, st>>>(a, first);
    else mx_rows<kX, 2, 8><<<grid, 512, 0, st>>>(a, first);
  });
}

}  // namespace

hipError_t launch_linear_mx(const LinearMx& a, hipStream_t st) {
  return a.format == SSDI8_FMT_MXFP8 ? run<kE4m3>(a, st) : run<kE2m1>(a, st);
}

}  // namespace ssdi8
