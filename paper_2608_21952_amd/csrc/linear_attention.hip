// Linear attention with a decay per head:
//   S_t = exp(g_t) S_{t-1} + k_t v_t^T,   y_t = scale S_t^T q_t          (S: keys x values, fp32)
// over chunks of C tokens, c_i the sum of g over the chunk's tokens up to i:
//   y_i = scale (exp(c_i) S_0^T q_i + sum_{j <= i} exp(c_i - c_j) (q_i . k_j) v_j)
//   S_C = exp(c_C) S_0 + sum_j exp(c_C - c_j) k_j v_j^T
// A workgroup of four waves walks the chunks of a head (of a span of it), each wave with its own columns of S, v and
// y; q, k and v of a chunk lie in LDS, the next chunk's are on their way in registers.
//
// Matrix products: the 16 x 16 instructions take eight values of a row per lane, for 32 along the sum (fp32: eight
// instructions of four).  A lane group g (of 16 lanes) has rows 4 g + (0..3) of a result tile, so the eight places of its
// part of an operand are given to its rows of two tiles: results become operands where they lie.  Of p, these are
// tokens 4 g + (0..3) and 16 + 4 g + (0..3); of S (keys x values, the operand of S^T q) the keys of two tiles are dealt
// out so that they are keys 8 g + (0..7), the ones that a read of 16 bytes of q gives.
//
// Roundings, of 16-bit types: p and S are rounded once on their way into the products for y, which adds to y's error
// about as much as its own rounding (0.00029 against 0.00021 of y, fp16): as two values each a call takes 316 us
// instead of 292 (4 x 4096 tokens of 80 heads, fp16), 221 instead of 207 (4 x 8192 of 16 heads, bf16).  fp16: p per row
// and S per column are brought to the top of the type's range by powers of two.  exp(c_C - c_j) v_j, which would leave its
// rounding in S with every chunk, enters as the sum of three bf16 values (two would be 2^-17 off), of fp16 too: two fp16
// values, brought into range by a power of two per column, lose what decays within a chunk have made small, though a key
// that is 0 for the later tokens has nothing else.  k of fp16 enters as two bf16 values then, five products in all: 4 x
// 4096 tokens of 80 heads 292 us, 232 in bf16, whose k is one value.
// Sums, S, and the decays' sums (these in fp64: differences of far sums) are not rounded.
// A value of v that is no number would reach earlier tokens of its chunk through 0 times it: it enters as 0, and its
// column is NaN from its token on.
//
// What bounds it: of a chunk's 9 us with two workgroups on a CU (fp16) the products take 3; the rest is LDS reads of the
// operands, S's conversion for every chunk, and the barriers between the phases.  Two heads that share q and k read them once.
// 4 x 4096 tokens, 80 heads of 64 with shared q and k of 128, fp16: 185 us, with the spans' states 94 and their join 12
// beside them (1.2 TB/s in all); 4 x 8192, 16 heads of 128 x 128, bf16: 123 + 69 + 14; 16384 of 8 heads of 64 x 128, fp32:
// 71 + 36 + 10.
#include <type_traits>
#include <utility>

#include "attention.hpp"
#include "block.hpp"
#include "common.hpp"
#include "ssdi8.h"

namespace ssdi8 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr double kLog2e = 1.4426950408889634074;

template <typename T> struct Frag {
  T v[8];
};
template <typename T> __device__ __forceinline__ v4f mma(const Frag<T>& a, const Frag<T>& b, v4f c) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
  } else if constexpr (std::is_same_v<T, bf16>) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
}
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef bf16 v2b __attribute__((ext_vector_type(2)));
template <typename T> struct TwoOf { typedef v2h type; };
template <> struct TwoOf<bf16> { typedef v2b type; };

// Eight values as a fragment, rounded to the type.
template <typename T> __device__ __forceinline__ Frag<T> round_frag(const float (&f)[8]) {
  Frag<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = f[e];
  } else {
    typedef typename TwoOf<T>::type Two;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const Two t = __builtin_convertvector(v2f{f[e], f[e + 1]}, Two);
      __builtin_memcpy(&r.v[e], &t, 4);
    }
  }
  return r;
}
// What that leaves of them, in their place.
template <typename T> __device__ __forceinline__ void take_off(float (&f)[8], const Frag<T>& hi) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] -= (float)hi.v[e];
}

// fp16: the exponent shift that brings values of which the largest has magnitude bits `big` (fp32) to where that lies in
// [2^14, 2^15), at most kMost; none for 0 and for what is no number.  Below fp16's normal range values are off by 2^-25:
// by 2^-39 of the largest, as long as that is 2^(14 - kMost) or more.
template <int kMost> __device__ __forceinline__ int range_shift(uint32_t big) {
  const int e = (int)(big >> 23);
  if (e == 0 || e == 255) return 0;
  const int s = 127 + 14 - e;
  return s > kMost ? kMost : s;
}
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
__device__ __forceinline__ uint32_t bits_max(uint32_t a, float v) {
  const uint32_t m = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
  return a > m ? a : m;
}
// The largest over the four lane groups, in each of them.
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = a[0] > a[1] ? a[0] : a[1];
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return b[0] > b[1] ? b[0] : b[1];
}
// The value of one lane, in scalar registers.
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// Sums over the lanes up to each.
__device__ __forceinline__ double wave_scan(double v) {
  v = dpp_add_f64<0x111, 0xf>(v);   // 1, 2, 4 and 8 lanes to the left within 16
  v = dpp_add_f64<0x112, 0xf>(v);
  v = dpp_add_f64<0x114, 0xf>(v);
  v = dpp_add_f64<0x118, 0xf>(v);
  v = dpp_add_f64<0x142, 0xa>(v);   // the last lane of a row of 16 into the next row, of 32 into the next half
  return dpp_add_f64<0x143, 0xc>(v);
}

// Eight values of an LDS row.
template <typename T> __device__ __forceinline__ Frag<T> row_frag(const T* p) {
  Frag<T> f;
  __builtin_memcpy(&f, __builtin_assume_aligned(p, 16), sizeof(f));
  return f;
}
// Of 16 columns of 32 LDS rows the lane's column, rows [4 g, 4 g + 4) and 16 further on.  at(row, c): where values
// 4 c .. 4 c + 3 of a row's 16 columns are.
template <typename T, typename At> __device__ __forceinline__ Frag<T> column_frag(const T* p, int lane, At at) {
  Frag<T> f;
  const int g = lane >> 4, m = lane & 15;
  if constexpr (sizeof(T) == 2) {
    // the four values that lane m of a group points at are a quarter of row m / 4 of a 4 x 16 block, which the
    // instruction hands out by columns
    typedef __attribute__((address_space(3))) v4s* Lds;
    T* q = const_cast<T*>(p);
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(q + at(4 * g + m / 4, m % 4)));
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(q + at(16 + 4 * g + m / 4, m % 4)));
    __builtin_memcpy(&f.v[0], &a, 8);
    __builtin_memcpy(&f.v[4], &b, 8);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = p[at(4 * g + e % 4 + e / 4 * 16, m / 4) + m % 4];
  }
  return f;
}

// Eight fp16 values as two bf16 each, which hold their 11 bits.
__device__ __forceinline__ void split_halves(const Frag<_Float16>& k, bf16* hi, bf16* lo) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (float)k.v[e];
  const Frag<bf16> h = round_frag<bf16>(f);
  take_off(f, h);
  const Frag<bf16> l = round_frag<bf16>(f);
  __builtin_memcpy(__builtin_assume_aligned(hi, 16), &h, 16);
  __builtin_memcpy(__builtin_assume_aligned(lo, 16), &l, 16);
}

// f(0), f(1) and so on, the numbers as types.
template <int... i, typename F> __device__ __forceinline__ void each_of(std::integer_sequence<int, i...>, F f) {
  (f(std::integral_constant<int, i>()), ...);
}

// A condition whose code is to lie out of the way.
__device__ __forceinline__ bool rarely(bool v) { return __builtin_expect(v, 0); }

struct Args {
  LinearAttention a;
  int slices, spans, chunks, span_chunks;   // column slices of a head; spans of the tokens and their chunks
  int groups;                               // of heads: those that a workgroup takes together
  float* final_state;
  int64_t first;                            // of the launch's workgroups
};

__device__ __host__ __forceinline__ int64_t state_floats(const LinearAttention& a) { return a.keys * a.values; }

// Memory from p on for loads and stores with offsets of less than 2^31 bytes; at kNowhere loads give 0 and stores do
// nothing, so that what is not there needs no branch.
constexpr uint32_t kNowhere = 0xfffffff0u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x80000000u, 0x00027000);
}

// A tile of rows on its way from memory to LDS: kRows rows of kWidth values (`width` of every kPart there, the parts
// `part` elements apart), by 256 threads in vectors of 16 bytes.  Offsets within the tile are of 32 bits (the host
// refuses tokens too far apart for them).
template <typename T, int kRows, int kWidth, int kPart> struct Stage {
  static constexpr int kPer = 16 / (int)sizeof(T), kVecs = kWidth / kPer, kStep = 256 / kVecs;
  static constexpr int kEach = kRows / kStep;
  static_assert(kRows % kStep == 0 && 256 % kVecs == 0 && kPart % kPer == 0, "stage");
  uint4 v[kEach];
  static __device__ __forceinline__ int column(int tid) { return tid % kVecs * kPer; }
  static __device__ __forceinline__ uint32_t offset(int64_t token_stride, int64_t part, int tid) {
    const int c = column(tid);
    return (uint32_t)((tid / kVecs * token_stride + (kPart < kWidth ? c / kPart * part : 0) + c % kPart) * sizeof(T));
  }
  // step: bytes from a load's rows to the next one's
  __device__ __forceinline__ void load(const char* base, uint32_t off, uint32_t step, int tokens, int width, int tid) {
    const int in = column(tid) % kPart, row0 = tid / kVecs;
    const auto tile = buffer_of(base);
    if (!rarely(tokens < kRows || width < kPart)) {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        v[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(
                                             tile, (int)off, (int)(i * step), 0));
      return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t at = i * kStep + row0 < tokens && in + kPer <= width ? off : kNowhere;
      const auto d = __builtin_amdgcn_raw_buffer_load_b128(tile, (int)at, (int)(i * step), 0);
      v[i] = __builtin_bit_cast(uint4, d);
    }
    if (!rarely(width % kPer != 0)) return;
    // the row's last vector, value by value
    if (in >= width || in + kPer <= width) return;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (i * kStep + row0 >= tokens) continue;
      uint64_t half[2] = {0, 0};
#pragma unroll 1
      for (int j = 0; j < width - in; ++j) {
        const int at = (int)(off + j * (uint32_t)sizeof(T)), row = (int)(i * step);
        uint64_t e;
        if constexpr (sizeof(T) == 2) e = __builtin_amdgcn_raw_buffer_load_b16(tile, at, row, 0);
        else e = __builtin_amdgcn_raw_buffer_load_b32(tile, at, row, 0);
        e <<= 8 * sizeof(T) * (j % (kPer / 2));
        half[0] |= j < kPer / 2 ? e : 0;
        half[1] |= j < kPer / 2 ? 0 : e;
      }
      __builtin_memcpy(&v[i], half, 16);
    }
  }
  template <typename At> __device__ __forceinline__ void put(T* lds, int tid, At at) const {   // at(row, column)
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      *reinterpret_cast<uint4*>(lds + at(i * kStep + tid / kVecs, column(tid))) = v[i];
  }
  // fp16: each value as two of bf16 that add up to it, at the same places of hi and lo.
  template <typename At> __device__ __forceinline__ void put_halves(bf16* hi, bf16* lo, int tid, At at) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int o = at(i * kStep + tid / kVecs, column(tid));
      split_halves(__builtin_bit_cast(Frag<_Float16>, v[i]), hi + o, lo + o);
    }
  }
};

// The magnitude bits of a fragment's largest value (as those of the type), 16-bit types.
__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
  typedef unsigned short v2u __attribute__((ext_vector_type(2)));
  const v2u x = __builtin_bit_cast(v2u, a), y = __builtin_bit_cast(v2u, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}
template <typename T> __device__ __forceinline__ uint32_t largest(const Frag<T>& f, uint32_t big) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) big = bits_max(big, f.v[e]);
  } else {
    uint32_t w[4];
    __builtin_memcpy(w, f.v, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) big = pk_max_u16(big, w[i] & 0x7fff7fffu);
  }
  return big;
}

// kKeys: keys filled up to 64, 128 or 256.  kHeads (1 or 2) heads of y that share q and k, each with 4 / kHeads waves of
// kTiles tiles of 16 columns.  kC: tokens of a chunk.  kOut: the walk with outputs; else the one for the states at
// the spans' ends.
template <typename T, int kKeys, int kTiles, int kHeads, int kC, bool kOut>
__global__ __launch_bounds__(256, kKeys > 128 ? 1 : 2) void attention_kernel(Args p) {
  const LinearAttention& a = p.a;
  constexpr bool kHalf = sizeof(T) == 2, kF16 = std::is_same_v<T, _Float16>;
  constexpr int kWH = 4 / kHeads, kSlice = 16 * kTiles * kWH;   // waves of a head, its columns in a workgroup
  constexpr int kSums = kC / 32, kRowsT = kC / 16, kKeyT = kKeys / 16, kKeyS = kKeys / 32;
  // v is read by four rows of 32 bytes: 8 banks from row to row.  Of q and k 16 rows at one chunk of 16 bytes are read
  // (lanes 0-3, 12-15 and 20-27 of 32 at a time), of k four rows at four chunks, too: chunks are exchanged so that
  // these lie in different banks.
  constexpr int kPerChunk = 16 / (int)sizeof(T), kV = kSlice * kHeads + 2 * kPerChunk;
  auto v_at = [](int row, int col) { return row * kV + col; };
  auto k_at = [](int row, int key) {
    constexpr int kChunks = kKeys / kPerChunk;
    const int quad = row / 4 % 4, low = ((quad ^ (quad >> 1)) & 1) * 2 + (quad >> 1);   // 0, 2, 3, 1
    const int f = (kChunks >= 16 ? row % 4 * 4 : row / 2 % 2 * 4) + low;
    // fp32: whole pairs of chunks
    return row * kKeys + ((key / kPerChunk) ^ (kHalf ? f : 2 * f % 16)) * kPerChunk + key % kPerChunk;
  };
  constexpr int kPairs = kRowsT * (kRowsT / 2 + 1) / 2;     // (row tile, 32 tokens) of p that are not 0
  constexpr int kOutSize = kC * kSlice * kHeads;             // of y's tile, which takes the place of q
  __shared__ __attribute__((aligned(16))) T q_lds[kOut ? (kC * kKeys > kOutSize ? kC * kKeys : kOutSize) : 8];
  __shared__ __attribute__((aligned(16))) T k_lds[kC * kKeys];
  // k as bf16 (fp16): with outputs its first values take its own place when p is there, the second ones that of v,
  // which all waves have in registers then
  constexpr int kVSize = kF16 && kOut && kC * kKeys > kC * kV ? kC * kKeys : kC * kV;
  __shared__ __attribute__((aligned(16))) T v_lds[kVSize];
  __shared__ __attribute__((aligned(16))) T rest_lds[kF16 && !kOut ? kC * kKeys : 8];
  bf16 *k_hi = reinterpret_cast<bf16*>(k_lds), *k_lo = reinterpret_cast<bf16*>(kOut ? v_lds : rest_lds);
  __shared__ __attribute__((aligned(16))) Frag<T> p_lds[kHeads][kOut ? kPairs * 64 : 1];
  __shared__ __attribute__((aligned(16))) double c_all[kHeads][kC];
  __shared__ __attribute__((aligned(16))) float w_all[kHeads][kC], e_all[kHeads][kC], row_all[kHeads][kC];
  __shared__ __attribute__((aligned(16))) float b_all[kHeads][kWH][kC];

  const int tid = threadIdx.x, lane = tid & 63, lane_g = lane >> 4, lane_m = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // the same in all lanes: branches by it are scalar
  const int sub = kHeads > 1 ? wave / kWH : 0, hw = wave % kWH;   // head of the workgroup, wave of the head
  double* c_lds = c_all[sub];
  float *w_lds = w_all[sub], *e_lds = e_all[sub], *row_scale = row_all[sub], *b_lds = b_all[sub][hw];
  int id = (int)p.first + xcd_remap(blockIdx.x, gridDim.x);
  const int slice = id % p.slices;
  id /= p.slices;
  // heads are neighbours: those that share q and k share an XCD's cache
  const int heads = (int)(kOut ? a.heads : a.v_heads);
  const int h0 = id % p.groups * kHeads, h = h0 + sub;
  id /= p.groups;
  const int span = id % (kOut ? p.spans : p.spans - 1);
  const int64_t b = id / (kOut ? p.spans : p.spans - 1);
  const int hq = (int)(h0 * a.q_heads / heads), hv0 = (int)(h0 * a.v_heads / heads), hv = hv0 + sub;
  const int hk = (int)(hv0 * a.k_heads / a.v_heads);
  const int col0 = slice * kSlice;
  const int cols = (int)(a.values - col0 < kSlice ? a.values - col0 : kSlice);
  const int keys = (int)a.keys;

  const T* qp = static_cast<const T*>(a.q) + b * a.qs.batch + hq * a.qs.head;
  const T* kp = static_cast<const T*>(a.k) + b * a.ks.batch + hk * a.ks.head;
  const T* vp = static_cast<const T*>(a.v) + b * a.vs.batch + hv0 * a.vs.head + col0;
  int64_t end = a.seqlen;
  if (a.lengths) {
    const int64_t n = a.lengths[b];
    end = n < 0 ? 0 : n < end ? n : end;
  }
  const int chunk0 = span * p.span_chunks;
  const int chunk1 = chunk0 + p.span_chunks < p.chunks ? chunk0 + p.span_chunks : p.chunks;
  const int live = (int)((end + kC - 1) / kC);               // chunks with tokens
  const int last = live < chunk1 ? live : chunk1;

  // The state: keys key_of(t, g) + (0..3) of key tile t, column m of column tile n.  The keys of two tiles are dealt
  // out so that a lane's eight rows of them are eight neighbouring keys: those of its part of q.
  auto key_of = [](int t, int quarter) { return t / 2 * 32 + 8 * quarter + t % 2 * 4; };
  const int my0 = hw * kTiles * 16;
  const int64_t states = a.batch * a.v_heads * state_floats(a);
  v4f S[kKeyT][kTiles];
  {
    const float* from = a.init ? a.init + (b * a.v_heads + hv) * state_floats(a) : nullptr;
    if (kOut && span > 0) from = a.workspace + (span - 1) * states + (b * a.v_heads + hv) * state_floats(a);
    if (!kOut) from = nullptr;
#pragma unroll
    for (int t = 0; t < kKeyT; ++t)
#pragma unroll
      for (int n = 0; n < kTiles; ++n) S[t][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    if (from) {
      from += col0 + my0;
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
        if (my0 + 16 * n + lane_m < cols) {
#pragma unroll
          for (int t = 0; t < kKeyT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (key_of(t, lane_g) + r < keys)
                S[t][n][r] = from[(int64_t)(key_of(t, lane_g) + r) * a.values + 16 * n + lane_m];
        }
    }
  }
  double total = 0.0;   // of the decays' logarithms (base 2) over the span

  typedef Stage<T, kC, kKeys, kKeys> KeyStage;
  typedef Stage<T, kC, kSlice * kHeads, kSlice> ValueStage;
  KeyStage q_next, k_next;
  ValueStage v_next;
  // Where the next chunk to be loaded and the next one to be stored begin, and steps in bytes: running values, as the
  // products with the strides and their way from the arguments took as long as a chunk's matrix products.
  const int64_t t_first = (int64_t)chunk0 * kC;
  const char *q_from = reinterpret_cast<const char*>(qp + t_first * a.qs.token),
             *k_from = reinterpret_cast<const char*>(kp + t_first * a.ks.token),
             *v_from = reinterpret_cast<const char*>(vp + t_first * a.vs.token);
  const uint32_t q_row = (uint32_t)(a.qs.token * sizeof(T)), k_row = (uint32_t)(a.ks.token * sizeof(T)),
                 v_row = (uint32_t)(a.vs.token * sizeof(T)), y_row = (uint32_t)(a.heads * a.values * sizeof(T));
  char* y_to = reinterpret_cast<char*>(static_cast<T*>(a.y) + ((b * a.seqlen + t_first) * a.heads + h) * a.values + col0 + my0);
  const float* g_from = !a.log_decay ? nullptr
                        : a.token_decay ? a.log_decay + b * a.g_batch + t_first * a.g_token + hv : a.log_decay + hv;
  const int64_t g_row = a.log_decay && a.token_decay ? a.g_token : 0;
  const uint32_t q_off = KeyStage::offset(a.qs.token, 0, tid), k_off = KeyStage::offset(a.ks.token, 0, tid);
  const uint32_t v_off = ValueStage::offset(a.vs.token, a.vs.head, tid);
  float g_next = 0.0f;
  // The chunk behind the one requested last, in three pieces.
  auto request = [&](int chunk, int piece) {
    const int64_t t0 = (int64_t)chunk * kC;
    const int tokens = (int)(end - t0 < kC ? end - t0 : kC);
    if (piece == 0) {
      g_next = 0.0f;
      if (g_from && lane < tokens) g_next = g_from[lane * g_row];
      if (g_from) g_from += kC * g_row;
      k_next.load(k_from, k_off, KeyStage::kStep * k_row, tokens, keys, tid);
      k_from += (int64_t)kC * k_row;
    } else if (piece == 1) {
      v_next.load(v_from, v_off, ValueStage::kStep * v_row, tokens, cols, tid);
      v_from += (int64_t)kC * v_row;
    } else if constexpr (kOut) {
      q_next.load(q_from, q_off, KeyStage::kStep * q_row, tokens, keys, tid);
      q_from += (int64_t)kC * q_row;
    }
  };

  if (chunk0 < last) {
    request(chunk0, 0);
    request(chunk0, 1);
    request(chunk0, 2);
  }
  for (int chunk = chunk0; chunk < last; ++chunk) {
    // The lane's places are formed anew for every chunk: kept over all of them, places and constants took up so many
    // registers that 50 went to memory, where their way back waits for the loads in flight.
    int g = lane_g, m = lane_m;
    asm volatile("" : "+v"(g), "+v"(m));
    g &= 3, m &= 15;   // their ranges, for the arithmetic of places
    const int lane = g * 16 + m;
    __syncthreads();   // the last chunk is read
    if constexpr (kOut) q_next.put(q_lds, tid, k_at);
    if constexpr (kF16 && !kOut) k_next.put_halves(k_hi, k_lo, tid, k_at);
    else k_next.put(k_lds, tid, k_at);
    v_next.put(v_lds, tid, v_at);
    // sums of the decays' logarithms, in base 2; below 2^-65536 is 0 all the same, and an infinite one would leave
    // no differences behind it
    double c = g_next < -65536.0f ? -65536.0 * kLog2e : (double)g_next * kLog2e;
    c = wave_scan(c);
    const double c_end = lane_value(c, kC - 1);
    if (hw == 0 && lane < kC) {
      c_lds[lane] = c;
      w_lds[lane] = __builtin_amdgcn_exp2f((float)(c_end - c));
      if constexpr (kOut) e_lds[lane] = a.scale * __builtin_amdgcn_exp2f((float)c);
    }
    __syncthreads();

    const int64_t t0 = (int64_t)chunk * kC;
    // v, 0 where its values are no numbers
    Frag<T> vf[kSums][kTiles];
    int first[kTiles];   // the first token of the column whose value is no number
    constexpr uint32_t kNoNumber = kF16 ? 0x7c00u : kHalf ? 0x7f80u : 0x7f800000u;
    bool odd = false;
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      first[n] = kC;
      uint32_t big = 0;
#pragma unroll
      for (int s = 0; s < kSums; ++s) {
        vf[s][n] = column_frag(v_lds + 32 * s * kV + sub * kSlice + my0 + 16 * n, lane,
                               [&](int row, int c) { return v_at(row, 4 * c); });
        big = largest(vf[s][n], big);
      }
      odd |= (!kHalf ? big : (big & 0xffffu) > (big >> 16) ? big & 0xffffu : big >> 16) >= kNoNumber;
    }
    const bool any_bad = __any(odd) != 0;
    if (rarely(any_bad)) {
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
#pragma unroll
        for (int s = 0; s < kSums; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!(__builtin_fabsf((float)vf[s][n].v[e]) < __builtin_inff())) {
              const int j = 32 * s + 16 * (e / 4) + 4 * g + e % 4;
              first[n] = j < first[n] ? j : first[n];
              vf[s][n].v[e] = (T)0.0f;
            }
#pragma unroll
        for (int d = 16; d < 64; d *= 2) {
          const int o = __shfl_xor(first[n], d);
          first[n] = o < first[n] ? o : first[n];
        }
      }
    }

    if constexpr (kOut) {
      // Priorities rise over a chunk: of two workgroups of a CU, which else go through their phases side by side and
      // share the matrix unit in one and leave it idle in the next, the one that is further on goes first (4 x 4096
      // tokens of 80 heads, fp16: 314 us without, 292 with).
      __builtin_amdgcn_s_setprio(1);
      // p^T: rows j, column i = m of row tile it; the waves of a head take one from each end of them in turn
#pragma unroll
      for (int u = 0; u < (kRowsT + kWH - 1) / kWH; ++u) {
        const int it = u % 2 == 0 ? u * kWH + hw : (u + 1) * kWH - 1 - hw;
        if (it >= kRowsT) continue;
        const int i = it * 16 + m;
        // exp(c_i - c_j) for tokens j of earlier row tiles is exp(c_i - c_x) exp(c_x - c_j), x the last of them: both
        // at most 1, the second one for all rows
        const double ci = c_lds[i], cx = c_lds[it > 0 ? it * 16 - 1 : 0];
        if (lane < kC) b_lds[lane] = __builtin_amdgcn_exp2f((float)(cx - c_lds[lane]));
        const float ai = a.scale * __builtin_amdgcn_exp2f((float)(ci - cx));
        double cj[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) cj[r] = c_lds[it * 16 + 4 * g + r];
        float wd[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) wd[r] = a.scale * __builtin_amdgcn_exp2f((float)(ci - cj[r]));
        constexpr int kAll = kRowsT;
        const int most = (u + 1) * kWH < kAll ? (u + 1) * kWH : kAll;   // tiles that any wave has in this turn
        v4f acc[kRowsT] = {};
#pragma unroll
        for (int s = 0; s < kKeyS; ++s) {
          const Frag<T> qf = row_frag(q_lds + k_at(i, 32 * s + 8 * g));
#pragma unroll
          for (int jt = 0; jt < kRowsT; ++jt)
            if (jt < most) acc[jt] = mma(row_frag(k_lds + k_at(jt * 16 + m, 32 * s + 8 * g)), qf, acc[jt]);
        }
        __builtin_amdgcn_wave_barrier();
        float big = 0.0f;
#pragma unroll
        for (int jt = 0; jt < kRowsT; ++jt) {
          if (jt >= most) continue;
          if (jt < it) {
            const float4 bj = *reinterpret_cast<const float4*>(b_lds + jt * 16 + 4 * g);
            acc[jt][0] *= bj.x * ai;
            acc[jt][1] *= bj.y * ai;
            acc[jt][2] *= bj.z * ai;
            acc[jt][3] *= bj.w * ai;
          } else {   // tokens behind the row are left out
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float v = acc[jt][r] * wd[r];
              acc[jt][r] = jt == it && 4 * g + r <= m ? v : 0.0f;
            }
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) big = __builtin_fmaxf(big, __builtin_fabsf(acc[jt][r]));
        }
        if constexpr (kF16) {
          // p below 2^-48 times 64 values is nothing to y; a row's sums stay finite where y is below 2^65
          const float by = power(range_shift<62>(group_max(__builtin_bit_cast(uint32_t, big))));
          if (g == 0) row_scale[i] = by;
#pragma unroll
          for (int jt = 0; jt < kRowsT; ++jt)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[jt][r] *= by;
        }
        const int pair0 = it / 2 * (it / 2 + 1) + it % 2 * (it / 2 + 1);
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
          if (2 * s > it) continue;
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = acc[2 * s + e / 4][e % 4];
          p_lds[sub][(pair0 + s) * 64 + lane] = round_frag<T>(f);
        }
      }
    }

    v4f acc[kOut ? kRowsT : 1][kTiles] = {};
    int s_shift[kTiles];        // of the lane's column of the state
    if constexpr (kOut) {
      // S^T q, the state rounded to the type
      __builtin_amdgcn_sched_barrier(0);   // phases stay apart: their operands do not fit the registers together
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        s_shift[n] = 0;
        if constexpr (kF16) {
          float most = 0.0f;
#pragma unroll
          for (int t = 0; t < kKeyT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(S[t][n][r]));
          s_shift[n] = range_shift<100>(group_max(__builtin_bit_cast(uint32_t, most)));
        }
      }
      Frag<T> qf[2][kRowsT];   // read a step ahead
      auto read_q = [&](int s) {
#pragma unroll
        for (int it = 0; it < kRowsT; ++it) qf[s % 2][it] = row_frag(q_lds + k_at(it * 16 + m, 32 * s + 8 * g));
      };
      read_q(0);
#pragma unroll
      for (int s = 0; s < kKeyS; ++s) {
        if (s + 1 < kKeyS) read_q(s + 1);
        Frag<T> sf[kTiles];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = kF16 ? S[2 * s + e / 4][n][e % 4] * power(s_shift[n]) : S[2 * s + e / 4][n][e % 4];
          sf[n] = round_frag<T>(f);
        }
#pragma unroll
        for (int it = 0; it < kRowsT; ++it)
#pragma unroll
          for (int n = 0; n < kTiles; ++n) acc[it][n] = mma(sf[n], qf[s % 2][it], acc[it][n]);
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();   // p is there
      if constexpr (kF16) k_next.put_halves(k_hi, k_lo, tid, k_at);
      __builtin_amdgcn_sched_barrier(0);
    }

    if constexpr (kOut) {
#pragma unroll
      for (int it = 0; it < kRowsT; ++it) {
        const int i = it * 16 + m;
        float e = e_lds[i];
        if constexpr (kF16) e *= row_scale[i];   // as p's rows are
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[it][n][r] *= e;
        }
      }
      if constexpr (kF16) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float by = power(-__shfl(s_shift[n], 4 * g + r));
#pragma unroll
            for (int it = 0; it < kRowsT; ++it) acc[it][n][r] *= by;
          }
      }
#pragma unroll
      for (int s = 0; s < kSums; ++s)
#pragma unroll
        for (int it = 2 * s; it < kRowsT; ++it) {
          const int pair0 = it / 2 * (it / 2 + 1) + it % 2 * (it / 2 + 1);
          const Frag<T> pf = p_lds[sub][(pair0 + s) * 64 + lane];
#pragma unroll
          for (int n = 0; n < kTiles; ++n) acc[it][n] = mma(vf[s][n], pf, acc[it][n]);
        }
      if constexpr (kF16) {
#pragma unroll
        for (int it = 0; it < kRowsT; ++it) {
          const float out = __builtin_amdgcn_rcpf(row_scale[it * 16 + m]);   // of a power of two: exact
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[it][n][r] *= out;
        }
      }
      if (rarely(any_bad)) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int from = __shfl(first[n], 4 * g + r);
#pragma unroll
            for (int it = 0; it < kRowsT; ++it)
              if (it * 16 + m >= from) acc[it][n][r] = __builtin_nanf("");
          }
      }
      __builtin_amdgcn_sched_barrier(0);
      // y leaves through the place of q, which all waves have read: the wave's rows in whole vectors of 16 bytes.
      // Chunk x of a row lies at x ^ (row / kPeriod): the 16 rows that are written at a time touch every bank once.
      constexpr int kChunks = kTiles * (int)sizeof(T), kPeriod = 16 / kChunks, kPer = 16 / (int)sizeof(T);
      char* out_lds = reinterpret_cast<char*>(q_lds) + wave * kC * kChunks * 16;
      const int64_t left = end - t0;
      if (rarely(left < kC)) {   // tokens behind the sequence's end: 0
#pragma unroll
        for (int it = 0; it < kRowsT; ++it)
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[it][n][r] = it * 16 + m < left ? acc[it][n][r] : 0.0f;
      }
#pragma unroll
      for (int it = 0; it < kRowsT; ++it)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          T v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = (T)acc[it][n][r];
          const int i = it * 16 + m, x = (n * 16 + 4 * g) / kPer, in = (4 * g) % kPer * (int)sizeof(T);
          __builtin_memcpy(__builtin_assume_aligned(out_lds + (i * kChunks + (x ^ (i / kPeriod % kChunks))) * 16 + in,
                                                    4 * sizeof(T)), v, sizeof(v));
        }
      __builtin_amdgcn_wave_barrier();
      const int rows = (int)(a.seqlen - t0 < kC ? a.seqlen - t0 : kC);
      const auto tile = buffer_of(y_to);
      const int x = lane % kChunks, row0 = lane / kChunks, mine = cols - my0 - x * kPer;   // columns from mine on
      const uint32_t y_off = (uint32_t)row0 * y_row + (uint32_t)(x * kPer * (int)sizeof(T));
#pragma unroll
      for (int u = 0; u < kC * kChunks / 64; ++u) {
        const int row = u * (64 / kChunks) + row0;
        typedef unsigned v4u __attribute__((ext_vector_type(4)));
        const v4u v = *reinterpret_cast<const v4u*>(out_lds + (row * kChunks + (x ^ (row / kPeriod % kChunks))) * 16);
        // The whole offset in the vector register: with a part of it in a scalar one the compiler leaves out the wait
        // state between a store of 16 bytes and the next write to its data registers, and the hardware stored the
        // first four bytes of some lanes from what was written there next.
        const uint32_t step = (uint32_t)(u * (64 / kChunks)) * y_row;
        const uint32_t at = row < rows && mine >= kPer ? y_off + step : kNowhere;
        __builtin_amdgcn_raw_buffer_store_b128(v, tile, (int)at, 0, 0);
      }
      y_to += (int64_t)kC * y_row;
      if (rarely(cols - my0 < 16 * kTiles && cols % kPer != 0)) {   // the rows' last vectors, value by value
        if (mine > 0 && mine < kPer)
#pragma unroll 1
          for (int row = row0; row < rows; row += 64 / kChunks) {
            const T* from = reinterpret_cast<const T*>(out_lds + (row * kChunks + (x ^ (row / kPeriod % kChunks))) * 16);
#pragma unroll 1
            for (int c = 0; c < mine; ++c) {
              const int at = (int)((uint32_t)row * y_row) + (x * kPer + c) * (int)sizeof(T);
              if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, from[c]), tile, at, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, from[c]), tile, at, 0, 0);
            }
          }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // The state behind the chunk: v times exp(c_end - c_j) as kTerms values, of 16-bit types of bf16, whose range is
    // fp32's: decays within a chunk span more than fp16's, and where k or v of the later tokens is 0 what is left of the
    // earlier ones is all there is.  k of fp16 enters as two of bf16, which hold its 11 bits.
    typedef std::conditional_t<kHalf, bf16, float> Term;
    constexpr int kTerms = kHalf ? 3 : 1;
    const float decay = __builtin_amdgcn_exp2f((float)c_end);
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      // a column with a value that is no number is NaN from here on
      const float by = first[n] < kC ? __builtin_nanf("") : decay;
#pragma unroll
      for (int t = 0; t < kKeyT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][n][r] *= by;
    }
    if constexpr (kF16 && kOut) __syncthreads();   // k's halves are there
    // k's columns are read several key tiles ahead: each read at its use, the products waited for it 16 times (4000 to
    // 5700 cycles for 1024 of products).
    constexpr int kAhead = kF16 ? 2 : kKeyT < 4 ? kKeyT : 4, kParts = kSums * kKeyT / kAhead;
    Frag<Term> kf[2][kAhead], kr[2][kF16 ? kAhead : 1];
    auto read_k = [&](auto part_) {
      constexpr int part = decltype(part_)::value, s = part * kAhead / kKeyT;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int t = part * kAhead % kKeyT + u;
        auto at = [&](int row, int c) { return k_at(row, key_of(t, c)); };
        if constexpr (kF16) {
          kf[part % 2][u] = column_frag(k_hi + 32 * s * kKeys, lane, at);
          kr[part % 2][u] = column_frag(k_lo + 32 * s * kKeys, lane, at);
        } else {
          kf[part % 2][u] = column_frag(k_lds + 32 * s * kKeys, lane, at);
        }
      }
    };
    read_k(std::integral_constant<int, 0>());
    __builtin_amdgcn_s_setprio(2);
    Frag<Term> w_v[kTerms][kTiles];
    each_of(std::make_integer_sequence<int, kParts>(), [&](auto part_) {
      constexpr int part = decltype(part_)::value, s = part * kAhead / kKeyT, t0 = part * kAhead % kKeyT;
      if constexpr (t0 == 0) {
        const float4 wa = *reinterpret_cast<const float4*>(w_lds + 32 * s + 4 * g);
        const float4 wb = *reinterpret_cast<const float4*>(w_lds + 32 * s + 16 + 4 * g);
        const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = (float)vf[s][n].v[e] * w[e];
#pragma unroll
          for (int i = 0; i < kTerms; ++i) {
            w_v[i][n] = round_frag<Term>(f);
            if (i + 1 < kTerms) take_off(f, w_v[i][n]);
          }
        }
      }
      // The next chunk's loads, between the products: all at once they hold the wave up while they are issued (12 of 16
      // bytes per lane, 1700 to 3000 cycles).  In front of a part's products, so that no branch lies between the last
      // products and the first use of S: behind one the compiler has left out wait states that such a use needs.
      if (chunk + 1 < last)
#pragma unroll
        for (int piece = part * 3 / kParts; piece < (part + 1) * 3 / kParts; ++piece) request(chunk + 1, piece);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (part + 1 < kParts) read_k(std::integral_constant<int, part + 1>());
      auto products = [&](auto& k, int i) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
          for (int n = 0; n < kTiles; ++n) S[t0 + u][n] = mma(k[u], w_v[i][n], S[t0 + u][n]);
      };
#pragma unroll
      for (int i = 0; i < kTerms; ++i) products(kf[part % 2], i);
      // the third term's product with k's second value is below 2^-25
      if constexpr (kF16) {
        products(kr[part % 2], 0);
        products(kr[part % 2], 1);
      }
      // Behind a branch, as the next loads have them, the compiler leaves out wait states that a register written by a
      // product, or overwritten after one, needs: eight of them here.
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 7");
      __builtin_amdgcn_sched_barrier(0);
    });
    __builtin_amdgcn_s_setprio(0);
    total += c_end;
  }

  if constexpr (kOut) {
    // tokens behind the last chunk with any
    for (int chunk = last > chunk0 ? last : chunk0; chunk < chunk1; ++chunk)
      for (int o = hw * 64 + lane; o < kC * kSlice; o += 64 * kWH) {
        const int64_t t = (int64_t)chunk * kC + o / kSlice;
        const int col = o % kSlice;
        if (t < a.seqlen && col < cols)
          static_cast<T*>(a.y)[((b * a.seqlen + t) * a.heads + h) * a.values + col0 + col] = (T)0.0f;
      }
  }
  float* to = kOut ? (p.final_state && span == p.spans - 1 && h * a.v_heads % heads == 0 ? p.final_state : nullptr)
                   : a.workspace + span * states;
  if (to) {
    to += (b * a.v_heads + hv) * state_floats(a) + col0 + my0;
    // the places are formed anew: those of the first loads would stay in registers over all chunks
    int group = lane_g, column = lane_m;
    asm volatile("" : "+v"(group), "+v"(column));
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
      if (my0 + 16 * n + column < cols) {
#pragma unroll
        for (int t = 0; t < kKeyT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (key_of(t, group) + r < keys) to[(int64_t)(key_of(t, group) + r) * a.values + 16 * n + column] = S[t][n][r];
      }
  }
  if (!kOut && hw == 0 && lane == 0 && slice == 0)
    (a.workspace + (p.spans - 1) * states)[(span * a.batch + b) * a.v_heads + hv] =
        __builtin_amdgcn_exp2f((float)total);
}

// The spans' own states into the states behind them: S_s = decay_s S_{s-1} + S_s, from the initial one.  Bound by the
// latency of the loads where there are many spans: kAtOnce of them are on their way together.
__global__ __launch_bounds__(256) void attention_join_kernel(Args p) {
  const LinearAttention& a = p.a;
  constexpr int kAtOnce = 8;
  const int n = p.spans - 1;
  const int64_t size = state_floats(a), states = a.batch * a.v_heads * size;
  const float* decays = a.workspace + (p.spans - 1) * states;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < states; i += (int64_t)gridDim.x * 256) {
    float s = a.init ? a.init[i] : 0.0f;
    const int64_t head = i / size;
    if (n < kAtOnce) {
      for (int k = 0; k < n; ++k) {
        float* at = a.workspace + k * states + i;
        s = __builtin_fmaf(s, decays[k * a.batch * a.v_heads + head], *at);
        *at = s;
      }
      continue;
    }
    for (int k0 = 0; k0 < n; k0 += kAtOnce) {
      float own[kAtOnce], d[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int k = k0 + u < n ? k0 + u : n - 1;
        own[u] = a.workspace[k * states + i];
        d[u] = decays[k * a.batch * a.v_heads + head];
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (k0 + u < n) a.workspace[(k0 + u) * states + i] = s = __builtin_fmaf(s, d[u], own[u]);
    }
  }
}

__global__ __launch_bounds__(256) void attention_copy_kernel(const float* from, float* to, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from[i];
}

// Four values at any alignment of one, past the caches: a state is read and written once.
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ float4 load4(const float* p) {
  const v4f_any v = __builtin_nontemporal_load(reinterpret_cast<const v4f_any*>(p));
  return make_float4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void store4(float* p, float4 f) {
  const v4f_any v = {f.x, f.y, f.z, f.w};
  __builtin_nontemporal_store(v, reinterpret_cast<v4f_any*>(p));
}

// One token.  A workgroup takes 64 columns of a head's state: 16 threads of four columns each, 16 such rows of
// threads.  Bound by the state's bytes: all of a thread's loads are on their way before the first is used.  128 x 80 heads
// of 128 x 64: 119 us, 5.7 TB/s, 134 through the caches, with other states in between.  The same states token after token,
// past the caches / through them: 21 MB 8.5 / 8.7, 42 MB 12.9 / 15.4, 84 MB 27 / 28, 168 MB 58 / 53, 336 MB 120 / 117.
template <typename T, int kRows>
__global__ __launch_bounds__(256) void attention_step_kernel(LinearAttention a, int slices, unsigned first) {
  constexpr int kMost = kRows * 16;
  __shared__ float k_lds[kMost], q_lds[kMost];
  __shared__ float sums[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned id = first + blockIdx.x;
  const int slice = (int)(id % slices);
  const int64_t head = id / slices, b = head / a.v_heads;
  const int hv = (int)(head % a.v_heads), keys = (int)a.keys;
  const int hk = (int)(hv * a.k_heads / a.v_heads);
  const int col = slice * 64 + tid % 16 * 4, kr = tid / 16;
  const int cols = (int)(a.values - col < 0 ? 0 : a.values - col < 4 ? a.values - col : 4);
  float* state = a.final_state + head * keys * a.values + col;
  float4 s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int key = i * 16 + kr;
    s[i] = make_float4(0, 0, 0, 0);
    if (key >= keys || cols == 0) continue;
    const float* at = state + (int64_t)key * a.values;
    if (cols == 4) {
      s[i] = load4(at);
    } else {
      s[i].x = at[0];
      if (cols > 1) s[i].y = at[1];
      if (cols > 2) s[i].z = at[2];
    }
  }
  const T* kp = static_cast<const T*>(a.k) + b * a.ks.batch + hk * a.ks.head;
  const T* vp = static_cast<const T*>(a.v) + b * a.vs.batch + hv * a.vs.head + col;
  const int per = (int)(a.heads / a.v_heads);   // heads of y that read this state
  auto query = [&](int r) {
    const int64_t hq = (hv * per + r) * a.q_heads / a.heads;
    const T* qp = static_cast<const T*>(a.q) + b * a.qs.batch + hq * a.qs.head;
    if (tid < kMost) q_lds[tid] = tid < keys ? (float)qp[tid] * a.scale : 0.0f;
  };
  if (tid < kMost) k_lds[tid] = tid < keys ? (float)kp[tid] : 0.0f;
  query(0);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < cols ? (float)vp[e] : 0.0f;
  float decay = 1.0f;
  if (a.log_decay) {
    const double d = (double)(a.token_decay ? a.log_decay[b * a.g_batch + hv] : a.log_decay[hv]) * kLog2e;
    decay = __builtin_amdgcn_exp2f((float)d);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int key = i * 16 + kr;
    const float k = k_lds[key];
    s[i].x = __builtin_fmaf(s[i].x, decay, k * v[0]);
    s[i].y = __builtin_fmaf(s[i].y, decay, k * v[1]);
    s[i].z = __builtin_fmaf(s[i].z, decay, k * v[2]);
    s[i].w = __builtin_fmaf(s[i].w, decay, k * v[3]);
    if (key >= keys || cols == 0) continue;
    float* at = state + (int64_t)key * a.values;
    if (cols == 4) {
      store4(at, s[i]);
    } else {
      at[0] = s[i].x;
      if (cols > 1) at[1] = s[i].y;
      if (cols > 2) at[2] = s[i].z;
    }
  }
  for (int r = 0; r < per; ++r) {
    if (r > 0) {
      __syncthreads();
      query(r);
      __syncthreads();
    }
    float y[4] = {};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int key = i * 16 + kr;
      if (key >= keys) continue;   // 0 times a state that is no number
      const float q = q_lds[key];
      y[0] = __builtin_fmaf(q, s[i].x, y[0]);
      y[1] = __builtin_fmaf(q, s[i].y, y[1]);
      y[2] = __builtin_fmaf(q, s[i].z, y[2]);
      y[3] = __builtin_fmaf(q, s[i].w, y[3]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] += __shfl_xor(y[e], 16);
      y[e] += __shfl_xor(y[e], 32);
    }
    if (lane < 16) *reinterpret_cast<float4*>(&sums[wave][lane * 4]) = make_float4(y[0], y[1], y[2], y[3]);
    __syncthreads();
    if (tid < 64 && slice * 64 + tid < a.values) {
      const float o = sums[0][tid] + sums[1][tid] + (sums[2][tid] + sums[3][tid]);
      static_cast<T*>(a.y)[(b * a.heads + hv * per + r) * a.values + slice * 64 + tid] = (T)o;
    }
  }
}

int chunk_of(int dtype) { return dtype == SSDI8_F32 ? 32 : 64; }

// Two heads to a workgroup where they are narrow and share q and k.
bool paired(const LinearAttention& a) {
  return a.values <= 64 && a.keys <= 128 && a.heads == a.v_heads && a.heads / a.q_heads % 2 == 0 && a.heads / a.k_heads % 2 == 0;
}

// Columns of a workgroup: 64 where 128 would leave half of the card without work, even with the tokens cut into spans of
// four chunks: a narrow workgroup is through a chunk sooner.  us with 64 / 128, bf16: 1 x 256 tokens, 16 heads of 128 x 128
// 19 / 26, 4 x 256, 64 heads 28 / 32, 4 x 2000, 8 heads 51 / 61; above, q k is formed twice: 4 x 8192, 16 heads 235 / 205.
int64_t slice_of(const LinearAttention& a) {
  if (a.values <= 64 || a.keys > 128) return 64;
  const int64_t chunks = (a.seqlen + chunk_of(a.dtype) - 1) / chunk_of(a.dtype), spans = chunks < 8 ? 1 : chunks / 4;
  return a.batch * a.heads * ((a.values + 127) / 128) * spans <= 256 ? 64 : 128;
}

Args plan(const LinearAttention& a) {
  Args p;
  p.a = a;
  p.first = 0;
  const int64_t c = chunk_of(a.dtype), slice = slice_of(a);
  p.slices = (int)((a.values + slice - 1) / slice);
  p.chunks = (int)((a.seqlen + c - 1) / c);
  p.groups = (int)(paired(a) ? a.heads / 2 : a.heads);
  // Spans: as many workgroups as the card holds at once (two for every CU), each with two chunks at least; none of
  // fewer than eight chunks.  us with and without, bf16: 8 chunks of 8 heads of 128 x 128 29 / 32, four chunks of 16 heads
  // 27 / 19.
  const int64_t wgs = a.batch * p.groups * p.slices, hold = a.keys > 128 ? 256 : 512, most = p.chunks < 8 ? 1 : p.chunks / 2;
  int64_t spans = wgs == 0 ? 1 : hold / wgs;
  spans = spans < most ? spans : most;
  if (spans < 1) spans = 1;
  p.span_chunks = (int)((p.chunks + spans - 1) / spans);
  p.spans = p.span_chunks ? (p.chunks + p.span_chunks - 1) / p.span_chunks : 1;
  return p;
}

// Whether other workgroups than the one that writes a final state read its initial one.
bool read_elsewhere(const Args& p) { return p.spans > 1 || p.a.heads > p.a.v_heads; }

template <typename T, int kKeys, int kTiles, int kHeads> hipError_t run(Args p, hipStream_t st) {
  constexpr int kC = sizeof(T) == 4 ? 32 : 64;
  const LinearAttention& a = p.a;
  const int64_t all = a.batch * a.v_heads * a.keys * a.values, wgs_all = (all + 255) / 256;
  const dim3 each((unsigned)(wgs_all < 4096 ? wgs_all : 4096));
  // over its own initial state a final one goes by way of the workspace
  const bool apart = a.final_state && a.final_state == a.init && read_elsewhere(p);
  p.final_state = apart ? a.workspace + (p.spans - 1) * (all + a.batch * a.v_heads) : a.final_state;
  auto walk = [&](auto out, Args s, int64_t spans) {
    return in_parts(a.batch * s.groups * s.slices * spans, 256, [&](int64_t first, dim3 grid) {
      s.first = first;
      attention_kernel<T, kKeys, kTiles, kHeads, kC, decltype(out)::value><<<grid, 256, 0, st>>>(s);
    });
  };
  hipError_t e = hipSuccess;
  if (p.spans > 1) {
    Args s = p;
    s.groups = (int)(a.v_heads / kHeads);
    e = walk(std::false_type(), s, p.spans - 1);
    if (e != hipSuccess) return e;
    attention_join_kernel<<<each, 256, 0, st>>>(p);
  }
  e = walk(std::true_type(), p, p.spans);
  if (e != hipSuccess) return e;
  if (apart) attention_copy_kernel<<<each, 256, 0, st>>>(p.final_state, a.final_state, all);
  return hipGetLastError();
}

template <typename T, int kKeys> hipError_t by_values(const Args& p, hipStream_t st) {
  if constexpr (kKeys > 128) {
    return run<T, kKeys, 1, 1>(p, st);
  } else {
    if (slice_of(p.a) > 64) return run<T, kKeys, 2, 1>(p, st);
    return paired(p.a) ? run<T, kKeys, 2, 2>(p, st) : run<T, kKeys, 1, 1>(p, st);
  }
}

template <typename T> hipError_t by_size(const Args& p, hipStream_t st) {
  if (p.a.keys <= 64) return by_values<T, 64>(p, st);
  if (p.a.keys <= 128) return by_values<T, 128>(p, st);
  return by_values<T, 256>(p, st);
}

template <typename T> hipError_t run_step(const LinearAttention& a, hipStream_t st) {
  const int slices = (int)((a.values + 63) / 64);
  return in_parts(a.batch * a.v_heads * slices, 256, [&](int64_t first, dim3 grid) {
    if (a.keys <= 64) attention_step_kernel<T, 4><<<grid, 256, 0, st>>>(a, slices, (unsigned)first);
    else if (a.keys <= 128) attention_step_kernel<T, 8><<<grid, 256, 0, st>>>(a, slices, (unsigned)first);
    else attention_step_kernel<T, 16><<<grid, 256, 0, st>>>(a, slices, (unsigned)first);
  });
}

}  // namespace

int64_t linear_attention_workspace(const LinearAttention& a) {
  const Args p = plan(a);
  const int64_t states = a.batch * a.v_heads * a.keys * a.values;
  return (p.spans - 1) * (states + a.batch * a.v_heads) + (read_elsewhere(p) ? states : 0);
}

hipError_t launch_linear_attention(const LinearAttention& a, hipStream_t st) {
  const Args p = plan(a);
  switch (a.dtype) {
    case SSDI8_F32: return by_size<float>(p, st);
    case SSDI8_F16: return by_size<_Float16>(p, st);
    default: return by_size<bf16>(p, st);
  }
}

hipError_t launch_linear_attention_step(const LinearAttention& a, hipStream_t st) {
  switch (a.dtype) {
    case SSDI8_F32: return run_step<float>(a, st);
    case SSDI8_F16: return run_step<_Float16>(a, st);
    default: return run_step<bf16>(a, st);
  }
}

}  // namespace ssdi8
