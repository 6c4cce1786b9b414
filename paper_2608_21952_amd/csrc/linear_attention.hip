// Linear attention with a decay per head:
//   S_t = exp(g_t) S_{t-1} + k_t v_t^T,   y_t = scale S_t^T q_t          (S: keys x values, fp32)
// over chunks of C tokens, c_i the sum of g over the chunk's tokens up to i:
//   y_i = scale (exp(c_i) S_0^T q_i + sum_{j <= i} exp(c_i - c_j) (q_i . k_j) v_j)
//   S_C = exp(c_C) S_0 + sum_j exp(c_C - c_j) k_j v_j^T
// A workgroup of four waves walks the chunks of a head (of a span of it), each wave with its own columns of S, v and
// y; q, k and v of a chunk lie in LDS, the next chunk's are on their way in registers.
//
// Matrix products: the 16 x 16 instructions take eight values of a row per lane, for 32 along the sum (fp32: eight
// instructions of four).  Lane group g (of 16 lanes) is given places 4 g + (0..3) of the first 16 and of the second
// 16 of the 32: these are the rows that a lane holds of two result tiles, so that results become operands where
// they lie.  S (keys x values) is the operand of S^T q, and p^T = (k . q) that of p v once all waves have it.
//
// Roundings, of 16-bit types: p, S and exp(c_C - c_j) v_j enter the matrix unit as the sum of two values of the
// type, which leaves 2^-17 (bf16) and 2^-22 (fp16) of them; as one value each would add as much error as y's own
// rounding, and 2^-9 of S with every chunk.  fp16: brought to the type's range by powers of two first (p per row, S
// per tile, v per column).  Sums, S, and the decays' sums (these in fp64: differences of far sums) are not rounded.
// A value of v that is no number would reach earlier tokens of its chunk through 0 times it: it enters as 0, and its
// column is NaN from its token on.
#include <type_traits>

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
// A value as the sum of two of the type (fp32: itself), in slot e of two fragments.
template <typename T> __device__ __forceinline__ void split(float f, Frag<T>& hi, Frag<T>& lo, int e) {
  hi.v[e] = (T)f;
  if constexpr (sizeof(T) == 2) lo.v[e] = (T)(f - (float)hi.v[e]);
}
template <typename T> __device__ __forceinline__ v4f mma_split(const Frag<T>& ahi, const Frag<T>& alo, const Frag<T>& b, v4f c) {
  c = mma(ahi, b, c);
  if constexpr (sizeof(T) == 2) c = mma(alo, b, c);
  return c;
}

// The exponent shift that brings magnitude bits `big` of fp32 to [2^14, 2^15); 0 for 0 and for what is no number.
__device__ __forceinline__ int range_shift(uint32_t big) {
  const int e = (int)(big >> 23);
  if (e == 0 || e == 255) return 0;
  const int s = 127 + 14 - e;
  return s > 100 ? 100 : s;
}
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
__device__ __forceinline__ uint32_t bits_max(uint32_t a, float v) {
  const uint32_t m = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
  return a > m ? a : m;
}
__device__ __forceinline__ uint32_t group_max(uint32_t v) {   // over the four lane groups
#pragma unroll
  for (int d = 16; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
    v = v > o ? v : o;
  }
  return v;
}

// Two times four values: places [at, at + 4) and [at + 16, at + 20) of an LDS row.
template <typename T> __device__ __forceinline__ Frag<T> row_frag(const T* p) {
  Frag<T> f;
  __builtin_memcpy(&f.v[0], __builtin_assume_aligned(p, 4 * sizeof(T)), 4 * sizeof(T));
  __builtin_memcpy(&f.v[4], __builtin_assume_aligned(p + 16, 4 * sizeof(T)), 4 * sizeof(T));
  return f;
}
// The same of a column: rows [4 g, 4 g + 4) and 16 further on, of 16 columns at p (p: row 0 of the 32, LDS).
template <typename T, int kStride> __device__ __forceinline__ Frag<T> column_frag(const T* p, int lane) {
  Frag<T> f;
  const int g = lane >> 4, m = lane & 15;
  if constexpr (sizeof(T) == 2) {
    // the four values that lane m of a group points at are a quarter of row m / 4 of a 4 x 16 block, which the
    // instruction hands out by columns
    typedef __attribute__((address_space(3))) v4s* Lds;
    T* q = const_cast<T*>(p) + (4 * g + m / 4) * kStride + 4 * (m % 4);
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(q));
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(q + 16 * kStride));
    __builtin_memcpy(&f.v[0], &a, 8);
    __builtin_memcpy(&f.v[4], &b, 8);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = p[(4 * g + e % 4 + e / 4 * 16) * kStride + m];
  }
  return f;
}

struct Args {
  LinearAttention a;
  int slices, spans, chunks, span_chunks;   // column slices of a head; spans of the tokens and their chunks
};

// Floats of a head's state in the workspace, and where the spans' decays lie behind the states.
__device__ __host__ __forceinline__ int64_t state_floats(const LinearAttention& a) { return a.keys * a.values; }

// A tile of rows on its way from memory to LDS: kRows rows of kWidth values (`width` of them there), by 256 threads
// in vectors of 16 bytes.
template <typename T, int kRows, int kWidth> struct Stage {
  static constexpr int kPer = 16 / (int)sizeof(T), kVecs = kWidth / kPer;
  static constexpr int kEach = (kRows * kVecs + 255) / 256;
  static_assert(kRows * kVecs % 256 == 0 || kEach == 1, "stage");
  uint4 v[kEach];
  __device__ __forceinline__ void load(const T* base, int64_t token_stride, int tokens, int width, int tid) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * 256 + tid, row = at / kVecs, c = at % kVecs * kPer;
      v[i] = make_uint4(0, 0, 0, 0);
      if (row >= tokens || row >= kRows) continue;
      const T* p = base + row * token_stride + c;
      if (c + kPer <= width) {
        __builtin_memcpy(&v[i], p, 16);
      } else {
        T e[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) e[j] = c + j < width ? p[j] : (T)0.0f;
        __builtin_memcpy(&v[i], e, 16);
      }
    }
  }
  __device__ __forceinline__ void put(T* lds, int stride, int tid) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * 256 + tid, row = at / kVecs, c = at % kVecs * kPer;
      if (row < kRows) *reinterpret_cast<uint4*>(lds + row * stride + c) = v[i];
    }
  }
};

// kKeys: keys filled up to 64, 128 or 256.  kTiles: tiles of 16 columns per wave.  kC: tokens of a chunk.
// kOut: the walk with outputs; else the one for the states at the spans' ends.
template <typename T, int kKeys, int kTiles, int kC, bool kOut>
__global__ __launch_bounds__(256) void attention_kernel(Args p) {
  const LinearAttention& a = p.a;
  constexpr int kSlice = 64 * kTiles;                       // columns of a workgroup
  constexpr int kSums = kC / 32, kRowsT = kC / 16, kKeyT = kKeys / 16, kKeyS = kKeys / 32;
  constexpr int kPad = 16 / (int)sizeof(T);
  constexpr int kQ = kKeys + kPad, kV = kSlice + kPad;      // LDS row lengths
  constexpr int kHalves = sizeof(T) == 2 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) T q_lds[kOut ? kC * kQ : 8];
  __shared__ __attribute__((aligned(16))) T k_lds[kC * kQ];
  __shared__ __attribute__((aligned(16))) T v_lds[kC * kV];
  __shared__ __attribute__((aligned(16))) Frag<T> p_lds[kOut ? kRowsT * kSums * kHalves * 64 : 1];
  __shared__ double c_lds[kC];
  __shared__ float row_scale[kC];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, m = lane & 15;
  int id = xcd_remap(blockIdx.x, gridDim.x);
  const int slice = id % p.slices;
  id /= p.slices;
  // heads are neighbours: those that share q and k share an XCD's cache
  const int heads = (int)(kOut ? a.heads : a.v_heads);
  const int h = id % heads;
  id /= heads;
  const int span = id % (kOut ? p.spans : p.spans - 1);
  const int64_t b = id / (kOut ? p.spans : p.spans - 1);
  const int hq = (int)(h * a.q_heads / heads), hv = (int)(h * a.v_heads / heads);
  const int hk = (int)(hv * a.k_heads / a.v_heads);
  const int col0 = slice * kSlice;
  const int cols = (int)(a.values - col0 < kSlice ? a.values - col0 : kSlice);
  const int keys = (int)a.keys;

  const T* qp = static_cast<const T*>(a.q) + b * a.qs.batch + hq * a.qs.head;
  const T* kp = static_cast<const T*>(a.k) + b * a.ks.batch + hk * a.ks.head;
  const T* vp = static_cast<const T*>(a.v) + b * a.vs.batch + hv * a.vs.head + col0;
  int64_t end = a.seqlen;
  if (a.lengths) {
    const int64_t n = a.lengths[b];
    end = n < 0 ? 0 : n < end ? n : end;
  }
  const int chunk0 = span * p.span_chunks;
  const int chunk1 = chunk0 + p.span_chunks < p.chunks ? chunk0 + p.span_chunks : p.chunks;
  const int live = (int)((end + kC - 1) / kC);               // chunks with tokens
  const int last = live < chunk1 ? live : chunk1;

  // the state: rows 16 t + 4 g + (0..3) of key tile t, column m of column tile n
  const int my0 = wave * kTiles * 16;
  const int64_t states = a.batch * a.v_heads * state_floats(a);
  v4f S[kKeyT][kTiles];
  {
    const float* from = a.init ? a.init + (b * a.v_heads + hv) * state_floats(a) : nullptr;
    if (kOut && span > 0) from = a.workspace + (span - 1) * states + (b * a.v_heads + hv) * state_floats(a);
    if (!kOut) from = nullptr;
#pragma unroll
    for (int t = 0; t < kKeyT; ++t)
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = 16 * t + 4 * g + r, col = my0 + 16 * n + m;
          S[t][n][r] = from && key < keys && col < cols ? from[(int64_t)key * a.values + col0 + col] : 0.0f;
        }
  }
  double total = 0.0;   // of the decays' logarithms (base 2) over the span

  Stage<T, kC, kKeys> q_next, k_next;
  Stage<T, kC, kSlice> v_next;
  float g_next = 0.0f;
  auto request = [&](int chunk) {
    const int64_t t0 = (int64_t)chunk * kC;
    const int tokens = (int)(end - t0 < kC ? end - t0 : kC);
    if constexpr (kOut) q_next.load(qp + t0 * a.qs.token, a.qs.token, tokens, keys, tid);
    k_next.load(kp + t0 * a.ks.token, a.ks.token, tokens, keys, tid);
    v_next.load(vp + t0 * a.vs.token, a.vs.token, tokens, cols, tid);
    g_next = 0.0f;
    if (a.log_decay && lane < tokens)
      g_next = a.token_decay ? a.log_decay[b * a.g_batch + (t0 + lane) * a.g_token + hv] : a.log_decay[hv];
  };

  if (chunk0 < last) request(chunk0);
  for (int chunk = chunk0; chunk < last; ++chunk) {
    __syncthreads();   // the last chunk is read
    if constexpr (kOut) q_next.put(q_lds, kQ, tid);
    k_next.put(k_lds, kQ, tid);
    v_next.put(v_lds, kV, tid);
    // sums of the decays' logarithms, in base 2; below 2^-100000 is 0 all the same, and an infinite one would leave
    // no differences behind it
    double c = g_next < -65536.0f ? -65536.0 * kLog2e : (double)g_next * kLog2e;
#pragma unroll
    for (int d = 1; d < kC; d *= 2) {
      const double o = __shfl_up(c, d);
      c = lane >= d ? c + o : c;
    }
    if (wave == 0 && lane < kC) c_lds[lane] = c;
    const double c_end = __shfl(c, kC - 1);
    __syncthreads();
    if (chunk + 1 < last) request(chunk + 1);

    const int64_t t0 = (int64_t)chunk * kC;
    if constexpr (kOut) {
      // p^T: rows j, column i = m of row tile `wave`
      for (int it = wave; it < kRowsT; it += 4) {
        const int i = it * 16 + m;
        const double ci = c_lds[i];
        v4f acc[kRowsT] = {};
#pragma unroll
        for (int s = 0; s < kKeyS; ++s) {
          const Frag<T> qf = row_frag(q_lds + i * kQ + 32 * s + 4 * g);
#pragma unroll
          for (int jt = 0; jt < kRowsT; ++jt)
            if (jt <= it) acc[jt] = mma(row_frag(k_lds + (jt * 16 + m) * kQ + 32 * s + 4 * g), qf, acc[jt]);
        }
        uint32_t big = 0;
#pragma unroll
        for (int jt = 0; jt < kRowsT; ++jt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = jt * 16 + 4 * g + r;
            const float w = a.scale * __builtin_amdgcn_exp2f((float)(ci - c_lds[j]));
            acc[jt][r] = j <= i ? acc[jt][r] * w : 0.0f;
            big = bits_max(big, acc[jt][r]);
          }
        float up = 1.0f;
        if constexpr (std::is_same_v<T, _Float16>) {
          const int s = range_shift(group_max(big));
          up = power(s);
          if (g == 0) row_scale[i] = power(-s);
        }
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
          Frag<T> hi, lo;
#pragma unroll
          for (int e = 0; e < 8; ++e) split(acc[2 * s + e / 4][e % 4] * up, hi, lo, e);
          p_lds[((it * kSums + s) * kHalves) * 64 + lane] = hi;
          if constexpr (kHalves == 2) p_lds[((it * kSums + s) * kHalves + 1) * 64 + lane] = lo;
        }
      }
      __syncthreads();
    }

    // v as it is (for p v) and times exp(c_end - c_j) (for the state), where its values are no numbers 0
    Frag<T> vf[kSums][kTiles], whi[kSums][kTiles], wlo[kSums][kTiles];
    float down[kTiles];
    int first[kTiles];   // the first token of the column whose value is no number
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      float w[kSums][8];
      uint32_t big = 0;
      bool odd = false;
      first[n] = kC;
#pragma unroll
      for (int s = 0; s < kSums; ++s) {
        vf[s][n] = column_frag<T, kV>(v_lds + 32 * s * kV + my0 + 16 * n, lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) odd |= !(__builtin_fabsf((float)vf[s][n].v[e]) < __builtin_inff());
      }
      if (__any(odd)) {
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
#pragma unroll
      for (int s = 0; s < kSums; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = 32 * s + 16 * (e / 4) + 4 * g + e % 4;
          w[s][e] = (float)vf[s][n].v[e] * __builtin_amdgcn_exp2f((float)(c_end - c_lds[j]));
          big = bits_max(big, w[s][e]);
        }
      float up = 1.0f;
      down[n] = 1.0f;
      if constexpr (std::is_same_v<T, _Float16>) {
        const int sh = range_shift(group_max(big));
        up = power(sh);
        down[n] = power(-sh);
      }
#pragma unroll
      for (int s = 0; s < kSums; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) split(w[s][e] * up, whi[s][n], wlo[s][n], e);
    }

    if constexpr (kOut) {
      const int64_t left = end - t0;
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        // the state as an operand
        Frag<T> shi[kKeyS], slo[kKeyS];
        float s_up = 1.0f, s_down = 1.0f;
        if constexpr (std::is_same_v<T, _Float16>) {
          uint32_t big = 0;
#pragma unroll
          for (int t = 0; t < kKeyT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) big = bits_max(big, S[t][n][r]);
#pragma unroll
          for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)big, d);
            big = big > o ? big : o;
          }
          const int sh = range_shift(big);
          s_up = power(sh);
          s_down = power(-sh);
        }
#pragma unroll
        for (int s = 0; s < kKeyS; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e) split(S[2 * s + e / 4][n][e % 4] * s_up, shi[s], slo[s], e);
        int bad[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) bad[r] = __shfl(first[n], 4 * g + r);
#pragma unroll
        for (int it = 0; it < kRowsT; ++it) {
          const int i = it * 16 + m;
          v4f before = {}, in = {};
#pragma unroll
          for (int s = 0; s < kKeyS; ++s)
            before = mma_split(shi[s], slo[s], row_frag(q_lds + i * kQ + 32 * s + 4 * g), before);
#pragma unroll
          for (int s = 0; s < kSums; ++s)
            if (2 * s <= it) {
              const Frag<T>* at = p_lds + ((it * kSums + s) * kHalves) * 64 + lane;
              in = mma(vf[s][n], at[0], in);
              if constexpr (kHalves == 2) in = mma(vf[s][n], at[64], in);
            }
          const float e = a.scale * __builtin_amdgcn_exp2f((float)c_lds[i]) * s_down;
          const float in_scale = std::is_same_v<T, _Float16> ? row_scale[i] : 1.0f;
          float o[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            o[r] = __builtin_fmaf(before[r], e, in[r] * in_scale);
            if (i >= bad[r]) o[r] = __builtin_nanf("");
          }
          const int col = my0 + 16 * n + 4 * g;
          if (t0 + i < a.seqlen && col < cols) {
            const bool dead = i >= left;   // behind the sequence's end: 0
            T* y = static_cast<T*>(a.y) + ((b * a.seqlen + t0 + i) * a.heads + h) * a.values + col0 + col;
            T out[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) out[r] = (T)(dead ? 0.0f : o[r]);
            if (col + 4 <= cols) {
              __builtin_memcpy(y, out, sizeof(out));
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (col + r < cols) y[r] = out[r];
            }
          }
        }
      }
    }

    // the state behind the chunk
    const float decay = __builtin_amdgcn_exp2f((float)c_end);
#pragma unroll
    for (int t = 0; t < kKeyT; ++t) {
      v4f add[kTiles] = {};
#pragma unroll
      for (int s = 0; s < kSums; ++s) {
        const Frag<T> kf = column_frag<T, kQ>(k_lds + 32 * s * kQ + 16 * t, lane);
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          add[n] = mma(kf, whi[s][n], add[n]);
          if constexpr (kHalves == 2) add[n] = mma(kf, wlo[s][n], add[n]);
        }
      }
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          S[t][n][r] = __builtin_fmaf(S[t][n][r], decay, add[n][r] * down[n]);
          if (first[n] < kC) S[t][n][r] = __builtin_nanf("");
        }
    }
    total += c_end;
  }

  if constexpr (kOut) {
    // tokens behind the last chunk with any
    for (int chunk = last > chunk0 ? last : chunk0; chunk < chunk1; ++chunk)
      for (int o = tid; o < kC * kSlice; o += 256) {
        const int64_t t = (int64_t)chunk * kC + o / kSlice;
        const int col = o % kSlice;
        if (t < a.seqlen && col < cols)
          static_cast<T*>(a.y)[((b * a.seqlen + t) * a.heads + h) * a.values + col0 + col] = (T)0.0f;
      }
  }
  float* to = kOut ? (a.final_state && span == p.spans - 1 && h * a.v_heads % heads == 0 ? a.final_state : nullptr)
                   : a.workspace + span * states;
  if (to) {
    to += (b * a.v_heads + hv) * state_floats(a);
#pragma unroll
    for (int t = 0; t < kKeyT; ++t)
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = 16 * t + 4 * g + r, col = my0 + 16 * n + m;
          if (key < keys && col < cols) to[(int64_t)key * a.values + col0 + col] = S[t][n][r];
        }
  }
  if (!kOut && tid == 0 && slice == 0)
    (a.workspace + (p.spans - 1) * states)[(span * a.batch + b) * a.v_heads + hv] =
        __builtin_amdgcn_exp2f((float)total);
}

// The spans' own states into the states behind them: S_s = decay_s S_{s-1} + S_s, from the initial one.
__global__ __launch_bounds__(256) void attention_join_kernel(Args p) {
  const LinearAttention& a = p.a;
  const int64_t size = state_floats(a), states = a.batch * a.v_heads * size;
  const float* decays = a.workspace + (p.spans - 1) * states;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < states; i += (int64_t)gridDim.x * 256) {
    float s = a.init ? a.init[i] : 0.0f;
    for (int k = 0; k < p.spans - 1; ++k) {
      float* at = a.workspace + k * states + i;
      s = __builtin_fmaf(s, decays[k * a.batch * a.v_heads + i / size], *at);
      *at = s;
    }
  }
}

// One token.  A workgroup takes 64 columns of a head's state: 16 threads of four columns each, 16 such rows of
// threads.  Bound by the state's bytes: all of a thread's loads are on their way before the first is used.
template <typename T, int kRows>
__global__ __launch_bounds__(256) void attention_step_kernel(LinearAttention a, int slices) {
  constexpr int kMost = kRows * 16;
  __shared__ float k_lds[kMost], q_lds[kMost];
  __shared__ float sums[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slice = (int)(blockIdx.x % slices);
  const int64_t head = blockIdx.x / slices, b = head / a.v_heads;
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
      __builtin_memcpy(&s[i], at, 16);
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
      __builtin_memcpy(at, &s[i], 16);
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
int tiles_of(int64_t values) { return values <= 64 ? 1 : 2; }

Args plan(const LinearAttention& a) {
  Args p;
  p.a = a;
  const int64_t c = chunk_of(a.dtype), slice = 64 * tiles_of(a.values);
  p.slices = (int)((a.values + slice - 1) / slice);
  p.chunks = (int)((a.seqlen + c - 1) / c);
  // Spans: two workgroups for every CU, each with four chunks at least.
  const int64_t wgs = a.batch * a.heads * p.slices;
  int64_t spans = wgs >= 256 || wgs == 0 ? 1 : (512 + wgs - 1) / wgs;
  spans = spans < p.chunks / 4 ? spans : p.chunks / 4;
  if (spans < 1) spans = 1;
  p.span_chunks = (int)((p.chunks + spans - 1) / spans);
  p.spans = p.span_chunks ? (p.chunks + p.span_chunks - 1) / p.span_chunks : 1;
  return p;
}

template <typename T, int kKeys, int kTiles> hipError_t run(const Args& p, hipStream_t st) {
  constexpr int kC = sizeof(T) == 4 ? 32 : 64;
  const LinearAttention& a = p.a;
  if (p.spans > 1) {
    attention_kernel<T, kKeys, kTiles, kC, false>
        <<<dim3((unsigned)(a.batch * a.v_heads * p.slices * (p.spans - 1))), 256, 0, st>>>(p);
    const int64_t states = a.batch * a.v_heads * a.keys * a.values, wgs = (states + 255) / 256;
    attention_join_kernel<<<dim3((unsigned)(wgs < 4096 ? wgs : 4096)), 256, 0, st>>>(p);
  }
  attention_kernel<T, kKeys, kTiles, kC, true>
      <<<dim3((unsigned)(a.batch * a.heads * p.slices * p.spans)), 256, 0, st>>>(p);
  return hipGetLastError();
}

template <typename T> hipError_t by_size(const Args& p, hipStream_t st) {
  const bool wide = tiles_of(p.a.values) == 2;
  if (p.a.keys <= 64) return wide ? run<T, 64, 2>(p, st) : run<T, 64, 1>(p, st);
  if (p.a.keys <= 128) return wide ? run<T, 128, 2>(p, st) : run<T, 128, 1>(p, st);
  return wide ? run<T, 256, 2>(p, st) : run<T, 256, 1>(p, st);
}

template <typename T> hipError_t run_step(const LinearAttention& a, hipStream_t st) {
  const int slices = (int)((a.values + 63) / 64);
  const dim3 grid((unsigned)(a.batch * a.v_heads * slices));
  if (a.keys <= 64) attention_step_kernel<T, 4><<<grid, 256, 0, st>>>(a, slices);
  else if (a.keys <= 128) attention_step_kernel<T, 8><<<grid, 256, 0, st>>>(a, slices);
  else attention_step_kernel<T, 16><<<grid, 256, 0, st>>>(a, slices);
  return hipGetLastError();
}

}  // namespace

int64_t linear_attention_workspace(const LinearAttention& a) {
  const Args p = plan(a);
  return (p.spans - 1) * a.batch * a.v_heads * (a.keys * a.values + 1);
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
