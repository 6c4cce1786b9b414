// The selective scan's kernel over prompts (described in selective_scan.hip).
#pragma once

#include <type_traits>

#include "block.hpp"

namespace ssdi8 {

namespace sel_scan {

constexpr int kThreads = 256;
constexpr int kSpanTokens = 64;   // the longest tile

// kCount elements as they lie in memory (a word each of fp32, half a word of a 16-bit type), turned into
// fp32 later.  A whole vector is requested without a choice between ways of loading it: where ways met, the
// compiler waited for the data.
template <int kCount> struct Raw {
  uint32_t w[kCount];
};
template <int kCount>
__device__ __forceinline__ void request_raw(Raw<kCount>& r, const char* p, int dtype) {
  __builtin_memcpy(r.w, p, 2 * kCount);
  if (dtype == 0) __builtin_memcpy(r.w + kCount / 2, p + 2 * kCount, 2 * kCount);
}
// The first n elements, the others 0.
template <int kCount>
__device__ __forceinline__ void request_part(Raw<kCount>& r, const char* p, int dtype, int n) {
#pragma unroll
  for (int i = 0; i < kCount; ++i) r.w[i] = 0;
#pragma unroll
  for (int i = 0; i < kCount; ++i)
    if (i < n) {
      if (dtype == 0) r.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
      else r.w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
    }
}
__device__ __forceinline__ uint32_t load_raw1(const void* base, int64_t off, int dtype) {
  return dtype == 0 ? static_cast<const uint32_t*>(base)[off]
                    : (uint32_t) static_cast<const uint16_t*>(base)[off];
}
__device__ __forceinline__ float as_float(uint32_t bits, int dtype) {
  if (dtype == 0) return __builtin_bit_cast(float, bits);
  if (dtype == 1) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  return __builtin_bit_cast(float, bits << 16);
}
template <int kCount>
__device__ __forceinline__ void as_floats(const Raw<kCount>& r, int dtype, float (&out)[kCount]) {
  if (dtype == 0) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) out[i] = __builtin_bit_cast(float, r.w[i]);
  } else if (dtype == 1) {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      out[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i / 2] >> (16 * (i & 1))));
  } else {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      out[i] = __builtin_bit_cast(float, i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
  }
}
template <typename T, int kCount>
__device__ __forceinline__ void store_n(T* p, int n, const float (&v)[kCount]) {
  if (n >= kCount) {
    T t[kCount];
#pragma unroll
    for (int i = 0; i < kCount; ++i) t[i] = (T)v[i];
    __builtin_memcpy(p, t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}
template <int kCount>
__device__ __forceinline__ void store_as(void* base, int64_t off, int dtype, int n, const float (&v)[kCount]) {
  if (dtype == 0) store_n(static_cast<float*>(base) + off, n, v);
  else if (dtype == 1) store_n(static_cast<_Float16*>(base) + off, n, v);
  else store_n(static_cast<bf16*>(base) + off, n, v);
}

// A in base 2; -inf (a decay of 0 for any positive delta) stays finite, so that delta = 0 gives 1.
__device__ __forceinline__ float decay_rate(float A) {
  const float a = A * kLog2eF;
  return a == -__builtin_inff() ? -__FLT_MAX__ : a;
}

// A lane's kS states lie in pieces of up to four neighbouring ones, the pieces of a channel's kLanes lanes side
// by side: 16 lanes then read 256 bytes of a row of B in a line, where eight states in a line per lane put
// every second lane on the same banks.
template <int kLanes, int kS> struct States {
  static constexpr int kPiece = kS < 4 ? kS : 4, kPieces = kS / kPiece;
  static __device__ __forceinline__ int at(int sub, int piece) { return (piece * kLanes + sub) * kPiece; }
  // of a row of N, 0 behind its end
  static __device__ __forceinline__ void load(const float* row, int sub, int N, float (&h)[kS]) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int n0 = at(sub, k);
      if (n0 + kPiece <= N) {
        __builtin_memcpy(&h[k * kPiece], row + n0, 4 * kPiece);
      } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) h[k * kPiece + i] = n0 + i < N ? row[n0 + i] : 0.0f;
      }
    }
  }
  static __device__ __forceinline__ void store(float* row, int sub, int N, const float (&h)[kS]) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int n0 = at(sub, k);
      if (n0 + kPiece <= N) {
        __builtin_memcpy(row + n0, &h[k * kPiece], 4 * kPiece);
      } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
          if (n0 + i < N) row[n0 + i] = h[k * kPiece + i];
      }
    }
  }
  // of a row of B or C in LDS
  static __device__ __forceinline__ void take(const float* row, int sub, float* v) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      __builtin_memcpy(v + k * kPiece, __builtin_assume_aligned(row + at(sub, k), 4 * kPiece), 4 * kPiece);
  }
};

// Where channel pair `pair` of a token's row of kCh channels lies.  With vectors of eight channels the low two
// bits of its place are exchanged so that the 16 lanes of an access, neighbouring vectors and tokens, touch
// every bank once; pairs by themselves lie in a line.
template <int kCh, int kSV> __device__ __forceinline__ int pair_slot(int row, int pair) {
  if (kSV != 8) return pair;
  int key;
  if (kCh == 64) key = (pair >> 4) ^ ((row & 1) << 1);
  else if (kCh == 32) key = row & 3;
  else if (kCh == 16) key = (row >> 1) & 3;
  else key = (row >> 2) & 3;
  return pair ^ key;
}

// The sums over kLanes lanes of kGroup tokens' values, each token's in lanes of its own: while more than one
// value is left, a lane keeps those of one half of the tokens and gives its partner the others, so that a
// step costs half of the one before it.  Partners in order: 16 lanes off, mirrored in 16 and in 8 (they
// differ in the bit that chooses, and hold the same tokens), then neighbours and pairs.
constexpr int kSumBits[5] = {4, 3, 2, 0, 1};
template <int kStep> __device__ __forceinline__ float partner(float v) {
  constexpr int kCtrl = kStep == 1 ? 0x140 : kStep == 2 ? 0x141 : kStep == 3 ? 0xB1 : 0x4E;
  if constexpr (kStep == 0) return __shfl_xor(v, 16);
  else
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf,
                                                                 0xf, true));
}
constexpr int sum_first(int lanes) {   // the first of the steps
  return lanes == 32 ? 0 : lanes == 16 ? 1 : lanes == 8 ? 2 : 3;
}
template <int kStep, int kCount>
__device__ __forceinline__ float sum_steps(const float (&v)[kCount], int lane) {
  if constexpr (kStep == 5) {
    return v[0];
  } else if constexpr (kCount == 1) {
    const float s[1] = {v[0] + partner<kStep>(v[0])};
    return sum_steps<kStep + 1, 1>(s, lane);
  } else {
    const bool odd = (lane >> kSumBits[kStep]) & 1;
    float s[kCount / 2];
#pragma unroll
    for (int i = 0; i < kCount / 2; ++i)
      s[i] = (odd ? v[2 * i + 1] : v[2 * i]) + partner<kStep>(odd ? v[2 * i] : v[2 * i + 1]);
    return sum_steps<kStep + 1, kCount / 2>(s, lane);
  }
}
template <int kLanes, int kGroup>
__device__ __forceinline__ float sum_tokens(const float (&v)[kGroup], int lane) {
  return sum_steps<sum_first(kLanes), kGroup>(v, lane);
}
// The token whose sum a lane ends up with, and whether it is the one lane that stores it.
template <int kLanes, int kGroup> __device__ __forceinline__ int token_of(int lane) {
  int t = 0, step = sum_first(kLanes);
#pragma unroll
  for (int k = 0; (1 << k) < kGroup; ++k) t |= ((lane >> kSumBits[step++]) & 1) << k;
  return t;
}
template <int kLanes, int kGroup> __device__ __forceinline__ bool writes_token(int lane) {
  int step = sum_first(kLanes);
#pragma unroll
  for (int k = 0; (1 << k) < kGroup; ++k) lane &= ~(1 << kSumBits[step++]);
  return lane == 0;
}

struct Args {
  SelScan s;
  int64_t span;          // tokens of a span (a multiple of kSpanTokens)
  int spans, D;
  int group_ch, group_tiles;   // channels of a group, workgroups that hold them
};

// The channels [first, end) of a workgroup: tiles do not cross from one group of B, C to the next.
struct Tile {
  int group, first, end;
};
__device__ __forceinline__ Tile tile_of(const Args& p, int ct, int channels) {
  Tile t;
  t.group = ct / p.group_tiles;
  t.first = t.group * p.group_ch + (ct % p.group_tiles) * channels;
  t.end = (t.group + 1) * p.group_ch;
  return t;
}

// kType, kDt: the types of the activations and of dt, -1 where they are only known at run time.  kFast: dt
// of a vector of channels is a vector (a decay per channel and state, headdim 1) or one head's (tied
// decay, headdim and group sizes multiples of kVec), and groups and states fill vectors.  The other form
// takes everything, element by element where it has to, and waits for its loads.
// Workspace of a cut scan: states [b, spans, d, n] (0: the initial state, c + 1: span c's from zero),
// then the spans' decays [b, spans, d].
// kTile: tokens of a tile.  kSV: channels of a thread's part of a tile, so that all threads have one.
// kPad: N is less than the lanes' states.  Those behind it hold no channel's state (B and C are 0 there, but
// 0 times an infinite delta u is NaN) and are left out of y: 8 x 2048 x 1536 x 8 205 us, 197 with them; 4 x 1000 x
// 24 heads of 64 x 100 160 and 157.  A form of its own, so that whole lanes pay nothing.
template <int kLanes, int kS, int kTile, int kSV, bool kTied, bool kStates, int kType, int kDt, bool kFast,
          bool kPad>
__global__ __launch_bounds__(kThreads, kS == 2 && kFast ? 3 : 1) void scan_kernel(Args p) {
  constexpr int kCh = kThreads / kLanes;            // channels of a workgroup
  constexpr int kN = kLanes * kS;                   // states, padded
  // Tokens whose operands are read together; with two states per lane as many as leave three waves per SIMD
  // (4 x 4096 x 5120 bf16: 565 us with eight and two waves, 503 with four and three; 8 x 2048 x 1536: 188, 196)
  constexpr int kGroup = kS > 4 || (kType == 0 && kS == 2) ? 2 : 4, kPair = 2 * kGroup;
  constexpr int kVecs = kCh / kSV;                  // vectors of a token's channels
  constexpr int kBcVecs = kTile * (kN / kVec);      // vectors of a tile of B (or C)
  constexpr int kBc = (kBcVecs + kThreads - 1) / kThreads;
  static_assert(kCh % kSV == 0 && 64 % kVecs == 0 && kVecs * kTile <= kThreads && kN % kVec == 0, "tile");
  // delta (or decay) and delta u of a tile, pairs of channels (16 bytes) exchanged by pair_slot; the sums
  // of y, rows apart by a quarter of the banks
  __shared__ __attribute__((aligned(16))) float s_du[kTile][kCh * 2];
  constexpr int kYRow = kCh + 16;
  __shared__ __attribute__((aligned(16))) float s_y[kStates ? 1 : kTile][kStates ? 4 : kYRow];
  __shared__ __attribute__((aligned(16))) float s_B[kTile][kN];
  __shared__ __attribute__((aligned(16))) float s_C[kStates ? 1 : kTile][kStates ? 4 : kN];

  __shared__ __attribute__((aligned(16))) float s_head[3][kCh];
  const SelScan& a = p.s;
  const int dtype = kType >= 0 ? kType : a.dtype, dt_dtype = kDt >= 0 ? kDt : a.dt_dtype;
  const int tid = threadIdx.x;
  const int nctile = p.group_tiles * (int)a.ngroups;
  const Tile tile = tile_of(p, (int)(blockIdx.x % nctile), kCh);
  const int group = tile.group;
  const int64_t rest = blockIdx.x / nctile;
  const int nsp = kStates ? p.spans - 1 : p.spans;
  const int span = (int)(rest % nsp);
  const int64_t b = rest / nsp;
  const int D = p.D, N = (int)a.dstate, P = (int)a.headdim;
  const int64_t L = a.seqlen;
  int64_t len = L;
  if (a.lengths) len = a.lengths[b] < 0 ? 0 : (a.lengths[b] < L ? a.lengths[b] : L);
  const int64_t t_begin = span * p.span;
  const int64_t t_end = t_begin + p.span < L ? t_begin + p.span : L;

  // the states of this lane
  const int ch = tid / kLanes, sub = tid % kLanes;
  using St = States<kLanes, kS>;
  const int d = tile.first + ch;
  const bool live = d < tile.end;
  float rate[kS], h[kS] = {};
  float* ws_decay = a.workspace + a.batch * p.spans * D * N;
  float* ws_state = a.workspace + (b * p.spans * D + d) * (int64_t)N;   // span 0
  const int64_t ws_span = (int64_t)D * N;
  const int64_t state_row = (b * D + d) * (int64_t)N;
#pragma unroll
  for (int i = 0; i < kS; ++i) rate[i] = 0.0f;
  if (live) {
    if constexpr (!kTied) {
      St::load(a.A + (int64_t)d * N, sub, N, rate);
#pragma unroll
      for (int i = 0; i < kS; ++i) rate[i] = decay_rate(rate[i]);
    }
    if constexpr (kStates) {
      if (span == 0) {   // the initial state into the workspace: the final one may overwrite it
        float init[kS] = {};
        if (a.init) St::load(a.init + state_row, sub, N, init);
        St::store(ws_state, sub, N, init);
      }
    } else if (p.spans == 1) {
      if (a.init) St::load(a.init + state_row, sub, N, h);
    } else {
      St::load(ws_state, sub, N, h);
      const float* decays = ws_decay + b * p.spans * D + d;
      constexpr int kAhead = 4;   // spans requested at a time
      for (int c = 0; c < span; c += kAhead) {
        float dec[kAhead], end[kAhead][kS];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int at = c + k < span ? c + k : span - 1;
          dec[k] = decays[(int64_t)at * D];
          St::load(ws_state + (at + 1) * ws_span, sub, N, end[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (c + k < span)
#pragma unroll
            for (int i = 0; i < kS; ++i) {
              const float f = kTied ? dec[k] : __builtin_amdgcn_exp2f(dec[k] * rate[i]);
              // a span's decay may be below the normal range, where none of its tokens' is: an infinite state stays
              // one, as it does token by token
              const bool stays = f == 0.0f && __builtin_fabsf(h[i]) == __builtin_inff();
              h[i] = __builtin_fmaf(stays ? 1.0f : f, h[i], end[k][i]);
            }
      }
    }
  }

  // what this thread brings in of a tile: a vector of channels of one token, vectors of B and C.  A last
  // vector that would pass the group's end (or N) is moved back to end there: the lanes it then shares
  // with its neighbour in the same wave carry the same values, and channels before the tile are left out.
  const int st = tid / kVecs;
  const bool stage = st < kTile;
  int c0 = tile.first + (tid % kVecs) * kSV;
  int nc = !stage || c0 >= tile.end ? 0 : kSV;
  if (nc > 0 && tile.end - c0 < kSV) {
    if (kFast) c0 = tile.end - kSV;
    else nc = tile.end - c0;
  }
  if (nc == 0) c0 = tile.first;   // for addresses that are not used
  // dt of a vector: a vector, one head's, several heads'
  const int mode = kFast ? (kTied ? 1 : 0) : 2;
  // of every channel: D, dt_bias and the tied rate, in LDS (a thread's own in registers cost it a wave per SIMD)
  for (int i = tid; i < kCh; i += kThreads) {
    const int c = tile.first + i;
    const bool in = c < tile.end;
    const int hd = in ? c / P : 0;
    s_head[0][i] = in && a.D ? a.D[hd] : 0.0f;
    s_head[1][i] = in && a.dt_bias ? a.dt_bias[hd] : 0.0f;
    if constexpr (kTied) s_head[2][i] = in ? decay_rate(a.A[hd]) : 0.0f;
  }
  const int lc = c0 - tile.first;   // of this thread's vector in LDS
  auto of_heads = [&](int what, float (&v)[kSV]) {
    if (kFast && lc % kSV == 0) {
      __builtin_memcpy(v, __builtin_assume_aligned(&s_head[what][lc], kSV > 2 ? 16 : 8), sizeof(v));
    } else {
#pragma unroll
      for (int i = 0; i < kSV; ++i) {
        const bool in = lc + i >= 0 && (kFast || i < nc);
        v[i] = in ? s_head[what][in ? lc + i : 0] : 0.0f;
      }
    }
  };
  const int es = dtype == 0 ? 4 : 2, ds = dt_dtype == 0 ? 4 : 2;
  auto column = [](const void* base, Rows r, int64_t batch, int64_t col, int size) {
    return static_cast<const char*>(base) + (batch * r.batch + col) * size;
  };
  const char* pu = column(a.u, a.ur, b, c0, es);
  const char* pz = column(a.z, a.zr, b, c0, es);
  const char* pdt = column(a.dt, a.dtr, b, c0 / P, ds);
  const char* pB = column(a.B, a.Br, b, (int64_t)group * N, es);
  const char* pC = column(a.C, a.Cr, b, (int64_t)group * N, es);
  const int64_t su = a.ur.token * es, sz = a.zr.token * es, sdt = a.dtr.token * ds,
                sB = a.Br.token * es, sC = a.Cr.token * es;
  const int64_t t_last = t_end < len ? t_end : len;   // tokens before it are read
  Raw<kSV> ru = {}, rz = {}, rdt = {};
  Raw<kVec> rB[kBc], rC[kStates ? 1 : kBc];
  auto bc_state = [&](int v) {   // first state of vector v of a tile of B, C
    const int n = (v % (kN / kVec)) * kVec;
    return kFast && n + kVec > N ? (n < N ? N - kVec : N) : n;
  };
  auto fetch = [&](int64_t t0) {
    const int64_t t = t0 + st;
    if (t < t_last && nc > 0) {
      if constexpr (kFast) {
        request_raw(ru, pu + t * su, dtype);
        if (!kStates && a.z) request_raw(rz, pz + t * sz, dtype);
      } else {
        request_part(ru, pu + t * su, dtype, nc);
        if (!kStates && a.z) request_part(rz, pz + t * sz, dtype, nc);
      }
      const char* row = pdt + t * sdt;
      if (mode == 0) {
        request_raw(rdt, row, dt_dtype);
      } else if (mode == 1) {
        rdt.w[0] = load_raw1(row, 0, dt_dtype);
      } else {
#pragma unroll
        for (int i = 0; i < kSV; ++i)
          if (i < nc) rdt.w[i] = load_raw1(row, (c0 + i) / P - c0 / P, dt_dtype);
      }
    }
#pragma unroll
    for (int k = 0; k < kBc; ++k) {
      const int v = tid + k * kThreads, n = bc_state(v);
      const int64_t tb = t0 + v / (kN / kVec);
      rB[k] = {};
      if constexpr (!kStates) rC[k] = {};
      if (v < kBcVecs && tb < t_last && n < N) {
        if constexpr (kFast) {
          request_raw(rB[k], pB + tb * sB + n * es, dtype);
          if constexpr (!kStates) request_raw(rC[k], pC + tb * sC + n * es, dtype);
        } else {
          request_part(rB[k], pB + tb * sB + n * es, dtype, N - n);
          if constexpr (!kStates) request_part(rC[k], pC + tb * sC + n * es, dtype, N - n);
        }
      }
    }
  };
  const int y_token = token_of<kLanes, kGroup>(sub);
  const bool y_writer = writes_token<kLanes, kGroup>(sub);
  // what no vector of B, C covers
  for (int i = tid; i < kTile * kN; i += kThreads) {
    (&s_B[0][0])[i] = 0.0f;
    if constexpr (!kStates) (&s_C[0][0])[i] = 0.0f;
  }
  __syncthreads();

  // A tile's y is stored behind the next tile's loads: loads and stores count down in one order, and the
  // wait for the loads, had it the store before it, would be for that too.
  float done[kSV] = {};
  auto put_y = [&](int64_t t0) {
    if (nc == 0 || t0 < t_begin || t0 + st >= t_end) return;
    const int64_t at = (b * L + t0 + st) * D + c0;
    if (lc >= 0) {
      store_as(a.y, at, dtype, kFast ? kSV : nc, done);
    } else {   // a vector moved back from the group's end: its last kSV + lc channels
      float own[kSV];
#pragma unroll
      for (int i = 0; i < kSV; ++i) own[i] = done[i];
      for (int k = lc; k < 0; ++k)
#pragma unroll
        for (int i = 0; i < kSV; ++i) own[i] = i + 1 < kSV ? own[i + 1] : 0.0f;
      store_as(a.y, at - lc, dtype, kSV + lc, own);
    }
  };
  float decay = kTied ? 1.0f : 0.0f;   // of the span (kStates)
  fetch(t_begin);
  for (int64_t t0 = t_begin; t0 < t_end; t0 += kTile) {
    Raw<kSV> ku, kz;
    const bool valid = t0 + st < t_last;
    // every load of this tile; said here, where every lane comes by, it spares the waits that the compiler
    // puts before the next requests on behalf of lanes that skip what follows
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
    if (nc > 0) {
      float dl[kSV], ml[kSV];
      float u[kSV];
      as_floats(ru, dtype, u);
      ku = ru, kz = rz;
      if (mode == 0) {
        as_floats(rdt, dt_dtype, dl);
      } else {
#pragma unroll
        for (int i = 0; i < kSV; ++i) dl[i] = as_float(rdt.w[mode == 1 ? 0 : i], dt_dtype);
      }
      of_heads(1, ml);
#pragma unroll
      for (int i = 0; i < kSV; ++i) dl[i] += ml[i];
      if (a.dt_softplus)
#pragma unroll
        for (int i = 0; i < kSV; ++i) dl[i] = softplus_fast(dl[i]);
      if (!valid)
#pragma unroll
        for (int i = 0; i < kSV; ++i) dl[i] = 0.0f, u[i] = 0.0f;
      if constexpr (kTied) of_heads(2, ml);
#pragma unroll
      for (int i = 0; i < kSV; ++i) {
        const float m = kTied ? __builtin_amdgcn_exp2f(dl[i] * ml[i]) : dl[i];
        dl[i] *= u[i];
        ml[i] = m;
      }
      if (kFast && lc % kSV == 0) {
#pragma unroll
        for (int i = 0; i < kSV; i += 2)
          *reinterpret_cast<float4*>(&s_du[st][4 * pair_slot<kCh, kSV>(st, (lc + i) / 2)]) =
              make_float4(ml[i], dl[i], ml[i + 1], dl[i + 1]);
      } else {
#pragma unroll
        for (int i = 0; i < kSV; ++i) {
          const int c = lc + i;
          if (c >= 0 && (kFast || i < nc))
            *reinterpret_cast<float2*>(&s_du[st][4 * pair_slot<kCh, kSV>(st, c / 2) + 2 * (c & 1)]) =
                make_float2(ml[i], dl[i]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kBc; ++k) {
      const int v = tid + k * kThreads, n = bc_state(v);
      if ((kBcVecs % kThreads == 0 || v < kBcVecs) && n < N) {
        const int row = v / (kN / kVec);
        auto keep = [&](const Raw<kVec>& r, float* dst) {
          float f[kVec];
          as_floats(r, dtype, f);
          if constexpr (kFast) {
            *reinterpret_cast<float4*>(dst) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(dst + 4) = make_float4(f[4], f[5], f[6], f[7]);
          } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) dst[i] = f[i];
          }
        };
        keep(rB[k], &s_B[row][n]);
        if constexpr (!kStates) keep(rC[k], &s_C[row][n]);
      }
    }
    if constexpr (!kStates) put_y(t0 - kTile);
    __syncthreads();
    if (t0 + kTile < t_end) fetch(t0 + kTile);
    // Tokens in groups of kGroup, the next group's operands on their way from LDS during one's arithmetic
    // (left to itself the compiler reads each token's right before their use, and a wave alone on its SIMD
    // waits out the LDS latency three times a token); within a group the exponentials, which depend on
    // nothing, come first.
    const int steps = t_end - t0 < kTile ? (int)(t_end - t0 + kPair - 1) / kPair * kPair : kTile;
    struct Token {
      float2 du;
      float B[kS], C[kStates ? 1 : kS];
    } q[2][kGroup];
    auto take = [&](int s0, Token (&g)[kGroup]) {
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        g[j].du = *reinterpret_cast<const float2*>(
            &s_du[s0 + j][4 * pair_slot<kCh, kSV>(s0 + j, ch / 2) + 2 * (ch & 1)]);
        St::take(s_B[s0 + j], sub, g[j].B);
        if constexpr (!kStates)
          St::take(s_C[s0 + j], sub, g[j].C);
      }
    };
    take(0, q[0]);
    for (int s0 = 0; s0 < steps; s0 += kPair) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int s1 = s0 + half * kGroup;
        Token(&g)[kGroup] = q[half];
        take(half == 0 ? s1 + kGroup : (s0 + kPair) % kTile, q[half ^ 1]);
        __builtin_amdgcn_sched_barrier(0);
        float m[kGroup][kS], y[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
#pragma unroll
          for (int i = 0; i < kS; ++i)
            m[j][i] = kTied ? g[j].du.x : __builtin_amdgcn_exp2f(g[j].du.x * rate[i]);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
          y[j] = 0.0f;
          float part = 0.0f;
#pragma unroll
          for (int i = 0; i < kS; ++i) {
            h[i] = __builtin_fmaf(m[j][i], h[i], g[j].du.y * g[j].B[i]);
            if constexpr (!kStates) {
              part = __builtin_fmaf(h[i], g[j].C[i], part);
              // kFast: N is a multiple of a piece, which is all there or not at all
              if (!kPad || !kFast || i % St::kPiece == St::kPiece - 1) {
                if (kPad) part = St::at(sub, i / St::kPiece) + (kFast ? 0 : i % St::kPiece) < N ? part : y[j];
                y[j] = part;
              }
            }
          }
          if constexpr (kStates) decay = kTied ? decay * g[j].du.x : decay + g[j].du.x;
        }
        if constexpr (!kStates) {
          const float sum = sum_tokens<kLanes, kGroup>(y, sub);
          if (y_writer) s_y[s1 + y_token][ch] = sum;
        }
      }
    }
    __syncthreads();
    if constexpr (!kStates) {
      if (nc > 0 && t0 + st < t_end) {
        float sum[kSV];
        if (kFast && lc % kSV == 0) {
          __builtin_memcpy(sum, __builtin_assume_aligned(&s_y[st][lc], kSV > 2 ? 16 : 8), sizeof(sum));
        } else {
#pragma unroll
          for (int i = 0; i < kSV; ++i) {
            const bool in = lc + i >= 0 && (kFast || i < nc);
            sum[i] = in ? s_y[st][in ? lc + i : 0] : 0.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < kSV; ++i) done[i] = sum[i];
        // u and z once more: as they lie in memory they take half the registers meanwhile
        float v[kSV], skip[kSV];
        as_floats(ku, dtype, v);
        of_heads(0, skip);
#pragma unroll
        for (int i = 0; i < kSV; ++i) done[i] = __builtin_fmaf(skip[i], v[i], done[i]);
        if (a.z) {
          as_floats(kz, dtype, v);
#pragma unroll
          for (int i = 0; i < kSV; ++i) done[i] *= silu(v[i]);
        }
        if (!valid)
#pragma unroll
          for (int i = 0; i < kSV; ++i) done[i] = 0.0f;
      }
    }
  }
  if constexpr (!kStates) put_y(t_begin + (t_end - t_begin - 1) / kTile * kTile);
  if (!live) return;
  if constexpr (kStates) {
    if (sub == 0) ws_decay[(b * p.spans + span) * D + d] = decay;
    St::store(ws_state + (span + 1) * ws_span, sub, N, h);
  } else if (a.final_state && span == p.spans - 1) {
    St::store(a.final_state + state_row, sub, N, h);
  }
}

// The forms of the kernel with types and layouts fixed at compile time, for the common sizes.
bool launch_fast(Args& p, hipStream_t st, hipError_t* e);

inline int64_t tiles_of(int64_t channels, int64_t groups, int64_t per) {
  return groups * ((channels / groups + per - 1) / per);
}

template <int kLanes, int kS, int kTile, int kSV, bool kTied, int kType, int kDt, bool kFast>
hipError_t launch_form(Args& p, hipStream_t st) {
  p.group_tiles = (int)tiles_of(p.group_ch, 1, kThreads / kLanes);
  const int64_t tiles = p.s.batch * p.s.ngroups * p.group_tiles;
  if (p.spans > 1) {
    scan_kernel<kLanes, kS, kTile, kSV, kTied, true, kType, kDt, kFast, false>
        <<<dim3((unsigned)(tiles * (p.spans - 1))), kThreads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  auto walk = [&](auto pad) {
    scan_kernel<kLanes, kS, kTile, kSV, kTied, false, kType, kDt, kFast, decltype(pad)::value>
        <<<dim3((unsigned)(tiles * p.spans)), kThreads, 0, st>>>(p);
  };
  if (p.s.dstate < kLanes * kS) walk(std::true_type());
  else walk(std::false_type());
  return hipGetLastError();
}

}  // namespace sel_scan
}  // namespace ssdi8
