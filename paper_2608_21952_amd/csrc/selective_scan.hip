// Selective state space scan: for every batch element and channel d of head h = d / P and group g
//   delta[t] = softplus(dt[t, h] + dt_bias[h])
//   s[t, n]  = exp(delta[t] A[d, n]) s[t-1, n] + delta[t] u[t, d] B[t, g, n]
//   y[t, d]  = (sum_n C[t, g, n] s[t, n] + D[h] u[t, d]) silu(z[t, d])
// with one decay per channel and state (A [d, n]) or per head (`tied`, A [h]), any length, from a
// given state.  The steps of several orders of magnitude more tokens than lanes are serial per
// (channel, state), so the work is laid over channels and states:
//   kLanes neighbouring lanes hold a channel, each kS of its states in registers; a workgroup of 256
//   threads holds 256 / kLanes channels and walks tiles of kTile tokens.  A tile's inputs come in
//   coalesced, are turned once into delta (or the tied decay) and delta u, and into fp32 B and C, in
//   LDS, where every lane of a channel reads them; the next tile's loads are in flight meanwhile.  The
//   lanes' partial sums of y meet by lane moves and leave through LDS, again coalesced.
// Few channels over many tokens are cut into spans: a first kernel leaves, per span, the state it
// reaches from zero and its decay (the sum of delta, or the tied decays' product); in the second the
// workgroup of a span joins those of the spans before it and walks its own.
//
// What bounds it: the vector unit.  Per (token, channel, state) one exponential on the quarter-rate
// unit and four full-rate operations, or three operations alone where the decay is tied.
//
// Everything is held in fp32; y is rounded once.  Tokens at or behind a sequence's length count as
// delta = 0 and u = 0, which leave the state as it is, and are not read.
#include <type_traits>

#include "block.hpp"

namespace ssdi8 {

namespace {

constexpr int kTile = 32;
constexpr int kThreads = 256;

// kVec elements as they lie in memory (8 words of fp32, 4 of a 16-bit type), turned into fp32 later.
struct Raw {
  uint32_t w[kVec];
};
__device__ __forceinline__ Raw load_raw(const void* base, int64_t off, int dtype, int n) {
  Raw r = {};
  if (dtype == 0) {
    const uint32_t* p = static_cast<const uint32_t*>(base) + off;
    if (n >= kVec) {
      __builtin_memcpy(r.w, p, 32);
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (i < n) r.w[i] = p[i];
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(base) + off;
    if (n >= kVec) {
      __builtin_memcpy(r.w, p, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (i < n) r.w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    }
  }
  return r;
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
__device__ __forceinline__ void as_floats(const Raw& r, int dtype, float (&out)[kVec]) {
  if (dtype == 0) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) out[i] = __builtin_bit_cast(float, r.w[i]);
  } else if (dtype == 1) {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      out[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i / 2] >> (16 * (i & 1))));
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      out[i] = __builtin_bit_cast(float, i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
  }
}
__device__ __forceinline__ void store_as(void* base, int64_t off, int dtype, int n,
                                         const float (&v)[kVec]) {
  if (dtype == 0) store_vec<float>(static_cast<float*>(base) + off, n, v);
  else if (dtype == 1) store_vec<_Float16>(static_cast<_Float16*>(base) + off, n, v);
  else store_vec<bf16>(static_cast<bf16*>(base) + off, n, v);
}

// A in base 2; -inf (a decay of 0 for any positive delta) stays finite, so that delta = 0 gives 1.
__device__ __forceinline__ float decay_rate(float A) {
  const float a = A * kLog2eF;
  return a == -__builtin_inff() ? -__FLT_MAX__ : a;
}

struct Args {
  SelScan s;
  int64_t span;          // tokens of a span (a multiple of kTile)
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

// Workspace of a cut scan: states [b, spans, d, n] (0: the initial state, c + 1: span c's from zero),
// then the spans' decays [b, spans, d].
template <int kLanes, int kS, bool kTied, bool kStates>
__global__ __launch_bounds__(kThreads) void scan_kernel(Args p) {
  constexpr int kCh = kThreads / kLanes;            // channels of a workgroup
  constexpr int kN = kLanes * kS;                   // states, padded
  constexpr int kVecs = kCh / kVec;                 // vectors of a token's channels
  constexpr int kBcVecs = kTile * (kN / kVec);      // vectors of a tile of B (or C)
  constexpr int kBc = (kBcVecs + kThreads - 1) / kThreads;
  static_assert(kCh % kVec == 0 && kVecs * kTile <= kThreads && kN % kVec == 0, "tile");
  __shared__ __attribute__((aligned(16))) float s_du[kTile][kCh][2];   // delta (or decay), delta u
  __shared__ __attribute__((aligned(16))) float s_B[kTile][kN];
  __shared__ __attribute__((aligned(16))) float s_C[kStates ? 1 : kTile][kStates ? 4 : kN];

  const SelScan& a = p.s;
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
  const int ch = tid / kLanes, sub = tid % kLanes, n0 = sub * kS;
  const int d = tile.first + ch;
  const bool live = d < tile.end;
  float rate[kS], h[kS];
  float* ws_decay = a.workspace + a.batch * p.spans * D * N;
  const int64_t ws_row = ((b * p.spans) * D + d) * (int64_t)N + n0;   // span 0
  const int64_t ws_span = (int64_t)D * N;
#pragma unroll
  for (int i = 0; i < kS; ++i) {
    const bool in = live && n0 + i < N;
    rate[i] = kTied ? 0.0f : (in ? decay_rate(a.A[(int64_t)d * N + n0 + i]) : 0.0f);
    h[i] = 0.0f;
    if (kStates) {
      if (span == 0 && in)   // the initial state into the workspace: the final one may overwrite it
        a.workspace[ws_row + i] = a.init ? a.init[(b * D + d) * (int64_t)N + n0 + i] : 0.0f;
    } else if (p.spans == 1) {
      if (a.init && in) h[i] = a.init[(b * D + d) * (int64_t)N + n0 + i];
    }
  }
  if (!kStates && p.spans > 1 && live) {
#pragma unroll
    for (int i = 0; i < kS; ++i)
      if (n0 + i < N) h[i] = a.workspace[ws_row + i];
    for (int c = 0; c < span; ++c) {
      const float dec = ws_decay[(b * p.spans + c) * D + d];
#pragma unroll
      for (int i = 0; i < kS; ++i)
        if (n0 + i < N) {
          const float m = kTied ? dec : __builtin_amdgcn_exp2f(dec * rate[i]);
          h[i] = __builtin_fmaf(m, h[i], a.workspace[ws_row + (c + 1) * ws_span + i]);
        }
    }
  }

  // what this thread brings in of a tile: a vector of channels of one token, vectors of B and C
  const int st = tid / kVecs, c0 = tile.first + (tid % kVecs) * kVec;
  const bool stage = st < kTile;
  const int nc = !stage || c0 >= tile.end ? 0 : (tile.end - c0 < kVec ? tile.end - c0 : kVec);
  // dt of a vector: a vector, one head's (heads and tiles begin at multiples of kVec), several heads'
  const int mode = P == 1 ? 0 : (P % kVec == 0 && p.group_ch % kVec == 0 ? 1 : 2);
  float head_D[kVec], head_bias[kVec], head_rate[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int hd = i < nc ? (c0 + i) / P : 0;
    head_D[i] = a.D && i < nc ? a.D[hd] : 0.0f;
    head_bias[i] = a.dt_bias && i < nc ? a.dt_bias[hd] : 0.0f;
    head_rate[i] = kTied && i < nc ? decay_rate(a.A[hd]) : 0.0f;
  }
  Raw ru = {}, rz = {}, rdt = {}, rB[kBc], rC[kStates ? 1 : kBc];
  auto fetch = [&](int64_t t0) {
    const int64_t t = t0 + st;
    const int n = t < t_end && t < len ? nc : 0;
    if (n > 0) {
      ru = load_raw(a.u, b * a.ur.batch + t * a.ur.token + c0, a.dtype, n);
      if (!kStates && a.z)
        rz = load_raw(a.z, b * a.zr.batch + t * a.zr.token + c0, a.dtype, n);
      const int64_t row = b * a.dtr.batch + t * a.dtr.token;
      if (mode == 0) {
        rdt = load_raw(a.dt, row + c0, a.dt_dtype, n);
      } else if (mode == 1) {
        rdt.w[0] = load_raw1(a.dt, row + c0 / P, a.dt_dtype);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (i < n) rdt.w[i] = load_raw1(a.dt, row + (c0 + i) / P, a.dt_dtype);
      }
    }
#pragma unroll
    for (int k = 0; k < kBc; ++k) {
      const int v = tid + k * kThreads;
      const int64_t tb = t0 + v / (kN / kVec);
      const int n = (v % (kN / kVec)) * kVec;
      const int m = v < kBcVecs && tb < t_end && tb < len && n < N ? (N - n < kVec ? N - n : kVec) : 0;
      rB[k] = Raw{};
      if (!kStates) rC[k] = Raw{};
      if (m > 0) {
        rB[k] = load_raw(a.B, b * a.Br.batch + tb * a.Br.token + (int64_t)group * N + n, a.dtype, m);
        if (!kStates)
          rC[k] = load_raw(a.C, b * a.Cr.batch + tb * a.Cr.token + (int64_t)group * N + n, a.dtype, m);
      }
    }
  };

  float decay = kTied ? 1.0f : 0.0f;   // of the span (kStates)
  fetch(t_begin);
  for (int64_t t0 = t_begin; t0 < t_end; t0 += kTile) {
    float u[kVec], z[kVec];
    const bool valid = t0 + st < t_end && t0 + st < len;
    if (stage) {
      float dl[kVec];
      as_floats(ru, a.dtype, u);
      if (!kStates && a.z) as_floats(rz, a.dtype, z);
      if (mode == 0) {
        as_floats(rdt, a.dt_dtype, dl);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) dl[i] = as_float(rdt.w[mode == 1 ? 0 : i], a.dt_dtype);
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        float v = dl[i] + head_bias[i];
        v = a.dt_softplus ? softplus_fast(v) : v;
        const bool in = valid && i < nc;
        dl[i] = in ? v : 0.0f;
        u[i] = in ? u[i] : 0.0f;
      }
      float* dst = &s_du[st][(tid % kVecs) * kVec][0];
#pragma unroll
      for (int i = 0; i < kVec; i += 2) {
        float4 q;
        q.x = kTied ? __builtin_amdgcn_exp2f(dl[i] * head_rate[i]) : dl[i];
        q.y = dl[i] * u[i];
        q.z = kTied ? __builtin_amdgcn_exp2f(dl[i + 1] * head_rate[i + 1]) : dl[i + 1];
        q.w = dl[i + 1] * u[i + 1];
        *reinterpret_cast<float4*>(dst + 2 * i) = q;
      }
    }
#pragma unroll
    for (int k = 0; k < kBc; ++k) {
      const int v = tid + k * kThreads;
      if (kBcVecs % kThreads == 0 || v < kBcVecs) {
        float q[kVec];
        as_floats(rB[k], a.dtype, q);
        float4* dst = reinterpret_cast<float4*>(&s_B[0][0] + v * kVec);
        dst[0] = make_float4(q[0], q[1], q[2], q[3]);
        dst[1] = make_float4(q[4], q[5], q[6], q[7]);
        if constexpr (!kStates) {
          as_floats(rC[k], a.dtype, q);
          dst = reinterpret_cast<float4*>(&s_C[0][0] + v * kVec);
          dst[0] = make_float4(q[0], q[1], q[2], q[3]);
          dst[1] = make_float4(q[4], q[5], q[6], q[7]);
        }
      }
    }
    __syncthreads();
    if (t0 + kTile < t_end) fetch(t0 + kTile);
    const int steps = t_end - t0 < kTile ? (int)((t_end - t0 + 3) & ~3) : kTile;
    for (int s4 = 0; s4 < steps; s4 += 4) {
      float ysel = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int s = s4 + j;
        const float2 du = *reinterpret_cast<const float2*>(&s_du[s][ch][0]);
        float Bv[kS], Cv[kS];
#pragma unroll
        for (int i = 0; i < kS; i += 4) {
          *reinterpret_cast<float4*>(&Bv[i]) = *reinterpret_cast<const float4*>(&s_B[s][n0 + i]);
          if constexpr (!kStates)
            *reinterpret_cast<float4*>(&Cv[i]) = *reinterpret_cast<const float4*>(&s_C[s][n0 + i]);
        }
        float y = 0.0f;
#pragma unroll
        for (int i = 0; i < kS; ++i) {
          const float m = kTied ? du.x : __builtin_amdgcn_exp2f(du.x * rate[i]);
          h[i] = __builtin_fmaf(m, h[i], du.y * Bv[i]);
          if constexpr (!kStates) y = __builtin_fmaf(h[i], Cv[i], y);
        }
        if constexpr (kStates) {
          decay = kTied ? decay * du.x : decay + du.x;
        } else {
          y = lane_sum<kLanes>(y);
          if (sub == j) ysel = y;
        }
      }
      if constexpr (!kStates)
        if (sub < 4) s_du[s4 + sub][ch][0] = ysel;   // read by this wave alone, and done
    }
    __syncthreads();
    if constexpr (!kStates) {
      if (nc > 0 && t0 + st < t_end) {
        float y[kVec];
        const float* src = &s_du[st][(tid % kVecs) * kVec][0];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          float v = __builtin_fmaf(head_D[i], u[i], src[2 * i]);
          if (a.z) v *= silu(z[i]);
          y[i] = valid ? v : 0.0f;
        }
        store_as(a.y, (b * L + t0 + st) * D + c0, a.dtype, nc, y);
      }
    }
  }
  if (!live) return;
  if (kStates) {
    if (sub == 0) ws_decay[(b * p.spans + span) * D + d] = decay;
#pragma unroll
    for (int i = 0; i < kS; ++i)
      if (n0 + i < N) a.workspace[ws_row + (span + 1) * ws_span + i] = h[i];
  } else if (a.final_state && span == p.spans - 1) {
#pragma unroll
    for (int i = 0; i < kS; ++i)
      if (n0 + i < N) a.final_state[(b * D + d) * (int64_t)N + n0 + i] = h[i];
  }
}

template <typename F> hipError_t for_states(int64_t N, F&& f) {
  using std::integral_constant;
  if (N <= 16) return f(integral_constant<int, 4>(), integral_constant<int, 4>());
  if (N <= 32) return f(integral_constant<int, 8>(), integral_constant<int, 4>());
  if (N <= 64) return f(integral_constant<int, 16>(), integral_constant<int, 4>());
  if (N <= 128) return f(integral_constant<int, 16>(), integral_constant<int, 8>());
  return f(integral_constant<int, 32>(), integral_constant<int, 8>());
}
int lanes_of(int64_t N) { return N <= 16 ? 4 : N <= 32 ? 8 : N <= 128 ? 16 : 32; }

int64_t tiles_of(int64_t channels, int64_t groups, int64_t per) {
  return groups * ((channels / groups + per - 1) / per);
}

// ---------------------------------------------------------------------------- one token
// kLanes lanes hold a channel, four states each: neighbouring ones (kWide: one 16-byte access, N a
// multiple of 4) or every kLanes-th.  A lane takes kRun channels, whose states are all requested
// before the first is used.
template <int kLanes, int kRun, bool kWide>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(Args p, float* state) {
  constexpr int kCh = kThreads / kLanes;
  const SelScan& a = p.s;
  const int nctile = p.group_tiles * (int)a.ngroups;
  const Tile tile = tile_of(p, (int)(blockIdx.x % nctile), kCh * kRun);
  const int64_t b = blockIdx.x / nctile;
  const int sub = threadIdx.x % kLanes, ch = threadIdx.x / kLanes;
  const int D = p.D, N = (int)a.dstate, P = (int)a.headdim;
  auto at = [&](int i) { return kWide ? sub * 4 + i : sub + kLanes * i; };
  auto value = [&](const void* t, int64_t off, int dtype) { return as_float(load_raw1(t, off, dtype), dtype); };

  float h[kRun][4], u[kRun], dt[kRun], z[kRun];
#pragma unroll
  for (int r = 0; r < kRun; ++r) {
    const int d = tile.first + r * kCh + ch;
    const bool live = d < tile.end;
    const float* sd = state + (b * D + d) * (int64_t)N;
    if (kWide) {
      float4 q = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (live && at(0) < N) q = *reinterpret_cast<const float4*>(sd + at(0));
      h[r][0] = q.x, h[r][1] = q.y, h[r][2] = q.z, h[r][3] = q.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) h[r][i] = live && at(i) < N ? sd[at(i)] : 0.0f;
    }
    u[r] = live ? value(a.u, b * a.ur.batch + d, a.dtype) : 0.0f;
    dt[r] = live ? value(a.dt, b * a.dtr.batch + d / P, a.dt_dtype) : 0.0f;
    z[r] = live && a.z ? value(a.z, b * a.zr.batch + d, a.dtype) : 0.0f;
  }
  float Bv[4], Cv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = at(i);
    Bv[i] = n < N ? value(a.B, b * a.Br.batch + (int64_t)tile.group * N + n, a.dtype) : 0.0f;
    Cv[i] = n < N ? value(a.C, b * a.Cr.batch + (int64_t)tile.group * N + n, a.dtype) : 0.0f;
  }
#pragma unroll
  for (int r = 0; r < kRun; ++r) {
    const int d = tile.first + r * kCh + ch;
    const bool live = d < tile.end;
    const int hd = live ? d / P : 0;
    float delta = dt[r] + (a.dt_bias ? a.dt_bias[hd] : 0.0f);
    if (a.dt_softplus) delta = softplus_fast(delta);
    const float du = delta * u[r];
    float tied = 0.0f, y = 0.0f;
    if (a.tied) tied = __builtin_amdgcn_exp2f(delta * decay_rate(a.A[hd]));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = at(i);
      float m = tied;
      if (!a.tied)
        m = live && n < N ? __builtin_amdgcn_exp2f(delta * decay_rate(a.A[(int64_t)d * N + n])) : 0.0f;
      h[r][i] = n < N ? __builtin_fmaf(m, h[r][i], du * Bv[i]) : 0.0f;
      y = __builtin_fmaf(h[r][i], Cv[i], y);
    }
    y = lane_sum<kLanes>(y);
    if (!live) continue;
    float* sd = state + (b * D + d) * (int64_t)N;
    if (kWide) {
      if (at(0) < N)
        *reinterpret_cast<float4*>(sd + at(0)) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (at(i) < N) sd[at(i)] = h[r][i];
    }
    if (sub == 0) {
      y = __builtin_fmaf(a.D ? a.D[hd] : 0.0f, u[r], y);
      if (a.z) y *= silu(z[r]);
      const int64_t o = b * D + d;
      if (a.dtype == 0) static_cast<float*>(a.y)[o] = y;
      else if (a.dtype == 1) static_cast<_Float16*>(a.y)[o] = (_Float16)y;
      else static_cast<bf16*>(a.y)[o] = (bf16)y;
    }
  }
}

}  // namespace

int sel_scan_spans(int64_t batch, int64_t seqlen, int64_t channels, int64_t groups, int64_t dstate) {
  const int64_t wgs = batch * tiles_of(channels, groups, kThreads / lanes_of(dstate));
  if (wgs >= 256 || wgs == 0) return 1;
  const int64_t most = (seqlen + 127) / 128;
  int64_t spans = 1024 / wgs;
  if (spans > most) spans = most;
  return spans < 2 ? 1 : (int)spans;
}

int64_t sel_scan_workspace(int64_t batch, int64_t seqlen, int64_t channels, int64_t groups,
                           int64_t dstate) {
  const int64_t spans = sel_scan_spans(batch, seqlen, channels, groups, dstate);
  return spans == 1 ? 0 : batch * spans * channels * (dstate + 1);
}

hipError_t launch_sel_scan(const SelScan& a, hipStream_t st) {
  Args p;
  p.s = a;
  p.D = (int)(a.nheads * a.headdim);
  p.group_ch = p.D / (int)a.ngroups;
  p.spans = sel_scan_spans(a.batch, a.seqlen, p.D, a.ngroups, a.dstate);
  const int64_t tokens = (a.seqlen + p.spans - 1) / p.spans;
  p.span = (tokens + kTile - 1) / kTile * kTile;
  // rounding up may leave spans without tokens: fewer are launched
  if (p.span > 0) p.spans = (int)((a.seqlen + p.span - 1) / p.span);
  if (p.spans < 1) p.spans = 1;
  return for_states(a.dstate, [&](auto lanes, auto states) {
    constexpr int kLanes = decltype(lanes)::value, kS = decltype(states)::value;
    p.group_tiles = (int)tiles_of(p.group_ch, 1, kThreads / kLanes);
    const int64_t tiles = a.batch * a.ngroups * p.group_tiles;
    auto go = [&](auto tied) {
      constexpr bool kTied = decltype(tied)::value;
      if (p.spans > 1) {
        scan_kernel<kLanes, kS, kTied, true>
            <<<dim3((unsigned)(tiles * (p.spans - 1))), kThreads, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
      scan_kernel<kLanes, kS, kTied, false>
          <<<dim3((unsigned)(tiles * p.spans)), kThreads, 0, st>>>(p);
      return hipGetLastError();
    };
    return a.tied ? go(std::true_type()) : go(std::false_type());
  });
}

hipError_t launch_sel_scan_step(const SelScan& a, float* state, hipStream_t st) {
  Args p;
  p.s = a;
  p.D = (int)(a.nheads * a.headdim);
  p.group_ch = p.D / (int)a.ngroups;
  p.spans = 1;
  p.span = 1;
  auto go = [&](auto lanes, auto run, auto wide) {
    constexpr int kLanes = decltype(lanes)::value, kRun = decltype(run)::value;
    p.group_tiles = (int)tiles_of(p.group_ch, 1, kThreads / kLanes * kRun);
    const int64_t grid = a.batch * a.ngroups * p.group_tiles;
    scan_step_kernel<kLanes, kRun, decltype(wide)::value>
        <<<dim3((unsigned)grid), kThreads, 0, st>>>(p, state);
    return hipGetLastError();
  };
  using std::integral_constant;
  auto by_run = [&](auto lanes, auto wide) {
    // four channels per lane once a channel each would already give every CU eight workgroups
    const int64_t wgs = a.batch * p.D / (kThreads / decltype(lanes)::value);
    return wgs >= 2048 ? go(lanes, integral_constant<int, 4>(), wide)
                       : go(lanes, integral_constant<int, 1>(), wide);
  };
  auto by_wide = [&](auto lanes) {
    return a.dstate % 4 == 0 ? by_run(lanes, std::true_type()) : by_run(lanes, std::false_type());
  };
  const int64_t N = a.dstate;
  if (N <= 16) return by_wide(integral_constant<int, 4>());
  if (N <= 32) return by_wide(integral_constant<int, 8>());
  if (N <= 64) return by_wide(integral_constant<int, 16>());
  if (N <= 128) return by_wide(integral_constant<int, 32>());
  return by_wide(integral_constant<int, 64>());
}

}  // namespace ssdi8
