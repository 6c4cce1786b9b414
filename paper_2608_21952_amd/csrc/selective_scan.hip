// Selective state space scan: for every batch element and channel d of head h = d / P and group g
//   delta[t] = softplus(dt[t, h] + dt_bias[h])
//   s[t, n]  = exp(delta[t] A[d, n]) s[t-1, n] + delta[t] u[t, d] B[t, g, n]
//   y[t, d]  = (sum_n C[t, g, n] s[t, n] + D[h] u[t, d]) silu(z[t, d])
// with one decay per channel and state (A [d, n]) or per head (`tied`, A [h]), any length, from a
// given state.  A (channel, state)'s tokens are serial, so the work is laid over channels and states:
//   kLanes neighbouring lanes hold a channel, each kS of its states in registers; a workgroup of 256
//   threads holds 256 / kLanes channels and walks tiles of kTile tokens.  A tile's inputs come in
//   coalesced, are turned once into delta (or the tied decay) and delta u, and into fp32 B and C, in
//   LDS, where every lane of a channel reads them; the next tile's loads are in flight meanwhile.  The
//   lanes' partial sums of y meet by lane moves and leave through LDS, again coalesced.
// Few channels over many tokens are cut into spans: a first kernel leaves, per span, the state it
// reaches from zero and its decay (the sum of delta, or the tied decays' product); in the second the
// workgroup of a span joins those of the spans before it and walks its own.
//
// What bounds it: the vector unit.  Per (token, channel, state) one exponential at half rate and four
// full-rate operations (three alone where the decay is tied), 61 us over the card's 1024 SIMDs for 8 x 2048 x
// 1536 x 16; softplus, gate and conversions of every element take about as long as half of that, the sums
// over a channel's lanes a quarter.  Measured there 197 us (fp16 with gate; 1.5 workgroups per CU, so that the
// fuller ones decide), 504 us for 4 x 4096 x 5120 x 16 in bf16, 220 us for one fp32 prompt of 16384 x 1536, 36 us
// for three remainders of 201 tokens, 24 heads of 64 x 128.
//
// Everything is held in fp32; y is rounded once.  Tokens at or behind a sequence's length count as
// delta = 0 and u = 0, which leave the state as it is, and are not read.
#include "selective_scan.hpp"

namespace ssdi8 {

namespace {

using namespace sel_scan;

template <typename F> hipError_t for_states(int64_t N, F&& f) {
  using std::integral_constant;
  if (N <= 16) return f(integral_constant<int, 8>(), integral_constant<int, 2>());
  if (N <= 32) return f(integral_constant<int, 8>(), integral_constant<int, 4>());
  if (N <= 64) return f(integral_constant<int, 16>(), integral_constant<int, 4>());
  if (N <= 128) return f(integral_constant<int, 16>(), integral_constant<int, 8>());
  return f(integral_constant<int, 32>(), integral_constant<int, 8>());
}
int lanes_of(int64_t N) { return N <= 32 ? 8 : N <= 128 ? 16 : 32; }

// ---------------------------------------------------------------------------- one token
// kLanes lanes hold a channel, four states each: neighbouring ones (kWide: one 16-byte access, N a
// multiple of 4) or every kLanes-th.  A lane takes kRun channels, whose states are all requested first;
// meanwhile a thread per channel forms what all its lanes need (delta or the tied decay, delta u), and
// later its y.  What bounds it: the states' bytes, read and written once: 128 x 5120 channels x 128 states in
// 127 us, 5.3 TB/s, the rate of a large copy.
template <int kLanes, int kRun, bool kWide>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(Args p, float* state) {
  constexpr int kCh = kThreads / kLanes, kAll = kCh * kRun;
  static_assert(kAll <= kThreads, "a thread per channel");
  __shared__ float2 s_du[kAll];
  __shared__ float s_y[kAll];
  const SelScan& a = p.s;
  const int nctile = p.group_tiles * (int)a.ngroups;
  const Tile tile = tile_of(p, (int)(blockIdx.x % nctile), kAll);
  const int64_t b = blockIdx.x / nctile;
  const int sub = threadIdx.x % kLanes, ch = threadIdx.x / kLanes;
  const int D = p.D, N = (int)a.dstate, P = (int)a.headdim;
  auto at = [&](int i) { return kWide ? sub * 4 + i : sub + kLanes * i; };
  auto value = [&](const void* t, int64_t off, int dtype) { return as_float(load_raw1(t, off, dtype), dtype); };
  // four values of a row of N, 0 behind its end
  auto four = [&](const float* row, bool live, float (&v)[4]) {
    if (kWide) {
      float4 q = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (live && at(0) < N) __builtin_memcpy(&q, row + at(0), 16);
      v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = live && at(i) < N ? row[at(i)] : 0.0f;
    }
  };

  float h[kRun][4], Bv[4], Cv[4];
#pragma unroll
  for (int r = 0; r < kRun; ++r) {
    const int d = tile.first + r * kCh + ch;
    four(state + (b * D + d) * (int64_t)N, d < tile.end, h[r]);
  }
  auto column = [&](const void* t, int64_t row, float (&v)[4]) {
    const char* q = static_cast<const char*>(t) + (row + (int64_t)tile.group * N) * (a.dtype == 0 ? 4 : 2);
    if (kWide && a.dtype != 0) {
      Raw<4> raw = {};
      if (at(0) < N) __builtin_memcpy(raw.w, q + 2 * at(0), 8);
      as_floats(raw, a.dtype, v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = at(i) < N ? value(q, at(i), a.dtype) : 0.0f;
    }
  };
  column(a.B, b * a.Br.batch, Bv);
  column(a.C, b * a.Cr.batch, Cv);
  // the channel of this thread
  const int own = tile.first + (int)threadIdx.x;
  const bool has = (int)threadIdx.x < kAll && own < tile.end;
  float skip = 0.0f, gate = 1.0f;
  if (has) {
    const int hd = own / P;
    const float u = value(a.u, b * a.ur.batch + own, a.dtype);
    float delta = value(a.dt, b * a.dtr.batch + hd, a.dt_dtype);
    if (a.z) gate = silu(value(a.z, b * a.zr.batch + own, a.dtype));
    if (a.D) skip = a.D[hd] * u;
    if (a.dt_bias) delta += a.dt_bias[hd];
    if (a.dt_softplus) delta = softplus_fast(delta);
    s_du[threadIdx.x] =
        make_float2(a.tied ? __builtin_amdgcn_exp2f(delta * decay_rate(a.A[hd])) : delta, delta * u);
  }
  __syncthreads();
  float y[kRun];
#pragma unroll
  for (int r = 0; r < kRun; ++r) {
    const int d = tile.first + r * kCh + ch;
    const bool live = d < tile.end;
    const float2 du = s_du[r * kCh + ch];   // of a channel behind the group's end: not used
    float m[4];
    if (a.tied) {
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = du.x;
    } else {
      four(a.A + (int64_t)d * N, live, m);
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = __builtin_amdgcn_exp2f(du.x * decay_rate(m[i]));
    }
    y[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[r][i] = live && at(i) < N ? __builtin_fmaf(m[i], h[r][i], du.y * Bv[i]) : 0.0f;
      y[r] = __builtin_fmaf(h[r][i], Cv[i], y[r]);
    }
    if (live) {
      float* sd = state + (b * D + d) * (int64_t)N;
      if (kWide) {
        if (at(0) < N)
          *reinterpret_cast<float4*>(sd + at(0)) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at(i) < N) sd[at(i)] = h[r][i];
      }
    }
  }
  lane_sums<kLanes, kRun>(y);
  if (sub == 0)
#pragma unroll
    for (int r = 0; r < kRun; ++r) s_y[r * kCh + ch] = y[r];
  __syncthreads();
  if (has) {
    const float v = (s_y[threadIdx.x] + skip) * gate;
    const int64_t o = b * D + own;
    if (a.dtype == 0) static_cast<float*>(a.y)[o] = v;
    else if (a.dtype == 1) static_cast<_Float16*>(a.y)[o] = (_Float16)v;
    else static_cast<bf16*>(a.y)[o] = (bf16)v;
  }
}

}  // namespace

int sel_scan_spans(int64_t batch, int64_t seqlen, int64_t channels, int64_t groups, int64_t dstate) {
  const int64_t wgs = batch * tiles_of(channels, groups, kThreads / lanes_of(dstate));
  // Uncut from a workgroup per CU on: a cut costs the walk a second time, less what only y needs (8 x 2048 x
  // 1536 x 16, 384 workgroups: 196 us uncut, 199 in 2 spans; 4 x 4096 x 5120, 640: 503 and 584; against it, a
  // tied decay of 80 heads over 2000 tokens, 320: 307 and 268).  Below, three workgroups per CU (1 x 16384 x
  // 1536 fp32, 48: 905 us uncut; 265, 220 and 240 in 10, 16 and 21 spans), of 128 tokens or more.
  if (wgs >= 256 || wgs == 0) return 1;
  const int64_t most = (seqlen + 127) / 128;
  int64_t spans = 768 / wgs;
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
  p.span = (tokens + kSpanTokens - 1) / kSpanTokens * kSpanTokens;
  // rounding up may leave spans without tokens: fewer are launched
  if (p.span > 0) p.spans = (int)((a.seqlen + p.span - 1) / p.span);
  if (p.spans < 1) p.spans = 1;
  hipError_t e = hipSuccess;
  if (launch_fast(p, st, &e)) return e;
  return for_states(a.dstate, [&](auto lanes, auto states) {
    constexpr int kLanes = decltype(lanes)::value, kS = decltype(states)::value;
    return a.tied ? launch_form<kLanes, kS, 32, 8, true, -1, -1, false>(p, st)
                  : launch_form<kLanes, kS, 32, 8, false, -1, -1, false>(p, st);
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
