// C ABI of the operators around the SSD layer (declared in include/ssdi8.h): argument validation and
// launches on the caller's stream.
#include "ssdi8.h"

#include <hip/hip_runtime.h>

#include "block.hpp"

namespace {

constexpr int64_t kMaxSize = (int64_t)1 << 31;    // of one dimension
constexpr double kMaxCount = 4.0e12;              // of a tensor's elements
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // elements
constexpr double kMaxGrid = 2147483647.0 / 2;     // workgroups

bool off(const void* p, uintptr_t align) { return ((uintptr_t)p & (align - 1)) != 0; }
bool is_float(int dtype) {
  return dtype == SSDI8_F32 || dtype == SSDI8_F16 || dtype == SSDI8_BF16;
}
uintptr_t size_of(int dtype) { return dtype == SSDI8_F32 ? 4 : dtype == SSDI8_I8 ? 1 : 2; }
bool bad_size(int64_t v, int64_t least) { return v < least || v >= kMaxSize; }
bool bad_stride(int64_t v) { return v < 0 || v > kMaxStride; }
ssdi8_status status_of(hipError_t e) { return e == hipSuccess ? SSDI8_OK : SSDI8_ERR_HIP; }

ssdi8_status check_conv(int64_t batch, int64_t seqlen, int64_t channels, const ssdi8_conv_args* a,
                        bool step, ssdi8::ConvOut* out) {
  if (bad_size(batch, 0) || bad_size(seqlen, 0) || bad_size(channels, 1)) return SSDI8_ERR_SHAPE;
  if (channels > kMaxSize - 4096 || (double)batch * (seqlen + 64) * channels > kMaxCount ||
      (double)batch * (seqlen / 32 + 1) * (channels / 512 + 2) > kMaxGrid)
    return SSDI8_ERR_SHAPE;
  if (!a) return SSDI8_ERR_NULL;
  if (!is_float(a->dtype)) return SSDI8_ERR_ARG;
  if (a->act != SSDI8_ACT_NONE && a->act != SSDI8_ACT_SILU) return SSDI8_ERR_ARG;
  if (a->width < 2 || a->width > 4) return SSDI8_ERR_UNSUPPORTED;
  if (bad_stride(a->x_batch_stride) || (!step && bad_stride(a->x_token_stride)))
    return SSDI8_ERR_SHAPE;
  int64_t cols = 0;
  for (int i = 0; i < 3; ++i) {
    if (a->y_cols[i] < 0 || a->y_cols[i] > channels) return SSDI8_ERR_SHAPE;
    cols += a->y_cols[i];
    out->y[i] = a->y[i];
    out->end[i] = (int)cols;
  }
  if (cols != channels) return SSDI8_ERR_SHAPE;
  if (batch == 0) return SSDI8_OK;
  if (!a->weight || (step && !a->final_state) || (seqlen > 0 && !a->x)) return SSDI8_ERR_NULL;
  const uintptr_t es = size_of(a->dtype);
  for (int i = 0; i < 3; ++i) {
    if (seqlen > 0 && a->y_cols[i] > 0 && !a->y[i]) return SSDI8_ERR_NULL;
    if (off(a->y[i], es)) return SSDI8_ERR_ALIGN;
  }
  if (off(a->x, es) || off(a->init_state, es) || off(a->final_state, es) || off(a->weight, 4) ||
      off(a->bias, 4) || off(a->lengths, 4))
    return SSDI8_ERR_ALIGN;
  return SSDI8_OK;
}

ssdi8_status check_scan_dims(const ssdi8_sel_scan_dims* d, bool step) {
  if (!d) return SSDI8_ERR_NULL;
  if (bad_size(d->batch, 0) || (!step && bad_size(d->seqlen, 0)) || bad_size(d->nheads, 1) ||
      bad_size(d->headdim, 1) || bad_size(d->ngroups, 1) || bad_size(d->dstate, 1))
    return SSDI8_ERR_SHAPE;
  const double D = (double)d->nheads * d->headdim, L = step ? 1.0 : (double)d->seqlen;
  if (D >= (double)kMaxSize - 4096) return SSDI8_ERR_SHAPE;
  if (d->nheads * d->headdim % d->ngroups != 0) return SSDI8_ERR_SHAPE;
  if (d->dstate > 256) return SSDI8_ERR_UNSUPPORTED;
  if ((double)d->batch * L * D > kMaxCount || (double)d->batch * D * 256 * 64 > kMaxCount * 16 ||
      (double)d->batch * L * d->ngroups * d->dstate > kMaxCount ||
      (double)d->batch * (D / 2 + d->ngroups) > kMaxGrid || L * 0.5 > kMaxGrid)
    return SSDI8_ERR_SHAPE;
  return SSDI8_OK;
}

ssdi8_status check_scan(const ssdi8_sel_scan_dims* d, const ssdi8_sel_scan_args* a, bool step,
                        ssdi8::SelScan* s) {
  if (!a) return SSDI8_ERR_NULL;
  if (!is_float(a->dtype)) return SSDI8_ERR_ARG;
  if (a->dt_dtype != SSDI8_F32 && a->dt_dtype != a->dtype) return SSDI8_ERR_ARG;
  const int64_t strides[] = {a->u_batch_stride, a->dt_batch_stride, a->B_batch_stride,
                             a->C_batch_stride, a->z_batch_stride};
  const int64_t tokens[] = {a->u_token_stride, a->dt_token_stride, a->B_token_stride,
                            a->C_token_stride, a->z_token_stride};
  for (int i = 0; i < 5; ++i)
    if (bad_stride(strides[i]) || (!step && bad_stride(tokens[i]))) return SSDI8_ERR_SHAPE;
  const bool work = d->batch > 0 && (step || d->seqlen > 0);
  if (work && (!a->u || !a->dt || !a->B || !a->C || !a->y)) return SSDI8_ERR_NULL;
  // the rates are read before the tokens are counted: by the launch that only copies the state, too
  if ((work || (d->batch > 0 && a->final_state)) && !a->A) return SSDI8_ERR_NULL;
  if (work && step && !a->final_state) return SSDI8_ERR_NULL;
  const uintptr_t es = size_of(a->dtype);
  if (off(a->u, es) || off(a->dt, size_of(a->dt_dtype)) || off(a->B, es) || off(a->C, es) ||
      off(a->z, es) || off(a->y, es) || off(a->A, 4) || off(a->D, 4) || off(a->dt_bias, 4) ||
      off(a->init_state, 4) || off(a->lengths, 4) || off(a->final_state, step ? 16 : 4) ||
      off(a->workspace, 4))
    return SSDI8_ERR_ALIGN;
  s->dtype = a->dtype;
  s->dt_dtype = a->dt_dtype;
  s->tied = a->tied != 0;
  s->dt_softplus = a->dt_softplus != 0;
  s->batch = d->batch;
  s->seqlen = step ? 1 : d->seqlen;
  s->nheads = d->nheads;
  s->headdim = d->headdim;
  s->ngroups = d->ngroups;
  s->dstate = d->dstate;
  s->u = a->u;
  s->dt = a->dt;
  s->B = a->B;
  s->C = a->C;
  s->z = a->z;
  s->ur = {a->u_batch_stride, a->u_token_stride};
  s->dtr = {a->dt_batch_stride, a->dt_token_stride};
  s->Br = {a->B_batch_stride, a->B_token_stride};
  s->Cr = {a->C_batch_stride, a->C_token_stride};
  s->zr = {a->z_batch_stride, a->z_token_stride};
  s->A = a->A;
  s->D = a->D;
  s->dt_bias = a->dt_bias;
  s->init = a->init_state;
  s->lengths = a->lengths;
  s->y = a->y;
  s->final_state = a->final_state;
  s->workspace = static_cast<float*>(a->workspace);
  return SSDI8_OK;
}

}  // namespace

extern "C" {

ssdi8_status ssdi8_causal_conv(int64_t batch, int64_t seqlen, int64_t channels,
                               const ssdi8_conv_args* a, void* stream) {
  ssdi8::ConvOut out;
  const ssdi8_status s = check_conv(batch, seqlen, channels, a, false, &out);
  if (s != SSDI8_OK || batch == 0 || (seqlen == 0 && !a->final_state)) return s;
  return status_of(ssdi8::launch_conv(
      a->dtype, a->width, batch, seqlen, channels, a->x, {a->x_batch_stride, a->x_token_stride},
      a->weight, a->bias, a->act == SSDI8_ACT_SILU, a->init_state, a->lengths, out, a->final_state,
      (hipStream_t)stream));
}

ssdi8_status ssdi8_causal_conv_step(int64_t batch, int64_t channels, const ssdi8_conv_args* a,
                                    void* stream) {
  ssdi8::ConvOut out;
  const ssdi8_status s = check_conv(batch, 1, channels, a, true, &out);
  if (s != SSDI8_OK || batch == 0) return s;
  return status_of(ssdi8::launch_conv_step(a->dtype, a->width, batch, channels, a->x,
                                           a->x_batch_stride, a->weight, a->bias,
                                           a->act == SSDI8_ACT_SILU, a->final_state, out,
                                           (hipStream_t)stream));
}

size_t ssdi8_selective_scan_workspace_size(const ssdi8_sel_scan_dims* d) {
  if (check_scan_dims(d, false) != SSDI8_OK) return 0;
  return (size_t)ssdi8::sel_scan_workspace(d->batch, d->seqlen, d->nheads * d->headdim, d->ngroups,
                                           d->dstate) * sizeof(float);
}

ssdi8_status ssdi8_selective_scan(const ssdi8_sel_scan_dims* d, const ssdi8_sel_scan_args* a,
                                  void* stream) {
  ssdi8::SelScan scan;
  ssdi8_status s = check_scan_dims(d, false);
  if (s == SSDI8_OK) s = check_scan(d, a, false, &scan);
  if (s != SSDI8_OK || d->batch == 0 || (d->seqlen == 0 && !a->final_state)) return s;
  const size_t need = ssdi8_selective_scan_workspace_size(d);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need)) return SSDI8_ERR_WORKSPACE;
  return status_of(ssdi8::launch_sel_scan(scan, (hipStream_t)stream));
}

ssdi8_status ssdi8_selective_scan_step(const ssdi8_sel_scan_dims* d, const ssdi8_sel_scan_args* a,
                                       void* stream) {
  ssdi8::SelScan scan;
  ssdi8_status s = check_scan_dims(d, true);
  if (s == SSDI8_OK) s = check_scan(d, a, true, &scan);
  if (s != SSDI8_OK || d->batch == 0) return s;
  return status_of(ssdi8::launch_sel_scan_step(scan, a->final_state, (hipStream_t)stream));
}

ssdi8_status ssdi8_gated_norm(int64_t rows, int64_t channels, int64_t groups,
                              const ssdi8_norm_args* a, void* stream) {
  if (bad_size(rows, 0) || bad_size(channels, 1) || bad_size(groups, 1) || channels % groups != 0)
    return SSDI8_ERR_SHAPE;
  if ((double)rows * channels > kMaxCount || (double)rows * groups > kMaxGrid) return SSDI8_ERR_SHAPE;
  if (channels / groups > 32768) return SSDI8_ERR_UNSUPPORTED;
  if (!a) return SSDI8_ERR_NULL;
  if (!is_float(a->dtype)) return SSDI8_ERR_ARG;
  if (!(a->eps >= 0.0f) || a->eps > 3.0e38f) return SSDI8_ERR_ARG;
  if (bad_stride(a->x_row_stride) || bad_stride(a->z_row_stride)) return SSDI8_ERR_SHAPE;
  if (rows == 0) return SSDI8_OK;
  if (!a->x || !a->weight || !a->y || (a->residual && !a->residual_out)) return SSDI8_ERR_NULL;
  if (!a->residual && a->residual_out) return SSDI8_ERR_ARG;
  const uintptr_t es = size_of(a->dtype);
  if (off(a->x, es) || off(a->z, es) || off(a->residual, es) || off(a->residual_out, es) ||
      off(a->y, es) || off(a->weight, 4))
    return SSDI8_ERR_ALIGN;
  return status_of(ssdi8::launch_gated_norm(a->dtype, rows, channels, groups, a->x, a->x_row_stride,
                                            a->z, a->z_row_stride, a->residual, a->weight, a->eps,
                                            a->norm_before_gate != 0, a->y, a->residual_out,
                                            (hipStream_t)stream));
}

ssdi8_status ssdi8_linear(int64_t rows, int64_t outputs, int64_t k, const ssdi8_linear_args* a,
                          void* stream) {
  if (bad_size(rows, 0) || bad_size(outputs, 1) || bad_size(k, 1)) return SSDI8_ERR_SHAPE;
  if ((double)rows * outputs > kMaxCount || (double)rows * k > kMaxCount ||
      (double)outputs * k > kMaxCount || ((double)rows / 64 + 1) * ((double)outputs / 16 + 1) > kMaxGrid)
    return SSDI8_ERR_SHAPE;
  if (!a) return SSDI8_ERR_NULL;
  if (a->dtype != SSDI8_F16 && a->dtype != SSDI8_BF16 && a->dtype != SSDI8_I8) return SSDI8_ERR_ARG;
  const bool quantized = a->dtype == SSDI8_I8;
  const int own = quantized ? SSDI8_F16 : a->dtype;
  if (a->y_dtype != SSDI8_F32 && a->y_dtype != own) return SSDI8_ERR_ARG;
  if (a->act < SSDI8_ACT_NONE || a->act > SSDI8_ACT_SOFTPLUS) return SSDI8_ERR_ARG;
  if (!quantized && (a->x_scale || a->weight_scale)) return SSDI8_ERR_ARG;
  if (quantized && k > 131072) return SSDI8_ERR_UNSUPPORTED;   // 127 * 128 k stays below 2^31
  if (bad_stride(a->x_row_stride) || bad_stride(a->weight_row_stride) ||
      bad_stride(a->residual_row_stride) || a->y_row_stride < outputs || bad_stride(a->y_row_stride))
    return SSDI8_ERR_SHAPE;
  const int64_t x_row = rows > 1 ? a->x_row_stride : 0;
  const int64_t w_row = outputs > 1 ? a->weight_row_stride : 0;
  if ((255.0 * (double)(x_row > w_row ? x_row : w_row) + (double)k) * (double)size_of(a->dtype) > 4.0e9)
    return SSDI8_ERR_UNSUPPORTED;   // the kernels take 256 rows with 32-bit offsets
  if (rows == 0) return SSDI8_OK;
  if (!a->x || !a->weight || !a->y || (quantized && (!a->x_scale || !a->weight_scale)))
    return SSDI8_ERR_NULL;
  const uintptr_t es = size_of(a->dtype), ys = size_of(a->y_dtype);
  if (off(a->x, es) || off(a->weight, es) || off(a->residual, ys) || off(a->y, ys) ||
      off(a->x_scale, 4) || off(a->weight_scale, 4) || off(a->bias, 4))
    return SSDI8_ERR_ALIGN;
  ssdi8::LinearArgs l;
  l.dtype = a->dtype;
  l.act = a->act;
  l.out_dtype = a->y_dtype;
  l.m = rows;
  l.n = outputs;
  l.k = k;
  l.x = a->x;
  l.w = a->weight;
  l.x_row = x_row;
  l.w_row = w_row;
  l.x_scale = a->x_scale;
  l.w_scale = a->weight_scale;
  l.bias = a->bias;
  l.residual = a->residual;
  l.residual_row = a->residual_row_stride;
  l.y = a->y;
  l.y_row = a->y_row_stride;
  return status_of(ssdi8::launch_linear(l, (hipStream_t)stream));
}

}  // extern "C"
