// C ABI of linear attention, the norm into few bits and the microscaled projections (declared in include/ssdi8.h):
// argument validation and launches on the caller's stream.
#include "ssdi8.h"

#include <hip/hip_runtime.h>

#include "attention.hpp"
#include "mx.hpp"

namespace {

constexpr int64_t kMaxSize = (int64_t)1 << 31;    // of one dimension
constexpr double kMaxCount = 4.0e12;              // of a tensor's elements
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // elements
constexpr double kMaxGrid = 2147483647.0 / 2;     // workgroups

bool off(const void* p, uintptr_t align) { return ((uintptr_t)p & (align - 1)) != 0; }
bool is_float(int dtype) {
  return dtype == SSDI8_F32 || dtype == SSDI8_F16 || dtype == SSDI8_BF16;
}
uintptr_t size_of(int dtype) { return dtype == SSDI8_F32 ? 4 : 2; }
bool bad_size(int64_t v, int64_t least) { return v < least || v >= kMaxSize; }
bool bad_stride(int64_t v) { return v < 0 || v > kMaxStride; }
bool finite(float v) { return v >= -3.4028235e38f && v <= 3.4028235e38f; }
ssdi8_status status_of(hipError_t e) { return e == hipSuccess ? SSDI8_OK : SSDI8_ERR_HIP; }

ssdi8_status check_attn_dims(const ssdi8_attn_dims* d, bool step) {
  if (!d) return SSDI8_ERR_NULL;
  if (bad_size(d->batch, 0) || (!step && bad_size(d->seqlen, 0)) || bad_size(d->q_heads, 1) ||
      bad_size(d->k_heads, 1) || bad_size(d->v_heads, 1) || bad_size(d->keys, 1) || bad_size(d->values, 1))
    return SSDI8_ERR_SHAPE;
  const int64_t heads = d->q_heads > d->v_heads ? d->q_heads : d->v_heads;
  if (heads % d->q_heads != 0 || heads % d->v_heads != 0 || d->v_heads % d->k_heads != 0) return SSDI8_ERR_SHAPE;
  if (d->keys > 256) return SSDI8_ERR_UNSUPPORTED;
  const double B = (double)d->batch, L = step ? 1.0 : (double)d->seqlen + 64.0, H = (double)heads;
  const double V = (double)d->values + 128.0;
  // the spans of a cut sequence are 512 workgroups more than the heads', at most
  if (B * L * H * V > kMaxCount || B * L * (double)d->q_heads * 256.0 > kMaxCount ||
      B * L * (double)d->k_heads * 256.0 > kMaxCount || B * H * 256.0 * V > kMaxCount ||
      B * H * (V / 64.0) + 1024.0 > kMaxGrid)
    return SSDI8_ERR_SHAPE;
  return SSDI8_OK;
}

void attn_sizes(const ssdi8_attn_dims* d, int dtype, bool step, ssdi8::LinearAttention* l) {
  l->dtype = dtype;
  l->batch = d->batch;
  l->seqlen = step ? 1 : d->seqlen;
  l->keys = d->keys;
  l->values = d->values;
  l->q_heads = d->q_heads;
  l->k_heads = d->k_heads;
  l->v_heads = d->v_heads;
  l->heads = d->q_heads > d->v_heads ? d->q_heads : d->v_heads;
}

ssdi8_status check_attn(const ssdi8_attn_dims* d, const ssdi8_attn_args* a, bool step, ssdi8::LinearAttention* l) {
  if (!a) return SSDI8_ERR_NULL;
  if (!is_float(a->dtype) || !finite(a->scale)) return SSDI8_ERR_ARG;
  const int64_t strides[] = {a->q_batch_stride, a->q_head_stride, a->k_batch_stride, a->k_head_stride,
                             a->v_batch_stride, a->v_head_stride};
  for (int64_t s : strides)
    if (bad_stride(s)) return SSDI8_ERR_SHAPE;
  if (!step && (bad_stride(a->q_token_stride) || bad_stride(a->k_token_stride) || bad_stride(a->v_token_stride)))
    return SSDI8_ERR_SHAPE;
  if (a->log_decay && a->token_decay &&
      (bad_stride(a->decay_batch_stride) || (!step && bad_stride(a->decay_token_stride))))
    return SSDI8_ERR_SHAPE;
  // a chunk's tokens, of two heads of v, are taken with 31-bit offsets; the stride of a single token or head is not used
  const double es_ = (double)size_of(a->dtype), most = 2.0e9 / (64.0 * es_);
  const bool many = d->seqlen > 1;
  const double v_head = d->v_heads > 1 ? (double)a->v_head_stride / 32.0 : 0.0;
  if (!step && d->seqlen > 0 &&
      ((many && ((double)a->q_token_stride + 256 > most || (double)a->k_token_stride + 256 > most)) ||
       (many ? (double)a->v_token_stride : 0.0) + v_head + 256 > most ||
       (many && (double)(d->q_heads > d->v_heads ? d->q_heads : d->v_heads) * (double)d->values > most)))
    return SSDI8_ERR_UNSUPPORTED;
  const bool work = d->batch > 0 && (step || d->seqlen > 0);
  if (work && (!a->q || !a->k || !a->v || !a->y)) return SSDI8_ERR_NULL;
  if (work && step && !a->final_state) return SSDI8_ERR_NULL;
  const uintptr_t es = size_of(a->dtype);
  if (off(a->q, es) || off(a->k, es) || off(a->v, es) || off(a->y, es) || off(a->log_decay, 4) ||
      off(a->init_state, 4) || off(a->lengths, 4) || off(a->final_state, 4) || off(a->workspace, 4))
    return SSDI8_ERR_ALIGN;
  attn_sizes(d, a->dtype, step, l);
  l->token_decay = a->token_decay != 0;
  l->q = a->q;
  l->k = a->k;
  l->v = a->v;
  l->qs = {a->q_batch_stride, a->q_token_stride, a->q_head_stride};
  l->ks = {a->k_batch_stride, a->k_token_stride, a->k_head_stride};
  l->vs = {a->v_batch_stride, a->v_token_stride, a->v_head_stride};
  l->log_decay = a->log_decay;
  l->g_batch = a->decay_batch_stride;
  l->g_token = a->decay_token_stride;
  l->scale = a->scale;
  l->init = a->init_state;
  l->lengths = a->lengths;
  l->y = a->y;
  l->final_state = a->final_state;
  l->workspace = static_cast<float*>(a->workspace);
  return SSDI8_OK;
}

}  // namespace

extern "C" {

size_t ssdi8_linear_attention_workspace_size(const ssdi8_attn_dims* d, int dtype) {
  if (check_attn_dims(d, false) != SSDI8_OK || !is_float(dtype)) return 0;
  ssdi8::LinearAttention l;
  attn_sizes(d, dtype, false, &l);
  return (size_t)ssdi8::linear_attention_workspace(l) * sizeof(float);
}

ssdi8_status ssdi8_linear_attention(const ssdi8_attn_dims* d, const ssdi8_attn_args* a, void* stream) {
  ssdi8::LinearAttention l;
  ssdi8_status s = check_attn_dims(d, false);
  if (s == SSDI8_OK) s = check_attn(d, a, false, &l);
  if (s != SSDI8_OK || d->batch == 0 || (d->seqlen == 0 && !a->final_state)) return s;
  const size_t need = ssdi8_linear_attention_workspace_size(d, a->dtype);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need)) return SSDI8_ERR_WORKSPACE;
  return status_of(ssdi8::launch_linear_attention(l, (hipStream_t)stream));
}

ssdi8_status ssdi8_linear_attention_step(const ssdi8_attn_dims* d, const ssdi8_attn_args* a, void* stream) {
  ssdi8::LinearAttention l;
  ssdi8_status s = check_attn_dims(d, true);
  if (s == SSDI8_OK) s = check_attn(d, a, true, &l);
  if (s != SSDI8_OK || d->batch == 0) return s;
  return status_of(ssdi8::launch_linear_attention_step(l, (hipStream_t)stream));
}

ssdi8_status ssdi8_norm_quantize(int64_t rows, int64_t channels, int64_t groups,
                                 const ssdi8_norm_quant_args* a, void* stream) {
  if (bad_size(rows, 0) || bad_size(channels, 1) || bad_size(groups, 1) || channels % groups != 0)
    return SSDI8_ERR_SHAPE;
  if ((double)rows * (channels + 32) > kMaxCount || (double)rows > kMaxGrid) return SSDI8_ERR_SHAPE;
  if (channels > 32768) return SSDI8_ERR_UNSUPPORTED;
  if (!a) return SSDI8_ERR_NULL;
  if (!is_float(a->dtype)) return SSDI8_ERR_ARG;
  if (a->format != SSDI8_FMT_I8 && a->format != SSDI8_FMT_MXFP8 && a->format != SSDI8_FMT_MXFP4) return SSDI8_ERR_ARG;
  if (!(a->eps >= 0.0f) || !finite(a->eps)) return SSDI8_ERR_ARG;
  if (bad_stride(a->x_row_stride) || bad_stride(a->z_row_stride)) return SSDI8_ERR_SHAPE;
  if (rows == 0) return SSDI8_OK;
  if (!a->x || !a->weight || !a->codes || !a->scales || (a->residual && !a->residual_out)) return SSDI8_ERR_NULL;
  if (!a->residual && a->residual_out) return SSDI8_ERR_ARG;
  const uintptr_t es = size_of(a->dtype);
  if (off(a->x, es) || off(a->z, es) || off(a->residual, es) || off(a->residual_out, es) || off(a->y, es) ||
      off(a->weight, 4) || (a->format == SSDI8_FMT_I8 && off(a->scales, 4)))
    return SSDI8_ERR_ALIGN;
  ssdi8::NormQuant q;
  q.dtype = a->dtype;
  q.format = a->format;
  q.before = a->norm_before_gate != 0;
  q.rows = rows;
  q.channels = channels;
  q.groups = groups;
  q.x = a->x;
  q.x_row = a->x_row_stride;
  q.z = a->z;
  q.z_row = a->z_row_stride;
  q.residual = a->residual;
  q.weight = a->weight;
  q.eps = a->eps;
  q.codes = a->codes;
  q.scales = a->scales;
  q.y = a->y;
  q.residual_out = a->residual_out;
  return status_of(ssdi8::launch_norm_quantize(q, (hipStream_t)stream));
}

ssdi8_status ssdi8_quantize_mx(int64_t rows, int64_t k, const void* x, int dtype, int64_t x_row_stride,
                               int format, void* codes, void* scales, void* stream) {
  if (bad_size(rows, 0) || bad_size(k, 1) || (double)rows * (k + 32) > kMaxCount ||
      (double)rows * (k + 32) / 8192 + 1 > kMaxGrid)
    return SSDI8_ERR_SHAPE;
  if (!is_float(dtype) || (format != SSDI8_FMT_MXFP8 && format != SSDI8_FMT_MXFP4)) return SSDI8_ERR_ARG;
  if (bad_stride(x_row_stride)) return SSDI8_ERR_SHAPE;
  if (rows == 0) return SSDI8_OK;
  if (!x || !codes || !scales) return SSDI8_ERR_NULL;
  if (off(x, size_of(dtype))) return SSDI8_ERR_ALIGN;
  return status_of(ssdi8::launch_quantize_mx(dtype, format, rows, k, x, x_row_stride, codes, scales,
                                             (hipStream_t)stream));
}

ssdi8_status ssdi8_linear_mx(int64_t rows, int64_t outputs, int64_t k, const ssdi8_linear_mx_args* a,
                             void* stream) {
  if (bad_size(rows, 0) || bad_size(outputs, 1) || bad_size(k, 1) || k % 32 != 0) return SSDI8_ERR_SHAPE;
  if ((double)rows * outputs > kMaxCount || (double)rows * k > kMaxCount || (double)outputs * k > kMaxCount ||
      ((double)rows / 64 + 1) * ((double)outputs / 16 + 1) > kMaxGrid)
    return SSDI8_ERR_SHAPE;
  if (!a) return SSDI8_ERR_NULL;
  if (a->x_format != SSDI8_FMT_MXFP8 && a->x_format != SSDI8_FMT_MXFP4) return SSDI8_ERR_ARG;
  if (!is_float(a->y_dtype)) return SSDI8_ERR_ARG;
  if (a->act < SSDI8_ACT_NONE || a->act > SSDI8_ACT_SOFTPLUS) return SSDI8_ERR_ARG;
  if (bad_stride(a->residual_row_stride) || a->y_row_stride < outputs || bad_stride(a->y_row_stride))
    return SSDI8_ERR_SHAPE;
  if (256.0 * (double)k > 4.0e9) return SSDI8_ERR_UNSUPPORTED;   // the kernels take 256 rows with 32-bit offsets
  if (rows == 0) return SSDI8_OK;
  if (!a->x_codes || !a->x_scales || !a->weight_codes || !a->weight_scales || !a->y) return SSDI8_ERR_NULL;
  const uintptr_t ys = size_of(a->y_dtype);
  if (off(a->x_codes, 16) || off(a->weight_codes, 16) || off(a->residual, ys) || off(a->y, ys) || off(a->bias, 4))
    return SSDI8_ERR_ALIGN;
  ssdi8::LinearMx l;
  l.format = a->x_format;
  l.act = a->act;
  l.out_dtype = a->y_dtype;
  l.m = rows;
  l.n = outputs;
  l.blocks = k / 32;
  l.x = static_cast<const uint8_t*>(a->x_codes);
  l.xs = static_cast<const uint8_t*>(a->x_scales);
  l.w = static_cast<const uint8_t*>(a->weight_codes);
  l.ws = static_cast<const uint8_t*>(a->weight_scales);
  l.bias = a->bias;
  l.residual = a->residual;
  l.residual_row = a->residual_row_stride;
  l.y = a->y;
  l.y_row = a->y_row_stride;
  return status_of(ssdi8::launch_linear_mx(l, (hipStream_t)stream));
}

}  // extern "C"
