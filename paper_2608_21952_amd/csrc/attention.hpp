// Linear attention with a decay per head: the launches of linear_attention.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ssdi8 {

// Element offsets between batch elements, tokens and heads of a tensor whose last dimension is dense.
struct Heads {
  int64_t batch = 0, token = 0, head = 0;
};

struct LinearAttention {
  int dtype = 0, token_decay = 0;
  int64_t batch = 0, seqlen = 0, keys = 0, values = 0;   // keys, values: sizes of a head
  int64_t q_heads = 0, k_heads = 0, v_heads = 0, heads = 0;   // heads: of y, the larger of q's and v's
  const void *q = nullptr, *k = nullptr, *v = nullptr;
  Heads qs, ks, vs;
  const float* log_decay = nullptr;   // per head, or per token at gs; NULL: none
  int64_t g_batch = 0, g_token = 0;
  float scale = 1.0f;
  const float* init = nullptr;
  const int* lengths = nullptr;
  void* y = nullptr;
  float* final_state = nullptr;
  float* workspace = nullptr;
};
// Floats of workspace that a call of these sizes needs.
int64_t linear_attention_workspace(const LinearAttention& a);
hipError_t launch_linear_attention(const LinearAttention& a, hipStream_t st);
// One token; the state, in and out, is final_state.
hipError_t launch_linear_attention_step(const LinearAttention& a, hipStream_t st);

}  // namespace ssdi8
