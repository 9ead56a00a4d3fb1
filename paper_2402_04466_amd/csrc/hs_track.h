// Device-side interface of the track decoder's operators (hs_norm_rotate, hs_retention, hs_cross_attention,
// hs_delta_rule, hs_differential_attention, hs_expert_layer): parameter blocks and launch functions.
#pragma once

#include "hs_kernels.h"

#include "hs.h"

namespace hs {

// The launch functions return hipErrorInvalidConfiguration, and launch nothing, where a call needs more workgroups
// than one launch can have.

// A tensor [batch][tokens][heads][dim]; strides in elements, dim contiguous.
struct Heads {
  void* p;
  int64_t batch, token, head;
};

struct NormRotateParams {
  Heads q, k, q_out, k_out;
  const float* wq;               // NULL: ones
  const float* wk;
  const double* freq;            // radians per position
  const int64_t* pos;            // NULL: first + token
  int64_t pos_batch, first;
  int dtype, batch, tokens, q_heads, k_heads, dim, rotary, interleaved, norm;
  float eps;
};
hipError_t launch(const NormRotateParams& p, hipStream_t stream);

struct RetentionParams {
  Heads q, k, v, out;
  const int32_t* lengths;        // NULL: all tokens
  const float* state_in;         // NULL: zeros
  float* state_out;
  int dtype, batch, tokens, q_heads, group, key_dim, value_dim;   // group: query heads per key head
  float scale;
  float decay[HS_MAX_HEADS], decay_rest[HS_MAX_HEADS];   // the decay in two parts, 48 bits of it together; 0 only for 0
  double log2_decay[HS_MAX_HEADS];
  float* parts;                  // workspace: retention_workspace() bytes
};
size_t retention_workspace(const RetentionParams& p);
hipError_t launch(const RetentionParams& p, hipStream_t stream);

struct CrossParams {
  Heads q, k, v, out;
  const int32_t* lengths;        // NULL: all keys
  const uint8_t* mask;           // NULL: all visible
  int64_t mask_batch;
  float* lse;                    // NULL: not wanted
  int dtype, batch, q_tokens, k_tokens, q_heads, group, dim;
  float scale;
  float* parts;                  // workspace: cross_workspace() bytes
};
size_t cross_workspace(const CrossParams& p);
hipError_t launch(const CrossParams& p, hipStream_t stream);

struct DeltaParams {
  Heads q, k, v, out;
  hs_gates log_decay, beta;      // d NULL: 0, 1
  const int32_t* lengths;        // NULL: all tokens
  const float* state_in;         // NULL: zeros
  float* state_out;
  int dtype, batch, tokens, heads, group, key_dim, value_dim;     // group: value heads per key head
  float scale;
  void* parts;                   // workspace: delta_workspace() bytes
};
size_t delta_workspace(const DeltaParams& p);
hipError_t launch(const DeltaParams& p, hipStream_t stream);

struct DifferentialParams {
  Heads q, k, v, out;
  const float* lambda;
  const float* weight;           // NULL: ones
  const int32_t* lengths;        // NULL: all keys
  const uint8_t* mask;           // NULL: all visible
  int64_t mask_batch;
  int dtype, batch, q_tokens, k_tokens, q_heads, group, dim, value_dim, norm;
  float scale, eps;
  float* parts;                  // workspace: differential_workspace() bytes
};
size_t differential_workspace(const DifferentialParams& p);
hipError_t launch(const DifferentialParams& p, hipStream_t stream);

struct ExpertParams {
  const void* x;
  int64_t x_stride;
  void* out;
  int64_t out_stride;
  const void* router;
  const void* w_in;
  const void* w_out;
  const uint8_t* mask;           // NULL: all tokens
  int32_t* chosen;               // NULL: not wanted
  float* weights;                // NULL: not wanted
  int dtype, tokens, channels, hidden, experts, top, renormalise;
  char* parts;                   // workspace: expert_workspace() bytes
};
size_t expert_workspace(const ExpertParams& p);
hipError_t launch(const ExpertParams& p, hipStream_t stream);

}  // namespace hs
