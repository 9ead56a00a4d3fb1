// The track decoder's operators behind the C boundary: checks of the descriptions, and launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <float.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "hs.h"
#include "hs_internal.h"
#include "hs_track.h"

namespace hs {
namespace {

constexpr int kMaxDim = 128;

bool aligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

Heads view(const hs_heads& t) { return Heads{t.d, t.batch, t.token, t.head}; }

hs_status check_type(const char* fn, int dtype) {
  if (dtype == HS_F16 || dtype == HS_BF16) return HS_OK;
  set_error("%s: dtype must be HS_F16 or HS_BF16, got %d", fn, dtype);
  return HS_E_INVAL;
}

hs_status check_dim(const char* fn, const char* name, int dim) {
  if (dim >= 8 && dim <= kMaxDim && dim % 8 == 0) return HS_OK;
  set_error("%s: %s must be a multiple of 8 in 8..%d, got %d", fn, name, kMaxDim, dim);
  return HS_E_INVAL;
}

hs_status check_sizes(const char* fn, int batch, int tokens, int more_tokens) {
  if (batch >= 0 && tokens >= 0 && more_tokens >= 0) return HS_OK;
  set_error("%s: batch and tokens must not be negative", fn);
  return HS_E_INVAL;
}

hs_status check_groups(const char* fn, int q_heads, int kv_heads) {
  if (q_heads >= 1 && kv_heads >= 1 && q_heads % kv_heads == 0) return HS_OK;
  set_error("%s: q_heads (%d) must be a positive multiple of kv_heads (%d)", fn, q_heads, kv_heads);
  return HS_E_INVAL;
}

// A tensor that is looked at at all: where, and with which strides.
hs_status check_heads(const char* fn, const char* name, const hs_heads& t) {
  if (!t.d || !aligned(t.d, 16)) {
    set_error("%s: %s must be a 16-byte aligned device pointer", fn, name);
    return HS_E_INVAL;
  }
  if (t.batch % 8 || t.token % 8 || t.head % 8) {
    set_error("%s: strides of %s must be multiples of 8 elements", fn, name);
    return HS_E_INVAL;
  }
  return HS_OK;
}

// An output besides: its heads must not overlap.  (Sorted by stride, each dimension has to step over all of the one
// before.)
hs_status check_output(const char* fn, const char* name, const hs_heads& t, int batch, int tokens, int heads, int dim) {
  const hs_status st = check_heads(fn, name, t);
  if (st != HS_OK) return st;
  struct { int64_t stride, n; } d[3] = {{t.batch, batch}, {t.token, tokens}, {t.head, heads}};
  for (auto& x : d) {
    if (x.stride == INT64_MIN) { set_error("%s: stride of %s out of range", fn, name); return HS_E_INVAL; }
    x.stride = std::llabs(x.stride);
  }
  std::sort(d, d + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
  __int128 reach = dim;
  for (const auto& x : d) {
    if (x.n <= 1) continue;
    if ((__int128)x.stride < reach) {
      set_error("%s: rows of %s overlap", fn, name);
      return HS_E_INVAL;
    }
    reach = (__int128)x.stride * (x.n - 1) + reach;
  }
  return HS_OK;
}

hs_status check_pointer(const char* fn, const char* name, const void* p, uintptr_t bytes) {
  if (aligned(p, bytes)) return HS_OK;
  set_error("%s: %s must be %d-byte aligned", fn, name, (int)bytes);
  return HS_E_INVAL;
}

hs_status check_workspace(const char* fn, const void* p, size_t bytes, size_t need) {
  if (bytes < need || (need && !p)) {
    set_error("%s: workspace too small: %zu bytes given, %zu needed", fn, p ? bytes : (size_t)0, need);
    return HS_E_NOMEM;
  }
  if (need && !aligned(p, 256)) {
    set_error("%s: d_workspace must be 256-byte aligned", fn);
    return HS_E_INVAL;
  }
  return HS_OK;
}

hs_status check_context(const char* fn, const hs_ctx* ctx) {
  if (ctx) return HS_OK;
  set_error("%s: NULL context", fn);
  return HS_E_INVAL;
}

// Launches on the context's device and leaves the caller's current device as it was.
template <class P>
hs_status run(const char* fn, const hs_ctx* ctx, const P& params, void* stream) {
  const int device = hs_internal_ctx_device(ctx), before = hs_internal_current_device();
  if (before != device) hs_internal_use_device(device);
  const hipError_t e = launch(params, (hipStream_t)stream);
  if (before != device) hs_internal_use_device(before);
  if (e == hipSuccess) return HS_OK;
  if (e == hipErrorInvalidConfiguration) {
    set_error("%s: more workgroups than one launch can have", fn);
    return HS_E_INVAL;
  }
  set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
  return HS_E_DEVICE;
}

#define HS_TRY(call)                    \
  do {                                  \
    const hs_status st_ = (call);       \
    if (st_ != HS_OK) return st_;       \
  } while (0)

// ---- norm and rotation ---------------------------------------------------------------------
hs_status check(const char* fn, const hs_norm_rotate_desc* d) {
  if (!d) { set_error("%s: NULL description", fn); return HS_E_INVAL; }
  HS_TRY(check_type(fn, d->dtype));
  HS_TRY(check_sizes(fn, d->batch, d->tokens, 0));
  HS_TRY(check_dim(fn, "head_dim", d->head_dim));
  if (d->q_heads < 0 || d->k_heads < 0 || d->q_heads + (int64_t)d->k_heads > INT32_MAX) {
    set_error("%s: bad number of heads (%d and %d)", fn, d->q_heads, d->k_heads);
    return HS_E_INVAL;
  }
  if ((int64_t)d->batch * d->tokens > INT32_MAX) {
    set_error("%s: too many tokens for one call (%d x %d)", fn, d->batch, d->tokens);
    return HS_E_INVAL;
  }
  if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 16) {
    set_error("%s: rotary_dim must be a multiple of 16 in 0..head_dim, got %d", fn, d->rotary_dim);
    return HS_E_INVAL;
  }
  if (d->norm && !(d->eps >= 0.0f && std::isfinite(d->eps))) {
    set_error("%s: eps must be finite and >= 0", fn);
    return HS_E_INVAL;
  }
  if (d->batch == 0 || d->tokens == 0) return HS_OK;
  const struct { const char* in; const char* out; const hs_heads &t, &o; int heads; const float* w; } side[2] = {
      {"q", "q_out", d->q, d->q_out, d->q_heads, d->d_q_weight}, {"k", "k_out", d->k, d->k_out, d->k_heads, d->d_k_weight}};
  bool any = false;
  for (const auto& s : side) {
    if (!s.heads) continue;
    any = true;
    HS_TRY(check_heads(fn, s.in, s.t));
    HS_TRY(check_output(fn, s.out, s.o, d->batch, d->tokens, s.heads, d->head_dim));
    HS_TRY(check_pointer(fn, "a weight", s.w, 4));
    if (s.t.d == s.o.d && (s.t.batch != s.o.batch || s.t.token != s.o.token || s.t.head != s.o.head)) {
      set_error("%s: %s is %s with other strides", fn, s.out, s.in);
      return HS_E_INVAL;
    }
  }
  if (any && d->rotary_dim) {
    if (!d->d_frequencies) { set_error("%s: NULL d_frequencies", fn); return HS_E_INVAL; }
    HS_TRY(check_pointer(fn, "d_frequencies", d->d_frequencies, 8));
    HS_TRY(check_pointer(fn, "d_positions", d->d_positions, 8));
  }
  return HS_OK;
}

// ---- retention ---------------------------------------------------------------------------------
hs_status check(const char* fn, const hs_retention_desc* d) {   // all but the pointers
  if (!d) { set_error("%s: NULL description", fn); return HS_E_INVAL; }
  HS_TRY(check_type(fn, d->dtype));
  HS_TRY(check_sizes(fn, d->batch, d->tokens, 0));
  HS_TRY(check_groups(fn, d->q_heads, d->kv_heads));
  if (d->q_heads > HS_MAX_HEADS) {
    set_error("%s: at most %d heads, got %d", fn, HS_MAX_HEADS, d->q_heads);
    return HS_E_INVAL;
  }
  HS_TRY(check_dim(fn, "key_dim", d->key_dim));
  HS_TRY(check_dim(fn, "value_dim", d->value_dim));
  if (!std::isfinite(d->scale)) { set_error("%s: scale must be finite", fn); return HS_E_INVAL; }
  if (!d->decay) { set_error("%s: NULL decay", fn); return HS_E_INVAL; }
  for (int h = 0; h < d->q_heads; ++h)
    if (!(d->decay[h] >= 0.0 && d->decay[h] <= 1.0)) {
      set_error("%s: decay of head %d must be in [0, 1]", fn, h);
      return HS_E_INVAL;
    }
  return HS_OK;
}

RetentionParams params_of(const hs_retention_desc* d) {
  RetentionParams p = {};
  p.q = view(d->q); p.k = view(d->k); p.v = view(d->v); p.out = view(d->out);
  p.lengths = d->d_lengths;
  p.state_in = d->d_state_in;
  p.state_out = d->d_state_out;
  p.dtype = d->dtype; p.batch = d->batch; p.tokens = d->tokens;
  p.q_heads = d->q_heads; p.group = d->q_heads / d->kv_heads;
  p.key_dim = d->key_dim; p.value_dim = d->value_dim;
  p.scale = d->scale;
  p.parts = (float*)d->d_workspace;
  for (int h = 0; h < d->q_heads; ++h) {
    p.decay[h] = d->decay[h] > 0.0 ? std::max((float)d->decay[h], FLT_TRUE_MIN) : 0.0f;   // (only a decay of 0 ends an infinity)
    p.decay_rest[h] = (float)(d->decay[h] - (double)p.decay[h]);
    p.log2_decay[h] = std::max(std::log2(d->decay[h]), -1e4);   // (a decay of 0: 2^0 = 1 after no step, 0 after one)
  }
  return p;
}

// ---- cross attention ---------------------------------------------------------------------------
hs_status check(const char* fn, const hs_cross_attention_desc* d) {   // all but the pointers
  if (!d) { set_error("%s: NULL description", fn); return HS_E_INVAL; }
  HS_TRY(check_type(fn, d->dtype));
  HS_TRY(check_sizes(fn, d->batch, d->q_tokens, d->k_tokens));
  HS_TRY(check_groups(fn, d->q_heads, d->kv_heads));
  HS_TRY(check_dim(fn, "head_dim", d->head_dim));
  if (!std::isfinite(d->scale)) { set_error("%s: scale must be finite", fn); return HS_E_INVAL; }
  if ((int64_t)d->batch * d->q_heads > INT32_MAX) {
    set_error("%s: too many heads of sequences for one call (%d x %d)", fn, d->batch, d->q_heads);
    return HS_E_INVAL;
  }
  if ((int64_t)d->q_tokens * (d->q_heads / d->kv_heads) > INT32_MAX - 1024) {
    set_error("%s: too many tokens for one call (%d, of %d heads each)", fn, d->q_tokens, d->q_heads / d->kv_heads);
    return HS_E_INVAL;
  }
  return HS_OK;
}

CrossParams params_of(const hs_cross_attention_desc* d) {
  CrossParams p = {};
  p.q = view(d->q); p.k = view(d->k); p.v = view(d->v); p.out = view(d->out);
  p.lengths = d->d_lengths;
  p.mask = d->d_mask; p.mask_batch = d->mask_batch_stride;
  p.lse = d->d_lse;
  p.dtype = d->dtype; p.batch = d->batch; p.q_tokens = d->q_tokens; p.k_tokens = d->k_tokens;
  p.q_heads = d->q_heads; p.group = d->q_heads / d->kv_heads;
  p.dim = d->head_dim;
  p.scale = d->scale;
  p.parts = (float*)d->d_workspace;
  return p;
}

// ---- delta rule ----------------------------------------------------------------------------------
hs_status check(const char* fn, const hs_delta_rule_desc* d) {   // all but the pointers
  if (!d) { set_error("%s: NULL description", fn); return HS_E_INVAL; }
  HS_TRY(check_type(fn, d->dtype));
  HS_TRY(check_sizes(fn, d->batch, d->tokens, 0));
  if (d->heads < 1 || d->qk_heads < 1 || d->heads % d->qk_heads) {
    set_error("%s: heads (%d) must be a positive multiple of qk_heads (%d)", fn, d->heads, d->qk_heads);
    return HS_E_INVAL;
  }
  HS_TRY(check_dim(fn, "key_dim", d->key_dim));
  HS_TRY(check_dim(fn, "value_dim", d->value_dim));
  if (!std::isfinite(d->scale)) { set_error("%s: scale must be finite", fn); return HS_E_INVAL; }
  if (d->tokens > INT32_MAX - 1024) {
    set_error("%s: too many tokens for one call (%d)", fn, d->tokens);
    return HS_E_INVAL;
  }
  if ((int64_t)d->batch * d->heads > INT32_MAX) {
    set_error("%s: too many heads of sequences for one call (%d x %d)", fn, d->batch, d->heads);
    return HS_E_INVAL;
  }
  return HS_OK;
}

DeltaParams params_of(const hs_delta_rule_desc* d) {
  DeltaParams p = {};
  p.q = view(d->q); p.k = view(d->k); p.v = view(d->v); p.out = view(d->out);
  p.log_decay = d->log_decay; p.beta = d->beta;
  p.lengths = d->d_lengths;
  p.state_in = d->d_state_in;
  p.state_out = d->d_state_out;
  p.dtype = d->dtype; p.batch = d->batch; p.tokens = d->tokens;
  p.heads = d->heads; p.group = d->heads / d->qk_heads;
  p.key_dim = d->key_dim; p.value_dim = d->value_dim;
  p.scale = d->scale;
  p.parts = d->d_workspace;
  return p;
}

// ---- differential attention ----------------------------------------------------------------------
hs_status check(const char* fn, const hs_differential_attention_desc* d) {   // all but the pointers
  if (!d) { set_error("%s: NULL description", fn); return HS_E_INVAL; }
  HS_TRY(check_type(fn, d->dtype));
  HS_TRY(check_sizes(fn, d->batch, d->q_tokens, d->k_tokens));
  HS_TRY(check_groups(fn, d->q_heads, d->kv_heads));
  HS_TRY(check_dim(fn, "head_dim", d->head_dim));
  HS_TRY(check_dim(fn, "value_dim", d->value_dim));
  if (!std::isfinite(d->scale)) { set_error("%s: scale must be finite", fn); return HS_E_INVAL; }
  if (d->norm && !(d->eps >= 0.0f && std::isfinite(d->eps))) {
    set_error("%s: eps must be finite and >= 0", fn);
    return HS_E_INVAL;
  }
  if ((int64_t)d->batch * d->q_heads * 2 > INT32_MAX) {
    set_error("%s: too many heads of sequences for one call (%d x 2 x %d)", fn, d->batch, d->q_heads);
    return HS_E_INVAL;
  }
  if ((int64_t)d->q_tokens * (d->q_heads / d->kv_heads) > INT32_MAX / 2 - 1024) {
    set_error("%s: too many tokens for one call (%d, of %d heads each)", fn, d->q_tokens, d->q_heads / d->kv_heads);
    return HS_E_INVAL;
  }
  return HS_OK;
}

DifferentialParams params_of(const hs_differential_attention_desc* d) {
  DifferentialParams p = {};
  p.q = view(d->q); p.k = view(d->k); p.v = view(d->v); p.out = view(d->out);
  p.lambda = d->d_lambda;
  p.weight = d->norm ? d->d_norm_weight : nullptr;
  p.lengths = d->d_lengths;
  p.mask = d->d_mask; p.mask_batch = d->mask_batch_stride;
  p.dtype = d->dtype; p.batch = d->batch; p.q_tokens = d->q_tokens; p.k_tokens = d->k_tokens;
  p.q_heads = d->q_heads; p.group = d->q_heads / d->kv_heads;
  p.dim = d->head_dim; p.value_dim = d->value_dim;
  p.norm = d->norm != 0; p.eps = d->eps;
  p.scale = d->scale;
  p.parts = (float*)d->d_workspace;
  return p;
}

// ---- expert layer --------------------------------------------------------------------------------
hs_status check_range(const char* fn, const char* name, int value, int least, int most, int step) {
  if (value >= least && value <= most && value % step == 0) return HS_OK;
  if (step > 1) set_error("%s: %s must be a multiple of %d in %d..%d, got %d", fn, name, step, least, most, value);
  else set_error("%s: %s must be in %d..%d, got %d", fn, name, least, most, value);
  return HS_E_INVAL;
}

hs_status check(const char* fn, const hs_expert_layer_desc* d) {   // all but the pointers
  if (!d) { set_error("%s: NULL description", fn); return HS_E_INVAL; }
  HS_TRY(check_type(fn, d->dtype));
  HS_TRY(check_range(fn, "tokens", d->tokens, 0, HS_MAX_EXPERT_TOKENS, 1));
  HS_TRY(check_range(fn, "channels", d->channels, 8, HS_MAX_CHANNELS, 8));
  HS_TRY(check_range(fn, "hidden", d->hidden, 8, HS_MAX_CHANNELS, 8));
  HS_TRY(check_range(fn, "experts", d->experts, 1, HS_MAX_EXPERTS, 1));
  HS_TRY(check_range(fn, "top", d->top, 1, std::min(HS_MAX_TOP, d->experts), 1));
  return HS_OK;
}

ExpertParams params_of(const hs_expert_layer_desc* d) {
  ExpertParams p = {};
  p.x = d->d_x; p.x_stride = d->x_stride;
  p.out = d->d_out; p.out_stride = d->out_stride;
  p.router = d->d_router; p.w_in = d->d_w_in; p.w_out = d->d_w_out;
  p.mask = d->d_mask;
  p.chosen = d->d_chosen; p.weights = d->d_weights;
  p.dtype = d->dtype; p.tokens = d->tokens; p.channels = d->channels; p.hidden = d->hidden;
  p.experts = d->experts; p.top = d->top; p.renormalise = d->renormalise != 0;
  p.parts = (char*)d->d_workspace;
  return p;
}

hs_status check_rows(const char* fn, const char* name, const void* d, int64_t stride) {
  if (!d || !aligned(d, 16)) {
    set_error("%s: %s must be a 16-byte aligned device pointer", fn, name);
    return HS_E_INVAL;
  }
  if (stride % 8) {
    set_error("%s: the stride of %s must be a multiple of 8 elements", fn, name);
    return HS_E_INVAL;
  }
  return HS_OK;
}

}  // namespace
}  // namespace hs

using namespace hs;

extern "C" {

hs_status hs_norm_rotate(hs_ctx* ctx, const hs_norm_rotate_desc* desc, void* hip_stream) {
  const char* const fn = "hs_norm_rotate";
  return guarded(fn, [&]() -> hs_status {
  HS_TRY(check(fn, desc));
  HS_TRY(check_context(fn, ctx));
  if (desc->batch == 0 || desc->tokens == 0 || desc->q_heads + desc->k_heads == 0) return HS_OK;
  NormRotateParams p = {};
  p.q = view(desc->q); p.k = view(desc->k); p.q_out = view(desc->q_out); p.k_out = view(desc->k_out);
  p.wq = desc->norm ? desc->d_q_weight : nullptr;
  p.wk = desc->norm ? desc->d_k_weight : nullptr;
  p.freq = desc->d_frequencies;
  p.pos = desc->d_positions;
  p.pos_batch = desc->position_batch_stride; p.first = desc->first_position;
  p.dtype = desc->dtype; p.batch = desc->batch; p.tokens = desc->tokens;
  p.q_heads = desc->q_heads; p.k_heads = desc->k_heads;
  p.dim = desc->head_dim; p.rotary = desc->rotary_dim; p.interleaved = desc->interleaved != 0;
  p.norm = desc->norm != 0; p.eps = desc->eps;
  return run(fn, ctx, p, hip_stream);
  });
}

hs_status hs_query_retention_workspace(const hs_retention_desc* desc, size_t* bytes) {
  const char* const fn = "hs_query_retention_workspace";
  return guarded(fn, [&]() -> hs_status {
  if (!bytes) { set_error("%s: NULL bytes", fn); return HS_E_INVAL; }
  HS_TRY(check(fn, desc));
  *bytes = retention_workspace(params_of(desc));
  return HS_OK;
  });
}

hs_status hs_retention(hs_ctx* ctx, const hs_retention_desc* desc, void* hip_stream) {
  const char* const fn = "hs_retention";
  return guarded(fn, [&]() -> hs_status {
  HS_TRY(check(fn, desc));
  if (desc->batch > 0) {
    if (desc->tokens > 0) {
      HS_TRY(check_heads(fn, "q", desc->q));
      HS_TRY(check_heads(fn, "k", desc->k));
      HS_TRY(check_heads(fn, "v", desc->v));
      HS_TRY(check_output(fn, "out", desc->out, desc->batch, desc->tokens, desc->q_heads, desc->value_dim));
    }
    if (!desc->d_state_out) { set_error("%s: NULL d_state_out", fn); return HS_E_INVAL; }
    HS_TRY(check_pointer(fn, "d_state_in", desc->d_state_in, 16));
    HS_TRY(check_pointer(fn, "d_state_out", desc->d_state_out, 16));
    HS_TRY(check_pointer(fn, "d_lengths", desc->d_lengths, 4));
  }
  HS_TRY(check_workspace(fn, desc->d_workspace, desc->workspace_bytes, retention_workspace(params_of(desc))));
  HS_TRY(check_context(fn, ctx));
  if (desc->batch == 0) return HS_OK;
  return run(fn, ctx, params_of(desc), hip_stream);
  });
}

hs_status hs_query_cross_attention_workspace(const hs_cross_attention_desc* desc, size_t* bytes) {
  const char* const fn = "hs_query_cross_attention_workspace";
  return guarded(fn, [&]() -> hs_status {
  if (!bytes) { set_error("%s: NULL bytes", fn); return HS_E_INVAL; }
  HS_TRY(check(fn, desc));
  *bytes = cross_workspace(params_of(desc));
  return HS_OK;
  });
}

hs_status hs_cross_attention(hs_ctx* ctx, const hs_cross_attention_desc* desc, void* hip_stream) {
  const char* const fn = "hs_cross_attention";
  return guarded(fn, [&]() -> hs_status {
  HS_TRY(check(fn, desc));
  const bool any = desc->batch > 0 && desc->q_tokens > 0;
  if (any) {
    HS_TRY(check_heads(fn, "q", desc->q));
    if (desc->k_tokens > 0) {
      HS_TRY(check_heads(fn, "k", desc->k));
      HS_TRY(check_heads(fn, "v", desc->v));
    }
    HS_TRY(check_output(fn, "out", desc->out, desc->batch, desc->q_tokens, desc->q_heads, desc->head_dim));
    HS_TRY(check_pointer(fn, "d_lengths", desc->d_lengths, 4));
    HS_TRY(check_pointer(fn, "d_lse", desc->d_lse, 4));
  }
  HS_TRY(check_workspace(fn, desc->d_workspace, desc->workspace_bytes, cross_workspace(params_of(desc))));
  HS_TRY(check_context(fn, ctx));
  if (!any) return HS_OK;
  return run(fn, ctx, params_of(desc), hip_stream);
  });
}

hs_status hs_query_delta_rule_workspace(const hs_delta_rule_desc* desc, size_t* bytes) {
  const char* const fn = "hs_query_delta_rule_workspace";
  return guarded(fn, [&]() -> hs_status {
  if (!bytes) { set_error("%s: NULL bytes", fn); return HS_E_INVAL; }
  HS_TRY(check(fn, desc));
  *bytes = delta_workspace(params_of(desc));
  return HS_OK;
  });
}

hs_status hs_delta_rule(hs_ctx* ctx, const hs_delta_rule_desc* desc, void* hip_stream) {
  const char* const fn = "hs_delta_rule";
  return guarded(fn, [&]() -> hs_status {
  HS_TRY(check(fn, desc));
  if (desc->batch > 0) {
    if (desc->tokens > 0) {
      HS_TRY(check_heads(fn, "q", desc->q));
      HS_TRY(check_heads(fn, "k", desc->k));
      HS_TRY(check_heads(fn, "v", desc->v));
      HS_TRY(check_output(fn, "out", desc->out, desc->batch, desc->tokens, desc->heads, desc->value_dim));
      HS_TRY(check_pointer(fn, "log_decay", desc->log_decay.d, 4));
      HS_TRY(check_pointer(fn, "beta", desc->beta.d, 4));
    }
    if (!desc->d_state_out) { set_error("%s: NULL d_state_out", fn); return HS_E_INVAL; }
    HS_TRY(check_pointer(fn, "d_state_in", desc->d_state_in, 16));
    HS_TRY(check_pointer(fn, "d_state_out", desc->d_state_out, 16));
    HS_TRY(check_pointer(fn, "d_lengths", desc->d_lengths, 4));
  }
  HS_TRY(check_workspace(fn, desc->d_workspace, desc->workspace_bytes, delta_workspace(params_of(desc))));
  HS_TRY(check_context(fn, ctx));
  if (desc->batch == 0) return HS_OK;
  return run(fn, ctx, params_of(desc), hip_stream);
  });
}

hs_status hs_query_differential_attention_workspace(const hs_differential_attention_desc* desc, size_t* bytes) {
  const char* const fn = "hs_query_differential_attention_workspace";
  return guarded(fn, [&]() -> hs_status {
  if (!bytes) { set_error("%s: NULL bytes", fn); return HS_E_INVAL; }
  HS_TRY(check(fn, desc));
  *bytes = differential_workspace(params_of(desc));
  return HS_OK;
  });
}

hs_status hs_differential_attention(hs_ctx* ctx, const hs_differential_attention_desc* desc, void* hip_stream) {
  const char* const fn = "hs_differential_attention";
  return guarded(fn, [&]() -> hs_status {
  HS_TRY(check(fn, desc));
  const bool any = desc->batch > 0 && desc->q_tokens > 0;
  if (any) {
    HS_TRY(check_heads(fn, "q", desc->q));
    if (desc->k_tokens > 0) {
      HS_TRY(check_heads(fn, "k", desc->k));
      HS_TRY(check_heads(fn, "v", desc->v));
    }
    HS_TRY(check_output(fn, "out", desc->out, desc->batch, desc->q_tokens, desc->q_heads, desc->value_dim));
    if (!desc->d_lambda) { set_error("%s: NULL d_lambda", fn); return HS_E_INVAL; }
    HS_TRY(check_pointer(fn, "d_lambda", desc->d_lambda, 4));
    HS_TRY(check_pointer(fn, "d_norm_weight", desc->norm ? desc->d_norm_weight : nullptr, 4));
    HS_TRY(check_pointer(fn, "d_lengths", desc->d_lengths, 4));
  }
  HS_TRY(check_workspace(fn, desc->d_workspace, desc->workspace_bytes, differential_workspace(params_of(desc))));
  HS_TRY(check_context(fn, ctx));
  if (!any) return HS_OK;
  return run(fn, ctx, params_of(desc), hip_stream);
  });
}

hs_status hs_query_expert_layer_workspace(const hs_expert_layer_desc* desc, size_t* bytes) {
  const char* const fn = "hs_query_expert_layer_workspace";
  return guarded(fn, [&]() -> hs_status {
  if (!bytes) { set_error("%s: NULL bytes", fn); return HS_E_INVAL; }
  HS_TRY(check(fn, desc));
  *bytes = expert_workspace(params_of(desc));
  return HS_OK;
  });
}

hs_status hs_expert_layer(hs_ctx* ctx, const hs_expert_layer_desc* desc, void* hip_stream) {
  const char* const fn = "hs_expert_layer";
  return guarded(fn, [&]() -> hs_status {
  HS_TRY(check(fn, desc));
  if (desc->tokens > 0) {
    HS_TRY(check_rows(fn, "d_x", desc->d_x, desc->x_stride));
    HS_TRY(check_rows(fn, "d_out", desc->d_out, desc->out_stride));
    if (desc->tokens > 1 && desc->out_stride > -desc->channels && desc->out_stride < desc->channels) {
      set_error("%s: rows of d_out overlap", fn);
      return HS_E_INVAL;
    }
    HS_TRY(check_rows(fn, "d_router", desc->d_router, 0));
    HS_TRY(check_rows(fn, "d_w_in", desc->d_w_in, 0));
    HS_TRY(check_rows(fn, "d_w_out", desc->d_w_out, 0));
    HS_TRY(check_pointer(fn, "d_chosen", desc->d_chosen, 4));
    HS_TRY(check_pointer(fn, "d_weights", desc->d_weights, 4));
  }
  HS_TRY(check_workspace(fn, desc->d_workspace, desc->workspace_bytes, expert_workspace(params_of(desc))));
  HS_TRY(check_context(fn, ctx));
  if (desc->tokens == 0) return HS_OK;
  return run(fn, ctx, params_of(desc), hip_stream);
  });
}

}  // extern "C"
