// hs_expert_layer: a router and the experts' networks for a few tokens.
#include "hs_track_device.h"

#include <math.h>

#include <algorithm>

namespace hs {
namespace {

struct ExpertParts {            // the workspace
  int32_t* chosen;              // [tokens][top]
  float* weights;               // [tokens][top]
  float* hidden;                // [tokens][top][hidden]
  size_t bytes;
};
ExpertParts parts_of(const ExpertParams& p) {
  ExpertParts w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* const here = p.parts + at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  const size_t pairs = (size_t)p.tokens * p.top;
  w.chosen = (int32_t*)take(pairs * 4);
  w.weights = (float*)take(pairs * 4);
  w.hidden = (float*)take(pairs * p.hidden * 4);
  w.bytes = at;
  return w;
}

// Scores as whole numbers in their order, those of NaN below all others.
__device__ __forceinline__ uint64_t rank_of(double x) {
  if (x != x) return 0;
  const uint64_t bits = __builtin_bit_cast(uint64_t, x == 0.0 ? 0.0 : x);
  return bits >> 63 ? ~bits : bits | 1ull << 63;
}

// A wave per token: scores in 64 bits, lane l has experts l, l + 64, ..
template <class T>
__global__ __launch_bounds__(64) void k_expert_route(ExpertParams p, ExpertParts w) {
  typedef typename Vec<T>::x8 x8;
  const int t = blockIdx.x, lane = threadIdx.x;
  if (p.mask && !p.mask[t]) {
    if (lane < p.top) {
      w.chosen[t * p.top + lane] = -1;
      w.weights[t * p.top + lane] = 0.0f;
      if (p.chosen) p.chosen[t * p.top + lane] = -1;
      if (p.weights) p.weights[t * p.top + lane] = 0.0f;
    }
    return;
  }
  const T* const x = (const T*)p.x + t * p.x_stride;
  double score[HS_MAX_EXPERTS / 64];
  for (int e = 0; e < p.experts; ++e) {
    const T* const r = (const T*)p.router + (int64_t)e * p.channels;
    double sum = 0.0;
    for (int c = 8 * lane; c < p.channels; c += 512) {
      const x8 a = *(const x8*)(x + c), g = *(const x8*)(r + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)(float)a[i], (double)(float)g[i], sum);
    }
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
#pragma unroll
    for (int i = 0; i < HS_MAX_EXPERTS / 64; ++i)
      if (lane + 64 * i == e) score[i] = sum;
  }
  double best[HS_MAX_TOP];
  uint32_t taken = 0;
  double most = 0.0;
  for (int n = 0; n < p.top; ++n) {
    uint64_t rank = 0;
    int index = INT32_MAX;
    double value = 0.0;
#pragma unroll
    for (int i = 0; i < HS_MAX_EXPERTS / 64; ++i) {
      if (lane + 64 * i >= p.experts || taken >> i & 1) continue;
      const uint64_t r = rank_of(score[i]);
      if (index == INT32_MAX || r > rank) rank = r, index = lane + 64 * i, value = score[i];
    }
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t r = __shfl_xor(rank, d);
      const int other = __shfl_xor(index, d);
      const double v = __shfl_xor(value, d);
      if (other != INT32_MAX && (index == INT32_MAX || r > rank || (r == rank && other < index))) rank = r, index = other, value = v;
    }
    if ((index & 63) == lane) taken |= 1u << (index >> 6);
    if (n == 0) most = value;
    if (lane == n) {
      w.chosen[t * p.top + n] = index;
      if (p.chosen) p.chosen[t * p.top + n] = index;
    }
#pragma unroll
    for (int i = 0; i < HS_MAX_TOP; ++i)
      if (i == n) best[i] = value;
  }
  double total = 0.0;
  if (p.renormalise) {
#pragma unroll
    for (int i = 0; i < HS_MAX_TOP; ++i)
      if (i < p.top) total += exp(best[i] - most);
  } else {
#pragma unroll
    for (int i = 0; i < HS_MAX_EXPERTS / 64; ++i)
      if (lane + 64 * i < p.experts) total += exp(score[i] - most);
    for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
  }
#pragma unroll
  for (int i = 0; i < HS_MAX_TOP; ++i)
    if (i < p.top && lane == i) {
      const float weight = (float)(exp(best[i] - most) / total);
      w.weights[t * p.top + i] = weight;
      if (p.weights) p.weights[t * p.top + i] = weight;
    }
}

template <class T>
__device__ __forceinline__ float dot(const T* a, const T* b, int n, int lane) {
  typedef typename Vec<T>::x8 x8;
  float sum = 0.0f;
  for (int c = 8 * lane; c < n; c += 512) {
    const x8 u = *(const x8*)(a + c), v = *(const x8*)(b + c);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf((float)u[i], (float)v[i], sum);
  }
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  return sum;
}

// A wave per token, chosen expert and value of the hidden layer.
template <class T>
__global__ __launch_bounds__(256) void k_expert_in(ExpertParams p, ExpertParts w) {
  const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, pair = id / p.hidden;
  if (pair >= (int64_t)p.tokens * p.top) return;
  const int f = id % p.hidden, e = w.chosen[pair], lane = threadIdx.x & 63;
  if (e < 0) return;
  const T* const x = (const T*)p.x + pair / p.top * p.x_stride;
  const T* const rows = (const T*)p.w_in + ((int64_t)e * 2 * p.hidden + f) * p.channels;
  const float gate = dot(x, rows, p.channels, lane), up = dot(x, rows + (int64_t)p.hidden * p.channels, p.channels, lane);
  if (lane == 0) w.hidden[pair * p.hidden + f] = gate / (1.0f + expf(-gate)) * up;
}

// A wave per token and channel.
template <class T>
__global__ __launch_bounds__(256) void k_expert_out(ExpertParams p, ExpertParts w) {
  const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, t = id / p.channels;
  if (t >= p.tokens) return;
  const int c = id % p.channels, lane = threadIdx.x & 63;
  float all = 0.0f;
  for (int i = 0; i < p.top; ++i) {
    const int e = w.chosen[t * p.top + i];
    if (e < 0) continue;
    const T* const row = (const T*)p.w_out + ((int64_t)e * p.channels + c) * p.hidden;
    const float* const h = w.hidden + (t * p.top + i) * p.hidden;
    float sum = 0.0f;
    for (int f = lane; f < p.hidden; f += 64) sum = fmaf(h[f], (float)row[f], sum);
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    all = fmaf(w.weights[t * p.top + i], sum, all);
  }
  if (lane == 0) ((T*)p.out)[t * p.out_stride + c] = (T)all;
}

template <class T>
hipError_t launch_of(const ExpertParams& p, hipStream_t stream) {
  ExpertParams params = p;
  ExpertParts parts = parts_of(p);
  void* args[] = {&params, &parts};
  hipError_t e = launch_kernel((const void*)k_expert_route<T>, p.tokens, 64, args, stream);
  if (e == hipSuccess) e = launch_kernel((const void*)k_expert_in<T>, ((int64_t)p.tokens * p.top * p.hidden + 3) / 4, 256, args, stream);
  if (e == hipSuccess) e = launch_kernel((const void*)k_expert_out<T>, ((int64_t)p.tokens * p.channels + 3) / 4, 256, args, stream);
  return e;
}
}  // namespace

size_t expert_workspace(const ExpertParams& p) {
  ExpertParams q = p;
  q.parts = nullptr;
  return parts_of(q).bytes;
}

hipError_t launch(const ExpertParams& p, hipStream_t stream) {
  return p.dtype == HS_F16 ? launch_of<f16>(p, stream) : launch_of<bf16>(p, stream);
}

}  // namespace hs
