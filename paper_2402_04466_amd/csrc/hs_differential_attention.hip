// hs_differential_attention: the difference of two softmax maps over the same values.
#include "hs_track_device.h"

#include <math.h>

#include <algorithm>

namespace hs {

// A wave per token and head: 64 keys at a time, a key per lane for the scores, two values per lane for the sums.
template <class T>
__global__ __launch_bounds__(64) void k_differential(DifferentialParams p) {
  typedef typename Vec<T>::x8 x8;
  __shared__ float q[2][128], w[2][64];
  const int lane = threadIdx.x;
  const int64_t id = blockIdx.x;
  const int h = id % p.q_heads, hk = h / p.group;
  const int64_t token = id / p.q_heads % p.q_tokens, b = id / p.q_heads / p.q_tokens;
  const int n = length_of(p.lengths, b, p.k_tokens);
  for (int i = lane; i < 2 * p.dim; i += 64) q[i / p.dim][i % p.dim] = (float)at<T>(p.q, b, token, 2 * h + i / p.dim)[i % p.dim];
  __syncthreads();
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {}, o[2][2] = {};
  for (int64_t j0 = 0; j0 < n; j0 += 64) {
    const int64_t j = j0 + lane;
    const bool seen = j < n && (!p.mask || p.mask[b * p.mask_batch + j]);
    const uint64_t visible = __ballot(seen);
    if (!visible) continue;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float s = -INFINITY;
      if (seen) {
        const T* const k = at<T>(p.k, b, j, 2 * hk + a);
        s = 0.0f;
        for (int d = 0; d < p.dim; d += 8) {
          const x8 kk = *(const x8*)(k + d);
#pragma unroll
          for (int i = 0; i < 8; ++i) s = fmaf((float)kk[i], q[a][d + i], s);
        }
        s *= p.scale;
      }
      float top = s;
      for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      const float raised = fmaxf(m[a], top), keep = m[a] == -INFINITY ? 0.0f : expf(m[a] - raised);
      const float e = !seen ? 0.0f : expf(s - (raised == -INFINITY ? 0.0f : raised));
      float sum = e;
      for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
      l[a] = l[a] * keep + sum;
      o[a][0] *= keep;
      o[a][1] *= keep;
      m[a] = raised;
      w[a][lane] = e;
    }
    __syncthreads();
    for (int i = 0; i < 64; ++i) {
      if (!(visible >> i & 1)) continue;
      const T* const v = at<T>(p.v, b, j0 + i, hk);
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        if (lane + 64 * d >= p.value_dim) continue;
        const float x = (float)v[lane + 64 * d];
        o[0][d] = fmaf(w[0][i], x, o[0][d]);
        o[1][d] = fmaf(w[1][i], x, o[1][d]);
      }
    }
    __syncthreads();
  }
  const float lambda = p.lambda[h];
  float y[2] = {}, square = 0.0f;
  const bool none = l[0] == 0.0f && l[1] == 0.0f;
#pragma unroll
  for (int d = 0; d < 2; ++d)
    if (!none && lane + 64 * d < p.value_dim) {
      y[d] = o[0][d] / l[0] - lambda * (o[1][d] / l[1]);
      square = fmaf(y[d], y[d], square);
    }
  for (int d = 1; d < 64; d *= 2) square += __shfl_xor(square, d);
  const float inv = !p.norm ? 1.0f : none ? 0.0f : rsqrtf(square / (float)p.value_dim + p.eps);
  T* const out = at_out<T>(p.out, b, token, h);
#pragma unroll
  for (int d = 0; d < 2; ++d)
    if (lane + 64 * d < p.value_dim) out[lane + 64 * d] = (T)(y[d] * inv * (p.weight ? p.weight[lane + 64 * d] : 1.0f));
}

size_t differential_workspace(const DifferentialParams&) { return 0; }

hipError_t launch(const DifferentialParams& p, hipStream_t stream) {
  DifferentialParams params = p;
  void* args[] = {&params};
  return launch_kernel(p.dtype == HS_F16 ? (const void*)k_differential<f16> : (const void*)k_differential<bf16>,
                       (int64_t)p.batch * p.q_tokens * p.q_heads, 64, args, stream);
}

}  // namespace hs
