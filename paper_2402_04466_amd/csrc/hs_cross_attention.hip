// hs_cross_attention: attention of tokens to an encoder's states of another length.
#include "hs_track_device.h"

#include <math.h>

namespace hs {

// One wave per token and head: 64 keys at a time, one per lane; running maximum and sum; then the values, two
// dimensions per lane.
template <class T>
__global__ __launch_bounds__(64) void k_cross_wave(CrossParams p) {
  typedef typename Vec<T>::x8 x8;
  __shared__ float s_q[128];
  __shared__ float s_p[64];
  const int lane = threadIdx.x;
  const int64_t id = blockIdx.x;
  const int t = (int)(id % p.q_tokens);
  const int64_t bh = id / p.q_tokens;
  const int h = (int)(bh % p.q_heads), hk = h / p.group;
  const int64_t b = bh / p.q_heads;
  for (int i = lane; i < p.dim; i += 64) s_q[i] = (float)at<T>(p.q, b, t, h)[i] * p.scale;
  __syncthreads();
  const int n = length_of(p.lengths, b, p.k_tokens);
  float top = -INFINITY, sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const bool seen = j < n && (!p.mask || p.mask[b * p.mask_batch + j]);
    float s = -INFINITY;
    if (seen) {
      const T* const k = at<T>(p.k, b, j, hk);
      s = 0.0f;
      for (int i = 0; i < p.dim; i += 8) {
        const x8 x = *(const x8*)(k + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(s_q[i + e], (float)x[e], s);
      }
    }
    uint64_t left = __ballot(seen);
    if (!left) continue;
    float m = s;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    m = fmaxf(m, top);
    const float e = seen ? expf(s - m) : 0.0f, keep = expf(top - m);
    top = m;
    float part = e;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) part += __shfl_xor(part, d);
    sum = fmaf(sum, keep, part);
    s_p[lane] = e;
    __syncthreads();
    o0 *= keep;
    o1 *= keep;
    while (left) {
      const int i = __ffsll((unsigned long long)left) - 1;
      left &= left - 1;
      const T* const v = at<T>(p.v, b, j0 + i, hk);
      if (lane < p.dim) o0 = fmaf(s_p[i], (float)v[lane], o0);
      if (lane + 64 < p.dim) o1 = fmaf(s_p[i], (float)v[lane + 64], o1);
    }
    __syncthreads();
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  T* const out = at_out<T>(p.out, b, t, h);
  if (lane < p.dim) out[lane] = (T)(o0 * inv);
  if (lane + 64 < p.dim) out[lane + 64] = (T)(o1 * inv);
  if (p.lse && lane == 0) p.lse[bh * p.q_tokens + t] = top + logf(sum);
}

hipError_t launch(const CrossParams& p, hipStream_t stream) {
  CrossParams params = p;
  void* args[] = {&params};
  return launch_kernel(p.dtype == HS_F16 ? (const void*)k_cross_wave<f16> : (const void*)k_cross_wave<bf16>,
                       (int64_t)p.batch * p.q_heads * p.q_tokens, 64, args, stream);
}

}  // namespace hs
