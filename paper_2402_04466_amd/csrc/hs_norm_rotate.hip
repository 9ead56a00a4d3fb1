// hs_norm_rotate: norms of queries and keys per head, and their rotation by position, in one pass.
#include "hs_track_device.h"

#include <algorithm>

namespace hs {

// y = x * rsqrt(mean(x^2) + eps) * w; pairs (a, b) of the first `rotary` values turned by t = position * frequency.
//
// Bound by reading and writing every value once.  A head is held by LANES = 2, 4, 8 or 16 lanes with 8 values (16
// bytes) each; a group of LANES lanes takes one token and up to HEADS of its heads one after the other, so that the
// token's sines and cosines, folded into the weights (own value times A plus partner's times B), are formed once
// and stay in registers.  The partner's values come from the lane that has them (half layout) or are the lane's
// own (interleaved).
template <class T, int LANES>
__global__ __launch_bounds__(256) void k_norm_rotate(NormRotateParams p, int heads_per_group, int q_blocks, int k_blocks) {
  typedef typename Vec<T>::x8 x8;
  const int lane = threadIdx.x % LANES, lane0 = (threadIdx.x & 63) - lane;
  const int64_t group = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int blocks = q_blocks + k_blocks;
  const int64_t row = group / blocks;
  if (row >= (int64_t)p.batch * p.tokens) return;
  const int block = (int)(group % blocks);
  const int64_t b = row / p.tokens, t = row % p.tokens;
  const bool is_q = block < q_blocks;
  const Heads& in = is_q ? p.q : p.k;
  const Heads& out = is_q ? p.q_out : p.k_out;
  const float* const w = is_q ? p.wq : p.wk;
  const int h0 = (is_q ? block : block - q_blocks) * heads_per_group;
  const int h1 = min(h0 + heads_per_group, is_q ? p.q_heads : p.k_heads);
  const int c0 = 8 * lane;                       // the lane's first value of the head
  const bool there = c0 < p.dim, turned = c0 < p.rotary;
  const int half = p.rotary / 2;
  // the lane that holds the other values of this lane's pairs (half layout)
  const int partner = lane0 + (p.interleaved || !turned ? lane : c0 < half ? lane + half / 8 : lane - half / 8);
  const int p0 = 8 * (partner - lane0);

  float A[8], B[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    A[i] = w && there ? w[c0 + i] : 1.0f;
    B[i] = 0.0f;
  }
  if (turned) {
    const double pos = (double)(p.pos ? p.pos[b * p.pos_batch + t] : p.first + t);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // whole turns are taken off in 64 bits: what is left is exact to 2^-53 of the position's turns
      const int f = p.interleaved ? (c0 + i) / 2 : (c0 + i) % half;
      const double turns = pos * p.freq[f] * 0.15915494309189533577;
      float sine, cosine;
      sincospif(2.0f * (float)(turns - rint(turns)), &sine, &cosine);
      const bool first = p.interleaved ? i % 2 == 0 : c0 < half;
      const int other = p.interleaved ? c0 + (i ^ 1) : p0 + i;
      B[i] = (first ? -sine : sine) * (w ? w[other] : 1.0f);
      A[i] *= cosine;
    }
  }
  for (int h = h0; h < h1; ++h) {
    x8 x = {};
    if (there) x = *(const x8*)(at<T>(in, b, t, h) + c0);
    float inv = 1.0f;
    if (p.norm) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf((float)x[i], (float)x[i], sum);
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
      inv = 1.0f / sqrtf(sum / (float)p.dim + p.eps);
    }
    x8 o = x;
    if (p.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = x[i ^ 1];
    } else {
      uint32_t words[4];
      __builtin_memcpy(words, &x, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) words[i] = __shfl(words[i], partner);
      __builtin_memcpy(&o, words, 16);
    }
    x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = (float)x[i] * inv * A[i];
      y[i] = (T)(turned ? fmaf((float)o[i] * inv, B[i], a) : a);
    }
    if (there) *(x8*)(at_out<T>(out, b, t, h) + c0) = y;
  }
}

template <class T>
static const void* kernel_of(int lanes) {
  switch (lanes) {
    case 2: return (const void*)k_norm_rotate<T, 2>;
    case 4: return (const void*)k_norm_rotate<T, 4>;
    case 8: return (const void*)k_norm_rotate<T, 8>;
    default: return (const void*)k_norm_rotate<T, 16>;
  }
}

hipError_t launch(const NormRotateParams& p, hipStream_t stream) {
  int lanes = 2;
  while (8 * lanes < p.dim) lanes *= 2;
  const int64_t rows = (int64_t)p.batch * p.tokens;
  // all heads of a token in one group where there are tokens enough for the device, else fewer
  int heads = std::max(p.q_heads, p.k_heads), q_blocks, k_blocks;
  for (;; heads = (heads + 1) / 2) {
    q_blocks = (p.q_heads + heads - 1) / heads;
    k_blocks = (p.k_heads + heads - 1) / heads;
    if (heads == 1 || rows * (q_blocks + k_blocks) * lanes >= 64 * 4096) break;
  }
  NormRotateParams params = p;
  void* args[] = {&params, &heads, &q_blocks, &k_blocks};
  const int64_t groups = rows * (q_blocks + k_blocks);
  return launch_kernel(p.dtype == HS_F16 ? kernel_of<f16>(lanes) : kernel_of<bf16>(lanes), (groups * lanes + 255) / 256, 256, args, stream);
}

}  // namespace hs
