// hs_norm_rotate: norms of queries and keys per head, and their rotation by position, in one pass.
#include "hs_track_device.h"

#include <algorithm>

namespace hs {

// y = x * rsqrt(mean(x^2) + eps) * w; pairs (a, b) of the first `rotary` values turned by t = position * frequency.
//
// Bound by reading and writing every value once (345600 tokens of 16 heads of 64: 263 us, 5.4 TB/s).  A head is held by LANES = 2, 4, 8 or 16 lanes with 8 values (16
// bytes) each; a group of LANES lanes takes one token and some of its heads, four at a time, so that the token's
// sines and cosines, folded into the weights (own value times A plus partner's times B), are formed once and stay in
// registers, behind the loads of the first four heads.  The partner's values come from the lane that has them (half layout)
// or are the lane's own (interleaved).

// Sum over the LANES lanes of a group, in each of them: neighbours, pairs, then mirrored halves, whose lanes agree by then.
template <int LANES>
__device__ __forceinline__ float group_sum(float x) {
  x += moved<0xb1>(x);                     // lane ^ 1
  if (LANES > 2) x += moved<0x4e>(x);      // lane ^ 2
  if (LANES > 4) x += moved<0x141>(x);     // 7 - lane
  if (LANES > 8) x += moved<0x140>(x);     // 15 - lane
  return x;
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));     // as the caller's pointers are aligned
typedef double f64x2_any __attribute__((ext_vector_type(2), aligned(8)));
__device__ __forceinline__ void load8(const float* from, float* to) {
  const f32x4_any a = *(const f32x4_any*)from, b = *(const f32x4_any*)(from + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    to[i] = a[i];
    to[4 + i] = b[i];
  }
}
// Eight pairs' frequencies, or the four of a lane that holds both values of its pairs.
__device__ __forceinline__ void load_frequencies(const double* from, bool four, double* to) {
  const f64x2_any a = *(const f64x2_any*)from, b = *(const f64x2_any*)(from + 2);
  to[0] = a[0], to[1] = a[1], to[2] = b[0], to[3] = b[1];
  if (four) return;
  const f64x2_any c = *(const f64x2_any*)(from + 4), d = *(const f64x2_any*)(from + 6);
  to[4] = c[0], to[5] = c[1], to[6] = d[0], to[7] = d[1];
}

template <class T, int LANES>
__global__ __launch_bounds__(256) void k_norm_rotate(NormRotateParams p, int heads_per_group, int q_blocks, int k_blocks) {
  typedef typename Vec<T>::x8 x8;
  constexpr int kAhead = 4;
  const int lane = threadIdx.x % LANES, lane0 = (threadIdx.x & 63) - lane;
  const uint32_t group = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, blocks = q_blocks + k_blocks;
  const uint32_t row = group / blocks, block = group % blocks;
  if (row >= (uint32_t)p.batch * (uint32_t)p.tokens) return;
  const uint32_t b = row / (uint32_t)p.tokens, t = row % (uint32_t)p.tokens;
  const bool is_q = block < (uint32_t)q_blocks;
  const int h0 = (is_q ? block : block - q_blocks) * heads_per_group;
  const int h1 = min(h0 + heads_per_group, is_q ? p.q_heads : p.k_heads);
  const int c0 = 8 * lane;                       // the lane's first value of the head
  const bool there = c0 < p.dim, turned = c0 < p.rotary;
  const int64_t in_head = is_q ? p.q.head : p.k.head, out_head = is_q ? p.q_out.head : p.k_out.head;
  const T* from = (is_q ? at<T>(p.q, b, t, h0) : at<T>(p.k, b, t, h0)) + c0;
  T* to = (is_q ? at_out<T>(p.q_out, b, t, h0) : at_out<T>(p.k_out, b, t, h0)) + c0;
  x8 x[kAhead];
#pragma unroll
  for (int e = 0; e < kAhead; ++e) {
    x[e] = x8{};
    if (there && h0 + e < h1) x[e] = *(const x8*)(from + e * in_head);
  }

  const float* const w = is_q ? p.wq : p.wk;
  const int half = p.rotary / 2;
  // the lane that holds the other values of this lane's pairs (half layout)
  const int partner = lane0 + (p.interleaved || !turned ? lane : c0 < half ? lane + half / 8 : lane - half / 8);
  const int p0 = 8 * (partner - lane0);
  // weights and frequencies: whole vectors, behind one branch each
  float weight[8], other[8], A[8], B[8];          // the lane's, and its pairs' other values'
#pragma unroll
  for (int i = 0; i < 8; ++i) weight[i] = other[i] = 1.0f;
  if (w && there) {
    load8(w + c0, weight);
    load8(w + p0, other);
  }
  double freq[8] = {};
  int64_t place = p.first + t;
  if (turned) {
    load_frequencies(p.freq + (p.interleaved ? c0 / 2 : c0 < half ? c0 : c0 - half), p.interleaved, freq);
    if (p.pos) place = p.pos[b * p.pos_batch + t];
  }
  const double pos = (double)place * 0.15915494309189533577;
  // Whole turns are taken off in 64 bits, which leaves 2^-53 of the position's turns; the sine and cosine instructions take
  // turns, and are within 1.25e-7 of the value over all of -1/2 .. 1/2.
  auto angle = [&](double f, float& sine, float& cosine) {
    const double turns = pos * f;
    const float part = (float)(turns - rint(turns));
    sine = __builtin_amdgcn_sinf(part);
    cosine = __builtin_amdgcn_cosf(part);
  };
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float sine, cosine;
      angle(freq[i / 2], sine, cosine);
      A[i] = cosine * weight[i];
      A[i + 1] = cosine * weight[i + 1];
      B[i] = -sine * weight[i + 1];
      B[i + 1] = sine * weight[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float sine, cosine;
      angle(freq[i], sine, cosine);
      A[i] = cosine * weight[i];
      B[i] = (c0 < half ? -sine : sine) * other[i];
    }
  }
  if (!turned) {
#pragma unroll
    for (int i = 0; i < 8; ++i) A[i] = weight[i];
  }
  const float mean = 1.0f / (float)p.dim;
  for (int h = h0; h < h1; h += kAhead) {
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      if (h + e >= h1) break;
      float inv = 1.0f;
      if (p.norm) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf((float)x[e][i], (float)x[e][i], sum);
        inv = rsqrtf(fmaf(group_sum<LANES>(sum), mean, p.eps));
      }
      x8 o;
      if (p.interleaved) {
        o = __builtin_shufflevector(x[e], x[e], 1, 0, 3, 2, 5, 4, 7, 6);
      } else {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        u32x4 words = __builtin_bit_cast(u32x4, x[e]);
#pragma unroll
        for (int i = 0; i < 4; ++i) words[i] = __shfl(words[i], partner);
        o = __builtin_bit_cast(x8, words);
      }
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = (float)x[e][i] * A[i];
        y[i] = inv * (turned ? fmaf((float)o[i], B[i], a) : a);
      }
      if (there) *(x8*)(to + (h - h0 + e) * out_head) = round8<T>(y);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
      if (there && h + kAhead + e < h1) x[e] = *(const x8*)(from + (h - h0 + kAhead + e) * in_head);
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
  // All heads of a token in one group, so that its angles are formed once, where that fills the device (2400 tokens of 16 and 4
  // heads of 128: 7.6 us, 11.4 if half as full is enough, 9.0 if twice is asked for), else fewer; and not so many that groups of
  // the side with more heads last far longer (14424 tokens of 8 and 2 heads of 96: 14.7 us, 16.5 without this).
  const int most = std::max(p.q_heads, p.k_heads), least = std::min(p.q_heads, p.k_heads);
  int heads = least && least < most / 2 ? 2 * least : most, q_blocks, k_blocks;
  for (;; heads = (heads + 1) / 2) {
    q_blocks = (p.q_heads + heads - 1) / heads;
    k_blocks = (p.k_heads + heads - 1) / heads;
    if (heads == 1 || rows * (q_blocks + k_blocks) * lanes >= 64 * 2048) break;
  }
  NormRotateParams params = p;
  void* args[] = {&params, &heads, &q_blocks, &k_blocks};
  const int64_t groups = rows * (q_blocks + k_blocks);
  return launch_kernel(p.dtype == HS_F16 ? kernel_of<f16>(lanes) : kernel_of<bf16>(lanes), (groups * lanes + 255) / 256, 256, args, stream);
}

}  // namespace hs
