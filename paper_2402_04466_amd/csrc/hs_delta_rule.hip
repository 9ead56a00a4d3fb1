// hs_delta_rule: linear attention whose state gives up what it holds for a key before it takes the key's new value.
#include "hs_track_device.h"

#include <algorithm>

namespace hs {

__device__ __forceinline__ const float* gate_at(const hs_gates& g, int64_t batch, int64_t head) {
  return g.d ? g.d + batch * g.batch + head * g.head : nullptr;
}

// Recurrent form, token by token: with a = S^T k and c = S^T q of the state before the token,
//   u = beta (v - g a),  out = scale (g c + (q.k) u),  S = g S + k u^T,
// so both sums over the state are formed in one pass and joined behind one barrier.  A workgroup holds key_dim x 64 values of
// one sequence's and head's state in registers: 16 lanes side by side have 4 values of 16 bytes each, and thread group g of
// 16 has ROWS rows from ROWS * g on.
template <class T, int ROWS>
__global__ __launch_bounds__(256) void k_delta_steps(DeltaParams p) {
  typedef typename Vec<T>::x4 x4;
  typedef T xr __attribute__((ext_vector_type(ROWS)));
  __shared__ f32x4 partial[2][2][4][16];
  __shared__ float partial_qk[2][4];
  const int blocks = (p.value_dim + 63) / 64;
  const int block = blockIdx.x % blocks;
  const int bh = blockIdx.x / blocks, h = bh % p.heads, hk = h / p.group, b = bh / p.heads;
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int dv0 = 64 * block + 4 * c, dk0 = ROWS * g;
  const bool in_v = dv0 < p.value_dim, in_k = dk0 < p.key_dim, there = in_v && in_k;
  const int64_t state0 = ((int64_t)bh * p.key_dim + dk0) * p.value_dim + dv0;
  const T* const q = at<T>(p.q, b, 0, hk) + dk0;
  const T* const k = at<T>(p.k, b, 0, hk) + dk0;
  const T* const v = at<T>(p.v, b, 0, h) + dv0;
  const float* const log_decay = gate_at(p.log_decay, b, h);
  const float* const beta = gate_at(p.beta, b, h);
  T* const out = at_out<T>(p.out, b, 0, h) + dv0;
  const int n = length_of(p.lengths, b, p.tokens);

  f32x4 s[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    s[r] = f32x4{0, 0, 0, 0};
    if (there && p.state_in) s[r] = *(const f32x4*)(p.state_in + state0 + (int64_t)r * p.value_dim);
  }
  xr kt = {}, qt = {};
  x4 vt = {};
  float lt = 0.0f, bt = 1.0f;
  auto fetch = [&](int64_t t) {
    if (in_k) {
      kt = *(const xr*)(k + t * p.k.token);
      qt = *(const xr*)(q + t * p.q.token);
    }
    if (in_v) vt = *(const x4*)(v + t * p.v.token);
    if (log_decay) lt = log_decay[t * p.log_decay.token];
    if (beta) bt = beta[t * p.beta.token];
  };
  if (n > 0) fetch(0);
  for (int t = 0; t < n; ++t) {
    const xr k0 = kt, q0 = qt;
    const x4 v0 = vt;
    const float decay = expf(lt), b0 = bt;
    if (t + 1 < n) fetch(t + 1);
    f32x4 a = {0, 0, 0, 0}, e = {0, 0, 0, 0};
    float qk = 0.0f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      a += (float)k0[r] * s[r];
      e += (float)q0[r] * s[r];
      qk = fmaf((float)q0[r], (float)k0[r], qk);
    }
#pragma unroll
    for (int d = 16; d < 64; d *= 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] += __shfl_xor(a[i], d);
        e[i] += __shfl_xor(e[i], d);
      }
      qk += __shfl_xor(qk, d);
    }
    const int buffer = t & 1;
    if ((threadIdx.x & 48) == 0) {
      partial[buffer][0][wave][c] = a;
      partial[buffer][1][wave][c] = e;
      if (c == 0) partial_qk[buffer][wave] = qk;
    }
    __syncthreads();
    a = (partial[buffer][0][0][c] + partial[buffer][0][1][c]) + (partial[buffer][0][2][c] + partial[buffer][0][3][c]);
    e = (partial[buffer][1][0][c] + partial[buffer][1][1][c]) + (partial[buffer][1][2][c] + partial[buffer][1][3][c]);
    qk = (partial_qk[buffer][0] + partial_qk[buffer][1]) + (partial_qk[buffer][2] + partial_qk[buffer][3]);
    f32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = b0 * ((float)v0[i] - decay * a[i]);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s[r] = decay * s[r] + (float)k0[r] * u;
    if (g == 0 && in_v) *(x4*)(out + t * p.out.token) = round4<T>(p.scale * (decay * e + qk * u));
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
    if (there) *(f32x4*)(p.state_out + state0 + (int64_t)r * p.value_dim) = s[r];
  if (in_v)
    for (int64_t t = n + g; t < p.tokens; t += 16) *(x4*)(out + t * p.out.token) = x4{};
}

size_t delta_workspace(const DeltaParams&) { return 0; }

template <class T>
static const void* steps_of(const DeltaParams& p) {
  return p.key_dim <= 64 ? (const void*)k_delta_steps<T, 4> : (const void*)k_delta_steps<T, 8>;
}

hipError_t launch(const DeltaParams& p, hipStream_t stream) {
  DeltaParams params = p;
  void* args[] = {&params};
  const int64_t workgroups = (int64_t)p.batch * p.heads * ((p.value_dim + 63) / 64);
  return launch_kernel(p.dtype == HS_F16 ? steps_of<f16>(p) : steps_of<bf16>(p), workgroups, 256, args, stream);
}

}  // namespace hs
