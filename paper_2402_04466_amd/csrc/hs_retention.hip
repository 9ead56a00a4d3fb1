// hs_retention: linear attention with a decay for each head.
#include "hs_track_device.h"

namespace hs {

// Recurrent form: S = decay * S + k v^T, out = scale * q S, token by token.  A workgroup holds key_dim x 64 values of
// one sequence's and head's state in registers: 16 lanes side by side have 4 values of 16 bytes each, so a row of
// the state is read in 256-byte pieces, and thread group g of 16 has the rows g, g + 16, ...
template <class T, int ROWS>
__global__ __launch_bounds__(256) void k_retain_steps(RetentionParams p) {
  typedef typename Vec<T>::x4 x4;
  __shared__ f32x4 partial[2][4][16];
  const int blocks = (p.value_dim + 63) / 64;
  const int block = blockIdx.x % blocks;
  const int64_t bh = blockIdx.x / blocks;
  const int h = (int)(bh % p.q_heads), hk = h / p.group;
  const int64_t b = bh / p.q_heads;
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int dv0 = 64 * block + 4 * c;
  const bool there = dv0 < p.value_dim;
  const int64_t state0 = bh * p.key_dim * p.value_dim + dv0;

  f32x4 S[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int dk = g + 16 * r;
    S[r] = f32x4{0, 0, 0, 0};
    if (p.state_in && there && dk < p.key_dim) S[r] = *(const f32x4*)(p.state_in + state0 + (int64_t)dk * p.value_dim);
  }
  const int n = length_of(p.lengths, b, p.tokens);
  // (an fp32 decay near one is 2^-25 off, which 7200 steps raise to 2e-4 of the state)
  const float decay = p.decay[h], rest = p.decay_rest[h];
  for (int t = 0; t < n; ++t) {
    const T* const q = at<T>(p.q, b, t, h);
    const T* const k = at<T>(p.k, b, t, hk);
    f32x4 v = {0, 0, 0, 0}, o = {0, 0, 0, 0};
    if (there) {
      const x4 raw = *(const x4*)(at<T>(p.v, b, t, hk) + dv0);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (float)raw[i];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int dk = g + 16 * r;
      if (dk < p.key_dim) {
        const float kk = (float)k[dk], qq = (float)q[dk];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          S[r][i] = fmaf(decay, S[r][i], fmaf(rest, S[r][i], kk * v[i]));
          o[i] = fmaf(qq, S[r][i], o[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] += __shfl_xor(o[i], 16);
      o[i] += __shfl_xor(o[i], 32);
    }
    if ((threadIdx.x & 63) < 16) partial[t & 1][wave][c] = o;
    __syncthreads();   // the other half of `partial` is written before the next one
    if (threadIdx.x < 16 && there) {
      x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        y[i] = (T)(p.scale * ((partial[t & 1][0][c][i] + partial[t & 1][1][c][i]) + (partial[t & 1][2][c][i] + partial[t & 1][3][c][i])));
      *(x4*)(at_out<T>(p.out, b, t, h) + dv0) = y;
    }
  }
  if (there)
    for (int t = n + g; t < p.tokens; t += 16) *(x4*)(at_out<T>(p.out, b, t, h) + dv0) = x4{};
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int dk = g + 16 * r;
    if (there && dk < p.key_dim) *(f32x4*)(p.state_out + state0 + (int64_t)dk * p.value_dim) = S[r];
  }
}

// Chunked form: 64 tokens at a time, products on the matrix pipe.  With c tokens in a chunk, S the state before it and
// i, j = 0 .. c - 1:
//   A_ij = scale * decay^(i - j) q_i k_j (j <= i)          out_i = sum_j A_ij v_j + scale * decay^(i + 1) S^T q_i
//   S   <- decay^c S + sum_j k_j (decay^(c - 1 - j) v_j)^T
// A workgroup has one sequence and head and 64 of the values' dimensions, 16 per wave.  The four waves share
// the lower triangle of A (through LDS); all else of a chunk is a wave's own: its slice of the state stays in the
// accumulators, whose layout is at once that of the operand S^T of the next chunk's S^T Q^T, if that product takes the
// key dimensions in the accumulators' order (Q is read in it).
//
// Rounded to 16 bits, as the matrix pipe takes them: A, and the copy of S that multiplies q (each term of out
// is then half a step off, as out itself); of the fp16 copy a power of two is taken out, so that it stays in
// that type's range whatever the state has grown to.  The state takes no such rounding: decayed values enter as a sum of
// three bf16 or two fp16 parts (the second scaled by 2^12, out of fp16's subnormal numbers).
constexpr int kChunk = 64;

template <class T, int KP>
__global__ __launch_bounds__(256) void k_retain_chunks(RetentionParams p) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int CH = KP / 8, KT = KP / 16, KS = KP / 32;
  constexpr int RP = 256 / CH, NL = kChunk / RP;    // rows per pass of the workgroup over Q or K, passes
  constexpr bool kHalf = __is_same(T, f16);
  constexpr int kQ = 0, kK = kChunk * KP * 2, kV = 2 * kK, kA = kV + kChunk * 64 * 2;
  __shared__ __align__(16) char lds[kA + kChunk * kChunk * 2];
  __shared__ double power[kChunk + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int blocks = (p.value_dim + 63) / 64;
  const int id = xcd_number(), block = id % blocks, bh = id / blocks, h = bh % p.q_heads, hk = h / p.group, b = bh / p.q_heads;
  const int n = length_of(p.lengths, b, p.tokens), chunks = (int)(((int64_t)n + kChunk - 1) / kChunk);
  const int dv0 = 64 * block + 16 * wave;           // the wave's 16 dimensions

  if (threadIdx.x <= kChunk) power[threadIdx.x] = exp2(p.log2_decay[h] * threadIdx.x);

  // staging: this thread's 16-byte chunk of rows r0, r0 + RP, ... of Q and K, and of V (8 chunks per row)
  const int r0 = threadIdx.x / CH, ch = threadIdx.x % CH, vr0 = threadIdx.x / 8, vch = threadIdx.x % 8;
  const bool in_k = 8 * ch < p.key_dim, in_v = 64 * block + 8 * vch < p.value_dim;
  const T* const qsrc = at<T>(p.q, b, 0, h) + 8 * ch;
  const T* const ksrc = at<T>(p.k, b, 0, hk) + 8 * ch;
  const T* const vsrc = at<T>(p.v, b, 0, hk) + 64 * block + 8 * vch;
  s16x8 qreg[NL], kreg[NL], vreg[2];
  auto fetch = [&](int t0) {
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int t = t0 + r0 + e * RP;
      qreg[e] = kreg[e] = s16x8{};
      if (t < n && in_k) {
        qreg[e] = *(const s16x8*)(qsrc + t * p.q.token);
        kreg[e] = *(const s16x8*)(ksrc + t * p.k.token);
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int t = t0 + vr0 + e * 32;
      vreg[e] = s16x8{};
      if (t < n && in_v) vreg[e] = *(const s16x8*)(vsrc + t * p.v.token);
    }
  };
  if (chunks) fetch(0);

  // the state's slice: lane has dimension dv0 + l16, key dimensions 16 t + 4 g + i
  f32x4 S[KT];
  const int64_t state0 = (int64_t)bh * p.key_dim * p.value_dim + dv0 + l16;
  const bool in_state = dv0 + l16 < p.value_dim;
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int dk = 16 * t + 4 * g + i;
      S[t][i] = p.state_in && in_state && dk < p.key_dim ? p.state_in[state0 + (int64_t)dk * p.value_dim] : 0.0f;
    }

  __syncthreads();
  float diagonal[4][4], after[4], weight[2][8];     // decays of A's tiles by distance, of S in out_i, of v_j in S
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    after[d] = p.scale * (float)power[16 * d + l16 + 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int apart = 16 * d + l16 - 4 * g - i;
      diagonal[d][i] = apart < 0 ? 0.0f : p.scale * (float)power[apart];
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) weight[s][i] = (float)power[kChunk - 1 - (32 * s + 8 * g + i)];
  float keep = (float)power[kChunk], keep_rest = (float)(power[kChunk] - (double)keep);

  for (int c = 0; c < chunks; ++c) {
    const int t0 = c * kChunk, left = min(n - t0, kChunk);
    if (c) __syncthreads();                         // the chunk before this one has been read
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      *(s16x8*)(lds + kQ + slot<CH>(r0 + e * RP, ch)) = qreg[e];
      *(s16x8*)(lds + kK + slot<CH>(r0 + e * RP, ch)) = kreg[e];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) *(s16x8*)(lds + kV + slot<8>(vr0 + e * 32, vch)) = vreg[e];
    __syncthreads();
    if (c + 1 < chunks) fetch(t0 + kChunk);

    // A's ten tiles on and below the diagonal, dealt to the waves: tile (row block, column block)
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      const int tile = wave + 4 * e;
      if (tile >= 10) break;
      const int rb = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, cb = tile - rb * (rb + 1) / 2;
      f32x4 a = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < KS; ++s)
        a = mfma16(*(const x8*)(lds + kK + slot<CH>(16 * cb + l16, 4 * s + g)), *(const x8*)(lds + kQ + slot<CH>(16 * rb + l16, 4 * s + g)), a);
      x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float d = diagonal[0][i];
        d = rb - cb == 1 ? diagonal[1][i] : d;
        d = rb - cb == 2 ? diagonal[2][i] : d;
        d = rb - cb == 3 ? diagonal[3][i] : d;
        r[i] = (T)(a[i] * d);
      }
      *(x4*)(lds + kA + slot<8>(16 * rb + l16, 2 * cb + (g >> 1)) + (g & 1) * 8) = r;
    }
    // (tile (0, 1) and (2, 3), right of the diagonal but within a step of 32 keys, are zeros from the start)
    if (c == 0 && wave < 2) *(x4*)(lds + kA + slot<8>(32 * wave + l16, 4 * wave + 2 + (g >> 1)) + (g & 1) * 8) = x4{};
    __syncthreads();

    // V^T, the operand of both products: dimension 16 * wave + l16, tokens 32 s + 8 g + i
    x8 v[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int r = 32 * s + 8 * g + (lane >> 2 & 3), cc = 2 * wave + (lane >> 1 & 1);
      v[s] = join8<T>(read_transposed(lds + kV + slot<8>(r, cc) + (lane & 1) * 8), read_transposed(lds + kV + slot<8>(r + 4, cc) + (lane & 1) * 8));
    }
    int exponent = 0;                               // of what is taken out of the copy
    if (kHalf) {
      float most = 0.0f;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(S[t][i]));
#pragma unroll
      for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
      exponent = max(min(__builtin_amdgcn_frexp_expf(most) - 12, 100), -100);
    }
    x8 s16[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) s16[s][i] = (T)(kHalf ? ldexpf(S[2 * s + i / 4][i % 4], -exponent) : S[2 * s + i / 4][i % 4]);
    f32x4 out[4];
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      f32x4 o = {0, 0, 0, 0};
      const int r = 16 * rb + l16;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const x4 q0 = *(const x4*)(lds + kQ + slot<CH>(r, 4 * s + (g >> 1)) + (g & 1) * 8);
        const x4 q1 = *(const x4*)(lds + kQ + slot<CH>(r, 4 * s + 2 + (g >> 1)) + (g & 1) * 8);
        o = mfma16(s16[s], __builtin_shufflevector(q0, q1, 0, 1, 2, 3, 4, 5, 6, 7), o);
      }
      o *= kHalf ? ldexpf(after[rb], exponent) : after[rb];
#pragma unroll
      for (int s = 0; s <= rb / 2; ++s) o = mfma16(v[s], *(const x8*)(lds + kA + slot<8>(r, 4 * s + g)), o);
      out[rb] = o;
    }

    // the state
    if (left < kChunk) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) weight[s][i] = (float)power[max(left - 1 - (32 * s + 8 * g + i), 0)];   // (later values are zeros)
      keep = (float)power[left];
      keep_rest = (float)(power[left] - (double)keep);
    }
    x8 part[2][3];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x = (float)v[s][i] * weight[s][i];
        asm("" : "+v"(x));   // the rounded product: rounded to 16 bits from the exact one in one place and from this in another, a part
                             // and what is left of it would not belong together
        part[s][0][i] = (T)x;
        x -= (float)part[s][0][i];
        if (kHalf) x *= 4096.0f;
        part[s][1][i] = (T)x;
        if (!kHalf) part[s][2][i] = (T)(x - (float)part[s][1][i]);
      }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) S[t][i] = fmaf(S[t][i], keep, S[t][i] * keep_rest);
      f32x4 low = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int r = 32 * s + 8 * g + (lane >> 2 & 3), cc = 2 * t + (lane >> 1 & 1);
        const x8 k = join8<T>(read_transposed(lds + kK + slot<CH>(r, cc) + (lane & 1) * 8), read_transposed(lds + kK + slot<CH>(r + 4, cc) + (lane & 1) * 8));
        S[t] = mfma16(k, part[s][0], S[t]);
        if (kHalf) {
          low = mfma16(k, part[s][1], low);
        } else {
          S[t] = mfma16(k, part[s][1], S[t]);
          S[t] = mfma16(k, part[s][2], S[t]);
        }
      }
      if (kHalf) S[t] += low * (1.0f / 4096.0f);
    }
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (T)out[rb][i];
      const int r = 16 * rb + l16;
      if (r < left && dv0 + 4 * g < p.value_dim) *(x4*)(at_out<T>(p.out, b, t0 + r, h) + dv0 + 4 * g) = y;
    }
  }
  if (in_v)
    for (int t = n + vr0; t < p.tokens; t += 32) *(s16x8*)(at_out<T>(p.out, b, t, h) + 64 * block + 8 * vch) = s16x8{};
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int dk = 16 * t + 4 * g + i;
      if (in_state && dk < p.key_dim) p.state_out[state0 + (int64_t)dk * p.value_dim] = S[t][i];
    }
}

hipError_t launch(const RetentionParams& p, hipStream_t stream) {
  RetentionParams params = p;
  void* args[] = {&params};
  const int64_t workgroups = (int64_t)p.batch * p.q_heads * ((p.value_dim + 63) / 64);
  const bool wide = p.key_dim > 64, half = p.dtype == HS_F16, steps = p.tokens <= 8;
  const void* kernel;
  if (steps) kernel = half ? wide ? (const void*)k_retain_steps<f16, 8> : (const void*)k_retain_steps<f16, 4>
                           : wide ? (const void*)k_retain_steps<bf16, 8> : (const void*)k_retain_steps<bf16, 4>;
  else kernel = half ? wide ? (const void*)k_retain_chunks<f16, 128> : (const void*)k_retain_chunks<f16, 64>
                     : wide ? (const void*)k_retain_chunks<bf16, 128> : (const void*)k_retain_chunks<bf16, 64>;
  return launch_kernel(kernel, workgroups, 256, args, stream);
}

}  // namespace hs
