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
// 16 has ROWS rows from ROWS * g on.  Bound by reading and writing the state (128 tracks of 16 heads of 128 x 128: 49 us, 5.5 TB/s, at five
// waves per SIMD; 78 at two); for few tracks by the chain of loads (8 of 8 heads of 64 x 64: 4.0 us).
template <class T, int ROWS>
__global__ __launch_bounds__(256, ROWS > 4 ? 4 : 6) void k_delta_steps(DeltaParams p) {
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

// ---- chunks of 32 tokens on the matrix pipe -------------------------------------------------------
//
// With L_i the sum of the decays' logarithms from the chunk's begin to token i, S the state before the chunk and
// Gamma_ij = 2^(L_i - L_j), the recurrence's u of the chunk's tokens solve a triangular system,
//   (1 + A) U = diag(beta) (V - diag(2^L) K S),     A_ij = beta_i Gamma_ij k_i.k_j for j < i,
// and  out = scale (diag(2^L) Q S + P U),           P_ij = Gamma_ij q_i.k_j for j <= i,
//      S'  = 2^L_end S + K^T diag(2^(L_end - L)) U.
// M = (1 + A)^-1 diag(beta) and P do not depend on the state: while the state's waves work on a chunk, one wave forms P of the chunk
// to come, one M from the A that another has left a chunk before, and one lays values and gates out.  A state wave has all rows of 16 of the state's columns in
// registers, and needs nothing of the others: in the layout in which products leave their results (rows 4g .. 4g + 3
// of a column in lane group g) pairs of 16 rows are operands of the next product, once its other operand is read in the order of rows
// 4g .. 4g + 3, 16 + 4g .. 16 + 4g + 3.
//
// Precision.  What enters the state is exact to 24 bits: the state and U go through the matrix pipe as three bf16 parts
// (8 bits each, rounded, what is left is exact; a value that bf16 rounds to infinity sends its chunk the way of infinities), fp16 keys and
// queries as two, M in fp32.  Outputs, which are rounded to 16 bits, take two parts of each and not the two second parts' product: at most 3 * 2^-17
// of a query times a value of the state, 2^-15 of a weight times a U.  Parts that are cut off, not rounded, lose four times that
// (8 x 7200 tokens 520 us, 531 rounded).
//
// Bound by a chunk's chain of products and splits in the state's waves, one of which a SIMD has beside one of the others: 8 x 7200 tokens of
// 16 heads of 128 x 128, 225 chunks one after the other in 256 workgroups, take 531 us, 2.4 us a chunk (vector pipe 49 %, matrix pipe 29 %, LDS
// 38 % busy; the state's waves alone 500, without their products with the state 365, without its splits 430).
constexpr int kChunk = 32, kStateWaves = 4, kOtherWaves = 4;
constexpr int kMPitch = 36;                          // floats per row of M: 16 rows' same 16 bytes lie in different banks
constexpr int kPPitch = 80;                          // bytes per row of P: as well

typedef Vec<bf16>::x8 b8;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight values as PARTS bf16 vectors that add up to them (exactly, for three), each part rounded: two parts leave at most 2^-17 of a value.
template <int PARTS>
__device__ __forceinline__ void split8(const float* x, b8* part) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int n = 0; n < PARTS; ++n) {
    part[n] = round8<bf16>(rest);
    if (n + 1 < PARTS)
#pragma unroll
      for (int i = 0; i < 8; ++i) rest[i] -= (float)part[n][i];
  }
}

// The larger of `most` and of the magnitudes, as whole numbers, of eight bf16 values: 0x7f80 and more of infinities and NaN.
__device__ __forceinline__ u16x2 most_of(u16x2 most, b8 x) {
  const u32x4 words = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, words[i] & 0x7fff7fffu));
  return most;
}

struct ChunkGates {                                  // of one chunk
  float upto_hi[kChunk], upto_lo[kChunk];            // L in two parts
  float since[kChunk], left[kChunk];                 // 2^L, 2^(L_end - L)
  float beta[kChunk], decay[kChunk];                 // decay: g itself
};

struct DeltaGrid {
  int blocks, waves;                                 // of 16 * waves value columns each
};

template <class T, int DK>
__global__ __launch_bounds__(64 * (kStateWaves + kOtherWaves)) void k_delta_chunks(DeltaParams p, DeltaGrid grid) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int NP = __is_same(T, f16) ? 2 : 1;      // bf16 parts of a key or query
  constexpr int CH = DK > 64 ? 16 : 8, KS = DK / 32, ST = DK / 16;
  constexpr int kTile = kChunk * CH * 16, kValues = kChunk * 8 * 16;
  constexpr int kQ = 0, kV = NP * kTile, kP = kV + kValues, kBuffer = kP + 2 * kChunk * kPPitch;
  __shared__ __align__(16) char lds[2 * kBuffer];
  __shared__ __align__(16) char keys[3][NP * kTile];
  __shared__ __align__(16) float ms[3][kChunk * kMPitch];      // A, then M
  __shared__ ChunkGates gates[4];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, g = lane >> 4;
  int id = xcd_number();
  const int block = id % grid.blocks, bh = id / grid.blocks, h = bh % p.heads, hk = h / p.group, b = bh / p.heads;
  const int n = length_of(p.lengths, b, p.tokens), chunks = (n + kChunk - 1) / kChunk;
  const int column0 = 16 * grid.waves * block;
  // roles: the state's waves first, then A, M, P, and values and gates
  const int role = wave < grid.waves ? 0 : 1 + wave - grid.waves;

  if (role == 0) {
    const int column = column0 + 16 * wave + row;
    const bool there = column < p.value_dim;
    const int64_t state0 = (int64_t)bh * p.key_dim * p.value_dim + column;
    f32x4 s[ST];
#pragma unroll
    for (int t = 0; t < ST; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = 16 * t + 4 * g + i;
        s[t][i] = there && p.state_in && k < p.key_dim ? p.state_in[state0 + (int64_t)k * p.value_dim] : 0.0f;
      }
    int koff[KS][2], toff[ST], voff;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) koff[k][e] = slot<CH>(row, 4 * k + 2 * e + (g >> 1)) + (g & 1) * 8;
#pragma unroll
    for (int t = 0; t < ST; ++t) toff[t] = slot<CH>(4 * g + (row >> 2), 2 * t + (row >> 1 & 1)) + (row & 1) * 8;
    voff = slot<8>(4 * g + (row >> 2), 2 * wave + (row >> 1 & 1)) + (row & 1) * 8;
    constexpr int kNext = 16 * CH * 16, kNextV = 16 * 8 * 16;     // 16 tokens further
    T* const out = at_out<T>(p.out, b, 0, h) + column0 + 16 * wave;
    const bool stored = column0 + 16 * wave + 4 * g < p.value_dim;

    __syncthreads();
    __syncthreads();
    __syncthreads();
    for (int c = 0; c < chunks; ++c) {
      const char* const here = lds + (c & 1) * kBuffer;
      const char* const k_here = keys[c % 3];
      const ChunkGates& gate = gates[c % 4];
      f32x4 ks[2] = {}, qs[2] = {};                  // K S: tokens x columns; (Q S)^T: columns x tokens
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = s[2 * k][i], x[4 + i] = s[2 * k + 1][i];
        b8 part[3];
        split8<3>(x, part);
        b8 kk[2][NP], qq[2][NP];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            const char* const at_k = k_here + e * kTile + tt * kNext;
            const char* const at_q = here + kQ + e * kTile + tt * kNext;
            kk[tt][e] = join8<bf16>(*(const s16x4*)(at_k + koff[k][0]), *(const s16x4*)(at_k + koff[k][1]));
            qq[tt][e] = join8<bf16>(*(const s16x4*)(at_q + koff[k][0]), *(const s16x4*)(at_q + koff[k][1]));
          }
        // (products that add to the same sums are kept apart: one would wait for the other)
        if (NP == 2) {
#pragma unroll
          for (int e = 1; e >= 0; --e) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) ks[tt] = mfma16(kk[tt][NP - 1], part[e], ks[tt]);
            if (e == 0)
#pragma unroll
              for (int tt = 0; tt < 2; ++tt) qs[tt] = mfma16(part[0], qq[tt][NP - 1], qs[tt]);
          }
        }
#pragma unroll
        for (int e = 2; e >= 0; --e) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) ks[tt] = mfma16(kk[tt][0], part[e], ks[tt]);
          if (e < 2)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) qs[tt] = mfma16(part[e], qq[tt][0], qs[tt]);
        }
      }
      f32x4 x[2], u[2] = {};
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const s16x4 raw = read_transposed(here + kV + voff + tt * kNextV);
        const x4 v = __builtin_bit_cast(x4, raw);
        const f32x4 since = *(const f32x4*)(gate.since + 16 * tt + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[tt][i] = (float)v[i] - since[i] * ks[tt][i];
      }
      const float* const m = ms[c % 3] + row * kMPitch + 4 * g;
      const f32x4 m00 = *(const f32x4*)m, m10 = *(const f32x4*)(m + 16 * kMPitch), m11 = *(const f32x4*)(m + 16 * kMPitch + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(m00[i], x[0][i], u[0], 0, 0, 0);
        u[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(m10[i], x[0][i], u[1], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) u[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(m11[i], x[1][i], u[1], 0, 0, 0);

      // Outputs and the state's new part are formed in one run with the above, so that their products fill the others' waits; what is
      // not finite is found out before they are kept.
      float y[8];
      b8 part[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = u[0][i], y[4 + i] = u[1][i];
      split8<2>(y, part);
      u16x2 most = most_of(u16x2{0, 0}, part[0]);
      f32x4 o[2] = {}, fresh[ST] = {};
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const char* const at_p = here + kP + (16 * tt + row) * kPPitch + 16 * g;
        const b8 hi = __builtin_bit_cast(b8, *(const s16x8*)at_p), lo = __builtin_bit_cast(b8, *(const s16x8*)(at_p + kChunk * kPPitch));
        o[tt] = mfma16(part[1], hi, o[tt]);
        o[tt] = mfma16(part[0], lo, o[tt]);
        o[tt] = mfma16(part[0], hi, o[tt]);
        const float since = gate.since[16 * tt + row];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[tt][i] = p.scale * fmaf(since, qs[tt][i], o[tt][i]);
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const f32x4 left = *(const f32x4*)(gate.left + 16 * tt + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[4 * tt + i] *= left[i];
      }
      split8<3>(y, part);
      most = most_of(most, part[0]);
      const float whole = gate.since[kChunk - 1];
#pragma unroll
      for (int t0 = 0; t0 < ST; t0 += 2) {
        b8 kk[2][NP];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            const char* const at_k = k_here + e * kTile + toff[t0 + t];
            kk[t][e] = join8<bf16>(read_transposed(at_k), read_transposed(at_k + kNext));
          }
        if (NP == 2) {
#pragma unroll
          for (int e = 1; e >= 0; --e)
#pragma unroll
            for (int t = 0; t < 2; ++t) fresh[t0 + t] = mfma16(kk[t][NP - 1], part[e], fresh[t0 + t]);
        }
#pragma unroll
        for (int e = 2; e >= 0; --e)
#pragma unroll
          for (int t = 0; t < 2; ++t) fresh[t0 + t] = mfma16(kk[t][0], part[e], fresh[t0 + t]);
      }

      // Something is not finite, or not as bf16: the recurrence says where it goes, token by token.
      if (__any(std::max(most[0], most[1]) >= 0x7f80)) {
        const int here_n = min(kChunk, n - c * kChunk);
        for (int j = 0; j < here_n; ++j) {
          const float decay = gate.decay[j], beta = gate.beta[j];
          float kt[ST][4], a = 0.0f, e = 0.0f;
          auto value = [&](const char* tile, int t, int i) {
            const int at_value = slot<CH>(j, 2 * t + (g >> 1)) + (g & 1) * 8 + 2 * i;
            float y = (float)*(const bf16*)(tile + at_value);
            if (NP == 2) y += (float)*(const bf16*)(tile + kTile + at_value);
            return y;
          };
#pragma unroll
          for (int t = 0; t < ST; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              kt[t][i] = value(k_here, t, i);
              if (16 * t + 4 * g + i < p.key_dim) a = fmaf(kt[t][i], s[t][i], a);
            }
          a += __shfl_xor(a, 16);
          a += __shfl_xor(a, 32);
          const float v = (float)*(const T*)(here + kV + slot<8>(j, 2 * wave + (row >> 3)) + (row & 7) * 2);
          const float uj = beta * (v - decay * a);
#pragma unroll
          for (int t = 0; t < ST; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (16 * t + 4 * g + i >= p.key_dim) continue;
              s[t][i] = fmaf(kt[t][i], uj, decay * s[t][i]);
              e = fmaf(value(here + kQ, t, i), s[t][i], e);
            }
          e += __shfl_xor(e, 16);
          e += __shfl_xor(e, 32);
          if (g == 0 && there) out[(int64_t)(c * kChunk + j) * p.out.token + row] = (T)(p.scale * e);
        }
        __syncthreads();
        continue;
      }

#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int token = c * kChunk + 16 * tt + row;
        if (token < n && stored) *(x4*)(out + (int64_t)token * p.out.token + 4 * g) = round4<T>(o[tt]);
      }
#pragma unroll
      for (int t = 0; t < ST; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][i] = fmaf(whole, s[t][i], fresh[t][i]);
      __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < ST; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = 16 * t + 4 * g + i;
        if (there && k < p.key_dim) p.state_out[state0 + (int64_t)k * p.value_dim] = s[t][i];
      }
    if (stored)
      for (int64_t t = n + row; t < p.tokens; t += 16) *(x4*)(out + t * p.out.token + 4 * g) = x4{};
    return;
  }

  if (role == 4) {   // values of chunk c + 1, gates of chunk c + 3
    const T* const v = at<T>(p.v, b, 0, h) + column0;
    const float* const log_decay = gate_at(p.log_decay, b, h);
    const float* const beta = gate_at(p.beta, b, h);
    s16x8 reg[4];
    float l = 0.0f, be = 0.0f;
    auto fetch_values = [&](int c) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at_row = e * 8 + (lane >> 3), ch = lane & 7;
        const int64_t t = (int64_t)c * kChunk + at_row;
        reg[e] = s16x8{};
        if (t < n && ch < 2 * grid.waves && column0 + 8 * ch < p.value_dim) reg[e] = load16(v + t * p.v.token + 8 * ch);
      }
    };
    auto fetch_gates = [&](int c) {
      const int64_t t = (int64_t)c * kChunk + (lane & 31);
      l = 0.0f;
      be = 0.0f;
      if (t < n) {
        if (log_decay) l = log_decay[t * p.log_decay.token];
        be = beta ? beta[t * p.beta.token] : 1.0f;
      }
    };
    fetch_gates(0);
    for (int c = -3; c < chunks; ++c) {
      if (c + 3 < chunks) {
        ChunkGates& gate = gates[(c + 3) % 4];
        // A decay of zero is 2^-10000 here: nothing of it is left in 32 bits, and no infinity enters the sums.
        double upto = (double)l * 1.4426950408889634074;
        if (upto < -1e4) upto = -1e4;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const double before = __shfl_up(upto, d, 32);
          if ((lane & 31) >= d) upto += before;
        }
        const double end = __shfl(upto, 31, 32);
        const float hi = (float)upto;
        if (lane < 32) {
          gate.upto_hi[lane] = hi;
          gate.upto_lo[lane] = (float)(upto - (double)hi);
          gate.since[lane] = __builtin_amdgcn_exp2f(hi);
          gate.left[lane] = __builtin_amdgcn_exp2f((float)(end - upto));
          gate.beta[lane] = be;
          gate.decay[lane] = expf(l);
        }
        fetch_gates(c + 4);
      }
      if (c + 1 >= 0 && c + 1 < chunks) {
        char* const next = lds + ((c + 1) & 1) * kBuffer + kV;
#pragma unroll
        for (int e = 0; e < 4; ++e) *(s16x8*)(next + slot<8>(e * 8 + (lane >> 3), lane & 7)) = reg[e];
      }
      if (c + 2 >= 0 && c + 2 < chunks) fetch_values(c + 2);
      __syncthreads();
    }
    return;
  }

  // A of chunk c + 2, and its keys in LDS (role 1); M of chunk c + 1 (role 2); P of chunk c + 1, and its queries in LDS (role 3)
  const T* const key = at<T>(p.k, b, 0, hk);
  const T* const query = at<T>(p.q, b, 0, hk);
  x8 kk[2][KS], qq[2][KS];
  // Whether a lane's last 8 dimensions are there; the others are where key_dim is more than 32 * (KS - 1), as most often it is.
  const bool in_dim = 32 * (KS - 1) + 8 * g < p.key_dim, others = p.key_dim > 32 * (KS - 1);
  auto fetch_rows = [&](const T* from, int64_t stride, int c, x8 (&to)[2][KS]) {
    const T* const first = from + ((int64_t)c * kChunk + row) * stride + 8 * g;
    const T* const at_row[2] = {first, first + 16 * stride};
    if (others && c * kChunk + kChunk <= n) {        // (the same for the whole workgroup)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int k = 0; k < KS - 1; ++k) to[tt][k] = __builtin_bit_cast(x8, load16(at_row[tt] + 32 * k));
      to[0][KS - 1] = to[1][KS - 1] = x8{};
      if (in_dim)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) to[tt][KS - 1] = __builtin_bit_cast(x8, load16(at_row[tt] + 32 * (KS - 1)));
      return;
    }
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        to[tt][k] = x8{};
        if (c * kChunk + 16 * tt + row < n && 32 * k + 8 * g < p.key_dim) to[tt][k] = __builtin_bit_cast(x8, load16(at_row[tt] + 32 * k));
      }
  };
  auto lay_out = [&](const x8 (&from)[2][KS], char* to) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        char* const at_row = to + slot<CH>(16 * tt + row, 4 * k + g);
        if (NP == 1) {
          *(s16x8*)at_row = __builtin_bit_cast(s16x8, from[tt][k]);
        } else {
          float x[8];
          b8 part[2];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = (float)from[tt][k][i];
          split8<2>(x, part);
          *(s16x8*)at_row = __builtin_bit_cast(s16x8, part[0]);
          *(s16x8*)(at_row + kTile) = __builtin_bit_cast(s16x8, part[1]);
        }
      }
  };
  // Gamma_ij of token i = 16 it + row and tokens j = 16 jt + 4 g + 0 .. 3
  auto gamma = [&](const ChunkGates& gate, int it, int jt) {
    const float hi = gate.upto_hi[16 * it + row], lo = gate.upto_lo[16 * it + row];
    const f32x4 hj = *(const f32x4*)(gate.upto_hi + 16 * jt + 4 * g), lj = *(const f32x4*)(gate.upto_lo + 16 * jt + 4 * g);
    f32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_exp2f((hi - hj[i]) + (lo - lj[i]));
    return y;
  };
  if (role == 1) {
    if (chunks > 0) fetch_rows(key, p.k.token, 0, kk);
    __syncthreads();
    for (int c = -2; c < chunks; ++c) {
      if (c + 2 < chunks) {
        const ChunkGates& gate = gates[(c + 2) % 4];
        float* const m = ms[(c + 2) % 3];
        lay_out(kk, keys[(c + 2) % 3]);
#pragma unroll
        for (int tile = 0; tile < 3; ++tile) {       // (it, jt) = (0, 0), (1, 0), (1, 1)
          const int it = tile > 0, jt = tile > 1;
          f32x4 d = {0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < KS; ++k) d = mfma16(kk[jt][k], kk[it][k], d);
          const f32x4 w = gamma(gate, it, jt);
          const float beta = gate.beta[16 * it + row];
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = it == jt && 4 * g + i >= row ? 0.0f : beta * w[i] * d[i];
          *(f32x4*)(m + (16 * it + row) * kMPitch + 16 * jt + 4 * g) = d;
        }
        if (c + 3 < chunks) fetch_rows(key, p.k.token, c + 3, kk);
      }
      __syncthreads();
    }
    return;
  }
  if (role == 2) {
    __syncthreads();
    __syncthreads();
    for (int c = -1; c < chunks; ++c) {
      if (c + 1 < chunks) {
        const ChunkGates& gate = gates[(c + 1) % 4];
        float* const m = ms[(c + 1) % 3];
        // the inverses of the diagonal blocks, a column per lane: lanes 0 .. 15 of the first, 16 .. 31 of the second
        float* const diagonal = m + (lane >> 4 & 1) * (16 * kMPitch + 16);
        const float beta = gate.beta[lane & 31];
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float y = i == row ? 1.0f : 0.0f;
#pragma unroll
          for (int j = 0; j < i; j += 4) {
            const f32x4 a = *(const f32x4*)(diagonal + i * kMPitch + j);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (j + e < i) y = fmaf(-a[e], x[j + e], y);
          }
          x[i] = y;
        }
        wave_order();
        // the first with beta, the second as it is, until the block below the first is formed: -T22 A21 T11
        if (lane < 32)
#pragma unroll
          for (int i = 0; i < 16; ++i) diagonal[i * kMPitch + row] = lane < 16 ? x[i] * beta : x[i];
        wave_order();
        const f32x4 a21 = *(const f32x4*)(m + (16 + row) * kMPitch + 4 * g), t22 = *(const f32x4*)(m + (16 + row) * kMPitch + 16 + 4 * g);
        f32x4 w = {0, 0, 0, 0}, y = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) w = __builtin_amdgcn_mfma_f32_16x16x4f32(a21[i], m[(4 * g + i) * kMPitch + row], w, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) y = __builtin_amdgcn_mfma_f32_16x16x4f32(t22[i], w[i], y, 0, 0, 0);
        wave_order();
#pragma unroll
        for (int i = 0; i < 4; ++i) m[(16 + 4 * g + i) * kMPitch + row] = -y[i];
        if (lane >= 16 && lane < 32)
#pragma unroll
          for (int i = 0; i < 16; ++i) diagonal[i * kMPitch + row] = x[i] * beta;
      }
      __syncthreads();
    }
    return;
  }
  if (chunks > 0) {
    fetch_rows(key, p.k.token, 0, kk);
    fetch_rows(query, p.q.token, 0, qq);
  }
  __syncthreads();
  __syncthreads();
  for (int c = -1; c < chunks; ++c) {
    if (c + 1 < chunks) {
      char* const next = lds + ((c + 1) & 1) * kBuffer;
      const ChunkGates& gate = gates[(c + 1) % 4];
      lay_out(qq, next + kQ);
#pragma unroll
      for (int tile = 0; tile < 4; ++tile) {         // (it, jt) = (0, 0), (0, 1): nothing, (1, 0), (1, 1)
        const int it = tile >> 1, jt = tile & 1;
        f32x4 d = {0, 0, 0, 0};
        if (tile != 1) {
#pragma unroll
          for (int k = 0; k < KS; ++k) d = mfma16(kk[jt][k], qq[it][k], d);
          const f32x4 w = gamma(gate, it, jt);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = it == jt && 4 * g + i > row ? 0.0f : w[i] * d[i];
        }
        char* const to = next + kP + (16 * it + row) * kPPitch + 16 * g + 8 * jt;
        const Vec<bf16>::x4 hi = round4<bf16>(d);
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] -= (float)hi[i];
        *(Vec<bf16>::x4*)to = hi;
        *(Vec<bf16>::x4*)(to + kChunk * kPPitch) = round4<bf16>(d);
      }
      if (c + 2 < chunks) {
        fetch_rows(key, p.k.token, c + 2, kk);
        fetch_rows(query, p.q.token, c + 2, qq);
      }
    }
    __syncthreads();
  }
}

namespace {
DeltaGrid grid_of(const DeltaParams& p) {
  const int columns = (p.value_dim + 15) / 16;
  DeltaGrid grid;
  // As many of the state's waves in a workgroup as leave a workgroup for every CU, since all of them wait for the waves that prepare its chunks:
  // 2048 tokens of 128 heads of 128 x 128 (8 sequences of 16) in four waves 170 us, in two 295, in one 552; of 64 of 64 x 64 in four 109, in one 99.
  grid.waves = std::min(kStateWaves, columns);
  while (grid.waves > 1 && (int64_t)p.batch * p.heads * ((columns + grid.waves - 1) / grid.waves) < 256) --grid.waves;
  grid.blocks = (columns + grid.waves - 1) / grid.waves;
  grid.waves = (columns + grid.blocks - 1) / grid.blocks;
  return grid;
}
template <class T>
const void* steps_of(const DeltaParams& p) {
  return p.key_dim <= 64 ? (const void*)k_delta_steps<T, 4> : (const void*)k_delta_steps<T, 8>;
}
template <class T>
const void* chunks_of(const DeltaParams& p) {
  return p.key_dim <= 64 ? (const void*)k_delta_chunks<T, 64> : p.key_dim <= 96 ? (const void*)k_delta_chunks<T, 96> : (const void*)k_delta_chunks<T, 128>;
}
}  // namespace

size_t delta_workspace(const DeltaParams&) { return 0; }

hipError_t launch(const DeltaParams& p, hipStream_t stream) {
  DeltaParams params = p;
  DeltaGrid grid = grid_of(p);
  void* args[] = {&params, &grid};
  // A chunk costs what it costs however few its tokens are, a token by itself more the fuller the device is.  Token by token and in chunks:
  // 12 and 8.5 us for 12 tokens of 8 tracks (8 heads of 64 x 64), 28 and 25 for 16 of 40 (8 of 96 x 80), 22 and 25 for 12; 166 and 161 for 24
  // of 128 (16 of 128 x 128), 124 and 149 for 16.
  const int64_t chunked = (int64_t)p.batch * p.heads * grid.blocks;
  if (p.tokens > (chunked <= 256 ? 8 : chunked <= 1024 ? 13 : 22))
    return launch_kernel(p.dtype == HS_F16 ? chunks_of<f16>(p) : chunks_of<bf16>(p), chunked, 64 * (grid.waves + kOtherWaves), args, stream);
  const int64_t workgroups = (int64_t)p.batch * p.heads * ((p.value_dim + 63) / 64);
  return launch_kernel(p.dtype == HS_F16 ? steps_of<f16>(p) : steps_of<bf16>(p), workgroups, 256, args, stream);
}

}  // namespace hs
