// hs_retention: linear attention with a decay for each head.
#include "hs_track_device.h"

#include <algorithm>

namespace hs {

// Recurrent form: S = decay * S + k v^T, out = scale * q S, token by token.  A workgroup holds key_dim x 64 values of
// one sequence's and head's state in registers: 16 lanes side by side have 4 values of 16 bytes each, so a row of
// the state is read in 256-byte pieces, and thread group g of 16 has ROWS rows from ROWS * g on.  Bound by reading and
// writing the state (5.2 TB/s at 128 tracks of 16 heads of 128 x 128); for few tracks by the chain of loads, so the first token's
// are issued beside the state's and the length's, and each further token's beside the sums of the one before.
template <class T, int ROWS>
__global__ __launch_bounds__(256) void k_retain_steps(RetentionParams p) {
  typedef typename Vec<T>::x4 x4;
  typedef T xr __attribute__((ext_vector_type(ROWS)));
  __shared__ f32x4 partial[2][4][16];
  const int blocks = (p.value_dim + 63) / 64;
  const int block = blockIdx.x % blocks;
  const int bh = blockIdx.x / blocks, h = bh % p.q_heads, hk = h / p.group, b = bh / p.q_heads;
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int dv0 = 64 * block + 4 * c, dk0 = ROWS * g;
  const bool in_v = dv0 < p.value_dim, in_k = dk0 < p.key_dim, there = in_v && in_k;
  const int64_t state0 = ((int64_t)bh * p.key_dim + dk0) * p.value_dim + dv0;
  const T* const q = at<T>(p.q, b, 0, h) + dk0;
  const T* const k = at<T>(p.k, b, 0, hk) + dk0;
  const T* const v = at<T>(p.v, b, 0, hk) + dv0;

  f32x4 S[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    S[r] = f32x4{0, 0, 0, 0};
    if (p.state_in && there) S[r] = *(const f32x4*)(p.state_in + state0 + (int64_t)r * p.value_dim);
  }
  xr qq = {}, kk = {};
  x4 vv = {};
  auto fetch = [&](int64_t t) {                     // (also of a token behind the sequence's end: then not used)
    if (in_k) {
      qq = *(const xr*)(q + t * p.q.token);
      kk = *(const xr*)(k + t * p.k.token);
    }
    if (in_v) vv = *(const x4*)(v + t * p.v.token);
  };
  if (p.tokens > 0) fetch(0);
  const int n = length_of(p.lengths, b, p.tokens);
  // (an fp32 decay near one is 2^-25 off, which 7200 steps raise to 2e-4 of the state)
  const float decay = p.decay[h], rest = p.decay_rest[h];
  for (int t = 0; t < n; ++t) {
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        S[r][i] = fmaf(decay, S[r][i], fmaf(rest, S[r][i], (float)kk[r] * (float)vv[i]));
        o[i] = fmaf((float)qq[r], S[r][i], o[i]);
      }
    if (t + 1 < n) fetch(t + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] += __shfl_xor(o[i], 16);
      o[i] += __shfl_xor(o[i], 32);
    }
    if ((threadIdx.x & 63) < 16) partial[t & 1][wave][c] = o;
    __syncthreads();   // the other half of `partial` is written before the next one
    if (threadIdx.x < 16 && in_v)
      *(x4*)(at_out<T>(p.out, b, t, h) + dv0) = round4<T>(p.scale * ((partial[t & 1][0][c] + partial[t & 1][1][c]) + (partial[t & 1][2][c] + partial[t & 1][3][c])));
  }
  if (in_v)
    for (int t = n + g; t < p.tokens; t += 16) *(x4*)(at_out<T>(p.out, b, t, h) + dv0) = x4{};
  if (there && !(n == 0 && p.state_out == p.state_in))
#pragma unroll
    for (int r = 0; r < ROWS; ++r) *(f32x4*)(p.state_out + state0 + (int64_t)r * p.value_dim) = S[r];
}

// Chunked form: 64 tokens at a time, products on the matrix pipe.  With c tokens in a chunk, S the state before it and
// i, j = 0 .. c - 1:
//   A_ij = scale * decay^(i - j) q_i k_j (j <= i)          out_i = sum_j A_ij v_j + scale * decay^(i + 1) S^T q_i
//   S   <- decay^c S + sum_j k_j (decay^(c - 1 - j) v_j)^T
// A workgroup has one sequence and head and 64 of the values' dimensions, and waves of two kinds, one of each per SIMD:
//   waves 0 .. 3 carry the state, 16 of the dimensions each, in their accumulators, and leave a 16-bit copy of it in LDS
//   for the next chunk;
//   waves 4 .. 7 form out, 16 of the chunk's rows each: A by K Q^T, so that a lane holds four keys of one row per tile
//   and A is the operand of the next product where it lies, if that one takes V's rows in the same order.
// While a chunk is worked on the next one goes from registers into the other half of LDS and the one behind it is on
// its way from memory; one barrier a chunk.
//
// Rounded to 16 bits, as the matrix pipe takes them: A, and the copy of S that multiplies q (each term of out
// is then half a step off, as out itself); of the fp16 copy a power of two is taken out, so that it stays in
// that type's range whatever the state has grown to.  The state takes no such rounding: decayed values enter as a sum of
// three bf16 or two fp16 parts (the second scaled by 2^12, out of fp16's subnormal numbers).
constexpr int kChunk = 64;

// Few sequences and heads: their chunks are cut into segments, a workgroup for each.  A first launch (kStates) finds what
// every segment but the last adds to a state of zeros, a second one (k_retain_starts) puts together by the decays of whole
// segments what each starts from, and the third goes on from there as above.
template <class T, int KP, bool kStates>
__global__ __launch_bounds__(512) void k_retain_chunks(RetentionParams p, int segments) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int CH = KP / 8, KT = KP / 16, KS = KP / 32;   // KT: 16-wide tiles of key dimensions, KS: steps of 32
  constexpr int RP = 512 / CH, NL = kChunk / RP;    // rows per pass of the workgroup over Q or K, passes
  constexpr bool kHalf = __is_same(T, f16);
  constexpr int kK = kChunk * KP * 2, kV = 2 * kK, kSlot = kV + kChunk * 64 * 2;   // Q, K and V of a chunk
  constexpr int kS = 2 * kSlot, kCopy = 64 * KP * 2;
  __shared__ __align__(16) char lds[kS + 2 * kCopy];
  __shared__ int exponents[2][4];
  __shared__ double power[kChunk + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w4 = wave & 3, l16 = lane & 15, g = lane >> 4;
  const int blocks = (p.value_dim + 63) / 64;
  int id = xcd_number();
  const int block = id % blocks;
  id /= blocks;
  const int parts = kStates ? segments - 1 : segments, segment = id % parts, bh = id / parts;
  const int h = bh % p.q_heads, hk = h / p.group, b = bh / p.q_heads;
  const int n = length_of(p.lengths, b, p.tokens), all_chunks = (int)(((int64_t)n + kChunk - 1) / kChunk);
  const int per_segment = (all_chunks + segments - 1) / segments;
  const int first = min(segment * per_segment, all_chunks), chunks = min(per_segment, all_chunks - first);
  const bool last = segment == (all_chunks ? (all_chunks - 1) / per_segment : 0);   // the one with the end
  if (kStates ? !chunks || last : !chunks && !last) return;

  // staging: this thread's 16-byte piece of rows r0, r0 + RP, ... of Q and K, and of a row of V (8 pieces).  Rows behind the
  // last token are read as that one and emptied on their way into LDS.
  const int r0 = threadIdx.x / CH, ch = threadIdx.x % CH, vr = threadIdx.x / 8, vch = threadIdx.x % 8;
  const bool in_k = 8 * ch < p.key_dim, in_v = 64 * block + 8 * vch < p.value_dim;
  const T *qsrc[NL], *ksrc[NL], *vsrc;              // of the chunk that is fetched next
#pragma unroll
  for (int e = 0; e < NL; ++e) {
    const int64_t t = (int64_t)first * kChunk + r0 + e * RP;
    qsrc[e] = at<T>(p.q, b, t, h) + 8 * ch;
    ksrc[e] = at<T>(p.k, b, t, hk) + 8 * ch;
  }
  vsrc = at<T>(p.v, b, (int64_t)first * kChunk + vr, hk) + 64 * block + 8 * vch;
  s16x8 qreg[NL] = {}, kreg[NL] = {}, vreg = {};
  auto left_of = [&](int c) { return (int)min((int64_t)n - (int64_t)(first + c) * kChunk, (int64_t)kChunk); };   // tokens of chunk c
  auto fetch = [&](int c) {                         // chunk c, after the ones before it
    if (c >= chunks) return;
    const int left = left_of(c);
    if (left < kChunk) {
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        const int64_t behind = max(r0 + e * RP - (left - 1), 0);
        qsrc[e] -= behind * p.q.token;
        ksrc[e] -= behind * p.k.token;
      }
      vsrc -= (int64_t)max(vr - (left - 1), 0) * p.v.token;
    }
    if (in_k) {
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        if (!kStates) qreg[e] = *(const s16x8*)qsrc[e];
        kreg[e] = *(const s16x8*)ksrc[e];
      }
    }
    if (in_v) vreg = *(const s16x8*)vsrc;
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      qsrc[e] += kChunk * p.q.token;
      ksrc[e] += kChunk * p.k.token;
    }
    vsrc += kChunk * p.v.token;
  };
  auto store = [&](int c, char* to) {
    const int left = left_of(c);
    if (left < kChunk) {
#pragma unroll
      for (int e = 0; e < NL; ++e)
        if (r0 + e * RP >= left) qreg[e] = kreg[e] = s16x8{};
      if (vr >= left) vreg = s16x8{};
    }
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      if (!kStates) *(s16x8*)(to + slot<CH>(r0 + e * RP, ch)) = qreg[e];
      *(s16x8*)(to + kK + slot<CH>(r0 + e * RP, ch)) = kreg[e];
    }
    *(s16x8*)(to + kV + slot<8>(vr, vch)) = vreg;
  };
  if (chunks) fetch(0);
  if (threadIdx.x >= 384 && threadIdx.x <= 384 + kChunk) power[threadIdx.x - 384] = exp2(p.log2_decay[h] * (threadIdx.x - 384));

  if (wave < 4) {
    // ---- the state: lane has dimension dv, key dimensions 16 t + 4 g + i
    const int dv = 64 * block + 16 * w4 + l16;
    const int64_t state0 = (int64_t)bh * p.key_dim * p.value_dim + dv;
    const int64_t states = (int64_t)p.batch * p.q_heads * p.key_dim * p.value_dim;
    const float* const from = kStates ? nullptr : segment ? p.parts + (segment - 1) * states : p.state_in;
    f32x4 S[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int dk = 16 * t + 4 * g + i;
        S[t][i] = from && dv < p.value_dim && dk < p.key_dim ? from[state0 + (int64_t)dk * p.value_dim] : 0.0f;
      }
    if (chunks) {
      store(0, lds);
      fetch(1);
    }
    // the state's 16-bit copy, [dimension][key dimension]
    auto leave_copy = [&](int to) {
      int exponent = 0;
      if (kHalf) {
        float most = 0.0f;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(S[t][i]));
        most = wave_max(most);
        if (most == INFINITY) {                     // (the finite values keep theirs)
          most = 0.0f;
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(S[t][i]) < INFINITY ? fabsf(S[t][i]) : 0.0f);
          most = wave_max(most);
        }
        exponent = max(min(__builtin_amdgcn_frexp_expf(most) - 12, 100), -100);
        if (lane == 0) exponents[to][w4] = exponent;
      }
      const float small = ldexpf(1.0f, -exponent);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        *(x4*)(lds + kS + to * kCopy + slot<CH>(16 * w4 + l16, 2 * t + (g >> 1)) + (g & 1) * 8) = round4<T>(kHalf ? S[t] * small : S[t]);
      }
    };
    if (!kStates) leave_copy(0);
    __syncthreads();
    float weight[2][8];                             // decays of v_j in S
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) weight[s][i] = (float)power[kChunk - 1 - (32 * s + 8 * g + i)];
    // A chunk's decay in fp32; what that drops is carried to the next one, so that many chunks' decay is as exact.
    const float keep = (float)power[kChunk], keep_rest = (float)(power[kChunk] - (double)keep);
    float carried = 0.0f;

    for (int c = 0; c < chunks; ++c) {
      char* const here = lds + (c & 1) * kSlot;
      if (c + 1 < chunks) {
        store(c + 1, lds + (~c & 1) * kSlot);
        fetch(c + 2);
      }
      carried += keep_rest;
      float now = keep + carried;
      carried -= now - keep;
      const int left = left_of(c);
      if (left < kChunk) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 8; ++i) weight[s][i] = (float)power[max(left - 1 - (32 * s + 8 * g + i), 0)];   // (later values are zeros)
        now = (float)power[left];
      }
      x8 part[2][3];                                // decayed values: dimension 16 w4 + l16, tokens 32 s + 8 g + i
      const int r = 8 * g + (lane >> 2 & 3), low8 = (lane & 1) * 8;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const char* const from = here + kV + 32 * s * 128 + low8;
        const int cc = 2 * w4 + (lane >> 1 & 1);
        const x8 v = join8<T>(read_transposed(from + slot<8>(r, cc)), read_transposed(from + slot<8>(r + 4, cc)));
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = (float)v[i] * weight[s][i];
          asm("" : "+v"(x[i]));   // the rounded product: rounded to 16 bits from the exact one in one place and from this in another, a
                                  // part and what is left of it would not belong together
        }
        part[s][0] = round8<T>(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] -= (float)part[s][0][i];
          if (kHalf) x[i] *= 4096.0f;
        }
        part[s][1] = round8<T>(x);
        if (!kHalf) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] -= (float)part[s][1][i];
          part[s][2] = round8<T>(x);
        }
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) S[t][i] *= now;
        f32x4 low = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const char* const from = here + kK + 32 * s * CH * 16 + low8;
          const int cc = 2 * t + (lane >> 1 & 1);
          const x8 k = join8<T>(read_transposed(from + slot<CH>(r, cc)), read_transposed(from + slot<CH>(r + 4, cc)));
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
      if (!kStates && c + 1 < chunks) leave_copy(~c & 1);
      __syncthreads();
    }
    float* to = p.state_out + state0;
    if (kStates) to = p.parts + segment * states + state0;
    else if (!last) return;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int dk = 16 * t + 4 * g + i;
        if (dv < p.value_dim && dk < p.key_dim) to[(int64_t)dk * p.value_dim] = S[t][i];
      }
  } else {
    // ---- out: rows 16 w4 .. + 15 of the chunk, lane has row 16 w4 + l16
    if (chunks) {
      store(0, lds);
      fetch(1);
    }
    __syncthreads();
    float decay[4][4];                              // of A's tiles: keys 16 cb + 4 g + i
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int apart = 16 * (w4 - cb) + l16 - 4 * g - i;
        decay[cb][i] = apart < 0 ? 0.0f : p.scale * (float)power[max(apart, 0)];
      }
    const float after = p.scale * (float)power[16 * w4 + l16 + 1];
    const int vrow = 4 * g + (lane >> 2 & 3), low8 = (lane & 1) * 8;
    for (int c = 0; c < chunks; ++c) {
      const char* const here = lds + (c & 1) * kSlot;
      const char* const copy = lds + kS + (c & 1) * kCopy;
      if (c + 1 < chunks) {
        store(c + 1, lds + (~c & 1) * kSlot);
        fetch(c + 2);
      }
      if (kStates) {
        __syncthreads();
        continue;
      }
      x8 q[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) q[s] = *(const x8*)(here + 16 * w4 * CH * 16 + slot<CH>(l16, 4 * s + g));
      f32x4 o[4];
      auto from_state = [&](int d) {
        o[d] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) o[d] = mfma16(*(const x8*)(copy + 16 * d * CH * 16 + slot<CH>(l16, 4 * s + g)), q[s], o[d]);
        o[d] *= kHalf ? ldexpf(after, exponents[c & 1][d]) : after;
      };
      auto scores = [&](int cb) {
        f32x4 t = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) t = mfma16(*(const x8*)(here + kK + 16 * cb * CH * 16 + slot<CH>(l16, 4 * s + g)), q[s], t);
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] *= decay[cb][i];
        return t;
      };
#pragma unroll
      for (int d = 0; d < 4; ++d) from_state(d);
#pragma unroll
      for (int j = 0; j < 2; ++j) {                 // 32 keys
        if (2 * j > w4) break;
        x8 a = {};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int cb = 2 * j + e;
          if (cb > w4) break;
          const f32x4 t = scores(cb);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[4 * e + i] = (T)t[i];
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const char* const from = here + kV + 32 * j * 128 + low8;
          const int cc = 2 * d + (lane >> 1 & 1);
          o[d] = mfma16(join8<T>(read_transposed(from + slot<8>(vrow, cc)), read_transposed(from + 16 * 128 + slot<8>(vrow, cc))), a, o[d]);
        }
      }
      float finite = 0.0f;                          // zero, or NaN
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) finite = fmaf(o[d][i], 0.0f, finite);
      if (__any(finite != 0.0f)) {
        // A product beyond fp16's range, or an input that is not finite, which must not reach earlier tokens through their zeros
        // in A: term by term, in fp32.
#pragma unroll
        for (int d = 0; d < 4; ++d) from_state(d);
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          if (cb > w4) break;
          const f32x4 t = scores(cb);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll 1
            for (int from = 0; from < 4; ++from) {
              const int key = 16 * cb + 4 * from + i;
              const float a = __shfl(t[i], 16 * from + l16);
              if (key > 16 * w4 + l16) continue;
#pragma unroll
              for (int d = 0; d < 4; ++d) {
                const x4 v = *(const x4*)(here + kV + slot<8>(key, 2 * d + (g >> 1)) + (g & 1) * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][e] = fmaf(a, (float)v[e], o[d][e]);
              }
            }
        }
      }
      const int64_t t = (int64_t)(first + c) * kChunk + 16 * w4 + l16;
      if (t < n) {
        T* const to = at_out<T>(p.out, b, t, h) + 64 * block + 4 * g;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          if (64 * block + 16 * d + 4 * g < p.value_dim) *(x4*)(to + 16 * d) = round4<T>(o[d]);
        }
      }
      __syncthreads();
    }
    if (last && in_v)
      for (int64_t t = (int64_t)n + vr - 32; t < p.tokens; t += 32) *(s16x8*)(at_out<T>(p.out, b, t, h) + 64 * block + 8 * vch) = s16x8{};
  }
}

// parts[s], s < segments - 1: what segment s adds, replaced by the state behind it.  Four values per thread.
__global__ __launch_bounds__(256) void k_retain_starts(RetentionParams p, int segments) {
  const int64_t size = (int64_t)p.key_dim * p.value_dim, states = (int64_t)p.batch * p.q_heads * size;
  const int64_t at_value = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (at_value >= states) return;
  const int64_t bh = at_value / size, b = bh / p.q_heads;
  const int n = p.lengths ? min(max(p.lengths[b], 0), p.tokens) : p.tokens, chunks = (int)(((int64_t)n + kChunk - 1) / kChunk), per_segment = (chunks + segments - 1) / segments;
  const int used = per_segment ? (chunks - 1) / per_segment : 0;   // segments before the sequence's last one
  const double far = exp2(p.log2_decay[bh % p.q_heads] * ((double)per_segment * kChunk));
  const float keep = (float)far, keep_rest = (float)(far - (double)keep);
  f32x4 S = {0, 0, 0, 0};
  if (p.state_in) S = *(const f32x4*)(p.state_in + at_value);
  float* part = p.parts + at_value;
#pragma unroll 4
  for (int s = 0; s < used; ++s, part += states) {
    const f32x4 add = *(const f32x4*)part;
#pragma unroll
    for (int i = 0; i < 4; ++i) S[i] = fmaf(S[i], keep, fmaf(S[i], keep_rest, add[i]));
    *(f32x4*)part = S;
  }
}

namespace {
struct RetentionPlan {
  bool steps;
  int segments;
  int64_t workgroups;            // of one segment
};
RetentionPlan plan_of(const RetentionParams& p) {
  RetentionPlan plan;
  plan.workgroups = (int64_t)p.batch * p.q_heads * ((p.value_dim + 63) / 64);
  plan.steps = p.tokens <= 8;
  plan.segments = 1;
  if (!plan.steps) {
    const int64_t chunks = ((int64_t)p.tokens + kChunk - 1) / kChunk;
    if (chunks >= 16) plan.segments = (int)std::max<int64_t>(1, std::min<int64_t>({256 / std::max<int64_t>(plan.workgroups, 1), chunks / 3, 32}));
  }
  return plan;
}

template <class T>
const void* chunks_kernel(bool wide, bool states) {
  return wide ? states ? (const void*)k_retain_chunks<T, 128, true> : (const void*)k_retain_chunks<T, 128, false>
              : states ? (const void*)k_retain_chunks<T, 64, true> : (const void*)k_retain_chunks<T, 64, false>;
}
}  // namespace

size_t retention_workspace(const RetentionParams& p) {
  const RetentionPlan plan = plan_of(p);
  return (size_t)(plan.segments - 1) * p.batch * p.q_heads * p.key_dim * p.value_dim * sizeof(float);
}

hipError_t launch(const RetentionParams& p, hipStream_t stream) {
  RetentionParams params = p;
  RetentionPlan plan = plan_of(p);
  const bool wide = p.key_dim > 64, half = p.dtype == HS_F16;
  void* args[] = {&params, &plan.segments};
  if (plan.steps) {
    const void* const kernel = half ? wide ? (const void*)k_retain_steps<f16, 8> : (const void*)k_retain_steps<f16, 4>
                                    : wide ? (const void*)k_retain_steps<bf16, 8> : (const void*)k_retain_steps<bf16, 4>;
    return launch_kernel(kernel, plan.workgroups, 256, args, stream);
  }
  if (plan.segments > 1) {
    const hipError_t e = launch_kernel(half ? chunks_kernel<f16>(wide, true) : chunks_kernel<bf16>(wide, true), plan.workgroups * (plan.segments - 1), 512, args, stream);
    if (e != hipSuccess) return e;
    const hipError_t joined = launch_kernel((const void*)k_retain_starts, ((int64_t)p.batch * p.q_heads * p.key_dim * p.value_dim / 4 + 255) / 256, 256, args, stream);
    if (joined != hipSuccess) return joined;
  }
  return launch_kernel(half ? chunks_kernel<f16>(wide, false) : chunks_kernel<bf16>(wide, false), plan.workgroups * plan.segments, 512, args, stream);
}

}  // namespace hs
