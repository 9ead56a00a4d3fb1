// hs_retention: linear attention with a decay for each head.
#include "hs_track_device.h"

#include <float.h>

#include <algorithm>
#include <type_traits>

namespace hs {

// Infinities of the state stay what they are (but for a decay of zero), as the recurrence has it: a correction to their decay would make
// NaN of them, and so would a power of the decay that underflows.
__device__ __forceinline__ float finite(float x) { return __builtin_amdgcn_fmed3f(x, -FLT_MAX, FLT_MAX); }
__device__ __forceinline__ float least_power(float decay) { return decay > 0.0f ? FLT_TRUE_MIN : 0.0f; }

// Recurrent form: S = decay * S + k v^T, out = scale * q S, token by token.  A workgroup holds key_dim x 64 values of
// one sequence's and head's state in registers: 16 lanes side by side have 4 values of 16 bytes each, so a row of
// the state is read in 256-byte pieces, and thread group g of 16 has ROWS rows from ROWS * g on.  Bound by reading and
// writing the state (5.6 TB/s at 128 tracks of 16 heads of 128 x 128); for few tracks by the chain of loads, so the first token's
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
    if (!there) return;                             // (zeros: a value that is not finite is not multiplied by what is not there)
    qq = *(const xr*)(q + t * p.q.token);
    kk = *(const xr*)(k + t * p.k.token);
    vv = *(const x4*)(v + t * p.v.token);
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
        S[r][i] = fmaf(decay, S[r][i], fmaf(rest, finite(S[r][i]), (float)kk[r] * (float)vv[i]));
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
//   A_ij = decay^(i - j) q_i k_j (j <= i)                  out_i = scale * (sum_j A_ij v_j + decay^(i + 1) S^T q_i)
//   S   <- decay^c S + sum_j k_j (decay^(c - 1 - j) v_j)^T
// A workgroup has one sequence and head and 48 or 64 of the values' dimensions, and waves of three kinds, one of each per SIMD:
//   waves 0 .. 3 carry the state, 16 of the dimensions each, in their accumulators, and leave a 16-bit copy of it in LDS
//   for the next chunk;
//   waves 4 .. 7 load: a chunk that is two ahead is on its way from memory into their registers while the next one goes
//   from there into the other half of LDS, with the values' decayed parts;
//   waves 8 .. 11 form out, 16 of the chunk's rows each: A by K Q^T, so that a lane holds four keys of one row per tile
//   and A is the operand of the next product where it lies, if that one takes V's rows in the same order.
// An infinity or NaN among the tokens would reach earlier ones through their zeros in A, and has no parts.  The waves that load
// multiply everything by zero on the side; where that has given NaN, the waves that carry the state go over the tokens a second
// time, one by one, and write what the recurrence has.
// One barrier a chunk.  The chain of LDS reads and products from barrier to barrier bounds it: 10 chunks of 64 sequences and heads of
// 64 x 64 take 16.1 us (19.9 with eight waves that shared the loads), 40 ragged clips of up to 257 tokens of 8 heads of 96 x 80 24.3 to 26
// (38.7), 113 chunks of 128 x 128 in 256 workgroups 240 to 259 by device, 3.7 to 4.0 TB/s (in one trace 285, of which the loads alone
// take 168).  The waves that form out are the longest, and go first.
//
// Rounded to 16 bits, as the matrix pipe takes them: A, and the copy of S that multiplies q (each term of out
// is then half a step off, as out itself).  In fp16 a power of two is taken out of each row of A, so that its largest is below 2^15
// and those of up to 2^-28 of that keep all their bits, and one out of each column of the copy, which lies
// in the same range then whatever the state has grown to.  The state takes no such rounding: decayed values enter as a sum of
// three bf16 or two fp16 parts.  The second of these is scaled by 2^11, out of fp16's subnormal numbers and no further: what a first
// part leaves is up to 16, of values from 32768 on.  So two parts keep 22 bits of what is above 2^-14, and 2^-36 of the rest.
constexpr int kChunk = 64;

// Few sequences and heads: their chunks are cut into segments, a workgroup for each.  A first launch (kStates) finds what
// every segment but the last adds to a state of zeros, a second one (k_retain_starts) puts together by the decays of whole
// segments what each starts from, and the third goes on from there as above.
template <class T, int KP, int DT, bool kStates>
__global__ __launch_bounds__(kStates ? 512 : 768) void k_retain_chunks(RetentionParams p, int segments) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int CH = KP > 64 ? 16 : 8, KT = KP / 16, KS = KP / 32;   // CH: 16-byte pieces per row in LDS; KT: 16-wide tiles of key dimensions, KS: steps of 32
  constexpr int kWide = 16 * DT;                    // of the values' dimensions
  constexpr int RP = 256 / CH, NL = kChunk / RP, NV = 2;   // rows per pass of the waves that load over Q or K, passes over them and V
  constexpr bool kHalf = __is_same(T, f16);
  constexpr int kParts = kHalf ? 2 : 3, kVTile = kChunk * 64 * 2;
  constexpr int kK = kChunk * CH * 16, kV = 2 * kK, kP = kV + kVTile, kSlot = kP + kParts * kVTile;   // Q, K, V of a chunk, V's decayed parts
  constexpr int kS = 2 * kSlot, kCopy = kWide * CH * 16;
  __shared__ __align__(16) char lds[kS + 2 * kCopy];
  __shared__ int4 exponents[kHalf ? 2 : 1][kHalf ? kWide / 4 : 1];   // of the copies' columns
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w4 = wave & 3, l16 = lane & 15, g = lane >> 4;
  const int blocks = (p.value_dim + kWide - 1) / kWide;
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

  auto left_of = [&](int c) { return (int)min((int64_t)n - (int64_t)(first + c) * kChunk, (int64_t)kChunk); };   // tokens of chunk c
  // the decay's powers below the chunk's: a wave has one per lane
  const double power64 = exp2(p.log2_decay[h] * lane);
  const float least = least_power(p.decay[h]), power = fmaxf((float)power64, least);
  auto power_of = [&](int steps) { return __shfl(power, steps); };

  // Behind the last chunk's barrier: whether a wave that loads has met an infinity or NaN.  (Where a further chunk would have its parts.)
  int* const met = (int*)(lds + (chunks & 1) * kSlot + kP);
  auto any_met = [&]() { return (met[0] | met[1] | met[2] | met[3]) != 0; };
  auto wait_for_chunks = [&]() {
    for (int c = -1; c < chunks; ++c) __syncthreads();
  };

  if (wave < 4 && w4 >= DT) {
    wait_for_chunks();
    if (any_met()) wait_for_chunks();
  } else if (wave < 4) {
    // ---- the state: lane has dimension dv, key dimensions 16 t + 4 g + i
    const int dv = kWide * block + 16 * w4 + l16;
    const int64_t state0 = (int64_t)bh * p.key_dim * p.value_dim + dv;
    const int64_t states = (int64_t)p.batch * p.q_heads * p.key_dim * p.value_dim;
    // (the first segment's, where the last one may have written over it already: as k_retain_starts has kept it)
    const float* const from = kStates ? nullptr : segment ? p.parts + (segment - 1) * states : segments > 1 && p.state_in == p.state_out ? p.parts + (segments - 1) * states : p.state_in;
    f32x4 S[KT];
    auto begin = [&](const float* from) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int dk = 16 * t + 4 * g + i;
          S[t][i] = from && dv < p.value_dim && dk < p.key_dim ? from[state0 + (int64_t)dk * p.value_dim] : 0.0f;
        }
    };
    begin(from);
    // the state's 16-bit copy, [dimension][key dimension]
    auto leave_copy = [&](int to) {
      int exponent = 0;
      if (kHalf) {
        float most = 0.0f;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(S[t][i]));
        most = column_max(most);
        if (__any(most == INFINITY)) {              // (the finite values keep theirs)
          most = 0.0f;
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(S[t][i]) < INFINITY ? fabsf(S[t][i]) : 0.0f);
          most = column_max(most);
        }
        exponent = max(__builtin_amdgcn_frexp_expf(most) - 15, -100);
        if (g == 0) ((int*)exponents[to])[16 * w4 + l16] = exponent;
      }
      const float small = ldexpf(1.0f, -exponent);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        *(x4*)(lds + kS + to * kCopy + slot<CH>(16 * w4 + l16, 2 * t + (g >> 1)) + (g & 1) * 8) = round4<T>(kHalf ? S[t] * small : S[t]);
      }
    };
    if (!kStates) leave_copy(0);
    // A chunk's decay in fp32; what that drops is carried to the next one, so that many chunks' decay is as exact.
    const double half_chunk = __shfl(power64, kChunk / 2), whole = half_chunk * half_chunk;
    const float keep = (float)whole, keep_rest = (float)(whole - (double)keep);
    float carried = 0.0f;
    const int r = 8 * g + (lane >> 2 & 3), low8 = (lane & 1) * 8;
    __syncthreads();

    for (int c = 0; c < chunks; ++c) {
      char* const here = lds + (c & 1) * kSlot;
      carried += keep_rest;
      float now = keep + carried;
      carried -= now - keep;
      now = fmaxf(now, least);
      const int left = left_of(c);
      if (left < kChunk) now = power_of(left);
      x8 part[2][kParts];                           // decayed values: dimension 16 w4 + l16, tokens 32 s + 8 g + i
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
          const char* const from = here + kP + e * kVTile + 32 * s * 128 + low8;
          const int cc = 2 * w4 + (lane >> 1 & 1);
          part[s][e] = join8<T>(read_transposed(from + slot<8>(r, cc)), read_transposed(from + slot<8>(r + 4, cc)));
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
        if (kHalf) S[t] += low * (1.0f / 2048.0f);
        if (t % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (reads further ahead would not fit the registers)
      }
      if (!kStates && c + 1 < chunks) leave_copy(~c & 1);
      __syncthreads();
    }
    if (any_met()) {                                // token by token from the start
      const float decay = p.decay[h], rest = p.decay_rest[h];
      const float* start = from;
      asm("" : "+s"(start));                        // (its addresses are formed here, not kept through the chunks)
      begin(start);
      __syncthreads();
      for (int c = 0; c < chunks; ++c) {
        const char* const here = lds + (c & 1) * kSlot;
        const int left = left_of(c);
#pragma unroll 1
        for (int j = 0; j < left; ++j) {
          const float v = (float)*(const T*)(here + kV + slot<8>(j, 2 * w4 + (l16 >> 3)) + (l16 & 7) * 2);
          x4 k[KT], q[KT] = {};
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            const int at_k = slot<CH>(j, 2 * t + (g >> 1)) + (g & 1) * 8;
            k[t] = *(const x4*)(here + kK + at_k);
            if (!kStates) q[t] = *(const x4*)(here + at_k);
          }
          float o = 0.0f;
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            const float in = 16 * t + 4 * g < p.key_dim ? v : 0.0f;   // (behind the keys there are zeros, as the first time)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              S[t][i] = fmaf(decay, S[t][i], fmaf(rest, finite(S[t][i]), (float)k[t][i] * in));
              if (!kStates) o = fmaf((float)q[t][i], S[t][i], o);
            }
          }
          if (kStates) continue;
          o += __shfl_xor(o, 16);
          o += __shfl_xor(o, 32);
          if (g == 0 && dv < p.value_dim) at_out<T>(p.out, b, (int64_t)(first + c) * kChunk + j, h)[dv] = (T)(p.scale * o);
        }
        __syncthreads();
      }
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
  } else if (wave < 8) {
    // ---- loads: this thread's 16-byte pieces of rows r0, r0 + RP, ... of Q and K, and of two rows of V (8 pieces).  Rows behind
    // the last token are read as that one and emptied on their way into LDS.
    const int tid = threadIdx.x & 255, r0 = tid / CH, ch = tid % CH, vr = tid / 8, vch = tid % 8;
    const bool in_k = 8 * ch < p.key_dim, in_v = vch < 2 * DT && kWide * block + 8 * vch < p.value_dim;
    const T* qsrc = at<T>(p.q, b, (int64_t)first * kChunk + r0, h) + 8 * ch;   // of the chunk that is fetched next
    const T* ksrc = at<T>(p.k, b, (int64_t)first * kChunk + r0, hk) + 8 * ch;
    const T* vsrc = at<T>(p.v, b, (int64_t)first * kChunk + vr, hk) + kWide * block + 8 * vch;
    struct Pieces { s16x8 q[NL], k[NL], v[NV]; } even = {}, odd = {};          // of chunks on their way
    auto fetch = [&](int c, Pieces& to) {           // chunk c, after the ones before it
      if (c >= chunks) return;
      const int left = left_of(c);
      const T *qa[NL], *ka[NL], *va[NV];
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        qa[e] = qsrc + e * RP * p.q.token;
        ka[e] = ksrc + e * RP * p.k.token;
      }
#pragma unroll
      for (int e = 0; e < NV; ++e) va[e] = vsrc + e * 32 * p.v.token;
      if (left < kChunk) {
#pragma unroll
        for (int e = 0; e < NL; ++e) {
          const int64_t behind = max(r0 + e * RP - (left - 1), 0);
          qa[e] -= behind * p.q.token;
          ka[e] -= behind * p.k.token;
        }
#pragma unroll
        for (int e = 0; e < NV; ++e) va[e] -= (int64_t)max(vr + e * 32 - (left - 1), 0) * p.v.token;
      }
      if (in_k) {
#pragma unroll
        for (int e = 0; e < NL; ++e) {
          if (!kStates) to.q[e] = load16(qa[e]);
          to.k[e] = load16(ka[e]);
        }
      }
      if (in_v) {
#pragma unroll
        for (int e = 0; e < NV; ++e) to.v[e] = load16(va[e]);
      }
      qsrc += kChunk * p.q.token;
      ksrc += kChunk * p.k.token;
      vsrc += kChunk * p.v.token;
    };
    float weight[NV];                               // v's decay until the chunk's end
#pragma unroll
    for (int e = 0; e < NV; ++e) weight[e] = power_of(kChunk - 1 - vr - e * 32);
    f32x4 zero = {0, 0, 0, 0};                      // what is loaded, times zero (on the matrix pipe 113 chunks of 128 x 128 take
                                                    // 249 us, 243 without; on the vector pipe 10 of 64 x 64 take 4 % more)
    auto store = [&](int c, Pieces& from) {
      if (c >= chunks) return;
      char* const to = lds + (c & 1) * kSlot;
      const int left = left_of(c);
      if (left < kChunk) {
#pragma unroll
        for (int e = 0; e < NL; ++e)
          if (r0 + e * RP >= left) from.q[e] = from.k[e] = s16x8{};
#pragma unroll
        for (int e = 0; e < NV; ++e) {
          weight[e] = power_of(max(left - 1 - vr - e * 32, 0));
          if (vr + e * 32 >= left) from.v[e] = s16x8{};
        }
      }
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        if (!kStates) *(s16x8*)(to + slot<CH>(r0 + e * RP, ch)) = from.q[e];
        *(s16x8*)(to + kK + slot<CH>(r0 + e * RP, ch)) = from.k[e];
      }
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        if (!kStates) zero = mfma16(__builtin_bit_cast(x8, from.q[e]), x8{}, zero);
        zero = mfma16(__builtin_bit_cast(x8, from.k[e]), x8{}, zero);
      }
#pragma unroll
      for (int e = 0; e < NV; ++e) zero = mfma16(__builtin_bit_cast(x8, from.v[e]), x8{}, zero);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int at_v = slot<8>(vr + u * 32, vch);
        if (!kStates) *(s16x8*)(to + kV + at_v) = from.v[u];
        const x8 v = __builtin_bit_cast(x8, from.v[u]);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = (float)v[i] * weight[u];
          asm("" : "+v"(x[i]));   // the rounded product: rounded to 16 bits from the exact one in one place and from this in another,
                                  // a part and what is left of it would not belong together
        }
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
          const x8 part = round8<T>(x);
          *(x8*)(to + kP + e * kVTile + at_v) = part;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = (x[i] - (float)part[i]) * (kHalf ? 2048.0f : 1.0f);
        }
      }
    };
    auto tell = [&]() {
      const bool it = __any((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.0f);
      if (lane == 0) met[w4] = it;
    };
    fetch(0, even);
    fetch(1, odd);
    store(0, even);
    fetch(2, even);
    if (chunks == 0) tell();
    __syncthreads();
    for (int c = 0; c < chunks; c += 2) {
      store(c + 1, odd);
      fetch(c + 3, odd);
      if (c + 1 == chunks) tell();
      __syncthreads();
      if (c + 1 >= chunks) break;
      store(c + 2, even);
      fetch(c + 4, even);
      if (c + 2 == chunks) tell();
      __syncthreads();
    }
    if (any_met()) {                                // the chunks as they are, one after the other
      auto bring = [&](int c) {
        char* const to = lds + (c & 1) * kSlot;
        const int64_t t0 = (int64_t)(first + c) * kChunk;
        const int left = c < chunks ? left_of(c) : 0;
        if (in_k)
          for (int r = r0; r < left; r += RP) {
            if (!kStates) *(s16x8*)(to + slot<CH>(r, ch)) = load16(at<T>(p.q, b, t0 + r, h) + 8 * ch);
            *(s16x8*)(to + kK + slot<CH>(r, ch)) = load16(at<T>(p.k, b, t0 + r, hk) + 8 * ch);
          }
        if (in_v)
          for (int r = vr; r < left; r += 32) *(s16x8*)(to + kV + slot<8>(r, vch)) = load16(at<T>(p.v, b, t0 + r, hk) + kWide * block + 8 * vch);
      };
      bring(0);
      __syncthreads();
      for (int c = 0; c < chunks; ++c) {
        bring(c + 1);
        __syncthreads();
      }
    }
    if (!kStates && last && in_v)
      for (int64_t t = (int64_t)n + vr; t < p.tokens; t += 32) *(s16x8*)(at_out<T>(p.out, b, t, h) + kWide * block + 8 * vch) = s16x8{};
  } else if (!kStates) {
    // ---- out: rows 16 w4 .. + 15 of the chunk, lane has row 16 w4 + l16
    __builtin_amdgcn_s_setprio(1);
    const int vrow = 4 * g + (lane >> 2 & 3), low8 = (lane & 1) * 8;
    auto run = [&](auto which) {                    // W = w4, so that each wave's share of the triangle is straight code
      constexpr int W = decltype(which)::value;
      float decay[W + 1][4];                        // of A's tiles: keys 16 cb + 4 g + i
#pragma unroll
      for (int cb = 0; cb <= W; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int apart = 16 * (W - cb) + l16 - 4 * g - i;
          decay[cb][i] = power_of(max(apart, 0));
        }
      const float after = fmaxf(power_of(16 * W + l16) * p.decay[h], least);
      __syncthreads();
      for (int c = 0; c < chunks; ++c) {
        const char* const here = lds + (c & 1) * kSlot;
        const char* const copy = lds + kS + (c & 1) * kCopy;
        x8 q[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *(const x8*)(here + 16 * W * CH * 16 + slot<CH>(l16, 4 * s + g));
        f32x4 o[DT] = {};
        auto from_state = [&](int d) {
          f32x4 t = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < KS; ++s) t = mfma16(*(const x8*)(copy + 16 * d * CH * 16 + slot<CH>(l16, 4 * s + g)), q[s], t);
          t *= after;
          if (!kHalf) return t;
          const int4 e = exponents[c & 1][4 * d + g];
          return f32x4{ldexpf(t[0], e.x), ldexpf(t[1], e.y), ldexpf(t[2], e.z), ldexpf(t[3], e.w)};
        };
        auto scores = [&](int cb) {
          f32x4 t = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < KS; ++s) t = mfma16(*(const x8*)(here + kK + 16 * cb * CH * 16 + slot<CH>(l16, 4 * s + g)), q[s], t);
          return t;
        };
        float x[W / 2 + 1][8] = {};                 // A, 32 keys each
#pragma unroll
        for (int cb = 0; cb <= W; ++cb) {
          const f32x4 t = scores(cb);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[cb / 2][cb % 2 * 4 + i] = cb == W && l16 < 4 * g + i ? 0.0f : t[i] * decay[cb][i];
        }
        f32x4 before[DT];                           // the state's part of out
#pragma unroll
        for (int d = 0; d < DT; ++d) before[d] = from_state(d);
        float up = 1.0f;                            // the power of two that is out of this lane's row
        if (kHalf) {
          float most = 0.0f;
#pragma unroll
          for (int cb = 0; cb <= W; ++cb)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(x[cb / 2][cb % 2 * 4 + i]));
          const int exponent = max(__builtin_amdgcn_frexp_expf(column_max(most)) - 15, -100);
          const float down = ldexpf(1.0f, -exponent);
          up = ldexpf(1.0f, exponent);
#pragma unroll
          for (int cb = 0; cb <= W; ++cb)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[cb / 2][cb % 2 * 4 + i] *= down;
        }
        x8 a[W / 2 + 1];
#pragma unroll
        for (int j = 0; j <= W / 2; ++j) a[j] = round8<T>(x[j]);
        __builtin_amdgcn_sched_barrier(0);          // (as above)
        if (!kHalf) {
#pragma unroll
          for (int d = 0; d < DT; ++d) o[d] = before[d];
        }
#pragma unroll
        for (int j = 0; j <= W / 2; ++j)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const char* const from = here + kV + 32 * j * 128 + low8;
            const int cc = 2 * d + (lane >> 1 & 1);
            o[d] = mfma16(join8<T>(read_transposed(from + slot<8>(vrow, cc)), read_transposed(from + 16 * 128 + slot<8>(vrow, cc))), a[j], o[d]);
          }
        if (kHalf) {
#pragma unroll
          for (int d = 0; d < DT; ++d) o[d] = o[d] * up + before[d];
        }
        const int64_t t = (int64_t)(first + c) * kChunk + 16 * W + l16;
        if (t < n) {
          T* const to = at_out<T>(p.out, b, t, h) + kWide * block + 4 * g;
#pragma unroll
          for (int d = 0; d < DT; ++d)
            if (kWide * block + 16 * d + 4 * g < p.value_dim) *(x4*)(to + 16 * d) = round4<T>(p.scale * o[d]);
        }
        __syncthreads();
      }
    };
    switch (w4) {
      case 0: run(std::integral_constant<int, 0>{}); break;
      case 1: run(std::integral_constant<int, 1>{}); break;
      case 2: run(std::integral_constant<int, 2>{}); break;
      default: run(std::integral_constant<int, 3>{}); break;
    }
    if (any_met()) wait_for_chunks();               // (the waves that carry the state write what is right)
  }
}

// parts[s], s < segments - 1: what segment s adds, replaced by the state behind it.  A state that is replaced in place is kept behind
// them, since the workgroups of one launch may end before others begin.  Four values per thread.
__global__ __launch_bounds__(256) void k_retain_starts(RetentionParams p, int segments) {
  const int64_t size = (int64_t)p.key_dim * p.value_dim, states = (int64_t)p.batch * p.q_heads * size;
  const int64_t at_value = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (at_value >= states) return;
  const int64_t bh = at_value / size, b = bh / p.q_heads;
  const int n = p.lengths ? min(max(p.lengths[b], 0), p.tokens) : p.tokens, chunks = (int)(((int64_t)n + kChunk - 1) / kChunk), per_segment = (chunks + segments - 1) / segments;
  const int used = per_segment ? (chunks - 1) / per_segment : 0;   // segments before the sequence's last one
  const double far = exp2(p.log2_decay[bh % p.q_heads] * ((double)per_segment * kChunk));
  const float keep = fmaxf((float)far, least_power(p.decay[bh % p.q_heads])), keep_rest = (float)(far - (double)keep);
  f32x4 S = {0, 0, 0, 0};
  if (p.state_in) S = *(const f32x4*)(p.state_in + at_value);
  float* part = p.parts + at_value;
  if (p.state_in == p.state_out) *(f32x4*)(part + (segments - 1) * states) = S;
#pragma unroll 4
  for (int s = 0; s < used; ++s, part += states) {
    const f32x4 add = *(const f32x4*)part;
#pragma unroll
    for (int i = 0; i < 4; ++i) S[i] = fmaf(S[i], keep, fmaf(finite(S[i]), keep_rest, add[i]));
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
  // Step by step up to 8 tokens: of 8 tokens 64 sequences of 8 heads of 64 take 9.8 us, 11.3 as a chunk, 16 sequences of 16 heads of 128
  // 14.1 and 15.6 (8 sequences of 8 heads of 64, though, 6.9 and 5.7); of 12 tokens the first take 12.6 us and 11.3.
  plan.steps = p.tokens <= 8;
  // Segments that fill the device once, of three chunks and more: 8 heads of 64 of one sequence of 2000 tokens take 21.7 us, 37.9 whole; of 8
  // sequences of 1000 tokens 22.7 and 22.5, of 1300 25.9 and 28.5, of 2000 32.3 and 40.2; the first of 16 chunks, 1000 tokens, 19.3 and 21.6
  // (17.5 in segments of two chunks, 24.8 of six), and of 600 tokens 17.4 and 14.8.  Two rounds of workgroups lose: 8 sequences of 2000 tokens 42.5 us.
  // Two segments alone do as well, 16 sequences of 2000 tokens 47.5 us, 42.2 whole.
  plan.segments = 1;
  if (!plan.steps) {
    const int64_t chunks = ((int64_t)p.tokens + kChunk - 1) / kChunk;
    if (chunks >= 16) plan.segments = (int)std::max<int64_t>(1, std::min<int64_t>({256 / std::max<int64_t>(plan.workgroups, 1), chunks / 3, 32}));
  }
  return plan;
}

// Key dimensions in steps of 32 from 64 on, the values' in workgroups of 48 or 64 each, whichever leaves less over: the ragged clips
// of 96 x 80 take 24.4 us, 26.3 as 128 x 128; 500 tokens of 80 x 40, 160 times, 16.7 and 18.9.
template <class T, int KP>
const void* chunks_kernel(int value_dim, bool states) {
  const int blocks = (value_dim + 63) / 64;
  return value_dim > 48 * blocks ? states ? (const void*)k_retain_chunks<T, KP, 4, true> : (const void*)k_retain_chunks<T, KP, 4, false>
                                 : states ? (const void*)k_retain_chunks<T, KP, 3, true> : (const void*)k_retain_chunks<T, KP, 3, false>;
}
template <class T>
const void* chunks_kernel(const RetentionParams& p, bool states) {
  return p.key_dim <= 64 ? chunks_kernel<T, 64>(p.value_dim, states)
                         : p.key_dim <= 96 ? chunks_kernel<T, 96>(p.value_dim, states) : chunks_kernel<T, 128>(p.value_dim, states);
}
}  // namespace

size_t retention_workspace(const RetentionParams& p) {
  const RetentionPlan plan = plan_of(p);
  return plan.segments == 1 ? 0 : (size_t)plan.segments * p.batch * p.q_heads * p.key_dim * p.value_dim * sizeof(float);
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
    const hipError_t e = launch_kernel(half ? chunks_kernel<f16>(p, true) : chunks_kernel<bf16>(p, true), plan.workgroups * (plan.segments - 1), 512, args, stream);
    if (e != hipSuccess) return e;
    const hipError_t joined = launch_kernel((const void*)k_retain_starts, ((int64_t)p.batch * p.q_heads * p.key_dim * p.value_dim / 4 + 255) / 256, 256, args, stream);
    if (joined != hipSuccess) return joined;
  }
  return launch_kernel(half ? chunks_kernel<f16>(p, false) : chunks_kernel<bf16>(p, false), plan.workgroups * plan.segments, 768, args, stream);
}

}  // namespace hs
