// hs_differential_attention: the difference of two softmax maps over the same values.
#include "hs_track_device.h"

#include <math.h>

#include <algorithm>

namespace hs {

// y = softmax(scale Q_0 K_0^T) V - lambda softmax(scale Q_1 K_1^T) V, out = y or its norm, by tiles of keys with a
// running maximum and sum for each map.  As in hs_cross_attention a wave has 32 rows (a row is a token and one of the heads that
// share keys), S^T = K Q^T leaves each row's scores in one lane pair, and O^T += V^T P^T takes them, rounded to 16 bits
// once, from the lanes that have them.
// That rounding spares a second product for what it leaves; where weights are spread over thousands of keys, and the difference
// is as small as what they average, half a step in each weight (bf16: up to 2^-8 of it) counts like the output's own rounding: an rms error
// of 2.55e-3 on 8160 keys, where the rounded output alone has 1.66e-3 (fp16: 3.2e-4 and 2.1e-4).  Weights in two parts, which need two thirds
// as many products again and registers that are not there, reach that for 840 -> 1230 us (2040 rows of 8 heads, 8 times); both maps' second
// parts in one product, by the ratio of the sums so far, for 1280; the first map's alone, 1003, would leave something of equal maps; bf16
// values as fp16 with weights of 11 bits, where that is exact, take a launch more and 924 -> 1076 us.
//
// Many rows (k_differential): eight waves, or four where heads and values are both of more than 64, have other rows and share the tiles; a wave
// forms both maps of its rows, so that each value that it reads from LDS is used twice: with a map per wave LDS would be busy as
// long as the matrix pipe.
// Few rows (k_differential_few): the waves of a workgroup have the same rows and take the keys in turn.
// Where either leaves the device idle the keys are cut further, over `splits` workgroups, which k_differential_join puts together.
//
// Many rows are bound by exponentials and products in turns (2040 rows of 8 heads of 64 on 8160 keys, values of 128, 8 times: 800 to 930 us,
// 0.88 to 1.0 PFLOP/s; vector pipe 56 %, matrix pipe 42 % busy), few by their keys' and values' way from memory and the
// chain of loads, products and join (8 on up to 6480 keys, 48 heads: 26 us, 3.1 TB/s, and 6 for the join; 8 on 405, 4 heads: 10 us).
struct DifferentialGrid {
  int row_tiles, splits;
};

// The sum over 16 lanes side by side, in each of them.
__device__ __forceinline__ float sum16(float x) {
  x += moved<0xb1>(x);                     // lane ^ 1
  x += moved<0x4e>(x);                     // lane ^ 2
  x += moved<0x141>(x);                    // 7 - lane
  return x + moved<0x140>(x);              // 15 - lane
}

// What a row's values are multiplied by: its norm's inverse.
__device__ __forceinline__ float row_factor(const DifferentialParams& p, float squares) {
  return p.norm ? rsqrtf(squares / (float)p.value_dim + p.eps) : 1.0f;
}

// a fa - b fb with both products rounded, so that equal maps leave nothing.
template <class V>
__device__ __forceinline__ V difference(V a, float fa, V b, float fb) {
#pragma clang fp contract(off)
  return a * fa - b * fb;
}

// Heads and values of more than 64 need more registers than two waves of a SIMD have.
__host__ __device__ constexpr int wide_waves(int dim, int value_dim) { return dim > 64 && value_dim > 64 ? 4 : 8; }
template <class T, int DP, int VP>
__global__ __launch_bounds__(64 * wide_waves(DP, VP), wide_waves(DP, VP) / 4) void k_differential(DifferentialParams p, DifferentialGrid grid) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int MAPS = 2, QW = wide_waves(DP, VP), BN = 64;
  constexpr int CK = DP > 64 ? 16 : 8, CV = VP > 64 ? 16 : 8, KS = DP / 16, DT = VP / 32, NB = BN / 32;   // CK, CV: 16-byte pieces per row in LDS
  constexpr int NT = 64 * QW;                       // threads that fill a tile together
  constexpr int NK = BN * CK / NT, NV = BN * CV / NT;   // 16-byte loads per thread for one map's keys, and for values
  constexpr int kKeys = BN * CK * 16, kTile = MAPS * kKeys + BN * CV * 16;   // bytes
  __shared__ __align__(16) char lds[2 * kTile];
  const int lane = threadIdx.x & 63, qw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row_in_wave = lane & 31, half = lane >> 5;

  // the workgroups of one batch and key head read the same keys: on the same XCD
  int id = xcd_number();
  const int row_tile = id % grid.row_tiles;
  id /= grid.row_tiles;
  const int split = id % grid.splits;
  const int bh = id / grid.splits, kv_heads = p.q_heads / p.group, hk = bh % kv_heads, b = bh / kv_heads;
  const uint32_t rows = (uint32_t)p.q_tokens * p.group, group = p.group;   // below 2^30
  const uint32_t row = (row_tile * QW + qw) * 32 + row_in_wave;
  const bool live = row < rows;
  const uint32_t token = live ? row / group : 0;
  const int head = hk * p.group + (live ? (int)(row - token * group) : 0);

  // the keys of this workgroup: tiles first .. last - 1
  const int n = length_of(p.lengths, b, p.k_tokens);
  const int all_tiles = (int)(((int64_t)n + BN - 1) / BN);
  const int first = (int)((int64_t)all_tiles * split / grid.splits), last = (int)((int64_t)all_tiles * (split + 1) / grid.splits);

  // the scale's sign, and a scale of zero, are taken into Q: maxima of scores are maxima of exponents
  const float c = positive_scale(p.scale) * kLog2e;
  x8 q[MAPS][KS];
#pragma unroll
  for (int a = 0; a < MAPS; ++a) {
    const T* const src = at<T>(p.q, b, token, 2 * head + a);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      q[a][k] = x8{};
      const int d0 = 16 * k + 8 * half;
      if (live && d0 < p.dim) q[a][k] = *(const x8*)(src + d0);
      if (p.scale < 0.0f) q[a][k] = -q[a][k];
      if (p.scale == 0.0f) q[a][k] = x8{};
    }
  }
  f32x16 o[MAPS][DT] = {};
  float m[MAPS], l[MAPS];
#pragma unroll
  for (int a = 0; a < MAPS; ++a) m[a] = -INFINITY, l[a] = 0.0f;

  // staging: this thread's chunk of rows r0, r0 + NT / CK, ...  Rows behind the last key are read as that one, so that every
  // tile's loads are the same instructions.
  const int tg = threadIdx.x % NT, kr = tg / CK, kc = tg % CK, vr = tg / CV, vc = tg % CV;
  const bool in_k = 8 * kc < p.dim, in_v = 8 * vc < p.value_dim;
  const T* const ksrc = at<T>(p.k, b, 0, 2 * hk) + 8 * kc;
  const T* const vsrc = at<T>(p.v, b, 0, hk) + 8 * vc;
  const uint8_t* const mask = p.mask ? p.mask + b * p.mask_batch : nullptr;
  s16x8 kreg[MAPS][NK] = {}, vreg[NV] = {};
  uint8_t seen = 0;
  auto fetch = [&](int tile) {
    const int64_t j0 = (int64_t)tile * BN, end = (int64_t)n - 1;
    const T *ka[NK], *va[NV];
#pragma unroll
    for (int e = 0; e < NK; ++e) ka[e] = ksrc + std::min(j0 + kr + e * (NT / CK), end) * p.k.token;
#pragma unroll
    for (int e = 0; e < NV; ++e) va[e] = vsrc + std::min(j0 + vr + e * (NT / CV), end) * p.v.token;
    if (in_k) {
#pragma unroll
      for (int e = 0; e < NK; ++e)
#pragma unroll
        for (int a = 0; a < MAPS; ++a) kreg[a][e] = load16(ka[e] + a * p.k.head);
    }
    if (in_v) {
#pragma unroll
      for (int e = 0; e < NV; ++e) vreg[e] = load16(va[e]);
    }
    if (mask) seen = mask[std::min(j0 + (lane & (BN - 1)), end)];
  };
  // the tile's keys as a bit set, and its values in LDS: hidden values as zeros, whatever they hold
  constexpr uint64_t kAll = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
  auto store = [&](int tile, char* at_tile) -> uint64_t {
    uint64_t visible = kAll;
    const int64_t left = n - (int64_t)tile * BN;
    if (left < BN) visible = (1ull << left) - 1;
    if (mask) visible &= __ballot(seen != 0);
    if (visible != kAll) {
#pragma unroll
      for (int e = 0; e < NV; ++e)
        if (!(visible >> (vr + e * (NT / CV)) & 1)) vreg[e] = s16x8{};
    }
#pragma unroll
    for (int e = 0; e < NK; ++e)
#pragma unroll
      for (int a = 0; a < MAPS; ++a) *(s16x8*)(at_tile + a * kKeys + slot<CK>(kr + e * (NT / CK), kc)) = kreg[a][e];
#pragma unroll
    for (int e = 0; e < NV; ++e) *(s16x8*)(at_tile + MAPS * kKeys + slot<CV>(vr + e * (NT / CV), vc)) = vreg[e];
    return visible;
  };
  // Chunk c of a row lies at c ^ swizzle: where chunks 4 d + .. lie is where chunk 0 + .. does but for the bits of 4 d.
  int koff[KS], voff[2];
#pragma unroll
  for (int k = 0; k < KS; ++k) koff[k] = slot<CK>(row_in_wave, 2 * k + half);
#pragma unroll
  for (int s = 0; s < 2; ++s)
    voff[s] = slot<CV>(8 * s + 4 * half + (lane >> 2 & 3), 2 * (lane >> 4 & 1) + (lane >> 1 & 1)) + (lane & 1) * 8;

  if (first < last) fetch(first);
  for (int tile = first; tile < last; ++tile) {
    char* const here = lds + ((tile - first) & 1) * kTile;
    const uint64_t visible = store(tile, here);
    __syncthreads();
    if (tile + 1 < last) fetch(tile + 1);
    if (!visible) continue;
#pragma unroll 1
    for (int kb = 0; kb < NB; ++kb) {
      const uint32_t bits = (uint32_t)(visible >> (32 * kb));
      if (!bits) continue;
      x8 w[MAPS][2];                                 // the maps' weights: 16 keys each
      // both maps' scores before either's softmax: those of the second are formed while the first's weights are (1120 us and 932 at 2040 rows of 8
      // heads on 8160 keys, 8 times)
      f32x16 scores[MAPS] = {};
#pragma unroll
      for (int a = 0; a < MAPS; ++a)
#pragma unroll
        for (int k = 0; k < KS; ++k) scores[a] = mfma32(*(const x8*)(here + a * kKeys + kb * 32 * CK * 16 + koff[k]), q[a][k], scores[a]);
#pragma unroll
      for (int a = 0; a < MAPS; ++a) {
        f32x16& s = scores[a];
        if (bits != ~0u) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!(bits >> (4 * half) >> (8 * (e / 4) + e % 4) & 1)) s[e] = -INFINITY;
        }
        float top = kLowest;                           // (some key is seen)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
        float lo, hi;
        both_halves(top, lo, hi);
        top = fmaxf(lo, hi);
        if (__any((top - m[a]) * c > kSlack)) {
          const float raised = fmaxf(m[a], top), keep = m[a] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m[a] - raised) * c);
          l[a] *= keep;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[a][d] *= keep;
          m[a] = raised;
        }
        const float mc = exponent_of<T>(m[a], c);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -mc));
        float part[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] = (s[e] + s[4 + e]) + (s[8 + e] + s[12 + e]);
        l[a] += (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float w8[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w8[e] = s[8 * j + e];
          w[a][j] = round8<T>(w8);
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const char* const at_v = here + MAPS * kKeys + (32 * kb + 16 * j) * CV * 16;
          const x8 v = join8<T>(read_transposed(at_v + (voff[0] ^ 64 * d)), read_transposed(at_v + (voff[1] ^ 64 * d)));
#pragma unroll
          for (int a = 0; a < MAPS; ++a) o[a][d] = mfma32(v, w[a][j], o[a][d]);
        }
    }
  }
#pragma unroll
  for (int a = 0; a < MAPS; ++a) {
    float lower, upper;
    both_halves(l[a], lower, upper);
    l[a] = lower + upper;
  }

  if (grid.splits > 1) {
    if (!live) return;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float* const part = p.parts + (((split * (int64_t)(p.batch * kv_heads) + bh) * rows + row) * 2 + a) * (p.value_dim + 4);
      if (half == 0) {
        part[0] = m[a];
        part[1] = l[a];
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const int d0 = 32 * d + 2 * e + 4 * half;
          if (d0 < p.value_dim) *(f32x4*)(part + 4 + d0) = f32x4{o[a][d][e], o[a][d][e + 1], o[a][d][e + 2], o[a][d][e + 3]};
        }
    }
    return;
  }
  const float f0 = inverse_sum(m[0], l[0]), f1 = p.lambda[head] * inverse_sum(m[1], l[1]);
  float squares = 0.0f;                            // (values behind the last are zero)
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    o[0][d] = difference(o[0][d], f0, o[1][d], f1);
#pragma unroll
    for (int e = 0; e < 16; ++e) squares = fmaf(o[0][d][e], o[0][d][e], squares);
  }
  float lower, upper;
  both_halves(squares, lower, upper);
  const float factor = row_factor(p, lower + upper);
  const bool saw = m[0] != -INFINITY;              // (both maps alike; else zeros, whatever lambda and the weights are)
  if (!live) return;
  T* const dst = at_out<T>(p.out, b, token, head);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int d0 = 32 * d + 2 * e + 4 * half;
      if (d0 >= p.value_dim) continue;
      x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (T)(saw ? o[0][d][e + i] * factor * (p.weight ? p.weight[d0 + i] : 1.0f) : 0.0f);
      *(x4*)(dst + d0) = y;
    }
}

// Few rows: 16 to a workgroup, whose eight waves take tiles of 32 keys in turn and are joined in LDS.  A wave forms both maps, on
// products of 16 x 16, whose results (keys 4g .. 4g + 3 of a row in lane group g, two tiles of 16 keys side by side) are
// operands of the next product.  Keys go from memory into the registers that multiply them; values, which are needed
// transposed, through LDS of the wave's own.
constexpr int kFewWaves = 8;
template <class T, int DP, int VP>
__global__ __launch_bounds__(64 * kFewWaves, 2) void k_differential_few(DifferentialParams p, DifferentialGrid grid) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int CV = VP > 64 ? 16 : 8, KS = DP / 32, DT = VP / 16, NV = 32 * CV / 64, kTile = 32 * CV * 16;
  constexpr int PT = VP + 4;                        // floats per row of a wave's part: reads and writes spread over the banks
  constexpr int kParts = kFewWaves * 2 * 16 * (PT + 2) * 4, kTiles = kFewWaves * kTile;
  __shared__ __align__(16) char lds[kParts > kTiles ? kParts : kTiles];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  char* const here = lds + wave * kTile;

  int id = xcd_number();                            // the workgroups of one batch and key head read the same keys: on the same XCD
  const int row_tile = id % grid.row_tiles;
  id /= grid.row_tiles;
  const int split = id % grid.splits;
  const int bh = id / grid.splits, kv_heads = p.q_heads / p.group, hk = bh % kv_heads, b = bh / kv_heads;
  const uint32_t rows = (uint32_t)p.q_tokens * p.group, group = p.group;   // below 2^30
  const uint32_t row = row_tile * 16 + col;
  const bool live = row < rows;
  const uint32_t token = live ? row / group : 0;
  const int head = hk * p.group + (live ? (int)(row - token * group) : 0);
  const int n = length_of(p.lengths, b, p.k_tokens), all_tiles = (int)(((int64_t)n + 31) / 32);
  const int first = (int)((int64_t)all_tiles * split / grid.splits), last = (int)((int64_t)all_tiles * (split + 1) / grid.splits);

  const float c = positive_scale(p.scale) * kLog2e;
  // a lane has DP / 4 dimensions side by side of a query, as of a key
  x8 q[2][KS];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const T* const src = at<T>(p.q, b, token, 2 * head + a);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      q[a][k] = x8{};
      const int d0 = (DP / 4) * g + 8 * k;
      if (live && d0 < p.dim) q[a][k] = *(const x8*)(src + d0);
      if (p.scale < 0.0f) q[a][k] = -q[a][k];
      if (p.scale == 0.0f) q[a][k] = x8{};
    }
  }
  f32x4 o[2][DT] = {};
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {};

  const int vr = lane / CV, vc = lane % CV;
  const bool in_v = 8 * vc < p.value_dim;
  const T* const ksrc = at<T>(p.k, b, 0, 2 * hk);
  const T* const vsrc = at<T>(p.v, b, 0, hk) + (in_v ? 8 * vc : 0);
  const uint8_t* const mask = p.mask ? p.mask + b * p.mask_batch : nullptr;
  x8 key[2][2][KS];                                 // [keys][map]
  s16x8 vreg[NV];
  uint8_t seen = 0;
  auto fetch = [&](int tile) {                      // (what lies behind the last key, or behind a head's dimensions, is read as what is there)
    const int64_t j0 = (int64_t)tile * 32, end = (int64_t)n - 1;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const T* const from = ksrc + std::min(j0 + 16 * t + col, end) * p.k.token;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int k = 0; k < KS; ++k) key[t][a][k] = __builtin_bit_cast(x8, load16(from + a * p.k.head + std::min((DP / 4) * g + 8 * k, p.dim - 8)));
    }
#pragma unroll
    for (int e = 0; e < NV; ++e) vreg[e] = load16(vsrc + std::min(j0 + vr + e * (64 / CV), end) * p.v.token);
    if (mask) seen = mask[std::min(j0 + (lane & 31), end)];
  };
  int voff[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) voff[d] = slot<CV>(4 * g + (col >> 2), 2 * d + (col >> 1 & 1)) + (col & 1) * 8;

  if (first + wave < last) fetch(first + wave);
  for (int tile = first + wave; tile < last; tile += kFewWaves) {
    uint32_t visible = ~0u;
    const int64_t left = n - (int64_t)tile * 32;
    if (left < 32) visible = (1u << left) - 1;
    if (mask) visible &= (uint32_t)__ballot(seen != 0);
#pragma unroll
    for (int e = 0; e < NV; ++e) {
      const int r = vr + e * (64 / CV);
      if (!(visible >> r & 1) || !in_v) vreg[e] = s16x8{};       // hidden values as zeros, whatever they hold
      *(s16x8*)(here + slot<CV>(r, vc)) = vreg[e];
    }
    f32x4 s[2][2];                                  // [map][keys]
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[a][t] = f32x4{};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const bool there = (DP / 4) * g + 8 * k < p.dim;
          s[a][t] = mfma16(there ? key[t][a][k] : x8{}, q[a][k], s[a][t]);
        }
      }
    if (tile + kFewWaves < last) fetch(tile + kFewWaves);
    if (!visible) continue;
    wave_order();
    x8 w[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      if (visible != ~0u) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(visible >> (16 * t + 4 * g + i) & 1)) s[a][t][i] = -INFINITY;
      }
      float top = kLowest;                             // (some key is seen)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(fmaxf(top, s[a][0][i]), s[a][1][i]);
      top = column_max(top);
      if (__any((top - m[a]) * c > kSlack)) {
        const float raised = fmaxf(m[a], top), keep = m[a] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m[a] - raised) * c);
        l[a] *= keep;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[a][d] *= keep;
        m[a] = raised;
      }
      const float mc = exponent_of<T>(m[a], c);
      float w8[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w8[i] = __builtin_amdgcn_exp2f(fmaf(s[a][i / 4][i % 4], c, -mc));
      l[a] += ((w8[0] + w8[1]) + (w8[2] + w8[3])) + ((w8[4] + w8[5]) + (w8[6] + w8[7]));
      w[a] = round8<T>(w8);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const x8 v = join8<T>(read_transposed(here + voff[d]), read_transposed(here + voff[d] + 16 * CV * 16));
#pragma unroll
      for (int a = 0; a < 2; ++a) o[a][d] = mfma16(v, w[a], o[a][d]);
    }
    wave_order();
  }

  // the waves' parts: lane l has values 16 d + 4 g + i of row l % 16
  float* const part_o = (float*)lds;
  float* const part_ml = part_o + kFewWaves * 2 * 16 * PT;
  __syncthreads();
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    l[a] += __shfl_xor(l[a], 16);
    l[a] += __shfl_xor(l[a], 32);
    const int at_part = (wave * 2 + a) * 16 + col;
    if (g == 0) {
      part_ml[2 * at_part] = m[a];
      part_ml[2 * at_part + 1] = l[a];
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) *(f32x4*)(part_o + at_part * PT + 16 * d + 4 * g) = o[a][d];
  }
  __syncthreads();
  // thread t: row t / 32, values 4 * (t % 32) .. + 3
  const int r = threadIdx.x / 32, d0 = 4 * (threadIdx.x % 32);
  const uint32_t at_row = row_tile * 16 + r;
  if (at_row >= rows) return;
  f32x4 sum[2] = {};
  float mm[2], ll[2];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    mm[a] = -INFINITY;
    ll[a] = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) mm[a] = fmaxf(mm[a], part_ml[2 * ((2 * w + a) * 16 + r)]);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const int at_part = (2 * w + a) * 16 + r;
      const float mw = part_ml[2 * at_part], f = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mw - mm[a]) * c);
      ll[a] = fmaf(part_ml[2 * at_part + 1], f, ll[a]);
      if (d0 < VP) sum[a] += f * *(const f32x4*)(part_o + at_part * PT + d0);
    }
  }
  const uint32_t tok = at_row / group;
  const int hh = hk * p.group + (int)(at_row - tok * group);
  if (grid.splits > 1) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float* const part = p.parts + (((split * (int64_t)(p.batch * kv_heads) + bh) * rows + at_row) * 2 + a) * (p.value_dim + 4);
      if (d0 == 0) {
        part[0] = mm[a];
        part[1] = ll[a];
      }
      if (d0 < p.value_dim) *(f32x4*)(part + 4 + d0) = sum[a];
    }
    return;
  }
  f32x4 y = difference(sum[0], inverse_sum(mm[0], ll[0]), sum[1], p.lambda[hh] * inverse_sum(mm[1], ll[1]));
  float squares = d0 < p.value_dim ? fmaf(y[0], y[0], fmaf(y[1], y[1], fmaf(y[2], y[2], y[3] * y[3]))) : 0.0f;
  squares = sum16(squares);
  squares += __shfl_xor(squares, 16);
  const float factor = row_factor(p, squares);
  if (d0 >= p.value_dim) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = mm[0] != -INFINITY ? y[e] * factor * (p.weight ? p.weight[d0 + e] : 1.0f) : 0.0f;
  *(x4*)(at_out<T>(p.out, b, tok, hh) + d0) = round4<T>(y);
}

// The splits' parts of a row, for each map a maximum, a sum and a weighted sum of values: a wave per row.  Lane s has what weighs
// part s; then the wave's halves take even and odd parts, four values per lane.
constexpr int kMostParts = 64;
template <class T>
__global__ __launch_bounds__(256) void k_differential_join(DifferentialParams p, int splits) {
  typedef typename Vec<T>::x4 x4;
  const int kv_heads = p.q_heads / p.group, lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t rows = (int64_t)p.q_tokens * p.group, all = (int64_t)p.batch * kv_heads * rows;
  const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (id >= all) return;
  const float c = positive_scale(p.scale) * kLog2e;
  const int64_t row = id % rows, bh = id / rows, b = bh / kv_heads, token = row / p.group;
  const int head = (int)(bh % kv_heads) * p.group + (int)(row % p.group);
  const int d0 = 4 * (lane & 31), pitch = p.value_dim + 4;
  f32x4 y = {0, 0, 0, 0};
  float first = 0.0f;
  bool saw = false;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const float* const parts = p.parts + (id * 2 + a) * pitch;
    float m = -INFINITY, l = 0.0f;
    if (lane < splits) {
      m = parts[lane * all * 2 * pitch];
      l = parts[lane * all * 2 * pitch + 1];
    }
    float top = m;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * c);
    l *= f;                                         // (a part that saw no key has 0, one whose scores are NaN keeps that)
#pragma unroll
    for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
    f32x4 sum = {0, 0, 0, 0};
    const int at_value = d0 < p.value_dim ? d0 : 0;
#pragma unroll 4
    for (int s = 0; s < splits; s += 2) {
      const int part = std::min(s + half, splits - 1);
      const float theirs = __shfl(f, part);                                // (from every lane: one that a branch leaves out gives zero)
      const float w = s + half < splits ? theirs : 0.0f;                   // (of a part that saw no key: 0, and so are its sums)
      sum += w * *(const f32x4*)(parts + part * all * 2 * pitch + 4 + at_value);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], 32);
    const float inv = inverse_sum(top, l);
    if (a == 0) {
      y = sum;
      first = inv;
    } else {
      y = difference(y, first, sum, p.lambda[head] * inv);
    }
    saw = top != -INFINITY;                        // (of both maps alike)
  }
  float squares = half || d0 >= p.value_dim ? 0.0f : fmaf(y[0], y[0], fmaf(y[1], y[1], fmaf(y[2], y[2], y[3] * y[3])));
#pragma unroll
  for (int d = 1; d < 64; d *= 2) squares += __shfl_xor(squares, d);
  const float factor = row_factor(p, squares);
  if (half || d0 >= p.value_dim) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = saw ? y[e] * factor * (p.weight ? p.weight[d0 + e] : 1.0f) : 0.0f;
  *(x4*)(at_out<T>(p.out, b, token, head) + d0) = round4<T>(y);
}

namespace {
struct DifferentialPlan {
  bool wide;                    // k_differential: eight or four waves with 32 rows each and the same keys; else eight with the same 16 rows
  DifferentialGrid grid;
  int64_t workgroups;
};
DifferentialPlan plan_of(const DifferentialParams& p) {
  const int64_t bh = (int64_t)p.batch * (p.q_heads / p.group), rows = (int64_t)p.q_tokens * p.group;
  DifferentialPlan plan;
  const int tile = 32 * wide_waves(p.dim, p.value_dim);
  const int64_t wide_tiles = (rows + tile - 1) / tile, wide = bh * wide_tiles, keys64 = ((int64_t)p.k_tokens + 63) / 64;
  auto at_most = [](int64_t room, int64_t base, int64_t parts) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({room / std::max<int64_t>(base, 1), parts, kMostParts}));
  };
  // Where row tiles are too few for the device their keys are cut into parts of eight tiles and more, if at least half of the rows are there
  // and that fills most of it: 256 tokens of 5 heads on 20000 keys 61 us, 72 by the other form; with parts of four tiles 66, of sixteen 72; 1000
  // on 2000 (4 times, 4 heads) 61, 63 and 72.  Where it fills less the other form is taken: 500 on 3000 (twice, 4 heads) 36 us and 48, 129 on 2100
  // (twice, 2 heads) 18 and 38; from about half of the device on it is the slower one: 1000 on 1100 (4 times, 4 heads on 2) 64 and 52.
  const int cut = at_most(256, wide, keys64 / 8);
  const int64_t tiles = ((int64_t)p.k_tokens + 31) / 32, few = bh * ((rows + 15) / 16);
  // Row tiles enough for the device are taken whatever their rows: 128 tokens on 405 keys (64 times, 4 heads) 37 us, 82 by the other form, 100
  // tokens 36 and 72, 40 tokens 32 and 32, 130 on 40 keys 13 and 58.  With fewer rows it is the slower one: 8 on 405 keys (64 times) 31 and 15,
  // (600 times) 296 and 146.  Rows that fill less than the device are taken by the other form on a few keys too, of whose waves most have none
  // then: 1755 tokens on 5 keys of 4 heads 14 us, 20 by row tiles, of 12 heads 38 and 20; 2040 on 405 of 12 heads 65 and 37.
  plan.wide = wide >= 256 || (2 * rows >= wide_tiles * tile && wide * cut >= 192);
  plan.grid.row_tiles = (int)std::min<int64_t>(plan.wide ? wide_tiles : (rows + 15) / 16, INT32_MAX);
  plan.grid.splits = wide >= 256 ? 1 : cut;
  if (!plan.wide) {
    // Parts of sixteen tiles and more (8 tokens of 4 heads on 6480 keys 19 us, with eight 21, with 24 21).  The second launch, which joins them,
    // costs as much as five rounds of tiles: on 1001 keys 15.6 us in one launch and 15.0 in two, on 2040 24.3 and 15.4; 5 x 77 on 1001 15.2 and 15.3.
    const int splits = at_most(256, few, tiles / 16);
    const bool apart = (tiles + 8 * splits - 1) / (8 * splits) + 5 < (few + 255) / 256 * ((tiles + 7) / 8);
    plan.grid.splits = apart ? splits : 1;
  }
  plan.workgroups = bh * plan.grid.row_tiles * plan.grid.splits;
  return plan;
}
template <class T, int DP, int VP>
const void* kernel_of(const DifferentialPlan& plan) {
  return plan.wide ? (const void*)k_differential<T, DP, VP> : (const void*)k_differential_few<T, DP, VP>;
}
template <class T>
const void* kernel_of(const DifferentialParams& p, const DifferentialPlan& plan) {
  if (p.dim <= 64) return p.value_dim <= 64 ? kernel_of<T, 64, 64>(plan) : kernel_of<T, 64, 128>(plan);
  return p.value_dim <= 64 ? kernel_of<T, 128, 64>(plan) : kernel_of<T, 128, 128>(plan);
}
}  // namespace

size_t differential_workspace(const DifferentialParams& p) {
  const DifferentialPlan plan = plan_of(p);
  return plan.grid.splits == 1 ? 0 : (size_t)plan.grid.splits * p.batch * p.q_heads * p.q_tokens * 2 * (p.value_dim + 4) * sizeof(float);
}

hipError_t launch(const DifferentialParams& p, hipStream_t stream) {
  DifferentialParams params = p;
  DifferentialPlan plan = plan_of(p);
  const unsigned threads = 64 * (plan.wide ? wide_waves(p.dim, p.value_dim) : kFewWaves);
  void* args[] = {&params, &plan.grid};
  const bool half = p.dtype == HS_F16;
  hipError_t e = launch_kernel(half ? kernel_of<f16>(p, plan) : kernel_of<bf16>(p, plan), plan.workgroups, threads, args, stream);
  if (e != hipSuccess || plan.grid.splits == 1) return e;
  void* join_args[] = {&params, &plan.grid.splits};
  return launch_kernel(half ? (const void*)k_differential_join<f16> : (const void*)k_differential_join<bf16>,
                       ((int64_t)p.batch * p.q_heads * p.q_tokens + 3) / 4, 256, join_args, stream);
}

}  // namespace hs
