// hs_cross_attention: attention of tokens to an encoder's states of another length.
#include "hs_track_device.h"

#include <math.h>

#include <algorithm>

namespace hs {

// out = softmax(scale * Q K^T) V by tiles of keys with a running maximum and sum.
//
// A wave has 32 rows (a row is a token and one of the query heads that share a key head) and forms, per tile of BN keys,
//   S^T = K Q^T          keys x rows: a lane's 16 values per 32 keys belong to ONE row, so maximum, sum and
//                        rescaling are per lane, with one exchange between the wave's halves;
//   O^T += V^T P^T       whose B operand is the lane's own P, rounded to 16 bits in place: the keys that a lane holds
//                        of S^T are taken as the product's k positions, and V^T is read from LDS (transposed) in that order.
// The weights P are rounded once to the inputs' type, as the matrix pipe takes them; their sum is formed
// before that, in fp32, as everything else.  Q stays in registers; K and V tiles go through registers into LDS
// while the tile before them is computed.
//
// QW waves side by side have other rows and share the tiles; KW groups of them take the keys in turn and are
// joined in LDS at the end.  Where that leaves the device idle the keys are cut further, over `splits`
// workgroups, whose partial results k_cross_join puts together.
//
// Large products (2040 tokens of 16 heads of 128 on 8160 keys, 8 times) take 1030 to 1080 us, 1.0 PFLOP/s: the matrix pipe is busy in
// 51 % of the cycles, the vector pipe in 47 %, most of it exponentials.  Few rows are bound by their keys and values (8 tokens on up
// to 6480 keys of 64, 96 heads: 3.8 TB/s in the first launch), the smallest by the chain of loads, products and join (7 us).
struct CrossGrid {
  int row_tiles, splits;
};

template <class T, int DP, int QW, int KW, int BN>
__global__ __launch_bounds__(64 * QW * KW, 2) void k_cross(CrossParams p, CrossGrid grid) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int CH = DP > 64 ? 16 : 8, KS = DP / 16, DT = DP / 32, NB = BN / 32;   // CH: 16-byte pieces per row in LDS
  constexpr int NT = 64 * QW;                       // threads that fill a tile together
  constexpr int NL = BN * CH / NT;                  // 16-byte loads per thread for K, and for V
  constexpr int kTile = BN * CH * 16;               // bytes
  constexpr int kBuffers = QW > 1 ? 2 : 1;          // a wave alone needs no second buffer: its accesses are in order
  constexpr int PT = DP + 4;                        // floats per row of a group's part: reads and writes spread over the banks
  constexpr int kTiles = KW * kBuffers * 2 * kTile, kParts = KW > 1 ? KW * QW * 32 * (PT + 2) * 4 : 0;
  constexpr int kLds = kTiles > kParts ? kTiles : kParts;
  __shared__ __align__(16) char lds[kLds];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qw = wave % QW, kw = wave / QW;
  const int row_in_wave = lane & 31, half = lane >> 5;
  char* const tiles = lds + kw * kBuffers * 2 * kTile;

  // the workgroups of one batch and key head read the same keys: on the same XCD
  int id = xcd_number();
  const int row_tile = id % grid.row_tiles;
  id /= grid.row_tiles;
  const int split = id % grid.splits;
  const int bh = id / grid.splits, kv_heads = p.q_heads / p.group, hk = bh % kv_heads, b = bh / kv_heads;
  const uint32_t rows = (uint32_t)p.q_tokens * p.group, group = p.group;   // below 2^31
  const uint32_t row = (row_tile * QW + qw) * 32 + row_in_wave;
  const bool live = row < rows;
  const uint32_t token = live ? row / group : 0;
  const int head = hk * p.group + (live ? (int)(row - token * group) : 0);

  // the keys of this workgroup: tiles first .. last - 1, of which group kw takes every KW-th
  const int n = length_of(p.lengths, b, p.k_tokens);
  const int all_tiles = (int)(((int64_t)n + BN - 1) / BN);
  const int first = (int)((int64_t)all_tiles * split / grid.splits), last = (int)((int64_t)all_tiles * (split + 1) / grid.splits);

  // the scale's sign, and a scale of zero, are taken into Q: maxima of scores are maxima of exponents
  const float scale = positive_scale(p.scale), c = scale * kLog2e;
  x8 q[KS];
  {
    const T* const src = at<T>(p.q, b, token, head);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      q[k] = x8{};
      const int d0 = 16 * k + 8 * half;
      if (live && d0 < p.dim) q[k] = *(const x8*)(src + d0);
      if (p.scale < 0.0f) q[k] = -q[k];
      if (p.scale == 0.0f) q[k] = x8{};
    }
  }
  f32x16 o[DT] = {};
  float m = -INFINITY, l = 0.0f;

  // staging: this thread's chunk of rows r0, r0 + NT / CH, ...  Rows behind the last key are read as that one, so that every
  // tile's loads are the same instructions: loads of two branches would be waited for where the branches meet.
  const int tg = threadIdx.x % NT, r0 = tg / CH, ch = tg % CH;
  const bool in_dim = 8 * ch < p.dim;
  const T* const ksrc = at<T>(p.k, b, 0, hk) + 8 * ch;
  const T* const vsrc = at<T>(p.v, b, 0, hk) + 8 * ch;
  const T* const klane = ksrc + r0 * p.k.token;
  const T* const vlane = vsrc + r0 * p.v.token;
  const uint8_t* const mask = p.mask ? p.mask + b * p.mask_batch : nullptr;
  s16x8 kreg[NL] = {}, vreg[NL] = {};
  uint8_t seen = 0;
  auto fetch = [&](int tile) {
    const int64_t j0 = (int64_t)tile * BN;
    const T *ka[NL], *va[NL];
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      ka[e] = klane + (j0 + e * (NT / CH)) * p.k.token;
      va[e] = vlane + (j0 + e * (NT / CH)) * p.v.token;
    }
    if (j0 + BN > n) {
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        const int64_t j = j0 + r0 + e * (NT / CH) < n ? j0 + r0 + e * (NT / CH) : (int64_t)n - 1;
        ka[e] = ksrc + j * p.k.token;
        va[e] = vsrc + j * p.v.token;
      }
    }
    if (in_dim) {
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        kreg[e] = load16(ka[e]);
        vreg[e] = load16(va[e]);
      }
    }
    if (mask) seen = mask[j0 + (lane & (BN - 1)) < n ? j0 + (lane & (BN - 1)) : (int64_t)n - 1];
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
      for (int e = 0; e < NL; ++e)
        if (!(visible >> (r0 + e * (NT / CH)) & 1)) vreg[e] = s16x8{};
    }
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int to = slot<CH>(r0 + e * (NT / CH), ch);
      *(s16x8*)(at_tile + to) = kreg[e];
      *(s16x8*)(at_tile + kTile + to) = vreg[e];
    }
    return visible;
  };
  int koff[KS], voff[DT][2];
#pragma unroll
  for (int k = 0; k < KS; ++k) koff[k] = slot<CH>(row_in_wave, 2 * k + half);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int r = 8 * s + 4 * half + (lane >> 2 & 3), cc = 4 * d + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
      voff[d][s] = kTile + slot<CH>(r, cc) + (lane & 1) * 8;
    }

  const int rounds = (last - first + KW - 1) / KW;
  if (first + kw < last) fetch(first + kw);
  for (int i = 0; i < rounds; ++i) {
    const int tile = first + kw + i * KW;
    char* const here = tiles + (kBuffers == 2 ? (i & 1) * 2 * kTile : 0);
    uint64_t visible = 0;
    if (tile < last) visible = store(tile, here);
    if (QW > 1) __syncthreads();
    if (tile + KW < last) fetch(tile + KW);
    if (!visible) continue;

    f32x16 s[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      s[kb] = f32x16{};
#pragma unroll
      for (int k = 0; k < KS; ++k) s[kb] = mfma32(*(const x8*)(here + koff[k] + kb * 32 * CH * 16), q[k], s[kb]);
    }
    if (QW > 1) reads_ahead<KS / 2, 2 * NB>();      // (2040 tokens on 8160 keys 1070 us, 1084 without)
    if (visible != kAll) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const uint32_t bits = (uint32_t)(visible >> (32 * kb)) >> (4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(bits >> (8 * (e / 4) + e % 4) & 1)) s[kb][e] = -INFINITY;
      }
    }
    float top = kLowest;                               // (some key is seen)
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
    float lo, hi;
    both_halves(top, lo, hi);
    top = fmaxf(lo, hi);
    if (__any((top - m) * c > kSlack)) {
      const float raised = fmaxf(m, top), keep = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - raised) * c);
      l *= keep;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= keep;
      m = raised;
    }
    const float mc = exponent_of<T>(m, c);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], c, -mc));
      float part[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) part[e] = (s[kb][e] + s[kb][4 + e]) + (s[kb][8 + e] + s[kb][12 + e]);
      l += (part[0] + part[1]) + (part[2] + part[3]);
    }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float w8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w8[e] = s[kb][8 * j + e];
        const x8 w = round8<T>(w8);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const char* const at_v = here + (32 * kb + 16 * j) * CH * 16;
          o[d] = mfma32(join8<T>(read_transposed(at_v + voff[d][0]), read_transposed(at_v + voff[d][1])), w, o[d]);
        }
      }
  }
  float lower, upper;
  both_halves(l, lower, upper);
  l = lower + upper;

  if (KW > 1) {   // the groups' parts of the same rows
    float* const part_o = (float*)lds;
    float* const part_ml = part_o + KW * QW * 32 * PT;
    __syncthreads();
    if (half == 0 && live) {
      part_ml[2 * (wave * 32 + row_in_wave)] = m;
      part_ml[2 * (wave * 32 + row_in_wave) + 1] = l;
    }
    if (live)
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *(f32x4*)(part_o + (wave * 32 + row_in_wave) * PT + 32 * d + 2 * e + 4 * half) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
    __syncthreads();
    // thread t: row t / 8 (of QW * 32), values 4 * (t % 8 + 8 * i)
    for (int r = threadIdx.x / 8; r < QW * 32; r += 8 * QW * KW) {
      const uint32_t at_row = row_tile * QW * 32 + r;
      if (at_row >= rows) break;
      float mm = -INFINITY, ll = 0.0f, f[KW];
#pragma unroll
      for (int g = 0; g < KW; ++g) mm = fmaxf(mm, part_ml[2 * (g * QW * 32 + r)]);
#pragma unroll
      for (int g = 0; g < KW; ++g) {
        const float mg = part_ml[2 * (g * QW * 32 + r)];
        f[g] = mg == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mg - mm) * c);
        ll = fmaf(part_ml[2 * (g * QW * 32 + r) + 1], f[g], ll);
      }
      const bool whole = grid.splits == 1;
      const float inv = whole ? inverse_sum(mm, ll) : 1.0f;
      const uint32_t tok = at_row / group;
      const int hh = hk * p.group + (int)(at_row - tok * group);
      const int64_t part_row = (int64_t)(split * (int64_t)(p.batch * kv_heads) + bh) * rows + at_row;
      for (int d0 = 4 * (threadIdx.x % 8); d0 < p.dim; d0 += 32) {
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < KW; ++g) sum += f[g] * *(const f32x4*)(part_o + (g * QW * 32 + r) * PT + d0);
        if (whole) {
          x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = (T)(sum[e] * inv);
          *(x4*)(at_out<T>(p.out, b, tok, hh) + d0) = y;
        } else {
          *(f32x4*)(p.parts + part_row * (p.dim + 4) + 4 + d0) = sum;
        }
      }
      if (threadIdx.x % 8 == 0) {
        if (!whole) {
          p.parts[part_row * (p.dim + 4)] = mm;
          p.parts[part_row * (p.dim + 4) + 1] = ll;
        } else if (p.lse) {
          p.lse[((int64_t)b * p.q_heads + hh) * p.q_tokens + tok] = ll == 0.0f ? -INFINITY : fmaf(mm, scale, logf(ll) - kRaise<T> * kLn2);
        }
      }
    }
    return;
  }
  if (!live) return;
  if (grid.splits > 1) {
    float* const part = p.parts + ((split * (int64_t)(p.batch * kv_heads) + bh) * rows + row) * (p.dim + 4);
    if (half == 0) {
      part[0] = m;
      part[1] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int d0 = 32 * d + 2 * e + 4 * half;
        if (d0 < p.dim) *(f32x4*)(part + 4 + d0) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
      }
    return;
  }
  const float inv = inverse_sum(m, l);
  T* const dst = at_out<T>(p.out, b, token, head);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int d0 = 32 * d + 2 * e + 4 * half;
      x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (T)(o[d][e + i] * inv);
      if (d0 < p.dim) *(x4*)(dst + d0) = y;
    }
  if (p.lse && half == 0) p.lse[((int64_t)b * p.q_heads + head) * p.q_tokens + token] = l == 0.0f ? -INFINITY : fmaf(m, scale, logf(l) - kRaise<T> * kLn2);
}

// The splits' parts of a row, each a maximum, a sum and a weighted sum of values: a wave per row.  Lane s has what weighs
// part s; then the wave's halves take even and odd parts, four values per lane.
constexpr int kMostSplits = 64;
template <class T>
__global__ __launch_bounds__(256) void k_cross_join(CrossParams p, int splits) {
  typedef typename Vec<T>::x4 x4;
  const int kv_heads = p.q_heads / p.group, lane = threadIdx.x & 63, half = lane >> 5;
  const int64_t rows = (int64_t)p.q_tokens * p.group, all = (int64_t)p.batch * kv_heads * rows;
  const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (id >= all) return;
  const float scale = positive_scale(p.scale), c = scale * kLog2e;
  const int64_t row = id % rows, bh = id / rows, b = bh / kv_heads, token = row / p.group;
  const int head = (int)(bh % kv_heads) * p.group + (int)(row % p.group);
  const int d0 = 4 * (lane & 31), pitch = p.dim + 4;
  const float* const parts = p.parts + id * pitch;
  float m = -INFINITY, l = 0.0f;
  if (lane < splits) {
    m = parts[lane * all * pitch];
    l = parts[lane * all * pitch + 1];
  }
  float top = m;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * c);
  l *= f;                                           // (a part that saw no key has 0, one whose scores are NaN keeps that)
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
  f32x4 sum = {0, 0, 0, 0};
  for (int s = 0; s < splits; s += 2) {
    const float w = __shfl(f, s + half);            // (of a part that is not there, or saw no key: 0)
    if (d0 < p.dim && w != 0.0f) sum += w * *(const f32x4*)(parts + (s + half) * all * pitch + 4 + d0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], 32);
  const float inv = inverse_sum(top, l);
  if (half == 0 && d0 < p.dim) *(x4*)(at_out<T>(p.out, b, token, head) + d0) = round4<T>(sum * inv);
  if (p.lse && lane == 0) p.lse[(b * p.q_heads + head) * p.q_tokens + token] = l == 0.0f ? -INFINITY : fmaf(top, scale, logf(l) - kRaise<T> * kLn2);
}

namespace {
struct CrossPlan {
  int wide;                     // so many waves with 32 rows each and the same keys, or
  int groups;                   // one set of 32 rows whose keys are dealt to so many waves
  CrossGrid grid;
  int64_t workgroups;
};
CrossPlan plan_of(const CrossParams& p) {
  const int64_t bh = (int64_t)p.batch * (p.q_heads / p.group), rows = (int64_t)p.q_tokens * p.group;
  CrossPlan plan;
  // Eight waves share a tile of wide heads, four one of narrow ones: 2040 tokens of 16 heads on 8160 keys, 8 times, take
  // 1095 and 1180 us of 128 dimensions, 757 and 721 of 64.
  const int waves = p.dim > 64 ? 8 : 4, tile = 32 * waves;
  const int64_t wide_tiles = (rows + tile - 1) / tile, wide = bh * wide_tiles, keys64 = ((int64_t)p.k_tokens + 63) / 64;
  auto at_most = [](int64_t room, int64_t base, int64_t parts) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({room / std::max<int64_t>(base, 1), parts, kMostSplits}));
  };
  // Where those tiles are too few for the device their keys are cut into parts of eight tiles and more, if at least half of the
  // rows are there and that fills most of it: 300 tokens on 3000 keys (18 heads of 64 in all) 33.4 us, by the form below 38.7;
  // 500 on 1000 (8 of 64) 9.6 and 12.4; with parts of four tiles 1000 on 2000 (8 heads of 128) takes 29.9 and not 23.3.
  const int cut = at_most(p.dim > 64 ? 256 : 512, wide, keys64 / 8);
  plan.groups = 0;
  // Row tiles enough for the device are taken whatever their rows: 40 tokens on 405 keys (64 times, 8 heads of 64) 15.4 us, 17.9 by the form
  // below, 8 tokens on 405 keys 14.5 and 16.0, 8 on 64 keys (40 times) 5.4 and 7.9.  With many more heads or keys than that and few rows it
  // is the slower one: 8 tokens on 405 keys (600 times) 112 and 95, (32 times) 10.6 and 7.9, of heads of 128 dimensions (600 times) 315 and 181.
  // And where the form below would need several rounds of workgroups for so few keys that most of its waves had none: 1755 tokens on
  // 5 keys (12 heads of 72) 7.6 us, 17.9; 113 on 4 (13 times, 6 heads of 96) 7.9, 12.3; 660 on 5 (3 times, 12 heads of 64) 7.3, 6.6.
  const int64_t tiles = ((int64_t)p.k_tokens + 31) / 32, few = bh * ((rows + 31) / 32);
  const bool short_keys = 2 * ((wide + 255) / 256) * keys64 < (few + 255) / 256 * ((tiles + 7) / 8 + 1);
  plan.wide = wide >= 256 || (2 * rows >= wide_tiles * tile && wide * cut >= 192) || short_keys ? waves : 0;
  plan.grid.row_tiles = (int)std::min<int64_t>(plan.wide ? wide_tiles : (rows + 31) / 32, INT32_MAX);
  plan.grid.splits = wide >= 256 ? 1 : cut;
  if (!plan.wide) {
    // Else each wave takes keys of its own: eight of one workgroup, or four of several, joined by a second launch, which costs
    // as much as three tiles more per wave (77 tokens on up to 1001 keys of 80 dimensions, 20 times: 14.6 us, 19.0 in three parts).
    const int splits = at_most(512, few, tiles / 16);
    const bool apart = (tiles + 4 * splits - 1) / (4 * splits) + 3 < (few + 255) / 256 * ((tiles + 7) / 8);
    plan.grid.splits = apart ? splits : 1;
    plan.groups = apart ? 4 : 8;
  }
  plan.workgroups = bh * plan.grid.row_tiles * plan.grid.splits;
  return plan;
}
// Steps of 32 dimensions from 64 on: 77 tokens on 1001 keys of 80 take 14.6 us, 15.5 as 128.
template <class T, int DP>
const void* kernel_of(const CrossPlan& plan) {
  if (plan.wide) return (const void*)k_cross<T, DP, (DP > 64 ? 8 : 4), 1, 64>;
  return plan.groups == 8 ? (const void*)k_cross<T, DP, 1, 8, 32> : (const void*)k_cross<T, DP, 1, 4, 32>;
}
template <class T>
const void* kernel_of(const CrossParams& p, const CrossPlan& plan) {
  return p.dim <= 64 ? kernel_of<T, 64>(plan) : p.dim <= 96 ? kernel_of<T, 96>(plan) : kernel_of<T, 128>(plan);
}
}  // namespace

size_t cross_workspace(const CrossParams& p) {
  const CrossPlan plan = plan_of(p);
  return plan.grid.splits == 1 ? 0 : (size_t)plan.grid.splits * p.batch * p.q_heads * p.q_tokens * (p.dim + 4) * sizeof(float);
}

hipError_t launch(const CrossParams& p, hipStream_t stream) {
  CrossParams params = p;
  CrossPlan plan = plan_of(p);
  void* args[] = {&params, &plan.grid};
  const bool half = p.dtype == HS_F16;
  const void* const kernel = half ? kernel_of<f16>(p, plan) : kernel_of<bf16>(p, plan);
  hipError_t e = launch_kernel(kernel, plan.workgroups, 64 * (plan.wide + plan.groups), args, stream);
  if (e != hipSuccess || plan.grid.splits == 1) return e;
  void* join_args[] = {&params, &plan.grid.splits};
  return launch_kernel(half ? (const void*)k_cross_join<f16> : (const void*)k_cross_join<bf16>,
                       ((int64_t)p.batch * p.q_heads * p.q_tokens + 3) / 4, 256, join_args, stream);
}

}  // namespace hs
