// hs_expert_layer: a router and the experts' networks for a few tokens.
#include "hs_track_device.h"

#include <math.h>

#include <algorithm>

namespace hs {
namespace {

constexpr int kSlice = 16;      // hidden values with a power of two of their own

struct ExpertParts {            // the workspace
  int32_t* chosen;              // [tokens][top]
  float* weights;               // [tokens][top]
  void* hidden;                 // [tokens][top][hidden], in the inputs' type
  int16_t* power;               // [tokens][top][hidden / 16]: what fp16 values were divided by, as a power of two
  float* products;              // [tokens][top][channels]
  int32_t* count;               // [experts]: pairs that chose it
  int32_t* list;                // [experts][tokens]: these pairs, in their order
  size_t bytes;
};
__host__ __device__ inline int slices_of(const ExpertParams& p) { return (p.hidden + kSlice - 1) / kSlice; }
ExpertParts parts_of(const ExpertParams& p) {
  ExpertParts w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* const here = p.parts + at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  const size_t pairs = (size_t)p.tokens * p.top;
  w.chosen = (int32_t*)take(pairs * 4);
  w.weights = (float*)take(pairs * 4);
  w.hidden = take(pairs * p.hidden * 2);
  w.power = (int16_t*)take(p.dtype == HS_F16 ? pairs * slices_of(p) * 2 : 0);
  w.products = (float*)take(pairs * p.channels * 4);
  w.count = (int32_t*)take((size_t)p.experts * 4);
  w.list = (int32_t*)take((size_t)p.experts * p.tokens * 4);
  w.bytes = at;
  return w;
}

// Scores as whole numbers in their order, those of NaN below all others.
__device__ __forceinline__ uint64_t rank_of(double x) {
  if (x != x) return 0;
  const uint64_t bits = __builtin_bit_cast(uint64_t, x == 0.0 ? 0.0 : x);
  return bits >> 63 ? ~bits : bits | 1ull << 63;
}

// A workgroup per token: scores in 64 bits, a quarter of the experts per wave; the first wave chooses, lane l with experts
// l, l + 64, ..
template <class T>
__global__ __launch_bounds__(256) void k_expert_route(ExpertParams p, ExpertParts w) {
  typedef typename Vec<T>::x8 x8;
  __shared__ double scores[HS_MAX_EXPERTS];
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (p.mask && !p.mask[t]) {
    if ((int)threadIdx.x < p.top) {
      w.chosen[t * p.top + lane] = -1;
      w.weights[t * p.top + lane] = 0.0f;
      if (p.chosen) p.chosen[t * p.top + lane] = -1;
      if (p.weights) p.weights[t * p.top + lane] = 0.0f;
    }
    return;
  }
  const T* const x = (const T*)p.x + t * p.x_stride;
  constexpr int kAtOnce = 4;
  for (int e0 = wave; e0 < p.experts; e0 += 4 * kAtOnce) {
    double sum[kAtOnce] = {};
    for (int c = 8 * lane; c < p.channels; c += 512) {
      const x8 a = *(const x8*)(x + c);
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const int e = min(e0 + 4 * n, p.experts - 1);
        const x8 r = *(const x8*)((const T*)p.router + (int64_t)e * p.channels + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[n] = fma((double)(float)a[i], (double)(float)r[i], sum[n]);
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) sum[n] += __shfl_xor(sum[n], d);
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n)
      if (lane == n && e0 + 4 * n < p.experts) scores[e0 + 4 * n] = sum[n];
  }
  __syncthreads();
  if (wave > 0) return;
  double score[HS_MAX_EXPERTS / 64];
#pragma unroll
  for (int i = 0; i < HS_MAX_EXPERTS / 64; ++i) score[i] = lane + 64 * i < p.experts ? scores[lane + 64 * i] : 0.0;
  double best[HS_MAX_TOP];
  uint32_t taken = 0;
  double most = 0.0;
  for (int n = 0; n < p.top; ++n) {
    uint64_t rank = 0;
    int index = INT32_MAX;
    double value = 0.0;
#pragma unroll
    for (int i = 0; i < HS_MAX_EXPERTS / 64; ++i) {
      if (lane + 64 * i >= p.experts || taken >> i & 1) continue;
      const uint64_t r = rank_of(score[i]);
      if (index == INT32_MAX || r > rank) rank = r, index = lane + 64 * i, value = score[i];
    }
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t r = __shfl_xor(rank, d);
      const int other = __shfl_xor(index, d);
      const double v = __shfl_xor(value, d);
      if (other != INT32_MAX && (index == INT32_MAX || r > rank || (r == rank && other < index))) rank = r, index = other, value = v;
    }
    if ((index & 63) == lane) taken |= 1u << (index >> 6);
    if (n == 0) most = value;
    if (lane == n) {
      w.chosen[t * p.top + n] = index;
      if (p.chosen) p.chosen[t * p.top + n] = index;
    }
#pragma unroll
    for (int i = 0; i < HS_MAX_TOP; ++i)
      if (i == n) best[i] = value;
  }
  double total = 0.0;
  if (p.renormalise) {
#pragma unroll
    for (int i = 0; i < HS_MAX_TOP; ++i)
      if (i < p.top) total += exp(best[i] - most);
  } else {
#pragma unroll
    for (int i = 0; i < HS_MAX_EXPERTS / 64; ++i)
      if (lane + 64 * i < p.experts) total += exp(score[i] - most);
    for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
  }
#pragma unroll
  for (int i = 0; i < HS_MAX_TOP; ++i)
    if (i < p.top && lane == i) {
      const float weight = (float)(exp(best[i] - most) / total);
      w.weights[t * p.top + i] = weight;
      if (p.weights) p.weights[t * p.top + i] = weight;
    }
}

// The pairs (token, place) that chose expert e, in their order: those numbered first .. first + most - 1 of them are left in
// `list`; returns how many these are.  For a whole workgroup of 256.
__device__ __forceinline__ int pairs_of(const ExpertParams& p, const int32_t* chosen, int e, int first, int most, int32_t* list, int* counts) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = p.tokens * p.top;
  int seen = 0;
  for (int at = 0; at < pairs && seen < first + most; at += 256) {
    const int i = at + threadIdx.x;
    const bool hit = i < pairs && chosen[i] == e;
    const uint64_t hits = __ballot(hit);
    if (lane == 0) counts[wave] = __popcll(hits);
    __syncthreads();
    int place = seen + __popcll(hits & ((1ull << lane) - 1));
    for (int n = 0; n < 4; ++n) {
      if (n < wave) place += counts[n];
      seen += counts[n];
    }
    if (hit && place >= first && place < first + most) list[place - first] = i;
    __syncthreads();
  }
  return min(max(seen - first, 0), most);
}

// Products of RT tiles of 16 weight rows with NT tiles of 16 vectors over steps first .. last - 1 of 64: a lane has 16 values side by
// side of a row, so that four lanes read 128 bytes of it, and of a vector; the matrix pipe takes them in the same order.
// Lane l has result [row 4 * (l / 16) + i][vector l % 16].  A step's loads are issued before the products of the one before.
template <class T, int RT, int NT, bool POWERS>
__device__ __forceinline__ void products(const T* const (&rows)[RT], const T* const (&vectors)[NT], const int16_t* const (&power)[NT],
                                         const int (&row_power)[NT], int first, int last, int length, f32x4 (&acc)[RT][NT]) {
  typedef typename Vec<T>::x8 x8;
  const int g = (threadIdx.x & 63) >> 4;
  struct Step {
    x8 a[RT][2], b[NT][2];
    int16_t power[NT];
  };
  auto load = [&](int step, Step& s) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int d0 = min(64 * step + 16 * g + 8 * e, length - 8);   // (what lies behind the row's end is left out below)
#pragma unroll
      for (int r = 0; r < RT; ++r) s.a[r][e] = __builtin_bit_cast(x8, load16(rows[r] + d0));
#pragma unroll
      for (int n = 0; n < NT; ++n) s.b[n][e] = __builtin_bit_cast(x8, load16(vectors[n] + d0));
    }
    if (POWERS)
#pragma unroll
      for (int n = 0; n < NT; ++n) s.power[n] = power[n][min(64 * step + 16 * g, length - 1) / kSlice];
  };
  auto multiply = [&](int step, Step& s) {
    if (64 * step + 64 > length) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (64 * step + 16 * g + 8 * e >= length) {
#pragma unroll
          for (int r = 0; r < RT; ++r) s.a[r][e] = x8{};
#pragma unroll
          for (int n = 0; n < NT; ++n) s.b[n][e] = x8{};
        }
    }
    if (POWERS)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const T f = (T)ldexpf(1.0f, max(s.power[n] - row_power[n], -40));
        s.b[n][0] *= f;
        s.b[n][1] *= f;
      }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = mfma16(s.a[r][e], s.b[n][e], acc[r][n]);
  };
  Step even, odd;
  if (first < last) load(first, even);
  for (int step = first; step < last; step += 2) {
    if (step + 1 < last) load(step + 1, odd);
    multiply(step, even);
    if (step + 1 >= last) break;
    if (step + 2 < last) load(step + 2, even);
    multiply(step + 1, odd);
  }
}

constexpr int kNoPower = -1000;   // of a slice of zeros

// Hidden layer: a workgroup has an expert, 16 of its hidden values and up to 16 * NT of its tokens; its four waves take a quarter
// of the channels each.
template <class T, int NT>
__global__ __launch_bounds__(256) void k_expert_in(ExpertParams p, ExpertParts w, int groups) {
  __shared__ int32_t list[16 * NT];
  __shared__ int counts[4];
  __shared__ f32x4 partial[4][2][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15;
  int id = xcd_number();
  const int group = id % groups, slices = slices_of(p);
  id /= groups;
  const int slice = id % slices, e = id / slices;
  const int n = pairs_of(p, w.chosen, e, group * 16 * NT, 16 * NT, list, counts);
  if (n == 0) return;
  const T* vectors[NT];                              // (a place without a token has the first's, and is left out below)
  const int16_t* none[NT] = {};
  int zero[NT] = {};
#pragma unroll
  for (int i = 0; i < NT; ++i) vectors[i] = (const T*)p.x + (int64_t)(list[16 * i + col < n ? 16 * i + col : 0] / p.top) * p.x_stride;
  const T* const gate = (const T*)p.w_in + ((int64_t)e * 2 * p.hidden + min(16 * slice + col, p.hidden - 1)) * p.channels;
  const T* const rows[2] = {gate, gate + (int64_t)p.hidden * p.channels};
  const int steps = (p.channels + 63) / 64;
  f32x4 acc[2][NT] = {};
  products<T, 2, NT, false>(rows, vectors, none, zero, steps * wave / 4, steps * (wave + 1) / 4, p.channels, acc);
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int i = 0; i < NT; ++i) partial[wave][r][i][lane] = acc[r][i];
  __syncthreads();
  // thread t: hidden value t % 16 of token t / 16
  const int u = threadIdx.x & 15, at = threadIdx.x >> 4, from = (u >> 2) * 16 + at;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (16 * i >= n) break;
    float y[2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
      y[r] = (partial[0][r][i][from][u & 3] + partial[1][r][i][from][u & 3]) + (partial[2][r][i][from][u & 3] + partial[3][r][i][from][u & 3]);
    float h = y[0] / (1.0f + expf(-y[0])) * y[1];
    const bool stored = 16 * i + at < n && 16 * slice + u < p.hidden;
    const int64_t pair = list[min(16 * i + at, n - 1)];
    if (__is_same(T, f16)) {
      float most = stored ? fabsf(h) : 0.0f;
#pragma unroll
      for (int d = 1; d < 16; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
      const int power = most > 0.0f && most < INFINITY ? ilogbf(most) - 14 : most > 0.0f ? 0 : kNoPower;
      if (power != kNoPower) h = ldexpf(h, -power);
      if (stored && u == 0) w.power[pair * slices + slice] = power;
    }
    if (stored) ((T*)w.hidden)[pair * p.hidden + 16 * slice + u] = (T)h;
  }
}

// What comes out of an expert: 16 channels per workgroup, a quarter of the hidden values per wave.
template <class T, int NT>
__global__ __launch_bounds__(256) void k_expert_out(ExpertParams p, ExpertParts w, int groups) {
  __shared__ int32_t list[16 * NT];
  __shared__ int counts[4];
  __shared__ f32x4 partial[4][NT][64];
  __shared__ int powers[16 * NT];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15;
  int id = xcd_number();
  const int group = id % groups, blocks = (p.channels + 15) / 16, slices = slices_of(p);
  id /= groups;
  const int block = id % blocks, e = id / blocks;
  const int n = pairs_of(p, w.chosen, e, group * 16 * NT, 16 * NT, list, counts);
  if (n == 0) return;
  constexpr bool kPowers = __is_same(T, f16);
  if (kPowers) {
    const int at = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (16 * i + at >= n) break;
      const int16_t* const power = w.power + (int64_t)list[16 * i + at] * slices;
      int most = kNoPower;
      for (int s = threadIdx.x & 15; s < slices; s += 16) most = max(most, (int)power[s]);
#pragma unroll
      for (int d = 1; d < 16; d *= 2) most = max(most, __shfl_xor(most, d));
      if ((threadIdx.x & 15) == 0) powers[16 * i + at] = most;
    }
    __syncthreads();
  }
  const T* vectors[NT];
  const int16_t* power[NT];
  int row_power[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int at = 16 * i + col < n ? 16 * i + col : 0;
    const int64_t pair = list[at];
    vectors[i] = (const T*)w.hidden + pair * p.hidden;
    power[i] = w.power + pair * slices;
    row_power[i] = kPowers ? powers[at] : 0;
  }
  const T* const rows[1] = {(const T*)p.w_out + ((int64_t)e * p.channels + min(16 * block + col, p.channels - 1)) * p.hidden};
  const int steps = (p.hidden + 63) / 64;
  f32x4 acc[1][NT] = {};
  products<T, 1, NT, kPowers>(rows, vectors, power, row_power, steps * wave / 4, steps * (wave + 1) / 4, p.hidden, acc);
#pragma unroll
  for (int i = 0; i < NT; ++i) partial[wave][i][lane] = acc[0][i];
  __syncthreads();
  const int u = threadIdx.x & 15, at = threadIdx.x >> 4, from = (u >> 2) * 16 + at;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (16 * i + at >= n || 16 * block + u >= p.channels) break;
    const int64_t pair = list[16 * i + at];
    float y = (partial[0][i][from][u & 3] + partial[1][i][from][u & 3]) + (partial[2][i][from][u & 3] + partial[3][i][from][u & 3]);
    if (kPowers) y = powers[16 * i + at] == kNoPower ? y : ldexpf(y, powers[16 * i + at]);
    w.products[pair * p.channels + 16 * block + u] = w.weights[pair] * y;
  }
}

// The pairs that chose each expert, a workgroup per expert: a thread looks at 16 pairs side by side.
__global__ __launch_bounds__(256) void k_expert_lists(ExpertParams p, ExpertParts w) {
  __shared__ int counts[4];
  const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = p.tokens * p.top;
  int seen = 0;
  for (int at = 0; at < pairs; at += 4096) {
    const int first = at + 16 * threadIdx.x;
    uint32_t hits = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (first + i < pairs && w.chosen[first + i] == e) hits |= 1u << i;
    int before = __popc(hits);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(before, d);
      if (lane >= d) before += other;
    }
    if (lane == 63) counts[wave] = before;
    __syncthreads();
    int place = seen + before - __popc(hits);
    for (int n = 0; n < 4; ++n) {
      if (n < wave) place += counts[n];
      seen += counts[n];
    }
    for (; hits; hits &= hits - 1) w.list[(int64_t)e * p.tokens + place++] = first + __ffs(hits) - 1;
    __syncthreads();
  }
  if (threadIdx.x == 0) w.count[e] = seen;
}

// Either product for many tokens of an expert: a workgroup has 128 hidden values (IN: 128 rows of each of the two weights) or channels
// and up to 32 * NT of the expert's tokens, 32 rows per wave.  Weights go from memory into the registers that multiply them, as
// no other wave needs them; the tokens' values, which all waves need, through LDS, 64 at a time.
template <class T, bool IN, int NT>
__global__ __launch_bounds__(256, 2) void k_expert_tiles(ExpertParams p, ExpertParts w, int groups) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int RT = IN ? 2 : 1, kTile = 32 * NT * 128;
  constexpr bool kPowers = __is_same(T, f16);
  __shared__ __align__(16) char lds[2 * kTile];
  __shared__ int powers[32 * NT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int rows = IN ? p.hidden : p.channels, length = IN ? p.channels : p.hidden, blocks = (rows + 127) / 128, slices = slices_of(p);
  // the groups of the tokens behind the first, most often empty, come last
  const int per_group = blocks * p.experts, group = blockIdx.x / per_group;
  const int id = blockIdx.x % per_group, block = id % blocks, e = id / blocks;
  const int n = min(w.count[e] - group * 32 * NT, 32 * NT);
  if (n <= 0) return;
  const int32_t* const list = w.list + (int64_t)e * p.tokens + group * 32 * NT;

  // staging: this thread's 16 bytes of vectors r0 + 32 i
  const int r0 = threadIdx.x >> 3, ch = threadIdx.x & 7;
  const T* from[NT];
  const int16_t* power[NT];
  int row_power[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int64_t pair = list[min(r0 + 32 * i, n - 1)];
    from[i] = IN ? (const T*)p.x + pair / p.top * p.x_stride : (const T*)w.hidden + pair * p.hidden;
    power[i] = w.power + pair * slices;
    row_power[i] = 0;
    if (!IN && kPowers) {                            // the eight threads of a vector look for its largest power
      int most = kNoPower;
      for (int s = ch; s < slices; s += 8) most = max(most, (int)power[i][s]);
#pragma unroll
      for (int d = 1; d < 8; d *= 2) most = max(most, __shfl_xor(most, d));
      row_power[i] = most;
      if (ch == 0) powers[r0 + 32 * i] = most;
    }
  }
  const int row = 128 * block + 32 * wave;
  const int64_t first_row = (int64_t)e * (IN ? 2 * p.hidden : p.channels) + min(row + col, rows - 1);
  const T* weights[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) weights[r] = (const T*)(IN ? p.w_in : p.w_out) + (first_row + (int64_t)r * p.hidden) * length + 8 * half;

  struct Step {
    x8 a[RT][4];
    x8 b[NT];
    int16_t power[NT];
  };
  auto load = [&](int step, Step& s) {
    const int d0 = min(64 * step + 8 * ch, length - 8);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      s.b[i] = __builtin_bit_cast(x8, load16(from[i] + d0));
      if (!IN && kPowers) s.power[i] = power[i][d0 / kSlice];
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int k = 0; k < 4; ++k) s.a[r][k] = __builtin_bit_cast(x8, load16(weights[r] + min(64 * step + 16 * k, length - 8 - 8 * half)));
  };
  int koff[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) koff[k] = slot<8>(col, 2 * k + half);
  f32x16 acc[RT][NT] = {};
  const int steps = (length + 63) / 64;
  auto multiply = [&](int step, Step& s, Step& next) {
    char* const here = lds + (step & 1) * kTile;
    const bool whole = 64 * step + 64 <= length;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (!whole && 64 * step + 8 * ch >= length) s.b[i] = x8{};
      if (!IN && kPowers) s.b[i] *= (T)ldexpf(1.0f, max(s.power[i] - row_power[i], -40));
      *(x8*)(here + slot<8>(r0 + 32 * i, ch)) = s.b[i];
    }
    if (step + 1 < steps) load(step + 1, next);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!whole && 64 * step + 16 * k + 8 * half >= length)
#pragma unroll
        for (int r = 0; r < RT; ++r) s.a[r][k] = x8{};
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const x8 b = *(const x8*)(here + koff[k] + i * 32 * 128);
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r][i] = mfma32(s.a[r][k], b, acc[r][i]);
      }
    }
  };
  Step even, odd;
  load(0, even);
  for (int step = 0; step < steps; step += 2) {
    multiply(step, even, odd);
    if (step + 1 < steps) multiply(step + 1, odd, even);
  }

  // lane l has vector l % 32 and rows 8 * (i / 4) + 4 * half + i % 4
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (32 * i >= n) break;
    const bool live = 32 * i + col < n;
    const int64_t pair = list[min(32 * i + col, n - 1)];
    if (IN) {
      f32x16 h;
#pragma unroll
      for (int j = 0; j < 16; ++j) h[j] = acc[0][i][j] / (1.0f + expf(-acc[0][i][j])) * acc[RT - 1][i][j];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        int own = 0;
        if (kPowers) {
          float most = 0.0f, lower, upper;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (row + 16 * s + 8 * (j / 4) + 4 * half < rows) most = fmaxf(most, fabsf(h[8 * s + j]));
          both_halves(most, lower, upper);
          most = fmaxf(lower, upper);
          own = most > 0.0f && most < INFINITY ? ilogbf(most) - 14 : most > 0.0f ? 0 : kNoPower;
          if (live && half == 0 && row + 16 * s < rows) w.power[pair * slices + row / kSlice + s] = own;
          if (own == kNoPower) own = 0;
        }
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const int unit = row + 16 * s + 2 * j + 4 * half;
          x4 y;
#pragma unroll
          for (int d = 0; d < 4; ++d) y[d] = (T)(kPowers ? ldexpf(h[8 * s + j + d], -own) : h[8 * s + j + d]);
          if (live && unit < rows) *(x4*)((T*)w.hidden + pair * p.hidden + unit) = y;
        }
      }
    } else {
      float f = w.weights[pair];
      const int own = kPowers ? powers[min(32 * i + col, n - 1)] : 0;
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        const int channel = row + 2 * j + 4 * half;
        f32x4 y;
#pragma unroll
        for (int d = 0; d < 4; ++d) y[d] = f * (kPowers && own != kNoPower ? ldexpf(acc[0][i][j + d], own) : acc[0][i][j + d]);
        if (live && channel < rows) *(f32x4*)(w.products + pair * p.channels + channel) = y;
      }
    }
  }
}

// A token's experts in the order of their choice: 8 channels per thread.
template <class T>
__global__ __launch_bounds__(256) void k_expert_sum(ExpertParams p, ExpertParts w) {
  const int pieces = p.channels / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, t = id / pieces;
  if (t >= p.tokens) return;
  const int c = (int)(id % pieces) * 8;
  float sum[8] = {};
  if (!p.mask || p.mask[t])
    for (int i = 0; i < p.top; ++i) {
      const float* const from = w.products + (t * p.top + i) * p.channels + c;
      const f32x4 a = *(const f32x4*)from, b = *(const f32x4*)(from + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += a[e], sum[4 + e] += b[e];
    }
  *(typename Vec<T>::x8*)((T*)p.out + t * p.out_stride + c) = round8<T>(sum);
}

template <class T, int NT>
hipError_t launch_tiles(const ExpertParams& p, void** args, hipStream_t stream) {
  int groups = (p.tokens + 32 * NT - 1) / (32 * NT);
  void* all[] = {args[0], args[1], &groups};
  hipError_t e = launch_kernel((const void*)k_expert_lists, p.experts, 256, args, stream);
  if (e == hipSuccess) e = launch_kernel((const void*)k_expert_tiles<T, true, NT>, (int64_t)p.experts * ((p.hidden + 127) / 128) * groups, 256, all, stream);
  if (e == hipSuccess) e = launch_kernel((const void*)k_expert_tiles<T, false, NT>, (int64_t)p.experts * ((p.channels + 127) / 128) * groups, 256, all, stream);
  return e;
}
template <class T>
hipError_t launch_few(const ExpertParams& p, void** args, hipStream_t stream) {
  int groups = 1;
  void* all[] = {args[0], args[1], &groups};
  hipError_t e = launch_kernel((const void*)k_expert_in<T, 1>, (int64_t)p.experts * slices_of(p), 256, all, stream);
  if (e == hipSuccess) e = launch_kernel((const void*)k_expert_out<T, 1>, (int64_t)p.experts * ((p.channels + 15) / 16), 256, all, stream);
  return e;
}
template <class T>
hipError_t launch_of(const ExpertParams& p, hipStream_t stream) {
  ExpertParams params = p;
  ExpertParts parts = parts_of(p);
  void* args[] = {&params, &parts};
  hipError_t e = launch_kernel((const void*)k_expert_route<T>, p.tokens, 256, args, stream);
  const int64_t each = (int64_t)p.tokens * p.top / p.experts;          // tokens of an expert, on average
  if (e == hipSuccess)
    e = p.tokens <= 16 ? launch_few<T>(p, args, stream) : each <= 24 ? launch_tiles<T, 1>(p, args, stream)
      : each <= 48 ? launch_tiles<T, 2>(p, args, stream) : launch_tiles<T, 4>(p, args, stream);
  if (e == hipSuccess) e = launch_kernel((const void*)k_expert_sum<T>, ((int64_t)p.tokens * (p.channels / 8) + 255) / 256, 256, args, stream);
  return e;
}
}  // namespace

size_t expert_workspace(const ExpertParams& p) {
  ExpertParams q = p;
  q.parts = nullptr;
  return parts_of(q).bytes;
}

hipError_t launch(const ExpertParams& p, hipStream_t stream) {
  return p.dtype == HS_F16 ? launch_of<f16>(p, stream) : launch_of<bf16>(p, stream);
}

}  // namespace hs
