// hs_expert_layer: a router and the experts' networks for a few tokens.
#include "hs_track_device.h"

#include <math.h>

#include <algorithm>

namespace hs {
namespace {

// The choice (k_expert_route), the hidden layer, what comes out of each expert, and the sum over a token's experts (k_expert_sum):
// up to 64 tokens by strips of 16 weight rows (k_expert_in, k_expert_out), a frame's 16 with the choice and the hidden layer in one
// launch (k_expert_frame); more by tiles of 64 (k_expert_tiles).
// Bound by the weights' way from memory: 128 tokens, 4 of 32 experts of 1024 x 2048, take 95 us, of them 50 and 33 for the products' 268 and 134
// MB (5.4 and 4.0 TB/s); a frame's 8 tokens 22 us for 33 MB, a chain of three launches; 1024 tokens 193 us, in which staging tokens, products and
// weights hide each other only in part (each left out saves 20 to 40).
// A product has a weight's rows as its first and tokens as its second operand, so that few tokens waste little of the matrix pipe, and
// every weight that is needed is read once, straight from memory into the registers that multiply it.
// Hidden values enter the second product rounded to 16 bits: a second part would double their way through memory and that product's work.
// It counts like the output's own rounding: an rms error of 2.3e-3 in bf16, where the rounded output alone has 1.65e-3, 3.0e-4 in fp16 and 2.1e-4.
//
// fp16: hidden values are kept divided by a power of two, one for each token and 16 of them, which lets them neither overflow nor lose
// bits; the second product takes all of a token's divided by their largest.
// Strips up to here: 3 of 6 experts of 520 x 1336 take 22.7 us for 24 tokens and 23.9 for 48, in tiles 25.3 and 26.2.  With more experts strips are
// the slower ones: 64 tokens, 4 of 32 of 1024 x 2048, 123 us and 95, 2 of 16 of 512 x 1024 28.6 and 26.9.
constexpr int kFewTokens = 64;
constexpr int kSlice = 16;
constexpr int kNoPower = -1000;                      // of a slice of zeros

struct ExpertParts {            // the workspace
  int32_t* chosen;              // [tokens][top]
  float* weights;               // [tokens][top]
  void* hidden;                 // [tokens][top][hidden], in the inputs' type
  int16_t* power;               // [tokens][top][power_pitch()], fp16
  float* products;              // [tokens][top][channels]
  size_t bytes;
};
__host__ __device__ inline int slices_of(const ExpertParams& p) { return (p.hidden + kSlice - 1) / kSlice; }
__host__ __device__ inline int power_pitch(const ExpertParams& p) { return (slices_of(p) + 7) / 8 * 8; }      // 16-byte pieces
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
  w.power = (int16_t*)take(p.dtype == HS_F16 ? pairs * power_pitch(p) * 2 : 0);
  w.products = (float*)take(pairs * p.channels * 4);
  w.bytes = at;
  return w;
}

// Scores as whole numbers in their order, those of NaN below all others.
__device__ __forceinline__ uint64_t rank_of(double x) {
  if (x != x) return 0;
  const uint64_t bits = __builtin_bit_cast(uint64_t, x == 0.0 ? 0.0 : x);
  return bits >> 63 ? ~bits : bits | 1ull << 63;
}

__device__ __forceinline__ double score_of(uint64_t rank) {
  return rank == 0 ? __builtin_nan("") : __builtin_bit_cast(double, rank >> 63 ? rank & ~(1ull << 63) : ~rank);
}

// A token's choice by one wave, from the scores' ranks in LDS: an expert's place is the number of experts before it.
__device__ __forceinline__ void choose(const ExpertParams& p, const uint64_t* ranks, int32_t* chosen) {
  const int lane = threadIdx.x & 63;
  for (int e0 = 0; e0 < p.experts; e0 += 64) {
    const int e = e0 + lane;
    const uint64_t own = e < p.experts ? ranks[e] : 0;
    int place = 0;
    for (int j0 = 0; j0 < p.experts; j0 += 64) {
      const uint64_t theirs = j0 + lane < p.experts ? ranks[j0 + lane] : 0;
      const int n = min(64, p.experts - j0);
      for (int j = 0; j < n; ++j) {
        const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(theirs >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)theirs, j);
        place += other > own || (other == own && j0 + j < e);
      }
    }
    if (e < p.experts && place < p.top) chosen[place] = e;
  }
  wave_order();
}

// The chosen experts of token t, in LDS, and their weights to memory.
__device__ __forceinline__ void publish(const ExpertParams& p, const ExpertParts& w, int t, const uint64_t* ranks, const int32_t* chosen) {
  const int lane = threadIdx.x & 63;
  const int e = chosen[lane < p.top ? lane : 0];
  const double most = score_of(ranks[chosen[0]]), own = lane < p.top ? exp(score_of(ranks[e]) - most) : 0.0;
  double total = own;
  if (!p.renormalise) {
    total = 0.0;
    for (int i = lane; i < p.experts; i += 64) total += exp(score_of(ranks[i]) - most);
  }
  const int sharers = p.renormalise ? HS_MAX_TOP : 64;
  for (int d = 1; d < sharers; d *= 2) total += __shfl_xor(total, d);
  if (lane >= p.top) return;
  const float weight = (float)(own / total);
  w.chosen[t * p.top + lane] = e;
  w.weights[t * p.top + lane] = weight;
  if (p.chosen) p.chosen[t * p.top + lane] = e;
  if (p.weights) p.weights[t * p.top + lane] = weight;
}

__device__ __forceinline__ void publish_none(const ExpertParams& p, const ExpertParts& w, int t) {
  const int lane = threadIdx.x & 63;
  if (lane >= p.top) return;
  w.chosen[t * p.top + lane] = -1;
  w.weights[t * p.top + lane] = 0.0f;
  if (p.chosen) p.chosen[t * p.top + lane] = -1;
  if (p.weights) p.weights[t * p.top + lane] = 0.0f;
}

// A workgroup per token: scores in 64 bits.  A wave has a quarter of the experts, eight at a time, a lane 8 of every 512 channels;
// the lanes' sums of the eight are joined together, half as many with every step (1024 tokens on 32 experts of 1024 channels: 13 us).
template <class T>
__global__ __launch_bounds__(256) void k_expert_route(ExpertParams p, ExpertParts w) {
  typedef typename Vec<T>::x8 x8;
  __shared__ uint64_t ranks[HS_MAX_EXPERTS];
  __shared__ int32_t chosen[HS_MAX_TOP];
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool here = !p.mask || p.mask[t];
  if (here) {
    const T* const x = (const T*)p.x + t * p.x_stride;
    constexpr int kAtOnce = 8;
    for (int e0 = kAtOnce * wave; e0 < p.experts; e0 += 4 * kAtOnce) {
      double sum[kAtOnce] = {};
      for (int c = 8 * lane; c < p.channels; c += 512) {
        const x8 a = __builtin_bit_cast(x8, load16(x + c));
        x8 r[kAtOnce];
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) r[n] = __builtin_bit_cast(x8, load16((const T*)p.router + (int64_t)min(e0 + n, p.experts - 1) * p.channels + c));
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[n] = fma((double)(float)a[i], (double)(float)r[n][i], sum[n]);
      }
#pragma unroll
      for (int half = kAtOnce / 2; half > 0; half /= 2) {     // lane bits 2, 1, 0: which of the eight a lane goes on with
        const bool upper = lane & half;
#pragma unroll
        for (int n = 0; n < half; ++n) {
          const double mine = upper ? sum[n + half] : sum[n], theirs = upper ? sum[n] : sum[n + half];
          sum[n] = mine + __shfl_xor(theirs, half);
        }
      }
#pragma unroll
      for (int d = kAtOnce; d < 64; d *= 2) sum[0] += __shfl_xor(sum[0], d);
      if (lane < kAtOnce && e0 + lane < p.experts) ranks[e0 + lane] = rank_of(sum[0]);
    }
  }
  __syncthreads();
  if (wave > 0) return;
  if (here) {
    choose(p, ranks, chosen);
    publish(p, w, t, ranks, chosen);
  } else {
    publish_none(p, w, t);
  }
}

// The same for up to 16 tokens and kFusedExperts experts, in a workgroup of 16 waves that goes on with the result, by matrix products in 64
// bits: a wave has 16 experts and every 4th to 16th 32 channels, then a token.  The choice is left in LDS.
constexpr int kFusedExperts = 64;
typedef double f64x4 __attribute__((ext_vector_type(4)));
struct RouteLds {
  double part[16 * 16 * 16];                         // [share of the channels][token][expert]
  uint64_t ranks[16][kFusedExperts];
  int32_t chosen[16][HS_MAX_TOP];
  int8_t place[kFusedExperts][16];                   // where in a token's choice the expert is, or -1
};
template <class T>
__device__ __forceinline__ void route_here(const ExpertParams& p, RouteLds& lds) {
  typedef typename Vec<T>::x8 x8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, g = lane >> 4;
  const int tiles = p.experts <= 16 ? 1 : p.experts <= 32 ? 2 : 4, shares = 16 / tiles, share = wave / tiles, e0 = 16 * (wave % tiles);
  ((int32_t*)lds.place)[threadIdx.x & 255] = -1;
  const T* const x = (const T*)p.x + min(row, p.tokens - 1) * p.x_stride;
  const T* const r = (const T*)p.router + (int64_t)min(e0 + row, p.experts - 1) * p.channels;
  f64x4 sum = {};
  for (int c = 32 * share; c < p.channels; c += 32 * shares) {
    const int c0 = min(c + 8 * g, p.channels - 8);
    x8 a = __builtin_bit_cast(x8, load16(x + c0)), b = __builtin_bit_cast(x8, load16(r + c0));
    if (c + 8 * g >= p.channels) a = b = x8{};
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)a[i], (double)(float)b[i], sum, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) lds.part[(share * 16 + g + 4 * i) * 16 * tiles + e0 + row] = sum[i];   // (row g + 4 i of the result, in 64 bits)
  __syncthreads();
  const int t = wave;
  if (t < p.tokens && (!p.mask || p.mask[t])) {
    if (lane < p.experts) {
      double score = 0.0;
      for (int n = 0; n < shares; ++n) score += lds.part[(n * 16 + t) * 16 * tiles + lane];
      lds.ranks[t][lane] = rank_of(score);
    }
    wave_order();
    choose(p, lds.ranks[t], lds.chosen[t]);
    if (lane < p.top) lds.place[lds.chosen[t][lane]][t] = lane;
  }
  __syncthreads();
}

// ---- few tokens: strips of 16 weight rows

// 64 values of each of RT * 16 weight rows and NT * 16 vectors: a lane has 16 values side by side of a row, so that four lanes read 128 bytes
// of it, and of a vector; the matrix pipe takes them in the same order.  Lane l has result [row 4 * (l / 16) + i][vector l % 16].
template <class T, int RT, int NT>
struct Strip {
  typedef typename Vec<T>::x8 x8;
  x8 a[RT][2], b[NT][2];
  static __device__ __forceinline__ int place(int step, int e, int length) {       // (what lies behind the row's end is left out below)
    return min(64 * step + 16 * (int)((threadIdx.x & 63) >> 4) + 8 * e, length - 8);
  }
  __device__ __forceinline__ void load_rows(const T* const (&rows)[RT], int step, int length) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int r = 0; r < RT; ++r) a[r][e] = __builtin_bit_cast(x8, load16(rows[r] + place(step, e, length)));
  }
  __device__ __forceinline__ void load_vectors(const T* const (&vectors)[NT], int step, int length) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int n = 0; n < NT; ++n) b[n][e] = __builtin_bit_cast(x8, load16(vectors[n] + place(step, e, length)));
  }
  __device__ __forceinline__ void multiply(int step, int length, f32x4 (&acc)[RT][NT]) {
    const int g = (threadIdx.x & 63) >> 4;
    if (64 * step + 64 > length) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (64 * step + 16 * g + 8 * e >= length) {
#pragma unroll
          for (int r = 0; r < RT; ++r) a[r][e] = x8{};
#pragma unroll
          for (int n = 0; n < NT; ++n) b[n][e] = x8{};
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = mfma16(a[r][e], b[n][e], acc[r][n]);
  }
};

// The strips first .. last - 1 of a wave.  The first two strips' rows are on their way (begin) while the caller finds out which
// vectors they are for (go on).
template <class T, int RT, int NT>
struct Strips {
  Strip<T, RT, NT> even, odd;
  int first, last, length;
  __device__ __forceinline__ void begin(const T* const (&rows)[RT]) {
    if (first < last) even.load_rows(rows, first, length);
    if (first + 1 < last) odd.load_rows(rows, first + 1, length);
  }
  // `prepare`: what is to be done to a strip's vectors before they are multiplied
  template <class F>
  __device__ __forceinline__ void go_on(const T* const (&rows)[RT], const T* const (&vectors)[NT], f32x4 (&acc)[RT][NT], F&& prepare) {
    if (first < last) even.load_vectors(vectors, first, length);
    for (int step = first; step < last; step += 2) {
      if (step + 1 < last) odd.load_vectors(vectors, step + 1, length);
      prepare(step, even);
      even.multiply(step, length, acc);
      if (step + 1 >= last) break;
      if (step + 2 < last) {
        even.load_rows(rows, step + 2, length);
        even.load_vectors(vectors, step + 2, length);
      }
      prepare(step + 1, odd);
      odd.multiply(step + 1, length, acc);
      if (step + 3 < last) odd.load_rows(rows, step + 3, length);
    }
  }
};

__device__ __forceinline__ int most_of(const int16_t* power, int first, int slices) {      // of eight powers
  const s16x8 eight = load16(power + first);
  int most = kNoPower;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (first + i < slices) most = max(most, (int)eight[i]);
  return most;
}

// Hidden values times 2^power, power <= 0, by two factors: fp16 has no 2^-25, and values times it that are normal ones keep their bits.
template <class T>
__device__ __forceinline__ void lower(typename Vec<T>::x8& values, int power) {
  const int whole = max(power, -40), half = whole / 2;               // (2^-40 of 2^15 rounds to zero)
  values *= (T)ldexpf(1.0f, half);
  values *= (T)ldexpf(1.0f, whole - half);
}

// The hidden value u of 16 from its gate and its other sum, for 16 threads side by side, which agree on the power of two that fp16 takes out.
template <class T>
__device__ __forceinline__ void store_hidden(const ExpertParams& p, const ExpertParts& w, int64_t pair, int slice, int u, bool there, float gate, float up) {
  float h = gate / (1.0f + expf(-gate)) * up;
  const bool stored = there && kSlice * slice + u < p.hidden;
  if (__is_same(T, f16)) {
    float most = stored ? fabsf(h) : 0.0f;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    const int power = most > 0.0f && most < INFINITY ? ilogbf(most) - 14 : most > 0.0f ? 0 : kNoPower;
    if (power != kNoPower) h = ldexpf(h, -power);
    if (stored && u == 0) w.power[pair * power_pitch(p) + slice] = power;
  }
  if (stored) ((T*)w.hidden)[pair * p.hidden + kSlice * slice + u] = (T)h;
}

// A frame's tokens, up to 16: the choice and the hidden layer.  A workgroup has an expert and 64 of its hidden values, 16 for every four waves,
// which take a quarter of the channels each; every workgroup works the choice out by itself, which costs less than a launch for it, and
// each token has a column of the products, whether it chose the expert or not.
// ahead: the first weights are asked for before it is known whether some token needs them.
template <class T>
__global__ __launch_bounds__(1024) void k_expert_frame(ExpertParams p, ExpertParts w, int ahead) {
  __shared__ union {
    RouteLds route;
    f32x4 partial[16][2][64];
  } lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, block = wave >> 2, quarter = wave & 3;
  const int id = xcd_number(), groups = (slices_of(p) + 3) / 4;
  const int slice = id % groups * 4 + block, e = id / groups;
  const T* const gate = (const T*)p.w_in + ((int64_t)e * 2 * p.hidden + min(kSlice * slice + col, p.hidden - 1)) * p.channels;
  const T* const rows[2] = {gate, gate + (int64_t)p.hidden * p.channels};
  const T* const vectors[1] = {(const T*)p.x + min(col, p.tokens - 1) * p.x_stride};     // (columns without a token are left out below)
  const int steps = (p.channels + 63) / 64;
  Strips<T, 2, 1> strips;
  strips.first = steps * quarter / 4;
  strips.last = steps * (quarter + 1) / 4;
  strips.length = p.channels;
  if (ahead) strips.begin(rows);
  route_here<T>(p, lds.route);
  if (slice == block) {                              // an expert's first workgroup: that of one without a token, if there is any, leaves the choice in memory
    const bool used = lane < p.experts && (*(const uint64_t*)lds.route.place[lane] & *(const uint64_t*)(lds.route.place[lane] + 8)) != ~0ull;
    const uint64_t unused = ~__ballot(used) & (p.experts < 64 ? (1ull << p.experts) - 1 : ~0ull);
    if (e == (unused ? __ffsll((unsigned long long)unused) - 1 : 0) && wave < p.tokens) {
      if (!p.mask || p.mask[wave]) publish(p, w, wave, lds.route.ranks[wave], lds.route.chosen[wave]);
      else publish_none(p, w, wave);
    }
  }
  const int u = threadIdx.x & 15, at = threadIdx.x >> 4 & 15, from = (u >> 2) * 16 + at;     // thread t finishes value t % 16 of token t / 16 % 16
  const int place = at < p.tokens ? lds.route.place[e][at] : -1;
  if (!__syncthreads_or(place >= 0)) return;
  if (!ahead) strips.begin(rows);
  f32x4 acc[2][1] = {};
  strips.go_on(rows, vectors, acc, [](int, Strip<T, 2, 1>&) {});
  lds.partial[wave][0][lane] = acc[0][0];
  lds.partial[wave][1][lane] = acc[1][0];
  __syncthreads();
  float y[2];
#pragma unroll
  for (int r = 0; r < 2; ++r)
    y[r] = (lds.partial[4 * block][r][from][u & 3] + lds.partial[4 * block + 1][r][from][u & 3])
         + (lds.partial[4 * block + 2][r][from][u & 3] + lds.partial[4 * block + 3][r][from][u & 3]);
  store_hidden<T>(p, w, (int64_t)at * p.top + place, slice, u, place >= 0, y[0], y[1]);
}

// The pairs (token, place) that chose expert e, in their order: those numbered first .. first + most - 1 of them are left in
// `list`; returns how many these are.  For a whole workgroup, a thread of which looks at 16 pairs side by side; `counts`: a place per wave.
__device__ __forceinline__ int pairs_of(const ExpertParams& p, const int32_t* chosen, int e, int first, int most, int32_t* list, int* counts) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, pairs = p.tokens * p.top;
  int seen = 0;
  for (int at = 0; at < pairs; at += 16 * blockDim.x) {
    const int own = at + 16 * threadIdx.x;
    uint32_t hits = 0;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      // (the array's room is a multiple of 256 bytes: what lies behind its end is read, and not looked at)
      const i32x4 c = own + i < pairs ? *(const i32x4*)(chosen + own + i) : i32x4{};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (own + i + j < pairs && c[j] == e) hits |= 1u << (i + j);
    }
    int before = __popc(hits);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(before, d);
      if (lane >= d) before += other;
    }
    if (lane == 63) counts[wave] = before;
    __syncthreads();
    int place = seen + before - __popc(hits);
    for (int n = 0; n < waves; ++n) {
      if (n < wave) place += counts[n];
      seen += counts[n];
    }
    for (; hits; hits &= hits - 1, ++place)
      if (place >= first && place < first + most) list[place - first] = own + __ffs(hits) - 1;
    __syncthreads();
  }
  return min(max(seen - first, 0), most);
}

// Hidden layer: a workgroup has an expert, 16 of its hidden values and up to 16 * NT of its tokens; its four waves take a quarter of the
// channels each.
template <class T, int NT>
__global__ __launch_bounds__(256) void k_expert_in(ExpertParams p, ExpertParts w, int ahead) {
  __shared__ int32_t list[16 * NT];
  __shared__ int counts[4];
  __shared__ f32x4 partial[4][2][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, slices = slices_of(p);
  const int slice = blockIdx.x % slices, e = blockIdx.x / slices;
  const T* const gate = (const T*)p.w_in + ((int64_t)e * 2 * p.hidden + min(kSlice * slice + col, p.hidden - 1)) * p.channels;
  const T* const rows[2] = {gate, gate + (int64_t)p.hidden * p.channels};
  const int steps = (p.channels + 63) / 64;
  Strips<T, 2, NT> strips;
  strips.first = steps * wave / 4;
  strips.last = steps * (wave + 1) / 4;
  strips.length = p.channels;
  for (int begin = 0; begin < p.tokens; begin += 16 * NT) {
  const bool early = ahead && begin == 0;
  if (early) strips.begin(rows);
  __syncthreads();                                   // the list's and the parts' last readers are done
  const int n = pairs_of(p, w.chosen, e, begin, 16 * NT, list, counts);
  if (n == 0) return;
  if (!early) strips.begin(rows);
  const T* vectors[NT];                              // (a place without a token has the first's, and is left out below)
#pragma unroll
  for (int i = 0; i < NT; ++i) vectors[i] = (const T*)p.x + (int64_t)(list[16 * i + col < n ? 16 * i + col : 0] / p.top) * p.x_stride;
  f32x4 acc[2][NT] = {};
  strips.go_on(rows, vectors, acc, [](int, Strip<T, 2, NT>&) {});
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int i = 0; i < NT; ++i) partial[wave][r][i][lane] = acc[r][i];
  __syncthreads();
  const int u = threadIdx.x & 15, at = threadIdx.x >> 4, from = (u >> 2) * 16 + at;   // thread t finishes value t % 16 of token t / 16
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (16 * i >= n) break;
    float y[2];
#pragma unroll
    for (int r = 0; r < 2; ++r)
      y[r] = (partial[0][r][i][from][u & 3] + partial[1][r][i][from][u & 3]) + (partial[2][r][i][from][u & 3] + partial[3][r][i][from][u & 3]);
    store_hidden<T>(p, w, list[min(16 * i + at, n - 1)], slice, u, 16 * i + at < n, y[0], y[1]);
  }
  if (n < 16 * NT) return;
  }
}

// What comes out of an expert: 16 channels per workgroup, a quarter of the hidden values per wave.
template <class T, int NT>
__global__ __launch_bounds__(256) void k_expert_out(ExpertParams p, ExpertParts w, int ahead) {
  constexpr bool kPowers = __is_same(T, f16);
  __shared__ int32_t list[16 * NT];
  __shared__ int counts[4], powers[16 * NT];
  __shared__ f32x4 partial[4][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, slices = slices_of(p);
  const int blocks = (p.channels + 15) / 16, block = blockIdx.x % blocks, e = blockIdx.x / blocks;
  const T* const rows[1] = {(const T*)p.w_out + ((int64_t)e * p.channels + min(16 * block + col, p.channels - 1)) * p.hidden};
  const int steps = (p.hidden + 63) / 64;
  Strips<T, 1, NT> strips;
  strips.first = steps * wave / 4;
  strips.last = steps * (wave + 1) / 4;
  strips.length = p.hidden;
  for (int begin = 0; begin < p.tokens; begin += 16 * NT) {
  const bool early = ahead && begin == 0;
  if (early) strips.begin(rows);
  __syncthreads();                                   // the list's and the parts' last readers are done
  const int n = pairs_of(p, w.chosen, e, begin, 16 * NT, list, counts);
  if (n == 0) return;
  if (!early) strips.begin(rows);
  const int u = threadIdx.x & 15, at = threadIdx.x >> 4, from = (u >> 2) * 16 + at;
  if (kPowers) {                                     // a token's largest power, by 16 threads
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (16 * i + at >= n) break;
      const int16_t* const power = w.power + (int64_t)list[16 * i + at] * power_pitch(p);
      int most = kNoPower;
      for (int s = 8 * u; s < slices; s += 128) most = max(most, most_of(power, s, slices));
#pragma unroll
      for (int d = 1; d < 16; d *= 2) most = max(most, __shfl_xor(most, d));
      if (u == 0) powers[16 * i + at] = most;
    }
    __syncthreads();
  }
  const T* vectors[NT];
  const int16_t* power[NT];
  int row_power[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int place = 16 * i + col < n ? 16 * i + col : 0;
    const int64_t pair = list[place];
    vectors[i] = (const T*)w.hidden + pair * p.hidden;
    power[i] = w.power + pair * power_pitch(p);
    row_power[i] = kPowers ? powers[place] : 0;
  }
  f32x4 acc[1][NT] = {};
  strips.go_on(rows, vectors, acc, [&](int step, Strip<T, 1, NT>& strip) {
    if (!kPowers) return;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int down = power[i][min(4 * step + (lane >> 4), slices - 1)] - row_power[i];
      lower<T>(strip.b[i][0], down);
      lower<T>(strip.b[i][1], down);
    }
  });
#pragma unroll
  for (int i = 0; i < NT; ++i) partial[wave][i][lane] = acc[0][i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (16 * i + at >= n || 16 * block + u >= p.channels) break;
    const int64_t pair = list[16 * i + at];
    float y = (partial[0][i][from][u & 3] + partial[1][i][from][u & 3]) + (partial[2][i][from][u & 3] + partial[3][i][from][u & 3]);
    if (kPowers && powers[16 * i + at] != kNoPower) y = ldexpf(y, powers[16 * i + at]);
    w.products[pair * p.channels + 16 * block + u] = w.weights[pair] * y;
  }
  if (n < 16 * NT) return;
  }
}

// ---- more tokens: tiles of 64 weight rows

// Either product for many tokens of an expert: a workgroup has 64 hidden values (IN: the rows of both weights) or channels and up to
// 16 * NT of the expert's tokens, a wave 16 of the rows.  Weights go from memory into the registers that multiply them, as no
// other wave needs them; the tokens' values, which all waves need, through LDS, 64 at a time.  Bound by the weights' way from
// memory: AHEAD steps of loads are on their way.
// (More tokens than that are taken in turn.)
// ahead: the first weights are asked for before it is known whether some token needs them.
template <class T, bool IN, int NT, int AHEAD>
__global__ __launch_bounds__(256, 2) void k_expert_tiles(ExpertParams p, ExpertParts w, int ahead) {
  typedef typename Vec<T>::x8 x8;
  typedef typename Vec<T>::x4 x4;
  constexpr int RT = IN ? 2 : 1, kVectors = 16 * NT, kTile = kVectors * 128, NB = (kVectors + 31) / 32;
  constexpr bool kPowers = __is_same(T, f16);
  __shared__ __align__(16) char lds[2 * kTile];
  __shared__ int powers[kVectors], counts[4];
  __shared__ int32_t list[kVectors];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const int rows = IN ? p.hidden : p.channels, length = IN ? p.channels : p.hidden, blocks = (rows + 63) / 64, slices = slices_of(p);
  const int steps = (length + 63) / 64;
  const int block = blockIdx.x % blocks, e = blockIdx.x / blocks;

  const int row = 64 * block + 16 * wave;
  const int64_t first_row = (int64_t)e * (IN ? 2 * p.hidden : p.channels) + min(row + col, rows - 1);
  const T* weights[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) weights[r] = (const T*)(IN ? p.w_in : p.w_out) + (first_row + (int64_t)r * p.hidden) * length;
  struct Step {
    x8 a[RT][2];
    x8 b[NB];
    int16_t power[NB];
  };
  auto load_weights = [&](int step, Step& s) {       // a lane has 16 values side by side: four lanes read 128 bytes of a row
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int k = 0; k < 2; ++k) s.a[r][k] = __builtin_bit_cast(x8, load16(weights[r] + min(64 * step + 16 * g + 8 * k, length - 8)));
  };
  for (int begin = 0; begin < p.tokens; begin += kVectors) {
  Step ring[AHEAD + 1];
  const bool early = ahead && begin == 0;
  if (early)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load_weights(min(i, steps - 1), ring[i]);
  __syncthreads();                                   // the list's and LDS's last readers are done
  const int n = pairs_of(p, w.chosen, e, begin, kVectors, list, counts);
  if (n == 0) return;
  if (!early)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load_weights(min(i, steps - 1), ring[i]);

  // staging: this thread's 16 bytes of vectors r0 + 32 i
  const int r0 = threadIdx.x >> 3, ch = threadIdx.x & 7;
  const T* from[NB];
  const int16_t* power[NB];
  int row_power[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int64_t pair = list[min(r0 + 32 * i, n - 1)];
    from[i] = IN ? (const T*)p.x + pair / p.top * p.x_stride : (const T*)w.hidden + pair * p.hidden;
    power[i] = w.power + pair * power_pitch(p);
    row_power[i] = 0;
    if (!IN && kPowers) {                            // the eight threads of a vector look for its largest power
      int most = kNoPower;
      for (int s = 8 * ch; s < slices; s += 64) most = max(most, most_of(power[i], s, slices));
#pragma unroll
      for (int d = 1; d < 8; d *= 2) most = max(most, __shfl_xor(most, d));
      row_power[i] = most;
      if (ch == 0 && r0 + 32 * i < kVectors) powers[r0 + 32 * i] = most;
    }
  }
  auto load_vectors = [&](int step, Step& s) {
    const int d0 = min(64 * step + 8 * ch, length - 8);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      s.b[i] = __builtin_bit_cast(x8, load16(from[i] + d0));
      if (!IN && kPowers) s.power[i] = power[i][d0 / kSlice];
    }
  };
  int boff[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) boff[k] = slot<8>(col, 2 * g + k);
  f32x4 acc[RT][NT] = {};
  const int tiles = (n + 15) / 16;
  auto multiply = [&](int step, Step& s) {
    char* const here = lds + (step & 1) * kTile;
    const bool whole = 64 * step + 64 <= length;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if (!whole && 64 * step + 8 * ch >= length) s.b[i] = x8{};
      if (!IN && kPowers) lower<T>(s.b[i], s.power[i] - row_power[i]);
      if (kVectors % 32 == 0 || r0 + 32 * i < kVectors) *(x8*)(here + slot<8>(r0 + 32 * i, ch)) = s.b[i];
    }
    if (!whole)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (64 * step + 16 * g + 8 * k >= length)
#pragma unroll
          for (int r = 0; r < RT; ++r) s.a[r][k] = x8{};
    __syncthreads();
    // (Five tiles at a time, or all there are: a branch around each of them would have every one wait for its own reads.)
    constexpr int kRun = NT % 5 ? NT : 5;
#pragma unroll
    for (int i0 = 0; i0 < NT; i0 += kRun) {
      if (i0 >= tiles) break;
#pragma unroll
      for (int i = i0; i < i0 + kRun; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const x8 b = *(const x8*)(here + boff[k] + i * 16 * 128);
#pragma unroll
          for (int r = 0; r < RT; ++r) acc[r][i] = mfma16(s.a[r][k], b, acc[r][i]);
        }
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load_vectors(min(i, steps - 1), ring[i]);
  int step = 0;
  // (Loads that a branch may leave out would be waited for where it ends: only the last steps have branches.)
  for (; step + 2 * AHEAD < steps; step += AHEAD + 1)
#pragma unroll
    for (int i = 0; i <= AHEAD; ++i) {
      Step& next = ring[(i + AHEAD) % (AHEAD + 1)];
      load_weights(step + i + AHEAD, next);
      load_vectors(step + i + AHEAD, next);
      multiply(step + i, ring[i]);
    }
#pragma unroll
  for (int i = 0; i < 2 * AHEAD; ++i) {
    if (step + i >= steps) break;
    if (step + i + AHEAD < steps) {
      Step& next = ring[(i + AHEAD) % (AHEAD + 1)];
      load_weights(step + i + AHEAD, next);
      load_vectors(step + i + AHEAD, next);
    }
    multiply(step + i, ring[i % (AHEAD + 1)]);
  }

  // lane l has vector l % 16 and rows 4 * (l / 16) + i
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (i >= tiles) continue;
    const int place = 16 * i + col;
    const bool live = place < n && row + 4 * g < rows;
    const int64_t pair = list[min(place, n - 1)];
    if (IN) {
      f32x4 h;
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = acc[0][i][j] / (1.0f + expf(-acc[0][i][j])) * acc[RT - 1][i][j];
      if (kPowers) {
        float most = 0.0f;
        if (row + 4 * g < rows) most = fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(h[2]), fabsf(h[3])));
        most = column_max(most);
        const int own = most > 0.0f && most < INFINITY ? ilogbf(most) - 14 : most > 0.0f ? 0 : kNoPower;
        if (live && g == 0) w.power[pair * power_pitch(p) + row / kSlice] = own;
        if (own != kNoPower)
#pragma unroll
          for (int j = 0; j < 4; ++j) h[j] = ldexpf(h[j], -own);
      }
      if (live) *(x4*)((T*)w.hidden + pair * p.hidden + row + 4 * g) = round4<T>(h);
    } else {
      const float f = w.weights[pair];
      const int own = kPowers ? powers[min(place, n - 1)] : 0;
      f32x4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = f * (kPowers && own != kNoPower ? ldexpf(acc[0][i][j], own) : acc[0][i][j]);
      if (live) *(f32x4*)(w.products + pair * p.channels + row + 4 * g) = y;
    }
  }
  if (n < kVectors) return;
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
hipError_t launch_few(const ExpertParams& p, bool frame, void** args, hipStream_t stream) {
  const hipError_t e = frame ? launch_kernel((const void*)k_expert_frame<T>, (int64_t)p.experts * ((slices_of(p) + 3) / 4), 1024, args, stream)
                             : launch_kernel((const void*)k_expert_in<T, NT>, (int64_t)p.experts * slices_of(p), 256, args, stream);
  return e != hipSuccess ? e : launch_kernel((const void*)k_expert_out<T, NT>, (int64_t)p.experts * ((p.channels + 15) / 16), 256, args, stream);
}
template <class T, int NT, int AHEAD_IN, int AHEAD_OUT>
hipError_t launch_tiles(const ExpertParams& p, void** args, hipStream_t stream) {
  const hipError_t e = launch_kernel((const void*)k_expert_tiles<T, true, NT, AHEAD_IN>, (int64_t)p.experts * ((p.hidden + 63) / 64), 256, args, stream);
  return e != hipSuccess ? e : launch_kernel((const void*)k_expert_tiles<T, false, NT, AHEAD_OUT>, (int64_t)p.experts * ((p.channels + 63) / 64), 256, args, stream);
}
template <class T>
hipError_t launch_of(const ExpertParams& p, hipStream_t stream) {
  ExpertParams params = p;
  ExpertParts parts = parts_of(p);
  // Weights are asked for before it is known that they are needed where each expert has a token on average: 8 tokens, 2 of 16 of 512 x 1024,
  // 20.9 us, 21.3 without.  Of experts without a token they are read in vain: 2 tokens, 2 of 64 of 1024 x 1024, 59 and 41, 8 tokens 70 and 54;
  // of large ones with one token each too many are, by chance: 16 tokens, 2 of 32 of 1024 x 2048, 81.6 and 76.5.
  int ahead = (int64_t)p.tokens * p.top >= p.experts;
  void* args[] = {&params, &parts, &ahead};
  // In one launch where every workgroup, which works the choice out by itself, has a CU of its own: 8 tokens on 16 experts of 512 x 1024 20.9 us,
  // 25.4 with the choice in a launch of its own; on 64 experts, four workgroups per CU, 73 and 38.  And where the router is small enough, of
  // which every workgroup reads all: 16 experts of 1024 x 1024 29.1 and 32.0, of 2048 channels 53.8 and 51.6, of 3584 82.5 and 76.3;
  // 32 of 512 x 512 22.8 and 22.5, of 1024 channels 33.6 and 28.7; 64 of 256 x 256 21.9 and 24.5, of 512 channels 29.9 and 29.2, of 1024 44.3 and 37.8.
  const bool frame = p.tokens <= 16 && p.experts <= kFusedExperts && p.experts * ((slices_of(p) + 3) / 4) <= 256 && (p.experts + 15) / 16 * p.channels <= 2048;
  hipError_t e = hipSuccess;
  if (!frame) e = launch_kernel((const void*)k_expert_route<T>, p.tokens, 256, args, stream);
  if (e != hipSuccess) return e;
  // Tiles of 32, 64 or 160 tokens by an expert's tokens on average, which are less than a tile holds, as some experts have more.
  // 4 of 32 experts of 1024 x 2048: 20 tokens each 100, 102 and 137 us, 24 118, 104 and 138, 48 178, 139 and 151, 56 190, 151 and 155,
  // 64 209, 171 and 162, 128 353, 255 and 226.
  const int64_t each = (int64_t)p.tokens * p.top / p.experts;
  if (p.tokens <= kFewTokens) e = p.tokens <= 16 ? launch_few<T, 1>(p, frame, args, stream) : launch_few<T, 2>(p, false, args, stream);
  else e = each <= 20 ? launch_tiles<T, 2, 3, 4>(p, args, stream) : each <= 48 ? launch_tiles<T, 4, 3, 3>(p, args, stream) : launch_tiles<T, 10, 2, 2>(p, args, stream);
  return e != hipSuccess ? e : launch_kernel((const void*)k_expert_sum<T>, ((int64_t)p.tokens * (p.channels / 8) + 255) / 256, 256, args, stream);
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
