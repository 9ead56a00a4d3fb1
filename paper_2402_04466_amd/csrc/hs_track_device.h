// Device helpers of the track decoder's kernels: the two 16-bit types and their vectors.
#pragma once

#include "hs_track.h"

#include <math.h>

namespace hs {

typedef __bf16 bf16;

template <class T> struct Vec;
template <> struct Vec<f16> {
  typedef f16 x4 __attribute__((ext_vector_type(4)));
  typedef f16 x8 __attribute__((ext_vector_type(8)));
};
template <> struct Vec<bf16> {
  typedef bf16 x4 __attribute__((ext_vector_type(4)));
  typedef bf16 x8 __attribute__((ext_vector_type(8)));
};
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// D[32][32] += A[32][16] B[16][32].  Lane l has A[l % 32][8 * (l / 32) + i], B[8 * (l / 32) + i][l % 32], i < 8, and
// D[8 * (i / 4) + 4 * (l / 32) + i % 4][l % 32], i < 16.
__device__ __forceinline__ f32x16 mfma32(Vec<f16>::x8 a, Vec<f16>::x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(Vec<bf16>::x8 a, Vec<bf16>::x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// D[16][16] += A[16][32] B[32][16].  Lane l has A[l % 16][8 * (l / 16) + i], B[8 * (l / 16) + i][l % 16], i < 8, and
// D[4 * (l / 16) + i][l % 16], i < 4.
__device__ __forceinline__ f32x4 mfma16(Vec<f16>::x8 a, Vec<f16>::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(Vec<bf16>::x8 a, Vec<bf16>::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A tile of 16-bit values in LDS, CH 16-byte chunks per row (8 or 16): chunk c of a row lies at c ^ swizzle(row).  16 rows' same
// chunk (an operand read along the rows), and two neighbouring chunks of rows 0 .. 3 and of 4 .. 7 or 8 .. 11
// behind them (transposed reads), then cover all banks once.
template <int CH>
__device__ __forceinline__ int swizzle(int row) {
  return (CH == 16 ? (row & 3) << 2 : (row >> 1 & 1) << 2) | ((row >> 2 ^ row >> 3) & 1) << 1 | (row >> 3 & 1);
}
template <int CH>   // byte offset of chunk c of a row
__device__ __forceinline__ int slot(int row, int c) {
  return (row * CH + (c ^ swizzle<CH>(row))) * 16;
}

// Workgroup i runs on XCD i % 8; this numbers the workgroups so that consecutive numbers share an XCD and its L2.
__device__ __forceinline__ int xcd_number() {
  const int total = gridDim.x, x = blockIdx.x % 8;
  return x * (total / 8) + min(x, total % 8) + blockIdx.x / 8;
}

// Transposed read from LDS: of each 16 lanes, lane l gives the address of 4 values of row l / 4, columns 4 * (l % 4) .. + 3,
// and receives column l of the four rows.
__device__ __forceinline__ s16x4 read_transposed(const char* lds) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)lds);
}
template <class T>
__device__ __forceinline__ typename Vec<T>::x8 join8(s16x4 a, s16x4 b) {
  return __builtin_bit_cast(typename Vec<T>::x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Eight sums, each rounded once.  (The conversion of a whole vector, not of its elements: that takes pairs.)
template <class T>
__device__ __forceinline__ typename Vec<T>::x8 round8(const float* x) {
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  const f32x8 v = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
  return __builtin_convertvector(v, typename Vec<T>::x8);
}
template <class T>
__device__ __forceinline__ typename Vec<T>::x4 round4(f32x4 v) { return __builtin_convertvector(v, typename Vec<T>::x4); }

// The value of lane l ^ 32 is among the two; both halves get both.
__device__ __forceinline__ void both_halves(float x, float& lower, float& upper) {
  const unsigned bits = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
  const unsigned r0 = r[0], r1 = r[1];   // (a bit cast of an element itself gives element 0)
  lower = __builtin_bit_cast(float, r0);
  upper = __builtin_bit_cast(float, r1);
}

// The largest of lanes l, l ^ 16, l ^ 32 and l ^ 48 (NaN is left out), in each of them.
__device__ __forceinline__ float column_max(float x) {
  const unsigned bits = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
  const unsigned r0 = r[0], r1 = r[1];
  x = fmaxf(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
  float lower, upper;
  both_halves(x, lower, upper);
  return fmaxf(lower, upper);
}

template <int CONTROL>
__device__ __forceinline__ float moved(float x) {   // from another lane of the row of 16
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}

template <class T>
__device__ __forceinline__ const T* at(const Heads& h, int64_t batch, int64_t token, int64_t head) {
  return (const T*)h.p + batch * h.batch + token * h.token + head * h.head;
}
template <class T>
__device__ __forceinline__ T* at_out(const Heads& h, int64_t batch, int64_t token, int64_t head) {
  return (T*)h.p + batch * h.batch + token * h.token + head * h.head;
}

// A 16-byte load that is known to be of global memory wherever its address comes from: one that might be of LDS (flat) is counted
// with the LDS accesses, so that a wait for those waits for memory.
__device__ __forceinline__ s16x8 load16(const void* from) {
  return *(const __attribute__((address_space(1))) s16x8*)from;
}

// A sequence's length as the caller gives it, taken into its range.  `batch` is the same for the whole wave, and so, said
// aloud, is the length: loops over it are the scalar unit's then.
__device__ __forceinline__ int length_of(const int32_t* lengths, int batch, int longest) {
  return __builtin_amdgcn_readfirstlane(lengths ? min(max(lengths[batch], 0), longest) : longest);
}

// The accesses of a wave to LDS before this come before those after it, whichever lane they are of.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---- softmax by tiles of keys, of the attentions
constexpr float kLog2e = 1.44269504088896340736f;
// A row's maximum is only raised, and what it has summed only rescaled, when the scores have grown by
// more than this many powers of two: weights then stay below 2^8, as exact as weights below 1.
constexpr float kSlack = 8.0f;
// fp16 weights are formed 2^7 times as large, below 2^15 then: those of up to 2^-21 of the largest keep all their bits, and
// what is lost of the others stays below 2^-32 of it.
template <class T> constexpr float kRaise = __is_same(T, f16) ? 7.0f : 0.0f;
// A row's maximum is at least this once it has seen a key, so that one whose scores are all minus infinity is told from one that sees none.
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2 = 0.69314718055994530942f;

// What is taken off scores times c: a maximum's, and a number where that is beyond fp32.
template <class T>
__device__ __forceinline__ float exponent_of(float m, float c) { return m == -INFINITY ? 0.0f : fmaxf(fmaf(m, c, -kRaise<T>), kLowest); }

// A softmax's sum is zero where no key is seen, which m = -INFINITY says, or where all scores are minus infinity, which leaves 0 / 0.
__device__ __forceinline__ float inverse_sum(float m, float l) { return m == -INFINITY ? 0.0f : 1.0f / l; }

__device__ __forceinline__ float positive_scale(float scale) { return scale == 0.0f ? 1.0f : fabsf(scale); }

// The order of the products before it and of the LDS reads that they take one each: two groups of reads, then each group's products
// before the reads of the one after next, so that none waits for a read that has only just been issued.
template <int GROUP, int GROUPS>
__device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, 2 * GROUP, 0);
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    __builtin_amdgcn_sched_group_barrier(0x8, GROUP, 0);
    if (g + 2 < GROUPS) __builtin_amdgcn_sched_group_barrier(0x100, GROUP, 0);
  }
}

inline hipError_t launch_kernel(const void* func, int64_t workgroups, unsigned threads, void** args, hipStream_t stream) {
  if (workgroups > (int64_t)(0xffffffffu / threads)) return hipErrorInvalidConfiguration;
  return hipLaunchKernel(func, dim3((unsigned)workgroups), dim3(threads), args, 0, stream);
}

}  // namespace hs
