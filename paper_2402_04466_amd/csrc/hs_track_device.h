// Device helpers of the track decoder's kernels: the two 16-bit types and their vectors.
#pragma once

#include "hs_track.h"

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

template <class T>
__device__ __forceinline__ const T* at(const Heads& h, int64_t batch, int64_t token, int64_t head) {
  return (const T*)h.p + batch * h.batch + token * h.token + head * h.head;
}
template <class T>
__device__ __forceinline__ T* at_out(const Heads& h, int64_t batch, int64_t token, int64_t head) {
  return (T*)h.p + batch * h.batch + token * h.token + head * h.head;
}

// A sequence's length as the caller gives it, taken into its range.
__device__ __forceinline__ int length_of(const int32_t* lengths, int batch, int longest) {
  return lengths ? min(max(lengths[batch], 0), longest) : longest;
}

inline hipError_t launch_kernel(const void* func, int64_t workgroups, unsigned threads, void** args, hipStream_t stream) {
  if (workgroups > (int64_t)(0xffffffffu / threads)) return hipErrorInvalidConfiguration;
  return hipLaunchKernel(func, dim3((unsigned)workgroups), dim3(threads), args, 0, stream);
}

}  // namespace hs
