// What the kernels of the operators around the step share: eight neighbouring values of a row at a time, whatever their type and
// alignment, and sums over lanes.  gfx950 only.
#pragma once
#include "fira_device.h"

// Storage types as the kernels name them.
struct FiraStoredF32 { typedef float raw; };
struct FiraStoredBf16 { typedef bf16_raw raw; };

constexpr int kVec = 8;   // values a lane takes at a time: 16 bytes of bf16, 32 of fp32

// Rows start at any element (odd widths, any leading dimension), so these are vectors with element alignment; the hardware
// takes such addresses.
template <typename T>
__device__ __forceinline__ float load1(const typename T::raw* p) {
  if constexpr (sizeof(typename T::raw) == 4) return *as_global(p);
  else return bf16_to_f32(*as_global(p));
}
template <typename T>
__device__ __forceinline__ void store1(typename T::raw* p, float x) {
  if constexpr (sizeof(typename T::raw) == 4) *as_global(p) = x;
  else *as_global(p) = f32_to_bf16(x);
}
template <typename T>
__device__ __forceinline__ void load8(const typename T::raw* p, float (&v)[kVec]) {
  if constexpr (sizeof(typename T::raw) == 4) {
    const f32x4 a = *(gptr<const f32x4_a4>)as_global(p), b = *(gptr<const f32x4_a4>)as_global(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
    const u32x4 a = *(gptr<const u32x4_a2>)as_global(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(a[i] << 16); v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
  }
}
template <typename T>
__device__ __forceinline__ void store8(typename T::raw* p, const float (&v)[kVec]) {
  if constexpr (sizeof(typename T::raw) == 4) {
    *(gptr<f32x4_a4>)as_global(p) = f32x4{v[0], v[1], v[2], v[3]};
    *(gptr<f32x4_a4>)as_global(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    *(gptr<u32x4_a2>)as_global(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
}
// The same for the n values of a row that are left, 0 <= n; what lies beyond is neither read nor written and counts as zero.
template <typename T>
__device__ __forceinline__ void load_some(const typename T::raw* p, long long n, float (&v)[kVec]) {
  if (n >= kVec) return load8<T>(p, v);
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = i < n ? load1<T>(p + i) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_some(typename T::raw* p, long long n, const float (&v)[kVec]) {
  if (n >= kVec) return store8<T>(p, v);
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (i < n) store1<T>(p + i, v[i]);
}

// Sum over the 64 lanes of a wavefront, in every lane.
template <typename F>
__device__ __forceinline__ F wave_sum(F x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}
// Sum over the workgroup's threads, in every thread, in an order that depends on their number only.  part: LDS, one value per wavefront.
template <typename F>
__device__ __forceinline__ F block_sum(F x, F* part) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  F s = part[0];
  for (unsigned w = 1; w < blockDim.x >> 6; ++w) s += part[w];
  return s;
}
