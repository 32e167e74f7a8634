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

// W neighbouring values (8, or 1 for rows shorter than 8) as they are stored: what is on its way is held like this, in half the
// registers where it is bf16.  One load each, without a branch, so that many stay on their way.
template <typename T, int W>
struct Raw;
template <>
struct Raw<FiraStoredF32, 8> {
  f32x4 a, b;
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void load(const float* p) { a = *(gptr<const f32x4_a4>)as_global(p); b = *(gptr<const f32x4_a4>)as_global(p + 4); }
};
template <>
struct Raw<FiraStoredBf16, 8> {
  u32x4 a;
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? a[i / 2] & 0xffff0000u : a[i / 2] << 16); }
  __device__ __forceinline__ void load(const bf16_raw* p) { a = *(gptr<const u32x4_a2>)as_global(p); }
};
template <typename T>
struct Raw<T, 1> {
  float a;
  __device__ __forceinline__ float get(int) const { return a; }
  __device__ __forceinline__ void load(const typename T::raw* p) { a = load1<T>(p); }
};
template <typename T, int W>
__device__ __forceinline__ void store_w(typename T::raw* p, const float (&v)[W]) {
  if constexpr (W == 8) store8<T>(p, v);
  else store1<T>(p, v[0]);
}

// A lane's W columns of rows that are `dim` >= W wide, by rights those from `c` on.  At the end of a row they start earlier, so that they are
// whole: the first `skip` of them are a neighbour's as well, who computes the same for them.  A lane beyond the end has none of its own.
template <int W>
struct Columns {
  long long at;
  int skip;
  bool any;
  __device__ __forceinline__ Columns(long long c, long long dim) : at(min(c, dim - W)), skip((int)(c - min(c, dim - W))), any(c < dim) {}
};

// Sum over each LANES neighbouring lanes, in all of them, between registers.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  if constexpr (LANES >= 64) x = add_xor<32>(x);
  if constexpr (LANES >= 32) x = add_xor<16>(x);
  if constexpr (LANES >= 16) x = add_xor<8>(x);
  return add_xor<1>(add_xor<2>(add_xor<4>(x)));
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
