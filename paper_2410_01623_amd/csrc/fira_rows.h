// What the kernels of the operators around the step share: eight neighbouring values of a row at a time, whatever their type and
// alignment, and sums over lanes.  gfx950 only.
#pragma once
#include "fira_device.h"

// Storage types as the kernels name them.
struct FiraStoredF32 { typedef float raw; };
struct FiraStoredBf16 { typedef bf16_raw raw; };

// W neighbouring values of a row, as many as make 16 bytes of the wider type that a kernel streams (8 where all is bf16, 4 with fp32; 1 for rows
// that are shorter): every load and store of a wavefront then covers whole lines, which fp32 in pieces of 32 bytes a lane does not (with those,
// streaming stores cost the embedding gradient of 131072 x 1024 in fp32 167 us instead of 144, and streaming loads the norm's gradient 94 instead of 80).
template <typename T, typename R = T>
constexpr int kWidth = sizeof(typename T::raw) == 4 || sizeof(typename R::raw) == 4 ? 4 : 8;
constexpr int kMostWidth = 8;

// Rows start at any element (odd widths, any leading dimension), so these are vectors with element alignment; the hardware
// takes such addresses.
typedef u32x2 __attribute__((aligned(2))) u32x2_a2;

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

// How W values of type T move: as one vector, or as two of fp32 where W is 8.
template <typename T, int W>
struct Moved;
template <> struct Moved<FiraStoredBf16, 8> { typedef u32x4 reg; typedef u32x4_a2 mem; };
template <> struct Moved<FiraStoredBf16, 4> { typedef u32x2 reg; typedef u32x2_a2 mem; };
template <> struct Moved<FiraStoredF32, 8> { typedef f32x4 reg; typedef f32x4_a4 mem; };
template <> struct Moved<FiraStoredF32, 4> { typedef f32x4 reg; typedef f32x4_a4 mem; };

// Values as they are stored: what is on its way is held like this, in half the registers where it is bf16.  load: one load (two for eight of fp32)
// without a branch, so that many stay on their way.  stream: the same for what is not needed again.
template <typename T, int W>
struct Raw {
  typedef typename Moved<T, W>::reg reg;
  typedef typename Moved<T, W>::mem mem;
  static constexpr bool F32 = sizeof(typename T::raw) == 4;
  static constexpr int N = F32 ? W / 4 : 1;
  reg a[N];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (F32) return a[i / 4][i % 4];
    else return __uint_as_float(i & 1 ? a[0][i / 2] & 0xffff0000u : a[0][i / 2] << 16);
  }
  __device__ __forceinline__ void load(const typename T::raw* p) {
#pragma unroll
    for (int k = 0; k < N; ++k) a[k] = *(gptr<const mem>)as_global(p + 4 * k);
  }
  __device__ __forceinline__ void stream(const typename T::raw* p) {
#pragma unroll
    for (int k = 0; k < N; ++k) a[k] = __builtin_nontemporal_load((gptr<const mem>)as_global(p + 4 * k));
  }
};
template <typename T>
struct Raw<T, 1> {
  float a;
  __device__ __forceinline__ float get(int) const { return a; }
  __device__ __forceinline__ void load(const typename T::raw* p) { a = load1<T>(p); }
  __device__ __forceinline__ void stream(const typename T::raw* p) { load(p); }
};
// STREAM: the result does not have to stay in the caches.
template <typename T, int W, bool STREAM = false>
__device__ __forceinline__ void store_w(typename T::raw* p, const float (&v)[W]) {
  if constexpr (W == 1) {
    store1<T>(p, v[0]);
  } else {
    typedef typename Moved<T, W>::reg reg;
    typedef typename Moved<T, W>::mem mem;
    constexpr bool F32 = sizeof(typename T::raw) == 4;
    constexpr int N = F32 ? W / 4 : 1;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      reg a;
      if constexpr (F32) {
        a = reg{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
      } else {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) a[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
      }
      if constexpr (STREAM) __builtin_nontemporal_store((mem)a, (gptr<mem>)as_global(p + 4 * k));
      else *(gptr<mem>)as_global(p + 4 * k) = a;
    }
  }
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
