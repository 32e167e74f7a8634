// The norm of a list of gradients taken together, and their scaling where it passes a limit.  gfx950 only.
#pragma once
#include "fira_rows.h"

// A piece of a gradient: rows of `cols` values.  The host cuts longer ones up so that all counts fit 32 bits.
struct FiraSpan {
  const void* g;
  void* out;
  int rows, cols;
  int ld, ld_out;
  int vecs;          // vectors of eight values per row, the last one of a row maybe shorter
  int tile0;         // first tile of this piece
};
constexpr int kSpans = 96;            // a launch's pieces travel as kernel arguments, of which there are 4 KB
constexpr int kClipTile = 2048;       // vectors of a tile
constexpr int kClipWorkgroups = 2048;
struct FiraSpans {
  FiraSpan s[kSpans];
  int count, tiles;
};

// Calls f(piece, row, column, values there) for this workgroup's vectors: tiles blockIdx.x, blockIdx.x + gridDim.x, ...
template <typename F>
__device__ __forceinline__ void for_each_vector(const FiraSpans& l, F f) {
  for (int tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
    int k = 0;
    while (k + 1 < l.count && l.s[k + 1].tile0 <= tile) ++k;
    const FiraSpan& s = l.s[k];
    const unsigned total = (unsigned)s.rows * (unsigned)s.vecs;
    const unsigned first = (unsigned)(tile - s.tile0) * kClipTile;
    for (unsigned i = first + threadIdx.x; i < first + kClipTile && i < total; i += blockDim.x) {
      const unsigned row = i / (unsigned)s.vecs, c = (i - row * (unsigned)s.vecs) * kVec;
      f(s, row, c, s.cols - (int)c);
    }
  }
}

// Sum of squares in fp64: neither a square nor a sum of them leaves its range, whatever the gradients are.
template <typename T>
__global__ __launch_bounds__(256) void fira_gradient_squares_kernel(FiraSpans l, double* partial) {
  __shared__ double part[4];
  double sum = 0.0;
  for_each_vector(l, [&](const FiraSpan& s, unsigned row, unsigned c, int left) {
    float v[kVec];
    load_some<T>((const typename T::raw*)s.g + (long long)row * s.ld + c, left, v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum += (double)v[i] * (double)v[i];
  });
  sum = block_sum(sum, part);
  if (threadIdx.x == 0) *as_global(partial + blockIdx.x) = sum;
}

// The norm from all launches' sums, in an order that every workgroup keeps.
__device__ __forceinline__ double norm_of(const double* partial, int n, double* part) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) s += *as_global(partial + i);
  return sqrt(block_sum(s, part));
}
__global__ __launch_bounds__(256) void fira_gradient_norm_kernel(const double* partial, int n, float* norm) {
  __shared__ double part[4];
  const double x = norm_of(partial, n, part);
  if (threadIdx.x == 0) *as_global(norm) = (float)x;
}

// out = min(1, max_norm / norm) g.  A norm that is not finite leaves the gradients as they are.
template <typename T, typename R>
__global__ __launch_bounds__(256) void fira_clip_kernel(FiraSpans l, const double* partial, int n, double max_norm) {
  __shared__ double part[4];
  const double norm = norm_of(partial, n, part);
  const bool cut = norm > max_norm && norm < INFINITY;
  const float factor = cut ? (float)(max_norm / norm) : 1.0f;
  for_each_vector(l, [&](const FiraSpan& s, unsigned row, unsigned c, int left) {
    if (!cut && s.g == s.out) return;     // in place: they are what they have to be
    float v[kVec];
    load_some<T>((const typename T::raw*)s.g + (long long)row * s.ld + c, left, v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] *= factor;
    store_some<R>((typename R::raw*)s.out + (long long)row * s.ld_out + c, left, v);
  });
}
