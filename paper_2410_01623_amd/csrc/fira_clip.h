// The norm of a list of gradients taken together, and their scaling where it passes a limit.  gfx950 only.
//
// Two passes: the factor is known when all has been read, and what has to be cut is read again.  Both are bound by memory.  60m shapes, f32 to bf16, cut:
// 106 us, with 8 or 3 values between the rows 108; where rows are apart and no whole number of vectors wide, the end of each is taken value by value from
// memory (511 x 1377 and the like 115 us dense, 197 apart).
#pragma once
#include "fira_rows.h"

// A piece of a gradient: rows of `cols` values.  The host cuts longer ones up so that all counts fit 32 bits.
struct FiraSpan {
  const void* g;
  void* out;
  int rows, cols;
  int ld, ld_out;
  int vecs;          // vectors of a row: of as many values as the kernel takes, the last one of a row maybe shorter, or of one where a row has fewer
  int tile0;         // first tile of this piece
};
constexpr int kSpans = 96;            // a launch's pieces travel as kernel arguments, of which there are 4 KB
constexpr int kClipUnroll = 4;        // vectors of a thread that are on their way together
constexpr int kClipTile = 256 * kClipUnroll;
constexpr int kClipWorkgroups = 1024;
struct FiraSpans {
  FiraSpan s[kSpans];
  int count, tiles;
  int each;          // tiles of a workgroup
};
static_assert(sizeof(FiraSpans) + 64 <= 4096, "kernel arguments");

// Calls f(piece, first vector) for this workgroup's tiles, which adjoin.
template <typename F>
__device__ __forceinline__ void for_each_tile(const FiraSpans& l, F f) {
  const int from = blockIdx.x * l.each, until = min(from + l.each, l.tiles);
  int k = 0;                                             // the last piece that does not begin after the first tile
#pragma unroll 1
  for (int step = 64; step; step >>= 1)
    if (k + step < l.count && l.s[k + step].tile0 <= from) k += step;
#pragma unroll 1
  for (int tile = from; tile < until; ++tile) {
    while (k + 1 < l.count && l.s[k + 1].tile0 <= tile) ++k;
    k = __builtin_amdgcn_readfirstlane(k);
    f(l.s[k], (unsigned)(tile - l.s[k].tile0) * kClipTile);
  }
}

// Calls f(row, place of the vector, values in front that are another vector's, whether there is such a vector) for this thread's vectors of a tile
// one after the other, so that f can put loads on their way; the last vector of a row starts earlier, so that it is whole.
template <int W, bool STRIDED, typename F>
__device__ __forceinline__ void for_each_vector(const FiraSpan& s, unsigned first, F f) {
  const unsigned total = (unsigned)s.rows * (unsigned)s.vecs;
#pragma unroll
  for (int u = 0; u < kClipUnroll; ++u) {
    const unsigned i = first + u * 256 + threadIdx.x, at = min(i, total - 1);
    const unsigned row = STRIDED ? at / (unsigned)s.vecs : 0u;
    const int c = (int)(at - row * (unsigned)s.vecs) * W, begin = min(c, s.cols - W);
    f(u, row, begin, c - begin, i < total);
  }
}
// Calls f with the constants for a piece: values of a vector, whether it has more than one row.
template <int W, typename F>
__device__ __forceinline__ void with_piece_shape(const FiraSpan& s, F f) {
  if (s.cols < W) f(std::integral_constant<int, 1>{}, std::true_type{});
  else if (s.rows > 1) f(std::integral_constant<int, W>{}, std::true_type{});
  else f(std::integral_constant<int, W>{}, std::false_type{});
}

// Sum of squares in fp64: neither a square nor a sum of them leaves its range, whatever the gradients are, and the vector unit has room for it
// beside the loads.
template <typename T>
__global__ __launch_bounds__(256) void fira_gradient_squares_kernel(FiraSpans l, double* partial) {
  __shared__ double part[4];
  double sum = 0.0;
  for_each_tile(l, [&](const FiraSpan& s, unsigned first) {
    with_piece_shape<kWidth<T>>(s, [&](auto w, auto strided) {
      constexpr int W = decltype(w)::value;
      Raw<T, W> x[kClipUnroll];
      const typename T::raw* p[kClipUnroll];
      int skip[kClipUnroll];
      for_each_vector<W, decltype(strided)::value>(s, first, [&](int u, unsigned row, int c, int before, bool here) {
        p[u] = (const typename T::raw*)s.g + (long long)row * s.ld + c;
        x[u].stream(p[u]);
        skip[u] = here ? before : -1;
      });
#pragma unroll
      for (int u = 0; u < kClipUnroll; ++u) {
        double q = 0.0;
#pragma unroll
        for (int j = 0; j < W; ++j) q += (double)x[u].get(j) * (double)x[u].get(j);
        sum += skip[u] == 0 ? q : 0.0;
        if (skip[u] > 0)
#pragma unroll 1
          for (int j = skip[u]; j < W; ++j) { const double v = load1<T>(p[u] + j); sum += v * v; }
      }
    });
  });
  sum = block_sum(sum, part);
  if (threadIdx.x == 0) *as_global(partial + blockIdx.x) = sum;
}

// The norm from all launches' sums, in an order that every workgroup keeps.
__device__ __forceinline__ double norm_of(const double* partial, int n, double* part) {
  double s = 0.0;
#pragma unroll 8
  for (int i = threadIdx.x; i < n; i += 256) s += *as_global(partial + i);
  return sqrt(block_sum(s, part));
}
template <typename = void>
__global__ __launch_bounds__(256) void fira_gradient_norm_kernel(const double* partial, int n, float* norm) {
  __shared__ double part[4];
  const double x = norm_of(partial, n, part);
  if (threadIdx.x == 0) *as_global(norm) = (float)x;
}

// out = min(1, max_norm / norm) g.  A norm that is not finite, as the fp32 value that the caller reads, leaves the gradients as they are.  Every
// workgroup works the norm out for itself, and one of them leaves it in *norm: no launch in between.
template <typename T, typename R>
__global__ __launch_bounds__(256) void fira_clip_kernel(FiraSpans l, const double* partial, int n, double max_norm, float* norm) {
  __shared__ double part[4];
  const double x = norm_of(partial, n, part);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *as_global(norm) = (float)x;
  const bool cut = x > max_norm && (float)x < INFINITY;
  const float factor = cut ? (float)(max_norm / x) : 1.0f;
  for_each_tile(l, [&](const FiraSpan& s, unsigned first) {
    if (!cut && s.g == s.out) return;                    // in place: they are what they have to be
    with_piece_shape<kWidth<T, R>>(s, [&](auto w, auto strided) {
      constexpr int W = decltype(w)::value;
      Raw<T, W> x[kClipUnroll];
      const typename T::raw* p[kClipUnroll];
      typename R::raw* to[kClipUnroll];
      int skip[kClipUnroll];
      for_each_vector<W, decltype(strided)::value>(s, first, [&](int u, unsigned row, int c, int before, bool here) {
        p[u] = (const typename T::raw*)s.g + (long long)row * s.ld + c;
        to[u] = (typename R::raw*)s.out + (long long)row * s.ld_out + c;
        x[u].stream(p[u]);
        skip[u] = here ? before : -1;
      });
#pragma unroll
      for (int u = 0; u < kClipUnroll; ++u) {
        float y[W];
#pragma unroll
        for (int j = 0; j < W; ++j) y[j] = factor * x[u].get(j);
        if (skip[u] == 0) store_w<R, W, true>(to[u], y);
        // (what another vector has as well may have been scaled by now, and is left to it)
        if (skip[u] > 0)
#pragma unroll 1
          for (int j = skip[u]; j < W; ++j) store1<R>(to[u] + j, factor * load1<T>(p[u] + j));
      }
    });
  });
}
