// Layer norm and root-mean-square norm of rows, and their gradients.  gfx950 only.
#pragma once
#include "fira_rows.h"

struct FiraNorm {
  long long rows, dim;
  long long ld_x, ld_y;      // y: the result (forward), the gradient of the result (backward)
  long long ld_dx;
  float eps;
  int rms;                   // 1: no mean
  int accumulate;            // backward: the weight's and the bias's gradients are added to what is there
};

// mu = mean x, rstd = (mean (x - mu)^2 + eps)^-1/2, y = w (x - mu) rstd + b.  One workgroup per row; mean before deviation, as their
// difference of large sums would cancel.
template <typename T, typename P>
__global__ __launch_bounds__(256) void fira_layer_norm_kernel(FiraNorm n, const typename T::raw* x, const typename P::raw* w, const typename P::raw* b,
                                                              typename T::raw* y, float* mean, float* rstd) {
  __shared__ float part[4];
  for (long long row = blockIdx.x; row < n.rows; row += gridDim.x) {
    const typename T::raw* xr = x + row * n.ld_x;
    float mu = 0.0f;
    if (!n.rms) {
      float s = 0.0f;
      for (long long c = threadIdx.x; c < n.dim; c += 256) s += load1<T>(xr + c);
      mu = block_sum(s, part) / (float)n.dim;
    }
    float s = 0.0f;
    for (long long c = threadIdx.x; c < n.dim; c += 256) { const float d = load1<T>(xr + c) - mu; s += d * d; }
    const float r = 1.0f / sqrtf(block_sum(s, part) / (float)n.dim + n.eps);
    for (long long c = threadIdx.x; c < n.dim; c += 256) {
      const float h = (load1<T>(xr + c) - mu) * r;
      store1<T>(y + row * n.ld_y + c, (w ? load1<P>(w + c) : 1.0f) * h + (b ? load1<P>(b + c) : 0.0f));
    }
    if (threadIdx.x == 0) {
      if (mean) *as_global(mean + row) = mu;
      if (rstd) *as_global(rstd + row) = r;
    }
  }
}

// g = w dy, h = (x - mu) rstd:  dx = rstd (g - mean g - h mean(g h)), without mean g where there is no mean.
template <typename T, typename P>
__global__ __launch_bounds__(256) void fira_layer_norm_dx_kernel(FiraNorm n, const typename T::raw* dy, const typename T::raw* x, const typename P::raw* w,
                                                                 const float* mean, const float* rstd, typename T::raw* dx) {
  __shared__ float part[4];
  for (long long row = blockIdx.x; row < n.rows; row += gridDim.x) {
    const float mu = n.rms ? 0.0f : *as_global(mean + row), r = *as_global(rstd + row);
    float s1 = 0.0f, s2 = 0.0f;
    for (long long c = threadIdx.x; c < n.dim; c += 256) {
      const float g = load1<T>(dy + row * n.ld_y + c) * (w ? load1<P>(w + c) : 1.0f);
      s1 += g;
      s2 += g * (load1<T>(x + row * n.ld_x + c) - mu) * r;
    }
    s1 = n.rms ? 0.0f : block_sum(s1, part) / (float)n.dim;
    s2 = block_sum(s2, part) / (float)n.dim;
    for (long long c = threadIdx.x; c < n.dim; c += 256) {
      const float g = load1<T>(dy + row * n.ld_y + c) * (w ? load1<P>(w + c) : 1.0f);
      const float h = (load1<T>(x + row * n.ld_x + c) - mu) * r;
      store1<T>(dx + row * n.ld_dx + c, r * (g - s1 - h * s2));
    }
  }
}

// dw = sum over rows of dy h, db = sum over rows of dy.  One workgroup per 64 columns, a quarter of the rows to each wavefront.
template <typename T, typename P>
__global__ __launch_bounds__(256) void fira_layer_norm_dw_kernel(FiraNorm n, const typename T::raw* dy, const typename T::raw* x, const float* mean,
                                                                 const float* rstd, typename P::raw* dw, typename P::raw* db) {
  __shared__ float part[2][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long c = blockIdx.x * 64LL + lane;
  float sw = 0.0f, sb = 0.0f;
  if (c < n.dim)
    for (long long row = wave; row < n.rows; row += 4) {
      const float g = load1<T>(dy + row * n.ld_y + c);
      sb += g;
      sw += g * (load1<T>(x + row * n.ld_x + c) - (n.rms ? 0.0f : *as_global(mean + row))) * *as_global(rstd + row);
    }
  part[0][wave][lane] = sw;
  part[1][wave][lane] = sb;
  __syncthreads();
  if (wave || c >= n.dim) return;
  for (int k = 1; k < 4; ++k) { sw += part[0][k][lane]; sb += part[1][k][lane]; }
  if (dw) store1<P>(dw + c, (n.accumulate ? load1<P>(dw + c) : 0.0f) + sw);
  if (db) store1<P>(db + c, (n.accumulate ? load1<P>(db + c) : 0.0f) + sb);
}
