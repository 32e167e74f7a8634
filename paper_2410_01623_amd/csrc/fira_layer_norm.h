// Layer norm and root-mean-square norm of rows, and their gradients.  gfx950 only.
#pragma once
#include "fira_rows.h"

struct FiraNorm {
  long long rows, dim;
  long long ld_x, ld_y;      // y: the result (forward), the gradient of the result (backward)
  long long ld_dx;
  float eps;
  int rms;                   // 1: no mean
};

// A row is held in registers by THREADS threads, NV vectors of W values to a thread (the first half of them, rounded down, inside the row), a part of
// a wavefront, a wavefront or a workgroup as its width asks for, so that it is read once and its sums are taken of what is there.
// kNormWidest: widest row that is held; wider ones are read again for every sum.
constexpr int kNormWidest = 16384;

// Sums of two values over a row's threads, in all of them.  part: LDS, two sets in turn, so that one barrier a row is enough.
template <int THREADS>
__device__ __forceinline__ void row_sums(float& a, float& b, float (*part)[16][2], int turn) {
  a = lanes_sum<THREADS < 64 ? THREADS : 64>(a);
  b = lanes_sum<THREADS < 64 ? THREADS : 64>(b);
  if constexpr (THREADS > 64) {
    if ((threadIdx.x & 63) == 0) { part[turn & 1][threadIdx.x >> 6][0] = a; part[turn & 1][threadIdx.x >> 6][1] = b; }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      const int wave = THREADS < 256 ? threadIdx.x / THREADS * (THREADS / 64) + w : w;
      a += part[turn & 1][wave][0];
      b += part[turn & 1][wave][1];
    }
  }
}

// mu = mean x, rstd = (mean (x - mu)^2 + eps)^-1/2, y = w (x - mu) rstd + b.  The deviation is taken from x - mu: E x^2 - mu^2 would cancel.
template <typename T, typename P, int W, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void fira_layer_norm_kernel(FiraNorm n, const typename T::raw* x, const typename P::raw* w,
                                                                                        const typename P::raw* b, typename T::raw* y, float* mean, float* rstd) {
  constexpr int GROUPS = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float part[2][16][2];
  const int me = threadIdx.x % THREADS;
  int turn = 0;
  for (long long row0 = (long long)blockIdx.x * GROUPS; row0 < n.rows; row0 += (long long)gridDim.x * GROUPS) {
    const long long row = row0 + threadIdx.x / THREADS;
    const bool here = row < n.rows;
    const typename T::raw* const xr = x + (here ? row : n.rows - 1) * n.ld_x;
    Raw<T, W> xs[NV];
    Raw<P, W> ws[NV], bs[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) xs[v].stream(xr + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
    if (w)
#pragma unroll
      for (int v = 0; v < NV; ++v) ws[v].load(w + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
    if (b)
#pragma unroll
      for (int v = 0; v < NV; ++v) bs[v].load(b + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
    int skip[NV];                                        // values of a vector that are not this thread's
#pragma unroll
    for (int v = NV / 2; v < NV; ++v) { const Columns<W> c((long long)(v * THREADS + me) * W, n.dim); skip[v] = c.any ? c.skip : W; }
    float mu = 0.0f, none = 0.0f;
    if (!n.rms) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) mu += v < NV / 2 || j >= skip[v] ? xs[v].get(j) : 0.0f;
      row_sums<THREADS>(mu, none, part, turn++);
      mu /= (float)n.dim;
    }
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float d = xs[v].get(j) - mu;
        s += v < NV / 2 || j >= skip[v] ? d * d : 0.0f;
      }
    row_sums<THREADS>(s, none, part, turn++);
    const float r = 1.0f / sqrtf(s / (float)n.dim + n.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Columns<W> c((long long)(v * THREADS + me) * W, n.dim);
      float o[W];
#pragma unroll
      for (int j = 0; j < W; ++j) {
        o[j] = (xs[v].get(j) - mu) * r;
        if (w) o[j] *= ws[v].get(j);
        if (b) o[j] += bs[v].get(j);
      }
      if (here && c.any) store_w<T, W, true>(y + row * n.ld_y + c.at, o);
    }
    if (here && me == 0) {
      if (mean) *as_global(mean + row) = mu;
      if (rstd) *as_global(rstd + row) = r;
    }
  }
}

// What the gradient's kernels do with a row, in the same roundings wherever it is done: this thread's part of the sums of g and g h, and of dw and db.
template <typename T, typename P, int W, int NV>
struct NormRow {
  Raw<T, W> x[NV], dy[NV];
  float mu, r;
  __device__ __forceinline__ void load(const FiraNorm& n, const typename T::raw* xs, const typename T::raw* dys, const float* mean, const float* rstd, long long row,
                                       int me, int threads) {
    mu = n.rms ? 0.0f : *as_global(mean + row);
    r = *as_global(rstd + row);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const long long c = Columns<W>((long long)(v * threads + me) * W, n.dim).at;
      x[v].stream(xs + row * n.ld_x + c);
      dy[v].stream(dys + row * n.ld_y + c);
    }
  }
  __device__ __forceinline__ void sums(const Raw<P, W> (&w)[NV], bool weighted, const int (&skip)[NV], bool here, float& s1, float& s2, float (&sw)[NV][W],
                                       float (&sb)[NV][W]) const {
#pragma clang fp contract(off)
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float d = here ? dy[v].get(j) : 0.0f, h = (x[v].get(j) - mu) * r, g = weighted ? d * w[v].get(j) : d;
        const bool mine = v < NV / 2 || j >= skip[v];
        s1 += mine ? g : 0.0f;
        s2 = mine ? __builtin_fmaf(g, h, s2) : s2;
        sw[v][j] = here ? __builtin_fmaf(d, h, sw[v][j]) : sw[v][j];
        sb[v][j] += d;
      }
  }
  // s1, s2: the means of g and g h
  __device__ __forceinline__ void write(const FiraNorm& n, const Raw<P, W> (&w)[NV], bool weighted, float s1, float s2, typename T::raw* dx, long long row, int me,
                                        int threads) const {
#pragma clang fp contract(off)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Columns<W> c((long long)(v * threads + me) * W, n.dim);
      float o[W];
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float h = (x[v].get(j) - mu) * r, g = weighted ? dy[v].get(j) * w[v].get(j) : dy[v].get(j);
        o[j] = r * (g - __builtin_fmaf(h, s2, s1));
      }
      if (c.any) store_w<T, W, true>(dx + row * n.ld_dx + c.at, o);
    }
  }
};

// g = w dy, h = (x - mu) rstd:  dx = rstd (g - mean g - h mean(g h)), without mean g where there is no mean;  dw = sum over rows of dy h,
// db = sum over rows of dy.  One pass: a workgroup takes every gridDim.x-th row (or set of rows side by side), the next one's values on their way
// while it works on one, and adds up dy h and dy of its columns in registers; fira_layer_norm_join_kernel adds up the workgroups' sums.
// partial: [2][gridDim.x][dim].
// Bound by memory: 131072 x 1024 bf16 154 us (5.2 TB/s), 8192 x 16384 bf16 175 (4.6) and f32 326 (4.9).  Rows wider than 8192 are held by 1024 threads, which have
// 128 registers each: 11 to 42 values more are kept in memory.
template <typename T, typename P, int W, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void fira_layer_norm_gradient_kernel(FiraNorm n, const typename T::raw* dy, const typename T::raw* x,
                                                                                                 const typename P::raw* w, const float* mean, const float* rstd,
                                                                                                 typename T::raw* dx, float* partial_w, float* partial_b) {
  constexpr int GROUPS = THREADS < 256 ? 256 / THREADS : 1;
  constexpr int BUFS = THREADS * NV * W > 8192 ? 1 : 2;      // (there are no registers for two rows then)
  __shared__ float part[2][16][2];
  __shared__ float joined[GROUPS > 1 ? GROUPS - 1 : 1][GROUPS > 1 ? THREADS * W : 1];
  const int me = threadIdx.x % THREADS, group = threadIdx.x / THREADS;
  Raw<P, W> ws[NV];
  if (w)
#pragma unroll
    for (int v = 0; v < NV; ++v) ws[v].load(w + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
  int skip[NV];                                          // values of a vector that are not this thread's
#pragma unroll
  for (int v = NV / 2; v < NV; ++v) { const Columns<W> c((long long)(v * THREADS + me) * W, n.dim); skip[v] = c.any ? c.skip : W; }
  float sw[NV][W] = {}, sb[NV][W] = {};
  NormRow<T, P, W, NV> rows[BUFS];
  const long long step = (long long)gridDim.x * GROUPS;
  auto load = [&](int to, long long row) { rows[to].load(n, x, dy, mean, rstd, min(row, n.rows - 1), me, THREADS); };
  int turn = 0;
  auto work = [&](int of, long long row0) {
    const long long row = row0 + group;
    const bool here = row < n.rows;
    float s1 = 0.0f, s2 = 0.0f;
    rows[of].sums(ws, w != nullptr, skip, here, s1, s2, sw, sb);
    row_sums<THREADS>(s1, s2, part, turn++);
    if (dx && here) rows[of].write(n, ws, w != nullptr, n.rms ? 0.0f : s1 / (float)n.dim, s2 / (float)n.dim, dx, row, me, THREADS);
  };
  // (two rows a turn, so that which registers hold which is known to the compiler)
  long long row0 = (long long)blockIdx.x * GROUPS;
  if constexpr (BUFS == 1) {
    for (; row0 < n.rows; row0 += step) { load(0, row0 + group); work(0, row0); }
  } else {
    load(0, row0 + group);
    for (; row0 < n.rows; row0 += 2 * step) {
      load(1, row0 + step + group);
      work(0, row0);
      if (row0 + step >= n.rows) break;
      load(0, row0 + 2 * step + group);
      work(1, row0 + step);
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* const partial = which ? partial_b : partial_w;
    if (!partial) continue;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float (&s)[W] = which ? sb[v] : sw[v];
      if constexpr (GROUPS > 1) {
        __syncthreads();
        if (group)
#pragma unroll
          for (int j = 0; j < W; ++j) joined[group - 1][j * THREADS + me] = s[j];
        __syncthreads();
        if (group) continue;
#pragma unroll 4
        for (int k = 0; k < GROUPS - 1; ++k)
#pragma unroll
          for (int j = 0; j < W; ++j) s[j] += joined[k][j * THREADS + me];
      }
      const Columns<W> c((long long)(v * THREADS + me) * W, n.dim);
      if (c.any) store_w<FiraStoredF32, W>(partial + (long long)blockIdx.x * n.dim + c.at, s);
    }
  }
}

// Sums of the parts: a workgroup takes 32 columns of dw (blockIdx.y 0) or db (1), a part of the parts to each of its 32 sets of eight lanes.
template <typename P>
__global__ __launch_bounds__(256) void fira_layer_norm_join_kernel(const float* partial_w, const float* partial_b, int parts, long long dim, typename P::raw* dw,
                                                                   typename P::raw* db, int accumulate) {
  constexpr int SETS = 32, N = 8;
  __shared__ float sums[SETS][33];
  const float* const partial = blockIdx.y ? partial_b : partial_w;
  typename P::raw* const to = blockIdx.y ? db : dw;
  if (!to) return;
  const int lane = threadIdx.x % 8, set = threadIdx.x / 8;
  const long long c0 = blockIdx.x * 32LL;
  const int cols = (int)min(32LL, dim - c0);
  float s[4] = {};
  for (int p0 = set; p0 < parts; p0 += SETS * N) {
    float x[N][4];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float* const from = partial + (long long)min(p0 + SETS * k, parts - 1) * dim + c0;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[k][j] = *as_global(from + min(j * 8 + lane, cols - 1));
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (p0 + SETS * k < parts)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += x[k][j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) sums[set][j * 8 + lane] = s[j];
  __syncthreads();
  if (threadIdx.x >= cols) return;
  float all = 0.0f;
#pragma unroll
  for (int k = 0; k < SETS; ++k) all += sums[k][threadIdx.x];
  store1<P>(to + c0 + threadIdx.x, accumulate ? load1<P>(to + c0 + threadIdx.x) + all : all);
}

// Few rows: all in one launch and without a workspace.  The first workgroups take the rows, the others 8 W columns each, for which they read all
// rows again: eight lanes to a row's columns, as many rows side by side as there are sets of eight lanes.
// Up to kFewRows; us here and in two launches: 512 rows bf16 x 256 5.5 and 6.4, x 2048 6.3 and 8.4, x 8192 13.6 and 21.9, x 16384 19.7 and 38.6; 768 rows f32 x 2048 13.3
// and 10.6, bf16 x 512 7.0 and 6.1, x 8192 18.7 and 26.3; 1024 rows bf16 x 512 8.5 and 6.5, x 8192 22.7 and 27.9; 2048 rows bf16 x 2048 30 and 14, x 8192 40 and 35.
constexpr int kFewRows = 512;
template <typename T, typename P, int W, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void fira_layer_norm_gradient_few_kernel(FiraNorm n, const typename T::raw* dy, const typename T::raw* x,
                                                                                                     const typename P::raw* w, const float* mean, const float* rstd,
                                                                                                     typename T::raw* dx, typename P::raw* dw, typename P::raw* db,
                                                                                                     int accumulate, int row_groups) {
  constexpr int ALL = THREADS < 256 ? 256 : THREADS, GROUPS = ALL / THREADS;
  __shared__ float part[2][16][2];
  __shared__ float sums[ALL / 64][2][8 * W];
  if ((int)blockIdx.x < row_groups) {
    const int me = threadIdx.x % THREADS;
    const long long row = (long long)blockIdx.x * GROUPS + threadIdx.x / THREADS;
    const bool here = row < n.rows;
    Raw<P, W> ws[NV];
    if (w)
#pragma unroll
      for (int v = 0; v < NV; ++v) ws[v].load(w + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
    int skip[NV];
#pragma unroll
    for (int v = NV / 2; v < NV; ++v) { const Columns<W> c((long long)(v * THREADS + me) * W, n.dim); skip[v] = c.any ? c.skip : W; }
    NormRow<T, P, W, NV> r;
    r.load(n, x, dy, mean, rstd, min(row, n.rows - 1), me, THREADS);
    float s1 = 0.0f, s2 = 0.0f, sw[NV][W] = {}, sb[NV][W] = {};      // (the sums over rows are not wanted here)
    r.sums(ws, w != nullptr, skip, here, s1, s2, sw, sb);
    row_sums<THREADS>(s1, s2, part, 0);
    if (here) r.write(n, ws, w != nullptr, n.rms ? 0.0f : s1 / (float)n.dim, s2 / (float)n.dim, dx, row, me, THREADS);
    return;
  }
  constexpr int SETS = ALL / 8, N = 4;
  const int lane = threadIdx.x % 8, set = threadIdx.x / 8;
  const Columns<W> c((long long)(blockIdx.x - row_groups) * (8 * W) + lane * W, n.dim);
  float sw[W] = {}, sb[W] = {};
  for (int row0 = set; row0 < (int)n.rows; row0 += N * SETS) {
    Raw<T, W> xs[N], gs[N];
    float mu[N], r[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const long long row = min((long long)row0 + k * SETS, n.rows - 1);
      xs[k].load(x + row * n.ld_x + c.at);
      gs[k].load(dy + row * n.ld_y + c.at);
      mu[k] = n.rms ? 0.0f : *as_global(mean + row);
      r[k] = *as_global(rstd + row);
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (row0 + k * SETS < (int)n.rows)
#pragma unroll
        for (int j = 0; j < W; ++j) {
          sw[j] += gs[k].get(j) * ((xs[k].get(j) - mu[k]) * r[k]);
          sb[j] += gs[k].get(j);
        }
  }
#pragma unroll
  for (int j = 0; j < W; ++j) {
    sw[j] = add_xor<8>(add_xor<16>(add_xor<32>(sw[j])));
    sb[j] = add_xor<8>(add_xor<16>(add_xor<32>(sb[j])));
  }
  if ((threadIdx.x & 63) < 8)
#pragma unroll
    for (int j = 0; j < W; ++j) { sums[threadIdx.x >> 6][0][j * 8 + lane] = sw[j]; sums[threadIdx.x >> 6][1][j * 8 + lane] = sb[j]; }
  __syncthreads();
  if (threadIdx.x >= 16) return;                         // eight lanes for dw, eight for db
  typename P::raw* const to = threadIdx.x < 8 ? dw : db;
  if (!to || !c.any) return;
#pragma unroll
  for (int j = 0; j < W; ++j) {
    float all = 0.0f;
#pragma unroll
    for (int k = 0; k < ALL / 64; ++k) all += sums[k][threadIdx.x >> 3][j * 8 + lane];
    if (j >= c.skip) store1<P>(to + c.at + j, accumulate ? load1<P>(to + c.at + j) + all : all);
  }
}

// Rows wider than kNormWidest: one workgroup per row, which reads it for each sum and for the result.
template <typename T, typename P>
__global__ __launch_bounds__(1024) void fira_layer_norm_wide_kernel(FiraNorm n, const typename T::raw* x, const typename P::raw* w, const typename P::raw* b,
                                                                    typename T::raw* y, float* mean, float* rstd) {
  __shared__ float part[16];
  for (long long row = blockIdx.x; row < n.rows; row += gridDim.x) {
    const typename T::raw* xr = x + row * n.ld_x;
    float mu = 0.0f;
    if (!n.rms) {
      float s = 0.0f;
      for (long long c = threadIdx.x; c < n.dim; c += 1024) s += load1<T>(xr + c);
      mu = block_sum(s, part) / (float)n.dim;
    }
    float s = 0.0f;
    for (long long c = threadIdx.x; c < n.dim; c += 1024) { const float d = load1<T>(xr + c) - mu; s += d * d; }
    const float r = 1.0f / sqrtf(block_sum(s, part) / (float)n.dim + n.eps);
    for (long long c = threadIdx.x; c < n.dim; c += 1024) {
      const float h = (load1<T>(xr + c) - mu) * r;
      store1<T>(y + row * n.ld_y + c, (w ? load1<P>(w + c) : 1.0f) * h + (b ? load1<P>(b + c) : 0.0f));
    }
    if (threadIdx.x == 0) {
      if (mean) *as_global(mean + row) = mu;
      if (rstd) *as_global(rstd + row) = r;
    }
  }
}
template <typename T, typename P>
__global__ __launch_bounds__(1024) void fira_layer_norm_wide_dx_kernel(FiraNorm n, const typename T::raw* dy, const typename T::raw* x, const typename P::raw* w,
                                                                       const float* mean, const float* rstd, typename T::raw* dx) {
  __shared__ float part[16];
  for (long long row = blockIdx.x; row < n.rows; row += gridDim.x) {
    const float mu = n.rms ? 0.0f : *as_global(mean + row), r = *as_global(rstd + row);
    float s1 = 0.0f, s2 = 0.0f;
    for (long long c = threadIdx.x; c < n.dim; c += 1024) {
      const float g = load1<T>(dy + row * n.ld_y + c) * (w ? load1<P>(w + c) : 1.0f);
      s1 += g;
      s2 += g * (load1<T>(x + row * n.ld_x + c) - mu) * r;
    }
    s1 = n.rms ? 0.0f : block_sum(s1, part) / (float)n.dim;
    s2 = block_sum(s2, part) / (float)n.dim;
    for (long long c = threadIdx.x; c < n.dim; c += 1024) {
      const float g = load1<T>(dy + row * n.ld_y + c) * (w ? load1<P>(w + c) : 1.0f);
      const float h = (load1<T>(x + row * n.ld_x + c) - mu) * r;
      store1<T>(dx + row * n.ld_dx + c, r * (g - s1 - h * s2));
    }
  }
}
// ... and the sums over rows, gridDim.y-th part of them: 256 columns per workgroup.
template <typename T>
__global__ __launch_bounds__(256) void fira_layer_norm_wide_dw_kernel(FiraNorm n, const typename T::raw* dy, const typename T::raw* x, const float* mean,
                                                                      const float* rstd, float* partial_w, float* partial_b) {
  const long long c = blockIdx.x * 256LL + threadIdx.x;
  if (c >= n.dim) return;
  float sw = 0.0f, sb = 0.0f;
  for (long long row = blockIdx.y; row < n.rows; row += gridDim.y) {
    const float g = load1<T>(dy + row * n.ld_y + c);
    sb += g;
    sw += g * (load1<T>(x + row * n.ld_x + c) - (n.rms ? 0.0f : *as_global(mean + row))) * *as_global(rstd + row);
  }
  if (partial_w) *as_global(partial_w + blockIdx.y * n.dim + c) = sw;
  if (partial_b) *as_global(partial_b + blockIdx.y * n.dim + c) = sb;
}
