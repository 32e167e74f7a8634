// What stands between two blocks on the residual stream: the block's norm, gate and scale, the sum, and the next block's norm; and the gradients.  gfx950 only.
#pragma once
#include "fira_layer_norm.h"

enum { kLayer = 0, kRms = 1, kNone = 2 };

struct FiraBlockNorm {
  long long rows, dim;
  long long ld_x, ld_b, ld_r, ld_y;       // x: in the gradient that of r from elsewhere; y: in the gradient that of y
  long long ld_dx, ld_db;
  float eps, post_eps, alpha, beta;       // alpha: of the block, beta: of the residual
  int norm, post;
};
template <typename P>
struct FiraBlockVectors {
  const typename P::raw *gate, *w, *b, *pw, *pb;
};
struct FiraBlockStats {
  float *mean, *rstd, *post_mean, *post_rstd;
};

// A row is held in registers as in fira_layer_norm.h: THREADS threads, NV vectors of W values to a thread.  Bound by memory: 131072 x 2048
// bf16 348 us (6.2 TB/s); 16385 x 2049 72 (3.7), whose rows begin at odd elements, x 2050 54.
template <typename T, typename P, int W, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void fira_block_norm_kernel(FiraBlockNorm n, const typename T::raw* x, const typename T::raw* b, FiraBlockVectors<P> vec,
                                                                                        typename T::raw* r, typename T::raw* y, FiraBlockStats to) {
  constexpr int GROUPS = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float part[2][16][2];
  const int me = GROUPS == 1 ? threadIdx.x : threadIdx.x % THREADS, group = GROUPS == 1 ? 0 : threadIdx.x / THREADS;   // (a row of a workgroup has a scalar address)
  const float dim = (float)n.dim;
  int turn = 0;
  for (long long row0 = (long long)blockIdx.x * GROUPS; row0 < n.rows; row0 += (long long)gridDim.x * GROUPS) {
    const long long row = row0 + group;
    const bool here = row < n.rows;
    const long long at = here ? row : n.rows - 1;
    Raw<T, W> xs[NV], bs[NV];
    int skip[NV];                                          // values of a vector that are not this thread's
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Columns<W> c((long long)(v * THREADS + me) * W, n.dim);
      bs[v].stream(b + at * n.ld_b + c.at);
      xs[v].stream(x + at * n.ld_x + c.at);
      skip[v] = v < NV / 2 ? 0 : c.any ? c.skip : W;
    }
    float u[NV][W];
    auto sum = [&](auto f) {
      float s = 0.0f, none = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) s += v < NV / 2 || j >= skip[v] ? f(u[v][j]) : 0.0f;
      row_sums<THREADS>(s, none, part, turn++);
      return s;
    };
    // u -= its mean; 1 / the deviation that is left
    auto stats = [&](int kind, float eps, float& mu, float& rs) {
      mu = 0.0f;
      if (kind == kLayer) {
        mu = sum([](float x) { return x; }) / dim;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < W; ++j) u[v][j] -= mu;
      }
      rs = 1.0f / sqrtf(sum([](float x) { return x * x; }) / dim + eps);
    };
    auto times = [&](const typename P::raw* w) {
      if (!w) return;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        Raw<P, W> ws;
        ws.load(w + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
#pragma unroll
        for (int j = 0; j < W; ++j) u[v][j] *= ws.get(j);
      }
    };
    auto plus = [&](const typename P::raw* w) {
      if (!w) return;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        Raw<P, W> ws;
        ws.load(w + Columns<W>((long long)(v * THREADS + me) * W, n.dim).at);
#pragma unroll
        for (int j = 0; j < W; ++j) u[v][j] += ws.get(j);
      }
    };
    auto put = [&](typename T::raw* out, long long ld) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Columns<W> c((long long)(v * THREADS + me) * W, n.dim);
        if (here && c.any) store_w<T, W, true>(out + row * ld + c.at, u[v]);
      }
    };
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) u[v][j] = bs[v].get(j);
    float pm = 0.0f, ps = 1.0f, mu = 0.0f, rs = 1.0f;
    if (n.post != kNone) {
      stats(n.post, n.post_eps, pm, ps);
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) u[v][j] *= ps;
      times(vec.pw);
      plus(vec.pb);
    }
    times(vec.gate);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) u[v][j] = n.beta * xs[v].get(j) + n.alpha * u[v][j];
    if (r) put(r, n.ld_r);
    if (n.norm != kNone) {
      stats(n.norm, n.eps, mu, rs);
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) u[v][j] *= rs;
      times(vec.w);
      plus(vec.b);
      put(y, n.ld_y);
    }
    if (here && me == 0) {
      if (to.mean && n.norm == kLayer) *as_global(to.mean + row) = mu;
      if (to.rstd && n.norm != kNone) *as_global(to.rstd + row) = rs;
      if (to.post_mean && n.post == kLayer) *as_global(to.post_mean + row) = pm;
      if (to.post_rstd && n.post != kNone) *as_global(to.post_rstd + row) = ps;
    }
  }
}

// Rows wider than kNormWidest: a workgroup for a row, which it reads again for every sum, value by value (4096 x 32768 bf16 1702 us, where 8192 x 16384 above take 215).
template <typename T, typename P>
__global__ __launch_bounds__(1024) void fira_block_norm_wide_kernel(FiraBlockNorm n, const typename T::raw* x, const typename T::raw* b, FiraBlockVectors<P> v, typename T::raw* r,
                                                                    typename T::raw* y, FiraBlockStats to) {
  __shared__ float part[16];
  const float dim = (float)n.dim;
  for (long long row = blockIdx.x; row < n.rows; row += gridDim.x) {
    const typename T::raw *const xr = x + row * n.ld_x, *const br = b + row * n.ld_b;
    auto total = [&](auto f) {
      float s = 0.0f;
      for (long long c = threadIdx.x; c < n.dim; c += blockDim.x) s += f(c);
      return block_sum(s, part);
    };
    // mean and 1 / deviation of f
    auto stats = [&](int kind, float eps, auto f, float& mu, float& rs) {
      mu = kind == kLayer ? total(f) / dim : 0.0f;
      rs = 1.0f / sqrtf(total([&](long long c) { const float d = f(c) - mu; return d * d; }) / dim + eps);
    };
    float pm = 0.0f, ps = 1.0f, mu = 0.0f, rs = 1.0f;
    if (n.post != kNone) stats(n.post, n.post_eps, [&](long long c) { return load1<T>(br + c); }, pm, ps);
    auto residual = [&](long long c) {
      float u = load1<T>(br + c);
      if (n.post != kNone) {
        u = (u - pm) * ps;
        if (v.pw) u *= load1<P>(v.pw + c);
        if (v.pb) u += load1<P>(v.pb + c);
      }
      if (v.gate) u *= load1<P>(v.gate + c);
      return n.beta * load1<T>(xr + c) + n.alpha * u;
    };
    if (n.norm != kNone) stats(n.norm, n.eps, residual, mu, rs);
    for (long long c = threadIdx.x; c < n.dim; c += blockDim.x) {
      const float s = residual(c);
      if (r) store1<T>(r + row * n.ld_r + c, s);
      if (y) {
        float o = (s - mu) * rs;
        if (v.w) o *= load1<P>(v.w + c);
        if (v.b) o += load1<P>(v.b + c);
        store1<T>(y + row * n.ld_y + c, o);
      }
    }
    if (threadIdx.x == 0) {
      if (to.mean && n.norm == kLayer) *as_global(to.mean + row) = mu;
      if (to.rstd && n.norm != kNone) *as_global(to.rstd + row) = rs;
      if (to.post_mean && n.post == kLayer) *as_global(to.post_mean + row) = pm;
      if (to.post_rstd && n.post != kNone) *as_global(to.post_rstd + row) = ps;
    }
  }
}

// What the gradient's kernel holds of a row: its values as they are stored, and the statistics.
template <typename T, int W, int NV>
struct BlockRowHeld {
  Raw<T, W> dr[NV], dy[NV], r[NV], b[NV];
  float mu, rs, pm, ps;
};

// t = dr + rstd (g - mean g - h mean(g h)), g = w dy;  dx = beta t;  q = alpha gate t pw,  db = rstd' (q - mean q - h' mean(q h')).  One pass as in fira_layer_norm_gradient_kernel: a workgroup takes
// every gridDim.x-th row, or set of rows side by side, and adds up its columns of dy h, dy, t h' and t, of which the vectors' gradients are
// made (block_vector_gradients): gate and post norm need no sums of their own.  partial: [4][gridDim.x][dim], of which `sums` (bits) are wanted.  Bound by memory: 65536 x 2048 bf16
// 312 us (5.2 TB/s), 16385 x 2049 f32 with means and biases 167 (4.8); with few rows by the latency of those of a workgroup (4097 x 2049 so 55, 3.6).
constexpr int kBlockWidest = 8192;      // of the gradient's rows in registers, 16 values a thread
// Ten wavefronts, in fp32 up to 2560 columns: two such workgroups fit a compute unit wherever they begin if six wavefronts fit a SIMD (with five, 16385 x 2049 with means and
// biases took 213 us, alone 203, so 175; with five wavefronts of two vectors 210, and without means 165 for 147; 16385 x 2560 224 for 188 and 195 for 178).
constexpr int kBlockTwo = 640;
// LEAN: no means and no sums of dy and t, as for root-mean-square norms without biases, which leaves registers for more wavefronts.
template <typename T, typename P, int W, int THREADS, int NV, bool LEAN>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS, THREADS == kBlockTwo ? 6 : 1) void fira_block_norm_gradient_kernel(FiraBlockNorm n, const typename T::raw* dr, const typename T::raw* dy, const typename T::raw* r,
                                                                                                 const typename T::raw* b, FiraBlockVectors<P> vec, FiraBlockStats stats,
                                                                                                 typename T::raw* dx, typename T::raw* db, float* partial, int sums) {
  constexpr int GROUPS = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float part[2][16][2];
  __shared__ float joined[GROUPS > 1 ? GROUPS - 1 : 1][GROUPS > 1 ? THREADS * W : 1];
  const int me = GROUPS == 1 ? threadIdx.x : threadIdx.x % THREADS, group = GROUPS == 1 ? 0 : threadIdx.x / THREADS;   // (a row of a workgroup has a scalar address)
  const float dim = (float)n.dim;
  const bool pre = n.norm != kNone, post = n.post != kNone, block = b != nullptr;
  // w, and alpha gate pw, of a thread's columns: in LDS, as the registers decide how many workgroups a compute unit holds (16385 x 2500 bf16, with means, 175 us with them
  // there and 114 here)
  constexpr int F = W < 4 ? W : 4, K = W / F;
  __shared__ __attribute__((aligned(16))) float factors[2][NV][K][THREADS][F];
  auto factor = [&](int which, int v, int j) { return factors[which][v][j / F][me][j % F]; };
  int skip[NV];                                          // values of a vector that are not this thread's
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Columns<W> c((long long)(v * THREADS + me) * W, n.dim);
    Raw<P, W> w, g, pw;
    if (vec.w) w.load(vec.w + c.at);
    if (vec.gate) g.load(vec.gate + c.at);
    if (vec.pw) pw.load(vec.pw + c.at);
    if (!group)
#pragma unroll
      for (int j = 0; j < W; ++j) {
        factors[0][v][j / F][me][j % F] = vec.w ? w.get(j) : 1.0f;
        factors[1][v][j / F][me][j % F] = n.alpha * (vec.gate ? g.get(j) : 1.0f) * (vec.pw ? pw.get(j) : 1.0f);
      }
    skip[v] = v < NV / 2 ? 0 : c.any ? c.skip : W;
  }
  if (GROUPS > 1) __syncthreads();                       // (else a thread's own)
  float s0[NV][W] = {}, s2[NV][W] = {}, s1[LEAN ? 1 : NV][W] = {}, s3[LEAN ? 1 : NV][W] = {};
  BlockRowHeld<T, W, NV> x;
  auto load = [&](long long row) {
    row = min(row, n.rows - 1);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const long long c = Columns<W>((long long)(v * THREADS + me) * W, n.dim).at;
      if (pre) { x.dy[v].stream(dy + row * n.ld_y + c); x.r[v].stream(r + row * n.ld_r + c); }
      if (dr) x.dr[v].stream(dr + row * n.ld_x + c);
      if (block) x.b[v].stream(b + row * n.ld_b + c);
    }
    x.mu = !LEAN && n.norm == kLayer ? *as_global(stats.mean + row) : 0.0f;
    x.rs = pre ? *as_global(stats.rstd + row) : 1.0f;
    x.pm = !LEAN && n.post == kLayer ? *as_global(stats.post_mean + row) : 0.0f;
    x.ps = post ? *as_global(stats.post_rstd + row) : 1.0f;
  };
  // Sums of f(v, j, a, b) over the row's values.  Those at the end of a row that are a neighbour's are left out again where there are some.
  int turn = 0;
  auto row_total = [&](float& a, float& b, auto f) {
    a = b = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float va = 0.0f, vb = 0.0f;
#pragma unroll
      for (int j = 0; j < W; ++j) f(v, j, va, vb);
      if (v >= NV / 2 && skip[v]) {
        va = vb = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
          float ja = 0.0f, jb = 0.0f;
          f(v, j, ja, jb);
          va += j >= skip[v] ? ja : 0.0f;
          vb += j >= skip[v] ? jb : 0.0f;
        }
      }
      a += va;
      b += vb;
    }
    row_sums<THREADS>(a, b, part, turn++);
  };
  auto work = [&](long long row0) {
    const long long row = row0 + group;
    const bool here = GROUPS == 1 || row < n.rows;       // (a set of rows may be short: its other rows count as zeros)
    auto hr = [&](int v, int j) { return (LEAN ? x.r[v].get(j) : x.r[v].get(j) - x.mu) * x.rs; };
    auto hb = [&](int v, int j) { return (LEAN ? x.b[v].get(j) : x.b[v].get(j) - x.pm) * x.ps; };
    auto put = [&](typename T::raw* out, long long ld, int v, const float (&o)[W]) {
      const Columns<W> c((long long)(v * THREADS + me) * W, n.dim);
      if (here && c.any) store_w<T, W, true>(out + row * ld + c.at, o);
    };
    float t[NV][W];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < W; ++j) t[v][j] = dr && here ? x.dr[v].get(j) : 0.0f;
    if (pre) {
      auto dy_of = [&](int v, int j) { return here ? x.dy[v].get(j) : 0.0f; };
      float a1, a2;
      row_total(a1, a2, [&](int v, int j, float& a, float& b) {
        const float g = dy_of(v, j) * factor(0, v, j);
        if (!LEAN) a += g;
        b = __builtin_fmaf(g, hr(v, j), b);
      });
      a1 = !LEAN && n.norm == kLayer ? a1 / dim : 0.0f;
      a2 /= dim;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float d = dy_of(v, j), h = hr(v, j);
          s0[v][j] = __builtin_fmaf(d, h, s0[v][j]);
          t[v][j] = __builtin_fmaf(x.rs, d * factor(0, v, j) - __builtin_fmaf(h, a2, a1), t[v][j]);
        }
      if (!LEAN && sums & 2)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < W; ++j) s1[v][j] += dy_of(v, j);
    }
    if (sums & 4)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) s2[v][j] = __builtin_fmaf(t[v][j], hb(v, j), s2[v][j]);
    if (!LEAN && sums & 8)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) s3[v][j] += t[v][j];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float o[W];
#pragma unroll
      for (int j = 0; j < W; ++j) o[j] = n.beta * t[v][j];
      if (dx) put(dx, n.ld_dx, v, o);
#pragma unroll
      for (int j = 0; j < W; ++j) t[v][j] *= factor(1, v, j);
    }
    if (!db) return;
    float q1 = 0.0f, q2 = 0.0f;
    if (post) {
      row_total(q1, q2, [&](int v, int j, float& a, float& b) {
        if (!LEAN) a += t[v][j];
        b = __builtin_fmaf(t[v][j], hb(v, j), b);
      });
      q1 = !LEAN && n.post == kLayer ? q1 / dim : 0.0f;
      q2 /= dim;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) t[v][j] = x.ps * (t[v][j] - __builtin_fmaf(hb(v, j), q2, q1));
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) put(db, n.ld_db, v, t[v]);
  };
  // (the next row on its way takes registers that more wavefronts can use: 32768 x 4096 bf16 279 us and 283 with it)
  for (long long row0 = (long long)blockIdx.x * GROUPS; row0 < n.rows; row0 += (long long)gridDim.x * GROUPS) {
    load(row0 + group);
    work(row0);
  }
#pragma unroll
  for (int which = 0; which < 4; ++which) {
    if ((LEAN && which % 2) || !(sums >> which & 1)) continue;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float (&s)[W] = which == 0 ? s0[v] : which == 1 ? s1[LEAN ? 0 : v] : which == 2 ? s2[v] : s3[LEAN ? 0 : v];
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
      if (c.any) store_w<FiraStoredF32, W>(partial + ((long long)which * gridDim.x + blockIdx.x) * n.dim + c.at, s);
    }
  }
}

// What the gradient's kernels read of a row's values.
template <typename T, typename P>
struct BlockRow {
  const typename T::raw *dr, *dy, *r, *b;
  float mu, rs, pm, ps;
  __device__ __forceinline__ BlockRow(const FiraBlockNorm& n, const typename T::raw* dr0, const typename T::raw* dy0, const typename T::raw* r0, const typename T::raw* b0,
                                      const FiraBlockStats& s, long long row) {
    dr = dr0 ? dr0 + row * n.ld_x : nullptr;
    dy = n.norm != kNone ? dy0 + row * n.ld_y : nullptr;
    r = n.norm != kNone ? r0 + row * n.ld_r : nullptr;
    b = b0 ? b0 + row * n.ld_b : nullptr;
    mu = n.norm == kLayer ? *as_global(s.mean + row) : 0.0f;
    rs = n.norm != kNone ? *as_global(s.rstd + row) : 1.0f;
    pm = n.post == kLayer ? *as_global(s.post_mean + row) : 0.0f;
    ps = n.post != kNone ? *as_global(s.post_rstd + row) : 1.0f;
  }
  __device__ __forceinline__ float h(long long c) const { return (load1<T>(r + c) - mu) * rs; }
  __device__ __forceinline__ float g(const FiraBlockVectors<P>& v, long long c) const { return load1<T>(dy + c) * (v.w ? load1<P>(v.w + c) : 1.0f); }
  // the gradient of r; s1, s2: the means of g and g h
  __device__ __forceinline__ float t(const FiraBlockVectors<P>& v, float s1, float s2, long long c) const {
    const float from = dr ? load1<T>(dr + c) : 0.0f;
    return dy ? from + rs * (g(v, c) - s1 - h(c) * s2) : from;
  }
  __device__ __forceinline__ float hb(long long c) const { return b ? (load1<T>(b + c) - pm) * ps : 0.0f; }
};

// Rows wider than kBlockWidest: a workgroup for a row, which it reads again for every sum, value by value.  means: of g and g h of every row, for the sums over rows, which read all of it once more (8192 x 16384
// bf16 2814 us and 637).
template <typename T, typename P>
__global__ __launch_bounds__(1024) void fira_block_norm_wide_rows_kernel(FiraBlockNorm n, const typename T::raw* dr, const typename T::raw* dy, const typename T::raw* r,
                                                                         const typename T::raw* b, FiraBlockVectors<P> v, FiraBlockStats stats, typename T::raw* dx,
                                                                         typename T::raw* db, float* means) {
  __shared__ float part[16];
  const float dim = (float)n.dim;
  for (long long row = blockIdx.x; row < n.rows; row += gridDim.x) {
    const BlockRow<T, P> at(n, dr, dy, r, b, stats, row);
    auto total = [&](auto f) {
      float s = 0.0f;
      for (long long c = threadIdx.x; c < n.dim; c += blockDim.x) s += f(c);
      return block_sum(s, part);
    };
    const float s1 = n.norm == kLayer ? total([&](long long c) { return at.g(v, c); }) / dim : 0.0f;
    const float s2 = n.norm != kNone ? total([&](long long c) { return at.g(v, c) * at.h(c); }) / dim : 0.0f;
    if (threadIdx.x == 0) { *as_global(means + 2 * row) = s1; *as_global(means + 2 * row + 1) = s2; }
    auto q = [&](long long c) {
      float x = n.alpha * at.t(v, s1, s2, c);
      if (v.gate) x *= load1<P>(v.gate + c);
      if (n.post != kNone && v.pw) x *= load1<P>(v.pw + c);
      return x;
    };
    const float q1 = db && n.post == kLayer ? total(q) / dim : 0.0f;
    const float q2 = db && n.post != kNone ? total([&](long long c) { return q(c) * at.hb(c); }) / dim : 0.0f;
    for (long long c = threadIdx.x; c < n.dim; c += blockDim.x) {
      if (dx) store1<T>(dx + row * n.ld_dx + c, n.beta * at.t(v, s1, s2, c));
      if (db) store1<T>(db + row * n.ld_db + c, n.post == kNone ? q(c) : at.ps * (q(c) - q1 - at.hb(c) * q2));
    }
  }
}

// Sums over rows, gridDim.y-th part of them: partial[k][blockIdx.y][dim] of dy h, dy, t h' and t.
template <typename T, typename P>
__global__ __launch_bounds__(256) void fira_block_norm_wide_sums_kernel(FiraBlockNorm n, const typename T::raw* dr, const typename T::raw* dy, const typename T::raw* r,
                                                                        const typename T::raw* b, FiraBlockVectors<P> v, FiraBlockStats stats, const float* means, float* partial) {
  const long long c = blockIdx.x * 256LL + threadIdx.x;
  if (c >= n.dim) return;
  float s[4] = {};
  for (long long row = blockIdx.y; row < n.rows; row += gridDim.y) {
    const BlockRow<T, P> at(n, dr, dy, r, b, stats, row);
    if (n.norm != kNone) {
      const float d = load1<T>(at.dy + c);
      s[0] += d * at.h(c);
      s[1] += d;
    }
    const float t = at.t(v, *as_global(means + 2 * row), *as_global(means + 2 * row + 1), c);
    s[2] += t * at.hb(c);
    s[3] += t;
  }
  for (int k = 0; k < 4; ++k) *as_global(partial + ((long long)k * gridDim.y + blockIdx.y) * n.dim + c) = s[k];
}

// The vectors' gradients from the sums S0 .. S3 over all rows: weight S0, bias S1, gate alpha (pw S2 + pb S3), post weight alpha gate S2, post bias alpha gate S3.
template <typename P>
struct FiraBlockGradients {
  typename P::raw *gate, *w, *b, *pw, *pb;
};
template <typename P>
__device__ __forceinline__ void block_vector_gradients(const FiraBlockNorm& n, const FiraBlockVectors<P>& v, const FiraBlockGradients<P>& to, const float (&s)[4], long long c,
                                                       int accumulate) {
  const float gate = v.gate ? load1<P>(v.gate + c) : 1.0f, pw = n.post != kNone && v.pw ? load1<P>(v.pw + c) : 1.0f, pb = n.post != kNone && v.pb ? load1<P>(v.pb + c) : 0.0f;
  auto put = [&](typename P::raw* p, float x) {
    if (p) store1<P>(p + c, accumulate ? load1<P>(p + c) + x : x);
  };
  put(to.w, s[0]);
  put(to.b, s[1]);
  put(to.gate, n.alpha * (pw * s[2] + pb * s[3]));
  put(to.pw, n.alpha * (gate * s[2]));
  put(to.pb, n.alpha * (gate * s[3]));
}
// Sums of the parts, for 16 columns a workgroup: four lanes of four columns, a part of the parts to each of the 64 sets of four lanes.
template <typename P>
__global__ __launch_bounds__(256) void fira_block_norm_join_kernel(FiraBlockNorm n, const float* partial, int parts, int sums, FiraBlockVectors<P> v, FiraBlockGradients<P> to,
                                                                   int accumulate) {
  constexpr int SETS = 64, N = 4;
  __shared__ float all[SETS][4][17];
  const int lane = threadIdx.x % 4, set = threadIdx.x / 4;
  const long long c0 = blockIdx.x * 16LL;
  const int cols = (int)min(16LL, n.dim - c0);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float s[4] = {};
    if (sums >> k & 1)
      for (int p0 = set; p0 < parts; p0 += SETS * N) {
        float x[N][4];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float* const from = partial + ((long long)k * parts + min(p0 + SETS * i, parts - 1)) * n.dim + c0;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = *as_global(from + min(j * 4 + lane, cols - 1));
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (p0 + SETS * i < parts)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += x[i][j];
      }
#pragma unroll
    for (int j = 0; j < 4; ++j) all[set][k][j * 4 + lane] = s[j];
  }
  __syncthreads();
  // a wavefront for each sum, four lanes to a column
  const int k = threadIdx.x >> 6, c = threadIdx.x & 15, quarter = (threadIdx.x & 63) >> 4;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < SETS / 4; ++i) s += all[quarter * (SETS / 4) + i][k][c];
  s = add_xor<16>(add_xor<32>(s));
  __syncthreads();
  if (quarter == 0) all[0][k][c] = s;
  __syncthreads();
  if (threadIdx.x >= cols) return;
  const float found[4] = {all[0][0][c], all[0][1][c], all[0][2][c], all[0][3][c]};
  block_vector_gradients(n, v, to, found, c0 + c, accumulate);
}
