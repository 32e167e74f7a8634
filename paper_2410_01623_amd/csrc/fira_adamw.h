// AdamW over the tensors of a list, with states in fp32 or in 8 bits.  gfx950 only.
#pragma once
#include "fira_rows.h"

constexpr int kAdamBlock = 256;       // values that share a scale

struct FiraAdamTensor {
  void* w;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  long long n, cols, ld_w, ld_g;
  double weight_decay;
  unsigned seed;
};
struct FiraAdamHp {
  double lr, log_beta1, log_beta2, max_norm;
  float b1, b2, omb1, omb2, eps;
};

// What a step multiplies by: 1 / (1 - b1^t) and the learning rate, 1 / sqrt(1 - b2^t), the factor that cuts the gradients, and t.
struct FiraAdamFactors {
  double lr;
  float m, v, cut;
  unsigned t;
};
__device__ __forceinline__ FiraAdamFactors adam_factors(const FiraAdamHp& hp, const float* lr, const float* norm, long long taken) {
  FiraAdamFactors f;
  const double t = (double)(taken + 1);
  f.lr = lr ? (double)*as_global(lr) : hp.lr;
  // (1 - b^t, without the cancellation of a beta next to one)
  f.m = (float)(f.lr / -expm1(t * hp.log_beta1));
  f.v = (float)(1.0 / sqrt(-expm1(t * hp.log_beta2)));
  f.cut = 1.0f;
  if (norm) {
    const float x = *as_global(norm);
    if ((double)x > hp.max_norm && x < INFINITY) f.cut = (float)(hp.max_norm / (double)x);
  }
  f.t = (unsigned)(taken + 1);
  return f;
}

// A hash of 32 bits; the constants are the fractions of the roots of two and three.
__host__ __device__ __forceinline__ unsigned adam_mix(unsigned x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ x >> 16;
}

// The e4m3 code of x (times `up` in [0, 448], but for what is not finite: NaN), rounded up where `random` says so: it is added below the three bits of
// mantissa that are kept, after which the rest is cut off.  Subnormal codes have the steps of the lowest normal ones, [2^-6, 2^-5), and are counted there.
// FLOOR: what is above zero stays so.
template <bool FLOOR>
__device__ __forceinline__ unsigned adam_code(float x, float up, unsigned random) {
  const float a = fminf(fabsf(x) * up, 448.0f);
  const bool below = a < 0x1p-6f;
  unsigned code = ((__float_as_uint(below ? a + 0x1p-6f : a) + (random << 4) + 8u) >> 20) - (below ? 968u : 960u);
  if (FLOOR) code = a > 0.0f ? max(code, 1u) : code;
  code |= __float_as_uint(x) >> 31 << 7;
  return fabsf(x) < INFINITY ? code : 127u;
}
__device__ __forceinline__ float adam_value(unsigned code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }
__device__ __forceinline__ float adam_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }
__device__ __forceinline__ float adam_up(float most) { return most < 0x1p-100f ? 0.0f : 448.0f / most; }
__device__ __forceinline__ float adam_scale(float most) { return most < 0x1p-100f ? 0.0f : most / 448.0f; }

// New moments and weight of one value; root = sqrt(v).  Each product and sum is rounded by itself, so that the moments are what elementary operations in fp32 give.
__device__ __forceinline__ void adam_update(const FiraAdamHp& hp, const FiraAdamFactors& f, float decay, float g, float& w, float& m, float& v, float& root) {
#pragma clang fp contract(off)
  g *= f.cut;
  m = m * hp.b1 + g * hp.omb1;
  v = v * hp.b2 + g * g * hp.omb2;
  root = sqrtf(v);
  w = w * decay - (m * f.m) / (root * f.v + hp.eps);
}

// A workgroup for 256 values at a time, a value to a thread.
template <typename T, typename R, bool EIGHT>
__global__ __launch_bounds__(kAdamBlock) void fira_adamw_kernel(FiraAdamTensor a, FiraAdamHp hp, const float* lr, const float* norm, const long long* taken) {
  __shared__ float most[2][4];
  const FiraAdamFactors f = adam_factors(hp, lr, norm, *as_global(taken));
  const float decay = (float)(1.0 - f.lr * a.weight_decay);
  const unsigned key = adam_mix(adam_mix(a.seed) + f.t);
  for (long long b = blockIdx.x; b * kAdamBlock < a.n; b += gridDim.x) {
    const long long i = b * kAdamBlock + threadIdx.x;
    const bool here = i < a.n;
    const long long row = here ? i / a.cols : 0, col = here ? i - row * a.cols : 0;
    typename T::raw* const to = (typename T::raw*)a.w + row * a.ld_w + col;
    float w = 0.0f, m = 0.0f, v = 0.0f, root = 0.0f;
    if (here) {
      w = load1<T>(to);
      if (EIGHT) {
        m = adam_value(*as_global((const unsigned char*)a.m + i)) * *as_global(a.m_scale + b);
        root = adam_value(*as_global((const unsigned char*)a.v + i)) * *as_global(a.v_scale + b);
        v = root * root;
      } else {
        m = *as_global((const float*)a.m + i);
        v = *as_global((const float*)a.v + i);
      }
      adam_update(hp, f, decay, load1<R>((const typename R::raw*)a.g + row * a.ld_g + col), w, m, v, root);
      store1<T>(to, w);
    }
    if (!EIGHT) {
      if (here) { *as_global((float*)a.m + i) = m; *as_global((float*)a.v + i) = v; }
      continue;
    }
    float mm = adam_size(m), mv = adam_size(root);
    for (int d = 32; d; d >>= 1) { mm = fmaxf(mm, __shfl_xor(mm, d, 64)); mv = fmaxf(mv, __shfl_xor(mv, d, 64)); }
    if ((threadIdx.x & 63) == 0) { most[0][threadIdx.x >> 6] = mm; most[1][threadIdx.x >> 6] = mv; }
    __syncthreads();
    mm = fmaxf(fmaxf(most[0][0], most[0][1]), fmaxf(most[0][2], most[0][3]));
    mv = fmaxf(fmaxf(most[1][0], most[1][1]), fmaxf(most[1][2], most[1][3]));
    __syncthreads();
    if (here) {
      const unsigned random = adam_mix((unsigned)i + key);
      *as_global((unsigned char*)a.m + i) = (unsigned char)adam_code<false>(m, adam_up(mm), random & 0xffffu);
      *as_global((unsigned char*)a.v + i) = (unsigned char)adam_code<true>(root, adam_up(mv), random >> 16);
    }
    if (threadIdx.x == 0) { *as_global(a.m_scale + b) = adam_scale(mm); *as_global(a.v_scale + b) = adam_scale(mv); }
  }
}

template <typename = void>
__global__ void fira_adamw_count_kernel(long long* taken) { *as_global(taken) += 1; }
