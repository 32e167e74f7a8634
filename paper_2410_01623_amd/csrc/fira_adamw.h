// AdamW over the tensors of a list, with states in fp32 or in 8 bits.  gfx950 only.
#pragma once
#include "fira_rows.h"

constexpr int kAdamBlock = 256;       // values that share a scale

// A piece of a tensor: n values, of the tensor's rows one after the other, from a whole block on.
struct FiraAdamSpan {
  void* w;                 // where the row of the first value begins, or with cols == 0 (no gaps) the value itself
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  long long ld_w, ld_g;
  double weight_decay;
  unsigned n, cols, col0;  // col0: the first value's column
  unsigned first, seed;    // first: its place in the tensor, modulo 2^32
  int tile0;               // first tile of this piece
};
constexpr int kAdamSpans = 40;        // a launch's pieces travel as kernel arguments, of which there are 4 KB
constexpr int kAdamUnroll = 2;        // vectors of a thread that are on their way together
constexpr int kAdamWorkgroups = 2048;
struct FiraAdamSpans {
  FiraAdamSpan s[kAdamSpans];
  int count, tiles;
  int each;                // tiles of a workgroup
  int last;                // the call's last launch: counts the step
};
// Values of a thread's vector and of a tile: 16 bytes of the widest type that is streamed.
template <typename T, typename R, bool EIGHT>
constexpr int kAdamWidth = EIGHT ? kWidth<T, R> : 4;

struct FiraAdamHp {
  double lr, log_beta1, log_beta2, max_norm;
  float b1, b2, omb1, omb2, eps;
};
static_assert(sizeof(FiraAdamSpans) + sizeof(FiraAdamHp) + 64 <= 4096, "kernel arguments");

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

// W values of type T in their stored form, one by one.
template <typename T, int W>
__device__ __forceinline__ void adam_set(Raw<T, W>& x, int k, typename T::raw value) {
  if constexpr (sizeof(typename T::raw) == 4) x.a[k / 4][k % 4] = value;
  else x.a[0][k / 2] = k & 1 ? (x.a[0][k / 2] & 0xffffu) | (unsigned)value << 16 : (x.a[0][k / 2] & 0xffff0000u) | value;
}

// Largest over the lanes that share a block.
template <int LANES>
__device__ __forceinline__ float adam_most(float x) {
#pragma unroll
  for (int d = LANES / 2; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
  return x;
}

// A thread's values on their way: weights and gradients as they are stored, and the states, which have no gaps.
template <typename T, typename R, bool EIGHT, int W>
struct AdamVector {
  Raw<T, W> w;
  Raw<R, W> g;
  unsigned m8[W / 4], v8[W / 4];
  f32x4 m, v;
  float ms, vs;
  unsigned j, row, col;    // place in the piece; row counted from the piece's first
  int here;                // values of the vector inside the piece
  bool whole;              // all W there, and neighbours

  __device__ __forceinline__ void load(const FiraAdamSpan& s, unsigned at) {
    j = at;
    here = j < s.n ? (int)min((unsigned)W, s.n - j) : 0;
    row = 0;
    col = j;
    if (s.cols) {
      const unsigned c = s.col0 + j;
      row = c / s.cols;
      col = c - row * s.cols;
    }
    whole = here == W && (!s.cols || s.cols - col >= W);
    const typename T::raw* const pw = (const typename T::raw*)s.w + row * s.ld_w + col;
    const typename R::raw* const pg = (const typename R::raw*)s.g + row * s.ld_g + col;
    if (whole) {
      w.stream(pw);
      g.stream(pg);
    } else if (here) {
#pragma unroll
      for (int k = 0; k < W; ++k) {
        long long ow = k, og = k;
        if (k < here && s.cols) {
          const unsigned down = (col + k) / s.cols;
          ow += down * (s.ld_w - s.cols);
          og += down * (s.ld_g - s.cols);
        }
        adam_set<T, W>(w, k, k < here ? *as_global(pw + ow) : (typename T::raw)0);
        adam_set<R, W>(g, k, k < here ? *as_global(pg + og) : (typename R::raw)0);
      }
    }
    if constexpr (EIGHT) {
      typedef unsigned __attribute__((aligned(1))) u32_a1;
      const unsigned char *const pm = (const unsigned char*)s.m + j, *const pv = (const unsigned char*)s.v + j;
      if (here == W) {
#pragma unroll
        for (int k = 0; k < W / 4; ++k) {
          m8[k] = __builtin_nontemporal_load((gptr<const u32_a1>)as_global(pm + 4 * k));
          v8[k] = __builtin_nontemporal_load((gptr<const u32_a1>)as_global(pv + 4 * k));
        }
      } else {
#pragma unroll
        for (int k = 0; k < W / 4; ++k) m8[k] = v8[k] = 0;
#pragma unroll
        for (int k = 0; k < W; ++k)
          if (k < here) {
            m8[k / 4] |= (unsigned)*as_global(pm + k) << 8 * (k % 4);
            v8[k / 4] |= (unsigned)*as_global(pv + k) << 8 * (k % 4);
          }
      }
      ms = here ? *as_global(s.m_scale + j / kAdamBlock) : 0.0f;
      vs = here ? *as_global(s.v_scale + j / kAdamBlock) : 0.0f;
    } else {
      const float *const pm = (const float*)s.m + j, *const pv = (const float*)s.v + j;
      if (here == W) {
        m = __builtin_nontemporal_load((gptr<const f32x4_a4>)as_global(pm));
        v = __builtin_nontemporal_load((gptr<const f32x4_a4>)as_global(pv));
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          m[k] = k < here ? *as_global(pm + k) : 0.0f;
          v[k] = k < here ? *as_global(pv + k) : 0.0f;
        }
      }
    }
  }

  __device__ __forceinline__ void step(const FiraAdamSpan& s, const FiraAdamHp& hp, const FiraAdamFactors& f, float decay, unsigned key) {
    float ow[W], om[W], ov[W], root[W];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ow[k] = w.get(k);
      if constexpr (EIGHT) {
        // (an immediate picks the byte)
        const float held[2] = {byte_value(m8[k / 4], k % 4), byte_value(v8[k / 4], k % 4)};
        om[k] = held[0] * ms;
        root[k] = held[1] * vs;
        ov[k] = root[k] * root[k];
      } else {
        om[k] = m[k];
        ov[k] = v[k];
      }
      adam_update(hp, f, decay, g.get(k), ow[k], om[k], ov[k], root[k]);
    }
    typename T::raw* const pw = (typename T::raw*)s.w + row * s.ld_w + col;
    if (whole) {
      store_w<T, W, true>(pw, ow);
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k)
        if (k < here) store1<T>(pw + k + (s.cols ? (col + k) / s.cols * (s.ld_w - s.cols) : 0), ow[k]);
    }
    if constexpr (EIGHT) {
      constexpr int LANES = kAdamBlock / W;
      float mm = 0.0f, mv = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        mm = fmaxf(mm, k < here ? adam_size(om[k]) : 0.0f);
        mv = fmaxf(mv, k < here ? adam_size(root[k]) : 0.0f);
      }
      mm = adam_most<LANES>(mm);
      mv = adam_most<LANES>(mv);
      const float up_m = adam_up(mm), up_v = adam_up(mv);
      unsigned cm[W / 4] = {}, cv[W / 4] = {};
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const unsigned random = adam_mix(s.first + j + k + key);
        cm[k / 4] |= adam_code<false>(om[k], up_m, random & 0xffffu) << 8 * (k % 4);
        cv[k / 4] |= adam_code<true>(root[k], up_v, random >> 16) << 8 * (k % 4);
      }
      unsigned char *const pm = (unsigned char*)s.m + j, *const pv = (unsigned char*)s.v + j;
      if (here == W) {
        typedef unsigned __attribute__((aligned(1))) u32_a1;
#pragma unroll
        for (int k = 0; k < W / 4; ++k) {
          __builtin_nontemporal_store(cm[k], (gptr<u32_a1>)as_global(pm + 4 * k));
          __builtin_nontemporal_store(cv[k], (gptr<u32_a1>)as_global(pv + 4 * k));
        }
      } else {
#pragma unroll
        for (int k = 0; k < W; ++k)
          if (k < here) {
            *as_global(pm + k) = (unsigned char)(cm[k / 4] >> 8 * (k % 4));
            *as_global(pv + k) = (unsigned char)(cv[k / 4] >> 8 * (k % 4));
          }
      }
      if (here && j % kAdamBlock == 0) {
        *as_global(s.m_scale + j / kAdamBlock) = adam_scale(mm);
        *as_global(s.v_scale + j / kAdamBlock) = adam_scale(mv);
      }
    } else {
      float *const pm = (float*)s.m + j, *const pv = (float*)s.v + j;
      if (here == W) {
        store_w<FiraStoredF32, W, true>(pm, om);
        store_w<FiraStoredF32, W, true>(pv, ov);
      } else {
#pragma unroll
        for (int k = 0; k < W; ++k)
          if (k < here) { *as_global(pm + k) = om[k]; *as_global(pv + k) = ov[k]; }
      }
    }
  }

  static __device__ __forceinline__ float byte_value(unsigned codes, int k) {
    switch (k) {
      case 0: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 0);
      case 1: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 1);
      case 2: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 2);
      default: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 3);
    }
  }
};

// A workgroup takes tiles that adjoin, of 256 threads times kAdamUnroll vectors; the lanes that hold a block of 256 values find its scale between them.
template <typename T, typename R, bool EIGHT>
__global__ __launch_bounds__(256) void fira_adamw_kernel(FiraAdamSpans l, FiraAdamHp hp, const float* lr, const float* norm, long long* counter) {
  constexpr int W = kAdamWidth<T, R, EIGHT>, TILE = 256 * W * kAdamUnroll;
  __shared__ FiraAdamFactors shared;
  if (threadIdx.x == 0) shared = adam_factors(hp, lr, norm, *as_global(counter));
  __syncthreads();
  const FiraAdamFactors f = shared;
  const int from = blockIdx.x * l.each, until = min(from + l.each, l.tiles);
  int k = 0;                                             // the last piece that does not begin after the first tile
#pragma unroll 1
  for (int step = 32; step; step >>= 1)
    if (k + step < l.count && l.s[k + step].tile0 <= from) k += step;
#pragma unroll 1
  for (int tile = from; tile < until; ++tile) {
    while (k + 1 < l.count && l.s[k + 1].tile0 <= tile) ++k;
    k = __builtin_amdgcn_readfirstlane(k);
    const FiraAdamSpan& s = l.s[k];
    const unsigned first = (unsigned)(tile - s.tile0) * TILE;
    AdamVector<T, R, EIGHT, W> x[kAdamUnroll];
#pragma unroll
    for (int u = 0; u < kAdamUnroll; ++u) x[u].load(s, first + (u * 256 + threadIdx.x) * W);
    const float decay = (float)(1.0 - f.lr * s.weight_decay);
    const unsigned key = adam_mix(adam_mix(s.seed) + f.t);
#pragma unroll
    for (int u = 0; u < kAdamUnroll; ++u) x[u].step(s, hp, f, decay, key);
  }
}

template <typename = void>
__global__ void fira_adamw_count_kernel(long long* taken) { *as_global(taken) += 1; }
