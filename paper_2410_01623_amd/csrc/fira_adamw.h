// AdamW over the tensors of a list, with states in fp32 or in 8 bits.  gfx950 only.
#pragma once
#include "fira_rows.h"

#include <algorithm>

constexpr int kAdamBlock = 256;       // values that share a scale

// A piece of a tensor: n values, of the tensor's rows one after the other, from a whole block on.
struct FiraAdamSpan {
  void* w;                 // where the row of the first value begins, or with cols == 0 (no gaps) the value itself
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  long long ld_w, ld_g;
  double per_col;          // 1 / cols
  float weight_decay;
  unsigned n, cols, col0;  // col0: the first value's column
  unsigned first, seed;    // first: its place in the tensor, modulo 2^32
  int tile0;               // first tile of this piece
  int stream;              // results that begin at whole lines, and go past the caches: 1 weights, 2 states
};
constexpr int kAdamSpans = 36;        // (a lane for each.)  A launch's pieces travel as kernel arguments, of which there are 4 KB
// Vectors of a thread that are on their way together, and workgroups of a launch of `tiles`: with states in 8 bits and rows apart that are not whole vectors wide (APART), where code and
// registers are many, one and those of two tiles each, else two and nearly all that there could be.  us with one vector and two: 60m bf16 265 and 235, embeddings in 8 bits 280 and 260, 62 m
// values bf16 with fp32 gradients in 8 bits 195 and 177; 511 x 1377 and the like in 8 bits with rows apart 58 and 64.  With 8192, 16384 and 65536 workgroups: 60m 244, 235 and 230, those 62 m
// values 184, 177 and 175; with rows apart and 8192, two tiles each and one tile each: 62 m values fp32 in 8 bits 341, 288 and 315, bf16 231, 237 and 245.
template <bool EIGHT, bool APART>
constexpr int kAdamUnroll = EIGHT && APART ? 1 : 2;
template <bool EIGHT, bool APART>
int adam_workgroups(int tiles) { return std::min(tiles, EIGHT && APART ? std::min(std::max(8192, (tiles + 1) / 2), (1 << 24) - 1) : 65536); }   // (a launch has less than 2^32 threads)
struct FiraAdamSpans {
  FiraAdamSpan s[kAdamSpans];
  int count, tiles;
  int counts;              // the call's last launch, of few workgroups: counts the step
};
// Values of a thread's vector: 16 bytes of the widest type that is streamed, but with states in 8 bits 32 bytes of fp32 weights or gradients beside bf16 (us so and with 16: 512 x 1376 and
// the like, bf16 with fp32 gradients 40 and 51, fp32 with bf16 ones 44 and 55; all fp32 50 and 45).  APART: 16 bytes, since the joining of rows' ends takes registers (the
// former two, 511 x 1377 with rows apart, 83 and 65, 85 and 70).
template <typename T, typename R, bool EIGHT, bool APART>
constexpr int kAdamWidth = !EIGHT ? 4 : APART || sizeof(typename T::raw) + sizeof(typename R::raw) == 8 ? kWidth<T, R> : 8;

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
  long long taken;
};
// Called by two lanes or more: one for each beta.
__device__ __forceinline__ void adam_factors(FiraAdamFactors& f, const FiraAdamHp& hp, const float* lr, const float* norm, long long taken) {
  // (1 - b^t, without the cancellation of a beta next to one)
  const double rest = -expm1((double)(taken + 1) * (threadIdx.x ? hp.log_beta2 : hp.log_beta1));
  if (threadIdx.x == 1) f.v = (float)(1.0 / sqrt(rest));
  if (threadIdx.x) return;
  f.lr = lr ? (double)*as_global(lr) : hp.lr;
  f.m = (float)(f.lr / rest);
  f.cut = 1.0f;
  if (norm) {
    const float x = *as_global(norm);
    if ((double)x > hp.max_norm && x < INFINITY) f.cut = (float)(hp.max_norm / (double)x);
  }
  f.t = (unsigned)(taken + 1);
  f.taken = taken;
}

// A hash of 32 bits; the constants are the fractions of the roots of two and three.
__host__ __device__ __forceinline__ unsigned adam_mix(unsigned x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ x >> 16;
}

// New moments and weight of one value with states in fp32.  Each product and sum is rounded by itself, so that the moments are what elementary operations give.
__device__ __forceinline__ void adam_update(const FiraAdamHp& hp, const FiraAdamFactors& f, float decay, float g, float& w, float& m, float& v) {
#pragma clang fp contract(off)
  g *= f.cut;
  m = m * hp.b1 + g * hp.omb1;
  v = v * hp.b2 + g * g * hp.omb2;
  w = w * decay - (m * f.m) / (sqrtf(v) * f.v + hp.eps);
}

enum { kStreamed, kWhole, kEnd, kRows, kApart };

// Calls f with whether to stream as a constant, which where rows are apart is known at run time only.  What the compiler finds twice, with and without
// streaming, it makes one of plain stores: the empty statements keep it from that.
template <int PLACE, typename F>
__device__ __forceinline__ void either_way(bool stream, F f) {
  if (PLACE == kStreamed || ((PLACE == kApart || PLACE == kRows) && stream)) {
    asm volatile("" ::: "memory");
    f(std::true_type{});
    asm volatile("" ::: "memory");
  } else {
    f(std::false_type{});
  }
}

// W values of type T in their stored form, one by one.
template <typename T, int W>
__device__ __forceinline__ void adam_set(Raw<T, W>& x, int k, typename T::raw value) {
  if constexpr (sizeof(typename T::raw) == 4) x.a[k / 4][k % 4] = value;
  else x.a[0][k / 2] = k & 1 ? (x.a[0][k / 2] & 0xffffu) | (unsigned)value << 16 : (x.a[0][k / 2] & 0xffff0000u) | value;
}

// Values back .. back + W of a and then b, left in a.
template <typename T, int W>
__device__ __forceinline__ void adam_joined(Raw<T, W>& a, const Raw<T, W>& b, int back) {
  constexpr bool F32 = sizeof(typename T::raw) == 4;
  constexpr int N = F32 ? W : W / 2;                       // 32-bit words
  unsigned x[2 * N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (F32) { x[i] = __float_as_uint(a.a[i / 4][i % 4]); x[N + i] = __float_as_uint(b.a[i / 4][i % 4]); }
    else { x[i] = a.a[0][i]; x[N + i] = b.a[0][i]; }
  }
  const int words = F32 ? back : back / 2;                 // 0 to N - 1
#pragma unroll
  for (int by = N / 2; by; by /= 2)
#pragma unroll
    for (int i = 0; i < 2 * N - by; ++i) x[i] = words & by ? x[i + by] : x[i];
  if constexpr (!F32)
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = back & 1 ? __builtin_amdgcn_alignbit(x[i + 1], x[i], 16) : x[i];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (F32) a.a[i / 4][i % 4] = __uint_as_float(x[i]);
    else a.a[0][i] = x[i];
  }
}

// The larger one, no number if one of the two is none; and over the lanes that share a block.
__device__ __forceinline__ float adam_larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
template <int OFF>
__device__ __forceinline__ float max_xor(float x) {
  if constexpr (OFF < 16) {
    return adam_larger(x, lane_xor<OFF>(x));
  } else {
    const unsigned u = __float_as_uint(x);
    const u32x2_s s = OFF == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return adam_larger(__uint_as_float((unsigned)s[0]), __uint_as_float((unsigned)s[1]));
  }
}
template <int LANES>
__device__ __forceinline__ float adam_most(float x) {
  x = max_xor<1>(max_xor<2>(max_xor<4>(max_xor<8>(max_xor<16>(x)))));
  if constexpr (LANES == 64) x = max_xor<32>(x);
  return x;
}

// a / b, correctly rounded (1 / b of every mantissa and 2^30 random quotients compared) but for what leaves fp32's range on the way.
__device__ __forceinline__ float adam_quotient(float a, float b) {
  const float r = __builtin_amdgcn_rcpf(b);
  float q = a * r;
  q = __builtin_fmaf(__builtin_fmaf(-b, q, a), r, q);
  return __builtin_amdgcn_div_fixupf(q, b, a);
}

// Root of x in [2^-126, 2^127], correctly rounded from 2^-102 on (every mantissa compared; the rest that the estimate leaves is exact there, and below rounded, so that up to one in twelve is off by an
// ulp).  (Of less it is too small, of 0 it is 0, of what is not finite no number.)  The root instruction, which is off by an ulp, is 1 % faster at embeddings in 8 bits (274 us and 277); an ulp more
// or less now and then rounds a code to the other side, whose block has another largest size from the next step on.
__device__ __forceinline__ float adam_root(float x) {
  const float y = __builtin_amdgcn_rsqf(fmaxf(x, 0x1p-126f)), q = x * y;
  return __builtin_fmaf(__builtin_fmaf(-q, q, x), 0.5f * y, q);
}

// The same with states in 8 bits, S times the moment m and root of v (and by S less what they are multiplied with).
template <bool FINITE>
struct AdamScaled {
  float cut, fm, fv;
  __device__ __forceinline__ AdamScaled(const FiraAdamFactors& f, float S) : cut(f.cut * S), fm(f.m / S), fv(f.v / S) {}
  __device__ __forceinline__ void update(const FiraAdamHp& hp, float decay, float g, float& w, float& m, float& root) const {
#pragma clang fp contract(off)
    g *= cut;
    m = m * hp.b1 + g * hp.omb1;
    root = root * root * hp.b2 + g * g * hp.omb2;
    root = FINITE ? adam_root(root) : sqrtf(root);
    w = w * decay - adam_quotient(m * fm, root * fv + hp.eps);
  }
};

// Four values' e4m3 codes in an unsigned.  The conversion adds the high 20 bits of `random` below the three bits of mantissa that it keeps and cuts the rest off, in
// steps of 2^-9 below 2^-6.  (An immediate picks the byte.)
__device__ __forceinline__ float adam_value(unsigned codes, int k) {
  switch (k) {
    case 0: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 2);
    default: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 3);
  }
}
__device__ __forceinline__ unsigned adam_put(unsigned codes, float x, unsigned random, int k) {
  switch (k) {
    case 0: return (unsigned)__builtin_amdgcn_cvt_sr_fp8_f32(x, (int)random, (int)codes, 0);
    case 1: return (unsigned)__builtin_amdgcn_cvt_sr_fp8_f32(x, (int)random, (int)codes, 1);
    case 2: return (unsigned)__builtin_amdgcn_cvt_sr_fp8_f32(x, (int)random, (int)codes, 2);
    default: return (unsigned)__builtin_amdgcn_cvt_sr_fp8_f32(x, (int)random, (int)codes, 3);
  }
}

// A thread's values on their way: weights and gradients as they are stored, and the states, which have no gaps.
// PLACE: whole vectors of a piece without gaps, whose results go past the caches (kStreamed) or not (kWhole); such vectors or a part of one at the piece's end (kEnd); of a piece
// whose rows are apart and whole vectors wide (kRows), or of any width (kApart).
template <typename T, typename R, bool EIGHT, int W, int PLACE>
struct AdamVector {
  static constexpr bool JOIN = PLACE == kApart, APART = JOIN || PLACE == kRows, FULL = PLACE == kStreamed || PLACE == kWhole;
  Raw<T, W> w;
  Raw<R, W> g;
  unsigned m8[W / 4], v8[W / 4];
  f32x4 m, v;
  float ms, vs;
  unsigned j, row, col;    // place in the piece; row counted from the piece's first
  int here;                // values of the vector inside the piece
  bool whole;              // all W there, and neighbours

  static __device__ __forceinline__ void stream_bytes(unsigned (&to)[W / 4], const unsigned char* p) {
    typedef unsigned __attribute__((aligned(1))) u32_a1;
#pragma unroll
    for (int k = 0; k < W / 4; ++k) to[k] = __builtin_nontemporal_load((gptr<const u32_a1>)as_global(p + 4 * k));
  }

  __device__ __forceinline__ void load(const FiraAdamSpan& s, unsigned at) {
    j = at;
    here = FULL ? W : j < s.n ? (int)min((unsigned)W, s.n - j) : 0;
    row = 0;
    col = j;
    if constexpr (APART) {
      // (c + 1/2) / cols is 1 / (2 cols) from a whole number at least, which fp64 keeps apart
      const unsigned c = s.col0 + j;
      row = (unsigned)(((double)c + 0.5) * s.per_col);
      col = c - row * s.cols;
    }
    whole = here == W && (!JOIN || s.cols - col >= W);
    const typename T::raw* const pw = (const typename T::raw*)s.w + row * s.ld_w + col;
    const typename R::raw* const pg = (const typename R::raw*)s.g + row * s.ld_g + col;
    auto vectors = [&] {
      w.stream(pw);
      g.stream(pg);
      stream_states(s);
    };
    if constexpr (FULL) {
      vectors();
      return;
    }
    if (whole) vectors();
    if (JOIN && !whole && here == W && s.cols >= W) {
      // the end of a row and the beginning of the next
      const int back = (int)(col + W - s.cols);
      Raw<T, W> w2;
      Raw<R, W> g2;
      w.stream(pw - back);
      g.stream(pg - back);
      w2.stream(pw + (s.ld_w - (long long)col));
      g2.stream(pg + (s.ld_g - (long long)col));
      stream_states(s);
      adam_joined<T, W>(w, w2, back);
      adam_joined<R, W>(g, g2, back);
    }
    if (here < W || (JOIN && !whole && s.cols < W)) {
      // value by value, zeros where there are none
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const bool is = PLACE != kRows && k < here;        // (there, all are or none is)
        const unsigned down = JOIN && is ? (col + k) / s.cols : 0u;
        adam_set<T, W>(w, k, is ? *as_global(pw + k + down * (s.ld_w - s.cols)) : (typename T::raw)0);
        adam_set<R, W>(g, k, is ? *as_global(pg + k + down * (s.ld_g - s.cols)) : (typename R::raw)0);
        if constexpr (EIGHT) {
          if (k % 4 == 0) m8[k / 4] = v8[k / 4] = 0;
          m8[k / 4] |= (is ? (unsigned)*as_global((const unsigned char*)s.m + j + k) : 0u) << 8 * (k % 4);
          v8[k / 4] |= (is ? (unsigned)*as_global((const unsigned char*)s.v + j + k) : 0u) << 8 * (k % 4);
        } else {
          m[k] = is ? *as_global((const float*)s.m + j + k) : 0.0f;
          v[k] = is ? *as_global((const float*)s.v + j + k) : 0.0f;
        }
      }
      if constexpr (EIGHT) {
        ms = here ? *as_global(s.m_scale + j / kAdamBlock) : 0.0f;
        vs = here ? *as_global(s.v_scale + j / kAdamBlock) : 0.0f;
      }
    }
  }

  __device__ __forceinline__ void stream_states(const FiraAdamSpan& s) {
    if constexpr (EIGHT) {
      stream_bytes(m8, (const unsigned char*)s.m + j);
      stream_bytes(v8, (const unsigned char*)s.v + j);
      ms = *as_global(s.m_scale + j / kAdamBlock);
      vs = *as_global(s.v_scale + j / kAdamBlock);
    } else {
      m = __builtin_nontemporal_load((gptr<const f32x4_a4>)as_global((const float*)s.m + j));
      v = __builtin_nontemporal_load((gptr<const f32x4_a4>)as_global((const float*)s.v + j));
    }
  }

  __device__ __forceinline__ void put_weights(const FiraAdamSpan& s, const float (&x)[W]) const {
    typename T::raw* const pw = (typename T::raw*)s.w + row * s.ld_w + col;
    if (FULL || whole) {
      either_way<PLACE>(s.stream & 1, [&](auto stream) { store_w<T, W, decltype(stream)::value>(pw, x); });
      return;
    }
    const bool one = s.cols >= W;                          // (no second end of a row then)
#pragma unroll
    for (int k = 0; k < W; ++k)
      if (PLACE != kRows && k < here) store1<T>(pw + k + (!JOIN ? 0u : one ? (unsigned)(col + k >= s.cols) : (col + k) / s.cols) * (s.ld_w - s.cols), x[k]);
  }
  static __device__ __forceinline__ void put_bytes(unsigned char* p, const unsigned (&x)[W / 4], bool stream) {
    typedef unsigned __attribute__((aligned(1))) u32_a1;
    either_way<PLACE>(stream, [&](auto past) {
#pragma unroll
      for (int k = 0; k < W / 4; ++k) {
        if constexpr (decltype(past)::value) __builtin_nontemporal_store(x[k], (gptr<u32_a1>)as_global(p + 4 * k));
        else *(gptr<u32_a1>)as_global(p + 4 * k) = x[k];
      }
    });
  }

  __device__ __forceinline__ void step_f32(const FiraAdamSpan& s, const FiraAdamHp& hp, const FiraAdamFactors& f, float decay) {
    float ow[W], om[W], ov[W];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ow[k] = w.get(k);
      om[k] = m[k];
      ov[k] = v[k];
      adam_update(hp, f, decay, g.get(k), ow[k], om[k], ov[k]);
    }
    put_weights(s, ow);
    if (FULL || here == W) {
      either_way<PLACE>(s.stream & 2, [&](auto stream) {
        store_w<FiraStoredF32, W, decltype(stream)::value>((float*)s.m + j, om);
        store_w<FiraStoredF32, W, decltype(stream)::value>((float*)s.v + j, ov);
      });
    } else {
#pragma unroll
      for (int k = 0; k < W - 1; ++k)
        if (PLACE != kRows && k < here) {
          *as_global((float*)s.m + j + k) = om[k];
          *as_global((float*)s.v + j + k) = ov[k];
        }
    }
  }

  // All that is of the gradients' size is held times 2^40, so that squares of roots down to 2^-103, below all that a block's scale is kept for, stay above 2^-126; where a product
  // leaves fp32's range for that (roots above 2^24), the value is worked out again without.
  __device__ __forceinline__ void step_e4m3(const FiraAdamSpan& s, const FiraAdamHp& hp, const FiraAdamFactors& f, float decay, unsigned key) {
    constexpr int LANES = kAdamBlock / W;
    constexpr float kMost = 0x1p120f;
    float S = 0x1p40f;
    const AdamScaled<true> scaled(f, S);
    float ow[W], om[W], root[W];
    float mm = 0.0f, mv = 0.0f;                            // the block's largest
    const float sm = ms * S, sv = vs * S;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ow[k] = w.get(k);
      om[k] = adam_value(m8[k / 4], k % 4) * sm;
      root[k] = adam_value(v8[k / 4], k % 4) * sv;
      scaled.update(hp, decay, g.get(k), ow[k], om[k], root[k]);
      mm = adam_larger(mm, fabsf(om[k]));
      mv = adam_larger(mv, root[k]);
    }
    mm = adam_most<LANES>(mm);
    mv = adam_most<LANES>(mv);
    bool lost_m[W] = {}, lost_v[W] = {};                   // what is not finite
    if (__any(!(adam_larger(mm, mv) < kMost))) {
      const AdamScaled<false> plain(f, 1.0f);
      mm = mv = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const bool fine = fabsf(om[k]) < INFINITY && root[k] < INFINITY;
        float w1 = w.get(k), m1 = adam_value(m8[k / 4], k % 4) * ms, r1 = adam_value(v8[k / 4], k % 4) * vs;
        plain.update(hp, decay, g.get(k), w1, m1, r1);
        ow[k] = fine ? ow[k] : w1;
        om[k] = fine ? om[k] * (1.0f / S) : m1;
        root[k] = fine ? root[k] * (1.0f / S) : r1;
        lost_m[k] = !(fabsf(om[k]) < INFINITY);
        lost_v[k] = !(root[k] < INFINITY);
        mm = adam_larger(mm, lost_m[k] ? 0.0f : fabsf(om[k]));
        mv = adam_larger(mv, lost_v[k] ? 0.0f : root[k]);
      }
      mm = adam_most<LANES>(mm);
      mv = adam_most<LANES>(mv);
      S = 1.0f;
    }
    const bool none_m = mm < 0x1p-100f * S, none_v = mv < 0x1p-100f * S;
    // (the reciprocal instruction has results below 2^-126 as zero)
    const float down_m = mm < kMost ? 1.0f : 0x1p-32f, down_v = mv < kMost ? 1.0f : 0x1p-32f;
    const float up_m = none_m ? 0.0f : adam_quotient(1.0f, mm * down_m) * 448.0f * down_m, up_v = none_v ? 0.0f : adam_quotient(1.0f, mv * down_v) * 448.0f * down_v;
    unsigned cm[W / 4] = {}, cv[W / 4] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const unsigned random = adam_mix(s.first + j + k + key);
      const float a = __builtin_amdgcn_fmed3f(om[k] * up_m, -448.0f, 448.0f);
      float b = root[k] * up_v;
      b = b > 0.0f ? __builtin_amdgcn_fmed3f(b, 0x1p-9f, 448.0f) : 0.0f;   // (at least the smallest code, which is not rounded down)
      cm[k / 4] = adam_put(cm[k / 4], a, random << 16 | 0x8000u, k % 4);
      cv[k / 4] = adam_put(cv[k / 4], b, (random & 0xffff0000u) | 0x8000u, k % 4);
      if (lost_m[k]) cm[k / 4] |= 127u << 8 * (k % 4);
      if (lost_v[k]) cv[k / 4] |= 127u << 8 * (k % 4);
    }
    put_weights(s, ow);
    if (FULL || here == W) {
      put_bytes((unsigned char*)s.m + j, cm, s.stream & 2);
      put_bytes((unsigned char*)s.v + j, cv, s.stream & 2);
    } else {
#pragma unroll
      for (int k = 0; k < W - 1; ++k)
        if (PLACE != kRows && k < here) {
          *as_global((unsigned char*)s.m + j + k) = (unsigned char)(cm[k / 4] >> 8 * (k % 4));
          *as_global((unsigned char*)s.v + j + k) = (unsigned char)(cv[k / 4] >> 8 * (k % 4));
        }
    }
    if (here && j % kAdamBlock == 0) {
      *as_global(s.m_scale + j / kAdamBlock) = none_m ? 0.0f : mm * (1.0f / 448.0f) / S;
      *as_global(s.v_scale + j / kAdamBlock) = none_v ? 0.0f : mv * (1.0f / 448.0f) / S;
    }
  }
};

// A workgroup takes every gridDim.x-th tile of 256 threads times kAdamUnroll vectors; the lanes that hold a block of 256 values find its scale between them.
// With fp32 states bound by memory: 60m bf16 with fp32 gradients 232 us (6.0 TB/s).  With states in 8 bits by vector instructions, about 70 a value, which at four cycles each take all cycles of the SIMDs at
// embeddings bf16 (270 us, 4.9 TB/s; 330 and more in the first passes after a pause, until the clock is up), 0.93 of them at 62 m values bf16 with fp32 gradients (176) and, with rows apart, whose ends are joined,
// 0.93 at 511 x 1377 and the like f32 (58, dense 47) and 0.89 at bf16 (57, dense 41).
// APART: some pieces' rows are, and not whole vectors wide.
template <typename T, typename R, bool EIGHT, bool APART>
__global__ __launch_bounds__(256) void fira_adamw_kernel(FiraAdamSpans l, FiraAdamHp hp, const float* lr, const float* norm, long long* counter) {
  constexpr int W = kAdamWidth<T, R, EIGHT, APART>, TILE = 256 * W * kAdamUnroll<EIGHT, APART>;
  __shared__ FiraAdamFactors shared;
  // (the other wavefronts' first loads are on their way meanwhile)
  if (threadIdx.x < 2) adam_factors(shared, hp, lr, norm, *as_global(counter));
  bool ready = false;
  FiraAdamFactors f;
  const int lane = threadIdx.x & 63, begins = lane < l.count ? l.s[lane].tile0 : 0x7fffffff;
#pragma unroll 1
  for (int tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
    const int k = __builtin_amdgcn_readfirstlane(__popcll(__ballot(begins <= tile)) - 1);      // the last piece that does not begin after the tile
    const FiraAdamSpan& s = l.s[k];
    const unsigned first = (unsigned)(tile - s.tile0) * TILE;
    // vectors that are on their way together: one where there are ends to look for, which take registers and branches
    auto work = [&](auto place, auto together) {
      constexpr int N = decltype(together)::value;
#pragma unroll 1
      for (int u0 = 0; u0 < kAdamUnroll<EIGHT, APART>; u0 += N) {
        AdamVector<T, R, EIGHT, W, decltype(place)::value> x[N];
#pragma unroll
        for (int u = 0; u < N; ++u) x[u].load(s, first + ((u0 + u) * 256 + threadIdx.x) * W);
        if (!ready) {
          __syncthreads();
          f = shared;
          ready = true;
          // the last workgroup to have read the count raises it
          if (l.counts && threadIdx.x == 0 &&
              __hip_atomic_fetch_add(counter + 1, 1LL, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (long long)gridDim.x - 1) {
            *as_global(counter + 1) = 0;
            *as_global(counter) = f.taken + 1;
          }
        }
        const float decay = (float)(1.0 - f.lr * (double)s.weight_decay);
        const unsigned key = adam_mix(adam_mix(s.seed) + f.t);
#pragma unroll
        for (int u = 0; u < N; ++u) {
          if constexpr (EIGHT) x[u].step_e4m3(s, hp, f, decay, key);
          else x[u].step_f32(s, hp, f, decay);
        }
      }
    };
    typedef std::integral_constant<int, kAdamUnroll<EIGHT, APART>> All;
    typedef std::integral_constant<int, 1> One;
    if constexpr (APART)
      if (s.cols % kMostWidth) {
        work(std::integral_constant<int, kApart>{}, One{});
        continue;
      }
    if (s.cols) work(std::integral_constant<int, kRows>{}, One{});
    else if (s.n - first < (unsigned)TILE) work(std::integral_constant<int, kEnd>{}, One{});
    else if (s.stream == 3) work(std::integral_constant<int, kStreamed>{}, All{});
    else work(std::integral_constant<int, kWhole>{}, All{});
  }
}

// Counting the step in the last launch saves a launch, but its workgroups queue at one address.  us in a graph so and with a launch for it: 17 vectors 4.6 and 5.4, 64 workgroups 5.2 and 5.1 (states
// in 8 bits 6.2 and 6.2), 128 6.6 and 5.3, 256 9.5 and 5.8, 512 19.9 and 6.9; call by call, 17 vectors 7.6 and 9.3.
constexpr int kAdamCounting = 64;
template <typename = void>
__global__ void fira_adamw_count_kernel(long long* taken) { *as_global(taken) += 1; }
