// Rotary positions and their gradient.  gfx950 only.
#pragma once
#include "fira_rows.h"

constexpr int kRotaryTensors = 4;
struct FiraRotaryTensor {
  const void* x;
  void* y;
  long long xs[3], ys[3];        // strides of sequences, tokens and heads
};
struct FiraRotary {
  FiraRotaryTensor t[kRotaryTensors];
  int first[kRotaryTensors];     // first head of each tensor, of all tensors' heads one after the other (not for the wide kernel, which takes one tensor)
  int count;
  unsigned token0, tokens;       // first token of a launch, and tokens of all sequences
  unsigned length;               // of a sequence
  long long position_stride;
  int half, rotated, copied;     // copied: values of a head that are not turned, none in place
  float scale, sign;             // sign: -1 for the gradient
  int wide;                      // positions of 64 bits
  // A unit is what a thread turns or copies at a time: W pairs as two vectors of W values, where pairs are interleaved one vector of W values (two with W = 1), or one that is
  // copied.  (Two neighbouring vectors a lane leave every load half a line: 65536 tokens of 32 heads of 128, bf16, interleaved 254 us so and 184 with one.)  A workgroup
  // takes `tile` tokens and of each `chunk` of the units of all heads.  Where a part of a head is no whole number of vectors, its last vector starts earlier and turns values that its neighbour
  // turns as well; a workgroup takes whole heads then, and has loaded all that it takes before it stores, so that this holds in place too (16384 tokens of 20 heads of 50, bf16, 32 us value
  // by value and 16 so; heads of 130 149 and 38).
  unsigned units, turned;        // of a head, and those of them that are turned
  unsigned all, tile, chunk, chunks;
  unsigned per_chunk, per_units; // 2^32 / chunk and 2^32 / units, rounded up
};
constexpr unsigned kRotaryTile = 128;         // most tokens of a workgroup
constexpr unsigned kRotaryTable = 2048;       // most pairs of all its tokens

// cos and sin of position times frequency, times the scale.  The angle is brought to a part of a turn in fp64; what is left fits fp32.
__device__ __forceinline__ void rotary_turn(long long position, double frequency, float scale, float sign, float& c, float& s) {
  const double turns = (double)position * frequency * 0.15915494309189533577;
  float sn, cs;
  sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
  c = scale * cs;
  s = sign * scale * sn;
}
// x / d for x d < 2^32
__device__ __forceinline__ unsigned rotary_quotient(unsigned x, unsigned d, unsigned per_d) { return d == 1 ? x : __umulhi(x, per_d); }

// First value of a unit that is turned.  OVERLAP: vectors may.
template <int W, bool INTERLEAVED, bool OVERLAP = true>
__host__ __device__ __forceinline__ unsigned rotary_place(const FiraRotary& r, unsigned unit) {
  if (INTERLEAVED && W == 1) return 2 * unit;
  if (!OVERLAP) return unit * W;
  const unsigned last = (unsigned)((INTERLEAVED ? r.rotated : r.half) - W);
  return unit * W < last ? unit * W : last;
}

// The sines and cosines of a workgroup's tokens are worked out once, for all heads, into LDS, while the values are on their way.  N: units of a thread.  STREAM: past the caches, and no vectors that overlap; but for halves
// that are no whole lines, which the caches put together (131072 tokens of 64 heads of 64, bf16: 438 us and 392 with them; heads of 128: 184 and 199).  Bound by memory.
template <typename T, int W, int N, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(256) void fira_rotary_kernel(FiraRotary r, const double* frequencies, const void* positions) {
  typedef typename T::raw raw;
  constexpr bool TWO = !INTERLEAVED || W == 1;             // a unit has two vectors
  __shared__ long long place[kRotaryTile];
  __shared__ unsigned long long from[kRotaryTensors][kRotaryTile], to[kRotaryTensors][kRotaryTile];
  __shared__ __attribute__((aligned(16))) float cosines[kRotaryTable], sines[kRotaryTable];
  const unsigned t0 = r.token0 + blockIdx.x / r.chunks * r.tile, c0 = blockIdx.x % r.chunks * r.chunk;
  const unsigned tokens = min(r.tile, r.tokens - t0), here = min(r.chunk, r.all - c0), head0 = c0 / r.units, unit0 = c0 - head0 * r.units;
  for (unsigned i = threadIdx.x; i < tokens * (unsigned)r.count; i += 256) {
    const unsigned k = i / tokens, t = i - k * tokens, batch = (t0 + t) / r.length, token = t0 + t - batch * r.length;
    const FiraRotaryTensor& x = r.t[k];
    from[k][t] = (unsigned long long)x.x + (batch * x.xs[0] + token * x.xs[1]) * (long long)sizeof(raw);
    to[k][t] = (unsigned long long)x.y + (batch * x.ys[0] + token * x.ys[1]) * (long long)sizeof(raw);
    if (k) continue;
    const long long p = batch * r.position_stride + token;
    place[t] = !positions ? (long long)token : r.wide ? *as_global((const long long*)positions + p) : (long long)*as_global((const int*)positions + p);
  }
  __syncthreads();
  auto fetch = [](Raw<T, W>& v, const raw* p) {
    if constexpr (STREAM) v.stream(p);
    else v.load(p);
  };
  Raw<T, W> a[N], b[N];
  raw* out[N];
  unsigned unit[N], row[N];
  bool is[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const unsigned i = n * 256 + threadIdx.x, t = rotary_quotient(i, r.chunk, r.per_chunk), c = i - t * r.chunk;
    is[n] = t < tokens && c < here;
    if (!is[n]) continue;
    const unsigned head = rotary_quotient(unit0 + c, r.units, r.per_units);
    unsigned h = head0 + head, k = 0;
    unit[n] = unit0 + c - head * r.units;
    row[n] = t;
    long long xh = r.t[0].xs[2], yh = r.t[0].ys[2];
#pragma unroll
    for (int j = 1; j < kRotaryTensors; ++j)
      if (j < r.count && h >= (unsigned)r.first[j]) { k = j; xh = r.t[j].xs[2]; yh = r.t[j].ys[2]; }
    h -= k ? (unsigned)(k == 1 ? r.first[1] : k == 2 ? r.first[2] : r.first[3]) : 0u;
    const raw* const in = (const raw*)from[k][t] + h * xh;
    out[n] = (raw*)to[k][t] + h * yh;
    if (unit[n] < r.turned) {
      const unsigned at = rotary_place<W, INTERLEAVED, !STREAM>(r, unit[n]);
      fetch(a[n], in + at);
      if (TWO) fetch(b[n], in + at + (INTERLEAVED ? 1 : r.half));
      out[n] += at;
    } else {
      const int c = (int)(unit[n] - r.turned) * W, at = r.rotated + (STREAM ? c : min(c, r.copied - W));
      fetch(a[n], in + at);
      out[n] += at;
    }
  }
  for (unsigned i = threadIdx.x; i < tokens * (unsigned)r.half; i += 256) {
    const unsigned t = i / (unsigned)r.half, j = i - t * (unsigned)r.half;
    rotary_turn(place[t], *as_global(frequencies + j), r.scale, r.sign, cosines[i], sines[i]);
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (!is[n]) continue;
    float p[W], q[W];
    if (unit[n] >= r.turned) {
#pragma unroll
      for (int j = 0; j < W; ++j) p[j] = a[n].get(j);
      if (STREAM || r.copied >= W) {
        store_w<T, W, STREAM>(out[n], p);
      } else {
        // (the vector begins among the values that are turned)
#pragma unroll
        for (int j = 0; j < W; ++j)
          if (j >= W - r.copied) store1<T>(out[n] + j, p[j]);
      }
      continue;
    }
    const unsigned pair = row[n] * r.half + rotary_place<W, INTERLEAVED, !STREAM>(r, unit[n]) / (INTERLEAVED ? 2 : 1);
    const float *const c = cosines + pair, *const s = sines + pair;
    if constexpr (!TWO) {
#pragma unroll
      for (int j = 0; j < W; j += 2) {
        const float x = a[n].get(j), y = a[n].get(j + 1);
        p[j] = x * c[j / 2] - y * s[j / 2];
        p[j + 1] = x * s[j / 2] + y * c[j / 2];
      }
      store_w<T, W, STREAM>(out[n], p);
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float x = a[n].get(j), y = b[n].get(j);
        p[j] = x * c[j] - y * s[j];
        q[j] = x * s[j] + y * c[j];
      }
      store_w<T, W, STREAM>(out[n], p);
      store_w<T, W, STREAM>(out[n] + (INTERLEAVED ? 1 : r.half), q);
    }
  }
}

// Heads of which more than kRotaryTable pairs are turned: a thread for a pair, or for a value that is copied, of tensor k.
template <typename T>
__global__ __launch_bounds__(256) void fira_rotary_wide_kernel(FiraRotary r, int k, unsigned heads, unsigned copied, int interleaved, const double* frequencies, const void* positions) {
  typedef typename T::raw raw;
  const FiraRotaryTensor& x = r.t[k];
  const unsigned long long units = (unsigned)r.half + copied, total = units * heads * r.tokens;
  for (unsigned long long i = blockIdx.x * 256ULL + threadIdx.x; i < total; i += gridDim.x * 256ULL) {
    const unsigned u = (unsigned)(i % units), head = (unsigned)(i / units % heads), all = (unsigned)(i / units / heads), batch = all / r.length, token = all - batch * r.length;
    const raw* const in = (const raw*)x.x + batch * x.xs[0] + token * x.xs[1] + head * x.xs[2];
    raw* const out = (raw*)x.y + batch * x.ys[0] + token * x.ys[1] + head * x.ys[2];
    if (u >= (unsigned)r.half) {
      const unsigned c = r.rotated + u - r.half;
      *as_global(out + c) = *as_global(in + c);
      continue;
    }
    const long long p = batch * r.position_stride + token;
    float c, s;
    rotary_turn(!positions ? (long long)token : r.wide ? *as_global((const long long*)positions + p) : (long long)*as_global((const int*)positions + p), *as_global(frequencies + u), r.scale,
                r.sign, c, s);
    const unsigned ia = interleaved ? 2 * u : u, ib = interleaved ? 2 * u + 1 : u + r.half;
    const float a = load1<T>(in + ia), b = load1<T>(in + ib);
    store1<T>(out + ia, a * c - b * s);
    store1<T>(out + ib, a * s + b * c);
  }
}
