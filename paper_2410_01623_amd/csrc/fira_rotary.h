// Rotary positions and their gradient.  gfx950 only.
#pragma once
#include "fira_rows.h"

struct FiraRotary {
  long long batch, length, heads, dim, rotated, position_stride;
  long long xs[3], ys[3];        // strides of sequences, tokens and heads
  float scale, sign;             // sign: -1 for the gradient
  int interleaved, wide;         // wide: positions of 64 bits
};

// cos and sin of position times frequency, times the scale.  The angle is brought to a part of a turn in fp64; what is left fits fp32.
__device__ __forceinline__ void rotary_turn(long long position, double frequency, float scale, float sign, float& c, float& s) {
  const double turns = (double)position * frequency * 0.15915494309189533577;
  float sn, cs;
  sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
  c = scale * cs;
  s = sign * scale * sn;
}
__device__ __forceinline__ long long rotary_position(const FiraRotary& r, const void* positions, long long batch, long long token) {
  if (!positions) return token;
  const long long i = batch * r.position_stride + token;
  return r.wide ? *as_global((const long long*)positions + i) : (long long)*as_global((const int*)positions + i);
}

// A thread for a pair, or for a value that is copied.
template <typename T>
__global__ __launch_bounds__(256) void fira_rotary_kernel(FiraRotary r, const typename T::raw* x, typename T::raw* y, const double* frequencies, const void* positions) {
  const long long half = r.rotated / 2, units = half + r.dim - r.rotated, total = r.batch * r.length * r.heads * units;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < total; i += gridDim.x * 256LL) {
    const long long u = i % units, head = i / units % r.heads, token = i / units / r.heads % r.length, batch = i / units / r.heads / r.length;
    const typename T::raw* const from = x + batch * r.xs[0] + token * r.xs[1] + head * r.xs[2];
    typename T::raw* const to = y + batch * r.ys[0] + token * r.ys[1] + head * r.ys[2];
    if (u >= half) {
      const long long c = r.rotated + u - half;
      to[c] = from[c];
      continue;
    }
    float c, s;
    rotary_turn(rotary_position(r, positions, batch, token), *as_global(frequencies + u), r.scale, r.sign, c, s);
    const long long ia = r.interleaved ? 2 * u : u, ib = r.interleaved ? 2 * u + 1 : u + half;
    const float a = load1<T>(from + ia), b = load1<T>(from + ib);
    store1<T>(to + ia, a * c - b * s);
    store1<T>(to + ib, a * s + b * c);
  }
}
