// Rows of an embedding table by token, and the table's gradient.  gfx950 only.
#pragma once
#include "fira_rows.h"

struct FiraEmbed {
  int vocab;              // rows of the table
  long long dim, ld;      // its width and leading dimension
  long long count, ld_rows;   // tokens, leading dimension of their rows
  float scale;
  int ids64;              // 1: ids are int64, 0: int32
};

// The table row that token t names, or -1 for an id outside the table (padding).
__device__ __forceinline__ int token_row(const FiraEmbed& e, const void* ids, long long t) {
  if (e.ids64) {
    const long long v = *as_global((const long long*)ids + t);
    return v >= 0 && v < e.vocab ? (int)v : -1;
  }
  const int v = *as_global((const int*)ids + t);
  return v >= 0 && v < e.vocab ? v : -1;
}

// out[t] = scale * table[id_t], zeros for an id outside the table.  One workgroup per token.
template <typename T, typename R>
__global__ __launch_bounds__(256) void fira_embed_lookup_kernel(FiraEmbed e, const typename T::raw* table, const void* ids, typename R::raw* out) {
  for (long long t = blockIdx.x; t < e.count; t += gridDim.x) {
    const int v = token_row(e, ids, t);
    for (long long c = threadIdx.x * kVec; c < e.dim; c += 256 * kVec) {
      float x[kVec] = {};
      if (v >= 0) load_some<T>(table + v * e.ld + c, e.dim - c, x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) x[i] *= e.scale;
      store_some<R>(out + t * e.ld_rows + c, e.dim - c, x);
    }
  }
}

// dtable[v] (+)= scale * sum of dout[t] over the tokens with id_t = v, in order of t, in fp32, rounded once.  One wavefront per table row
// and 512 columns, which looks through all ids.
template <typename T, typename R>
__global__ __launch_bounds__(64) void fira_embed_gradient_kernel(FiraEmbed e, const typename R::raw* dout, const void* ids, typename T::raw* dtable, int accumulate) {
  const int lane = threadIdx.x;
  for (long long v = blockIdx.x; v < e.vocab; v += gridDim.x) {
    for (long long c = lane * kVec; c - lane * kVec < e.dim; c += 64 * kVec) {
      float sum[kVec] = {};
      for (long long t0 = 0; t0 < e.count; t0 += 64) {
        unsigned long long hit = __ballot(t0 + lane < e.count && token_row(e, ids, t0 + lane) == v);
        for (; hit; hit &= hit - 1) {
          const long long t = t0 + __builtin_ctzll(hit);
          float x[kVec] = {};
          if (c < e.dim) load_some<R>(dout + t * e.ld_rows + c, e.dim - c, x);
#pragma unroll
          for (int i = 0; i < kVec; ++i) sum[i] += x[i];
        }
      }
      if (c >= e.dim) continue;
      typename T::raw* to = dtable + v * e.ld + c;
      float old[kVec] = {};
      if (accumulate) load_some<T>(to, e.dim - c, old);
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum[i] = old[i] + e.scale * sum[i];
      store_some<T>(to, e.dim - c, sum);
    }
  }
}
