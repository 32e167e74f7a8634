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

// ---- gradient ------------------------------------------------------------------------------------------------------
// dtable[v] (+)= scale * sum of dout[t] over the tokens with id_t = v, in order of t.  The tokens are sorted by id, stably, so that every row's
// tokens stand together in order of t and the sums have one order, whatever runs when:
//   1. fira_embed_chunk_kernel    a chunk of tokens per workgroup, sorted by the low eight bits of the id (a bucket: neighbouring ids, which
//                                 text uses together, go to different ones)
//   2. fira_embed_bucket_kernel   a bucket per workgroup: its tokens out of all chunks, sorted by the rest of the id; where each row's tokens are
//   3. fira_embed_sum_kernel      every row of the table: its tokens' rows added up in registers and written once; rows of more than
//                                 kPieceTokens tokens (text has a few that hold a large share of all) in pieces side by side
//   4. fira_embed_join_kernel     the pieces of those
// A row is cut by its own tokens alone, so that its bits depend on nothing else.
constexpr int kBuckets = 256, kMostChunks = 256;
constexpr int kPieceTokens = 32;
constexpr int kCounters = 15360;                        // LDS of a bucket's workgroup: a counter for each of its rows and wavefronts
constexpr int64_t kMostEmbedRows = 1 << 21;             // ... of which there are kBuckets times fewer than rows of the table

struct FiraEmbedSort {       // the sort's part of the workspace
  int chunk, chunks;         // tokens of a chunk, number of chunks
  int bins;                  // rows of a bucket
  int bits;                  // ... and bits that number them
  u32x2* sorted;             // [chunks][chunk]       (id >> 8, token), by bucket
  u32x2* part;               // [kBuckets][chunks]    first entry and number of entries of a bucket in a chunk
  unsigned* order;           // [count]               tokens by row
  u32x2* rows;               // [kBuckets][bins]      first entry in `order` and number of entries of a row
  int* counters;             // entries of `order` handed out, pieces, rows in pieces
  u32x2* pieces;             // (row, piece of it)
  u32x2* cut;                // rows in pieces: (row, their first piece)
  float* partial;            // [pieces][dim]
};

// Lanes that are `in` and have this lane's key of `bits` bits.
__device__ __forceinline__ unsigned long long lanes_alike(unsigned key, int bits, bool in) {
  unsigned long long m = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long one = __ballot((key >> b) & 1);
    m &= (key >> b) & 1 ? one : ~one;
  }
  return m;
}
// Sum of x over the threads before this one; *total: over all.  part: LDS, 17 values.
__device__ __forceinline__ int block_scan(int x, int* part, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) { const int y = __shfl_up(s, d, 64); s += lane >= d ? y : 0; }
  __syncthreads();
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < waves; ++w) { before += w < wave ? part[w] : 0; all += part[w]; }
  *total = all;
  return before + s - x;
}

__global__ __launch_bounds__(256) void fira_embed_chunk_kernel(FiraEmbed e, const void* ids, FiraEmbedSort s) {
  __shared__ int count[4][kBuckets];
  __shared__ int part[17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x == 0 && threadIdx.x < 3) *as_global(s.counters + threadIdx.x) = 0;   // for the next kernel
  for (int w = 0; w < 4; ++w) count[w][threadIdx.x] = 0;
  __syncthreads();
  const long long begin = (long long)blockIdx.x * s.chunk, end = min(begin + s.chunk, e.count);
  const long long mine = begin + wave * (s.chunk / 4), until = min(mine + s.chunk / 4, end);
  // (a wavefront's counters are its own, and of the lanes with one bucket only the first one writes)
  auto each = [&](auto f) {
    for (long long t0 = mine; t0 < until; t0 += 64) {
      const long long t = t0 + lane;
      const int v = t < until ? token_row(e, ids, t) : -1;
      const unsigned long long alike = lanes_alike(v & (kBuckets - 1), 8, v >= 0);
      const unsigned long long below = alike & ((1ull << lane) - 1);
      volatile int* const c = &count[wave][v & (kBuckets - 1)];
      const int before = *c + __popcll(below);
      __builtin_amdgcn_wave_barrier();
      if (v >= 0 && !below) *c = before + __popcll(alike);
      __builtin_amdgcn_wave_barrier();
      if (v >= 0) f(v, t, before);
    }
  };
  each([](int, long long, int) {});
  __syncthreads();
  int sum = 0;
  for (int w = 0; w < 4; ++w) sum += count[w][threadIdx.x];
  int total;
  int first = block_scan(sum, part, &total);
  *as_global(s.part + (long long)threadIdx.x * s.chunks + blockIdx.x) = u32x2{(unsigned)first, (unsigned)sum};
  for (int w = 0; w < 4; ++w) { const int c = count[w][threadIdx.x]; count[w][threadIdx.x] = first; first += c; }
  __syncthreads();
  each([&](int v, long long t, int at) { *as_global(s.sorted + begin + at) = u32x2{(unsigned)v >> 8, (unsigned)t}; });
}

// (dynamic LDS: a counter per wavefront and row of the bucket)
__global__ __launch_bounds__(1024) void fira_embed_bucket_kernel(FiraEmbed e, FiraEmbedSort s) {
  extern __shared__ int count[];
  __shared__ int first_of[kMostChunks], at_of[kMostChunks];
  __shared__ int part[17];
  __shared__ int base_s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, bucket = blockIdx.x;
  int n = 0;                                            // tokens of this bucket
  for (int c0 = 0; c0 < s.chunks; c0 += blockDim.x) {
    const int c = c0 + threadIdx.x;
    const u32x2 p = c < s.chunks ? *as_global(s.part + (long long)bucket * s.chunks + c) : u32x2{0, 0};
    int total;
    const int before = n + block_scan((int)p.y, part, &total);
    if (c < s.chunks) { first_of[c] = before; at_of[c] = (int)p.x; }
    n += total;
  }
  for (int i = threadIdx.x; i < waves * s.bins; i += blockDim.x) count[i] = 0;
  // where in `order` does not matter to any result
  if (threadIdx.x == 0) base_s = n ? atomicAdd(s.counters, n) : 0;
  __syncthreads();
  const int base = base_s;
  const int per = ((n + waves - 1) / waves + 63) / 64 * 64;
  const int mine = min(wave * per, n), until = min(mine + per, n);
  volatile int* const own = count + wave * s.bins;
  auto each = [&](auto f) {
    for (int i0 = mine; i0 < until; i0 += 64) {
      const int i = i0 + lane;
      u32x2 entry{0, 0};
      if (i < until) {
        int c = 0;                                       // the last chunk whose first entry is not after i
        for (int step = kMostChunks / 2; step; step >>= 1)
          if (c + step < s.chunks && first_of[c + step] <= i) c += step;
        entry = *as_global(s.sorted + (long long)c * s.chunk + at_of[c] + (i - first_of[c]));
      }
      const unsigned long long alike = lanes_alike(entry.x, s.bits, i < until);
      const unsigned long long below = alike & ((1ull << lane) - 1);
      const int before = own[entry.x] + __popcll(below);
      __builtin_amdgcn_wave_barrier();
      if (i < until && !below) own[entry.x] = before + __popcll(alike);
      __builtin_amdgcn_wave_barrier();
      if (i < until) f(entry.y, before);
    }
  };
  each([](unsigned, int) {});
  __syncthreads();
  int start = 0;
  for (int b0 = 0; b0 < s.bins; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    int sum = 0;
    if (b < s.bins)
      for (int w = 0; w < waves; ++w) sum += count[w * s.bins + b];
    int total;
    int first = start + block_scan(sum, part, &total);
    start += total;
    if (b >= s.bins) continue;                          // (the barriers are behind; the next round's are in block_scan, which needs all)
    *as_global(s.rows + (long long)bucket * s.bins + b) = u32x2{(unsigned)(base + first), (unsigned)sum};
    if (sum > kPieceTokens) {
      const int pieces = (sum + kPieceTokens - 1) / kPieceTokens, p = atomicAdd(s.counters + 1, pieces);
      const unsigned row = (unsigned)b * kBuckets + bucket;
      for (int k = 0; k < pieces; ++k) *as_global(s.pieces + p + k) = u32x2{row, (unsigned)k};
      *as_global(s.cut + atomicAdd(s.counters + 2, 1)) = u32x2{row, (unsigned)p};
    }
    for (int w = 0; w < waves; ++w) { const int c = count[w * s.bins + b]; count[w * s.bins + b] = first; first += c; }
  }
  __syncthreads();
  each([&](unsigned t, int at) { *as_global(s.order + base + at) = t; });
}

__device__ __forceinline__ u32x2 tokens_of_row(const FiraEmbedSort& s, unsigned row) {
  return *as_global(s.rows + (long long)(row & (kBuckets - 1)) * s.bins + (row >> 8));
}

// sum += dout[order[first + i]] for i < n, columns c to c + 7, in order of i; eight rows are on their way at a time.
template <typename R>
__device__ __forceinline__ void sum_of_tokens(const FiraEmbed& e, const typename R::raw* dout, const unsigned* order, unsigned n, long long c, float (&sum)[kVec]) {
  const long long left = e.dim - c;
  for (unsigned i0 = 0; i0 < n; i0 += 8) {
    float x[8][kVec];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k < n) load_some<R>(dout + *as_global(order + i0 + k) * e.ld_rows + c, left, x[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k < n)
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum[j] += x[k][j];
  }
}
template <typename T>
__device__ __forceinline__ void write_gradient(const FiraEmbed& e, typename T::raw* dtable, unsigned row, long long c, int accumulate, float (&sum)[kVec]) {
  typename T::raw* to = dtable + row * e.ld + c;
  float old[kVec] = {};
  if (accumulate) load_some<T>(to, e.dim - c, old);
#pragma unroll
  for (int j = 0; j < kVec; ++j) sum[j] = old[j] + e.scale * sum[j];
  store_some<T>(to, e.dim - c, sum);
}

// LANES lanes to a row, or to 512 columns of one; the pieces first, as they take longest.
template <typename T, typename R, int LANES>
__global__ __launch_bounds__(256) void fira_embed_sum_kernel(FiraEmbed e, const typename R::raw* dout, typename T::raw* dtable, int accumulate, FiraEmbedSort s) {
  const int lane = threadIdx.x % LANES;
  const long long tiles = (e.dim + LANES * kVec - 1) / (LANES * kVec);
  const long long pieces = *as_global(s.counters + 1) * tiles, all = pieces + e.vocab * tiles;
  for (long long i = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; i < all; i += (long long)gridDim.x * (256 / LANES)) {
    const bool piece = i < pieces;
    const long long k = piece ? i / tiles : (i - pieces) / tiles;
    const long long c = ((piece ? i : i - pieces) - k * tiles) * (LANES * kVec) + lane * kVec;
    if (c >= e.dim) continue;
    float sum[kVec] = {};
    if (piece) {
      const u32x2 p = *as_global(s.pieces + k), r = tokens_of_row(s, p.x);
      sum_of_tokens<R>(e, dout, s.order + r.x + p.y * kPieceTokens, min((unsigned)kPieceTokens, r.y - p.y * kPieceTokens), c, sum);
      store_some<FiraStoredF32>(s.partial + k * e.dim + c, e.dim - c, sum);
    } else {
      const u32x2 r = tokens_of_row(s, (unsigned)k);
      if (r.y > kPieceTokens || (r.y == 0 && accumulate)) continue;
      sum_of_tokens<R>(e, dout, s.order + r.x, r.y, c, sum);
      write_gradient<T>(e, dtable, (unsigned)k, c, accumulate, sum);
    }
  }
}

// 512 columns of a row in pieces per workgroup: its wavefronts take every 16th piece each, and their sums are added in turn.
template <typename T>
__global__ __launch_bounds__(1024) void fira_embed_join_kernel(FiraEmbed e, typename T::raw* dtable, int accumulate, FiraEmbedSort s) {
  __shared__ float part[16][64 * kVec];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long tiles = (e.dim + 64 * kVec - 1) / (64 * kVec), all = *as_global(s.counters + 2) * tiles;
  for (long long i = blockIdx.x; i < all; i += gridDim.x) {
    const u32x2 row = *as_global(s.cut + i / tiles);
    const long long c = i % tiles * (64 * kVec) + lane * kVec;
    const unsigned pieces = (tokens_of_row(s, row.x).y + kPieceTokens - 1) / kPieceTokens;
    float sum[kVec] = {};
    if (c < e.dim)
#pragma unroll 4
      for (unsigned k = wave; k < pieces; k += 16) {
        float x[kVec];
        load_some<FiraStoredF32>(s.partial + (long long)(row.y + k) * e.dim + c, e.dim - c, x);
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum[j] += x[j];
      }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kVec; ++j) part[wave][lane * kVec + j] = sum[j];
    __syncthreads();
    if (wave == 0 && c < e.dim) {
#pragma unroll 1
      for (int w = 1; w < 16; ++w)
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum[j] += part[w][lane * kVec + j];
      write_gradient<T>(e, dtable, row.x, c, accumulate, sum);
    }
  }
}
