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

// out[t] = scale * table[id_t], zeros for an id outside the table.  A wavefront takes TOKENS tokens at a time, 64 / LANES of them side by side, and
// NV vectors of each per lane.  131072 tokens x 2048, a table of 32000 rows in fp32, bf16 out: 168 us with two tokens and 2048 columns a wavefront, 172 with
// one, 175 and 182 with 512 columns and two or four tokens; 179 to 198 where every XCD goes through columns of its own, so that more of the rows
// that a text uses all the time are in its L2.
template <typename T, typename R, int W, int LANES, int NV, int TOKENS>
__global__ __launch_bounds__(256) void fira_embed_lookup_kernel(FiraEmbed e, const typename T::raw* table, const void* ids, typename R::raw* out) {
  constexpr int SIDE = 64 / LANES, EACH = TOKENS / SIDE;
  const int lane = threadIdx.x & 63;
  const unsigned tiles = (unsigned)((e.dim + NV * LANES * W - 1) / (NV * LANES * W));
  const long long all = (e.count + TOKENS - 1) / TOKENS * tiles;
  for (long long i = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < all; i += gridDim.x * 4LL) {
    const long long unit = i / tiles, c0 = (i - unit * tiles) * (NV * LANES * W) + lane % LANES * W, t0 = unit * TOKENS + lane / LANES;
    int row[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) row[k] = token_row(e, ids, min(t0 + k * SIDE, e.count - 1));
    Raw<T, W> x[EACH][NV];
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int v = 0; v < NV; ++v) x[k][v].load(table + max(row[k], 0) * e.ld + Columns<W>(c0 + v * (LANES * W), e.dim).at);
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Columns<W> c(c0 + v * (LANES * W), e.dim);
        const long long t = t0 + k * SIDE;
        float y[W];
#pragma unroll
        for (int j = 0; j < W; ++j) y[j] = row[k] >= 0 ? e.scale * x[k][v].get(j) : 0.0f;
        if (c.any && t < e.count) store_w<R, W, true>(out + t * e.ld_rows + c.at, y);
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
constexpr int kCounters = 15360;                        // LDS of a bucket's workgroup, in words: a counter for each of its rows and wavefronts, then entries
constexpr int64_t kMostEmbedRows = 1 << 21;             // ... of which there are kBuckets times fewer than rows of the table

struct FiraEmbedSort {       // the sort's part of the workspace
  int chunk, chunks;         // tokens of a chunk, number of chunks
  int bins;                  // rows of a bucket
  int bits;                  // ... and bits that number them
  u32x2* sorted;             // [chunks][chunk]       (id >> 8, token), by bucket
  u32x2* gathered;           // [count]               the same, a bucket's side by side, where they do not fit LDS
  u32x2* part;               // [kBuckets][chunks]    first entry and number of entries of a bucket in a chunk
  unsigned* order;           // [count]               tokens by row
  u32x2* rows;               // [kBuckets][bins]      first entry in `order` and number of entries of a row
  int* counters;             // pieces, rows in pieces
  u32x4* pieces;             // (row, first entry of `order`, number of entries)
  u32x4* cut;                // rows in pieces: (row, first piece, number of pieces)
  float* partial;            // [pieces][dim]
};

// Lanes that are `in` and have this lane's key of `bits` bits.  (Taking keys out one after the other instead, or four of them before this, as the bucket of a
// text's most frequent token has mostly one: 131072 tokens 130.9 and 129.8 us for 127.4.)
__device__ __forceinline__ unsigned long long lanes_alike(unsigned key, int bits, bool in) {
  unsigned long long m = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const int mine = (int)(key << (31 - b)) >> 31;      // all ones where the bit is set
    m &= ~(__ballot(mine) ^ (unsigned long long)(long long)mine);
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
  if (blockIdx.x == 0 && threadIdx.x < 2) *as_global(s.counters + threadIdx.x) = 0;   // for the next kernel
  for (int w = 0; w < 4; ++w) count[w][threadIdx.x] = 0;
  __syncthreads();
  const long long begin = (long long)blockIdx.x * s.chunk, end = min(begin + s.chunk, e.count);
  const long long mine = begin + wave * (s.chunk / 4), until = min(mine + s.chunk / 4, end);
  int id[2];                                             // a wavefront's ids, where there are so few
  auto load = [&](long long t0) {
#pragma unroll
    for (int k = 0; k < 2; ++k) { const long long t = t0 + k * 64 + lane; id[k] = t < until ? token_row(e, ids, t) : -1; }
  };
  for (long long t0 = mine; t0 < until; t0 += 128) {
    load(t0);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (id[k] >= 0) atomicAdd(&count[wave][id[k] & (kBuckets - 1)], 1);
  }
  __syncthreads();
  int sum = 0;
  for (int w = 0; w < 4; ++w) sum += count[w][threadIdx.x];
  int total;
  int first = block_scan(sum, part, &total);
  *as_global(s.part + (long long)threadIdx.x * s.chunks + blockIdx.x) = u32x2{(unsigned)first, (unsigned)sum};
  for (int w = 0; w < 4; ++w) { const int c = count[w][threadIdx.x]; count[w][threadIdx.x] = first; first += c; }
  __syncthreads();
  // (a wavefront's counters are its own, and of the lanes with one bucket only the first one writes)
  for (long long t0 = mine; t0 < until; t0 += 128) {
    if (until - mine > 128) load(t0);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int v = id[k];
      const unsigned long long alike = lanes_alike(v & (kBuckets - 1), 8, v >= 0);
      const unsigned long long below = alike & ((1ull << lane) - 1);
      volatile int* const c = &count[wave][v & (kBuckets - 1)];
      const int at = *c + __popcll(below);
      __builtin_amdgcn_wave_barrier();
      if (v >= 0 && !below) *c = at + __popcll(alike);
      __builtin_amdgcn_wave_barrier();
      if (v >= 0) *as_global(s.sorted + begin + at) = u32x2{(unsigned)v >> 8, (unsigned)(t0 + k * 64 + lane)};
    }
  }
}

// How a row of n < 2^31 tokens is cut: at most 256 pieces, which the join has to read one after the other.  (256 pieces of the next length may be 2^31
// tokens, and so may whole spans of all wavefronts: nothing here goes past 32 bits for it.)
__host__ __device__ __forceinline__ int piece_tokens(int n) {
  int len = kPieceTokens;
  while ((n - 1) / 256 >= len) len *= 2;
  return len;
}
__host__ __device__ __forceinline__ int row_pieces(int n) { return n > kPieceTokens ? (n - 1) / piece_tokens(n) + 1 : 0; }
// Entries of a bucket with `total` that each of its wavefronts places: whole groups of 64.
__host__ __device__ __forceinline__ unsigned wave_span(unsigned total, unsigned waves) {
  const unsigned each = total / waves + (total % waves != 0);
  return each ? (each + 63) / 64 * 64 : 64;
}

// The bucket's entries come out of all chunks at once, a few threads to a chunk, side by side into LDS (those of the bucket of a text's most frequent
// token may be too many: into the workspace then), and are counted on the way; a wavefront then places a part of them.  What has to wait for memory
// waits once for all of it: with a group of 64 entries after the other, each fetched from another XCD's work, the largest of the 256 buckets of 131072
// tokens took 21 us.  The workgroup is alone with its bucket: with a fifth of those tokens one id it takes 54 us, with all of them 218 (the whole gradient,
// x 1024 in fp32, 127, 163 and 345 us).
// (dynamic LDS: a counter per wavefront and row of the bucket, then the entries)
__global__ __launch_bounds__(1024) void fira_embed_bucket_kernel(FiraEmbed e, FiraEmbedSort s) {
  extern __shared__ int count[];
  __shared__ int part[17];
  __shared__ unsigned long long given;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, bucket = blockIdx.x;
  u32x2* const staged = (u32x2*)(count + (waves * s.bins + 1) / 2 * 2);
  const int room = (kCounters - (waves * s.bins + 1) / 2 * 2) / 2;
  // `each` threads to a chunk, the chunks in their order
  int each = 1;
  while (2 * each * s.chunks <= (int)blockDim.x) each *= 2;
  const int steps = (s.chunks * each + blockDim.x - 1) / blockDim.x;      // 1 but for few wavefronts
  for (int i = threadIdx.x; i < waves * s.bins; i += blockDim.x) count[i] = 0;
  int before = 0, n = 0;                                // entries of the buckets before this one, and of this one
  u32x2 mine{0, 0};
  for (int k = 0; k < steps; ++k) {
    const int c = (k * blockDim.x + threadIdx.x) / each;
    mine = u32x2{0, 0};
    if (c < s.chunks) mine = *as_global(s.part + (long long)bucket * s.chunks + c);
    const bool first = threadIdx.x % each == 0;
    before += first ? (int)mine[0] : 0;
    n += first ? (int)mine[1] : 0;
  }
  int base, total;
  block_scan(before, part, &base);
  int at = block_scan(n, part, &total);                 // (where steps is 1: entries of the chunks before this thread's)
  const unsigned span = wave_span(total, waves);
  const bool in_lds = total <= room;
  int done = 0;
  for (int k = 0; k < steps; ++k) {
    const int c = (k * blockDim.x + threadIdx.x) / each, j0 = threadIdx.x % each;
    if (steps > 1) {
      mine = u32x2{0, 0};
      if (c < s.chunks) mine = *as_global(s.part + (long long)bucket * s.chunks + c);
      int here;
      at = done + block_scan(j0 == 0 ? (int)mine[1] : 0, part, &here);
      done += here;
    }
    if (j0) at -= (int)mine[1];                         // (the scan has counted the chunk itself for all but its first thread)
    const u32x2* const src = s.sorted + (long long)c * s.chunk + mine[0];
    for (int j = j0; j < (int)mine[1]; j += 4 * each) {
      u32x2 entry[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (j + u * each < (int)mine[1]) entry[u] = *as_global(src + j + u * each);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (j + u * each < (int)mine[1]) {
          const unsigned to = at + j + u * each;
          if (in_lds) staged[to] = entry[u];
          else *as_global(s.gathered + base + to) = entry[u];
          atomicAdd(count + to / span * s.bins + entry[u][0], 1);
        }
    }
  }
  __syncthreads();
  // the rows' first places, and each wavefront's among them
  int start = 0;
  for (int b0 = 0; b0 < s.bins; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    int sum = 0;
    if (b < s.bins)
#pragma unroll 8
      for (int w = 0; w < waves; ++w) sum += count[w * s.bins + b];
    int here;
    int first = start + block_scan(sum, part, &here);
    start += here;
    if (b < s.bins) {
      *as_global(s.rows + (long long)bucket * s.bins + b) = u32x2{(unsigned)(base + first), (unsigned)sum};
      int next = first;
#pragma unroll 8
      for (int w = 0; w < waves; ++w) { const int c = count[w * s.bins + b]; count[w * s.bins + b] = next; next += c; }
    }
    // rows in pieces: one addition per workgroup hands out the places for all of them, as those of all workgroups wait for one another;
    // which places does not matter to any result
    const int len = piece_tokens(sum), pieces = row_pieces(sum);
    if (__syncthreads_or(pieces)) {
      int all_pieces, all_rows;
      const int my_pieces = block_scan(pieces, part, &all_pieces), my_row = block_scan(pieces > 0, part, &all_rows);
      if (threadIdx.x == 0) given = atomicAdd((unsigned long long*)s.counters, (unsigned long long)all_rows << 32 | (unsigned)all_pieces);
      __syncthreads();
      const unsigned row = (unsigned)b * kBuckets + bucket, p = (unsigned)given + my_pieces;
      if (pieces) *as_global(s.cut + (given >> 32) + my_row) = u32x4{row, p, (unsigned)pieces, 0};
      for (unsigned long long m = __ballot(pieces > 0); m; m &= m - 1) {      // a wavefront lists one row's pieces after the other
        const int l = __builtin_ctzll(m), n = __builtin_amdgcn_readlane(pieces, l), size = __builtin_amdgcn_readlane(len, l);
        const int from = base + __builtin_amdgcn_readlane(first, l), all = __builtin_amdgcn_readlane(sum, l);
        u32x4* const to = s.pieces + (unsigned)__builtin_amdgcn_readlane((int)p, l);
        for (int k = lane; k < n; k += 64)
          *as_global(to + k) = u32x4{(unsigned)__builtin_amdgcn_readlane((int)row, l), (unsigned)(from + k * size), (unsigned)min(size, all - k * size), 0};
      }
    }
  }
  __syncthreads();
  volatile int* const own = count + wave * s.bins;
  const unsigned until = min((wave + 1) * span, (unsigned)total);
#pragma unroll 1
  for (unsigned i = wave * span + lane; i - lane < until; i += 64) {
    const bool in = i < until;
    u32x2 entry{0, 0};
    if (in_lds) { if (in) entry = staged[i]; }
    else if (in) entry = *as_global(s.gathered + base + i);
    const unsigned long long alike = lanes_alike(entry[0], s.bits, in);
    const unsigned long long below = alike & ((1ull << lane) - 1);
    const int to = own[entry[0]] + __popcll(below);
    __builtin_amdgcn_wave_barrier();
    if (in && !below) own[entry[0]] = to + __popcll(alike);   // (of the lanes with one row only the first one writes)
    __builtin_amdgcn_wave_barrier();
    if (in) *as_global(s.order + base + to) = entry[1];
  }
}

__device__ __forceinline__ u32x2 tokens_of_row(const FiraEmbedSort& s, unsigned row) {
  return *as_global(s.rows + (long long)(row & (kBuckets - 1)) * s.bins + (row >> 8));
}

template <typename T, int W, bool ADD>
__device__ __forceinline__ void write_gradient(const FiraEmbed& e, typename T::raw* dtable, unsigned row, const Columns<W>& c, const float (&sum)[W]) {
  typename T::raw* const to = dtable + row * e.ld + c.at;
  float y[W];
#pragma unroll
  for (int j = 0; j < W; ++j) y[j] = e.scale * sum[j];
  if constexpr (ADD) {
    Raw<T, W> old;
    old.load(to);
#pragma unroll
    for (int j = 0; j < W; ++j) y[j] += old.get(j);
    if (c.skip) {                                        // (the neighbour may be another wavefront, before its own reading)
#pragma unroll
      for (int j = 1; j < W; ++j)
        if (j >= c.skip) store1<T>(to + j, y[j]);
      return;
    }
  }
  store_w<T, W, !ADD>(to, y);
}

// Loads of N rows are put on their way together, without a branch between them; beyond the last row it is loaded again.  (One copy of the loop's
// body: with blocks of 8, 4, 2 and 1 for the remainder the wavefronts of fira_embed_sum_kernel waited for instructions half of their time.)

// Widths up to 32 W: LANES lanes to a row; four tokens' rows are on their way at a time.  The pieces come first, as they take longest.  Bound by memory and
// by what has to be waited for one after the other: 131072 tokens x 128 bf16, 50257 rows, 16.5 us (2.8 TB/s) of the gradient's 43, the sort being 22.
template <typename T, typename R, int W, int LANES, bool ADD>
__global__ __launch_bounds__(256) void fira_embed_sum_narrow_kernel(FiraEmbed e, const typename R::raw* dout, typename T::raw* dtable, FiraEmbedSort s) {
  constexpr int N = 4;
  const Columns<W> c(threadIdx.x % LANES * W, e.dim);
  if (!c.any) return;
  const long long pieces = *as_global(s.counters), all = pieces + e.vocab;
  for (long long i = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; i < all; i += (long long)gridDim.x * (256 / LANES)) {
    const bool piece = i < pieces;
    u32x2 r{0, 0};
    if (piece) {
      const u32x4 p = *as_global(s.pieces + i);
      r = u32x2{p[1], p[2]};
    } else {
      r = tokens_of_row(s, (unsigned)(i - pieces));
      if (r[1] > kPieceTokens || (ADD && r[1] == 0)) continue;
    }
    float sum[W] = {};
    const unsigned* const order = s.order + r[0];
    for (unsigned first = 0; first < r[1]; first += N) {
      unsigned t[N];
      Raw<R, W> x[N];
#pragma unroll
      for (int k = 0; k < N; ++k) t[k] = *as_global(order + min(first + k, r[1] - 1));
#pragma unroll
      for (int k = 0; k < N; ++k) x[k].load(dout + t[k] * e.ld_rows + c.at);
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (first + k < r[1])
#pragma unroll
          for (int j = 0; j < W; ++j) sum[j] += x[k].get(j);
    }
    if (piece) store_w<FiraStoredF32, W>(s.partial + i * e.dim + c.at, sum);
    else write_gradient<T, W, ADD>(e, dtable, (unsigned)(i - pieces), c, sum);
  }
}

// Wider ones: a wavefront takes 512 columns of kBatch neighbouring rows of a bucket (whose tokens it finds with one load), or of a piece.
// The tokens of all its rows make one sequence, of which eight are on their way at a time, whatever row they belong to: most rows have one
// token or none, and one row after the other would wait for its place, its tokens and their rows in turn.
constexpr int kBatch = 8;
template <typename T, typename R, bool ADD>
__global__ __launch_bounds__(256) void fira_embed_sum_kernel(FiraEmbed e, const typename R::raw* dout, typename T::raw* dtable, FiraEmbedSort s) {
  constexpr int W = kWidth<T, R>, NV = 8 / W, N = 8;
  const int lane = threadIdx.x & 63;
  const unsigned tiles = (unsigned)((e.dim + 511) / 512), batches = (s.bins + kBatch - 1) / kBatch;
  const long long pieces = (long long)*as_global(s.counters) * tiles, all = pieces + (long long)batches * kBuckets * tiles;
  for (long long i = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < all; i += gridDim.x * 4LL) {
    const bool piece = i < pieces;
    const long long unit = (piece ? i : i - pieces) / tiles;
    const long long c0 = ((piece ? i : i - pieces) - unit * tiles) * 512 + lane * W;
    auto columns = [&](int v) { return Columns<W>(c0 + v * (64 * W), e.dim); };
    // lane k < kBatch: first token and number of tokens of row k
    unsigned row0 = 0;
    u32x2 r{0, 0};
    if (piece) {
      const u32x4 p = *as_global(s.pieces + unit);
      if (lane == 0) r = u32x2{p[1], p[2]};
    } else {
      const unsigned bucket = (unsigned)unit & (kBuckets - 1), key0 = (unsigned)(unit >> 8) * kBatch;
      row0 = key0 * kBuckets + bucket;                   // row k is row0 + k * kBuckets
      if (lane < kBatch && key0 + lane < (unsigned)s.bins) r = *as_global(s.rows + (long long)bucket * s.bins + key0 + lane);
    }
    const int n = !piece && r[1] > kPieceTokens ? 0 : (int)r[1];      // (such rows are in pieces, which may be longer than that)
    int upto = n;                                        // tokens of the rows up to this lane's
#pragma unroll
    for (int d = 1; d < kBatch; d <<= 1) { const int y = __shfl_up(upto, d, 64); upto += lane >= d ? y : 0; }
    const int total = __builtin_amdgcn_readlane(upto, kBatch - 1);
    float sum[NV][W] = {};
    auto finish = [&](unsigned to) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Columns<W> c = columns(v);
        if (c.any) write_gradient<T, W, ADD>(e, dtable, to, c, sum[v]);
      }
    };
    if (!ADD && !piece) {
      const bool none = r[1] == 0 && lane < kBatch && row0 + lane * kBuckets < (unsigned)e.vocab;
      for (unsigned long long m = __ballot(none); m; m &= m - 1) finish(row0 + __builtin_ctzll(m) * kBuckets);
    }
    int row = -1;                                        // the one that is being summed
    for (int j0 = 0; j0 < total; j0 += 64) {
      // token and row of place j0 + lane in the sequence
      const int at = min(j0 + lane, total - 1);
      int of = 0;
#pragma unroll
      for (int k = 0; k < kBatch - 1; ++k) of += at >= __builtin_amdgcn_readlane(upto, k);
      const int before = __shfl(upto, of, 64) - __shfl(n, of, 64);
      const unsigned token = *as_global(s.order + (__shfl(r[0], of, 64) + at - before));
      for (int first = 0; first < 64 && j0 + first < total; first += N) {
        Raw<R, W> x[N][NV];
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
          for (int v = 0; v < NV; ++v) x[k][v].load(dout + (unsigned)__builtin_amdgcn_readlane(token, first + k) * e.ld_rows + columns(v).at);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          if (j0 + first + k >= total) break;
          const int next = __builtin_amdgcn_readlane(of, first + k);
          if (next != row) {
            if (row >= 0) {
              finish(row0 + row * kBuckets);
#pragma unroll
              for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < W; ++j) sum[v][j] = 0.0f;
            }
            row = next;
          }
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < W; ++j) sum[v][j] += x[k][v].get(j);
        }
      }
    }
    if (piece) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (columns(v).any) store_w<FiraStoredF32, W>(s.partial + unit * e.dim + columns(v).at, sum[v]);
    } else if (row >= 0) {
      finish(row0 + row * kBuckets);
    }
  }
}

// 32 W columns of a row in pieces per workgroup: its eight half wavefronts take every eighth piece each, and their sums are added in turn.  (With
// 64 W columns and sixteen wavefronts the chip holds fewer rows at a time than a text of 131072 tokens has, and a row is mostly latency.)
template <typename T, int W, bool ADD>
__global__ __launch_bounds__(256) void fira_embed_join_kernel(FiraEmbed e, typename T::raw* dtable, FiraEmbedSort s) {
  constexpr int PARTS = 8, N = 8;
  __shared__ float part[PARTS][32 * W];
  const int lane = threadIdx.x & 31, mine = threadIdx.x >> 5;
  const long long tiles = (e.dim + 32 * W - 1) / (32 * W), all = *as_global(s.counters + 1) * tiles;
  for (long long i = blockIdx.x; i < all; i += gridDim.x) {
    const u32x4 row = *as_global(s.cut + i / tiles);
    const Columns<W> c(i % tiles * (32 * W) + lane * W, e.dim);
    const int pieces = (int)row[2];
    const float* const from = s.partial + (long long)row[1] * e.dim + c.at;
    float sum[W] = {};
    for (int first = mine; first < pieces; first += PARTS * N) {
      Raw<FiraStoredF32, W> x[N];
#pragma unroll
      for (int k = 0; k < N; ++k) x[k].load(from + (long long)min(first + PARTS * k, pieces - 1) * e.dim);
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (first + PARTS * k < pieces)
#pragma unroll
          for (int j = 0; j < W; ++j) sum[j] += x[k].get(j);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < W; ++j) part[mine][j * 32 + lane] = sum[j];
    __syncthreads();
    if (mine == 0 && c.any) {
#pragma unroll
      for (int w = 1; w < PARTS; ++w)
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] += part[w][j * 32 + lane];
      write_gradient<T, W, ADD>(e, dtable, row[0], c, sum);
    }
  }
}

// Few tokens: no sort, every workgroup looks through all ids for kFewBatch neighbouring rows of the table and 64 W columns.  A row's tokens are summed in
// the pieces and parts of the kernels above, so that it gets the same bits whatever the number of other tokens; of a row with more than one piece each
// wavefront takes two of the eight parts (one token for all of 256: 34 us with one wavefront for it, 19 with four).
// Up to kFewTokens, the most that two pieces a part hold; us here and with the sort, bf16: 512 tokens x 512 of 32000 rows 9.6 and 20.4, x 2048 24.7 and 36.5, x 512
// of 131072 rows 25 and 38, x 192 of 768 rows 15.0 and 15.9; the sort is ahead where most tokens are one id of a small table (512 x 512, all of them 36 and 24).
constexpr int kFewTokens = 512, kFewBatch = 32;
template <typename T, typename R, int W, bool ADD>
__global__ __launch_bounds__(256) void fira_embed_few_kernel(FiraEmbed e, const typename R::raw* dout, const void* ids, typename T::raw* dtable) {
  constexpr int N = 8, PARTS = 8, GROUPS = kFewTokens / 64;
  static_assert(kFewTokens <= 2 * PARTS * kPieceTokens, "a part is of two pieces at most");
  __shared__ short found[4][kFewTokens];
  __shared__ float parts[PARTS][64 * W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned tiles = (unsigned)((e.dim + 64 * W - 1) / (64 * W));
  const long long all = (e.vocab + kFewBatch - 1LL) / kFewBatch * tiles;
  int id[GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) id[g] = g * 64 + lane < e.count ? token_row(e, ids, g * 64 + lane) : -1;
  volatile short* const mine = found[wave];
  for (long long i = blockIdx.x; i < all; i += gridDim.x) {
    const long long unit = i / tiles;
    const Columns<W> c((i - unit * tiles) * (64 * W) + lane * W, e.dim);
    const int row0 = (int)unit * kFewBatch, rows = min(kFewBatch, e.vocab - row0);
    unsigned named = 0, several = 0;                     // rows of these with a token, with more than one piece
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      unsigned long long m = __ballot((unsigned)(id[g] - row0) < (unsigned)rows && id[g] >= 0);
      for (; m; m &= m - 1) named |= 1u << (__builtin_amdgcn_readlane(id[g], __builtin_ctzll(m)) - row0);
    }
    // the row's tokens in order, in this wavefront's list; their number
    auto find = [&](int k) {
      int total = 0;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const bool is = id[g] == row0 + k;
        const unsigned long long m = __ballot(is);
        if (is) mine[total + __popcll(m & ((1ull << lane) - 1))] = (short)(g * 64 + lane);
        total += __popcll(m);
      }
      __builtin_amdgcn_wave_barrier();
      return total;
    };
    auto add_piece = [&](int p0, int total, float (&sum)[W]) {
      float piece[W] = {};
      const int until = min(p0 + kPieceTokens, total);
      const int token = mine[min(p0 + (lane & (kPieceTokens - 1)), until - 1)];
#pragma unroll 1
      for (int first = 0; p0 + first < until; first += N) {
        Raw<R, W> x[N];
#pragma unroll
        for (int u = 0; u < N; ++u) x[u].load(dout + (long long)__builtin_amdgcn_readlane(token, first + u) * e.ld_rows + c.at);
#pragma unroll
        for (int u = 0; u < N; ++u)
          if (p0 + first + u < until)
#pragma unroll
            for (int j = 0; j < W; ++j) piece[j] += x[u].get(j);
      }
#pragma unroll
      for (int j = 0; j < W; ++j) sum[j] += piece[j];
    };
    float zeros[W] = {};
    if (!ADD)                                            // rows without a token, a quarter for each wavefront
      for (unsigned m = ~named & (rows == 32 ? ~0u : (1u << rows) - 1) & (0xffu << 8 * wave); m; m &= m - 1)
        if (c.any) write_gradient<T, W, ADD>(e, dtable, row0 + __builtin_ctz(m), c, zeros);
#pragma unroll 1
    for (unsigned m = named; m; m &= m - 1) {            // rows of one piece: a wavefront each
      const int k = __builtin_ctz(m), total = find(k);
      if (total > kPieceTokens) { several |= 1u << k; continue; }
      if (k / 8 != wave) continue;
      float sum[W] = {};
      add_piece(0, total, sum);
      if (c.any) write_gradient<T, W, ADD>(e, dtable, row0 + k, c, sum);
    }
    for (; several; several &= several - 1) {            // (the same rows for all wavefronts)
      const int k = __builtin_ctz(several), total = find(k);
#pragma unroll 1
      for (int part = wave; part < PARTS; part += 4) {
        float sum[W] = {};
#pragma unroll 1
        for (int p0 = part * kPieceTokens; p0 < total; p0 += PARTS * kPieceTokens) add_piece(p0, total, sum);
#pragma unroll
        for (int j = 0; j < W; ++j) parts[part][j * 64 + lane] = sum[j];
      }
      __syncthreads();
      if (wave == 0) {
        float sum[W];
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] = parts[0][j * 64 + lane];
#pragma unroll
        for (int part = 1; part < PARTS; ++part)
#pragma unroll
          for (int j = 0; j < W; ++j) sum[j] += parts[part][j * 64 + lane];
        if (c.any) write_gradient<T, W, ADD>(e, dtable, row0 + k, c, sum);
      }
      __syncthreads();
    }
  }
}
