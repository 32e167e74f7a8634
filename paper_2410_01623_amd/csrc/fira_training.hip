// Host side of the operators around the step (include/fira.h): checks of the arguments and launches.  gfx950 only; no state, no
// allocation, nothing that throws.
#include "../../include/fira.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "fira_error.h"
#include "fira_embed.h"
#include "fira_layer_norm.h"
#include "fira_clip.h"

namespace {

constexpr int64_t kMost = 0x7fffffff, kMostDim = 1 << 24;

__attribute__((format(printf, 2, 3))) fira_status refuse(fira_status st, const char* format, ...) {
  char msg[256];
  va_list args;
  va_start(args, format);
  std::vsnprintf(msg, sizeof msg, format, args);
  va_end(args);
  return fira_fail_without_context(st, msg);
}

fira_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FIRA_OK : refuse(FIRA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

template <int N>
using Int = std::integral_constant<int, N>;

bool known(int32_t dtype) { return dtype == FIRA_F32 || dtype == FIRA_BF16; }
size_t size_of(int32_t dtype) { return dtype == FIRA_F32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// A pointer that has to be there and aligned to its elements.
#define FIRA_POINTER(p, bytes)                                                                              \
  do {                                                                                                      \
    if (!(p)) return refuse(FIRA_ERR_INVALID_ARG, #p " is null");                                           \
    if (!aligned(p, bytes)) return refuse(FIRA_ERR_INVALID_ARG, #p " is not aligned to its elements");      \
  } while (0)
#define FIRA_LEADING(ld, width, rows)                                                                       \
  do {                                                                                                      \
    if ((ld) < (width)) return refuse(FIRA_ERR_SHAPE, #ld " is below the width");                           \
    int64_t span_;                                                                                          \
    if (__builtin_mul_overflow((int64_t)(ld), (int64_t)(rows) + 1, &span_) || span_ > INT64_MAX / 4)        \
      return refuse(FIRA_ERR_SHAPE, #ld " is out of range");                                                \
  } while (0)

fira_status check_workspace(const void* p, size_t have, size_t need) {
  if (have < need || (need && !p)) return refuse(FIRA_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", p ? have : (size_t)0, need);
  if (!aligned(p, 256)) return refuse(FIRA_ERR_WORKSPACE, "workspace is not aligned to 256 bytes");
  return FIRA_OK;
}

// Calls f with the types that two fira_dtypes stand for.
template <typename F>
void with_types(int32_t a, int32_t b, F f) {
  if (a == FIRA_F32) { if (b == FIRA_F32) f(FiraStoredF32{}, FiraStoredF32{}); else f(FiraStoredF32{}, FiraStoredBf16{}); }
  else { if (b == FIRA_F32) f(FiraStoredBf16{}, FiraStoredF32{}); else f(FiraStoredBf16{}, FiraStoredBf16{}); }
}

// Calls f with `flag` as a constant.
template <typename F>
void with_flag(bool flag, F f) {
  if (flag) f(std::true_type{});
  else f(std::false_type{});
}

fira_status check_embed(const fira_embed_desc* d, int64_t count) {
  if (!d) return refuse(FIRA_ERR_INVALID_ARG, "null descriptor");
  if (d->rows < 1 || d->rows > kMostEmbedRows || d->dim < 1 || d->dim > kMostDim) return refuse(FIRA_ERR_SHAPE, "embedding table of %lld x %lld", (long long)d->rows, (long long)d->dim);
  FIRA_LEADING(d->ld, d->dim, d->rows);
  if (count < 0 || count > kMost) return refuse(FIRA_ERR_SHAPE, "%lld tokens", (long long)count);
  if (!known(d->dtype) || !known(d->row_dtype)) return refuse(FIRA_ERR_DTYPE, "embedding types %d and %d", d->dtype, d->row_dtype);
  if (d->id_type != FIRA_I32 && d->id_type != FIRA_I64) return refuse(FIRA_ERR_DTYPE, "index type %d", d->id_type);
  if (!std::isfinite((float)d->scale)) return refuse(FIRA_ERR_INVALID_ARG, "scale is not finite");
  return FIRA_OK;
}

FiraEmbed embed_of(const fira_embed_desc* d, int64_t count, int64_t ld_rows) {
  return FiraEmbed{(int)d->rows, d->dim, d->ld, count, ld_rows, (float)d->scale, d->id_type == FIRA_I64};
}

// The gradient's workspace.
struct EmbedSort {
  FiraEmbedSort s;
  int64_t pieces;     // at most so many: rows in pieces have more than kPieceTokens tokens each
  size_t bytes;
};
EmbedSort embed_sort(const fira_embed_desc* d, int64_t count, char* at) {
  EmbedSort r{};
  FiraEmbedSort& s = r.s;
  if (count <= kFewTokens) { r.bytes = FIRA_UNUSED_WORKSPACE_BYTES; return r; }      // no sort
  char* const begin = at;
  auto take = [&](auto*& p, int64_t n) { p = (std::remove_reference_t<decltype(p)>)at; at += up256(n * sizeof *p); };
  s.chunk = (int)std::max<int64_t>(512, up256((count + kMostChunks - 1) / kMostChunks));
  s.chunks = (int)std::max<int64_t>(1, (count + s.chunk - 1) / s.chunk);
  s.bins = (int)((d->rows + kBuckets - 1) / kBuckets);
  while (1 << s.bits < s.bins) ++s.bits;
  r.pieces = 2 * (count / kPieceTokens);
  take(s.sorted, (int64_t)s.chunks * s.chunk);
  take(s.gathered, count);
  take(s.part, (int64_t)kBuckets * s.chunks);
  take(s.order, count);
  take(s.rows, (int64_t)kBuckets * s.bins);
  take(s.counters, 2);
  take(s.pieces, r.pieces);
  take(s.cut, r.pieces);
  take(s.partial, r.pieces * d->dim);
  r.bytes = at - begin;                                 // (more than that, of the lists' parts alone)
  return r;
}

fira_status check_norm(const fira_layer_norm_desc* d) {
  if (!d) return refuse(FIRA_ERR_INVALID_ARG, "null descriptor");
  if (d->rows < 0 || d->rows > kMost || d->dim < 1 || d->dim > kMostDim) return refuse(FIRA_ERR_SHAPE, "norm of %lld rows of %lld", (long long)d->rows, (long long)d->dim);
  if (!known(d->dtype) || !known(d->param_dtype)) return refuse(FIRA_ERR_DTYPE, "norm types %d and %d", d->dtype, d->param_dtype);
  if (d->kind != FIRA_LAYER_NORM && d->kind != FIRA_RMS_NORM) return refuse(FIRA_ERR_INVALID_ARG, "norm kind %d", d->kind);
  if (!(d->eps >= 0.0) || !std::isfinite((float)d->eps)) return refuse(FIRA_ERR_INVALID_ARG, "eps is negative or not finite");
  return FIRA_OK;
}

// Calls f with the constants that a row of `dim` <= kNormWidest values of type T is held by: values of a vector, threads, vectors of a thread.
// EACH: values of a thread where a row takes more than a wavefront, 8 or 16.
template <typename T, int EACH, typename F>
void with_row_shape(int64_t dim, F f) {
  constexpr int W = kWidth<T>, N = 8 / W, D = EACH / 8;
  if (dim < kMostWidth) f(Int<1>{}, Int<8>{}, Int<1>{});
  else if (dim <= 8 * W) f(Int<W>{}, Int<8>{}, Int<1>{});
  else if (dim <= 16 * W) f(Int<W>{}, Int<16>{}, Int<1>{});
  else if (dim <= 32 * W) f(Int<W>{}, Int<32>{}, Int<1>{});
  else if (dim <= 64 * W) f(Int<W>{}, Int<64>{}, Int<1>{});
  else if (dim <= 512) f(Int<W>{}, Int<64>{}, Int<N>{});
  else if (dim <= 1024) f(Int<W>{}, Int<128 / D>{}, Int<D * N>{});
  else if (dim <= 2048) f(Int<W>{}, Int<256 / D>{}, Int<D * N>{});
  else if (dim <= 4096) f(Int<W>{}, Int<512 / D>{}, Int<D * N>{});
  else if (dim <= 8192) f(Int<W>{}, Int<1024 / D>{}, Int<D * N>{});
  else f(Int<W>{}, Int<1024>{}, Int<2 * N>{});
}
// Workgroups of the norm's gradient, each of which leaves its sums over rows: as many as the chip holds, but fewer where that leaves each less than ten
// turns (of a row, or of the rows that it has side by side), and a quarter of that at least.  2048 rows x 2048 f32: 16.5 us with 256 workgroups, 17.6
// with 512, 24.7 with 1024; 5840 x 1680 f32: 34, 29.6 and 33.7; 16384 x 2048 bf16: 57, 49.7 and 49.3.
int64_t norm_parts(const fira_layer_norm_desc* d) {
  if (d->dim > kNormWidest) return std::min<int64_t>(d->rows, 64);
  int64_t parts = 1;
  auto shape = [&](auto, auto threads, auto) {
    constexpr int THREADS = decltype(threads)::value, GROUPS = std::max(1, 256 / THREADS);
    constexpr int64_t full = 256 * 1024 / std::max(256, THREADS);
    const int64_t turns = std::max<int64_t>(1, (d->rows + GROUPS - 1) / GROUPS);
    const int64_t each = std::min(std::max<int64_t>(10, (turns + full - 1) / full), (4 * turns + full - 1) / full);
    parts = (turns + each - 1) / each;
  };
  if (d->dtype == FIRA_F32) with_row_shape<FiraStoredF32, 8>(d->dim, shape);
  else with_row_shape<FiraStoredBf16, 8>(d->dim, shape);
  return parts;
}

fira_status check_gradients(const fira_gradient_desc* d, int count, bool outs) {
  if (count < 0) return refuse(FIRA_ERR_INVALID_ARG, "%d gradients", count);
  if (count && !d) return refuse(FIRA_ERR_INVALID_ARG, "null descriptors");
  for (int i = 0; i < count; ++i) {
    if (d[i].rows < 0 || d[i].cols < 0 || d[i].rows > kMost) return refuse(FIRA_ERR_SHAPE, "gradient %d of %lld x %lld", i, (long long)d[i].rows, (long long)d[i].cols);
    if (!known(d[i].dtype) || (outs && !known(d[i].out_dtype))) return refuse(FIRA_ERR_DTYPE, "type of gradient %d", i);
    FIRA_LEADING(d[i].ld, d[i].cols, d[i].rows);
    if (outs) FIRA_LEADING(d[i].ld_out, d[i].cols, d[i].rows);
  }
  return FIRA_OK;
}

// Cuts a gradient into pieces that the kernels take, in vectors of `width` values: at most kPiece values a row and kPiece vectors in all.
constexpr int64_t kPiece = 1 << 30;
template <typename F>
void cut_up(const fira_gradient_desc& d, const void* g, void* out, bool outs, int width, F piece) {
  int64_t rows = d.rows, cols = d.cols, ld = d.ld, ld_out = outs ? d.ld_out : d.ld;
  if (!rows || !cols) return;
  const size_t size = size_of(d.dtype), size_out = size_of(outs ? d.out_dtype : d.dtype);
  if (ld == cols && ld_out == cols) { cols *= rows; rows = 1; }                       // dense: one long row
  const bool by_row = ld > kPiece || ld_out > kPiece || cols > kPiece;
  const int64_t vecs = cols < width ? cols : (cols + width - 1) / width, some = by_row ? 1 : std::min(rows, kPiece / std::min(vecs, kPiece));
  for (int64_t r = 0; r < rows; r += some)
    for (int64_t c = 0; c < cols; c += kPiece) {
      const int64_t n = std::min(kPiece, cols - c);
      piece(FiraSpan{(const char*)g + (r * ld + c) * size, (char*)out + (r * ld_out + c) * size_out, (int)std::min(some, rows - r), (int)n,
                     by_row ? 0 : (int)ld, by_row ? 0 : (int)ld_out, (int)(n < width ? n : (n + width - 1) / width), 0});
    }
}

// Collects the pieces of one pair of types and hands them over a launch at a time.
struct Batch {
  FiraSpans l{};
  void add(FiraSpan s) {
    s.tile0 = l.tiles;
    l.s[l.count++] = s;
    l.tiles += (int)(((int64_t)s.rows * s.vecs + kClipTile - 1) / kClipTile);
  }
  // (2^30 vectors are 2^20 tiles a piece, so a launch's tiles fit 32 bits)
  bool full() const { return l.count == kSpans; }
};
int workgroups(const FiraSpans& l) { return (l.tiles + l.each - 1) / l.each; }

// Calls f(types, pieces) for every launch that the list takes, types by types; by_out: the results' types as well.
template <typename F>
void for_each_launch(const fira_gradient_desc* d, int count, const void* const* G, void* const* out, bool by_out, F f) {
  for (int in = 0; in < 2; ++in)
    for (int to = 0; to < (by_out ? 2 : 1); ++to) {
      Batch b;
      const int width = in == FIRA_F32 || (by_out && to == FIRA_F32) ? kWidth<FiraStoredF32> : kWidth<FiraStoredBf16>;
      auto flush = [&] {
        b.l.each = (b.l.tiles + kClipWorkgroups - 1) / kClipWorkgroups;
        if (b.l.count) f(in, to, b.l);
        b.l.count = b.l.tiles = 0;
      };
      for (int i = 0; i < count; ++i) {
        if (d[i].dtype != in || (by_out && (out ? d[i].out_dtype : d[i].dtype) != to)) continue;
        cut_up(d[i], G ? G[i] : nullptr, out ? out[i] : G ? const_cast<void*>(G[i]) : nullptr, by_out && out, width, [&](const FiraSpan& s) { b.add(s); if (b.full()) flush(); });
      }
      flush();
    }
}

// Partial sums of all launches.
int64_t partials(const fira_gradient_desc* d, int count) {
  int64_t n = 0;
  for_each_launch(d, count, nullptr, nullptr, false, [&](int, int, const FiraSpans& l) { n += workgroups(l); });
  return n;
}

fira_status check_gradient_pointers(const fira_gradient_desc* d, int count, const void* const* G, void* const* out) {
  if (count && !G) return refuse(FIRA_ERR_INVALID_ARG, "null list of gradients");
  for (int i = 0; i < count; ++i) {
    if (!d[i].rows || !d[i].cols) continue;
    if (!G[i] || !aligned(G[i], size_of(d[i].dtype))) return refuse(FIRA_ERR_INVALID_ARG, "gradient %d is null or not aligned to its elements", i);
    if (!out) continue;
    if (!out[i] || !aligned(out[i], size_of(d[i].out_dtype))) return refuse(FIRA_ERR_INVALID_ARG, "result %d is null or not aligned to its elements", i);
    if (out[i] == G[i] && (d[i].dtype != d[i].out_dtype || (d[i].rows > 1 && d[i].ld != d[i].ld_out)))
      return refuse(FIRA_ERR_INVALID_ARG, "gradient %d in place with another type or leading dimension", i);
  }
  return FIRA_OK;
}

void launch_squares(const fira_gradient_desc* d, int count, const void* const* G, double* partial, hipStream_t q) {
  for_each_launch(d, count, G, nullptr, false, [&](int in, int, const FiraSpans& l) {
    const int n = workgroups(l);
    if (in == FIRA_F32) hipLaunchKernelGGL(fira_gradient_squares_kernel<FiraStoredF32>, dim3(n), dim3(256), 0, q, l, partial);
    else hipLaunchKernelGGL(fira_gradient_squares_kernel<FiraStoredBf16>, dim3(n), dim3(256), 0, q, l, partial);
    partial += n;
  });
}

}  // namespace

extern "C" {

fira_status fira_embed_lookup(const fira_embed_desc* d, const void* dev_table, const void* dev_ids, int64_t count, void* dev_out,
                              int64_t ld_out, void* hip_stream) {
  if (const fira_status st = check_embed(d, count)) return st;
  if (!count) return FIRA_OK;
  FIRA_LEADING(ld_out, d->dim, count);
  FIRA_POINTER(dev_table, size_of(d->dtype));
  FIRA_POINTER(dev_ids, d->id_type == FIRA_I64 ? 8 : 4);
  FIRA_POINTER(dev_out, size_of(d->row_dtype));
  const FiraEmbed e = embed_of(d, count, ld_out);
  with_types(d->dtype, d->row_dtype, [&](auto t, auto r) {
    typedef decltype(t) T;
    typedef decltype(r) R;
    auto launch = [&](auto w, auto lanes, auto nv, auto tokens) {
      constexpr int W = decltype(w)::value, LANES = decltype(lanes)::value, NV = decltype(nv)::value, TOKENS = decltype(tokens)::value;
      const int64_t units = (count + TOKENS - 1) / TOKENS * ((d->dim + NV * LANES * W - 1) / (NV * LANES * W));
      hipLaunchKernelGGL((fira_embed_lookup_kernel<T, R, W, LANES, NV, TOKENS>), dim3(std::min<int64_t>((units + 3) / 4, 1 << 20)), dim3(256), 0,
                         (hipStream_t)hip_stream, e, (const typename T::raw*)dev_table, dev_ids, (typename R::raw*)dev_out);
    };
    constexpr int W = kWidth<T, R>;
    if (d->dim < kMostWidth) launch(Int<1>{}, Int<8>{}, Int<1>{}, Int<8>{});
    else if (d->dim <= 8 * W) launch(Int<W>{}, Int<8>{}, Int<1>{}, Int<16>{});
    else if (d->dim <= 16 * W) launch(Int<W>{}, Int<16>{}, Int<1>{}, Int<8>{});
    else if (d->dim <= 32 * W) launch(Int<W>{}, Int<32>{}, Int<1>{}, Int<4>{});
    // (2048 or 1024 columns where a row is made of such, else 512.  Wide ones pay where tables and results leave the caches, and cost where few wavefronts are
    // left to wait.  us with 512, 1024 and 2048 columns, 32000 rows: 131072 tokens x 2048, f32 to bf16 176, 175, 169, bf16 120, 115, 117, bf16 to f32 190, 209, 203;
    // 65536 x 4096 bf16 153, 132, 143; 131072 x 1024 bf16 55, 57, 57, of 131072 rows 70, 60, 61; 4096 x 2048 bf16 6.4, 6.0, 5.9; 16384 x 4096 bf16 31, 34, 34;
    // 256 x 2048 bf16 3.0, 3.2, 3.7, which is less than the call takes to reach the GPU)
    else if ((d->dim + 511) / 512 % 4 == 0) launch(Int<W>{}, Int<64>{}, Int<32 / W>{}, Int<2>{});
    else if ((d->dim + 511) / 512 % 2 == 0) launch(Int<W>{}, Int<64>{}, Int<16 / W>{}, Int<2>{});
    else launch(Int<W>{}, Int<64>{}, Int<8 / W>{}, Int<2>{});
  });
  return launched("embedding lookup");
}

size_t fira_embed_gradient_workspace_bytes(const fira_embed_desc* d, int64_t count) {
  return check_embed(d, count) ? 0 : embed_sort(d, count, nullptr).bytes;
}

fira_status fira_embed_gradient(const fira_embed_desc* d, const void* dev_dout, int64_t ld_dout, const void* dev_ids, int64_t count,
                                void* dev_dtable, int accumulate, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  if (const fira_status st = check_embed(d, count)) return st;
  if (count) {
    FIRA_LEADING(ld_dout, d->dim, count);
    FIRA_POINTER(dev_dout, size_of(d->row_dtype));
    FIRA_POINTER(dev_ids, d->id_type == FIRA_I64 ? 8 : 4);
  }
  FIRA_POINTER(dev_dtable, size_of(d->dtype));
  const EmbedSort sort = embed_sort(d, count, (char*)dev_workspace);
  if (const fira_status st = check_workspace(dev_workspace, workspace_bytes, sort.bytes)) return st;
  if (!count && accumulate) return FIRA_OK;
  const FiraEmbed e = embed_of(d, count, ld_dout);
  const FiraEmbedSort& s = sort.s;   // (not made for few tokens)
  const hipStream_t q = (hipStream_t)hip_stream;
  with_types(d->dtype, d->row_dtype, [&](auto t, auto r) {
    typedef decltype(t) T;
    typedef decltype(r) R;
    const typename R::raw* const dout = (const typename R::raw*)dev_dout;
    typename T::raw* const dtable = (typename T::raw*)dev_dtable;
    const int64_t dim = d->dim;
    auto grid = [](int64_t units, int64_t per) { return dim3(std::min<int64_t>((units + per - 1) / per, 1 << 20)); };
    with_flag(accumulate, [&](auto add) {
      constexpr bool ADD = decltype(add)::value;
      if (count <= kFewTokens) {
        auto few = [&](auto w) {
          constexpr int W = decltype(w)::value;
          hipLaunchKernelGGL((fira_embed_few_kernel<T, R, W, ADD>), grid((d->rows + kFewBatch - 1) / kFewBatch * ((dim + 64 * W - 1) / (64 * W)), 1), dim3(256), 0, q, e,
                             dout, dev_ids, dtable);
        };
        if (dim < kMostWidth) few(Int<1>{});
        else few(Int<kWidth<T, R>>{});
        return;
      }
      hipLaunchKernelGGL(fira_embed_chunk_kernel, dim3(s.chunks), dim3(256), 0, q, e, dev_ids, s);
      const int waves = std::min(16, kCounters / s.bins);
      hipLaunchKernelGGL(fira_embed_bucket_kernel, dim3(kBuckets), dim3(64 * waves), 4 * kCounters, q, e, s);
      auto narrow = [&](auto w, auto lanes) {
        constexpr int W = decltype(w)::value, LANES = decltype(lanes)::value;
        hipLaunchKernelGGL((fira_embed_sum_narrow_kernel<T, R, W, LANES, ADD>), grid(sort.pieces + d->rows, 256 / LANES), dim3(256), 0, q, e, dout, dtable, s);
      };
      const int64_t batches = (int64_t)((s.bins + kBatch - 1) / kBatch) * kBuckets;
      constexpr int W = kWidth<T, R>;
      if (dim < kMostWidth) narrow(Int<1>{}, Int<8>{});
      else if (dim <= 8 * W) narrow(Int<W>{}, Int<8>{});
      else if (dim <= 16 * W) narrow(Int<W>{}, Int<16>{});
      else if (dim <= 32 * W) narrow(Int<W>{}, Int<32>{});
      else hipLaunchKernelGGL((fira_embed_sum_kernel<T, R, ADD>), grid((sort.pieces + batches) * ((dim + 511) / 512), 4), dim3(256), 0, q, e, dout, dtable, s);
      // (a row in pieces has kPieceTokens + 1 tokens at least)
      auto join = [&](auto w) {
        constexpr int W = decltype(w)::value;
        hipLaunchKernelGGL((fira_embed_join_kernel<T, W, ADD>), dim3(std::min<int64_t>(count / (kPieceTokens + 1) * ((dim + 32 * W - 1) / (32 * W)), 4096)), dim3(256),
                           0, q, e, dtable, s);
      };
      if (dim < kMostWidth) join(Int<1>{});
      else join(Int<kWidth<FiraStoredF32>>{});
    });
  });
  return launched("embedding gradient");
}

fira_status fira_layer_norm(const fira_layer_norm_desc* d, const void* dev_x, int64_t ld_x, const void* dev_weight, const void* dev_bias,
                            void* dev_y, int64_t ld_y, float* dev_mean, float* dev_rstd, void* hip_stream) {
  if (const fira_status st = check_norm(d)) return st;
  if (!d->rows) return FIRA_OK;
  FIRA_LEADING(ld_x, d->dim, d->rows);
  FIRA_LEADING(ld_y, d->dim, d->rows);
  FIRA_POINTER(dev_x, size_of(d->dtype));
  FIRA_POINTER(dev_y, size_of(d->dtype));
  if (!aligned(dev_weight, size_of(d->param_dtype)) || !aligned(dev_bias, size_of(d->param_dtype)) || !aligned(dev_mean, 4) || !aligned(dev_rstd, 4))
    return refuse(FIRA_ERR_INVALID_ARG, "weight, bias, mean or rstd is not aligned to its elements");
  const FiraNorm n{d->rows, d->dim, ld_x, ld_y, 0, (float)d->eps, d->kind == FIRA_RMS_NORM};
  with_types(d->dtype, d->param_dtype, [&](auto t, auto p) {
    typedef decltype(t) T;
    typedef decltype(p) P;
    const typename T::raw* const x = (const typename T::raw*)dev_x;
    const typename P::raw *const w = (const typename P::raw*)dev_weight, *const b = (const typename P::raw*)dev_bias;
    typename T::raw* const y = (typename T::raw*)dev_y;
    float* const mean = n.rms ? nullptr : dev_mean;
    const hipStream_t q = (hipStream_t)hip_stream;
    if (d->dim > kNormWidest) {
      hipLaunchKernelGGL((fira_layer_norm_wide_kernel<T, P>), dim3(std::min<int64_t>(d->rows, 1 << 20)), dim3(1024), 0, q, n, x, w, b, y, mean, dev_rstd);
      return;
    }
    with_row_shape<T, 16>(d->dim, [&](auto width, auto threads, auto nv) {
      constexpr int W = decltype(width)::value, THREADS = decltype(threads)::value, NV = decltype(nv)::value, GROUPS = std::max(1, 256 / THREADS);
      hipLaunchKernelGGL((fira_layer_norm_kernel<T, P, W, THREADS, NV>), dim3(std::min<int64_t>((d->rows + GROUPS - 1) / GROUPS, 1 << 20)),
                         dim3(std::max(256, THREADS)), 0, q, n, x, w, b, y, mean, dev_rstd);
    });
  });
  return launched("layer norm");
}

size_t fira_layer_norm_gradient_workspace_bytes(const fira_layer_norm_desc* d) {
  if (check_norm(d)) return 0;
  return d->rows <= kFewRows && d->dim <= kNormWidest ? FIRA_UNUSED_WORKSPACE_BYTES : std::max<size_t>(2 * FIRA_UNUSED_WORKSPACE_BYTES, up256(2 * norm_parts(d) * d->dim * 4));
}

fira_status fira_layer_norm_gradient(const fira_layer_norm_desc* d, const void* dev_dy, int64_t ld_dy, const void* dev_x, int64_t ld_x,
                                     const void* dev_weight, const float* dev_mean, const float* dev_rstd, void* dev_dx, int64_t ld_dx,
                                     void* dev_dweight, void* dev_dbias, int accumulate, void* dev_workspace, size_t workspace_bytes,
                                     void* hip_stream) {
  if (const fira_status st = check_norm(d)) return st;
  if (d->rows) {
    FIRA_LEADING(ld_dy, d->dim, d->rows);
    FIRA_LEADING(ld_x, d->dim, d->rows);
    if (dev_dx) FIRA_LEADING(ld_dx, d->dim, d->rows);
    FIRA_POINTER(dev_dy, size_of(d->dtype));
    FIRA_POINTER(dev_x, size_of(d->dtype));
    FIRA_POINTER(dev_rstd, 4);
    if (d->kind == FIRA_LAYER_NORM) FIRA_POINTER(dev_mean, 4);
    if (!aligned(dev_dx, size_of(d->dtype))) return refuse(FIRA_ERR_INVALID_ARG, "dev_dx is not aligned to its elements");
  }
  if (!aligned(dev_weight, size_of(d->param_dtype)) || !aligned(dev_dweight, size_of(d->param_dtype)) || !aligned(dev_dbias, size_of(d->param_dtype)))
    return refuse(FIRA_ERR_INVALID_ARG, "weight, dweight or dbias is not aligned to its elements");
  if (const fira_status st = check_workspace(dev_workspace, workspace_bytes, fira_layer_norm_gradient_workspace_bytes(d))) return st;
  const FiraNorm n{d->rows, d->dim, ld_x, ld_dy, ld_dx, (float)d->eps, d->kind == FIRA_RMS_NORM};
  with_types(d->dtype, d->param_dtype, [&](auto t, auto p) {
    typedef decltype(t) T;
    typedef decltype(p) P;
    const typename T::raw *const dy = (const typename T::raw*)dev_dy, *const x = (const typename T::raw*)dev_x;
    const typename P::raw* const w = (const typename P::raw*)dev_weight;
    typename T::raw* const dx = (typename T::raw*)dev_dx;
    const hipStream_t q = (hipStream_t)hip_stream;
    if (d->rows <= kFewRows && d->dim <= kNormWidest) {
      with_row_shape<T, 8>(d->dim, [&](auto width, auto threads, auto nv) {
        constexpr int W = decltype(width)::value, THREADS = decltype(threads)::value, NV = decltype(nv)::value, GROUPS = std::max(1, 256 / THREADS);
        const int rows = dx ? (int)((d->rows + GROUPS - 1) / GROUPS) : 0;
        const int columns = (dev_dweight || dev_dbias) && (d->rows || !accumulate) ? (int)((d->dim + 8 * W - 1) / (8 * W)) : 0;
        if (rows + columns)
          hipLaunchKernelGGL((fira_layer_norm_gradient_few_kernel<T, P, W, THREADS, NV>), dim3(rows + columns), dim3(std::max(256, THREADS)), 0, q, n, dy, x, w, dev_mean,
                             dev_rstd, dx, (typename P::raw*)dev_dweight, (typename P::raw*)dev_dbias, accumulate, rows);
      });
      return;
    }
    const int parts = (int)norm_parts(d);
    float* const pw = dev_dweight ? (float*)dev_workspace : nullptr;
    float* const pb = dev_dbias ? (float*)dev_workspace + (int64_t)parts * d->dim : nullptr;
    if (d->dim > kNormWidest) {
      if (dx && d->rows) hipLaunchKernelGGL((fira_layer_norm_wide_dx_kernel<T, P>), dim3(std::min<int64_t>(d->rows, 1 << 20)), dim3(1024), 0, q, n, dy, x, w, dev_mean, dev_rstd, dx);
      if ((pw || pb) && d->rows) hipLaunchKernelGGL(fira_layer_norm_wide_dw_kernel<T>, dim3((d->dim + 255) / 256, parts), dim3(256), 0, q, n, dy, x, dev_mean, dev_rstd, pw, pb);
    } else if (dx || pw || pb) {
      with_row_shape<T, 8>(d->dim, [&](auto width, auto threads, auto nv) {
        constexpr int W = decltype(width)::value, THREADS = decltype(threads)::value, NV = decltype(nv)::value;
        hipLaunchKernelGGL((fira_layer_norm_gradient_kernel<T, P, W, THREADS, NV>), dim3(parts), dim3(std::max(256, THREADS)), 0, q, n, dy, x, w, dev_mean, dev_rstd, dx,
                           pw, pb);
      });
    }
    if ((pw || pb) && (d->rows || !accumulate))
      hipLaunchKernelGGL(fira_layer_norm_join_kernel<P>, dim3((d->dim + 31) / 32, 2), dim3(256), 0, q, pw, pb, parts, d->dim, (typename P::raw*)dev_dweight,
                         (typename P::raw*)dev_dbias, accumulate);
  });
  return launched("layer norm gradient");
}

size_t fira_gradient_workspace_bytes(const fira_gradient_desc* d, int count) {
  return check_gradients(d, count, false) ? 0 : up256(8 * (partials(d, count) + 1));
}

fira_status fira_gradient_norm(const fira_gradient_desc* d, int count, const void* const* dev_G, float* dev_norm, void* dev_workspace,
                               size_t workspace_bytes, void* hip_stream) {
  if (const fira_status st = check_gradients(d, count, false)) return st;
  if (const fira_status st = check_gradient_pointers(d, count, dev_G, nullptr)) return st;
  FIRA_POINTER(dev_norm, 4);
  const int64_t n = partials(d, count);
  if (const fira_status st = check_workspace(dev_workspace, workspace_bytes, up256(8 * (n + 1)))) return st;
  launch_squares(d, count, dev_G, (double*)dev_workspace, (hipStream_t)hip_stream);
  hipLaunchKernelGGL(fira_gradient_norm_kernel<>, dim3(1), dim3(256), 0, (hipStream_t)hip_stream, (const double*)dev_workspace, (int)n, dev_norm);
  return launched("gradient norm");
}

fira_status fira_clip_gradients(const fira_gradient_desc* d, int count, void* const* dev_G, void* const* dev_out, double max_norm, float* dev_norm,
                                void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  if (const fira_status st = check_gradients(d, count, dev_out != nullptr)) return st;
  if (const fira_status st = check_gradient_pointers(d, count, dev_G, dev_out)) return st;
  if (!(max_norm >= 0.0)) return refuse(FIRA_ERR_INVALID_ARG, "max_norm is negative or not a number");
  FIRA_POINTER(dev_norm, 4);
  const int64_t n = partials(d, count);
  if (const fira_status st = check_workspace(dev_workspace, workspace_bytes, up256(8 * (n + 1)))) return st;
  const hipStream_t q = (hipStream_t)hip_stream;
  launch_squares(d, count, dev_G, (double*)dev_workspace, q);
  if (!n) hipLaunchKernelGGL(fira_gradient_norm_kernel<>, dim3(1), dim3(256), 0, q, (const double*)dev_workspace, 0, dev_norm);   // nothing in the list
  float* norm = dev_norm;                                // the first launch writes it
  for_each_launch(d, count, dev_G, dev_out, true, [&](int in, int to, const FiraSpans& l) {
    with_types(in, to, [&](auto t, auto r) {
      hipLaunchKernelGGL((fira_clip_kernel<decltype(t), decltype(r)>), dim3(workgroups(l)), dim3(256), 0, q, l, (const double*)dev_workspace, (int)n, max_norm, norm);
      norm = nullptr;
    });
  });
  return launched("gradient clipping");
}

}  // extern "C"
