// Host side of the operators that complete a training step (include/fira.h): checks of the arguments and launches.  gfx950 only; no
// state, no allocation, nothing that throws.
#include "fira_host.h"
#include "fira_adamw.h"
#include "fira_rotary.h"
#include "fira_block_norm.h"

namespace {

fira_status check_adamw(const fira_adamw_desc* d, int i) {
  if (d->rows < 0 || d->cols < 0 || d->rows > kMost) return refuse(FIRA_ERR_SHAPE, "tensor %d of %lld x %lld", i, (long long)d->rows, (long long)d->cols);
  if (!known(d->dtype) || !known(d->grad_dtype)) return refuse(FIRA_ERR_DTYPE, "types of tensor %d", i);
  if (d->state_type != FIRA_STATE_F32 && d->state_type != FIRA_STATE_E4M3) return refuse(FIRA_ERR_DTYPE, "state type of tensor %d", i);
  if (!(d->weight_decay >= 0.0) || !std::isfinite((float)d->weight_decay)) return refuse(FIRA_ERR_INVALID_ARG, "weight decay of tensor %d", i);
  FIRA_LEADING(d->ld_w, d->cols, d->rows);
  FIRA_LEADING(d->ld_g, d->cols, d->rows);
  if (d->rows > 1 && (d->ld_w != d->cols || d->ld_g != d->cols) && d->cols > kMost) return refuse(FIRA_ERR_SHAPE, "tensor %d has rows apart of %lld", i, (long long)d->cols);
  return FIRA_OK;
}

fira_status check_adamw_hparams(const fira_adamw_hparams* hp, bool norm) {
  if (!hp) return refuse(FIRA_ERR_INVALID_ARG, "null hyper-parameters");
  if (!std::isfinite((float)hp->lr)) return refuse(FIRA_ERR_INVALID_ARG, "lr is not finite");
  // (1 - beta has to be there in fp32, as beta itself)
  if (!(hp->beta1 >= 0.0 && hp->beta2 >= 0.0) || !((float)hp->beta1 < 1.0f && (float)hp->beta2 < 1.0f)) return refuse(FIRA_ERR_INVALID_ARG, "a beta is not in [0, 1)");
  if (!((float)hp->eps > 0.0f) || !std::isfinite((float)hp->eps)) return refuse(FIRA_ERR_INVALID_ARG, "eps is not positive and finite");
  if (norm && !(hp->max_norm >= 0.0)) return refuse(FIRA_ERR_INVALID_ARG, "max_norm is negative or not a number");
  return FIRA_OK;
}

bool adamw_apart(const fira_adamw_desc& d) { return d.rows > 1 && d.cols && (d.ld_w != d.cols || d.ld_g != d.cols); }

// Cuts a tensor into pieces that the kernel takes: from a whole block on, up to 2^30 values.
constexpr int64_t kAdamPiece = 1 << 30;
template <typename F>
void cut_adamw(const fira_adamw_desc& d, void* w, const void* g, const fira_adamw_state& s, F piece) {
  const int64_t n = d.rows * d.cols;
  const bool dense = !adamw_apart(d);
  const bool eight = d.state_type == FIRA_STATE_E4M3;
  for (int64_t i = 0; i < n; i += kAdamPiece) {
    const int64_t row = dense ? 0 : i / d.cols, col = dense ? 0 : i % d.cols, b = i / kAdamBlock;
    const int64_t at_w = dense ? i : row * d.ld_w, at_g = dense ? i : row * d.ld_g;
    FiraAdamSpan p{(char*)w + at_w * size_of(d.dtype), (const char*)g + at_g * size_of(d.grad_dtype), (char*)s.m + i * (eight ? 1 : 4), (char*)s.v + i * (eight ? 1 : 4),
                   eight ? s.m_scale + b : nullptr, eight ? s.v_scale + b : nullptr, d.ld_w, d.ld_g, 1.0 / (double)d.cols, (float)d.weight_decay,
                   (unsigned)std::min(kAdamPiece, n - i), dense ? 0u : (unsigned)d.cols, (unsigned)col, (unsigned)i, d.seed, 0, 0};
    // Lines that two wavefronts write parts of are put together in the caches, where stores have to leave them (511 x 1377 and the like, f32 and 8 bits: 61 us without, 52
    // with; 512 x 1376: 85 and 78 with fp32 states).
    if (aligned(p.w, 128) && (dense || d.ld_w * size_of(d.dtype) % 128 == 0)) p.stream |= 1;
    if (aligned(p.m, 128) && aligned(p.v, 128)) p.stream |= 2;
    piece(p);
  }
}

// Calls f(types, states in 8 bits, whether rows are apart and not whole vectors wide, pieces) for every launch that the list takes, types by types.
template <typename F>
void for_each_adamw_launch(const fira_adamw_desc* d, int count, void* const* W, const void* const* G, const fira_adamw_state* state, F f) {
  for (int kind = 0; kind < 8; ++kind) {
    const int in = kind & 1, grad = kind >> 1 & 1, eight = kind >> 2;
    auto of_kind = [&](const fira_adamw_desc& x) { return x.dtype == in && x.grad_dtype == grad && (x.state_type == FIRA_STATE_E4M3) == (eight != 0); };
    // All of a kind go through that kernel then.  A launch more for the others would cost about 1 us, which short lists save; long ones lose more: one such tensor beside 60m bf16 267 us and
    // without it 232, beside 62 m values bf16 with fp32 gradients in 8 bits 217 and 185.
    bool any = false;
    for (int i = 0; i < count; ++i) any = any || (of_kind(d[i]) && adamw_apart(d[i]) && d[i].cols % kMostWidth);
    with_types(in, grad, [&](auto t, auto r) {
      with_flag(eight, [&](auto e) {
        with_flag(any, [&](auto apart) {
          constexpr int64_t tile = 256 * kAdamUnroll<decltype(e)::value, decltype(apart)::value> * kAdamWidth<decltype(t), decltype(r), decltype(e)::value, decltype(apart)::value>;
          FiraAdamSpans l{};
          auto flush = [&] {
            if (l.count) f(t, r, e, apart, l);
            l.count = l.tiles = 0;
          };
          for (int i = 0; i < count; ++i) {
            if (!of_kind(d[i])) continue;
            cut_adamw(d[i], W[i], G[i], state[i], [&](FiraAdamSpan s) {
              s.tile0 = l.tiles;
              l.s[l.count++] = s;
              l.tiles += (int)((s.n + tile - 1) / tile);   // (2^30 values are 2^20 tiles at most)
              if (l.count == kAdamSpans) flush();
            });
          }
          flush();
        });
      });
    });
  }
}

// Whether the elements of a result are apart: strides in the order of their size, each at least what those before it span.  span: of all.
bool strides_apart(const int64_t (&size)[3], const int64_t (&stride)[3], int64_t dim, bool result, int64_t* span) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
  int64_t extent = dim, most = dim;
  for (int k : order) {
    int64_t far;
    if (size[k] <= 1) continue;
    if (result && stride[k] < extent) return false;
    if (stride[k] < 0 || __builtin_mul_overflow(stride[k], size[k] - 1, &far) || far > INT64_MAX / 16) return false;
    extent = far + extent;
    most += far;
  }
  *span = most;
  return true;
}

fira_status check_rotary(const fira_rotary_desc* d, const fira_rotary_heads* h, int count, const double* frequencies, const void* positions) {
  if (!d || !h) return refuse(FIRA_ERR_INVALID_ARG, "null descriptor");
  if (count < 1 || count > 4) return refuse(FIRA_ERR_INVALID_ARG, "%d tensors to turn", count);
  if (d->batch < 0 || d->length < 0 || d->batch > kMost || d->length > kMost || d->batch * d->length > kMost)
    return refuse(FIRA_ERR_SHAPE, "%lld sequences of %lld tokens", (long long)d->batch, (long long)d->length);
  if (d->dim < 1 || d->dim > 1 << 16 || d->rotated < 2 || d->rotated > d->dim || d->rotated % 2) return refuse(FIRA_ERR_SHAPE, "heads of %lld, %lld turned", (long long)d->dim, (long long)d->rotated);
  if (!known(d->dtype) || (d->position_type != FIRA_I32 && d->position_type != FIRA_I64)) return refuse(FIRA_ERR_DTYPE, "rotary types %d and %d", d->dtype, d->position_type);
  if (d->layout != FIRA_ROTARY_HALVES && d->layout != FIRA_ROTARY_INTERLEAVED) return refuse(FIRA_ERR_INVALID_ARG, "rotary layout %d", d->layout);
  if (!std::isfinite((float)d->scale)) return refuse(FIRA_ERR_INVALID_ARG, "scale is not finite");
  if (d->position_stride < 0 || d->position_stride > kMost) return refuse(FIRA_ERR_SHAPE, "position stride %lld", (long long)d->position_stride);
  if (!d->batch || !d->length) return FIRA_OK;
  for (int i = 0; i < count; ++i) {
    if (h[i].heads < 0 || h[i].heads > kMost) return refuse(FIRA_ERR_SHAPE, "%lld heads", (long long)h[i].heads);
    if (!h[i].heads) continue;
    const int64_t size[3] = {d->batch, d->length, h[i].heads};
    int64_t span;
    if (!strides_apart(size, h[i].x_stride, d->dim, false, &span)) return refuse(FIRA_ERR_SHAPE, "strides of tensor %d are negative or out of range", i);
    if (!strides_apart(size, h[i].y_stride, d->dim, true, &span)) return refuse(FIRA_ERR_SHAPE, "strides of result %d let elements overlap, or are out of range", i);
    if (!h[i].dev_x || !h[i].dev_y || !aligned(h[i].dev_x, size_of(d->dtype)) || !aligned(h[i].dev_y, size_of(d->dtype)))
      return refuse(FIRA_ERR_INVALID_ARG, "tensor or result %d is null or not aligned to its elements", i);
    if (h[i].dev_x == h[i].dev_y)
      for (int k = 0; k < 3; ++k)
        if (size[k] > 1 && h[i].x_stride[k] != h[i].y_stride[k]) return refuse(FIRA_ERR_INVALID_ARG, "tensor %d in place with other strides", i);
  }
  FIRA_POINTER(frequencies, 8);
  if (!aligned(positions, d->position_type == FIRA_I64 ? 8 : 4)) return refuse(FIRA_ERR_INVALID_ARG, "positions are not aligned to their elements");
  return FIRA_OK;
}

// How the kernel cuts its work up, in units of `pairs` or `width` values, at most `most` units a workgroup; whole: those of whole heads.
void cut_rotary(FiraRotary& r, int64_t heads, int pairs, int width, unsigned most, bool whole) {
  r.turned = (unsigned)(r.half + pairs - 1) / pairs;
  r.units = r.turned + (unsigned)(r.copied + width - 1) / width;
  r.all = (unsigned)heads * r.units;
  r.chunk = std::min(r.all, whole ? most / r.units * r.units : most);
  r.chunks = (r.all + r.chunk - 1) / r.chunk;
  r.tile = std::max(1u, std::min({most / r.chunk, kRotaryTile, kRotaryTable / (unsigned)r.half}));
  r.per_chunk = (unsigned)((((uint64_t)1 << 32) + r.chunk - 1) / r.chunk);
  r.per_units = (unsigned)((((uint64_t)1 << 32) + r.units - 1) / r.units);
}

fira_status rotary(const fira_rotary_desc* d, const fira_rotary_heads* h, int count, const double* frequencies, const void* positions, float sign, void* hip_stream) {
  if (const fira_status st = check_rotary(d, h, count, frequencies, positions)) return st;
  if (!d->batch || !d->length) return FIRA_OK;
  FiraRotary r{};
  r.tokens = (unsigned)(d->batch * d->length);
  r.length = (unsigned)d->length;
  r.position_stride = d->position_stride;
  r.half = (int)(d->rotated / 2);
  r.rotated = (int)d->rotated;
  r.scale = (float)d->scale;
  r.sign = sign;
  const bool interleaved = d->layout == FIRA_ROTARY_INTERLEAVED;
  r.wide = d->position_type == FIRA_I64;
  int64_t heads = 0, of[kRotaryTensors] = {};              // all tensors', which may be 2^31 and more, and each one's
  bool in_place = true;
  for (int i = 0; i < count; ++i) {
    if (!h[i].heads) continue;
    FiraRotaryTensor& t = r.t[r.count];
    t = {h[i].dev_x, h[i].dev_y, {}, {}};
    for (int k = 0; k < 3; ++k) { t.xs[k] = h[i].x_stride[k]; t.ys[k] = h[i].y_stride[k]; }
    of[r.count++] = h[i].heads;
    heads += h[i].heads;
    in_place = in_place && h[i].dev_x == h[i].dev_y;
  }
  if (!heads) return FIRA_OK;
  r.copied = in_place ? 0 : (int)(d->dim - d->rotated);
  const int64_t copied = r.copied, total = (int64_t)r.tokens * heads * (r.half + copied);
  const hipStream_t q = (hipStream_t)hip_stream;
  with_types(d->dtype, d->dtype, [&](auto t, auto) {
    typedef decltype(t) T;
    // (a head's units are below 2^15, and those of all heads below 2^21, so that their products stay in 32 bits)
    if ((unsigned)r.half > kRotaryTable || r.half + copied > 1 << 15 || heads * (r.half + copied) > 1 << 21) {
      for (int k = 0; k < r.count; ++k)
        hipLaunchKernelGGL(fira_rotary_wide_kernel<T>, dim3(std::min<int64_t>((r.tokens * of[k] * (r.half + copied) + 255) / 256, 1 << 20)), dim3(256), 0, q, r, k, (unsigned)of[k],
                           (unsigned)copied, interleaved, frequencies, positions);
      return;
    }
    for (int k = 1; k < r.count; ++k) r.first[k] = r.first[k - 1] + (int)of[k - 1];
    auto launch = [&](auto width, auto each, auto inter, bool whole) {
      constexpr int W = decltype(width)::value, N = decltype(each)::value;
      constexpr bool INTER = decltype(inter)::value;
      cut_rotary(r, heads, INTER && W > 1 ? W / 2 : W, W, 256 * N, whole);
      // (a launch has less than 2^32 threads)
      const int64_t step = (int64_t)((1 << 24) - 1) / r.chunks * r.tile;
      for (int64_t at = 0; at < r.tokens; at += step) {
        r.token0 = (unsigned)at;
        with_flag(!whole && (INTER || r.half * size_of(d->dtype) % 128 == 0), [&](auto stream) {
          hipLaunchKernelGGL((fira_rotary_kernel<T, W, N, INTER, decltype(stream)::value>), dim3((std::min<int64_t>(step, r.tokens - at) + r.tile - 1) / r.tile * r.chunks),
                             dim3(256), 0, q, r, frequencies, positions);
        });
      }
    };
    // Few units are spread over more workgroups.  us with one unit a thread and with four, in a graph, 40 heads of 128: bf16 512 tokens (0.3 of the limit) 4.3 and 5.9, 1024 7.1 and 6.5, 2048 12.0
    // and 8.4; fp32 512 tokens (0.6) 4.9 and 5.5, 1024 8.8 and 7.5.
    auto many = [&](auto width, bool whole) {
      with_flag(interleaved, [&](auto inter) {
        if (total / decltype(width)::value > 1 << 19) launch(width, Int<4>{}, inter, whole);
        else launch(width, Int<1>{}, inter, whole);
      });
    };
    constexpr int W = kWidth<T>;
    const int64_t turned = interleaved ? d->rotated : r.half;
    auto vectors = [&](int w) { return turned % w == 0 && copied % w == 0; };
    // (vectors may overlap where there are some and a workgroup takes a whole head)
    auto overlapping = [&](int w) { return turned >= w && (turned + w - 1) / w + (copied + w - 1) / w <= 256; };
    if (vectors(W)) many(Int<W>{}, false);
    else if (overlapping(W)) many(Int<W>{}, true);
    else if (vectors(4)) many(Int<4>{}, false);
    else if (overlapping(4)) many(Int<4>{}, true);
    else many(Int<1>{}, false);
  });
  return launched("rotary positions");
}

bool kind_known(int32_t k) { return k == FIRA_LAYER_NORM || k == FIRA_RMS_NORM || k == FIRA_NO_NORM; }
static_assert(FIRA_LAYER_NORM == (int)kLayer && FIRA_RMS_NORM == (int)kRms && FIRA_NO_NORM == (int)kNone, "kinds");

fira_status check_block(const fira_block_norm_desc* d, const fira_block_norm_params* p) {
  if (!d) return refuse(FIRA_ERR_INVALID_ARG, "null descriptor");
  if (d->rows < 0 || d->rows > kMost || d->dim < 1 || d->dim > kMostDim) return refuse(FIRA_ERR_SHAPE, "block norm of %lld rows of %lld", (long long)d->rows, (long long)d->dim);
  if (!known(d->dtype) || !known(d->param_dtype)) return refuse(FIRA_ERR_DTYPE, "block norm types %d and %d", d->dtype, d->param_dtype);
  if (!kind_known(d->norm) || !kind_known(d->post)) return refuse(FIRA_ERR_INVALID_ARG, "norm kinds %d and %d", d->norm, d->post);
  if (!(d->eps >= 0.0) || !std::isfinite((float)d->eps) || !(d->post_eps >= 0.0) || !std::isfinite((float)d->post_eps))
    return refuse(FIRA_ERR_INVALID_ARG, "an eps is negative or not finite");
  if (!std::isfinite((float)d->residual_scale) || !std::isfinite((float)d->block_scale)) return refuse(FIRA_ERR_INVALID_ARG, "a scale is not finite");
  if (p) {
    const size_t to = size_of(d->param_dtype);
    if (!aligned(p->gate, to) || !aligned(p->weight, to) || !aligned(p->bias, to) || !aligned(p->post_weight, to) || !aligned(p->post_bias, to))
      return refuse(FIRA_ERR_INVALID_ARG, "a vector is not aligned to its elements");
  }
  return FIRA_OK;
}

template <typename P>
FiraBlockVectors<P> block_vectors(const fira_block_norm_desc* d, const fira_block_norm_params* p) {
  FiraBlockVectors<P> v{};
  typedef const typename P::raw* at;
  if (!p) return v;
  v.gate = (at)p->gate;
  if (d->norm != FIRA_NO_NORM) { v.w = (at)p->weight; v.b = (at)p->bias; }
  if (d->post != FIRA_NO_NORM) { v.pw = (at)p->post_weight; v.pb = (at)p->post_bias; }
  return v;
}

// Calls f with the constants that a row is held by: values of a vector, threads, vectors of a thread.  FORWARD: up to kNormWidest values, 16 a thread where a row takes more
// than a wavefront; else up to kBlockWidest, 8 a thread and 16 from 4097 on.  Steps above 2048 are less than a factor of two, since lanes without a value cost most there
// (8192 x 4100 bf16 forward 70 us with powers of two, 57 with these).
template <typename T, bool FORWARD, typename F>
void with_block_shape(int64_t dim, F f) {
  constexpr int W = kWidth<T>, N = 8 / W, D = FORWARD ? 2 : 1;
  if (dim < kMostWidth) f(Int<1>{}, Int<8>{}, Int<1>{});
  else if (dim <= 8 * W) f(Int<W>{}, Int<8>{}, Int<1>{});
  else if (dim <= 16 * W) f(Int<W>{}, Int<16>{}, Int<1>{});
  else if (dim <= 32 * W) f(Int<W>{}, Int<32>{}, Int<1>{});
  else if (dim <= 64 * W) f(Int<W>{}, Int<64>{}, Int<1>{});
  else if (dim <= 512) f(Int<W>{}, Int<64>{}, Int<N>{});
  else if (dim <= 1024) f(Int<W>{}, Int<128 / D>{}, Int<D * N>{});
  else if (dim <= 2048) f(Int<W>{}, Int<256 / D>{}, Int<D * N>{});
  else if (dim <= 2560) f(Int<W>{}, Int<FORWARD ? 192 : 320 * N>{}, Int<FORWARD ? D * N : 1>{});   // (kBlockTwo with fp32)
  else if (!FORWARD && dim <= 3584) f(Int<W>{}, Int<448>{}, Int<N>{});
  else if (dim <= 4096) f(Int<W>{}, Int<512 / D>{}, Int<D * N>{});
  else if (dim <= 5120) f(Int<W>{}, Int<320>{}, Int<2 * N>{});
  else if (dim <= 6144) f(Int<W>{}, Int<384>{}, Int<2 * N>{});
  else if (dim <= 7168) f(Int<W>{}, Int<448>{}, Int<2 * N>{});
  else if (!FORWARD || dim <= 8192) f(Int<W>{}, Int<512>{}, Int<2 * N>{});
  else if constexpr (FORWARD) f(Int<W>{}, Int<1024>{}, Int<2 * N>{});
}
static_assert(kBlockWidest == 8192 && kNormWidest == 16384, "shapes");

// Workgroups of the gradient, each of which leaves its sums over rows; the workspace: the sums, then two means of every row where rows are read again.
// As many as the chip holds at a time or somewhat fewer, by what was measured, and fewer where that leaves each less than ten turns (of a row, or of the rows that it has side
// by side), with a quarter of that at least.  us with 1024 threads a compute unit, 1280 and 2048: 65536 x 2048 bf16 323, 354 and 327; with one workgroup a compute unit and two:
// 16385 x 2049 f32 165 and 147, with means and biases 203 and 175; 131072 x 256 bf16 with those (768 threads, 1024, 1536) 84, 94 and 94, 16385 x 2049 (two workgroups of 320 threads,
// three, four) 120, 142 and 182, x 2560 109, 133 and 152, and 32768 x 4096 with one workgroup a compute unit and two 372 and 294.
int64_t block_parts(const fira_block_norm_desc* d) {
  if (d->dim > kBlockWidest) return std::max<int64_t>(1, std::min<int64_t>(d->rows, 64));
  const bool lean = d->norm != FIRA_LAYER_NORM && d->post != FIRA_LAYER_NORM, f32 = d->dtype == FIRA_F32;
  int64_t threads = 0, side = 1;
  auto shape = [&](auto, auto t, auto) {
    threads = std::max(256, decltype(t)::value);
    side = std::max(1, 256 / decltype(t)::value);
  };
  f32 ? with_block_shape<FiraStoredF32, false>(d->dim, shape) : with_block_shape<FiraStoredBf16, false>(d->dim, shape);
  const int64_t held = d->dim > kBlockWidest / 2 ? 512 : f32 && d->dim > 256 ? (threads == kBlockTwo ? 2 * kBlockTwo : lean ? 1024 : 512) : lean || f32 ? 1024 : 768;
  const int64_t full = 256 * std::max<int64_t>(f32 || lean || d->dim > kBlockWidest / 2 ? 1 : 2, held / threads), turns = std::max<int64_t>(1, (d->rows + side - 1) / side);
  const int64_t each = std::min(std::max<int64_t>(10, (turns + full - 1) / full), (4 * turns + full - 1) / full);
  return (turns + each - 1) / each;
}
size_t block_sums_bytes(const fira_block_norm_desc* d) { return up256(4 * block_parts(d) * d->dim * 4); }

}  // namespace

extern "C" {

int64_t fira_adamw_scales(const fira_adamw_desc* d) {
  if (!d || check_adamw(d, 0) || d->state_type != FIRA_STATE_E4M3) return 0;
  return (d->rows * d->cols + kAdamBlock - 1) / kAdamBlock;
}

fira_status fira_adamw_step(const fira_adamw_desc* d, int count, const fira_adamw_hparams* hp, void* const* dev_W, const void* const* dev_G,
                            const fira_adamw_state* dev_state, int64_t* dev_t, const float* dev_lr, const float* dev_norm, void* hip_stream) {
  if (count < 0 || (count && (!d || !dev_W || !dev_G || !dev_state))) return refuse(FIRA_ERR_INVALID_ARG, "%d tensors, or a null list", count);
  if (const fira_status st = check_adamw_hparams(hp, dev_norm != nullptr)) return st;
  FIRA_POINTER(dev_t, 8);
  if (!aligned(dev_lr, 4) || !aligned(dev_norm, 4)) return refuse(FIRA_ERR_INVALID_ARG, "dev_lr or dev_norm is not aligned to its elements");
  for (int i = 0; i < count; ++i) {
    if (const fira_status st = check_adamw(d + i, i)) return st;
    if (!d[i].rows || !d[i].cols) continue;
    const fira_adamw_state& s = dev_state[i];
    const bool eight = d[i].state_type == FIRA_STATE_E4M3;
    if (!dev_W[i] || !dev_G[i] || !s.m || !s.v || (eight && (!s.m_scale || !s.v_scale))) return refuse(FIRA_ERR_INVALID_ARG, "tensor %d has a null pointer", i);
    if (!aligned(dev_W[i], size_of(d[i].dtype)) || !aligned(dev_G[i], size_of(d[i].grad_dtype)) ||
        (eight ? !aligned(s.m_scale, 4) || !aligned(s.v_scale, 4) : !aligned(s.m, 4) || !aligned(s.v, 4)))
      return refuse(FIRA_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
    if (dev_W[i] == dev_G[i] || s.m == s.v) return refuse(FIRA_ERR_INVALID_ARG, "tensor %d overlaps its gradient or its states each other", i);
  }
  const hipStream_t q = (hipStream_t)hip_stream;
  const FiraAdamHp h{hp->lr, std::log(hp->beta1), std::log(hp->beta2), hp->max_norm, (float)hp->beta1, (float)hp->beta2, (float)(1.0 - hp->beta1), (float)(1.0 - hp->beta2),
                     (float)hp->eps};
  int launches = 0, at = 0;
  bool counted = false;
  for_each_adamw_launch(d, count, dev_W, dev_G, dev_state, [&](auto, auto, auto, auto, FiraAdamSpans&) { ++launches; });
  for_each_adamw_launch(d, count, dev_W, dev_G, dev_state, [&](auto t, auto r, auto eight, auto apart, FiraAdamSpans& l) {
    const int workgroups = adam_workgroups<decltype(eight)::value, decltype(apart)::value>(l.tiles);
    l.counts = counted = ++at == launches && workgroups <= kAdamCounting;
    hipLaunchKernelGGL((fira_adamw_kernel<decltype(t), decltype(r), decltype(eight)::value, decltype(apart)::value>), dim3(workgroups), dim3(256), 0, q, l, h, dev_lr, dev_norm, (long long*)dev_t);
  });
  if (!counted) hipLaunchKernelGGL(fira_adamw_count_kernel<>, dim3(1), dim3(1), 0, q, (long long*)dev_t);
  return launched("AdamW step");
}

fira_status fira_rotary(const fira_rotary_desc* d, const fira_rotary_heads* h, int count, const double* dev_frequencies, const void* dev_positions, void* hip_stream) {
  return rotary(d, h, count, dev_frequencies, dev_positions, 1.0f, hip_stream);
}

fira_status fira_rotary_gradient(const fira_rotary_desc* d, const fira_rotary_heads* h, int count, const double* dev_frequencies, const void* dev_positions, void* hip_stream) {
  return rotary(d, h, count, dev_frequencies, dev_positions, -1.0f, hip_stream);
}

fira_status fira_rotary_frequencies(int64_t rotated, double base, int32_t context, double factor, double trained, double low, double high, double* host_frequencies,
                                    double* scale) {
  if (rotated < 2 || rotated > 1 << 16 || rotated % 2) return refuse(FIRA_ERR_SHAPE, "%lld values turned", (long long)rotated);
  if (!host_frequencies) return refuse(FIRA_ERR_INVALID_ARG, "host_frequencies is null");
  if (!(base > 0.0) || !std::isfinite(base)) return refuse(FIRA_ERR_INVALID_ARG, "base is not positive and finite");
  if (context < FIRA_ROTARY_PLAIN || context > FIRA_ROTARY_BY_PARTS) return refuse(FIRA_ERR_INVALID_ARG, "context %d", context);
  if (context != FIRA_ROTARY_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return refuse(FIRA_ERR_INVALID_ARG, "factor is below one or not finite");
  if (context == FIRA_ROTARY_BY_PARTS && !(trained > 0.0 && std::isfinite(trained) && low >= 0.0 && high > low && std::isfinite(high)))
    return refuse(FIRA_ERR_INVALID_ARG, "trained context, low or high out of range");
  for (int64_t j = 0; j < rotated / 2; ++j) {
    const double f = std::pow(base, -2.0 * (double)j / (double)rotated);
    double keep = context == FIRA_ROTARY_PLAIN ? 1.0 : 0.0;
    if (context == FIRA_ROTARY_BY_PARTS) keep = std::min(1.0, std::max(0.0, (trained * f / 6.283185307179586477 - low) / (high - low)));
    host_frequencies[j] = keep == 1.0 ? f : f * keep + f / factor * (1.0 - keep);
  }
  if (scale) *scale = context == FIRA_ROTARY_BY_PARTS ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return FIRA_OK;
}

fira_status fira_block_norm(const fira_block_norm_desc* d, const void* dev_x, int64_t ld_x, const void* dev_block, int64_t ld_block, const fira_block_norm_params* params,
                            void* dev_residual, int64_t ld_residual, void* dev_y, int64_t ld_y, float* dev_mean, float* dev_rstd, float* dev_post_mean, float* dev_post_rstd,
                            void* hip_stream) {
  if (const fira_status st = check_block(d, params)) return st;
  if (!d->rows) return FIRA_OK;
  const size_t size = size_of(d->dtype);
  FIRA_LEADING(ld_x, d->dim, d->rows);
  FIRA_LEADING(ld_block, d->dim, d->rows);
  FIRA_POINTER(dev_x, size);
  FIRA_POINTER(dev_block, size);
  if (dev_residual) {
    FIRA_LEADING(ld_residual, d->dim, d->rows);
    FIRA_POINTER(dev_residual, size);
  }
  if (d->norm == FIRA_NO_NORM && dev_y) return refuse(FIRA_ERR_INVALID_ARG, "y without a norm");
  if (d->norm != FIRA_NO_NORM) {
    FIRA_LEADING(ld_y, d->dim, d->rows);
    FIRA_POINTER(dev_y, size);
  }
  if ((dev_residual && (dev_residual == dev_x || dev_residual == dev_block || dev_residual == dev_y)) || (dev_y && (dev_y == dev_x || dev_y == dev_block)))
    return refuse(FIRA_ERR_INVALID_ARG, "a result is an input, or the other result");
  if (!aligned(dev_mean, 4) || !aligned(dev_rstd, 4) || !aligned(dev_post_mean, 4) || !aligned(dev_post_rstd, 4)) return refuse(FIRA_ERR_INVALID_ARG, "statistics are not aligned to their elements");
  const FiraBlockNorm n{d->rows, d->dim, ld_x, ld_block, ld_residual, ld_y, 0, 0, (float)d->eps, (float)d->post_eps, (float)d->block_scale, (float)d->residual_scale, d->norm, d->post};
  const FiraBlockStats to{dev_mean, dev_rstd, dev_post_mean, dev_post_rstd};
  with_types(d->dtype, d->param_dtype, [&](auto t, auto p) {
    typedef decltype(t) T;
    typedef decltype(p) P;
    typedef typename T::raw raw;
    const FiraBlockVectors<P> v = block_vectors<P>(d, params);
    const hipStream_t q = (hipStream_t)hip_stream;
    if (d->dim > kNormWidest) {
      hipLaunchKernelGGL((fira_block_norm_wide_kernel<T, P>), dim3(std::min<int64_t>(d->rows, 1 << 20)), dim3(1024), 0, q, n, (const raw*)dev_x, (const raw*)dev_block, v,
                         (raw*)dev_residual, (raw*)dev_y, to);
      return;
    }
    with_block_shape<T, true>(d->dim, [&](auto width, auto threads, auto nv) {
      constexpr int W = decltype(width)::value, THREADS = decltype(threads)::value, NV = decltype(nv)::value, GROUPS = std::max(1, 256 / THREADS);
      hipLaunchKernelGGL((fira_block_norm_kernel<T, P, W, THREADS, NV>), dim3(std::min<int64_t>((d->rows + GROUPS - 1) / GROUPS, 1 << 20)), dim3(GROUPS * THREADS), 0, q, n,
                         (const raw*)dev_x, (const raw*)dev_block, v, (raw*)dev_residual, (raw*)dev_y, to);
    });
  });
  return launched("block norm");
}

size_t fira_block_norm_gradient_workspace_bytes(const fira_block_norm_desc* d) {
  if (check_block(d, nullptr)) return 0;
  return std::max<size_t>(2 * FIRA_UNUSED_WORKSPACE_BYTES, block_sums_bytes(d) + (d->dim > kBlockWidest ? up256(8 * d->rows) : 0));
}

fira_status fira_block_norm_gradient(const fira_block_norm_desc* d, const void* dev_dresidual, int64_t ld_dresidual, const void* dev_dy, int64_t ld_dy, const void* dev_residual,
                                     int64_t ld_residual, const void* dev_block, int64_t ld_block, const fira_block_norm_params* params, const float* dev_mean, const float* dev_rstd,
                                     const float* dev_post_mean, const float* dev_post_rstd, void* dev_dx, int64_t ld_dx, void* dev_dblock, int64_t ld_dblock,
                                     const fira_block_norm_gradients* gradients, int accumulate, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  if (const fira_status st = check_block(d, params)) return st;
  const size_t size = size_of(d->dtype), psize = size_of(d->param_dtype);
  const fira_block_norm_gradients none{}, &g = gradients ? *gradients : none;
  if (!aligned(g.gate, psize) || !aligned(g.weight, psize) || !aligned(g.bias, psize) || !aligned(g.post_weight, psize) || !aligned(g.post_bias, psize))
    return refuse(FIRA_ERR_INVALID_ARG, "a vector's gradient is not aligned to its elements");
  if (d->norm == FIRA_NO_NORM && (g.weight || g.bias || dev_dy)) return refuse(FIRA_ERR_INVALID_ARG, "gradients of a norm that is not there");
  if (d->post == FIRA_NO_NORM && (g.post_weight || g.post_bias)) return refuse(FIRA_ERR_INVALID_ARG, "gradients of a post norm that is not there");
  // (the block's values: for the post norm's gradient, the gate's and the post weight's)
  const bool block = (d->post != FIRA_NO_NORM && dev_dblock) || g.gate || g.post_weight, sums = g.gate || g.weight || g.bias || g.post_weight || g.post_bias;
  if (d->rows) {
    if (dev_dresidual) {
      FIRA_LEADING(ld_dresidual, d->dim, d->rows);
      FIRA_POINTER(dev_dresidual, size);
    }
    if (d->norm != FIRA_NO_NORM) {
      FIRA_LEADING(ld_dy, d->dim, d->rows);
      FIRA_LEADING(ld_residual, d->dim, d->rows);
      FIRA_POINTER(dev_dy, size);
      FIRA_POINTER(dev_residual, size);
      FIRA_POINTER(dev_rstd, 4);
      if (d->norm == FIRA_LAYER_NORM) FIRA_POINTER(dev_mean, 4);
    }
    if (block) {
      FIRA_LEADING(ld_block, d->dim, d->rows);
      FIRA_POINTER(dev_block, size);
    }
    if (d->post != FIRA_NO_NORM) {
      FIRA_POINTER(dev_post_rstd, 4);
      if (d->post == FIRA_LAYER_NORM) FIRA_POINTER(dev_post_mean, 4);
    }
    if (dev_dx) {
      FIRA_LEADING(ld_dx, d->dim, d->rows);
      FIRA_POINTER(dev_dx, size);
    }
    if (dev_dblock) {
      FIRA_LEADING(ld_dblock, d->dim, d->rows);
      FIRA_POINTER(dev_dblock, size);
    }
    if (dev_dx && dev_dx == dev_dblock) return refuse(FIRA_ERR_INVALID_ARG, "one buffer for two results");
    for (const void* in : {dev_dresidual, dev_dy, dev_residual, dev_block})
      if (in && (in == dev_dx || in == dev_dblock)) return refuse(FIRA_ERR_INVALID_ARG, "a result is an input");
  }
  if (const fira_status st = check_workspace(dev_workspace, workspace_bytes, fira_block_norm_gradient_workspace_bytes(d))) return st;
  if ((!sums && (!d->rows || (!dev_dx && !dev_dblock))) || (!d->rows && accumulate)) return FIRA_OK;
  const FiraBlockNorm n{d->rows, d->dim, ld_dresidual, ld_block, ld_residual, ld_dy, ld_dx, ld_dblock, (float)d->eps, (float)d->post_eps, (float)d->block_scale, (float)d->residual_scale,
                        d->norm, d->post};
  const FiraBlockStats stats{(float*)dev_mean, (float*)dev_rstd, (float*)dev_post_mean, (float*)dev_post_rstd};   // (read only)
  with_types(d->dtype, d->param_dtype, [&](auto t, auto p) {
    typedef decltype(t) T;
    typedef decltype(p) P;
    typedef typename T::raw raw;
    typedef typename P::raw praw;
    const FiraBlockVectors<P> v = block_vectors<P>(d, params);
    const FiraBlockGradients<P> to{(praw*)g.gate, (praw*)g.weight, (praw*)g.bias, (praw*)g.post_weight, (praw*)g.post_bias};
    const raw *const dr = (const raw*)dev_dresidual, *const dy = (const raw*)dev_dy, *const r = (const raw*)dev_residual, *const b = block ? (const raw*)dev_block : nullptr;
    const hipStream_t q = (hipStream_t)hip_stream;
    const int parts = (int)block_parts(d);
    float* const partial = (float*)dev_workspace;
    float* const means = (float*)((char*)dev_workspace + block_sums_bytes(d));
    // (which of the sums of dy h, dy, t h' and t are wanted)
    const int wanted = (g.weight ? 1 : 0) | (g.bias ? 2 : 0) | (g.gate || g.post_weight ? 4 : 0) | ((g.gate && v.pb) || g.post_bias ? 8 : 0);
    if (!d->rows) {                                        // (nothing to add up)
    } else if (d->dim > kBlockWidest) {
      hipLaunchKernelGGL((fira_block_norm_wide_rows_kernel<T, P>), dim3(std::min<int64_t>(d->rows, 1 << 20)), dim3(1024), 0, q, n, dr, dy, r, b, v, stats, (raw*)dev_dx, (raw*)dev_dblock, means);
      if (sums) hipLaunchKernelGGL((fira_block_norm_wide_sums_kernel<T, P>), dim3((d->dim + 255) / 256, parts), dim3(256), 0, q, n, dr, dy, r, b, v, stats, (const float*)means, partial);
    } else {
      auto launch = [&](auto width, auto threads, auto nv) {
        constexpr int W = decltype(width)::value, THREADS = decltype(threads)::value, NV = decltype(nv)::value;
        with_flag(d->norm != FIRA_LAYER_NORM && d->post != FIRA_LAYER_NORM && !(wanted & 10), [&](auto lean) {
          hipLaunchKernelGGL((fira_block_norm_gradient_kernel<T, P, W, THREADS, NV, decltype(lean)::value>), dim3(parts), dim3(std::max(256, THREADS)), 0, q, n, dr, dy, r, b, v, stats,
                             (raw*)dev_dx, (raw*)dev_dblock, partial, wanted);
        });
      };
      with_block_shape<T, false>(d->dim, launch);
    }
    if (sums) hipLaunchKernelGGL(fira_block_norm_join_kernel<P>, dim3((d->dim + 15) / 16), dim3(256), 0, q, n, (const float*)partial, d->rows ? parts : 0, wanted, v, to, accumulate);
  });
  return launched("block norm gradient");
}

}  // extern "C"
