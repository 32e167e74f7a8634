// Host-only check of the operators around the step: their host code (csrc/fira_training.hip) over a stand-in for the HIP runtime (host_hip.h), which
// hands every launch to this program.  The pieces that a list of gradients is cut into cover every value once, whatever the sizes (to beyond 32
// bits), and fit the kernels' counts; the workspaces' parts are disjoint and inside; no grid has more threads than a launch may have.
// Built and run on the CPU by tests/test_host_training.py.
#include "../paper_2410_01623_amd/csrc/fira_training.hip"

#include <cstring>
#include <random>
#include <string>
#include <vector>

// (the stand-in leaves launch shapes out: kept here, as launches are made of a shape pushed and popped)
#define __hipPushCallConfiguration stand_in_push
#define __hipPopCallConfiguration stand_in_pop
#include "host_hip.h"
#undef __hipPushCallConfiguration
#undef __hipPopCallConfiguration
namespace {
dim3 pushed_grid, pushed_block;
size_t pushed_lds;
}
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t) {
  pushed_grid = grid;
  pushed_block = block;
  pushed_lds = lds;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* q) {
  *grid = pushed_grid;
  *block = pushed_block;
  *lds = pushed_lds;
  *q = nullptr;
  return hipSuccess;
}

namespace {
std::string message;
}
fira_status fira_fail_without_context(fira_status st, const char* msg) noexcept {
  message = msg;
  return st;
}

namespace {

struct Piece { const char* g; char* out; int64_t rows, cols, ld, ld_out; int dtype, out_dtype; };
std::vector<Piece> scaled, squared;
int64_t most_threads = 0;

template <typename K>
bool is(const void* f, K kernel) { return f == (const void*)kernel; }

void take(std::vector<Piece>& to, const FiraSpans& l, dim3 grid, int in, int out, int width) {
  CHECK(l.count >= 1 && l.count <= kSpans && l.each >= 1);
  CHECK((int)grid.x <= kClipWorkgroups && (int64_t)grid.x * l.each >= l.tiles && (int64_t)(grid.x - 1) * l.each < l.tiles);
  int64_t tiles = 0;
  for (int i = 0; i < l.count; ++i) {
    const FiraSpan& s = l.s[i];
    CHECK(s.tile0 == tiles && s.rows >= 1 && s.cols >= 1);
    CHECK(s.vecs == (s.cols < width ? s.cols : (s.cols + width - 1) / width));
    const int64_t vecs = (int64_t)s.rows * s.vecs;
    CHECK(vecs < (int64_t)1 << 31);
    tiles += (vecs + kClipTile - 1) / kClipTile;
    to.push_back(Piece{(const char*)s.g, (char*)s.out, s.rows, s.cols, s.ld, s.ld_out, in, out});
  }
  CHECK(tiles == l.tiles && tiles < (int64_t)1 << 31);
}

void launched(const void* f, dim3 grid, void** args) {
  most_threads = std::max<int64_t>(most_threads, (int64_t)grid.x * grid.y * grid.z * pushed_block.x);
  const FiraSpans& l = *(const FiraSpans*)args[0];
  if (is(f, fira_gradient_squares_kernel<FiraStoredF32>)) take(squared, l, grid, FIRA_F32, FIRA_F32, 4);
  else if (is(f, fira_gradient_squares_kernel<FiraStoredBf16>)) take(squared, l, grid, FIRA_BF16, FIRA_BF16, 8);
  else if (is(f, fira_clip_kernel<FiraStoredF32, FiraStoredF32>)) take(scaled, l, grid, FIRA_F32, FIRA_F32, 4);
  else if (is(f, fira_clip_kernel<FiraStoredF32, FiraStoredBf16>)) take(scaled, l, grid, FIRA_F32, FIRA_BF16, 4);
  else if (is(f, fira_clip_kernel<FiraStoredBf16, FiraStoredF32>)) take(scaled, l, grid, FIRA_BF16, FIRA_F32, 4);
  else if (is(f, fira_clip_kernel<FiraStoredBf16, FiraStoredBf16>)) take(scaled, l, grid, FIRA_BF16, FIRA_BF16, 8);
}

// The pieces of one gradient at g (values of `size` bytes) put together again: whole rows of pieces, or parts of rows.
void covers(const std::vector<Piece>& pieces, const fira_gradient_desc& d, const char* g, const char* out, bool outs) {
  const int64_t size = d.dtype == FIRA_F32 ? 4 : 2, size_out = (outs ? d.out_dtype : d.dtype) == FIRA_F32 ? 4 : 2;
  const int64_t ld_out = outs ? d.ld_out : d.ld;
  const bool dense = (d.ld == d.cols || d.rows <= 1) && (!outs || d.ld_out == d.cols || d.rows <= 1);
  int64_t at = 0, values = 0;                          // next value in order
  for (const Piece& p : pieces) {
    const int64_t offset = (p.g - g) / size;
    const int64_t row = dense ? 0 : offset / d.ld, col = offset - row * (dense ? 0 : d.ld);
    CHECK((p.g - g) % size == 0 && col >= 0 && col + p.cols <= (dense ? d.rows * d.cols : d.cols));
    CHECK(at == row * d.cols + col);
    if (p.out) CHECK((p.out - out) == (row * ld_out + col) * size_out);
    if (p.rows > 1) CHECK(p.cols == d.cols && p.ld == d.ld && (!p.out || p.ld_out == ld_out));
    at += p.rows * p.cols;
    values += p.rows * p.cols;
  }
  CHECK(values == d.rows * d.cols);
}

void check_gradients() {
  std::mt19937_64 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
  const int64_t sizes[] = {0, 1, 2, 7, 8, 9, 100, 1376, 4099, 70001, (1ll << 30) - 1, 1ll << 30, (1ll << 30) + 5, (1ll << 31) + 9, 5ll << 30};
  for (int round = 0; round < 400; ++round) {
    const int n = (int)pick(0, round % 10 == 0 ? 300 : 12);
    std::vector<fira_gradient_desc> d(n);
    std::vector<const void*> G(n);
    std::vector<void*> out(n), in_place(n);
    char* next = (char*)(1ll << 20);
    for (int i = 0; i < n; ++i) {
      const bool large = pick(0, 15) == 0;
      int64_t rows = large ? pick(1, 3) : sizes[pick(0, 9)], cols = sizes[pick(0, large ? 14 : 9)];
      const int64_t pads[] = {0, 0, 3, 8, large ? 1ll << 31 : 64};
      d[i] = fira_gradient_desc{rows, cols, cols + pads[pick(0, 4)], (int32_t)pick(0, 1), (int32_t)pick(0, 1), cols + pads[pick(0, 4)]};
      // (a list of one kind at a time is put together again in order; kinds are launched one after the other)
      G[i] = next;
      in_place[i] = next;
      next += ((rows + 1) * d[i].ld + 64) * 4;
      out[i] = next;
      next += ((rows + 1) * d[i].ld_out + 64) * 4;
    }
    const size_t bytes = fira_gradient_workspace_bytes(d.data(), n);
    CHECK(bytes >= 8);
    void* const ws = (void*)4096;
    for (int outs = 0; outs < 2; ++outs) {
      scaled.clear();
      squared.clear();
      CHECK(fira_clip_gradients(d.data(), n, in_place.data(), outs ? out.data() : nullptr, 1.0, (float*)4096, ws, bytes, nullptr) == FIRA_OK);
      for (int i = 0; i < n; ++i) {
        const char* const g = (const char*)G[i];
        const char* const end = g + ((d[i].rows + 1) * d[i].ld + 64) * 4;
        std::vector<Piece> a, b;
        for (const Piece& p : squared) if (p.g >= g && p.g < end) { a.push_back(p); a.back().out = nullptr; CHECK(p.dtype == d[i].dtype); }
        for (const Piece& p : scaled) if (p.g >= g && p.g < end) { b.push_back(p); CHECK(p.dtype == d[i].dtype && p.out_dtype == (outs ? d[i].out_dtype : d[i].dtype)); }
        covers(a, d[i], g, nullptr, false);
        covers(b, d[i], g, outs ? (char*)out[i] : g, outs);
      }
      CHECK((int64_t)bytes >= 8 * partials(d.data(), n));
    }
  }
}

void check_workspaces() {
  std::mt19937_64 rng(11);
  for (int round = 0; round < 3000; ++round) {
    const double u = (double)(rng() % 1000) / 1000, v = (double)(rng() % 1000) / 1000, w = (double)(rng() % 1000) / 1000;
    const int64_t rows = 1 + (int64_t)(std::exp2(21 * u)) - 1, dim = (int64_t)std::exp2((round % 8 ? 14 : 24) * v), count = (int64_t)std::exp2(31 * w) - 1;
    const fira_embed_desc d{rows, dim, dim, (int32_t)(rng() & 1), (int32_t)(rng() & 1), (int32_t)(rng() & 1), 1.0};
    const size_t bytes = fira_embed_gradient_workspace_bytes(&d, count);
    CHECK(bytes >= 256 && bytes % 256 == 0);
    char* const at = (char*)(1ll << 20);
    const EmbedSort r = embed_sort(&d, count, at);
    CHECK(r.bytes == bytes);
    if (count > kFewTokens) {
      const FiraEmbedSort& s = r.s;
      CHECK(s.chunks >= 1 && s.chunks <= kMostChunks && (int64_t)s.chunks * s.chunk >= count && s.chunk % 256 == 0);
      CHECK((int64_t)s.bins * kBuckets >= rows && s.bins <= kCounters && (1 << s.bits) >= s.bins);
      const std::pair<char*, int64_t> parts[] = {{(char*)s.sorted, 8ll * s.chunks * s.chunk}, {(char*)s.gathered, 8 * count}, {(char*)s.part, 8ll * kBuckets * s.chunks},
                                                 {(char*)s.order, 4 * count}, {(char*)s.rows, 8ll * kBuckets * s.bins}, {(char*)s.counters, 8}, {(char*)s.pieces, 16 * r.pieces},
                                                 {(char*)s.cut, 16 * r.pieces}, {(char*)s.partial, 4 * r.pieces * dim}};
      char* end = at;
      for (const auto& p : parts) {
        CHECK(p.first >= end && ((uintptr_t)p.first & 255) == 0);
        end = p.first + p.second;
      }
      CHECK(end <= at + bytes);
      // rows of more than kPieceTokens tokens, in pieces of kPieceTokens: no more than there is room for, in the worst case
      CHECK(count / (kPieceTokens + 1) * 2 <= r.pieces);
    }
    const fira_layer_norm_desc n{count, dim, (int32_t)(rng() & 1), (int32_t)(rng() & 1), (int32_t)(rng() & 1), 1e-5};
    CHECK(fira_layer_norm_gradient_workspace_bytes(&n) >= (count <= kFewRows && dim <= kNormWidest ? (size_t)256 : 2 * (size_t)norm_parts(&n) * dim * 4));
    void* const p = (void*)(1ll << 20);
    CHECK(fira_embed_lookup(&d, p, p, count, p, dim, nullptr) == FIRA_OK);
    CHECK(fira_embed_gradient(&d, p, dim, p, count, p, round & 1, p, bytes, nullptr) == FIRA_OK);
    CHECK(fira_layer_norm(&n, p, dim, p, p, p, dim, (float*)p, (float*)p, nullptr) == FIRA_OK);
    CHECK(fira_layer_norm_gradient(&n, p, dim, p, dim, p, (const float*)p, (const float*)p, p, dim, p, p, round & 1, p, fira_layer_norm_gradient_workspace_bytes(&n), nullptr) == FIRA_OK);
  }
  CHECK(most_threads < (int64_t)1 << 32);
}

}  // namespace

int main() {
  on_launch = launched;
  check_gradients();
  on_launch = [](const void*, dim3 grid, void**) { most_threads = std::max<int64_t>(most_threads, (int64_t)grid.x * grid.y * grid.z * pushed_block.x); };
  check_workspaces();
  // a launch that fails is reported
  launches_fail = true;
  const fira_gradient_desc d{2, 3, 3, 0, 0, 3};
  void* const g[1] = {(void*)4096};
  CHECK(fira_clip_gradients(&d, 1, g, nullptr, 1.0, (float*)4096, (void*)4096, 4096, nullptr) == FIRA_ERR_HIP && message.find("clipping") != std::string::npos);
  std::printf("%d failure(s)\n", failures);
  return failures != 0;
}
