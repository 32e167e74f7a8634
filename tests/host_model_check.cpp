// Host-only check of AdamW, rotary positions and the block norm: their host code (csrc/fira_model.hip) over a stand-in for the HIP runtime (host_hip.h), which hands every launch
// to this program.  The pieces that a list of tensors is cut into cover every value once, from whole blocks on, to beyond 32 bits; the step is counted once; a workgroup's
// units of heads, in the kernel's own index arithmetic, cover every value of every head once and stay inside its tables; the gradient's sums fit the
// workspace; no grid has more threads than a launch may have.  Built and run on the CPU by tests/test_host_model.py.
#include "../paper_2410_01623_amd/csrc/fira_model.hip"

#include <cstring>
#include <functional>
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
}
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  pushed_grid = grid;
  pushed_block = block;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* q) {
  *grid = pushed_grid;
  *block = pushed_block;
  *lds = 0;
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

int64_t most_threads = 0;
std::function<void(const void*, dim3, void**)> look;
void launched_here(const void* f, dim3 grid, void** args) {
  most_threads = std::max<int64_t>(most_threads, (int64_t)grid.x * grid.y * grid.z * pushed_block.x);
  CHECK(grid.x >= 1 && pushed_block.x >= 1 && pushed_block.x <= 1024);
  if (look) look(f, grid, args);
}

std::mt19937_64 rng(7);
int64_t pick(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); }

// ---- AdamW: a list whose tensors lie apart in an imagined memory -------------------------------------------------------

struct Seen { FiraAdamSpan s; int dtype, grad, eight; };

template <typename T, typename R, bool EIGHT, bool APART>
bool adamw_launch_of(const void* f, dim3 grid, void** args, std::vector<Seen>& seen, int& counts, int dtype, int grad) {
  if (f != (const void*)fira_adamw_kernel<T, R, EIGHT, APART>) return false;
  const FiraAdamSpans& l = *(const FiraAdamSpans*)args[0];
  constexpr int64_t tile = 256 * kAdamUnroll<EIGHT, APART> * kAdamWidth<T, R, EIGHT, APART>;
  CHECK(l.count >= 1 && l.count <= kAdamSpans && ((int)grid.x == adam_workgroups<EIGHT, APART>(l.tiles)) && (int)grid.x <= l.tiles && (int64_t)grid.x * 256 < (int64_t)1 << 32 && pushed_block.x == 256);
  int64_t tiles = 0;
  for (int i = 0; i < l.count; ++i) {
    CHECK(APART || l.s[i].cols % kMostWidth == 0);
    CHECK(l.s[i].tile0 == tiles && l.s[i].n >= 1 && (int64_t)l.s[i].n <= kAdamPiece);
    // (a thread's place in a piece, and in the columns, beyond its last vector)
    CHECK((int64_t)l.s[i].n + tile < (int64_t)1 << 32 && (int64_t)l.s[i].col0 + l.s[i].n + tile < (int64_t)1 << 32);
    tiles += (l.s[i].n + tile - 1) / tile;
    seen.push_back({l.s[i], dtype, grad, EIGHT});
  }
  CHECK(tiles == l.tiles);
  CHECK(!l.counts || (int)grid.x <= kAdamCounting);
  counts += l.counts != 0;
  return true;
}

template <typename T, typename R, bool EIGHT>
bool adamw_launch(const void* f, dim3 grid, void** args, std::vector<Seen>& seen, int& counts, int dtype, int grad) {
  return adamw_launch_of<T, R, EIGHT, false>(f, grid, args, seen, counts, dtype, grad) || adamw_launch_of<T, R, EIGHT, true>(f, grid, args, seen, counts, dtype, grad);
}

void check_adamw_lists() {
  typedef FiraStoredF32 F;
  typedef FiraStoredBf16 B;
  const int64_t sizes[] = {0, 1, 2, 7, 8, 255, 256, 257, 1376, 70001, (1ll << 30) - 1, 1ll << 30, (1ll << 30) + 5, (1ll << 31) - 1, 5ll << 30};
  for (int round = 0; round < 300; ++round) {
    const int n = (int)pick(0, round % 10 == 0 ? 200 : 10);
    std::vector<fira_adamw_desc> d(n);
    std::vector<void*> W(n);
    std::vector<const void*> G(n);
    std::vector<fira_adamw_state> S(n);
    char* next = (char*)(1ll << 20);
    auto room = [&](int64_t bytes) { char* const p = next; next += (bytes + 4096) / 256 * 256; return p; };
    for (int i = 0; i < n; ++i) {
      const bool large = pick(0, 15) == 0;
      const int64_t rows = large ? pick(1, 3) : sizes[pick(0, 9)], cols = sizes[pick(0, large ? 14 : 9)];
      const bool apart = cols < (1ll << 31) && pick(0, 1);
      d[i] = fira_adamw_desc{rows, cols, cols + (apart ? pick(0, 9) : 0), cols + (apart ? pick(0, 9) : 0), (int32_t)pick(0, 1), (int32_t)pick(0, 1), (int32_t)pick(0, 1), (uint32_t)rng(), 0.1};
      W[i] = room((rows + 1) * d[i].ld_w * 4) + (d[i].dtype ? 2 : 4) * pick(0, 1);
      G[i] = room((rows + 1) * d[i].ld_g * 4);
      S[i] = fira_adamw_state{room(rows * cols * 4), room(rows * cols * 4), (float*)room(rows * cols / 64 + 4), (float*)room(rows * cols / 64 + 4)};
      CHECK(fira_adamw_scales(&d[i]) == (d[i].state_type ? (rows * cols + 255) / 256 : 0));
    }
    std::vector<Seen> seen;
    int counts = 0, counted_apart = 0, others = 0;
    look = [&](const void* f, dim3 grid, void** args) {
      if (f == (const void*)fira_adamw_count_kernel<>) { ++counted_apart; return; }
      const bool known = adamw_launch<F, F, false>(f, grid, args, seen, counts, 0, 0) || adamw_launch<F, B, false>(f, grid, args, seen, counts, 0, 1) ||
                         adamw_launch<B, F, false>(f, grid, args, seen, counts, 1, 0) || adamw_launch<B, B, false>(f, grid, args, seen, counts, 1, 1) ||
                         adamw_launch<F, F, true>(f, grid, args, seen, counts, 0, 0) || adamw_launch<F, B, true>(f, grid, args, seen, counts, 0, 1) ||
                         adamw_launch<B, F, true>(f, grid, args, seen, counts, 1, 0) || adamw_launch<B, B, true>(f, grid, args, seen, counts, 1, 1);
      others += !known;
    };
    const fira_adamw_hparams hp{1e-3, 0.9, 0.999, 1e-8, 1.0};
    CHECK(fira_adamw_step(d.data(), n, &hp, W.data(), G.data(), S.data(), (int64_t*)4096, nullptr, nullptr, nullptr) == FIRA_OK);
    CHECK(others == 0 && counts + counted_apart == 1);
    size_t used = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t all = d[i].rows * d[i].cols, size = d[i].dtype ? 2 : 4, gsize = d[i].grad_dtype ? 2 : 4, state = d[i].state_type ? 1 : 4;
      const bool dense = d[i].rows <= 1 || (d[i].ld_w == d[i].cols && d[i].ld_g == d[i].cols);
      int64_t at = 0;
      for (const Seen& x : seen) {
        if ((char*)x.s.m < (char*)S[i].m || (char*)x.s.m >= (char*)S[i].m + std::max<int64_t>(1, all * state)) continue;
        ++used;
        const FiraAdamSpan& s = x.s;
        CHECK(x.dtype == d[i].dtype && x.grad == d[i].grad_dtype && x.eight == d[i].state_type && at % 256 == 0);
        CHECK((char*)s.m == (char*)S[i].m + at * state && (char*)s.v == (char*)S[i].v + at * state && s.first == (unsigned)at && s.seed == d[i].seed);
        if (d[i].state_type) CHECK(s.m_scale == S[i].m_scale + at / 256 && s.v_scale == S[i].v_scale + at / 256);
        CHECK((s.cols == 0) == dense);
        if (dense) CHECK((char*)s.w == (char*)W[i] + at * size && (const char*)s.g == (const char*)G[i] + at * gsize);
        else {
          CHECK(s.cols == d[i].cols && s.col0 == at % d[i].cols && (char*)s.w == (char*)W[i] + at / d[i].cols * d[i].ld_w * size && (const char*)s.g == (const char*)G[i] + at / d[i].cols * d[i].ld_g * gsize);
          // the quotient in fp64, at the ends of rows and of the piece
          for (int k = 0; k < 200; ++k) {
            unsigned c = s.col0 + (unsigned)pick(0, (int64_t)s.n - 1);
            if (k & 1) c = std::min<unsigned>(c / s.cols * s.cols + (k & 2 ? s.cols - 1 : 0), s.col0 + s.n - 1);
            CHECK((unsigned)(((double)c + 0.5) * s.per_col) == c / s.cols);
          }
        }
        if (s.stream & 1) CHECK((uintptr_t)s.w % 128 == 0);
        if (s.stream & 2) CHECK((uintptr_t)s.m % 128 == 0 && (uintptr_t)s.v % 128 == 0);
        at += s.n;
      }
      CHECK(at == all);
    }
    CHECK(used == seen.size());
  }
}

// ---- rotary: the kernel's index arithmetic, over counters of what is touched -----------------------------------------------

unsigned quotient(unsigned x, unsigned d, unsigned per_d) { return d == 1 ? x : (unsigned)((uint64_t)x * per_d >> 32); }

// Turns one launch's arguments into counts: touched[tensor][token][head][value].
void count_rotary(const FiraRotary& r, dim3 grid, int W, int N, bool inter, int64_t dim, std::vector<std::vector<int>>& touched, std::vector<std::vector<int>>& owner, const std::vector<int64_t>& heads) {
  const bool two = !inter || W == 1;
  CHECK(r.tile >= 1 && r.tile <= kRotaryTile && (int64_t)r.tile * r.half <= kRotaryTable);
  CHECK((int64_t)r.tile * r.chunk <= 256 * N && r.chunk >= 1 && (int64_t)r.chunks * r.chunk >= r.all);
  for (unsigned b = 0; b < grid.x; ++b) {
    const unsigned t0 = r.token0 + b / r.chunks * r.tile, c0 = b % r.chunks * r.chunk;
    CHECK(t0 < r.tokens);
    const unsigned tokens = std::min(r.tile, r.tokens - t0), here = std::min(r.chunk, r.all - c0), head0 = c0 / r.units, unit0 = c0 - head0 * r.units;
    for (unsigned i = 0; i < 256u * N; ++i) {
      const unsigned t = quotient(i, r.chunk, r.per_chunk), c = i - t * r.chunk;
      CHECK(t == i / r.chunk);
      if (!(t < tokens && c < here)) continue;
      const unsigned head = quotient(unit0 + c, r.units, r.per_units);
      CHECK(head == (unit0 + c) / r.units);
      unsigned h = head0 + head, k = 0;
      const unsigned unit = unit0 + c - head * r.units;
      for (int j = 1; j < r.count; ++j)
        if (h >= (unsigned)r.first[j]) k = j;
      h -= r.first[k];
      CHECK(h < heads[k]);
      auto touch = [&](int64_t at, int n) {
        CHECK(at >= 0 && at + n <= dim);
        for (int v = 0; v < n; ++v) {
          const int64_t place = ((int64_t)(t0 + t) * heads[k] + h) * dim + at + v;
          ++touched[k][place];
          // (what is turned twice is turned by one workgroup)
          CHECK(!owner[k][place] || owner[k][place] == (int)b + 1);
          owner[k][place] = (int)b + 1;
        }
      };
      if (unit < r.turned) {
        const unsigned at = W == 8 ? (inter ? rotary_place<8, true>(r, unit) : rotary_place<8, false>(r, unit)) : W == 4 ? (inter ? rotary_place<4, true>(r, unit) : rotary_place<4, false>(r, unit)) :
                            (inter ? rotary_place<1, true>(r, unit) : rotary_place<1, false>(r, unit));
        CHECK((int64_t)t * r.half + at / (inter ? 2 : 1) + (two ? W : W / 2) <= kRotaryTable && at / (inter ? 2 : 1) + (two ? W : W / 2) <= (unsigned)r.half);
        touch(at, W);
        if (two) touch(at + (inter ? 1 : r.half), W);
      } else {
        const int64_t at = r.rotated + std::min<int64_t>((int64_t)(unit - r.turned) * W, r.copied - W), skip = std::max(0, W - r.copied);
        CHECK(at >= 0);
        touch(at + skip, W - skip);
      }
    }
  }
}

template <typename T, int W, int N>
bool rotary_launch(const void* f, int& w, int& n, bool& inter) {
  const bool a = f == (const void*)fira_rotary_kernel<T, W, N, false, false> || f == (const void*)fira_rotary_kernel<T, W, N, false, true>, b = f == (const void*)fira_rotary_kernel<T, W, N, true, false> || f == (const void*)fira_rotary_kernel<T, W, N, true, true>;
  if (!a && !b) return false;
  w = W;
  n = N;
  inter = b;
  return true;
}

void check_rotary_units() {
  typedef FiraStoredF32 F;
  typedef FiraStoredBf16 B;
  for (int round = 0; round < 1200; ++round) {
    const bool big = round % 40 == 0;
    const int64_t dim = pick(0, 3) ? pick(2, big ? 5000 : 300) : (int64_t[]){64, 128, 96, 256}[pick(0, 3)], rotated = pick(0, 1) ? dim / 2 * 2 : 2 * pick(1, dim / 2);
    const int64_t batch = pick(1, 3), length = big ? pick(1, 2) : pick(1, 60);
    const int count = (int)pick(1, 4);
    fira_rotary_desc d{batch, length, dim, rotated, (int32_t)pick(0, 1), (int32_t)pick(0, 1), (int32_t)pick(0, 1), length, 1.0};
    fira_rotary_heads h[4];
    std::vector<int64_t> heads;
    std::vector<std::vector<int>> touched, owner;
    const bool in_place = pick(0, 3) == 0;
    for (int i = 0; i < count; ++i) {
      const int64_t n = pick(0, 9) ? pick(1, big ? 40 : 12) : 0;
      h[i] = fira_rotary_heads{(void*)(1ll << (30 + i)), (void*)((1ll << (30 + i)) + (in_place ? 0 : 1ll << 29)), n, {length * n * dim, n * dim, dim}, {length * n * dim, n * dim, dim}};
      if (!n) continue;
      heads.push_back(n);
      touched.emplace_back((size_t)(batch * length * n * dim));
      owner.emplace_back((size_t)(batch * length * n * dim));
    }
    int wide = 0;
    look = [&](const void* f, dim3 grid, void** args) {
      int w = 0, n = 0;
      bool inter = false;
      const FiraRotary& r = *(const FiraRotary*)args[0];
      if (rotary_launch<F, 4, 4>(f, w, n, inter) || rotary_launch<F, 4, 1>(f, w, n, inter) || rotary_launch<F, 1, 4>(f, w, n, inter) || rotary_launch<F, 1, 1>(f, w, n, inter) ||
          rotary_launch<B, 8, 4>(f, w, n, inter) || rotary_launch<B, 8, 1>(f, w, n, inter) || rotary_launch<B, 4, 4>(f, w, n, inter) || rotary_launch<B, 4, 1>(f, w, n, inter) ||
          rotary_launch<B, 1, 4>(f, w, n, inter) || rotary_launch<B, 1, 1>(f, w, n, inter)) {
        CHECK(inter == (d.layout == FIRA_ROTARY_INTERLEAVED) && r.count == (int)heads.size());
        count_rotary(r, grid, w, n, inter, dim, touched, owner, heads);
      } else {
        ++wide;
        CHECK(rotated / 2 > kRotaryTable);
      }
    };
    CHECK(fira_rotary(&d, h, count, (const double*)4096, nullptr, nullptr) == FIRA_OK);
    if (wide) { CHECK(wide == (int)heads.size()); continue; }
    for (const auto& t : touched)
      for (size_t i = 0; i < t.size(); ++i) {
        const bool want = !in_place || (int64_t)(i % dim) < rotated;
        if ((t[i] != 0) != want || t[i] > 2) { CHECK((t[i] != 0) == want && t[i] <= 2); break; }
      }
  }
  // the same with more tokens than one launch has threads for: launches adjoin
  int64_t next = 0, launches = 0;
  const fira_rotary_desc d{1, (1ll << 31) - 1, 6, 6, 1, 0, 0, 0, 1.0};
  const fira_rotary_heads h{(void*)4096, (void*)(1ll << 50), 300, {0, 0, 0}, {0, 1800, 6}};
  look = [&](const void*, dim3 grid, void** args) {
    const FiraRotary& r = *(const FiraRotary*)args[0];
    CHECK(r.token0 == next && grid.x % r.chunks == 0);
    next += (int64_t)(grid.x / r.chunks) * r.tile;
    ++launches;
  };
  CHECK(fira_rotary(&d, &h, 1, (const double*)4096, nullptr, nullptr) == FIRA_OK);
  CHECK(next >= d.length && launches > 1);
}

// ---- block norm -----------------------------------------------------------------------------------------------------------

void check_block_norms() {
  look = nullptr;
  void* const p[] = {(void*)(1ll << 20), (void*)(2ll << 20), (void*)(3ll << 20), (void*)(4ll << 20), (void*)(5ll << 20), (void*)(6ll << 20)};
  for (int round = 0; round < 4000; ++round) {
    const int64_t rows = (int64_t)std::exp2(31.0 * (double)(rng() % 1000) / 1000) - 1, dim = (int64_t)std::exp2((round % 8 ? 14.5 : 24.0) * (double)(rng() % 1000) / 1000);
    const fira_block_norm_desc d{rows, dim, (int32_t)pick(0, 1), (int32_t)pick(0, 1), (int32_t)pick(0, 2), (int32_t)pick(0, 2), 1e-5, 1e-5, 1.0, 1.0};
    const fira_block_norm_params v{p[0], nullptr, nullptr, nullptr, nullptr};
    const fira_block_norm_gradients g{p[0], nullptr, nullptr, nullptr, nullptr};
    const int64_t parts = block_parts(&d);
    const size_t bytes = fira_block_norm_gradient_workspace_bytes(&d);
    CHECK(parts >= 1 && parts < 1 << 20 && bytes >= (size_t)(16 * parts * dim) + (dim > kBlockWidest ? (size_t)(8 * rows) : 0) && bytes > FIRA_UNUSED_WORKSPACE_BYTES);
    const bool y = d.norm != FIRA_NO_NORM;
    CHECK(fira_block_norm(&d, p[0], dim, p[1], dim, &v, p[2], dim, y ? p[3] : nullptr, dim, (float*)p[0], (float*)p[0], (float*)p[0], (float*)p[0], nullptr) == FIRA_OK);
    CHECK(fira_block_norm_gradient(&d, p[0], dim, y ? p[1] : nullptr, dim, p[2], dim, p[3], dim, &v, (const float*)p[0], (const float*)p[0], (const float*)p[0], (const float*)p[0], p[4], dim, p[5],
                                   dim, &g, round & 1, p[0], bytes, nullptr) == FIRA_OK);
  }
}

}  // namespace

int main() {
  on_launch = launched_here;
  check_adamw_lists();
  check_rotary_units();
  check_block_norms();
  CHECK(most_threads < (int64_t)1 << 32);
  // a launch that fails is reported
  launches_fail = true;
  look = nullptr;
  const fira_adamw_hparams hp{1e-3, 0.9, 0.999, 1e-8, 1.0};
  CHECK(fira_adamw_step(nullptr, 0, &hp, nullptr, nullptr, nullptr, (int64_t*)4096, nullptr, nullptr, nullptr) == FIRA_ERR_HIP && message.find("AdamW") != std::string::npos);
  std::printf("%d failure(s)\n", failures);
  return failures != 0;
}
