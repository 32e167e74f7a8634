// Host-only check of the largest calls that include/fira.h allows of AdamW and of rotary positions, and of every width of the block norm: their host code (csrc/fira_model.hip) over a stand-in for the HIP runtime
// (host_hip.h), which hands every launch to this program.  Built and run on the CPU by tests/test_host_model_limits.py.
#include "../paper_2410_01623_amd/csrc/fira_model.hip"

#include <cstring>
#include <functional>
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
std::string message;
std::function<void(const void*, dim3, void**)> look;
void launched_here(const void* f, dim3 grid, void** args) {
  CHECK(grid.x >= 1 && pushed_block.x >= 1 && pushed_block.x <= 1024 && (int64_t)grid.x * grid.y * grid.z * pushed_block.x < (int64_t)1 << 32);
  look(f, grid, args);
}
}  // namespace
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
fira_status fira_fail_without_context(fira_status st, const char* msg) noexcept {
  message = msg;
  return st;
}

namespace {

// Up to four tensors of any heads below 2^31, more than that together: each is turned by a launch of its own heads.
void check_rotary_heads() {
  const int64_t most = 0x7fffffff;
  const std::vector<std::vector<int64_t>> lists = {{most}, {most, most}, {most, most, most}, {most, most, most, most}, {most, 5, most, 7}, {1, most, 0, most}, {1 << 30, 1 << 30, 1 << 30, 1 << 30}};
  for (const auto& heads : lists)
    for (int layout = 0; layout < 2; ++layout)
      for (int64_t dim : {2, 6}) {
        std::vector<fira_rotary_heads> h;
        for (size_t i = 0; i < heads.size(); ++i)
          h.push_back({(void*)((1ll << 44) * (int64_t)(i + 1)), (void*)((1ll << 44) * (int64_t)(i + 9)), heads[i], {0, 0, 0}, {0, heads[i] * dim, dim}});
        const fira_rotary_desc d{1, 3, dim, 2, FIRA_BF16, layout, FIRA_I64, 0, 1.0};
        std::vector<int64_t> seen;
        look = [&](const void* f, dim3 grid, void** args) {
          CHECK(f == (const void*)fira_rotary_wide_kernel<FiraStoredBf16>);
          const FiraRotary& r = *(const FiraRotary*)args[0];
          const int k = *(const int*)args[1];
          const unsigned n = *(const unsigned*)args[2];
          CHECK(k == (int)seen.size() && k < r.count && (int64_t)grid.x <= 1 << 20);
          size_t i = 0;                                    // the k-th tensor that has heads
          for (int j = k; i < heads.size(); ++i)
            if (heads[i] && j-- == 0) break;
          CHECK(i < heads.size() && (int64_t)n == heads[i] && r.t[k].x == h[i].dev_x && r.t[k].y == h[i].dev_y);
          seen.push_back(n);
        };
        CHECK(fira_rotary(&d, h.data(), (int)h.size(), (const double*)4096, nullptr, nullptr) == FIRA_OK);
        size_t some = 0;
        for (int64_t n : heads) some += n != 0;
        CHECK(seen.size() == some);
      }
}

// 2^35 values and more in one list, rows apart and not whole vectors wide, states in 8 bits: each launch has a grid that it may have, and covers its pieces.
void check_adamw_threads() {
  typedef FiraStoredF32 F;
  typedef FiraStoredBf16 B;
  const int64_t rows = 1047552, cols = 1025;               // nearly a whole piece, so that a launch has 36 of them
  for (int n : {33, 36, 40})
    for (int kind = 0; kind < 4; ++kind) {
      std::vector<fira_adamw_desc> d((size_t)n, fira_adamw_desc{rows, cols, cols + 3, cols + 3, kind & 1, kind >> 1, FIRA_STATE_E4M3, 0, 0.0});
      std::vector<void*> W;
      std::vector<const void*> G;
      std::vector<fira_adamw_state> S;
      for (int64_t i = 0; i < n; ++i) {
        char* const at = (char*)((i + 1) << 36);
        W.push_back(at);
        G.push_back(at + (1ll << 33));
        S.push_back({at + (2ll << 33), at + (3ll << 33), (float*)(at + (4ll << 33)), (float*)(at + (5ll << 33))});
      }
      int64_t values = 0;
      look = [&](const void* f, dim3 grid, void** args) {
        if (f == (const void*)fira_adamw_count_kernel<>) return;
        CHECK(f == (kind == 0 ? (const void*)fira_adamw_kernel<F, F, true, true> : kind == 1 ? (const void*)fira_adamw_kernel<B, F, true, true> :
                    kind == 2 ? (const void*)fira_adamw_kernel<F, B, true, true> : (const void*)fira_adamw_kernel<B, B, true, true>));
        const FiraAdamSpans& l = *(const FiraAdamSpans*)args[0];
        CHECK((int)grid.x <= l.tiles);
        for (int i = 0; i < l.count; ++i) values += l.s[i].n;
      };
      const fira_adamw_hparams hp{1e-3, 0.9, 0.999, 1e-8, 1.0};
      CHECK(fira_adamw_step(d.data(), n, &hp, W.data(), G.data(), S.data(), (int64_t*)4096, nullptr, nullptr, nullptr) == FIRA_OK);
      CHECK(values == n * rows * cols);
    }
}

// Every width that a row of the block norm is held by: a row's vectors cover it, none begins before it, and the first half of a thread's vectors, which the kernels take
// as wholly its own, lie wholly inside; a column is one thread's own.
template <typename T, bool FORWARD>
void check_block_shapes() {
  for (int64_t dim = 1; dim <= (FORWARD ? kNormWidest : kBlockWidest); ++dim)
    with_block_shape<T, FORWARD>(dim, [&](auto width, auto threads, auto nv) {
      constexpr int W = decltype(width)::value, THREADS = decltype(threads)::value, NV = decltype(nv)::value;
      CHECK((int64_t)THREADS * W * NV >= dim && (int64_t)THREADS * W * (NV / 2) <= dim && dim >= W);
      CHECK(THREADS <= 1024 && (THREADS >= 64 ? THREADS % 64 == 0 : 64 % THREADS == 0));
      if (dim % 97 && dim % 64 > 1) return;
      std::vector<int> own((size_t)dim, 0);
      for (int v = 0; v < NV; ++v)
        for (int me = 0; me < THREADS; ++me) {
          // (as Columns has it)
          const int64_t c = ((int64_t)v * THREADS + me) * W, at = std::min(c, dim - W), skip = v < NV / 2 ? 0 : c < dim ? c - at : W;
          CHECK(at >= 0 && (v >= NV / 2 || at == c));
          for (int64_t j = skip; j < W; ++j) ++own[(size_t)(at + j)];
        }
      for (int n : own)
        if (n != 1) { CHECK(n == 1); break; }
    });
}

}  // namespace

int main() {
  on_launch = launched_here;
  check_block_shapes<FiraStoredF32, true>();
  check_block_shapes<FiraStoredF32, false>();
  check_block_shapes<FiraStoredBf16, true>();
  check_block_shapes<FiraStoredBf16, false>();
  check_adamw_threads();
  check_rotary_heads();
  std::printf("%d failure(s)\n", failures);
  return failures != 0;
}
