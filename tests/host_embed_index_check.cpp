// Host-only check of the embedding gradient's index arithmetic (csrc/fira_embed.h) up to the 2^31 - 1 tokens that a call may have: how rows are cut into
// pieces and how a bucket's entries are shared among wavefronts, against the same in 64 bits.  Run by tests/test_host_embed_index.py.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>

#include "../paper_2410_01623_amd/csrc/fira_embed.h"
#include "host_hip.h"

namespace {

void check_pieces(int64_t n) {
  const int64_t len = piece_tokens((int)n), pieces = row_pieces((int)n);
  if (n <= kPieceTokens) { CHECK(len == kPieceTokens && pieces == 0); return; }
  CHECK(len >= kPieceTokens && len % kPieceTokens == 0);
  CHECK(pieces >= 2 && pieces <= 256 && pieces * len >= n && (pieces - 1) * len < n);
  CHECK(len == kPieceTokens || n > 256 * (len / 2));                      // no longer than it has to be
  CHECK(pieces <= 2 * (n / kPieceTokens));                                // ... and as many as the workspace has room for
}

void check_spans(int64_t total) {
  for (int64_t waves = 1; waves <= 16; ++waves) {
    const int64_t span = wave_span((unsigned)total, (unsigned)waves);
    CHECK(span >= 64 && span % 64 == 0 && waves * span >= total);
    CHECK(span == 64 || waves * (span - 64) < total);
    CHECK(waves * span + 64 < (int64_t)1 << 32);                          // the last wavefront's last group
    CHECK(total == 0 || (total - 1) / span < waves);
  }
}

}  // namespace

int main() {
  const int64_t last = 0x7fffffff;
  for (int64_t n = 0; n <= 70000; ++n) { check_pieces(n); check_spans(n); }
  for (int shift = 13; shift <= 31; ++shift)
    for (int64_t d = -300; d <= 300; ++d) {
      const int64_t n = ((int64_t)1 << shift) + d;
      if (n <= last) { check_pieces(n); check_spans(n); }
    }
  std::mt19937_64 rng(3);
  for (int i = 0; i < 200000; ++i) { const int64_t n = (int64_t)(rng() % (uint64_t)(last + 1)); check_pieces(n); check_spans(n); }
  std::printf("%d failure(s)\n", failures);
  return failures != 0;
}
