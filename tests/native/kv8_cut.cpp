// Evaluates csrc/kv8_cut.h on the host: the steps that an attention tile's parts walk, over lengths, new rows,
// windows, numbers of parts and pages.
#include <cstdio>
#include <vector>

#include "kv8_cut.h"

namespace {

int g_fail = 0;
void expect(bool ok, const char* what, int len, int fresh, int window, int parts, int tok) {
  if (ok || ++g_fail > 20) return;
  std::fprintf(stderr, "FAIL %s: len %d, new %d, window %d, parts %d, steps of %d\n", what, len, fresh, window, parts, tok);
}

// One tile with all rows of the sequence: every token that a row sees is in one step of one part, and every step of
// a page that holds whole steps begins in a page that the sequence has.
void check(int len, int fresh, int window, int parts, int tok) {
  const int first = len - fresh, last = len - 1;            // first: below 0 where rows have no place
  const int low = window > 0 && int64_t(first) - window + 1 > 0 ? first - window + 1 : 0;
  std::vector<int> seen(size_t(len) / tok + 3, 0);
  for (int p = 0; p < parts; ++p) {
    const moe::Kv8Steps s = moe::kv8_steps(first, last, window, p, parts, tok);
    for (int i = s.begin; i < s.end; ++i) {
      for (int page : {32, 64, 96, 128, 160, 192})
        if (page % tok == 0)
          expect(i >= 0 && i * tok / page < (len + page - 1) / page, "a page past the sequence's", len, fresh, window, parts,
                 tok);
      if (i >= 0 && size_t(i) < seen.size()) ++seen[size_t(i)];
    }
  }
  for (size_t i = 0; i < seen.size(); ++i) {
    const int from = int(i) * tok, to = from + tok - 1;
    const bool needed = from <= last && to >= low;
    expect(seen[i] <= 1 && (!needed || seen[i] == 1), "a step left out or walked twice", len, fresh, window, parts, tok);
  }
}

}  // namespace

int main() {
  for (int len = 0; len <= 700; ++len)
    for (int fresh : {1, 2, 17, 64, 65, 130, 699})
      for (int window : {0, 1, 33, 100, 500, INT32_MAX})
        for (int parts : {1, 2, 3, 7})
          for (int tok : {32, 64}) check(len, fresh, window, parts, tok);
  // the largest lengths that a block table has place for, and tiles up to two a compute unit of 256
  for (int64_t len : {int64_t(0), int64_t(1), int64_t(64), int64_t(65), int64_t(1) << 28, int64_t(INT32_MAX) - 15,
                      int64_t(INT32_MAX)}) {
    const int64_t chunks = (len + moe::kChunk - 1) / moe::kChunk;
    expect(moe::kv8_chunks(int(len)) == chunks, "chunks", int(len), 0, 0, 0, 0);
    for (int tiles = 1; tiles < 512; ++tiles)
      expect(moe::kv8_counts_fit(tiles, int(len)) == (tiles * chunks <= INT32_MAX), "counts", int(len), tiles, 0, 0, 0);
  }
  if (g_fail == 0) std::puts("ok");
  return g_fail != 0;
}
