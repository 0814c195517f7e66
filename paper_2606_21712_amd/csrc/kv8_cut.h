// How attention over the 8-bit cache is cut up.  Plain C++, no HIP dependency, so that a host can
// evaluate it; what the kernels share is constexpr.
#pragma once
#include <algorithm>
#include <cstdint>

namespace moe {

constexpr int kChunk = 64;                    // tokens: the unit in which work is dealt

// Chunks of `len` tokens.
constexpr int kv8_chunks(int len) { return len > 0 ? (len - 1) / kChunk + 1 : 0; }

// Whether the chunks of `tiles` tiles of up to `capacity` tokens are counted in 32 bits, as the kernel adds
// them up where it cuts tiles: 511 tiles of 268 million tokens are not.
constexpr bool kv8_counts_fit(int64_t tiles, int capacity) { return tiles * kv8_chunks(capacity) <= INT32_MAX; }

// Steps [begin, end) of `tok` tokens (kChunk or a divisor of it); end <= begin: none.
struct Kv8Steps {
  int begin, end;
};

// The steps of part `part` of `parts` of a tile whose rows are at positions first .. last: equal numbers
// of the chunks that its rows see.  The last chunk's steps end with the one that holds `last`: the next
// one's page need not have a place in the block table.
constexpr Kv8Steps kv8_steps(int first, int last, int window, int part, int parts, int tok) {
  const int low = window > 0 ? std::max(std::max(first, 0) - window + 1, 0) : 0;   // first: maybe below 0
  const int c0 = low / kChunk, c1 = last < 0 ? c0 : std::max(last / kChunk + 1, c0);
  const int each = (std::max(c1 - c0, 0) + parts - 1) / parts;
  const int begin = std::min(c0 + part * each, c1), end = std::min(c0 + (part + 1) * each, c1);
  return {begin * (kChunk / tok), std::min(end * (kChunk / tok), last / tok + 1)};
}

}  // namespace moe
