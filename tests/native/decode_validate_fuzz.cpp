// Host-side fuzz of the argument checks of the entry points for few sequences (4-bit weights, the
// layer for few tokens, the paged 8-bit cache), as validate_fuzz.cpp does for the layer's calls.
#include <cstdint>
#include <cstdio>

#include "moe_validate.h"

namespace {

uint64_t g_state = 0x243F6A8885A308D3ull;
uint64_t next() {                       // splitmix64
  uint64_t z = (g_state += 0x9E3779B97F4A7C15ull);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

const int64_t k64[] = {INT64_MIN, -1, 0, 1, 2, 15, 16, 17, 64, 1000, 1 << 20, 1ll << 24, (1ll << 31) - 1, 1ll << 31,
                       1ll << 40, INT64_MAX / 2, INT64_MAX};
const int32_t k32[] = {INT32_MIN, -1, 0, 1, 2, 3, 8, 16, 17, 32, 63, 64, 65, 128, 192, 256, 4096, 14336, 65535, 65536,
                       1 << 20, 1 << 23, 1 << 24, INT32_MAX - 1, INT32_MAX};

int64_t pick64() { return (next() & 1) ? k64[next() % (sizeof k64 / sizeof k64[0])] : int64_t(next() % 64); }
int32_t pick32() { return (next() & 1) ? k32[next() % (sizeof k32 / sizeof k32[0])] : int32_t(32 * (next() % 300)); }

alignas(16) unsigned char g_buf[64];
void* pickp() {
  switch (next() % 16) {
    case 0: return nullptr;
    case 1: return g_buf + 4;           // misaligned
    default: return g_buf;
  }
}

int g_fail = 0;
long g_accepted = 0;
void expect(bool ok, const char* what, long long a, long long b) {
  if (ok) return;
  std::fprintf(stderr, "FAIL %s (%lld, %lld)\n", what, a, b);
  ++g_fail;
}

}  // namespace

int main() {
  using namespace moe;
  for (int i = 0; i < 300000; ++i) {
    const int64_t T = pick64(), rows = pick64(), mats = pick64();
    const int32_t H = pick32(), E = pick32(), k = pick32(), F = pick32(), Fs = pick32(), K = pick32(), N = pick32();
    const int32_t group = (next() & 1) ? 32 << next() % 3 : pick32(), flag = int32_t(next() % 3);
    const size_t ws = (next() & 1) ? size_t(next() % (1ull << 34)) : ~size_t(0);
    Check c = validate_quantize_int4(pickp(), rows, K, group, pickp(), pickp(), pickp());
    g_accepted += c.ok();
    c = validate_pack_int4(pickp(), pickp(), pickp(), mats, rows, K, group, pickp(), pickp());
    if (c.ok() && mats > 0 && rows > 0) {
      const int64_t tiles = int64_t(int4_code_bytes(rows, K) / 1024);
      expect(tiles > 0 && mats <= ((1 << 26) / tiles), "packed tiles", mats, tiles);
      expect(int4_scale_bytes(rows, K, group, 0) == size_t(tiles) * 16 * (128 / group) * 2, "scale bytes", rows, K);
    }
    c = validate_matvec_int4(pickp(), pickp(), pickp(), flag, T, N, K, group, pickp());
    if (c.ok()) {
      expect(int4_code_bytes(N, K) < (size_t(1) << 31), "32-bit offsets", N, K);
      expect(int64_t(64) * K * 2 < (int64_t(1) << 31), "32-bit offsets of x", K, 0);
    }
    const void* w[6];
    moe_int4 w4[6];
    for (int j = 0; j < 6; ++j) {
      w[j] = pickp();
      w4[j] = {static_cast<const uint8_t*>(pickp()), static_cast<const uint8_t*>(pickp())};
    }
    const Check few = validate_few(pickp(), pickp(), T, H, E, k, F, Fs, flag, w, pickp(), pickp(), pickp(), pickp(), ws);
    const Check few4 = validate_few_int4(pickp(), pickp(), T, H, E, k, F, Fs, flag, group, int32_t(next() % 3),
                                         next() % 8 ? w4 : nullptr, pickp(), pickp(), pickp(), pickp(), ws);
    if ((few.ok() || few4.ok()) && T > 0) {
      expect(few_workspace_bytes(T, H, k, F, Fs) <= ws, "few: short workspace accepted", T, H);
      expect(few_partial_offset(T, k, F, Fs) < (size_t(1) << 31), "few: 32-bit offsets of h", k, F);
      expect(T <= MOE_FEW_TOKENS && H % 64 == 0 && F % 64 == 0 && Fs % 64 == 0, "few: sizes", H, F);
    }
    const moe_kv8_cache cache = {static_cast<uint8_t*>(pickp()), static_cast<uint8_t*>(pickp()),
                                 static_cast<uint8_t*>(pickp()), static_cast<uint8_t*>(pickp()), pick64(),
                                 (next() & 1) ? int32_t(16 << next() % 4) : pick32(),
                                 (next() & 1) ? int32_t(1 + next() % 8) : pick32(),
                                 (next() & 1) ? int32_t(64 << next() % 3) : pick32()};
    const int32_t q_heads = (next() & 1) && cache.heads > 0 && cache.heads < 1000 ? cache.heads * int32_t(1 + next() % 8)
                                                                                  : pick32();
    const int32_t cols = pick32(), B = pick32(), new_most = pick32(), len = pick32(), window = pick32();
    c = validate_kv8_append(pickp(), pick64(), pickp(), pick64(), pickp(), pick64(), T, q_heads, pickp(), pick64(), pick32(),
                            flag, next() % 8 ? &cache : nullptr, pickp(), cols, pickp(), pickp(), B, pickp());
    g_accepted += c.ok();
    const float scale = next() % 8 ? 0.125f : next() % 2 ? -1.0f : 0.0f / (next() % 2 ? 1.0f : -1.0f);
    const size_t need = next() % 2 ? 0 : size_t(next() % (1ull << 34));
    c = validate_kv8_attention(pickp(), T, q_heads, next() % 8 ? &cache : nullptr, pickp(), cols, pickp(), pickp(), B,
                               new_most, len, window, scale, pickp(), pickp(), ws, need);
    if (c.ok() && T > 0) {
      expect(kv8_plan_sizes_ok(B, q_heads, cache.heads, cache.dim, new_most, len, window), "plan sizes", B, new_most);
      expect(scale > 0 && need <= ws && int64_t(cols) * cache.page <= INT32_MAX, "attention", cols, cache.page);
      // tiles of 16 rows at most, and the workgroups that cut them, are counted in 32 bits
      const int64_t tiles = (int64_t(new_most) * (q_heads / cache.heads) + 15) / 16;
      expect(tiles * B * cache.heads < INT32_MAX / 2, "attention workgroups", tiles, B);
      ++g_accepted;
    }
  }
  expect(g_accepted > 1000, "some arguments are accepted", g_accepted, 0);
  if (g_fail) {
    std::fprintf(stderr, "%d failures\n", g_fail);
    return 1;
  }
  std::printf("decode_validate_fuzz: 300000 rounds, no failures\n");
  return 0;
}
