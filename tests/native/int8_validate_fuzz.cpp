// Host-side fuzz of the argument checks of the dense half in 8-bit integers, as validate_fuzz.cpp does for the
// layer's calls: no check may overflow, and what it lets through has to fit the launches.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "moe_validate.h"

namespace {

uint64_t g_state = 0x452821E638D01377ull;
uint64_t next() {                       // splitmix64
  uint64_t z = (g_state += 0x9E3779B97F4A7C15ull);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

const int64_t k64[] = {INT64_MIN, -1, 0, 1, 2, 16, 1000, 1 << 20, (1 << 20) + 1, 1ll << 24, (1ll << 24) + 1, 1ll << 31,
                       1ll << 40, INT64_MAX / 2, INT64_MAX};
const int32_t k32[] = {INT32_MIN, -1, 0, 1, 8, 16, 24, 4096, 14336, 32768, 131056, 131072, 1 << 24, INT32_MAX};

int64_t pick64() { return (next() & 1) ? k64[next() % (sizeof k64 / sizeof k64[0])] : int64_t(8 * (next() % 5000)); }
int32_t pick32() { return (next() & 1) ? k32[next() % (sizeof k32 / sizeof k32[0])] : int32_t(16 * (next() % 300)); }
int32_t small() { return int32_t(next() % 6) - 1; }
float number() {
  const float f[] = {0.f, 1.f, -1.f, 1e-6f, 1e38f, INFINITY, NAN};
  return f[next() % 7];
}

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
    const int64_t T = pick64(), a = pick64(), b = pick64(), c64 = pick64();
    const int32_t H = pick32(), N = pick32();
    const float eps = number();
    const int kind = small();
    Check c = validate_norm_join(pickp(), a, small(), pickp(), b, small() & 1, pickp(), kind > 0 ? pickp() : nullptr, c64, kind,
                                 small() & 1, number(), pickp(), number(), eps, T, H, pickp(), a, 1, pickp(), pickp());
    if (c.ok()) {
      ++g_accepted;
      expect(H > 0 && H % 8 == 0 && H <= 32768 && T >= 0 && eps >= 0, "norm sizes", T, H);
      expect(T == 0 || (a >= H && a % 4 == 0), "strides", a, H);
    }
    c = validate_quantize_int8(pickp(), a, T, H, pickp(), pickp());
    if (c.ok()) {
      ++g_accepted;
      expect(H % 16 == 0 && H <= 131056 && T >= 0 && (T == 0 || (a >= H && a % 8 == 0)), "rows", T, H);
    }
    c = validate_pack_int8(pickp(), T, H, pickp());
    if (c.ok() && T > 0) {
      ++g_accepted;
      const size_t n = int8_code_bytes(T, H);
      expect(n > 0 && n % 2048 == 0 && n / 1024 <= (1u << 26), "packed pieces", T, H);
    }
    const size_t ws = (next() & 1) ? 0 : ~size_t(0), need = next() % 3 ? 0 : 1000;
    c = validate_matmul_int8(pickp(), pickp(), pickp(), pickp(), pickp(), T, N, H, pickp());
    if (c.ok()) {
      ++g_accepted;
      expect(T >= 0 && T <= (1 << 20) && N >= 1 && N <= (1 << 24) && H % 16 == 0 && H <= 131056, "product", T, N);
      expect(int8_sizes_ok(T, N, H) == (T > 0), "sizes", T, N);
      expect(T == 0 || T * int64_t(N) <= (int64_t(1) << 37), "outputs", T, N);
    }
    c = validate_gated_int8(pickp(), pickp(), pickp(), pickp(), pickp(), pickp(), T, N, H, pickp());
    if (c.ok()) ++g_accepted;
    c = validate_int8_workspace("call", pickp(), ws, need);
    if (c.ok()) expect(ws >= need, "workspace", (long long)ws, (long long)need);
  }
  if (g_accepted < 20000) {
    std::fprintf(stderr, "FAIL only %ld accepted\n", g_accepted);
    ++g_fail;
  }
  if (g_fail == 0) std::printf("no failures (%ld accepted)\n", g_accepted);
  return g_fail != 0;
}
