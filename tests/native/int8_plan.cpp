// Evaluates the rule for products of 8-bit codes (csrc/launch_rules.h): "T N K gated compute-units" per input line,
// "form parts tiles part_bytes stream" per output line.
#include <iostream>

#include "launch_rules.h"

int main() {
  int64_t T, N, K;
  int gated, cus;
  while (std::cin >> T >> N >> K >> gated >> cus) {
    const moe::Int8Plan p = moe::int8_plan(T, N, K, gated != 0, cus);
    std::cout << int(p.form) << " " << p.parts << " " << p.tiles << " " << p.part_bytes << " " << p.stream << "\n";
  }
}
