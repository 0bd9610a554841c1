// The kernel that zipmoe_expert_ffn takes for few tokens (paper_2601_21198_b200/csrc/resident_choice.h) against times
// measured with either kernel on a B200 (148 SMs): the one taken is never more than 5 % slower than the other.
#include <cstdio>

#include "resident_choice.h"

struct Measured {
  uint32_t tokens, k, experts, hidden, inter;   // as many experts active as tokens * k choices can reach
  double whole_rows_us, shares_us;
};

int main() {
  const Measured all[] = {
      // whole 64 columns
      {8, 4, 30, 512, 512, 50.4, 27.6}, {8, 4, 30, 1024, 1024, 65.6, 45.2}, {8, 4, 30, 2048, 1408, 95.4, 90.0},
      {8, 4, 30, 1536, 1536, 85.4, 79.7}, {8, 4, 8, 768, 768, 25.5, 25.8}, {8, 4, 30, 64, 64, 47.1, 17.1},
      // columns behind the last whole 64
      {8, 4, 30, 520, 520, 55.8, 29.8}, {8, 4, 8, 520, 520, 24.7, 25.6}, {1, 4, 8, 520, 520, 14.6, 23.3},
      {8, 4, 8, 776, 776, 28.4, 27.5}, {4, 4, 8, 776, 776, 25.7, 26.9}, {8, 4, 12, 1000, 520, 33.0, 28.1},
      {8, 4, 30, 1000, 1000, 72.0, 46.6}, {8, 4, 8, 1032, 1032, 29.0, 31.0}, {8, 4, 30, 1032, 1032, 71.9, 49.0},
      {1, 6, 60, 1032, 1032, 22.5, 28.8}, {8, 4, 16, 1488, 1488, 53.7, 51.3}, {8, 4, 30, 1480, 1480, 90.8, 79.2},
      {8, 4, 10, 1544, 1544, 39.7, 43.3}, {8, 4, 30, 1544, 1544, 91.9, 84.6}, {8, 8, 60, 1896, 1896, 229.6, 219.4},
      {8, 4, 24, 2040, 1424, 83.5, 83.5}, {4, 4, 60, 2056, 1416, 47.3, 51.7}, {8, 4, 30, 2056, 1416, 100.8, 94.3},
      {8, 4, 30, 2048, 1416, 98.2, 92.6}, {8, 4, 16, 2568, 2568, 109.3, 110.3}, {8, 4, 30, 2568, 2568, 190.5, 194.6},
      {8, 4, 20, 2568, 1032, 71.1, 68.2}, {8, 4, 30, 3016, 1544, 131.9, 141.1}, {8, 4, 16, 4104, 1032, 80.2, 81.0},
      {8, 4, 16, 4104, 4104, 247.7, 251.7}, {8, 4, 30, 72, 72, 55.1, 20.6}, {8, 4, 30, 40, 40, 42.7, 16.5},
      {1, 8, 30, 40, 40, 16.9, 16.5},
  };
  int wrong = 0;
  for (const Measured &m : all) {
    const bool whole = zipmoe_host::whole_rows_pay(m.tokens * m.k, m.experts, m.hidden, m.inter, 148);
    const double taken = whole ? m.whole_rows_us : m.shares_us, other = whole ? m.shares_us : m.whole_rows_us;
    if (taken <= 1.05 * other) continue;
    std::printf("%u tokens, top %u of %u experts of %u x %u: %s taken, %.1f us against %.1f\n", m.tokens, m.k, m.experts, m.hidden,
                m.inter, whole ? "whole rows" : "shares", taken, other);
    wrong = 1;
  }
  if (!wrong) std::puts("ok");
  return wrong;
}
