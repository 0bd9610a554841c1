// Which of its two kernels takes a grouped product, and how the one for few tokens splits it.  Plain C++ without CUDA, so that the
// choice can be checked against measured times on a CPU.
#pragma once
#include <algorithm>
#include <cstdint>

namespace zipmoe_host {

struct GroupedSizes {
  uint32_t groups, rows;   // rows: of the product, of all groups together
  uint32_t N, Kb;          // output columns; bytes of a row of x
  bool int8, pair, gathered;
};

// What either kernel takes, in ns on a device of `sms` SMs, if the rows are spread evenly over the groups.  (How they are spread is
// known on the device alone: where most rows fall on one of many experts the kernel for few tokens reads that expert's weights once
// per 64 of them.)  Both forms are sums of what the kernels do, with rates fitted to 264 measured pairs of times.  Of those they
// are: few, 0.45 to 1.53 of the measured time; many, 0.56 to 1.48; about one in five is off by more than a fifth.  They err
// alike where it matters: the kernel that is taken costs at most 1.29 of the other's time.
//   Few: weights from memory at 6.5 TB/s, whatever is taken in again for every further 64 tokens, and the tokens, at 10 TB/s (from the
//   second-level cache), 2.5 us per block that an SM takes after another, 5.5 us besides.
inline uint64_t few_ns(const GroupedSizes &s, uint32_t sms) {
  const uint64_t groups = std::min(s.groups, s.rows), each = (s.rows + groups - 1) / groups, tiles = groups * ((each + 63) / 64);
  const uint64_t units = tiles * ((s.N + (s.pair ? 63 : 127)) / (s.pair ? 64 : 128)), steps = (s.Kb + 127) / 128;
  const uint64_t weights = groups * s.N * s.Kb * (s.pair ? 2 : 1), all = units * steps * (16384 + std::min<uint64_t>(64, (each + 15) / 16 * 16) * 128);
  return 5500 + weights / 6500 + (all > weights ? (all - weights) / 10000 : 0) + 2500 * ((units + 2 * sms - 1) / (2 * sms));
}
//   Many: the longer of the weights from memory at 5.8 TB/s and rounds of 512 rows of weights x up to 256 tokens per pair of blocks,
//   0.45 (8-bit integers) to 0.6 us a step and 0.15 to 0.25 more with 256 tokens, 2.2 us besides; 6 us; the gathered rows' packing.
inline uint64_t wide_ns(const GroupedSizes &s, uint32_t sms) {
  const uint64_t groups = std::min(s.groups, s.rows), each = (s.rows + groups - 1) / groups, pairs = std::max(1u, sms / 2);
  const uint64_t deep = (each + 255) / 256, steps = (s.Kb + 127) / 128;
  const uint64_t tiles = groups * deep * ((s.N + (s.pair ? 255 : 511)) / (s.pair ? 256 : 512)), rounds = (tiles + pairs - 1) / pairs;
  const uint64_t cols = (each + deep - 1) / deep / (tiles * 2 <= pairs ? 2 : 1);   // (few tiles are cut by tokens)
  const uint64_t step = s.int8 ? 450 + cols : 600 + cols * 6 / 10, weights = groups * s.N * s.Kb * (s.pair ? 2 : 1);
  return 6000 + std::max(weights / 5800, rounds * (steps * step + 2200)) + (s.gathered ? 3000 + (uint64_t)s.rows * s.Kb * 2 / 5000 : 0);
}

inline bool grouped_wide_pays(const GroupedSizes &s, uint32_t sms) { return s.rows > 0 && wide_ns(s, sms) < few_ns(s, sms); }

}  // namespace zipmoe_host
