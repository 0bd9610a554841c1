// How zipmoe_expert_ffn lays out few tokens' calls, and which of its two kernels takes them.  Plain C++ without CUDA, so
// that the choice can be checked against measured times on a CPU.
#pragma once
#include <algorithm>
#include <cstdint>

namespace zipmoe_host {

// Rows of W1 (and W3) and of W2 that a block of the whole-rows kernel owns, and takes at once (the box rows of the sliced maps).
inline void resident_few_rows(uint32_t H, uint32_t I, uint32_t grid, uint32_t *R1, uint32_t *S1, uint32_t *R2, uint32_t *S2) {
  auto up = [](uint32_t v, uint32_t d) { return (v + d - 1) / d; };
  *R1 = up(I, grid);
  *S1 = up(*R1, up(*R1, 16));
  *R2 = up(H, grid);
  *S2 = up(*R2, up(*R2, 32));
}

// Whether a block's whole rows are the faster way for few tokens.  They save 13 us of a call, but every expert takes a block 0.3 us,
// every chunk of 512 columns of a set of rows 0.42 us however few rows it has, and the columns behind a row's last whole 64, a
// chunk of their own, 0.1 us; where that is longer than an expert's bytes take, experts cost what is over.  8 tokens, whole rows
// against shares: 8 experts of 2048 x 1408 35 against 43 us, 30 of them 99 against 95; 30 of 3008 x 1536 128 against 140; 30 of
// 4096 x 256 119 against 53; 60 of 1024 x 512 116 against 48, but 8 of them (one token) 24 against 28; 30 of 2056 x 1416 104
// against 100; 60 of 1896 x 1896 239 against 221; 10 of 1544 x 1544 42 against 45.  (A second column of eight tokens was built and
// taken out: 16 tokens, 16 experts of 1096 x 904: 60 us against 44.)
inline bool whole_rows_pay(uint32_t choices, uint32_t E, uint32_t H, uint32_t I, uint32_t grid) {
  uint32_t R1, S1, R2, S2;
  resident_few_rows(H, I, grid, &R1, &S1, &R2, &S2);
  auto row_ns = [](uint32_t K) { return 420ull * std::max(1u, (K / 64 + 7) / 8) + (K % 64 ? 100 : 0); };    // of a set of rows
  const uint64_t expert_ns = 300 + (R1 + S1 - 1) / S1 * row_ns(H) + (R2 + S2 - 1) / S2 * row_ns(I);
  const uint64_t byte_ns = 6ull * H * I / 6464;
  return expert_ns <= byte_ns || std::min(choices, E) * (expert_ns - byte_ns) <= 13000;
}

}  // namespace zipmoe_host
