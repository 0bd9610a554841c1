// Reads sizes (groups, rows per group, columns and rows of the weights, pair, 8 bits, gathered), prints what
// paper_2601_21198_b200/csrc/grouped_choice.h reckons that either kernel takes on 148 SMs, in us.
#include <cstdio>

#include "grouped_choice.h"

int main() {
  unsigned groups, each, cols, rows, pair, int8, gathered;
  while (std::scanf("%u %u %u %u %u %u %u", &groups, &each, &cols, &rows, &pair, &int8, &gathered) == 7) {
    const zipmoe_host::GroupedSizes s = {groups, groups * each, rows, cols * (int8 ? 1 : 2), int8 != 0, pair != 0, gathered != 0};
    std::printf("%.4f %.4f %d\n", zipmoe_host::few_ns(s, 148) / 1e3, zipmoe_host::wide_ns(s, 148) / 1e3, (int)zipmoe_host::grouped_wide_pays(s, 148));
  }
}
