// Which kernel a product with weights of 4 bits is launched with, as the library's own rule says it.
// Usage: linear4_plan <units> {<rows> <width in> <width out> <group>}...: a line each
#include <cstdio>
#include <cstdlib>
#include "../../paper_2411_01830_amd/csrc/ft_linear4_plan.h"

int main(int argc, char **argv) {
  const int units = std::atoi(argv[1]);
  for (int i = 2; i + 3 < argc; i += 4) {
    const uint32_t rows = std::strtoul(argv[i], nullptr, 10), ni = std::strtoul(argv[i + 1], nullptr, 10), no = std::strtoul(argv[i + 2], nullptr, 10),
                   group = std::strtoul(argv[i + 3], nullptr, 10);
    const ft::Linear4Plan p = ft::linear4_plan(ni, no, group, rows, units);
    // of wide ones how many pieces of a row's groups have their scales brought in turn by one workgroup
    if (p.any) std::printf("any\n");
    else if (p.narrow) std::printf("narrow %d\n", rows > 8 ? 16 : rows > 2 ? 8 : 2);
    else std::printf("wide %u %s %u\n", p.tiles, p.parts > 1 ? "shared" : "whole", (p.each + group / 4 - 1) / (group / 4));
  }
}
