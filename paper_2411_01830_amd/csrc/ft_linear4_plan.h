// Which kernel a product with weights of 4 bits is launched with (ft_linear4.hip), from its sizes alone.
#pragma once
#include <stdint.h>

namespace ft {

constexpr uint32_t kMostGroups = 1024;  // of a row, for what has a workgroup's scales in shared memory from the start

// Which kernel multiplies, and what of it a workgroup has.
struct Linear4Plan {
  bool any, narrow;
  uint32_t tiles, waves;  // wide: tiles of 16 rows of x, wavefronts along the rows of weights
  uint32_t each, parts;   // chunks of 256 elements to a workgroup, workgroups along them
};

// What the kernels take for more than two rows, in nanoseconds, from the widths and rows alone; the shortest is launched. (One or two rows are at least as
// fast in the narrow one: of 4096 to 32768 the same, below that 2 to 5 us less.) A workgroup of the wide kernel takes a time for 256 elements that depends
// on its tiles of 16 rows of x and on whether a compute unit has one or two of them (of four tiles, with 128 rows of weights, one; registers have room
// for no more); what several workgroups have of the same sums goes through memory and a second launch. The narrow one has a workgroup to a compute unit, of up
// to eight rows two that share it. Measured, us, narrow and wide of 1, 2 and 4 tiles, * with the work along the rows shared out (8: wide of 9 rows):
//    8 rows of 2048 to 32768  18.7 12.8              8 of 4096 to 14336     13.5 15.0             8 of 8192 to 8192     12.3 15.5*
//   16 rows of 2048 to 8192    8.2  9.3             16 of 4096 to 4096      6.0  9.4*            16 of 8192 to 8192     18.0 15.9*
//   32 rows of 1024 to 8192   12.7  6.6  7.8        32 of 4096 to 4096     10.3 10.9* 11.1*      32 of 8192 to 32768       -  64.0  47.1 58.5
//   64 rows of 2048 to 4096   14.6  8.4 10.9* 14.4* 64 of 4096 to 4096     18.4 12.0 13.5* 15.8* 64 of 2048 to 32768      -  33.6  27.4 20.8
//   64 rows of 8192 to 8192      - 29.2 27.3* 25.2* 64 of 8192 to 32768       -  106   86  65   128 of 4096 to 14336      -  47.0  41.0 31.1
//  128 rows of 2048 to 8192      - 17.2 13.4 18.7* 128 of 4096 to 4096     35.1 15.6 15.7 18.7* 256 of 4096 to 4096      -  26.4  21.2 24.0*
// These are of groups of 128, and the rule does not know of others, whose chunks take longer in the wide kernel. Of the sizes above the shortest of all ways
// is at most 8 % below the one taken in groups of 128 and of 64 (32 rows of 8192 to 32768 57 us, 62 taken); in groups of 32 too, but for 64 rows of 4096 to
// 4096, 17.8 in tiles of two shared out and 24.5 taken, and 16 of 4096 to 14336, 20.5 shared out and 26 taken.
inline uint64_t linear4_narrow_time(uint32_t width_in, uint32_t width_out, uint32_t rows, uint32_t units) {
  const uint64_t workgroups = (uint64_t)((width_out + 15) / 16) * ((rows + 15) / 16);
  return 2500 + (workgroups + units - 1) / units * (rows > 8 ? 1200 + (uint64_t)width_in * 4 / 5 : 600 + width_in / 2);
}
inline uint64_t linear4_wide_time(const Linear4Plan &p, uint64_t workgroups, uint64_t result, uint32_t units) {
  const uint64_t one = p.tiles == 4 ? 1700 : p.tiles == 2 ? 700 : 520, two = p.tiles == 2 ? 1100 : 720;
  const uint64_t most = p.tiles == 4 ? units : 2 * units, all = workgroups * p.parts, rest = all % most;
  const uint64_t chunk = all / most * (p.tiles == 4 ? one : two) + (rest == 0 ? 0 : rest <= units ? one : two);
  return 5000 + p.each * chunk + (p.parts > 1 ? 3000 + result * p.parts / 600 : 0);  // (elements of 32 bits, written and read at 5 TB/s)
}

inline Linear4Plan linear4_plan(uint32_t width_in, uint32_t width_out, uint32_t group, uint32_t rows, int cu_count) {
  const uint64_t groups = (width_in + (uint64_t)group - 1) / group;
  Linear4Plan best{};
  best.any = group < 32 || groups > kMostGroups || width_in < 32 || width_out * groups < 16;  // (loads are of 16 bytes)
  best.narrow = true;
  if (best.any || rows <= 2) return best;
  const uint32_t chunks = (width_in + 255) / 256, units = (uint32_t)cu_count;
  uint64_t shortest = linear4_narrow_time(width_in, width_out, rows, units);
  for (uint32_t tiles = 1; tiles <= 4 && (tiles == 1 || 8 * tiles < rows); tiles *= 2) {
    // With four tiles 128 rows of weights to a workgroup, else 64: 64 rows of 8192 to 32768 64 us and 93 with 64 rows of weights, 32 rows 51 and 48, 16 45 and 37.
    Linear4Plan p{};
    p.tiles = tiles;
    p.waves = tiles == 4 ? 4 : 2;
    const uint64_t workgroups = (uint64_t)((width_out + 32 * p.waves - 1) / (32 * p.waves)) * ((rows + 16 * tiles - 1) / (16 * tiles));
    for (uint32_t fill = 0; fill <= (tiles == 4 ? 1 : 2); ++fill) {  // not shared out; to one workgroup a unit, to two: four chunks each at least
      uint64_t parts = fill * units / workgroups;
      if (parts > chunks / 4) parts = chunks / 4;
      if (parts < 1) parts = 1;
      p.each = (chunks + (uint32_t)parts - 1) / (uint32_t)parts;
      p.parts = (chunks + p.each - 1) / p.each;
      const uint64_t time = linear4_wide_time(p, workgroups, (uint64_t)rows * width_out, units);
      if (time <= shortest) {
        shortest = time;
        best = p;
      }
    }
  }
  return best;
}

}  // namespace ft
