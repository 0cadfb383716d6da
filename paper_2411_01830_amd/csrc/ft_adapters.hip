// Low-rank adapters of many requests beside a shared projection: out[t] = base[t] + s B (A x[t]) with the A, B and s of row t.
//
// Rows are put in the order of their adapters and cut into tiles of up to 64 rows of one adapter (ft_adapter_group_kernel), so that a
// tile's products are matrix products. H^T = A X^T first, with the long axis split over workgroups and wavefronts whose sums are put
// into the workspace; then out^T = B H^T, where the parts of H are added up, scaled and held as the sum of two numbers of 16 bits: the matrix
// unit's operands, together 16 bits of a value (22 in float16) where the result has 8 (11). Against 64 bits results are as far off as with H in 32 bits,
// 0.0016 (0.0002) of their size.
// Rows without an adapter are tiles of their own that are copied.
//
// 64 rows of 32 adapters of ranks 8 to 64, 4096 to 4096, in bfloat16: 17.6 us, three launches of 3.8 (grouping), 5.7 and 7.8 us that latency bounds, for
// 15 MB. 8192 rows of 8 adapters, 4096 to 6144: 107 us for 273 MB, 8 + 25.5 + 67; the first product reads X at 2.7 TB/s, the second reads and
// writes 3 TB/s. Of the second one's time writing is 23 us, base 12, adding up the parts of H 16 and the products none: wavefronts wait for
// memory (base and B one after the other), two workgroups to a unit (three, with wavefronts of 32 rows: 118). One kernel for both products takes 122 alone, as a unit then holds one workgroup of the 137; tiles of
// 32 rows 125 for all three.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

constexpr uint32_t kTileRows = 64;
constexpr uint32_t kGroupThreads = 1024;
constexpr uint32_t kAtOnce = 8;  // rows of a thread of the sort

struct Tile {
  int32_t adapter;  // -1: none
  uint32_t first;   // of its rows in `order`
  uint32_t count;
  uint32_t _pad;
};

// What ft_adapters_group leaves for the other kernels.
struct Groups {
  uint32_t *tiles_there;  // a line of its own
  Tile *tiles;
  int32_t *order;
};

__host__ __device__ inline uint64_t most_tiles(uint32_t rows, uint32_t count) {
  const uint64_t kinds = (uint64_t)count + 1 < rows ? (uint64_t)count + 1 : rows;
  return rows / kTileRows + kinds;
}

__host__ __device__ inline Groups groups_at(void *p, uint32_t rows, uint32_t count) {
  char *at = static_cast<char *>(p);
  return {reinterpret_cast<uint32_t *>(at), reinterpret_cast<Tile *>(at + 64), reinterpret_cast<int32_t *>(at + 64 + most_tiles(rows, count) * sizeof(Tile))};
}

// Adds one for every lane that takes part to its bin, and gives each where it comes among them. Neighbouring rows are mostly of one request:
// lanes with the first one's bin add once together.
__device__ inline uint32_t take(uint32_t *bin, uint32_t id, bool takes) {
  const uint64_t active = __ballot(takes);
  if (active == 0) return 0;
  const int lane = threadIdx.x & 63, leader = __builtin_ctzll(active);
  const bool same = takes && id == (uint32_t)__shfl((int)id, leader);
  const uint64_t with = __ballot(same);
  uint32_t at = 0;
  if (lane == leader) at = atomicAdd(&bin[id], (uint32_t)__popcll(with));
  at = (uint32_t)__shfl((int)at, leader) + (uint32_t)__popcll(with & ((1ull << lane) - 1));
  if (takes && !same) at = atomicAdd(&bin[id], 1u);
  return at;
}

// A counting sort in one workgroup: 3.8 us for 64 rows, 8 for 8192, once a step for all of its projections. Where a row comes among those of its adapter depends on the order of atomics, and nothing else does: every
// row's result is its own column of a product.
__global__ __launch_bounds__(kGroupThreads) void ft_adapter_group_kernel(const int32_t *__restrict__ ids, uint32_t rows, uint32_t count, Groups out) {
  extern __shared__ uint32_t bin[];  // count + 1: rows, then where the next one goes
  __shared__ uint32_t part[2][kGroupThreads / 64];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (uint32_t i = tid; i <= count; i += kGroupThreads) bin[i] = 0;
  __syncthreads();
  uint32_t id[kAtOnce];  // of rows i0 + tid, i0 + kGroupThreads + tid, ..: asked for together
  const auto load = [&](uint32_t i0) {
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t i = i0 + k * kGroupThreads + tid;
      id[k] = (uint32_t)ids[i < rows ? i : rows - 1];
    }
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) id[k] = id[k] < count ? id[k] : count;
  };
  for (uint32_t i0 = 0; i0 < rows; i0 += kAtOnce * kGroupThreads) {
    load(i0);
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) take(bin, id[k], i0 + k * kGroupThreads + tid < rows);
  }
  uint32_t rows_before = 0, tiles_before = 0;
  for (uint32_t i0 = 0; i0 <= count; i0 += kGroupThreads) {
    __syncthreads();
    const uint32_t i = i0 + tid, n = i <= count ? bin[i] : 0, tiles = (n + kTileRows - 1) / kTileRows;
    uint32_t a = n, b = tiles;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t x = __shfl_up(a, d), y = __shfl_up(b, d);
      if (lane >= (uint32_t)d) {
        a += x;
        b += y;
      }
    }
    if (lane == 63) {
      part[0][wave] = a;
      part[1][wave] = b;
    }
    __syncthreads();
    uint32_t first = rows_before + a - n, tile = tiles_before + b - tiles;
    for (uint32_t w = 0; w < kGroupThreads / 64; ++w) {
      if (w < wave) {
        first += part[0][w];
        tile += part[1][w];
      }
      rows_before += part[0][w];
      tiles_before += part[1][w];
    }
    if (i <= count) {
      bin[i] = first;
      for (uint32_t k = 0; k < tiles; ++k)
        out.tiles[tile + k] = {i < count ? (int32_t)i : -1, first + k * kTileRows, n - k * kTileRows < kTileRows ? n - k * kTileRows : kTileRows, 0};
    }
  }
  __syncthreads();
  for (uint32_t i0 = 0; i0 < rows; i0 += kAtOnce * kGroupThreads) {
    if (rows > kAtOnce * kGroupThreads) load(i0);  // (else they are still there)
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t i = i0 + k * kGroupThreads + tid, at = take(bin, id[k], i < rows);
      if (i < rows) out.order[at] = (int32_t)i;
    }
  }
  if (tid == 0) *out.tiles_there = tiles_before;
}

struct Adapt {
  ft_adapters_call c;
  Groups g;
  float *h;          // splits x rows (in their order) x pitch
  uint32_t pitch;    // max_rank rounded up to 16
  uint32_t splits, split;  // of the long axis: how many, elements of one (a multiple of 256)
  uint32_t blocks;   // of 64 columns that a workgroup of the second product has
};

// 8 elements of a row from `at`, those from `end` on zero.
__device__ inline Words4 load_to(const uint16_t *row, uint32_t at, uint32_t end) {
  if (at + 8 <= end) return load16(row + at);
  Words4 w{0, 0, 0, 0};
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i)
    if (at + i < end) w[i / 2] |= (uint32_t)row[at + i] << (i % 2 * 16);
  return w;
}

// Tiles of 16 rows of X times tiles of 16 rows of A, over this wavefront's part of the long axis; 64 elements of it at a time, all of their loads
// before the first product. The tile is as small as its rows and its rank allow: products with nothing cost their loads.
template <class T, int NT, int RT>
__device__ inline void shrink(const Adapt &p, const Tile &tile, const ft_adapter_record &rec, uint32_t rank, uint32_t r0, uint32_t k0, uint32_t k1, float *lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g = lane >> 4;
  const uint16_t *x[NT], *a[RT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint32_t i = t * 16 + n16 < tile.count ? t * 16 + n16 : tile.count - 1;
    x[t] = static_cast<const uint16_t *>(p.c.x) + (uint64_t)p.g.order[tile.first + i] * p.c.x_stride;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const uint32_t r = r0 + t * 16 + n16;
    a[t] = reinterpret_cast<const uint16_t *>(rec.a) + (uint64_t)(r < rank ? r : rank - 1) * p.c.width_in;
  }
  Floats4 acc[NT][RT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < RT; ++u) acc[t][u] = Floats4{0, 0, 0, 0};
  uint32_t k = k0 + wave * 64;
  for (; k + 64 <= k1; k += 256) {
    Words4 xf[2][NT], af[2][RT];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int u = 0; u < RT; ++u) af[s][u] = load16(a[u] + k + s * 32 + 8 * g);
#pragma unroll
      for (int t = 0; t < NT; ++t) xf[s][t] = load16(x[t] + k + s * 32 + 8 * g);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int u = 0; u < RT; ++u) acc[t][u] = T::mfma(af[s][u], xf[s][t], acc[t][u]);
  }
  for (; k < k1; k += k % 64 == 32 ? 224 : 32) {  // what is left of the last 64, where a row may end anywhere
    Words4 xf[NT], af[RT];
#pragma unroll
    for (int u = 0; u < RT; ++u) af[u] = load_to(a[u], k + 8 * g, k1);
#pragma unroll
    for (int t = 0; t < NT; ++t) xf[t] = load_to(x[t], k + 8 * g, k1);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < RT; ++u) acc[t][u] = T::mfma(af[u], xf[t], acc[t][u]);
  }
  Floats4 *room = reinterpret_cast<Floats4 *>(lds);
  __syncthreads();
  if (wave != 0)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < RT; ++u) room[((wave - 1) * NT * RT + t * RT + u) * 64 + lane] = acc[t][u];
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < RT; ++u) {
      for (int w = 0; w < 3; ++w) acc[t][u] += room[(w * NT * RT + t * RT + u) * 64 + lane];
      const uint32_t r = r0 + u * 16 + 4 * g;
      if (t * 16 + n16 < tile.count && r < p.pitch)
        *reinterpret_cast<Floats4 *>(p.h + ((uint64_t)blockIdx.y * p.c.rows + tile.first + t * 16 + n16) * p.pitch + r) = acc[t][u];
    }
}

template <class T>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void ft_adapter_shrink_kernel(Adapt p) {
  __shared__ float lds[3 * 16 * 256];
  const Tile tile = p.g.tiles[blockIdx.x];  // (there is room for as many as the grid has, and not all of them are there)
  if (blockIdx.x >= *p.g.tiles_there || tile.adapter < 0) return;
  const ft_adapter_record rec = p.c.records[tile.adapter];
  const uint32_t rank = rec.rank < p.c.max_rank ? rec.rank : p.c.max_rank;
  const uint32_t k0 = blockIdx.y * p.split, k1 = k0 + p.split < p.c.width_in ? k0 + p.split : p.c.width_in;
  for (uint32_t r0 = 0; r0 < rank; r0 += 64) {
    if (tile.count <= 16) {
      if (rank - r0 <= 16) shrink<T, 1, 1>(p, tile, rec, rank, r0, k0, k1, lds);
      else if (rank - r0 <= 32) shrink<T, 1, 2>(p, tile, rec, rank, r0, k0, k1, lds);
      else shrink<T, 1, 4>(p, tile, rec, rank, r0, k0, k1, lds);
    } else {
      if (rank - r0 <= 16) shrink<T, 4, 1>(p, tile, rec, rank, r0, k0, k1, lds);
      else if (rank - r0 <= 32) shrink<T, 4, 2>(p, tile, rec, rank, r0, k0, k1, lds);
      else shrink<T, 4, 4>(p, tile, rec, rank, r0, k0, k1, lds);
    }
  }
}

template <class T>
__device__ inline void add_up(const Adapt &p, const Tile &tile, const ft_adapter_record &rec, uint32_t rank, uint16_t *halves, uint32_t row_pitch, float *size) {
  // The parts of a row of H added up, 16 lanes to a row. Each is brought to between 1 and 2 by a power of two that multiplies the result, so that
  // the range of 16 bits neither cuts large ones off nor takes digits from small ones. The high part is cut off, so that the low one has its sign, and
  // is never zero beside it: an infinity of B has to meet two numbers of one sign, or would be NaN. (16 bits of a value, 22 in float16.)
  const uint32_t rows16 = (tile.count + 15) / 16 * 16;
  for (uint32_t i = threadIdx.x >> 4; i < rows16; i += 16) {
    const uint32_t q = threadIdx.x & 15, from = tile.first + (i < tile.count ? i : tile.count - 1);
    Floats4 v[4];  // elements 64 k + 4 q .. + 3
    float most = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = Floats4{0, 0, 0, 0};
      const uint32_t r = 64 * k + 4 * q;
      if (64 * k >= (int)rank) continue;
      const float *part = p.h + (uint64_t)from * p.pitch + (r < p.pitch ? r : 0);
#pragma unroll 8
      for (uint32_t s = 0; s < p.splits; ++s) v[k] += *reinterpret_cast<const Floats4 *>(part + (uint64_t)s * p.c.rows * p.pitch);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (r + x >= rank) v[k][x] = 0;
        most = fmaxf(most, fabsf(v[k][x]));
      }
    }
    for (int d = 1; d < 16; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    int e = (int)(__float_as_uint(most) >> 23) - 127;
    if (most == 0 || e > 126) e = 0;
    e = e < -120 ? -120 : e;
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    if (q == 0) size[i] = __uint_as_float((uint32_t)(127 + e) << 23) * rec.scale;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t r = 64 * k + 4 * q;
      if (r >= row_pitch) continue;
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int x = 0; x < 4; x += 2) {
        const float a = v[k][x] * down, b = v[k][x + 1] * down;
        hi[x / 2] = T::pack_cut(a, b);
        const float ra = a - T::to_float((uint16_t)hi[x / 2]), rb = b - T::to_float((uint16_t)(hi[x / 2] >> 16));
        lo[x / 2] = T::pack(fabsf(a) == INFINITY ? 0 : ra, fabsf(b) == INFINITY ? 0 : rb);
        if ((lo[x / 2] & 0x7fff) == 0 && a != 0) lo[x / 2] |= (hi[x / 2] & 0x8000) | T::kTiny;
        if ((lo[x / 2] & 0x7fff0000) == 0 && b != 0) lo[x / 2] |= (hi[x / 2] & 0x80000000) | (uint32_t)T::kTiny << 16;
      }
      typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
      *reinterpret_cast<Words2 *>(&halves[i * row_pitch + r]) = Words2{hi[0], hi[1]};
      *reinterpret_cast<Words2 *>(&halves[(kTileRows + i) * row_pitch + r]) = Words2{lo[0], lo[1]};
    }
  }
}

// Two neighbouring lanes have two vectors each of their own row, or one each of both: from the one to the other, either way.
__device__ inline void exchange(Words4 (&v)[2], uint32_t odd) {
  Words4 there;
#pragma unroll
  for (int y = 0; y < 4; ++y) there[y] = (uint32_t)__builtin_amdgcn_mov_dpp((int)(odd ? v[0][y] : v[1][y]), 0xb1, 0xf, 0xf, true);
  v[0] = odd ? there : v[0];
  v[1] = odd ? v[1] : there;
}

// 64 columns of a tile's rows. Columns are dealt to the products so that a lane's 16 results, acc[j][i], are two groups of 8 neighbours: columns
// 8 g + 4 (i % 2) + j of the first 32 (i < 2) and of the second. A block's part of base is asked for before the products of the block ahead of it, but
// is waited for there too: its loads lie in branches, which the compiler does not count past, so that base's and B's time in memory add up. What
// lanes read and write is whole lines of 128 bytes of every other row, and is exchanged with the neighbour's: 3.5 us less for 8192 rows.
template <class T, int NT>
__device__ inline void expand(const Adapt &p, const Tile &tile, const ft_adapter_record &rec, uint32_t rank, uint16_t *high, uint32_t row_pitch, float *size) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g = lane >> 4;
  const uint16_t *low = high + kTileRows * row_pitch;
  const uint32_t end = p.c.width_out, first_block = blockIdx.y * p.blocks;
  const uint32_t odd = n16 & 1, pair = n16 & ~1u;
  uint64_t row[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (uint32_t x = 0; x < 2; ++x) row[t][x] = (uint64_t)p.g.order[tile.first + (t * 16 + pair + x < tile.count ? t * 16 + pair + x : tile.count - 1)];
  const uint32_t last_block = first_block + p.blocks < (end + 63) / 64 ? first_block + p.blocks : (end + 63) / 64;
  const auto load_base = [&](uint32_t block, Words4 (&into)[NT][2]) {
    const uint32_t at = block * 64 + 8 * g + 32 * odd;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint16_t *b = static_cast<const uint16_t *>(p.c.base) + row[t][x] * p.c.base_stride;
        into[t][x] = block * 64 + 64 <= end ? load16(b + at) : load_to(b, at, end);
      }
  };
  Words4 base[NT][2] = {}, next[NT][2] = {};
  if (p.c.base != nullptr && first_block + wave < last_block) load_base(first_block + wave, base);
  add_up<T>(p, tile, rec, rank, high, row_pitch, size);
  __syncthreads();
  for (uint32_t block = first_block + wave; block < last_block; block += 4) {
    const uint32_t n0 = block * 64;
    const bool whole = n0 + 64 <= end;
    if (p.c.base != nullptr && block + 4 < last_block) load_base(block + 4, next);
    Floats4 acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[t][j] = Floats4{0, 0, 0, 0};
    for (uint32_t r = 0; r < rank; r += 32) {
      Words4 b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t n = n0 + (n16 >> 1 & 1) * 32 + (n16 >> 2) * 8 + (n16 & 1) * 4 + j, k = r + 8 * g;
        const uint16_t *row_of_b = reinterpret_cast<const uint16_t *>(rec.b) + (uint64_t)(n < end ? n : end - 1) * rec.rank;
        if (rank % 8 == 0) {
          b[j] = Words4{0, 0, 0, 0};
          if (k < rank) b[j] = load16(row_of_b + k);
        } else {
          b[j] = load_to(row_of_b, k, rank);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t at = (t * 16 + n16) * row_pitch + r + 8 * g;
        const Words4 hi = *reinterpret_cast<const Words4 *>(high + at), lo = *reinterpret_cast<const Words4 *>(low + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[t][j] = T::mfma(b[j], lo, acc[t][j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[t][j] = T::mfma(b[j], hi, acc[t][j]);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float by = size[t * 16 + n16];
      exchange(base[t], odd);
      Words4 w[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {  // elements 2 y and 2 y + 1 of 8: i = 2 x + y / 2, j = 2 (y % 2) and the next
          const uint32_t two = base[t][x][y];
          const float lo = T::to_float((uint16_t)two), hi = T::to_float((uint16_t)(two >> 16));
          w[x][y] = T::pack(__builtin_fmaf(acc[t][y % 2 * 2][2 * x + y / 2], by, lo), __builtin_fmaf(acc[t][y % 2 * 2 + 1][2 * x + y / 2], by, hi));
        }
      exchange(w, odd);
#pragma unroll
      for (uint32_t x = 0; x < 2; ++x) {
        if (t * 16 + pair + x >= tile.count) continue;
        const uint32_t n = n0 + 8 * g + 32 * odd;
        uint16_t *out = static_cast<uint16_t *>(p.c.out) + row[t][x] * p.c.out_stride + n;
        if (whole) {
          *reinterpret_cast<Loose4 *>(out) = Loose4{{w[x][0], w[x][1], w[x][2], w[x][3]}};
        } else {
#pragma unroll
          for (uint32_t i = 0; i < 8; ++i)
            if (n + i < end) out[i] = (uint16_t)(w[x][i / 2] >> (i % 2 * 16));
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) base[t][x] = next[t][x];
  }
}

template <class T>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void ft_adapter_expand_kernel(Adapt p) {
  extern __shared__ uint16_t halves[];  // 64 rows x (rank rounded up to 32, and 8): the high parts, then the low ones
  __shared__ float size[kTileRows];
  const Tile tile = p.g.tiles[blockIdx.x];
  if (blockIdx.x >= *p.g.tiles_there) return;
  if (tile.adapter < 0) {
    // rows without an adapter: base as it is, or zero
    if (p.c.out == p.c.base && p.c.out_stride == p.c.base_stride) return;
    const uint32_t first = blockIdx.y * p.blocks * 64, end = first + p.blocks * 64 < p.c.width_out ? first + p.blocks * 64 : p.c.width_out;
    for (uint32_t i = threadIdx.x >> 6; i < tile.count; i += 4) {
      const uint64_t row = (uint64_t)p.g.order[tile.first + i];
      const uint16_t *from = static_cast<const uint16_t *>(p.c.base) + row * p.c.base_stride;
      uint16_t *to = static_cast<uint16_t *>(p.c.out) + row * p.c.out_stride;
      for (uint32_t n = first + (threadIdx.x & 63) * 8; n < end; n += 512) {
        const Words4 w = p.c.base == nullptr ? Words4{0, 0, 0, 0} : load_to(from, n, end);
        if (n + 8 <= end) *reinterpret_cast<Loose4 *>(to + n) = Loose4{{w[0], w[1], w[2], w[3]}};
        else
          for (uint32_t k = 0; n + k < end; ++k) to[n + k] = (uint16_t)(w[k / 2] >> (k % 2 * 16));
      }
    }
    return;
  }
  const ft_adapter_record rec = p.c.records[tile.adapter];
  const uint32_t rank = rec.rank < p.c.max_rank ? rec.rank : p.c.max_rank, row_pitch = (rank + 31) / 32 * 32 + 8;
  if (tile.count <= 16) expand<T, 1>(p, tile, rec, rank, halves, row_pitch, size);
  else expand<T, 4>(p, tile, rec, rank, halves, row_pitch, size);
}

uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// Workgroups that keep the chip busy; the long axis is split until there are as many, into pieces of 256 elements and more. (Eight splits cost 8192
// rows 20 us, whose parts have to be written and added up; half as many workgroups do as well there.)
constexpr uint64_t kEnough = 512;

void split_of(const ft_adapters_call &c, uint32_t *splits, uint32_t *split) {
  const uint64_t tiles = most_tiles(c.rows, c.count), most = (c.width_in + 255) / 256;
  uint64_t n = (kEnough + tiles - 1) / tiles;
  n = n > most ? most : n;
  *split = (uint32_t)up((c.width_in + n - 1) / n, 256);
  *splits = (c.width_in + *split - 1) / *split;
}

}  // namespace

uint64_t adapter_tiles(uint32_t rows, uint32_t count) { return most_tiles(rows, count); }

uint64_t adapter_group_bytes(uint32_t rows, uint32_t count) { return 64 + up(most_tiles(rows, count) * sizeof(Tile) + (uint64_t)rows * 4, 16); }

hipError_t launch_adapter_group(const int32_t *ids, uint32_t rows, uint32_t count, void *groups, hipStream_t stream) {
  hipLaunchKernelGGL(ft_adapter_group_kernel, dim3(1), dim3(kGroupThreads), (count + 1) * 4, stream, ids, rows, count, groups_at(groups, rows, count));
  return hipGetLastError();
}

uint64_t adapter_workspace(const ft_adapters_call &c) {
  uint32_t splits, split;
  split_of(c, &splits, &split);
  return (uint64_t)splits * c.rows * up(c.max_rank, 16) * 4;
}

template <class T>
hipError_t launch(const Adapt &p, hipStream_t stream) {
  const uint32_t tiles = (uint32_t)most_tiles(p.c.rows, p.c.count), blocks = (p.c.width_out + 63) / 64;
  hipLaunchKernelGGL(ft_adapter_shrink_kernel<T>, dim3(tiles, p.splits), dim3(256), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(ft_adapter_expand_kernel<T>, dim3(tiles, (blocks + p.blocks - 1) / p.blocks), dim3(256), kTileRows * (up(p.c.max_rank, 32) + 8) * 4, stream, p);
  return hipGetLastError();
}

hipError_t launch_adapters(const ft_adapters_call &call, hipStream_t stream) {
  Adapt p{call};
  p.g = groups_at(const_cast<void *>(call.groups), call.rows, call.count);
  p.h = static_cast<float *>(call.workspace);
  p.pitch = (uint32_t)up(call.max_rank, 16);
  split_of(call, &p.splits, &p.split);
  // A workgroup's four wavefronts take a block at least each, and no more where that is two rounds of kEnough workgroups at most (64 rows of 33 tiles:
  // 17.6 us, with 8 blocks 20.5). Beyond that each has H to add up before its blocks, which costs about what four blocks do, and the last round may
  // be all but empty (8192 rows of 6144 columns: 117 us with 8 blocks, 111 with 12, 107 with 16, 114 with 24).
  const uint64_t blocks = (call.width_out + 63) / 64, tiles = most_tiles(call.rows, call.count);
  const uint32_t most = tiles * ((blocks + 3) / 4) <= 2 * kEnough ? 4 : 16;
  uint64_t least = ~0ull;
  for (uint32_t n = 4; n <= most; n += 4) {
    const uint64_t cost = (tiles * ((blocks + n - 1) / n) + kEnough - 1) / kEnough * (n + 4);
    if (cost < least) {
      least = cost;
      p.blocks = n;
    }
  }
  return call.type == FT_BF16 ? launch<Bf16>(p, stream) : launch<Fp16>(p, stream);
}

}  // namespace ft
