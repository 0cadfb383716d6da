// Products of few rows with weights of 4 bits and group scales, read as they lie in the pool.
//
// The matrix instruction multiplies 16 rows of x with 16 rows of weights, 32 elements at a time. A code becomes a number of 16 bits by two
// instructions for two codes: put into the low places of a number's mantissa it is that number plus the code, 128 + code in bfloat16, 64 + code in float16,
// exactly. What is too much is taken away behind the products, for a group of elements at once, with the zero:
//   sum of x (code - zero) = sum of x (128 + code) - (128 + zero) sum of x,
// where the sums of x are a product with ones. So nothing is rounded but sums, in 32 bits, and the scale is applied to their difference (to each of them it
// may be too much for 32 bits where a weight is not). An infinite or NaN
// element of x makes its row of the result NaN or infinite, as does a scale its column.
//
// Every weight is read once for 16, 32 or 64 rows of x, by the kernel that the rule in ft_linear4_plan.h takes, or for 8 by the plain one. Up to 16 rows the codes'
// way from memory is the bound: 8192 to 32768 takes 32 us with one row (4.4 TB/s of the 5.2 that a long read reaches) and 38 with 16 (3.7); with 64 rows, 65 us,
// it is what a wavefront does with a code - one of two instructions, one of 32 in products and sums - beside loads that only half overlap with it: without
// the products the same kernel takes 40 us, without the loads 52, without putting them down either 43 to 46. Small
// projections are bound by a launch and by one way to memory behind which come products, sums and the way back: 5.2 us for one row of 4096 to 4096.
#include <hip/hip_runtime.h>

#include "ft_linear4_plan.h"
#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

constexpr uint32_t kBlock = 128;   // elements of a row that four instructions multiply

// 16 bytes at any address
struct __attribute__((packed, aligned(1))) Bytes16 {
  uint32_t w[4];
};
__device__ inline Words4 load_codes(const uint8_t *p) {
  typedef const __attribute__((address_space(1))) Bytes16 *P;
  const P q = (P)global(p);
  return Words4{q->w[0], q->w[1], q->w[2], q->w[3]};
}
// 16 bytes without the first `bytes`, and zeros behind
__device__ inline Words4 without(Words4 v, uint32_t bytes) {
  uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
  if (bytes >= 8) {
    lo = hi;
    hi = 0;
  }
  if (bytes >= 16) lo = 0;
  const uint32_t by = 8 * (bytes % 8);
  lo = lo >> by | hi << 1 << (63 - by);
  hi >>= by;
  return Words4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// Bytes [at, at + 16) of `size`, 16 or more, from p: zeros behind the last one, and nothing read there.
__device__ inline Words4 load_upto(const void *p, uint64_t at, uint64_t size) {
  const uint64_t from = at + 16 <= size ? at : size - 16;
  return without(load_codes(static_cast<const uint8_t *>(p) + from), at - from < 16 ? (uint32_t)(at - from) : 16);
}

// Eight codes as numbers, in the order 0, 4, 1, 5, 2, 6, 3, 7.
template <class T>
struct Code;
template <>
struct Code<Bf16> {
  static constexpr float kMore = 128;
  static constexpr uint32_t kOnes = 0x3f803f80;
  static constexpr uint32_t kMask = 0x000f000f, kExponent = 0x43004300;
  // (the exponents come in a register: one instruction does not take two constants)
  static __device__ Words4 numbers(uint32_t w, uint32_t more) {
    return Words4{(w & kMask) | more, ((w >> 4) & kMask) | more, ((w >> 8) & kMask) | more, ((w >> 12) & kMask) | more};
  }
};
template <>
struct Code<Fp16> {
  static constexpr float kMore = 64;
  static constexpr uint32_t kOnes = 0x3c003c00;
  static constexpr uint32_t kMask = 0x00f000f0, kExponent = 0x54005400;
  static __device__ Words4 numbers(uint32_t w, uint32_t more) {
    return Words4{((w << 4) & kMask) | more, (w & kMask) | more, ((w >> 4) & kMask) | more, ((w >> 8) & kMask) | more};
  }
};

// Eight elements of x in the order of the codes.
__device__ inline Words4 in_order(Words4 v) {
  constexpr uint32_t low = 0x05040100, high = 0x07060302;
  return Words4{__builtin_amdgcn_perm(v[2], v[0], low), __builtin_amdgcn_perm(v[2], v[0], high), __builtin_amdgcn_perm(v[3], v[1], low),
                __builtin_amdgcn_perm(v[3], v[1], high)};
}

// Four lanes that are 16 apart hold four words each, as rows of a matrix: turned, lane g has word g of each.
__device__ inline Words4 turned(Words4 v) {
  typedef uint32_t Two __attribute__((ext_vector_type(2)));
  const Two a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false), b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
  const Two c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  return Words4{c[0], c[1], d[0], d[1]};
}

// What a wavefront does with a block of 128 elements of 16 rows of weights: `codes` is a lane's 32 of them - row l % 16, elements 32 (l / 16) to + 31 -,
// x(tile, step) its eight elements of 16 rows of x for one of four instructions, element(step). SG: groups that a block has exactly, 0: any, of 32
// elements or more. SG = 1: an instruction multiplies 8 of every 32 elements; otherwise neighbours, and the lanes exchange codes for it.
template <int SG>
__device__ inline uint32_t element(int g, int step) { return SG == 1 ? 32 * g + 8 * step : 32 * step + 8 * g; }

// NT tiles of 16 rows of weights and TT of x; scale(tile, group), zero(tile, group): of the lane's row of weights.
template <class T, int SG, int NT, int TT, class X, class Scale, class Zero>
__device__ inline void multiply(const Linear4View &w, Words4 (&codes)[NT], uint32_t k0, int g, const X &x, const Scale &scale, const Zero &zero,
                                Floats4 (&acc)[NT][TT]) {
  const Words4 ones{Code<T>::kOnes, Code<T>::kOnes, Code<T>::kOnes, Code<T>::kOnes};
  const Floats4 nothing{0, 0, 0, 0};
  uint32_t exponent = Code<T>::kExponent;
  asm volatile("" : "+v"(exponent));
  Floats4 products[NT][TT], sums[TT];
  const auto add = [&](const float (&by)[NT], const float (&more)[NT]) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][tt][j] = __builtin_fmaf(by[i], __builtin_fmaf(more[i], sums[tt][j], products[i][tt][j]), acc[i][tt][j]);
    }
  };
  const auto factors = [&](uint32_t group, float (&by)[NT], float (&more)[NT]) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      by[i] = scale(i, group);
      more[i] = -(Code<T>::kMore + zero(i, group));
    }
  };
  constexpr int G = SG == 0 ? 1 : SG;
  float by[G][NT], more[G][NT];
  if (SG != 0)
#pragma unroll
    for (int j = 0; j < G; ++j) factors(w.group.of(k0 + 128 / G * j), by[j], more[j]);
  if (SG != 1)
#pragma unroll
    for (int i = 0; i < NT; ++i) codes[i] = turned(codes[i]);
  constexpr int each = SG == 0 ? 1 : 4 / (SG == 0 ? 1 : SG);  // instructions to a group
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const uint32_t k = k0 + 32 * s;
    Words4 a[TT], b[NT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) a[tt] = x(tt, s);
#pragma unroll
    for (int i = 0; i < NT; ++i) b[i] = Code<T>::numbers(codes[i][s], exponent);
    if (SG != 0) {
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) {
        sums[tt] = T::mfma(a[tt], ones, s % each == 0 ? nothing : sums[tt]);
#pragma unroll
        for (int i = 0; i < NT; ++i) products[i][tt] = T::mfma(a[tt], b[i], s % each == 0 ? nothing : products[i][tt]);
      }
      if ((s + 1) % each == 0) add(by[s / each % G], more[s / each % G]);
    } else {
      // a lane's eight elements are in one group, and 32 in two at most
      const uint32_t first = w.group.of(k), last = w.group.of(k + 31);
      const bool mine = w.group.of(k + 8 * g) == first;
      float by0[NT], more0[NT];
      factors(first, by0, more0);
      if (TT == 4) {  // (one after the other, with the same code: registers do not hold both)
#pragma unroll 1
        for (int part = 0; part < (first == last ? 1 : 2); ++part) {
#pragma unroll
          for (int tt = 0; tt < TT; ++tt) {
            Words4 some;
#pragma unroll
            for (int i = 0; i < 4; ++i) some[i] = mine == (part == 0) ? a[tt][i] : 0;
            sums[tt] = T::mfma(some, ones, nothing);
#pragma unroll
            for (int i = 0; i < NT; ++i) products[i][tt] = T::mfma(some, b[i], nothing);
          }
          if (part == 1) factors(last, by0, more0);
          add(by0, more0);
        }
        continue;
      }
      if (first != last) {
        float by1[NT], more1[NT];
        factors(last, by1, more1);
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) {
          Words4 some;
#pragma unroll
          for (int i = 0; i < 4; ++i) some[i] = mine ? 0 : a[tt][i];
          sums[tt] = T::mfma(some, ones, nothing);
#pragma unroll
          for (int i = 0; i < NT; ++i) products[i][tt] = T::mfma(some, b[i], nothing);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[tt][i] = mine ? a[tt][i] : 0;
        }
        add(by1, more1);
      }
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) {
        sums[tt] = T::mfma(a[tt], ones, nothing);
#pragma unroll
        for (int i = 0; i < NT; ++i) products[i][tt] = T::mfma(a[tt], b[i], nothing);
      }
      add(by0, more0);
    }
  }
}

// An offset that stays 32 bits: widened ahead of a loop it would take two registers in it, and an addition for each load.
__device__ inline uint32_t here32(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

// A barrier for shared memory alone: loads from global memory stay on their way.
__device__ inline void fence() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Strides of a workgroup's scales and zeros in shared memory, in bytes: an odd number of words, so that 16 rows lie in different banks.
__host__ __device__ inline uint32_t scale_stride(uint32_t groups) { return 4 * ((groups + 1) / 2 | 1); }
__host__ __device__ inline uint32_t zero_stride(uint32_t groups) { return 4 * ((groups + 3) / 4 | 1); }

// Scales or zeros, `size` bytes each, of rows n0 to n0 + ROWS - 1, groups g0 to g0 + groups - 1, to shared memory: a thread asks for 16 bytes, and puts
// them down when others are on their way; then the rest. (All rows' scales together are 16 bytes at least, and so are their zeros.)
template <int ROWS, int THREADS>
struct Scales {
  const char *from;
  uint32_t size, pieces, stride, n0, g0;
  uint64_t all;
  Words4 first;

  __device__ Scales(const Linear4View &w, const void *at, uint32_t size, uint32_t n0, uint32_t g0, uint32_t groups, uint32_t stride)
      : from(static_cast<const char *>(at)), size(size), pieces((groups * size + 15) / 16), stride(stride), n0(n0), g0(g0),
        all((uint64_t)w.width_out * w.groups * size) {
    first = piece(w, threadIdx.x < ROWS * pieces ? threadIdx.x : 0);
  }
  __device__ Words4 piece(const Linear4View &w, uint32_t i) const {
    const uint32_t r = i / pieces, j = i - r * pieces, n = n0 + r < w.width_out ? n0 + r : w.width_out - 1;
    return load_upto(from, ((uint64_t)n * w.groups + g0) * size + 16 * j, all);
  }
  __device__ void put(char *to, uint32_t i, Words4 v) const {
    const uint32_t r = i / pieces, j = i - r * pieces;
    uint32_t *out = reinterpret_cast<uint32_t *>(to + r * stride + 16 * j);
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
      if (16 * j + 4 * k < stride) out[k] = v[k];
  }
  __device__ void bring(const Linear4View &w, char *to) const {
    if (threadIdx.x < ROWS * pieces) put(to, threadIdx.x, first);
    for (uint32_t i = threadIdx.x + THREADS; i < ROWS * pieces; i += THREADS) put(to, i, piece(w, i));
  }
};

// Eight neighbouring elements of a row of the result, or `there` of them, from 32 bits, base added.
template <class T>
__device__ inline void write8(const ft_linear4_call &c, uint32_t row, uint32_t n, uint32_t there, const float *sums) {
  uint16_t *out = static_cast<uint16_t *>(c.out) + row * c.out_stride + n;
  const uint16_t *base = static_cast<const uint16_t *>(c.base) + row * c.base_stride + n;
  if (there >= 8) {
    Words4 b{0, 0, 0, 0};
    if (c.base != nullptr) b = load16(base);
    Loose4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v.w[i] = T::pack(sums[2 * i] + T::to_float((uint16_t)b[i]), sums[2 * i + 1] + T::to_float((uint16_t)(b[i] >> 16)));
    *reinterpret_cast<Loose4 *>(out) = v;
  } else {
    for (uint32_t i = 0; i < there; ++i) out[i] = T::from_float(sums[i] + (c.base != nullptr ? T::to_float(base[i]) : 0));
  }
}

// 16 rows of weights to a workgroup, and 16 rows of x, 2 XL of which there are. Its wavefronts have every KW-th 256 elements and add up what they
// have at the end. A wavefront brings what it multiplies by itself, neighbouring lanes neighbouring pieces - 128 bytes of eight rows of weights to an
// instruction; as the matrix instruction has them, four pieces of 16 bytes from each of 16 rows, the loads are bound by their addresses -, and turns it
// round in shared memory of its own, without a barrier. There are 16 rows to a workgroup, not more, so that small projections have workgroups for all
// compute units: 256 of eight wavefronts for 4096 rows. All loads up to the first product leave together: 16 rows of 4096 to 4096 take 6.3 us, one 5.2.
template <class T, int SG, int XL, int KW>
__global__ __launch_bounds__(64 * KW) __attribute__((amdgpu_waves_per_eu(XL != 1 ? 4 : SG != 0 ? 6 : 5))) void ft_linear4_narrow_kernel(Linear4View w,
                                                                                                                                   ft_linear4_call c) {
  constexpr int R = 2 * XL, kDepth = XL == 1 ? 2 : 1;  // (pieces on their way; of 8 rows with two: 4096 to 14336 15.5 us instead of 14.0)
  __shared__ Words4 codes_lds[KW][16 * 8], x_lds[KW][R * 32];
  __shared__ float parts[KW][4][64];
  extern __shared__ __attribute__((aligned(16))) char scales_lds[];
  char *zeros_lds = scales_lds + 16 * scale_stride(w.groups);
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, col = lane % 16;
  const uint32_t n0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  // where this lane's pieces come from, in bytes behind the workgroup's first rows, and where they go
  const uint8_t *weights = w.weights + (uint64_t)n0 * w.row_bytes;
  const char *rows = reinterpret_cast<const char *>(static_cast<const uint16_t *>(c.x) + t0 * c.x_stride);
  uint32_t from[2], to[2], x_from[XL], x_to[XL];
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i) {
    const uint32_t r = 8 * i + lane / 8;
    from[i] = (n0 + r < w.width_out ? r : w.width_out - 1 - n0) * w.row_bytes + 16 * (lane % 8);
    to[i] = r * 8 + (lane % 8 ^ r >> 1);
  }
#pragma unroll
  for (uint32_t i = 0; i < XL; ++i) {
    const uint32_t r = 2 * i + lane / 32;
    x_from[i] = (t0 + r < c.rows ? r : c.rows - 1 - t0) * (2 * (uint32_t)c.x_stride) + 16 * (lane % 32);
    x_to[i] = r * 32 + (lane % 32 ^ r);
  }
  const uint32_t pieces = w.width_in / 256, all = (w.width_in + 255) / 256;
  // of the result a thread has one element at most
  const uint32_t row = t0 + 4 * (lane / 16) + wave % 4, n = n0 + col;
  const bool mine = wave < 4 && row < c.rows && n < w.width_out;
  const bool based = mine && c.base != nullptr;
  const uint16_t base = *(based ? static_cast<const uint16_t *>(c.base) + row * c.base_stride + n : w.scales);  // (in any case: a branch would wait for it)
  __builtin_amdgcn_sched_barrier(0);
  const Scales<16, 64 * KW> scales(w, w.scales, 2, n0, 0, w.groups, scale_stride(w.groups));
  const Scales<16, 64 * KW> zeros(w, w.zeros != nullptr ? static_cast<const void *>(w.zeros) : w.scales, 1, n0, 0, w.groups, zero_stride(w.groups));
  Words4 codes[kDepth][2], x[kDepth][XL];
  const auto load = [&](Words4 (&to_codes)[2], Words4 (&to_x)[XL], uint32_t piece, uint32_t some = ~0u) {
    const uint8_t *codes_at = weights + 128 * piece;
    const char *x_at = rows + 512 * piece;
#pragma unroll
    for (int i = 0; i < 2; ++i) to_codes[i] = load_codes(codes_at + here32(from[i] & some));
#pragma unroll
    for (int i = 0; i < XL; ++i) to_x[i] = load16(x_at + here32(x_from[i] & some));
  };
  // (in any case, whether this wavefront has a piece or not: behind loads that are on their way in one case only, all would be waited for)
#pragma unroll
  for (int i = 0; i < kDepth; ++i) {
    load(codes[i], x[i], (wave + i * KW < pieces ? wave + i * KW : pieces - 1) & (pieces != 0 ? ~0u : 0), pieces != 0 ? ~0u : 0);
    __builtin_amdgcn_sched_barrier(0);  // (asked for in another order they would have to be waited for together)
  }
  scales.bring(w, scales_lds);
  if (w.zeros != nullptr) zeros.bring(w, zeros_lds);
  __syncthreads();
  Floats4 acc[1][1] = {{Floats4{0, 0, 0, 0}}};
  // (of elements behind a row's last, which are zeros, the last group's)
  const auto there = [&](uint32_t group) { return group < w.groups ? group : w.groups - 1; };
  const auto scale = [&](int, uint32_t group) { return T::to_float(*reinterpret_cast<const uint16_t *>(scales_lds + col * scale_stride(w.groups) + 2 * there(group))); };
  const auto zero = [&](int, uint32_t group) { return w.zeros == nullptr ? 8.0f : (float)(uint8_t)zeros_lds[col * zero_stride(w.groups) + there(group)]; };
  const auto put = [&](const Words4 (&my_codes)[2], const Words4 (&my_x)[XL]) {
    wave_fence();  // other lanes have read what was there
#pragma unroll
    for (int i = 0; i < 2; ++i) codes_lds[wave][to[i]] = my_codes[i];
#pragma unroll
    for (int i = 0; i < XL; ++i) x_lds[wave][x_to[i]] = in_order(my_x[i]);
    wave_fence();
  };
  const auto use = [&](uint32_t piece) {
    const uint32_t x_row = col & (R - 1);
#pragma unroll
    for (uint32_t block = 0; block < 2; ++block) {
      const uint32_t k0 = 256 * piece + kBlock * block;
      if (k0 >= w.width_in) break;
      Words4 mine[1] = {codes_lds[wave][col * 8 + (4 * block + g ^ col >> 1)]};
      multiply<T, SG, 1, 1>(w, mine, k0, g, [&](int, int s) { return x_lds[wave][x_row * 32 + (16 * block + element<SG>(g, s) / 8 ^ x_row)]; }, scale, zero, acc);
    }
  };
  for (uint32_t p = wave; p < pieces; p += kDepth * KW) {
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      if (p + i * KW < pieces) {
        put(codes[i], x[i]);
        use(p + i * KW);
      }
      const uint32_t next = p + (i + kDepth) * KW;
      load(codes[i], x[i], next < pieces ? next : pieces - 1);
    }
  }
  if (pieces < all && wave == pieces % KW) {
#pragma unroll
    for (int i = 0; i < 2; ++i) codes[0][i] = load_upto(weights + (from[i] - 16 * (lane % 8)), 128 * pieces + 16 * (lane % 8), w.row_bytes);
#pragma unroll
    for (int i = 0; i < XL; ++i) x[0][i] = load_upto(rows + (x_from[i] - 16 * (lane % 32)), 512 * pieces + 16 * (lane % 32), 2 * w.width_in);
    put(codes[0], x[0]);
    use(pieces);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) parts[wave][j][lane] = acc[0][0][j];
  __syncthreads();
  static_assert(KW >= 4);
  if (!mine) return;
  float sum = 0;
#pragma unroll
  for (int k = 0; k < KW; ++k) sum += parts[k][wave][lane];
  static_cast<uint16_t *>(c.out)[row * c.out_stride + n] = T::from_float(sum + (based ? T::to_float(base) : 0));
}

// 32 NW rows of weights to a workgroup - 32 to a wavefront, and two wavefronts take turns along the rows -, and 16 TT rows of x, which all wavefronts
// multiply and bring to shared memory together, 256 elements at a time, the next ones while these are multiplied. A row of x is read by as many
// workgroups as there are tiles along the weights: with 128 rows of weights and 64 of x that is 32 KB beside 16 KB of codes for every 256 elements, out
// of the second-level cache. Registers, about 240, allow two wavefronts to a SIMD; what they leave alone waits for each other at the one barrier
// of a chunk, and what they do adds up: of 65 us for 64 rows of 8192 to 32768, 44 are products, 8 putting down and 13 loads, 4000 cycles a chunk of which
// matrix instructions have 1536 and others 1160. Not faster, all within 2 us of it: sums of x by one wavefront for all, what the zeros take off by one
// more product at the end (a fifth fewer instructions), products of one tile of x while those of the one before are scaled, reads of shared
// memory a step ahead, half of the wavefronts putting down before they multiply and half behind, one chunk on its way instead of two, pieces of 128
// bytes of a row to an instruction, chunks in another order for every workgroup.
struct Wide {
  Linear4View w;
  ft_linear4_call c;
  uint32_t each;   // chunks of 256 elements to a workgroup
  float *partial;  // where several have parts of the same sums
};

template <class T, int SG, int TT, int NW>
__global__ __launch_bounds__(128 * NW) __attribute__((amdgpu_waves_per_eu(2))) void ft_linear4_wide_kernel(Wide given) {
  const Linear4View &w = given.w;
  const uint32_t each = given.each;
  constexpr uint32_t NT = 2, kGroups = 66, kRows = 32 * NW, XP = TT * 4 / NW;
  constexpr uint32_t kDepth = TT == 4 && SG == 2 ? 1 : 2;  // (chunks that are on their way: what registers hold)
  __shared__ Words4 x_lds[2][TT * 16 * 32], codes_lds[2 * NW][NT][16 * 4];
  __shared__ __attribute__((aligned(16))) char scales_lds[kRows * 4 * (kGroups / 2 | 1)], zeros_lds[kRows * 4 * (kGroups / 4 | 1)];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, col = lane % 16;
  const uint32_t kw = wave / NW, nw = wave % NW, n0 = blockIdx.x * kRows, t0 = blockIdx.y * (16 * TT);
  // offsets in bytes from the workgroup's first row: of 128 rows of weights less than 2^30, of 64 rows of x less than 2^31
  const uint8_t *weights = w.weights + (uint64_t)n0 * w.row_bytes;
  const char *rows = reinterpret_cast<const char *>(static_cast<const uint16_t *>(given.c.x) + t0 * given.c.x_stride);
  uint32_t from[NT], x_from[XP], x_to[XP];
  const uint32_t piece = 64 * kw + 16 * (lane % 4), x_piece = 16 * (threadIdx.x % 32);
#pragma unroll
  for (uint32_t i = 0; i < NT; ++i) {
    const uint32_t r = 32 * nw + 16 * i + lane / 4;
    from[i] = (n0 + r < w.width_out ? r : w.width_out - 1 - n0) * w.row_bytes + piece;
  }
  const uint32_t to = lane / 4 * 4 + (lane % 4 ^ lane / 16);
#pragma unroll
  for (uint32_t i = 0; i < XP; ++i) {
    const uint32_t r = 4 * NW * i + threadIdx.x / 32;
    x_from[i] = (t0 + r < given.c.rows ? r : given.c.rows - 1 - t0) * (2 * (uint32_t)given.c.x_stride) + x_piece;
    x_to[i] = r * 32 + (threadIdx.x % 32 ^ r % 16);
  }
  const uint32_t whole = w.width_in / 256;  // and a part
  struct Chunk {
    Words4 codes[NT], x[XP];
  };
  // (`all`: 0 where there is no whole chunk, and what is read is not used)
  const auto load = [&](Chunk &f, uint32_t chunk, uint32_t end, uint32_t all = ~0u) {
    if (chunk >= end) chunk = (end - 1) & all;
    const uint8_t *codes_at = weights + 128 * chunk;
    const char *x_at = rows + 512 * chunk;
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i) f.codes[i] = load_codes(codes_at + here32(from[i] & all));
#pragma unroll
    for (uint32_t i = 0; i < XP; ++i) f.x[i] = load16(x_at + here32(x_from[i] & all));
  };
  Floats4 acc[NT][TT];
#pragma unroll
  for (uint32_t i = 0; i < NT; ++i)
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) acc[i][tt] = Floats4{0, 0, 0, 0};
  uint32_t g0 = 0;
  const uint32_t part = w.group.d / 4;  // chunks whose scales are in shared memory together: of 64 groups and parts of two more
  const auto put = [&](const Chunk &f, uint32_t chunk) {
    wave_fence();  // other lanes have read the codes that were there
#pragma unroll
    for (uint32_t i = 0; i < XP; ++i) x_lds[chunk & 1][x_to[i]] = in_order(f.x[i]);
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i) codes_lds[wave][i][to] = f.codes[i];
  };
  // (of elements behind a row's last, which are zeros, the last group's: the next row's scale may be infinite)
  const auto there = [&](uint32_t group) { return group < w.groups ? group : w.groups - 1; };
  const auto use = [&](uint32_t chunk) {
    fence();
    const Words4 *here = x_lds[chunk & 1];
    const uint32_t r = 32 * nw + col;
    Words4 turn[NT];
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i) turn[i] = codes_lds[wave][i][col * 4 + (g ^ col / 4)];
    multiply<T, SG, NT, TT>(
        w, turn, 256 * chunk + kBlock * kw, g, [&](int tt, int s) { return here[(16 * tt + col) * 32 + (16 * kw + element<SG>(g, s) / 8 ^ col)]; },
        [&](int i, uint32_t group) {
          return T::to_float(*reinterpret_cast<const uint16_t *>(scales_lds + (r + 16 * i) * scale_stride(kGroups) + 2 * (there(group) - g0)));
        },
        [&](int i, uint32_t group) {
          const float zero = (float)(uint8_t)zeros_lds[(r + 16 * i) * zero_stride(kGroups) + (there(group) - g0)];
          return w.zeros == nullptr ? 8.0f : zero;  // (read in any case, without a branch)
        },
        acc);
  };
  // of the chunks a workgroup has `each`
  const uint32_t all = (w.width_in + 255) / 256, stop = (blockIdx.z + 1) * each < all ? (blockIdx.z + 1) * each : all;
  for (uint32_t begin = blockIdx.z * each; begin < stop; begin += part) {
    if (begin != blockIdx.z * each) fence();  // the scales before are no longer read
    g0 = w.group.of(256 * begin);
    const uint32_t here = begin + part < stop ? begin + part : stop, end = here < whole ? here : whole;
    Chunk f[kDepth];
    {
      const Scales<kRows, 128 * NW> scales(w, w.scales, 2, n0, g0, kGroups, scale_stride(kGroups));
      const Scales<kRows, 128 * NW> zeros(w, w.zeros != nullptr ? static_cast<const void *>(w.zeros) : w.scales, 1, n0, g0, kGroups, zero_stride(kGroups));
      // (in any case: behind loads that are on their way in one case only, all would be waited for)
#pragma unroll
      for (uint32_t i = 0; i < kDepth; ++i) {
        load(f[i], begin + i, end, whole != 0 ? ~0u : 0);
        __builtin_amdgcn_sched_barrier(0);  // (asked for in another order they would have to be waited for together)
      }
      scales.bring(w, scales_lds);
      if (w.zeros != nullptr) zeros.bring(w, zeros_lds);
    }
    uint32_t chunk = begin;
    for (; chunk + kDepth <= end; chunk += kDepth) {
#pragma unroll
      for (uint32_t i = 0; i < kDepth; ++i) {
        put(f[i], chunk + i);
        load(f[i], chunk + i + kDepth, end);
        use(chunk + i);
      }
    }
    // one more that is there, and a part
#pragma unroll 1
    for (; chunk < here; ++chunk) {
      if (chunk == whole) {
#pragma unroll
        for (uint32_t i = 0; i < NT; ++i) f[0].codes[i] = load_upto(weights + (from[i] - piece), 128 * whole + piece, w.row_bytes);
#pragma unroll
        for (uint32_t i = 0; i < XP; ++i) f[0].x[i] = load_upto(rows + (x_from[i] - x_piece), 512 * whole + x_piece, 2 * w.width_in);
      }
      put(f[0], chunk);
      use(chunk);
    }
  }
  // The two halves of the sums, and then whole rows of the result: 8 elements to a thread.
  constexpr uint32_t kStride = kRows + 4;  // (floats: whole 16 bytes)
  float *sums = reinterpret_cast<float *>(x_lds);
  static_assert(sizeof(x_lds) >= 16 * TT * kStride * sizeof(float));
#pragma unroll
  for (uint32_t half = 0; half < 2; ++half) {
    fence();
    if (kw != 1 - half) continue;
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i)
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float &at = sums[(16 * tt + 4 * g + j) * kStride + 32 * nw + 16 * i + col];
          at = half == 0 ? acc[i][tt][j] : at + acc[i][tt][j];
        }
  }
  fence();
  // (read where they are used: as registers they would have to be kept all along)
  typedef const __attribute__((address_space(4))) Wide *Argument;
  Argument at_end = reinterpret_cast<Argument>(reinterpret_cast<uintptr_t>(__builtin_amdgcn_kernarg_segment_ptr()));
  asm volatile("" : "+s"(at_end));
  ft_linear4_call c;
  c.out = at_end->c.out;
  c.base = at_end->c.base;
  c.out_stride = at_end->c.out_stride;
  c.base_stride = at_end->c.base_stride;
  c.rows = at_end->c.rows;
  float *partial = at_end->partial;
  const uint32_t width = at_end->w.width_out;
  for (uint32_t i = threadIdx.x; i < 16 * TT * kRows / 8; i += 128 * NW) {
    const uint32_t r = i / (kRows / 8), row = t0 + r, n = n0 + 8 * (i % (kRows / 8));
    if (row >= c.rows || n >= width) continue;
    const float *from = sums + r * kStride + 8 * (i % (kRows / 8));
    if (partial != nullptr) {
      float *to = partial + ((uint64_t)blockIdx.z * c.rows + row) * ((width + 7) / 8 * 8) + n;
      *reinterpret_cast<Floats4 *>(to) = *reinterpret_cast<const Floats4 *>(from);
      *reinterpret_cast<Floats4 *>(to + 4) = *reinterpret_cast<const Floats4 *>(from + 4);
      continue;
    }
    write8<T>(c, row, n, width - n, from);
  }
}

// What several workgroups have of the same sums, in their order: eight neighbouring elements of a row of the result to a thread, which asks for four
// workgroups' at a time. (Rows of sums are padded to eight elements.)
template <class T>
__global__ __launch_bounds__(256) void ft_linear4_join_kernel(ft_linear4_call c, uint32_t width, uint32_t parts, const float *partial) {
  const uint32_t eights = (width + 7) / 8;
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x, all = (uint64_t)c.rows * eights;
  if (i >= all) return;
  const uint32_t row = (uint32_t)(i / eights), n = 8 * (uint32_t)(i - (uint64_t)row * eights);
  const Floats4 *from = reinterpret_cast<const Floats4 *>(partial) + 2 * i;
  Floats4 a{0, 0, 0, 0}, b{0, 0, 0, 0};
  for (uint32_t z = 0; z < parts; z += 4) {
    Floats4 v[4][2];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      const uint64_t at = 2 * all * (z + j < parts ? z + j : parts - 1);
      v[j][0] = from[at];
      v[j][1] = from[at + 1];
    }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
      if (z + j < parts) {
        a += v[j][0];
        b += v[j][1];
      }
  }
  const float sums[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  write8<T>(c, row, n, width - n, sums);
}

// What the others do not take: groups below 32 elements, more than 1024 of them to a row, matrices of fewer than 16 scales, rows of x whose offsets 32 bits do
// not hold. A wavefront to an output column, eight rows at a time, a byte of codes to a lane: 129 us for 16 rows of 4096 to 4096, where the others take 7.
template <class T>
__global__ __launch_bounds__(256) void ft_linear4_any_kernel(Linear4View w, ft_linear4_call c) {
  const uint32_t lane = threadIdx.x & 63, n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= w.width_out) return;
  const uint8_t *codes = w.weights + (uint64_t)n * w.row_bytes;
  const uint16_t *x = static_cast<const uint16_t *>(c.x), *base = static_cast<const uint16_t *>(c.base);
  uint16_t *out = static_cast<uint16_t *>(c.out);
  for (uint32_t t0 = blockIdx.y * 8; t0 < c.rows; t0 += gridDim.y * 8) {
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (uint32_t b = lane; b < w.row_bytes; b += 64) {
      const uint32_t k = 2 * b, g = w.group.of(k);  // (a group has an even number of elements)
      const uint64_t at = (uint64_t)n * w.groups + g;
      const float scale = T::to_float(w.scales[at]), zero = w.zeros == nullptr ? 8.0f : (float)w.zeros[at];
      const uint32_t two = codes[b];
      const float lo = scale * ((float)(two & 15) - zero), hi = k + 1 < w.width_in ? scale * ((float)(two >> 4) - zero) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (t0 + i >= c.rows) break;
        const uint16_t *row = x + (t0 + i) * c.x_stride + k;
        sum[i] += T::to_float(row[0]) * lo;
        if (k + 1 < w.width_in) sum[i] += T::to_float(row[1]) * hi;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      for (int d = 32; d > 0; d >>= 1) sum[i] += __shfl_xor(sum[i], d);
      if (lane == 0 && t0 + i < c.rows) {
        if (base != nullptr) sum[i] += T::to_float(base[(t0 + i) * c.base_stride + n]);
        out[(t0 + i) * c.out_stride + n] = T::from_float(sum[i]);
      }
    }
  }
}

template <class T, int SG, int XL>
void launch_narrow(const Linear4View &w, const ft_linear4_call &c, hipStream_t stream) {
  const dim3 grid((w.width_out + 15) / 16, (c.rows + 15) / 16);
  hipLaunchKernelGGL((ft_linear4_narrow_kernel<T, SG, XL, 8>), grid, dim3(512), 16 * (scale_stride(w.groups) + zero_stride(w.groups)), stream, w, c);
}

template <class T, int SG, int TT, int NW>
void launch_wide(const Linear4View &w, const ft_linear4_call &c, const Linear4Plan &p, hipStream_t stream) {
  const dim3 grid((w.width_out + 32 * NW - 1) / (32 * NW), (c.rows + 16 * TT - 1) / (16 * TT), p.parts);
  float *partial = p.parts > 1 ? static_cast<float *>(c.workspace) : nullptr;
  hipLaunchKernelGGL((ft_linear4_wide_kernel<T, SG, TT, NW>), grid, dim3(128 * NW), 0, stream, Wide{w, c, p.each, partial});
}

template <class T, int SG>
void launch(const Linear4View &w, const ft_linear4_call &c, const Linear4Plan &p, hipStream_t stream) {
  if (p.narrow) {
    if (c.rows > 8) launch_narrow<T, SG, 8>(w, c, stream);
    else if (c.rows > 2) launch_narrow<T, SG, 4>(w, c, stream);
    else launch_narrow<T, SG, 1>(w, c, stream);
    return;
  }
  if (p.tiles == 4) launch_wide<T, SG, 4, 4>(w, c, p, stream);
  else if (p.tiles == 2) launch_wide<T, SG, 2, 2>(w, c, p, stream);
  else launch_wide<T, SG, 1, 2>(w, c, p, stream);
  if (p.parts > 1)
    hipLaunchKernelGGL(ft_linear4_join_kernel<T>, dim3((uint32_t)(((uint64_t)c.rows * ((w.width_out + 7) / 8) + 255) / 256)), dim3(256), 0, stream, c,
                       w.width_out, p.parts,
                       static_cast<const float *>(c.workspace));
}

template <class T>
hipError_t launch(const Linear4View &w, const ft_linear4_call &c, int cu_count, hipStream_t stream) {
  const uint32_t group = w.group.d;
  const Linear4Plan p = linear4_plan(w.width_in, w.width_out, group, c.rows, cu_count);
  const bool far = c.rows > 1 && c.x_stride >= 1u << 24;  // offsets of 32 bits would not reach
  if (p.any || far) {
    const uint32_t parts = (c.rows + 7) / 8;
    hipLaunchKernelGGL(ft_linear4_any_kernel<T>, dim3((w.width_out + 3) / 4, parts < 1024 ? parts : 1024), dim3(256), 0, stream, w, c);
  } else if (group % 128 == 0) {
    launch<T, 1>(w, c, p, stream);
  } else if (group == 64) {
    launch<T, 2>(w, c, p, stream);
  } else {
    launch<T, 0>(w, c, p, stream);
  }
  return hipGetLastError();
}

}  // namespace

uint64_t linear4_workspace(const ft_linear4 &w, uint32_t rows, int cu_count) {
  const Linear4Plan p = linear4_plan(w.width_in, w.width_out, w.group, rows, cu_count);
  return p.parts > 1 ? (uint64_t)p.parts * rows * ((w.width_out + 7) / 8 * 8) * sizeof(float) : 0;
}

hipError_t launch_linear4(const Linear4View &w, const ft_linear4_call &c, int cu_count, hipStream_t stream) {
  return w.type == FT_BF16 ? launch<Bf16>(w, c, cu_count, stream) : launch<Fp16>(w, c, cu_count, stream);
}

}  // namespace ft
