// Products of few rows with weights of 4 bits and group scales, read as they lie in the pool.
//
// The matrix instruction multiplies 16 rows of x with 16 rows of weights, 32 elements at a time. A code becomes a number of 16 bits by two
// instructions for two codes: put into the low places of a number's mantissa it is that number plus the code, 128 + code in bfloat16, 64 + code in float16,
// exactly. What is too much is taken away behind the products, for a group of elements at once, with the zero:
//   sum of x (code - zero) = sum of x (128 + code) - (128 + zero) sum of x,
// where the sums of x are a product with ones. So nothing is rounded but sums, in 32 bits, and the scale is applied to a group's sum.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

constexpr uint32_t kBlock = 128;   // elements of a row that four instructions multiply
constexpr uint32_t kMostGroups = 1024;  // of a row, for what has a workgroup's scales in shared memory from the start

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
  const auto add = [&](uint32_t group) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float by = scale(i, group), more = -by * (Code<T>::kMore + zero(i, group));
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][tt][j] = __builtin_fmaf(by, products[i][tt][j], __builtin_fmaf(more, sums[tt][j], acc[i][tt][j]));
    }
  };
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
      if ((s + 1) % each == 0) add(w.group.of(k + 32 - 32 * each));
    } else {
      // a lane's eight elements are in one group, and 32 in two at most
      const uint32_t first = w.group.of(k), last = w.group.of(k + 31);
      const bool mine = w.group.of(k + 8 * g) == first;
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        if (part == 1 && first == last) break;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) {
          Words4 some;
#pragma unroll
          for (int i = 0; i < 4; ++i) some[i] = mine == (part == 0) ? a[tt][i] : 0;
          sums[tt] = T::mfma(some, ones, nothing);
#pragma unroll
          for (int i = 0; i < NT; ++i) products[i][tt] = T::mfma(some, b[i], nothing);
        }
        add(part == 0 ? first : last);
      }
    }
  }
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

// Scales and zeros of rows n0 to n0 + ROWS - 1, groups g0 to g0 + groups - 1, to shared memory, 16 bytes a thread. (All rows' scales together are 16 bytes at least, and so are their zeros.)
template <int ROWS, int THREADS>
struct Scales {
  __device__ static void bring(const Linear4View &w, uint32_t n0, uint32_t g0, uint32_t groups, char *scales, char *zeros) {
    some(reinterpret_cast<const char *>(w.scales), 2, w, n0, g0, groups, scales, scale_stride(groups));
    if (w.zeros != nullptr) some(reinterpret_cast<const char *>(w.zeros), 1, w, n0, g0, groups, zeros, zero_stride(groups));
  }
  __device__ static void some(const char *from, uint32_t size, const Linear4View &w, uint32_t n0, uint32_t g0, uint32_t groups, char *to, uint32_t stride) {
    const uint32_t pieces = (groups * size + 15) / 16;  // of a row
    const uint64_t all = (uint64_t)w.width_out * w.groups * size;
    for (uint32_t i = threadIdx.x; i < ROWS * pieces; i += THREADS) {
      const uint32_t r = i % ROWS, j = i / ROWS, n = n0 + r < w.width_out ? n0 + r : w.width_out - 1;
      const Words4 v = load_upto(from, ((uint64_t)n * w.groups + g0) * size + 16 * j, all);
      uint32_t *out = reinterpret_cast<uint32_t *>(to + r * stride + 16 * j);
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k)
        if (16 * j + 4 * k < stride) out[k] = v[k];
    }
  }
};

// 16 rows of weights to a workgroup, and 16 rows of x, 2 XL of which there are. Its wavefronts have every KW-th 256 elements and add up what they
// have at the end. A wavefront brings what it multiplies by itself, neighbouring lanes neighbouring pieces, and turns it round in shared memory of
// its own.
template <class T, int SG, int XL, int KW>
__global__ __launch_bounds__(64 * KW) void ft_linear4_narrow_kernel(Linear4View w, ft_linear4_call c) {
  constexpr int R = 2 * XL, kDepth = XL <= 2 ? 4 : 2;
  __shared__ Words4 codes_lds[KW][16 * 8], x_lds[KW][R * 32];
  __shared__ float parts[KW][4][64];
  extern __shared__ char scales_lds[];
  char *zeros_lds = scales_lds + 16 * scale_stride(w.groups);
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, col = lane % 16;
  const uint32_t n0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  // where this lane's pieces come from, and where they go
  const uint8_t *from[2];
  uint32_t to[2];
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i) {
    const uint32_t r = 8 * i + lane / 8, n = n0 + r < w.width_out ? n0 + r : w.width_out - 1;
    from[i] = w.weights + (uint64_t)n * w.row_bytes;
    to[i] = r * 8 + (lane % 8 ^ r >> 1);
  }
  const uint16_t *x_from[XL];
  uint32_t x_to[XL];
#pragma unroll
  for (uint32_t i = 0; i < XL; ++i) {
    const uint32_t r = 2 * i + lane / 32, t = t0 + r < c.rows ? t0 + r : c.rows - 1;
    x_from[i] = static_cast<const uint16_t *>(c.x) + t * c.x_stride;
    x_to[i] = r * 32 + (lane % 32 ^ r);
  }
  const uint32_t pieces = w.width_in / 256, all = (w.width_in + 255) / 256;
  Words4 codes[kDepth][2], x[kDepth][XL];
  const auto load = [&](Words4 (&to_codes)[2], Words4 (&to_x)[XL], uint32_t piece) {
#pragma unroll
    for (int i = 0; i < 2; ++i) to_codes[i] = load_codes(from[i] + 128 * piece + 16 * (lane % 8));
#pragma unroll
    for (int i = 0; i < XL; ++i) to_x[i] = load16(x_from[i] + 256 * piece + 8 * (lane % 32));
  };
  if (wave < pieces)
#pragma unroll
    for (int i = 0; i < kDepth; ++i) load(codes[i], x[i], wave + i * KW < pieces ? wave + i * KW : pieces - 1);
  Scales<16, 64 * KW>::bring(w, n0, 0, w.groups, scales_lds, zeros_lds);
  __syncthreads();
  Floats4 acc[1][1] = {{Floats4{0, 0, 0, 0}}};
  // (of elements behind a row's last, which are zeros, the last group's)
  const auto there = [&](uint32_t group) { return group < w.groups ? group : w.groups - 1; };
  const auto scale = [&](int, uint32_t group) { return T::to_float(*reinterpret_cast<const uint16_t *>(scales_lds + col * scale_stride(w.groups) + 2 * there(group))); };
  const auto zero = [&](int, uint32_t group) { return w.zeros == nullptr ? 8.0f : (float)(uint8_t)zeros_lds[col * zero_stride(w.groups) + there(group)]; };
  const auto use = [&](const Words4 (&my_codes)[2], const Words4 (&my_x)[XL], uint32_t piece) {
#pragma unroll
    for (int i = 0; i < 2; ++i) codes_lds[wave][to[i]] = my_codes[i];
#pragma unroll
    for (int i = 0; i < XL; ++i) x_lds[wave][x_to[i]] = in_order(my_x[i]);
    const uint32_t row = col & (R - 1);
#pragma unroll
    for (uint32_t block = 0; block < 2; ++block) {
      const uint32_t k0 = 256 * piece + kBlock * block;
      if (k0 >= w.width_in) break;
      Words4 mine[1] = {codes_lds[wave][col * 8 + (4 * block + g ^ col >> 1)]};
      multiply<T, SG, 1, 1>(w, mine, k0, g, [&](int, int s) { return x_lds[wave][row * 32 + (16 * block + element<SG>(g, s) / 8 ^ row)]; }, scale, zero, acc);
    }
  };
  for (uint32_t p = wave; p < pieces; p += kDepth * KW) {
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      if (p + i * KW < pieces) use(codes[i], x[i], p + i * KW);
      const uint32_t next = p + (i + kDepth) * KW;
      load(codes[i], x[i], next < pieces ? next : pieces - 1);
    }
  }
  if (pieces < all && wave == pieces % KW) {
#pragma unroll
    for (int i = 0; i < 2; ++i) codes[0][i] = load_upto(from[i], 128 * pieces + 16 * (lane % 8), w.row_bytes);
#pragma unroll
    for (int i = 0; i < XL; ++i) x[0][i] = load_upto(x_from[i], 512 * pieces + 16 * (lane % 32), 2 * w.width_in);
    use(codes[0], x[0], pieces);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) parts[wave][j][lane] = acc[0][0][j];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < 256; i += 64 * KW) {
    const uint32_t l = i % 64, row = t0 + 4 * (l / 16) + i / 64, n = n0 + l % 16;
    if (row >= c.rows || n >= w.width_out) continue;
    float sum = 0;
#pragma unroll
    for (int k = 0; k < KW; ++k) sum += parts[k][i / 64][l];
    if (c.base != nullptr) sum += T::to_float(static_cast<const uint16_t *>(c.base)[row * c.base_stride + n]);
    static_cast<uint16_t *>(c.out)[row * c.out_stride + n] = T::from_float(sum);
  }
}

// 128 rows of weights to a workgroup - 32 to a wavefront, and two wavefronts take turns along the rows -, and 16 TT rows of x, which all wavefronts
// multiply and bring to shared memory together, 256 elements at a time, the next ones while these are multiplied.
template <class T, int SG, int TT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void ft_linear4_wide_kernel(Linear4View w, ft_linear4_call c) {
  constexpr uint32_t NT = 2, kGroups = 64, kDepth = TT == 4 ? 3 : 4;  // (chunks that are on their way)
  __shared__ Words4 x_lds[2][TT * 16 * 32], codes_lds[8][NT][16 * 4];
  __shared__ char scales_lds[128 * 4 * (kGroups / 2 | 1)], zeros_lds[128 * 4 * (kGroups / 4 | 1)];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, col = lane % 16;
  const uint32_t kw = wave / 4, nw = wave % 4, n0 = blockIdx.x * 128, t0 = blockIdx.y * (16 * TT);
  // offsets in bytes from the workgroup's first row: of 128 rows of weights less than 2^30, of 64 rows of x less than 2^31
  const uint8_t *weights = w.weights + (uint64_t)n0 * w.row_bytes;
  const char *rows = reinterpret_cast<const char *>(static_cast<const uint16_t *>(c.x) + t0 * c.x_stride);
  uint32_t from[NT], x_from[TT], x_to[TT];
#pragma unroll
  for (uint32_t i = 0; i < NT; ++i) {
    const uint32_t r = 32 * nw + 16 * i + lane / 4;
    from[i] = (n0 + r < w.width_out ? r : w.width_out - 1 - n0) * w.row_bytes;
  }
  const uint32_t to = lane / 4 * 4 + (lane % 4 ^ lane / 16), piece = 64 * kw + 16 * (lane % 4), x_piece = 16 * (threadIdx.x % 32);
#pragma unroll
  for (uint32_t i = 0; i < TT; ++i) {
    const uint32_t r = 16 * i + threadIdx.x / 32;
    x_from[i] = (t0 + r < c.rows ? r : c.rows - 1 - t0) * (2 * (uint32_t)c.x_stride);
    x_to[i] = r * 32 + (threadIdx.x % 32 ^ r % 16);
  }
  const uint32_t whole = w.width_in / 256;  // and a part
  struct Chunk {
    Words4 codes[NT], x[TT];
  };
  const auto load = [&](Chunk &f, uint32_t chunk) {
    if (chunk >= whole) chunk = whole - 1;
    const uint8_t *codes_at = weights + 128 * chunk;
    const char *x_at = rows + 512 * chunk;
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i) f.codes[i] = load_codes(codes_at + (from[i] + piece));
#pragma unroll
    for (int i = 0; i < TT; ++i) f.x[i] = load16(x_at + (x_from[i] + x_piece));
  };
  Floats4 acc[NT][TT];
#pragma unroll
  for (uint32_t i = 0; i < NT; ++i)
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) acc[i][tt] = Floats4{0, 0, 0, 0};
  uint32_t g0 = 0;
  const uint32_t part = w.group.d / (256 / kGroups);  // chunks whose scales are in shared memory together
  const auto scales_of = [&](uint32_t chunk) {
    if (chunk % part != 0) return;
    fence();  // those before are no longer read
    g0 = chunk / part * kGroups;
    Scales<128, 512>::bring(w, n0, g0, kGroups, scales_lds, zeros_lds);
  };
  const auto put = [&](const Chunk &f, uint32_t chunk) {
#pragma unroll
    for (int i = 0; i < TT; ++i) x_lds[chunk & 1][x_to[i]] = in_order(f.x[i]);
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i) codes_lds[wave][i][to] = f.codes[i];
  };
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
          return T::to_float(*reinterpret_cast<const uint16_t *>(scales_lds + (r + 16 * i) * scale_stride(kGroups) + 2 * (group - g0)));
        },
        [&](int i, uint32_t group) {
          return w.zeros == nullptr ? 8.0f : (float)(uint8_t)zeros_lds[(r + 16 * i) * zero_stride(kGroups) + (group - g0)];
        },
        acc);
  };
  if (whole != 0) {
    Chunk f[kDepth];
#pragma unroll
    for (uint32_t i = 0; i < kDepth; ++i) load(f[i], i);
    for (uint32_t chunk = 0; chunk < whole; chunk += kDepth) {
#pragma unroll
      for (uint32_t i = 0; i < kDepth; ++i) {
        if (chunk + i >= whole) break;
        scales_of(chunk + i);
        put(f[i], chunk + i);
        load(f[i], chunk + i + kDepth);
        use(chunk + i);
      }
    }
  }
  if (256 * whole < w.width_in) {
    scales_of(whole);
    Chunk f;
#pragma unroll
    for (uint32_t i = 0; i < NT; ++i) f.codes[i] = load_upto(weights + from[i], 128 * whole + piece, w.row_bytes);
#pragma unroll
    for (int i = 0; i < TT; ++i) f.x[i] = load_upto(rows + x_from[i], 512 * whole + x_piece, 2 * w.width_in);
    put(f, whole);
    use(whole);
  }
  // the two halves of the sums
  fence();
  Floats4 *parts = reinterpret_cast<Floats4 *>(x_lds);
  static_assert(sizeof(x_lds) >= 4 * NT * TT * 64 * sizeof(Floats4));
#pragma unroll
  for (uint32_t i = 0; i < NT; ++i)
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
      if (kw == 1) parts[((nw * NT + i) * TT + tt) * 64 + lane] = acc[i][tt];
  fence();
  if (kw == 1) return;
#pragma unroll
  for (uint32_t i = 0; i < NT; ++i) {
    const uint32_t n = n0 + 32 * nw + 16 * i + col;
    if (n >= w.width_out) continue;
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
      const Floats4 sum = acc[i][tt] + parts[((nw * NT + i) * TT + tt) * 64 + lane];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t row = t0 + 16 * tt + 4 * g + j;
        if (row >= c.rows) continue;
        const float base = c.base != nullptr ? T::to_float(static_cast<const uint16_t *>(c.base)[row * c.base_stride + n]) : 0;
        static_cast<uint16_t *>(c.out)[row * c.out_stride + n] = T::from_float(sum[j] + base);
      }
    }
  }
}

// A wavefront to an output column, eight rows at a time; any widths, groups and alignment.
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

}  // namespace

uint64_t linear4_workspace(const ft_linear4 &, uint32_t, int) { return 0; }

namespace {

template <class T, int SG, int XL>
void launch_narrow(const Linear4View &w, const ft_linear4_call &c, hipStream_t stream) {
  const dim3 grid((w.width_out + 15) / 16, (c.rows + 15) / 16);
  hipLaunchKernelGGL((ft_linear4_narrow_kernel<T, SG, XL, 8>), grid, dim3(512), 16 * (scale_stride(w.groups) + zero_stride(w.groups)), stream, w, c);
}

template <class T, int SG, int TT>
void launch_wide(const Linear4View &w, const ft_linear4_call &c, hipStream_t stream) {
  const dim3 grid((w.width_out + 127) / 128, (c.rows + 16 * TT - 1) / (16 * TT));
  hipLaunchKernelGGL((ft_linear4_wide_kernel<T, SG, TT>), grid, dim3(512), 0, stream, w, c);
}

template <class T, int SG>
void launch(const Linear4View &w, const ft_linear4_call &c, hipStream_t stream) {
  const bool far = c.rows > 1 && c.x_stride >= 1u << 24;  // offsets of 32 bits would not reach
  if (far) launch_narrow<T, SG, 8>(w, c, stream);
  else if (c.rows > 32) launch_wide<T, SG, 4>(w, c, stream);
  else if (c.rows > 16) launch_wide<T, SG, 2>(w, c, stream);
  else if (w.width_out >= 16384) launch_wide<T, SG, 1>(w, c, stream);
  else if (c.rows > 8) launch_narrow<T, SG, 8>(w, c, stream);
  else if (c.rows > 2) launch_narrow<T, SG, 4>(w, c, stream);
  else launch_narrow<T, SG, 1>(w, c, stream);
}

template <class T>
hipError_t launch(const Linear4View &w, const ft_linear4_call &c, hipStream_t stream) {
  const uint32_t group = w.group.d;
  if (group < 32 || w.groups > kMostGroups || w.width_in < 32 || (uint64_t)w.width_out * w.groups < 16) {  // (loads are of 16 bytes)
    const uint32_t parts = (c.rows + 7) / 8;
    hipLaunchKernelGGL(ft_linear4_any_kernel<T>, dim3((w.width_out + 3) / 4, parts < 1024 ? parts : 1024), dim3(256), 0, stream, w, c);
  } else if (group % 128 == 0) {
    launch<T, 1>(w, c, stream);
  } else if (group == 64) {
    launch<T, 2>(w, c, stream);
  } else {
    launch<T, 0>(w, c, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear4(const Linear4View &w, const ft_linear4_call &c, int, hipStream_t stream) {
  return w.type == FT_BF16 ? launch<Bf16>(w, c, stream) : launch<Fp16>(w, c, stream);
}

}  // namespace ft
