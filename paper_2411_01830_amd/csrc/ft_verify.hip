// Drafted tokens judged against the target's probabilities, and the token behind those that stand.
//
// Of a request's rows only those are read whole whose sum is asked for: the row that the next token comes from, and, where tokens were
// drawn, that of every sibling which falls with another one behind it. All other tests need two numbers each, which are gathered for all of a
// request's rows at once. A row's sum is that of chunks of 1024 tokens; the next token is looked for in their sums first, then in one chunk.
//
// One sum waits for another: a sibling is tested against what is left behind the one before it. A sum by one workgroup takes 4.5 us over 50001 tokens of
// bfloat16 with a draft, bound by instructions on 64-bit numbers, five for a token; spread over many workgroups it is bound by memory: 64 rows of 131072 tokens
// of float32 with their draft, 67 MB, take 12 us (5.6 TB/s). So a request's first sum, which most are done with, is spread, in a launch of its own
// (Stop is what it hands on), and those behind it are its one workgroup's: 64 chains of 4 to 8 take 17 us, 32 trees of 9 to 16 rows, with up to four sums one
// behind the other, 27. A further launch for each of these that gathers and goes down the rows again would not be shorter: that takes 3 to 4 us before its first
// load. One that is handed where the way stopped, and its siblings' numbers, was not tried.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

constexpr uint32_t kChunk = 1024;  // of the vocabulary: 16 tokens to a lane
constexpr uint32_t kMostChunks = (1u << 22) / kChunk;

struct Fp32 {
  typedef uint32_t Bits;
};
template <class T>
struct Probability {
  typedef uint16_t Bits;
  static __device__ float value(Bits b) { return T::to_float(b); }
  // 8 of them as they lie, at any element's address
  struct Raw {
    Words4 w;
  };
  static __device__ Raw load8(const Bits *p) { return {load16(p)}; }
  static __device__ void values(const Raw &r, float (&out)[8]) {
    const Words4 w = r.w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      out[2 * i] = value((uint16_t)w[i]);
      out[2 * i + 1] = value((uint16_t)(w[i] >> 16));
    }
  }
};
template <>
struct Probability<Fp32> {
  typedef uint32_t Bits;
  static __device__ float value(Bits b) { return __uint_as_float(b); }
  struct Raw {
    Words4 a, b;
  };
  static __device__ Raw load8(const Bits *p) { return {load16(p), load16(p + 4)}; }
  static __device__ void values(const Raw &r, float (&out)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      out[i] = value(r.a[i]);
      out[4 + i] = value(r.b[i]);
    }
  }
};

// What is left of a token's probability p where `taken` of the draft's q is gone; of NaN nothing is. (A maximum with a NaN is the other number.)
__device__ inline double left_of(double p, double taken, double q) { return __builtin_fmax(__builtin_fma(-taken, q, p), 0.0); }
__device__ inline double left_of(float p) { return __builtin_fmaxf(p, 0.0f); }

// v of another lane: of the same 16 lanes by a pattern, of 16 or 32 lanes further
template <int PATTERN>
__device__ inline double other_lane(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, PATTERN, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(bits >> 32), PATTERN, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// The sum over a wavefront, in all lanes: neighbours, pairs, quads mirrored, eights mirrored, and then what lies 16 and 32 lanes apart. (By shuffles through
// shared memory the six steps take longer than a chunk's loads.)
__device__ inline double wave_sum(double v) {
  v += other_lane<0xb1>(v);   // quad_perm 1 0 3 2
  v += other_lane<0x4e>(v);   // quad_perm 2 3 0 1
  v += other_lane<0x141>(v);  // row_half_mirror
  v += other_lane<0x140>(v);  // row_mirror
  typedef uint32_t Two __attribute__((ext_vector_type(2)));
  uint64_t bits = __builtin_bit_cast(uint64_t, v);
  Two lo = __builtin_amdgcn_permlane16_swap((uint32_t)bits, (uint32_t)bits, false, false);
  Two hi = __builtin_amdgcn_permlane16_swap((uint32_t)(bits >> 32), (uint32_t)(bits >> 32), false, false);
  v = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
  bits = __builtin_bit_cast(uint64_t, v);
  lo = __builtin_amdgcn_permlane32_swap((uint32_t)bits, (uint32_t)bits, false, false);
  hi = __builtin_amdgcn_permlane32_swap((uint32_t)(bits >> 32), (uint32_t)(bits >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}

// The sums over the lanes up to each: within 16 lanes, then with those of the 16 and of the 32 before.
template <int PATTERN, int ROWS>
__device__ inline double lane_before(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, PATTERN, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(bits >> 32), PATTERN, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ inline double wave_upto(double v) {
  v += lane_before<0x111, 0xf>(v);  // row_shr 1
  v += lane_before<0x112, 0xf>(v);
  v += lane_before<0x114, 0xf>(v);
  v += lane_before<0x118, 0xf>(v);
  v += lane_before<0x142, 0xa>(v);  // row_bcast 15: to the second and the fourth 16 lanes
  v += lane_before<0x143, 0xc>(v);  // row_bcast 31: to the upper 32
  return v;
}

__device__ inline double of_lane(double v, int lane) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)bits, lane), hi = __builtin_amdgcn_readlane((int)(bits >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ inline int32_t clamped(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : v > hi ? hi : v; }

struct Rows {
  int32_t parent[kMostVerifyRows], token[kMostVerifyRows];  // (a token outside the vocabulary: -1)
  float p[kMostVerifyRows], q[kMostVerifyRows], accept[kMostVerifyRows];
  int32_t fallen[kMostVerifyRows];
};

// A request's way down its rows. Every wavefront of the workgroup goes it by itself, its state is the same in all lanes.
template <class T, int THREADS>
struct Walk {
  typedef Probability<T> Pr;
  typedef typename Pr::Bits Bits;
  const ft_verify_call &v;
  Rows &s;
  int32_t first, n;  // rows of the request
  int32_t node, cursor;  // the last row that stands; rows from here on have not been looked at
  double taken, mass;    // A and T
  int32_t fell;          // rows that hang from the node and fell
  bool lacking;          // drawn: the mass is not known, as a sum over the row is due

  __device__ int lane() const { return threadIdx.x & 63; }
  __device__ const Bits *target(int32_t row) const { return static_cast<const Bits *>(v.target) + (uint64_t)(first + row) * v.target_stride; }
  __device__ const Bits *draft(int32_t row) const { return static_cast<const Bits *>(v.draft) + (uint64_t)(first + row) * v.draft_stride; }

  // the rows' own numbers to shared memory; a barrier is behind it
  __device__ void gather() {
    for (int32_t j = threadIdx.x; j < n; j += THREADS) {
      int32_t parent = v.parent == nullptr ? j - 1 : v.parent[first + j];
      if (parent < 0 || parent >= j) parent = -1;
      const int64_t token = v.tokens[first + j];
      const bool known = token >= 0 && token < (int64_t)v.vocab;
      float p = 0, q = 0;
      if (known && parent >= 0) {
        p = Pr::value(target(parent)[token]);
        if (v.draft != nullptr) q = Pr::value(draft(parent)[token]);
      }
      s.parent[j] = parent;
      s.token[j] = known ? (int32_t)token : -1;
      s.p[j] = p;
      s.q[j] = q;
      s.accept[j] = v.accept[first + j];
    }
    __syncthreads();
    stand(0);
  }

  __device__ void stand(int32_t row) {
    node = row;
    cursor = row + 1;
    taken = 0;
    mass = 1;
    fell = 0;
    lacking = false;
  }

  // the first row from the cursor on that hangs from the node, or n
  __device__ int32_t next() const {
    for (int32_t j = cursor; j < n; j += 64) {
      const uint64_t all = __ballot(j + lane() < n && s.parent[j + lane()] == node);
      if (all != 0) return j + __builtin_ctzll(all);
    }
    return n;
  }

  // not drawn: whether a row before `row` has its token and hangs from the node too
  __device__ bool before(int32_t row) const {
    for (int32_t j = node + 1; j < row; j += 64) {
      const int32_t i = j + lane();
      if (__ballot(i < row && s.parent[i] == node && s.token[i] == s.token[row]) != 0) return true;
    }
    return false;
  }

  // Goes on until a sum is lacking (which may not be asked for: then it is the token's), or all that hang from the node fell.
  __device__ void go() {
    while (!lacking) {
      const int32_t j = next();
      cursor = j;
      if (j >= n) return;
      cursor = j + 1;
      const float p = s.p[j], q = s.q[j], u = s.accept[j];
      if (v.draft != nullptr) {
        if ((double)u * mass * (double)q < (fell == 0 ? left_of(p) : left_of(p, taken, q))) {
          stand(j);
        } else {
          taken += mass;
          ++fell;
          lacking = true;
        }
      } else {
        const double left = before(j) ? 0 : left_of(p);
        if ((double)u * mass < left) {
          stand(j);
        } else {
          mass = mass > left ? mass - left : 0;
          ++fell;
        }
      }
    }
  }

  // not drawn: the tokens that fell, to shared memory; how many
  __device__ int32_t list() {
    if (v.draft != nullptr || fell == 0) return 0;
    int32_t count = 0;
    for (int32_t j = node + 1; j < n; j += 64) {
      const int32_t i = j + lane();
      const bool one = i < n && s.parent[i] == node && s.token[i] >= 0;
      const uint64_t all = __ballot(one);
      if (one && threadIdx.x < 64) s.fallen[count + __popcll(all & ((1ull << lane()) - 1))] = s.token[i];
      count += __popcll(all);
    }
    __syncthreads();
    return count;
  }

  // the same of a way that another workgroup went, by a wavefront
  __device__ int32_t fallen(int32_t fell_there) const {
    if (v.draft != nullptr || fell_there == 0) return 0;
    int32_t count = 0;
    for (int32_t j = node + 1; j < n; j += 64) {
      const int32_t i = j + lane();
      int64_t token = -1;
      if (i < n && (v.parent == nullptr ? i - 1 : v.parent[first + i]) == node) token = v.tokens[first + i];
      const bool one = token >= 0 && token < (int64_t)v.vocab;
      const uint64_t all = __ballot(one);
      if (one) s.fallen[count + __popcll(all & ((1ull << lane()) - 1))] = (int32_t)token;
      count += __popcll(all);
    }
    wave_fence();
    return count;
  }

  // what is left of 8 neighbouring tokens whose probabilities are a and b (Q) or a alone. The drop is of those that were not drawn.
  template <bool Q>
  __device__ void left8(const float (&a)[8], const float (&b)[8], uint32_t drop, double (&out)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = Q ? left_of(a[i], taken, b[i]) : left_of(a[i]);
    if (!Q && __ballot(drop != 0) != 0)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (drop >> i & 1) out[i] = 0;
  }
  // of the node's row, `at` to at + 7, whatever of them there is
  __device__ void left8(const Bits *p, const Bits *q, uint32_t at, uint32_t drop, double (&out)[8]) const {
    float a[8], b[8];
    if (at + 8 <= v.vocab) {
      Pr::values(Pr::load8(p + at), a);
      Pr::values(Pr::load8((q != nullptr ? q : p) + at), b);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = at + i < v.vocab ? Pr::value(p[at + i]) : 0;
        b[i] = q != nullptr && at + i < v.vocab ? Pr::value(q[at + i]) : 0;
      }
    }
    if (q != nullptr) left8<true>(a, b, drop, out);
    else left8<false>(a, b, drop, out);
  }

  // which of 8 neighbouring tokens fell. (All lanes come here.)
  __device__ uint32_t dropped(uint32_t chunk, uint32_t at, int32_t count) const {
    uint32_t drop = 0;
    for (int32_t j = 0; j < count; j += 64) {
      const uint32_t token = j + lane() < count ? (uint32_t)s.fallen[j + lane()] : 0xffffffffu;
      for (uint64_t all = __ballot(token / kChunk == chunk); all != 0; all &= all - 1) {
        const uint32_t off = (uint32_t)__shfl((int)token, __builtin_ctzll(all)) - at;
        if (off < 8) drop |= 1u << off;
      }
    }
    return drop;
  }

  // the sum of a chunk, in all lanes of a wavefront; what its two runs of eight tokens a lane give is added in their order
  __device__ double chunk_sum(const Bits *p, const Bits *q, uint32_t chunk, int32_t count) const {
    double sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
      const uint32_t at = chunk * kChunk + i * 512 + lane() * 8;
      double left[8];
      left8(p, q, at, dropped(chunk, at, count), left);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += left[e];
    }
    return wave_sum(sum);
  }
  // The same of N chunks, `step` apart and before `stop`, all whole. Their loads are on their way before the first is looked at; where there are
  // fewer, the last one's again.
  template <int N, bool Q>
  __device__ void some_sums(const Bits *p, const Bits *q, uint32_t chunk, uint32_t step, uint32_t stop, int32_t count, double *out) const {
    typename Pr::Raw a[N][2], b[N][2];
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t c = chunk + j * step < stop ? chunk + j * step : stop - 1, at = c * kChunk + i * 512 + lane() * 8;
        a[j][i] = Pr::load8(p + at);
        if (Q) b[j][i] = Pr::load8(q + at);
      }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t c = chunk + j * step;
      double sum = 0;
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        float x[8], y[8];
        Pr::values(a[j][i], x);
        if (Q) Pr::values(b[j][i], y);
        double left[8];
        left8<Q>(x, y, dropped(c, c * kChunk + i * 512 + lane() * 8, count), left);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += left[e];
      }
      sum = wave_sum(sum);
      if (lane() == 0 && c < stop) out[c] = sum;
    }
  }
  // of the chunks from `chunk` to before `end`
  __device__ void chunk_sums(const Bits *p, const Bits *q, uint32_t chunk, uint32_t step, uint32_t end, int32_t count, double *out) const {
    constexpr int N = 2;  // (four in flight do not fit into registers: 38 us where two take 27)
    const uint32_t whole = v.vocab / kChunk, stop = end < whole ? end : whole, begin = chunk;
    for (; chunk < stop; chunk += N * step) {
      if (q != nullptr) {
        if (chunk + step >= stop) some_sums<1, true>(p, q, chunk, step, stop, count, out);
        else some_sums<N, true>(p, q, chunk, step, stop, count, out);
      } else {
        if (chunk + step >= stop) some_sums<1, false>(p, q, chunk, step, stop, count, out);
        else some_sums<N, false>(p, q, chunk, step, stop, count, out);
      }
    }
    if (whole < end && begin <= whole && (whole - begin) % step == 0) {
      const double one = chunk_sum(p, q, whole, count);
      if (lane() == 0) out[whole] = one;
    }
  }

  __device__ uint32_t chunks() const { return (v.vocab + kChunk - 1) / kChunk; }

  // the chunks' sums to shared memory
  __device__ void sum(const Bits *q, int32_t count, double *chunk) const {
    chunk_sums(target(node), q, threadIdx.x >> 6, THREADS / 64, chunks(), count, chunk);
    __syncthreads();
  }

  // all chunks' sums together, the same in every wavefront
  __device__ double total(const double *chunk) const {
    double mine = 0;
    for (uint32_t c = lane(); c < chunks(); c += 64) mine += chunk[c];
    return wave_sum(mine);
  }

  // The token with which the sum over what is left exceeds `limit`: a wavefront looks for its chunk, then in it.
  __device__ int64_t choose(const Bits *q, int32_t count, const double *sums, double limit) const {
    double before = 0, there = 0;  // of the chunk: what is before it
    uint32_t chunk = 0xffffffffu, last = 0;
    double last_before = 0;
    for (uint32_t c0 = 0; c0 < chunks() && chunk == 0xffffffffu; c0 += 64) {
      const uint32_t c = c0 + lane();
      const double one = c < chunks() ? sums[c] : 0;
      const double upto = wave_upto(one);
      const uint64_t over = __ballot(one > 0 && before + upto > limit), some = __ballot(one > 0);
      if (over != 0) {
        const int at = __builtin_ctzll(over);
        chunk = c0 + at;
        there = before + (of_lane(upto, at) - of_lane(one, at));
      } else if (some != 0) {
        const int at = 63 - __builtin_clzll(some);
        last = c0 + at;
        last_before = before + (of_lane(upto, at) - of_lane(one, at));
      }
      before += of_lane(upto, 63);
    }
    if (chunk == 0xffffffffu) {
      chunk = last;
      there = last_before;
    }
    // 16 neighbouring tokens to a lane
    const uint32_t at = chunk * kChunk + lane() * 16;
    double left[2][8], sum = 0;
    left8(target(node), q, at, dropped(chunk, at, count), left[0]);
    left8(target(node), q, at + 8, dropped(chunk, at + 8, count), left[1]);
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += left[i / 8][i % 8];
    const double upto = wave_upto(sum);
    double here = there + (upto - sum);
    int over = -1, some = -1;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const double one = left[i / 8][i % 8];
      here += one;
      if (one > 0) {
        some = i;
        if (over < 0 && here > limit) over = i;
      }
    }
    const uint64_t overs = __ballot(over >= 0), somes = __ballot(some >= 0);
    const int who = overs != 0 ? __builtin_ctzll(overs) : 63 - __builtin_clzll(somes | 1);
    return (int64_t)chunk * kChunk + who * 16 + __builtin_amdgcn_readlane(overs != 0 ? over : some, who);
  }
};

// The rows of request r; n of them are judged.
__device__ inline void rows_of(const ft_verify_call &v, uint32_t r, int32_t *first, int32_t *all, int32_t *n) {
  *first = clamped(v.starts[r], 0, (int32_t)v.rows);
  *all = clamped(v.starts[r + 1], *first, (int32_t)v.rows) - *first;
  *n = (uint32_t)*all > v.drafts ? (int32_t)v.drafts : *all;
}

// Where a request's way stops for the first time.
struct Stop {
  double taken;
  int32_t node, fell;
  int32_t last;  // whether it ends there
  int32_t _pad;
};

// Which rows stand: those on the way to `node`. All threads of the workgroup come here.
template <int THREADS>
__device__ inline void write_kept(const ft_verify_call &v, Rows &s, int32_t first, int32_t all, int32_t n, int32_t node) {
  __syncthreads();
  int32_t *on = s.fallen;
  for (int32_t j = threadIdx.x; j < n; j += THREADS) on[j] = 0;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int32_t j = node; j >= 0; j = s.parent[j]) on[j] = 1;  // (parents are before their rows)
  __syncthreads();
  for (int32_t j = threadIdx.x; j < all; j += THREADS) v.keep[first + j] = j < n ? (uint8_t)on[j] : 0;
}

// The chunks' sums of the first row whose sum a request asks for, several workgroups to a request: each goes the way there by itself, and has
// `each` chunks. The first one says where that was, and which rows stand if the way ends there.
template <class T>
__global__ __launch_bounds__(256) void ft_verify_sums_kernel(ft_verify_call v, uint32_t each, double *sums, Stop *stops) {
  __shared__ Rows s;
  const uint32_t r = blockIdx.y;
  int32_t first, all, n;
  rows_of(v, r, &first, &all, &n);
  if (n == 0) return;
  Walk<T, 256> walk{v, s, first, n};
  walk.gather();
  walk.go();
  const int32_t count = walk.list();
  const auto *p = walk.target(walk.node), *q = v.draft != nullptr && walk.fell != 0 ? walk.draft(walk.node) : nullptr;
  const uint32_t chunks = walk.chunks(), end = (blockIdx.x + 1) * each < chunks ? (blockIdx.x + 1) * each : chunks;
  walk.chunk_sums(p, q, blockIdx.x * each + (threadIdx.x >> 6), 4, end, count, sums + (uint64_t)r * chunks);
  if (blockIdx.x != 0) return;
  const bool last = !walk.lacking || walk.next() >= n;
  if (threadIdx.x == 0) stops[r] = Stop{walk.taken, walk.node, walk.fell, last, 0};
  if (last) write_kept<256>(v, s, first, all, n, walk.node);
}

// The last row that stands and the token behind it, by a wavefront.
template <class W, class Bits>
__device__ inline void finish(const ft_verify_call &v, uint32_t r, int32_t first, const W &walk, const Bits *q, int32_t count, const double *sums,
                              double *spare) {
  const double pick = v.pick[r];
  double sum = walk.total(sums);
  if (!(sum > 0)) {  // nothing is left: the target itself
    q = nullptr;
    count = 0;
    wave_fence();  // (the spare ones may be the sums themselves)
    walk.chunk_sums(walk.target(walk.node), q, 0, 1, walk.chunks(), 0, spare);
    wave_fence();
    sums = spare;
    sum = walk.total(sums);
  }
  const int64_t token = sum > 0 ? walk.choose(q, count, sums, __dmul_rn(pick, sum)) : -1;
  if (threadIdx.x == 0) {
    v.last[r] = first + walk.node;
    v.token[r] = token;
  }
}

// A workgroup to a request, of 16 wavefronts, each with every 16th chunk. SUMS: those of the first row that is asked for are there; where the way ends with it a wavefront does the rest.
template <class T, bool SUMS>
__global__ __launch_bounds__(1024) void ft_verify_kernel(ft_verify_call v, const double *sums, const Stop *stops) {
  constexpr int kThreads = 1024;
  __shared__ Rows s;
  __shared__ double chunk[kMostChunks];
  const int32_t rows = (int32_t)v.rows;
  if (blockIdx.x == v.requests) {  // rows of no request
    const int32_t lo = v.requests != 0 ? clamped(v.starts[0], 0, rows) : rows, hi = v.requests != 0 ? clamped(v.starts[v.requests], lo, rows) : rows;
    for (int64_t i = threadIdx.x; i < lo; i += kThreads) v.keep[i] = 0;
    for (int64_t i = (int64_t)hi + threadIdx.x; i < rows; i += kThreads) v.keep[i] = 0;
    return;
  }
  const uint32_t r = blockIdx.x;
  int32_t first, all, n;
  rows_of(v, r, &first, &all, &n);
  Stop stop{};
  if (SUMS) stop = stops[r];  // (of a request without rows it is not there)
  if (n == 0) {
    if (threadIdx.x == 0) {
      v.last[r] = -1;
      v.token[r] = -1;
    }
    return;
  }
  Walk<T, kThreads> walk{v, s, first, n};
  if (SUMS) {
    const double *mine = sums + (uint64_t)r * walk.chunks();
    if (stop.last != 0) {
      if (threadIdx.x >= 64) return;
      walk.node = stop.node;
      walk.taken = stop.taken;
      finish(v, r, first, walk, v.draft != nullptr && stop.fell != 0 ? walk.draft(stop.node) : nullptr, walk.fallen(stop.fell), mine, chunk);
      return;
    }
    for (uint32_t c = threadIdx.x; c < walk.chunks(); c += kThreads) chunk[c] = mine[c];
  }
  walk.gather();
  typedef typename Walk<T, kThreads>::Bits Bits;
  const Bits *q;
  int32_t count;
  for (bool there = SUMS;; there = false) {
    walk.go();
    q = v.draft != nullptr && walk.fell != 0 ? walk.draft(walk.node) : nullptr;
    count = walk.list();
    if (!there) walk.sum(q, count, chunk);
    if (!walk.lacking) break;
    if (walk.next() >= walk.n) break;
    walk.lacking = false;
    walk.mass = walk.total(chunk);
    __syncthreads();
  }
  if (threadIdx.x < 64) finish(v, r, first, walk, q, count, chunk, chunk);
  write_kept<kThreads>(v, s, first, all, n, walk.node);
}

// Workgroups that a request's first sum is spread over, 0: its own does it, and there is one launch. What spreading saves is a workgroup's way along
// its rows, what it costs is a launch and, with as many requests as compute units, units that wait for no one: it is done for up to a third as
// many requests, and for up to five eighths where a request's rows have 1 MiB. In two launches and in one, us, four rows a request:
//   with a draft     float32   32768 tokens   1:  7.0  7.3   64:  8.4  8.6    85:  9.9  9.2   128: 11.9 10.1
//                              65536          1:  6.6  9.1   64: 12.0 12.6    85: 13.2 12.9   128: 15.8 14.4
//                             131072          1:  7.1 12.8   64: 16.3 19.1   128: 25.7 29.4   160: 30.4 31.5   192: 36.8 36.3   256: 48.5 47.0
//                             262144          1:  8.1 19.9   64: 26.3 46.7   128: 51.5 64.6   160: 67.2 71.8   192: 77.2 79.5   256: 98.4 93.0
//                   bfloat16  65536          1:  7.1  9.3   64:  9.7 11.1    85: 10.6 11.3   128: 12.8 11.7
//                             131072          1:  7.2 13.5   64: 13.2 16.1    85: 14.5 16.2   128: 17.7 17.3
//                             262144          1:  7.7 21.3   64: 18.1 25.2   128: 27.1 29.8   160: 32.4 32.0   192: 39.1 35.8
//   without          float32  131072          1:  7.4 13.7   64: 14.9 15.7    85: 17.9 15.8   128: 23.6 18.1
//                             262144          1:  8.6 21.8   64: 20.5 24.4   128: 30.8 33.4   160: 38.3 42.6   192: 43.6 49.2   256: 63.9 61.6
//                   bfloat16 131072          1:  7.9 14.5   64: 12.0 16.1    85: 14.0 16.2   128: 16.4 16.5
uint32_t slices_of(const ft_verify_call &v, bool drawn, int cu_count) {
  const uint32_t chunks = (v.vocab + kChunk - 1) / kChunk, most = (chunks + 3) / 4, units = (uint32_t)cu_count;
  const uint64_t bytes = (uint64_t)v.vocab * (v.type == FT_FP32 ? 4 : 2) * (drawn ? 2 : 1);
  if (chunks <= 32 || (bytes < 1u << 20 ? 3 * v.requests > units : 8 * v.requests > 5 * units)) return 0;
  const uint32_t want = 4 * units / v.requests;  // of four wavefronts each
  return want < most ? want : most;
}

template <class T>
void launch(const ft_verify_call &v, int cu_count, hipStream_t stream) {
  const uint32_t slices = v.requests == 0 || v.rows == 0 ? 0 : slices_of(v, v.draft != nullptr, cu_count), chunks = (v.vocab + kChunk - 1) / kChunk;
  if (slices != 0) {
    const uint32_t each = (chunks + slices - 1) / slices;
    Stop *stops = static_cast<Stop *>(v.workspace);
    double *sums = reinterpret_cast<double *>(stops + v.requests);
    hipLaunchKernelGGL(ft_verify_sums_kernel<T>, dim3((chunks + each - 1) / each, v.requests), dim3(256), 0, stream, v, each, sums, stops);
    hipLaunchKernelGGL((ft_verify_kernel<T, true>), dim3(v.requests + 1), dim3(1024), 0, stream, v, sums, stops);
  } else {
    hipLaunchKernelGGL((ft_verify_kernel<T, false>), dim3(v.requests + 1), dim3(1024), 0, stream, v, nullptr, nullptr);
  }
}

}  // namespace

uint64_t verify_workspace(const ft_verify_call &v, int cu_count) {
  // (for either kind of call: with a draft it is spread wherever it is without)
  if (v.requests == 0 || v.rows == 0 || slices_of(v, true, cu_count) == 0) return 0;
  return v.requests * (sizeof(Stop) + (uint64_t)((v.vocab + kChunk - 1) / kChunk) * sizeof(double));
}

hipError_t launch_verify(const ft_verify_call &v, int cu_count, hipStream_t stream) {
  if (v.type == FT_FP32) launch<Fp32>(v, cu_count, stream);
  else if (v.type == FT_BF16) launch<Bf16>(v, cu_count, stream);
  else launch<Fp16>(v, cu_count, stream);
  return hipGetLastError();
}

}  // namespace ft
