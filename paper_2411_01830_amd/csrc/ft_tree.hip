// Attention of drafted tokens over a paged cache and over each other.
//
// The rows of a request that read one key head - its drafted tokens times the query heads of that key head - are a matrix Q. 32 keys at
// a time, S^T = K Q^T and O^T += V^T P^T by the matrix instruction, with the running maximum and sum of a softmax in
// between. Both products have the rows of Q as columns, so a lane deals with the same row throughout: its scores, its maximum, its sum and
// its part of O, and the weights P^T leave the first product in the registers that the second one reads them from - the 32 keys of a
// step are numbered so that lane group g (of four, 16 lanes each) holds keys 4g .. 4g+3 and 16+4g .. 16+4g+3 in both. Keys are read as
// the instruction wants them, 16 bytes a lane; of values a lane reads a piece of 8 rows and turns it round by byte permutes.
//
// The wavefronts of a workgroup bring 32 keys and values to shared memory together and read all of them, each for its own rows; heads
// of more than 128 elements, whose sums take the registers that this needs, are read into registers by each for itself. The chip holds
// a fixed number of workgroups, and the steps of all requests and key heads are dealt out to them evenly, whatever the lengths: a worker's part
// begins and ends anywhere, and what several have of one segment is joined by a second kernel, from sums in the workspace.
//
// What it costs, on a card that reads 6.1 to 6.9 TB/s and multiplies 1240 TFLOP/s in bfloat16 (caches of several inputs in turn, heads of 128):
//   one request, 2000 tokens of 8 key heads, a token          17.5 us: latency, 10 us until the first product is under way, and 5 of the join
//   64 requests of 16 to 8192, a token, 276 MB                70 us, 3.9 TB/s: the same at either end, the reads between (50 us if they were still in cache)
//   32 of 256 to 4096, trees of 9 to 16 under 4 heads, 175 MB 57 us, 3.1 TB/s
//   4 of 20000 to 32768, trees of 64 under 8 heads, 232 GFLOP 282 to 290 us, 810 TFLOP/s: vector instructions, 150 a step of 32 MFMA and 32 rows, which
//     take turns with the matrix unit: of what a step takes, products are a third, reads from shared memory an eighth, exponents a tenth
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kStep = 32;     // keys
// What a segment costs beside its steps, in steps, when they are dealt out. 64 requests of 16 to 8192 tokens: 81.5 us, 85.5 with 2, 81 with 4, 82.5 with 6;
// 256 of 16 to 2000: 110, 117.5, 107.5, 110; 24 of 16 to 3000, 9 rows of 64 elements: 26, 28, 24.5, 24; 5 of 16 to 400: 14.6, 14.2, 15.1, 16.5.
constexpr uint32_t kSegment = 3;
// How far, in powers of two, a score may pass the maximum that weights are relative to before sums are brought to a new one: weights
// stay below 2^8 and sums of them far from the end of any range, and most steps have no maximum to agree on over the lanes.
constexpr float kSlack = 8.0f;

// Where a wavefront has left out values that are not finite and that a row may see: its first and its last step with such, in units of work back from
// the end of its worker's range (0: none; the largest number stands for larger ones too).
struct LeftOut {
  uint32_t first, last;
};

struct Tree {
  KvView c;
  ft_tree_call t;
  uint32_t group;        // query heads of a key head
  uint32_t cluster;      // workgroups of a worker, which have different rows
  Divisor by_group;
  uint32_t workers, least;  // workgroups, and steps that each takes at least
  float scale;           // of products, times log2 e: more than 0
  uint32_t flip;         // the signs of queries where it was less
  uint64_t *prefix;      // requests + 2: work of the requests before; the workers' rate; all work
  LeftOut *left_out;     // of every wavefront
  float *sums;           // partial results, see Partial
};

__device__ inline uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline uint64_t uniform(uint64_t v) { return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }

// A barrier for shared memory alone: loads from global memory stay on their way.
__device__ inline void fence() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ inline uint64_t from_lane(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__shfl((int)(v >> 32), lane) << 32 | (uint32_t)__shfl((int)(uint32_t)v, lane);
}

// over the four lanes that have a row in common
__device__ inline float row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ inline float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// read through the scalar cache where the index is the same for all lanes: a vector load's answer would have to wait for all keys and
// values that were asked for before it
typedef const __attribute__((address_space(4))) int32_t *Constants;
__device__ inline Constants constants(const int32_t *p) { return reinterpret_cast<Constants>(reinterpret_cast<uintptr_t>(p)); }

// Workers' ranges: worker w has units [begin_of(w), begin_of(w + 1)), `rate` of them on average in 48.16 bits. All are as long but for
// one, so that no die has less to read than another.
__device__ inline uint64_t rate_of(uint64_t all, uint32_t workers, uint32_t least) {
  const uint64_t rate = ((all << 16) + workers - 1) / workers;
  return rate < (uint64_t)least << 16 ? (uint64_t)least << 16 : rate;
}
__device__ inline uint64_t begin_of(uint32_t worker, uint64_t rate) { return worker * rate >> 16; }
__device__ inline uint32_t worker_of(uint64_t unit, uint64_t rate) { return (uint32_t)(((unit + 1 << 16) - 1) / rate); }

// n / d; both are nearly always small, and a division of 64 bits is long
__device__ inline uint64_t quotient(uint64_t n, uint32_t d) { return n >> 32 == 0 ? (uint32_t)n / d : n / d; }

// A kernel's argument where it lies. What is read through it is read where it is used: the compiler would have all of it in scalar
// registers from the start, which are too few.
typedef const __attribute__((address_space(4))) Tree *Argument;
__device__ inline Argument argument() {
  Argument a = reinterpret_cast<Argument>(reinterpret_cast<uintptr_t>(__builtin_amdgcn_kernarg_segment_ptr()));
  asm volatile("" : "+s"(a));
  return a;
}
template <class D>
__device__ inline Divisor divisor(const D &d) {
  Divisor out;
  out.d = d.d;
  out.m = d.m;
  out.shift = d.shift;
  return out;
}

struct Request {
  int start, n, len;  // drafted tokens from `start`, cached ones
};

template <class A>
__device__ inline Request request(const A &a, uint32_t r) {
  const int tokens = (int)a.t.tokens;
  const Constants starts = constants(a.t.starts);
  int s = starts[r], e = starts[r + 1], len = constants(a.t.lens)[r];
  s = s < 0 ? 0 : s > tokens ? tokens : s;
  e = e < s ? s : e > tokens ? tokens : e;
  const uint64_t room = (uint64_t)a.t.blocks * a.c.page_tokens.d;
  len = len < 0 ? 0 : (uint64_t)len > room ? (int)room : len;
  const int n = e - s;
  return {s, n > (int)a.t.drafts ? (int)a.t.drafts : n, len};
}

__device__ inline uint32_t steps_for(int keys) { return ((uint32_t)keys + (kStep - 1)) >> 5; }  // (there may be 2^31 - 1 of them)
__device__ inline uint32_t steps_of(const Request &q) { return steps_for(q.len) + steps_for(q.n); }

// Work of a request: for each key head and each cluster's tiles of `rows` rows, which are a segment, what it costs to begin with and all of its
// steps.
template <class A>
__device__ inline uint64_t work_of(const A &a, const Request &q, uint32_t rows) {
  const uint32_t tiles = ((uint32_t)q.n * a.group + rows - 1) / rows;
  return (uint64_t)a.c.heads * ((tiles + a.cluster - 1) / a.cluster) * (steps_of(q) + kSegment);
}

// A worker's sums of a segment that it has a part of: [16 rows][4 elements x 64 lanes of every product], then a row's maximum and sum.
template <int DT>
struct Partial {
  static constexpr uint32_t kTile = 16 * DT + 32;  // floats of 16 rows
};

// The elements of one row that a lane holds: O[E (4 g + i) + j] in acc[j][i].
template <class T, int DT, class A>
__device__ inline void write_row(const A &a, const Floats4 (&acc)[DT / 16], float l, float m, const Request &q, uint32_t row, uint32_t kv_head, int g) {
  constexpr int E = DT / 16;
  const uint32_t token = divisor(a.by_group).of(row), head = kv_head * a.group + (row - token * a.group);
  if ((int)token >= q.n) return;
  const uint64_t t = (uint64_t)(q.start + (int)token);
  uint16_t *out = static_cast<uint16_t *>(a.t.out) + t * a.t.out_token_stride + head * a.t.out_head_stride + 4 * E * g;
  const float by = l == 0 ? 0 : 1 / l;
  uint32_t w[2 * E];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < E; j += 2) w[(i * E + j) / 2] = T::pack(acc[j][i] * by, acc[j + 1][i] * by);
#pragma unroll
  for (int x = 0; x < 2 * E; x += 4)  // 8 elements; the head's size is a multiple of that
    if (4 * E * g + 2 * x < (int)a.c.dim) *reinterpret_cast<Loose4 *>(out + 2 * x) = Loose4{{w[x], w[x + 1], w[x + 2], w[x + 3]}};
  if (g == 0 && a.t.lse != nullptr) a.t.lse[t * a.t.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Wavefronts to each of a compute unit's four parts: what their registers leave room for.
constexpr int waves(int dt) { return dt <= 128 ? 2 : 1; }

// Which of two elements are infinite or NaN: their exponents of all ones carry into the places of their signs.
template <class T>
__device__ inline uint32_t not_finite(uint32_t v) {
  return ((v & T::kExponent * 0x10001u) + T::kLowest * 0x10001u) & 0x80008000u;
}

// Two bytes of each of eight rows, as the matrix instruction wants them.
template <int W>
__device__ inline Words4 turned(const uint32_t (&v)[8][W], int word, uint32_t bytes) {
  Words4 out;
#pragma unroll
  for (int x = 0; x < 4; ++x) out[x] = __builtin_amdgcn_perm(v[2 * x + 1][word], v[2 * x][word], bytes);
  return out;
}

// NR: tiles of 16 rows a wavefront has. WR: wavefronts of a workgroup, which have different rows and read the same keys.
// PAGED: the head has DT elements and a page a multiple of 16 tokens, so 16 keys are read from one base address that is the same for all
// lanes; without it every lane finds the row of one key, and hands it on to those that read it.
// SHARED: keys and values go through shared memory, which the WR wavefronts of a workgroup fill together; several workgroups, a cluster, have
// the rows beyond those and are next to each other on one die, where the second finds in the cache what the first has read.
template <class T, int DT, int NR, int WR, bool PAGED, bool SHARED>
__global__ __launch_bounds__(64 * WR) __attribute__((amdgpu_waves_per_eu(waves(DT), waves(DT)))) void ft_tree_kernel(Tree) {
  constexpr int E = DT / 16, KS = DT / 32, RT = 16 * NR, ROWS = RT * WR;
  // SHARED: 16-byte pieces of a row, those of a step that a thread has, steps that are on their way besides the one in shared memory
  constexpr int CH = DT / 8, N = SHARED ? CH / (2 * WR) : 1, DEPTH = SHARED ? (NR == 1 ? 4 : 2) / N : 1, NI = SHARED ? N : 2;
  static_assert(!SHARED || (N >= 1 && N * 2 * WR == CH));
  __shared__ Words4 tile_lds[SHARED ? 2 : 1][2][SHARED ? 32 * CH : 1];
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
  const uint32_t wave = uniform((uint32_t)threadIdx.x >> 6);
  // SHARED: where a lane's pieces of a step's first keys and values are, in bytes; those of the others are an exclusive or and a distance away
  const uint32_t key_at = 16 * (n16 * CH + (g ^ (n16 % CH)));
  const uint32_t value_at = E == 4 ? 16 * (4 * g * CH + ((n16 / 2) ^ (4 * g % CH))) + 8 * (n16 & 1) : 16 * (4 * g * CH + (n16 ^ (4 * g % CH)));

  // The workers next to each other go to the same die: they read the same pages for other rows.
  const uint32_t per_die = gridDim.x / 8;
  const uint32_t place = (blockIdx.x % 8) * per_die + blockIdx.x / 8, worker = place / argument()->cluster, member = place - worker * argument()->cluster;
  // Every wavefront sums up the requests' work for itself, a lane a few that are neighbours, and finds where it begins.
  uint32_t r;
  uint64_t at, left;
  Request q;
  {
    const auto &a = *argument();
    const uint32_t requests = a.t.requests, each = (requests + 63) / 64, r0 = lane * each < requests ? lane * each : requests;
    const uint32_t r1 = r0 + each < requests ? r0 + each : requests;
    uint64_t mine = 0, sum;
    Request one{0, 0, 0};
    for (uint32_t i = r0; i < r1; ++i) {
      one = request(a, i);
      mine += work_of(a, one, ROWS);
    }
    sum = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    const uint64_t all = from_lane(sum, 63), before = sum - mine, rate = rate_of(all, a.workers, a.least);
    if (place == 0 && wave == 0) {
      uint64_t sofar = before;
      for (uint32_t i = r0; i < r1; ++i) {
        a.prefix[i] = sofar;
        sofar += r1 - r0 == 1 ? mine : work_of(a, request(a, i), ROWS);
      }
      if (lane == 0) {
        a.prefix[requests] = rate;
        a.prefix[requests + 1] = all;
      }
    }
    const uint64_t begin = begin_of(worker, rate), end = begin_of(worker + 1, rate);
    if (begin >= all) return;
    left = uniform((end < all ? end : all) - begin);
    uint32_t i = r0;
    uint64_t sofar = before;
    const bool here = begin >= before && begin < before + mine;
    if (here && r1 - r0 > 1)
      for (;; ++i) {
        one = request(a, i);
        const uint64_t w = work_of(a, one, ROWS);
        if (begin < sofar + w) break;
        sofar += w;
      }
    const int finder = __builtin_ctzll(__ballot(here));
    r = uniform((uint32_t)__shfl((int)i, finder));
    at = uniform(from_lane(begin - sofar, finder));
    q = {(int)uniform((uint32_t)__shfl(one.start, finder)), (int)uniform((uint32_t)__shfl(one.n, finder)), (int)uniform((uint32_t)__shfl(one.len, finder))};
  }
  // What the loop over keys goes by, each in a register of its own (as parts of the argument's words they would come and go with those). PAGED only.
  const Argument all = argument();
  uint32_t row_bytes = 2 * (uint32_t)all->c.token_stride, k_bytes = 2 * (uint32_t)all->t.k_token_stride, v_bytes = 2 * (uint32_t)all->t.v_token_stride;
  uint32_t pages = all->c.pages, page_d = all->c.page_tokens.d, page_m = all->c.page_tokens.m, page_shift = all->c.page_tokens.shift;
  uint64_t page_bytes = 2 * all->c.page_stride;
  float scale = all->scale;
  asm volatile("" : "+s"(row_bytes), "+s"(k_bytes), "+s"(v_bytes), "+s"(pages), "+s"(page_d), "+s"(page_m), "+s"(page_shift), "+s"(page_bytes), "+s"(scale));

  LeftOut left_out{0, 0};
  for (;;) {
    const uint32_t cluster = argument()->cluster, heads = argument()->c.heads, group = argument()->group;
    const uint32_t steps = steps_of(q), tiles = ((uint32_t)q.n * group + ROWS - 1) / ROWS, cost = steps + kSegment;
    const uint32_t cached = steps_for(q.len);
    const uint32_t groups = (tiles + cluster - 1) / cluster;
    const uint64_t segments = (uint64_t)heads * groups;
    uint64_t seg = quotient(at, cost);
    for (at -= seg * cost; seg < segments && left != 0; ++seg, at = 0) {
      // this worker's part of the segment's cost, and of its steps
      const uint32_t from = (uint32_t)at, to = cost - from < left ? cost : from + (uint32_t)left;
      left -= to - from;
      const uint32_t first = from < kSegment ? 0 : from - kSegment, last = to < kSegment ? 0 : to - kSegment;
      if (first == last) continue;
      const auto &a = *argument();
      const auto &t = a.t;
      const auto &c = a.c;
      const Constants table = constants(t.table + (uint64_t)r * t.blocks);
      const uint32_t head = uniform((uint32_t)quotient(seg, groups)), tile = uniform((uint32_t)(seg - (uint64_t)head * groups) * cluster + member);
      if (tile >= tiles) continue;
      const uint32_t row0 = tile * ROWS + wave * RT;
      const char *kc = c.k + 2 * (head * c.head_stride), *vc = c.v + 2 * (head * c.head_stride);
      const char *kd = static_cast<const char *>(t.k) + 2 * (q.start * t.k_token_stride + head * t.k_head_stride);
      const char *vd = static_cast<const char *>(t.v) + 2 * (q.start * t.v_token_stride + head * t.v_head_stride);

      Words4 qf[NR][KS];
      // rows behind the last one are answered as that one is, and not written
      const auto row_of = [&](int nr) -> uint32_t {
        const uint32_t row = row0 + nr * 16 + n16, most = (uint32_t)q.n * group - 1;
        return row < most ? row : most;
      };
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        const uint32_t row = row_of(nr), tok = divisor(a.by_group).of(row);
        const uint16_t *p = static_cast<const uint16_t *>(t.q) + (q.start + (int)tok) * t.q_token_stride + (head * group + (row - tok * group)) * t.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int d = ks * 32 + 8 * g;
          if (PAGED || d < (int)c.dim) qf[nr][ks] = load16(p + d);
          else qf[nr][ks] = Words4{0, 0, 0, 0};
#pragma unroll
          for (int x = 0; x < 4; ++x) qf[nr][ks][x] ^= a.flip;
        }
      }
      Floats4 acc[NR][E];
      float m[NR], l[NR];
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        m[nr] = -INFINITY;
        l[nr] = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) acc[nr][j] = Floats4{0, 0, 0, 0};
      }

      Words4 kf[2][KS];
      uint32_t vf[8][E / 2];

      // A step's rows. PAGED: 16 cached keys have a page in common, whose number is read two steps ahead; rows behind the last
      // key, in that page still, are read and not looked at. Otherwise lane l % 32 finds key l % 32, behind the last one that one again. So
      // it is with drafted keys. (No branches here: loads under a condition, of either outcome, would be waited for as if they were not there.)
      const uint32_t end_key = q.len > 0 ? (uint32_t)q.len - 1 : 0;
      // SHARED: which 16 of a step's keys this wavefront brings, of its i-th pieces
      const auto half_of = [&](int i) -> uint32_t { return (i * 64 * WR + wave * 64) / CH >> 4; };
      const auto pages_of = [&](uint32_t st, uint32_t (&ids)[NI]) {
        if (st >= cached) return;
        if constexpr (PAGED) {
#pragma unroll
          for (int kk = 0; kk < NI; ++kk) {
            const uint32_t key = st * kStep + (SHARED ? half_of(kk) : kk) * 16;
            ids[kk] = (uint32_t)table[uniform(__umulhi(key < end_key ? key : end_key, page_m) >> page_shift)];
          }
        } else {
#pragma unroll
          for (int i = 0; i < (SHARED ? N : 1); ++i) {
            const uint32_t key = st * kStep + (SHARED ? (i * 64 * WR + threadIdx.x) / CH : lane & 31);
            ids[i] = (uint32_t)table[divisor(c.page_tokens).of(key < end_key ? key : end_key)];
          }
        }
      };
      // A row of a step as an offset in bytes from the head's first one (without PAGED), of cached and of drafted keys.
      const auto lane_row = [&](uint32_t st, uint32_t of_step, uint32_t page, uint64_t draft_stride) -> uint64_t {
        uint32_t key = st * kStep + of_step, draft = key - cached * kStep;
        key = key < end_key ? key : end_key;
        draft = draft < (uint32_t)q.n ? draft : (uint32_t)q.n - 1;
        const uint64_t in_cache = (page < c.pages ? page : 0) * c.page_stride + divisor(c.page_tokens).rest(key) * c.token_stride;
        return 2 * (st < cached ? in_cache : draft * draft_stride);
      };
      // PAGED: where 16 keys of a step begin, in bytes from the head's first one, and how many rows there are behind that one.
      struct Half {
        uint64_t row;
        uint32_t behind;
      };
      const auto half = [&](uint32_t st, int kk, uint32_t page, uint32_t draft_stride) -> Half {
        const uint32_t key = st * kStep + kk * 16, end = (uint32_t)q.n - 1;
        const uint32_t draft = key - cached * kStep < end ? key - cached * kStep : end;
        const bool in_cache = st < cached;
        page = in_cache && page < pages ? page : 0;
        const uint32_t row = in_cache ? key - (__umulhi(key, page_m) >> page_shift) * page_d : draft;
        return {page * page_bytes + (uint64_t)row * (in_cache ? row_bytes : draft_stride), in_cache ? 15 : end - draft};
      };
      const auto load_keys = [&](uint32_t st, const uint32_t (&ids)[NI]) {
        const uint64_t row = PAGED ? 0 : lane_row(st, lane & 31, ids[0], t.k_token_stride);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          Global base = global(st < cached ? kc : kd);
          uint32_t off = 16 * g;
          if constexpr (PAGED) {
            const Half h = half(st, kk, ids[kk], k_bytes);
            base += h.row;
            off += __umul24((uint32_t)n16 < h.behind ? n16 : h.behind, st < cached ? row_bytes : k_bytes);
            asm volatile("" : "+s"(base), "+v"(off));  // (32 bits beside a base in scalar registers: the sum of both would take two registers a row)
          } else {
            base += from_lane(row, kk * 16 + n16);
          }
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            if (PAGED || ks * 32 + 8 * g < (int)c.dim) kf[kk][ks] = load16(base + off + ks * 64);
            else kf[kk][ks] = Words4{0, 0, 0, 0};
          }
        }
      };
      const auto load_values = [&](uint32_t st, const uint32_t (&ids)[NI]) {
        const uint64_t row = PAGED ? 0 : lane_row(st, lane & 31, ids[0], t.v_token_stride);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          Global half_base = global(st < cached ? vc : vd);
          Half h{0, 0};
          if constexpr (PAGED) {
            h = half(st, kk, ids[kk], v_bytes);
            half_base += h.row;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int e = 4 * kk + i;
            Global base = half_base;
            uint32_t off = 2 * E * n16;
            if constexpr (PAGED) {
              off += __umul24((uint32_t)(4 * g + i) < h.behind ? 4 * g + i : h.behind, st < cached ? row_bytes : v_bytes);
              asm volatile("" : "+s"(base), "+v"(off));
            } else {
              base += from_lane(row, kk * 16 + 4 * g + i);
            }
            // a lane's piece of a row: E elements, some multiple of 8 of which the head has
#pragma unroll
            for (int x = 0; x < E / 8; ++x) {
              Words4 w{0, 0, 0, 0};
              if (PAGED || E * n16 + 8 * x < (int)c.dim) w = load16(base + off + 16 * x);
#pragma unroll
              for (int y = 0; y < 4; ++y) vf[e][4 * x + y] = w[y];
            }
          }
        }
      };
      // SHARED: where a thread's pieces of a step's keys and values are. Row r has its pieces in the order that counting up to CH and an exclusive
      // or with r give: wavefronts read 16 bytes of each of several rows, and so meet different banks.
      struct Place {
        Global k, v;
        uint32_t k_off, v_off;
      };
      uint32_t lane_off[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t index = i * 64 * WR + threadIdx.x, row = index / CH;
        lane_off[i] = 16 * ((index % CH) ^ (row % CH)) + (PAGED ? __umul24(row & 15, row_bytes) : 0);
      }
      const auto place = [&](uint32_t st, uint32_t page, int i) -> Place {
        const uint32_t end = (uint32_t)q.n - 1;
        Place at;
        if constexpr (PAGED) {
          const uint32_t key = st * kStep + half_of(i) * 16;
          if (st < cached) {
            const uint32_t row = key - (__umulhi(key, page_m) >> page_shift) * page_d;
            const uint64_t first_row = (page < pages ? page : 0) * page_bytes + (uint64_t)row * row_bytes;
            at = {global(kc) + first_row, global(vc) + first_row, lane_off[i], lane_off[i]};
          } else {
            const uint32_t draft = key - cached * kStep < end ? key - cached * kStep : end, index = i * 64 * WR + threadIdx.x, row = index / CH;
            const uint32_t of_half = (row & 15) < end - draft ? row & 15 : end - draft, piece = 16 * ((index % CH) ^ (row % CH));
            at = {global(kd) + (uint64_t)draft * k_bytes, global(vd) + (uint64_t)draft * v_bytes, piece + __umul24(of_half, k_bytes), piece + __umul24(of_half, v_bytes)};
          }
          asm volatile("" : "+s"(at.k), "+s"(at.v), "+v"(at.k_off), "+v"(at.v_off));
        } else {
          uint32_t index = i * 64 * WR + threadIdx.x;
          asm volatile("" : "+v"(index));
          at.k_off = lane_off[i] >= 2 * c.dim ? 0 : lane_off[i];  // (what is behind the head)
          at.v_off = at.k_off;
          at.k = global(st < cached ? kc : kd) + lane_row(st, index / CH, page, t.k_token_stride);
          at.v = global(st < cached ? vc : vd) + lane_row(st, index / CH, page, t.v_token_stride);
        }
        return at;
      };
      const auto put = [&](Words4 *to, const Words4 (&from)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i)  // behind the head queries are zero, and keys too: what was read there may be an infinity
          to[i * 64 * WR + threadIdx.x] = PAGED || lane_off[i] < 2 * c.dim ? from[i] : Words4{0, 0, 0, 0};
      };
      // (the empty statements keep places from being worked out once and held: registers are scarcer than instructions)
      const auto get_keys = [&](int buf) {
        uint32_t at = key_at;
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const char *p = reinterpret_cast<const char *>(tile_lds[0][0]) + (at ^ (ks * 64));
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) kf[kk][ks] = *reinterpret_cast<const Words4 *>(p + buf * (int)sizeof(tile_lds[0]) + kk * 256 * CH);
        }
      };
      const auto get_values = [&](int buf) {
        uint32_t at = value_at;
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const char *p = reinterpret_cast<const char *>(tile_lds[0][0]) + (at ^ (i * 16));
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            const char *row = p + buf * (int)sizeof(tile_lds[0]) + (int)sizeof(tile_lds[0][0]) + (16 * kk + i) * 16 * CH;
            if constexpr (E == 4) {
              typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
              const Words2 w = *reinterpret_cast<const Words2 *>(row);
              vf[4 * kk + i][0] = w[0];
              vf[4 * kk + i][1] = w[1];
            } else if constexpr (E == 8) {
              const Words4 w = *reinterpret_cast<const Words4 *>(row);
#pragma unroll
              for (int y = 0; y < 4; ++y) vf[4 * kk + i][y] = w[y];
            }
          }
        }
      };
      // which of a step's keys a row sees
      const auto sees_of = [&](int nr, uint32_t st) -> uint32_t {
        const bool drafted = st >= cached;
        const uint32_t js = st - cached, valid = drafted ? (uint32_t)q.n - js * kStep : (uint32_t)q.len - st * kStep;
        uint32_t w = ~0u;
        if (drafted) {
          const int token = (int)divisor(a.by_group).of(row_of(nr));
          if (t.mask != nullptr) {
            w = reinterpret_cast<const uint32_t *>(t.mask)[(uint64_t)(q.start + token) * 2 * t.mask_words + js];
          } else {
            const int d = token - (int)(js * kStep);
            w = d < 0 ? 0 : d >= 31 ? ~0u : (2u << d) - 1;
          }
        }
        return valid < 32 ? w & ((1u << valid) - 1) : w;
      };

      Floats4 s[NR][2];
      const auto scores = [&] {
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            s[nr][kk] = Floats4{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s[nr][kk] = T::mfma(kf[kk][ks], qf[nr][ks], s[nr][kk]);
          }
      };
      Words4 p[NR];
      uint32_t far = 0;  // a maximum is or was beyond 2^24, on either side
      const auto weights = [&] {
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
          float x[8], w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = s[nr][i >> 2][i & 3];
          const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
          if (__any(top * scale > m[nr] + kSlack)) {
            // (at most the largest number: relative to an infinite maximum every weight would be zero, and the row one that sees nothing)
            const float now = fminf(fmaxf(m[nr], row_max(top) * scale), __FLT_MAX__);
            const float shrink = now == -INFINITY ? 1 : __builtin_amdgcn_exp2f(m[nr] - now);
            m[nr] = now;
            far |= uniform((uint32_t)(__any(now != -INFINITY && fabsf(now) > 0x1p24f) ? 1 : 0));
            l[nr] *= shrink;
#pragma unroll
            for (int j = 0; j < E; ++j) acc[nr][j] *= shrink;
          }
          const float from = m[nr] == -INFINITY ? 0 : m[nr];
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = __builtin_fmaf(x[i], scale, -from);
          // The maximum is a rounded score. All weights are off by the one factor that its rounding makes, which the row's sum takes out again, but
          // from 2^24 on that may be too much for any range: there each score is rounded as the maximum was.
          if (far != 0)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float score = x[i] * scale;
              asm("" : "+v"(score));
              w[i] = score - from;
            }
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_exp2f(w[i]);
          l[nr] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
          // rounded to the matrix unit's 16 bits for the product with the values; the sum has them as they were. Against 64 bits results are off by 0.0022 of their
          // size in bfloat16 and 0.00025 in float16, with weights of 32 bits by 0.0017 and 0.0002: most of it is the result's own rounding.
          p[nr] = Words4{T::pack(w[0], w[1]), T::pack(w[2], w[3]), T::pack(w[4], w[5]), T::pack(w[6], w[7])};
        }
      };
      const auto outputs = [&] {
#pragma unroll
        for (int j = 0; j < E; j += 2) {
          const Words4 lo = turned(vf, j / 2, 0x05040100), hi = turned(vf, j / 2, 0x07060302);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            acc[nr][j] = T::mfma(lo, p[nr], acc[nr][j]);
            acc[nr][j + 1] = T::mfma(hi, p[nr], acc[nr][j + 1]);
          }
        }
      };

      // Steps in which not everything is seen: the last cached keys where they are no whole step, and drafted ones. What a row does not see
      // has a weight of zero, and its value, which may be anything, must not be met by it where it is not finite: such values
      // are left out of the product. Where a row may see one, the kernel behind this one adds it.
      const auto edge = [&](uint32_t st) {
        if ((st + 1) * kStep <= (uint32_t)q.len) return;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
          const uint32_t sees = sees_of(nr, st);
#pragma unroll
          for (int i = 0; i < 8; ++i) s[nr][i >> 2][i & 3] = sees >> ((i >> 2) * 16 + 4 * g + (i & 3)) & 1 ? s[nr][i >> 2][i & 3] : -INFINITY;
        }
      };
      const auto edge_values = [&](uint32_t st) {
        if ((st + 1) * kStep <= (uint32_t)q.len) return;
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int x = 0; x < E / 2; ++x) any |= not_finite<T>(vf[e][x]);
        if (!__any(any != 0)) return;
        const int valid = st >= cached ? q.n - (int)(st - cached) * kStep : q.len - (int)(st * kStep);
        uint32_t seen = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t may = (e >> 2) * 16 + 4 * g + (e & 3) < valid ? ~0u : 0;
#pragma unroll
          for (int x = 0; x < E / 2; ++x) {
            const uint32_t bit = not_finite<T>(vf[e][x]) >> 15;
            seen |= bit & may;
            vf[e][x] &= ~((bit << 16) - bit);
          }
        }
        // (no branch here: the compiler would hold the values twice)
        const uint64_t back = left + (last - st);
        const uint32_t here = back >> 32 == 0 ? (uint32_t)back : ~0u, now = uniform((uint32_t)(__any(seen != 0) ? 1 : 0));
        left_out.last = uniform(now != 0 ? here : left_out.last);
        left_out.first = uniform(now != 0 && left_out.first == 0 ? here : left_out.first);
      };

      // A step's keys are on their way while the one before weighs its values, its values from there on, and the pages of the one behind it
      // are asked for first of all. The last step asks for its own rows once more, which are near by then: were there a
      // condition on these loads, what is asked for before them would be waited for together with them.
      const auto softmax = [&](uint32_t st) {
        edge(st);
        weights();
      };
      uint32_t st = first;
      uint32_t ids[NI] = {}, ahead[NI] = {};
      pages_of(st, ids);
      if (st + 1 < last) pages_of(st + 1, ahead);
      if constexpr (!SHARED) {
        load_keys(st, ids);
        __builtin_amdgcn_sched_barrier(0);  // (loads are waited for in their order: in the loop keys come first)
        load_values(st, ids);
        bool more;
        do {
          more = st + 1 < last;
          const uint32_t next = more ? st + 1 : st;
          if (more) {
#pragma unroll
            for (int i = 0; i < NI; ++i) ids[i] = ahead[i];
          }
          scores();
          load_keys(next, ids);
          __builtin_amdgcn_sched_barrier(0);  // (scalar loads come back in any order: to wait for these pages is to wait for the next ones)
          if (next + 1 < last) pages_of(next + 1, ahead);
          softmax(st);
          edge_values(st);
          outputs();
          load_values(next, ids);
          st = next;
        } while (more);
      } else {
        // The step that is worked on lies in one half of shared memory, the next one is put into the other half, those behind it are on their way
        // in registers. (Not all of the time: as it is compiled the first `put` of every DEPTH steps waits for all loads, the last one's too.) One barrier a step: it says that the half to work on is full, and that the other one has been read.
        const bool works = NR > 1 || row0 < (uint32_t)q.n * group;  // wavefronts without rows of their own bring theirs and wait
        Words4 k[DEPTH][N], v[DEPTH][N];
        uint32_t asked = st;  // the step that `ids` are the pages of
        const auto ask = [&](Words4 (&into_k)[N], Words4 (&into_v)[N]) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const Place at = place(asked, ids[i], i);
            into_k[i] = load16(at.k + at.k_off);
            into_v[i] = load16(at.v + at.v_off);
          }
          if (asked + 1 < last) {
            ++asked;
#pragma unroll
            for (int i = 0; i < NI; ++i) ids[i] = ahead[i];
          }
          __builtin_amdgcn_sched_barrier(0);
          if (asked + 1 < last) pages_of(asked + 1, ahead);
        };
        fence();  // what the segment before has left in shared memory has been read
        ask(k[0], v[0]);
        put(tile_lds[0][0], k[0]);
        put(tile_lds[0][1], v[0]);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) ask(k[d], v[d]);
        for (bool more = true; more;) {
#pragma unroll
          for (int d = 0; d < (DEPTH > 1 ? DEPTH : 2); ++d)
            if (more) {
              fence();
              put(tile_lds[d + 1 & 1][0], k[d % DEPTH]);
              put(tile_lds[d + 1 & 1][1], v[d % DEPTH]);
              ask(k[d % DEPTH], v[d % DEPTH]);
              __builtin_amdgcn_sched_barrier(0);  // (keys and values at once would not leave registers for what is on its way)
              if (works) {
                get_keys(d & 1);
                scores();
                __builtin_amdgcn_sched_barrier(0);
                softmax(st);
                __builtin_amdgcn_sched_barrier(0);
                get_values(d & 1);
                edge_values(st);
                outputs();
              }
              ++st;
              more = st < last;
            }
        }
      }
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) l[nr] = row_sum(l[nr]);
      if (row0 < (uint32_t)q.n * group) {  // (it is the most of all sums that wavefronts without rows would write)
        if (first == 0 && last == steps) {
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) write_row<T, DT>(a, acc[nr], l[nr], m[nr], q, row0 + nr * 16 + n16, head, g);
        } else {
          // a worker has at most two segments that it shares: the one it begins in, which others have begun, and the one it ends in
          float *sums = a.sums + ((((uint64_t)worker * 2 + (first == 0 ? 1 : 0)) * cluster + member) * WR + wave) * (NR * Partial<DT>::kTile);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
            for (int j = 0; j < E; ++j) reinterpret_cast<Floats4 *>(sums + nr * Partial<DT>::kTile)[j * 64 + lane] = acc[nr][j];
            if (g == 0) {
              sums[nr * Partial<DT>::kTile + 16 * DT + n16] = m[nr];
              sums[nr * Partial<DT>::kTile + 16 * DT + 16 + n16] = l[nr];
            }
          }
        }
      }
    }
    at = 0;
    q.n = 0;
    while (left != 0 && q.n == 0 && ++r < argument()->t.requests) q = request(*argument(), r);
    if (left == 0 || q.n == 0) {
      if (lane == 0) argument()->left_out[place * WR + wave] = left_out;
      return;
    }
  }
}

// Infinities and NaN among the values that a row sees, of the last cached keys and of drafted ones in steps [from, to], are added to its
// sums, whatever else these are: it cannot matter how much of them. Every fourth step to a wavefront: two lanes look at a key's values,
// then those with any are gone through, each lane for the elements of write_row.
template <class T, int DT, class A>
__device__ __forceinline__ void add_left_out(const A &a, const Request &q, uint32_t r, uint32_t row, uint32_t head, uint32_t from, uint32_t to, Floats4 (&acc)[DT / 16]) {
  constexpr int E = DT / 16;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const uint32_t cached = steps_for(q.len), whole = (uint32_t)q.len >> 5;
  uint32_t token = divisor(a.by_group).of(row);
  token = token < (uint32_t)q.n ? token : (uint32_t)q.n - 1;
  for (uint32_t st = (from < whole ? whole : from) + (threadIdx.x >> 6); st <= to; st += 4) {
    const bool drafted = st >= cached;
    const uint32_t first = drafted ? (st - cached) * kStep : st * kStep, end = (uint32_t)(drafted ? q.n : q.len);
    const uint32_t key = first + (lane >> 1) < end ? first + (lane >> 1) : end - 1;
    const uint16_t *v;
    if (drafted) {
      v = static_cast<const uint16_t *>(a.t.v) + ((uint64_t)q.start + key) * a.t.v_token_stride + head * a.t.v_head_stride;
    } else {
      const uint32_t block = divisor(a.c.page_tokens).of(key), page = (uint32_t)a.t.table[(uint64_t)r * a.t.blocks + block];
      v = reinterpret_cast<const uint16_t *>(a.c.v) + (page < a.c.pages ? page : 0) * a.c.page_stride + (key - block * a.c.page_tokens.d) * a.c.token_stride +
          head * a.c.head_stride;
    }
    uint32_t any = 0;
    for (uint32_t d = 8 * (lane & 1); d < a.c.dim; d += 16) {
      const Words4 w = load16(v + d);
#pragma unroll
      for (int y = 0; y < 4; ++y) any |= not_finite<T>(w[y]);
    }
    uint32_t sees = ~0u;
    if (drafted && a.t.mask != nullptr) {
      sees = reinterpret_cast<const uint32_t *>(a.t.mask)[((uint64_t)q.start + token) * 2 * a.t.mask_words + (st - cached)];
    } else if (drafted) {
      const int d = (int)token - (int)first;
      sees = d < 0 ? 0 : d >= 31 ? ~0u : (2u << d) - 1;
    }
    for (uint64_t found = __ballot(any != 0 && first + (lane >> 1) < end); found != 0;) {
      const int i = __builtin_ctzll(found) >> 1;
      found &= ~(3ull << 2 * i);
      const uint16_t *values = reinterpret_cast<const uint16_t *>(from_lane(reinterpret_cast<uintptr_t>(v), 2 * i)) + 4 * E * g;
      const bool seen = (sees >> i & 1) != 0;
#pragma unroll
      for (int x = 0; x < E / 2; ++x) {
        Words4 w{0, 0, 0, 0};
        if (seen && 4 * E * g + 8 * x < (int)a.c.dim) w = load16(values + 8 * x);
#pragma unroll
        for (int y = 0; y < 8; ++y) {  // element E k + j of the lane's 4 E
          const uint16_t bits = (uint16_t)(w[y / 2] >> (y % 2 * 16));
          acc[(8 * x + y) % E][(8 * x + y) / E] += (bits & T::kExponent) == T::kExponent ? T::to_float(bits) : 0;
        }
      }
    }
  }
}

// What add_left_out has found, on top of a result that is in place already.
template <class T, int DT, class A>
__device__ inline void add_to_row(const A &a, const Floats4 (&acc)[DT / 16], const Request &q, uint32_t row, uint32_t kv_head, int g) {
  constexpr int E = DT / 16;
  const uint32_t token = divisor(a.by_group).of(row), head = kv_head * a.group + (row - token * a.group);
  if ((int)token >= q.n) return;
  uint16_t *out = static_cast<uint16_t *>(a.t.out) + ((uint64_t)q.start + token) * a.t.out_token_stride + head * a.t.out_head_stride + 4 * E * g;
#pragma unroll
  for (int j = 0; j < E; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (acc[j][i] != 0) out[E * i + j] = T::from_float(T::to_float(out[E * i + j]) + acc[j][i]);
}

// The sums of segments that several workers share, 16 rows to a workgroup, whose wavefronts take every fourth worker's each. A kernel of its own: 5 to 8
// us, most of them its start and three dependent reads; done by the worker that comes last it would need each one's sums written past its
// die's cache, and counters cleared before each call.
template <class T, int DT, int NR, int WR>
__global__ __launch_bounds__(256) void ft_tree_join_kernel(Tree) {
  const auto &a = *argument();
  constexpr int E = DT / 16, ROWS = 16 * NR * WR;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g = lane >> 4;
  __shared__ float top[16][16], total[4][16];
  __shared__ Floats4 join[3][E][64];
  const uint32_t r = blockIdx.x / a.c.heads, head = blockIdx.x - r * a.c.heads;
  const uint32_t tile = blockIdx.y / (NR * WR), part = blockIdx.y - tile * (NR * WR);
  const Request q = request(a, r);
  const uint32_t tiles = ((uint32_t)q.n * a.group + ROWS - 1) / ROWS;
  if (tile >= tiles || tile * ROWS + part * 16 >= (uint32_t)q.n * a.group) return;
  const uint32_t steps = steps_of(q);
  const uint64_t rate = a.prefix[a.t.requests], groups = (tiles + a.cluster - 1) / a.cluster;
  const uint64_t begin = a.prefix[r] + ((uint64_t)head * groups + tile / a.cluster) * (steps + kSegment) + kSegment;
  const uint32_t w0 = worker_of(begin, rate), w1 = worker_of(begin + steps - 1, rate);
  const auto left_out_by = [&](uint32_t w) { return a.left_out[(w * a.cluster + tile % a.cluster) * WR + part / NR]; };
  const uint32_t row = tile * ROWS + part * 16 + n16;
  const auto at = [&](uint32_t w) { return a.sums + ((((uint64_t)w * 2 + (w == w0 ? 1 : 0)) * a.cluster + tile % a.cluster) * (WR * NR) + part) * Partial<DT>::kTile; };
  float now = -INFINITY, l = 0;
  Floats4 acc[E];
#pragma unroll
  for (int j = 0; j < E; ++j) acc[j] = Floats4{0, 0, 0, 0};
  // of what the workers have left out, in all that they did, the steps of this segment
  const auto with_left_out = [&] {
    const uint64_t all = a.prefix[a.t.requests + 1];
    uint64_t lo = ~0ull, hi = 0;
    for (uint32_t w = w0; w <= w1; ++w) {
      const LeftOut out = left_out_by(w);
      const uint64_t end = begin_of(w + 1, rate) < all ? begin_of(w + 1, rate) : all;
      if (out.first == 0) continue;
      const uint64_t first = out.first == ~0u ? 0 : end - out.first, last = end - out.last;
      lo = first < lo ? first : lo;
      hi = last > hi ? last : hi;
    }
    lo = lo < begin ? begin : lo;
    hi = hi < begin + steps - 1 ? hi : begin + steps - 1;
    if (lo <= hi) add_left_out<T, DT>(a, q, r, row, head, (uint32_t)(lo - begin), (uint32_t)(hi - begin), acc);
  };
  // the wavefronts' sums to the first one
  const auto gather = [&] {
    if (g == 0) total[wave][n16] = l;
    if (wave != 0)
#pragma unroll
      for (int j = 0; j < E; ++j) join[wave - 1][j][lane] = acc[j];
    __syncthreads();
    if (wave != 0) return;
    l = ((total[0][n16] + total[1][n16]) + total[2][n16]) + total[3][n16];
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] += join[w][j][lane];
  };
  if (w0 == w1) {  // the result is in place
    if (left_out_by(w0).first == 0) return;
    with_left_out();
    gather();
    if (wave == 0) add_to_row<T, DT>(a, acc, q, row, head, g);
    return;
  }
  bool left_out = false;
  for (uint32_t w = w0 + (threadIdx.x >> 4); w <= w1; w += 16) {
    now = fmaxf(now, at(w)[16 * DT + n16]);
    left_out |= left_out_by(w).first != 0;
  }
  top[threadIdx.x >> 4][n16] = now;
  left_out = __syncthreads_or(left_out);
  for (int i = 0; i < 16; ++i) now = fmaxf(now, top[i][n16]);
  const float from = now == -INFINITY ? 0 : now;
  for (uint32_t w = w0 + wave; w <= w1; w += 4) {
    const float *sums = at(w);
    const float shrink = __builtin_amdgcn_exp2f(sums[16 * DT + n16] - from);
    l += sums[16 * DT + 16 + n16] * shrink;
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] += reinterpret_cast<const Floats4 *>(sums)[j * 64 + lane] * shrink;
  }
  if (left_out) with_left_out();
  gather();
  if (wave == 0) write_row<T, DT>(a, acc, l, now, q, row, head, g);
}

struct Shape {
  int dt, nr, wr;
  bool shared;
  uint32_t cluster;
};

// Heads are padded to 64, 128 or 256 elements. Four wavefronts of 16 rows share keys and values in shared memory, also where there are fewer
// rows: a wavefront to itself, with four times the workers, takes 121 us instead of 105 for 64 requests of 2000 tokens and 4 rows a key head (8
// key heads of 128), 46 instead of 33 for one of 20000, 28 and 21 for 17 of 700, 74 and 70 for 64 of 16 to 8192; it is faster only where there is next
// to nothing to do (13 instead of 13.8 for one of 300). Beyond 64 rows, 16 requests of 4096: eight wavefronts
// of 16 rows take 77 us for 96 rows, four 84, eight of 32 rows 98; for 192 rows 124, 142 and 102. With heads of 64 elements four of 32 rows do what
// eight do there (43 for 96 and 128). Beyond that up to four workgroups share the die's cache: 384 instead of 394 for 64 requests of 2000 and 512 rows,
// 259 instead of 274 with heads of 64. Heads of 256 do not leave registers for what is on its way to shared memory.
Shape shape_of(uint32_t dim, uint64_t rows) {
  const int dt = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
  if (dt == 256) return {dt, 1, rows <= 16 ? 1 : 4, false, 1};
  if (rows <= 64) return {dt, 1, 4, true, 1};
  if (rows <= 128 && dt == 128) return {dt, 1, 8, true, 1};
  const int most = dt == 64 ? 4 : 8;
  const uint64_t tiles = (rows + 32 * most - 1) / (32 * most);
  return {dt, 2, most, true, tiles > 4 ? 4 : (uint32_t)tiles};
}

// As many as the chip holds, a multiple of its dies.
uint32_t workers_of(const Shape &s, int cu_count) {
  return (uint32_t)(cu_count * 4 * waves(s.dt) / (s.wr * (int)s.cluster) + 7) / 8 * 8;
}

// Wavefronts of all workers, at most: workers are rounded up to the dies.
uint64_t waves_of(const Shape &s, int cu_count) { return (uint64_t)cu_count * 4 * waves(s.dt) + 256; }

uint64_t up16(uint64_t v) { return (v + 15) / 16 * 16; }

template <class T, int DT, int NR, int WR, bool SHARED>
hipError_t launch(const Tree &a, bool paged, uint64_t rows, hipStream_t stream) {
  const dim3 grid(a.workers * a.cluster), threads(64 * WR);
  if (paged) hipLaunchKernelGGL((ft_tree_kernel<T, DT, NR, WR, true, SHARED>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((ft_tree_kernel<T, DT, NR, WR, false, SHARED>), grid, threads, 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint64_t tiles = (rows + 16 * NR * WR - 1) / (16 * NR * WR) * NR * WR;
  hipLaunchKernelGGL((ft_tree_join_kernel<T, DT, NR, WR>), dim3(a.t.requests * a.c.heads, (uint32_t)tiles), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <class T, int DT>
hipError_t launch_rows(const Tree &a, const Shape &s, bool paged, uint64_t rows, hipStream_t stream) {
  if constexpr (DT == 256) {
    return s.wr == 1 ? launch<T, DT, 1, 1, false>(a, paged, rows, stream) : launch<T, DT, 1, 4, false>(a, paged, rows, stream);
  } else {
    if (s.nr == 1 && s.wr == 4) return launch<T, DT, 1, 4, true>(a, paged, rows, stream);
    if constexpr (DT == 64) return launch<T, DT, 2, 4, true>(a, paged, rows, stream);
    else return s.nr == 1 ? launch<T, DT, 1, 8, true>(a, paged, rows, stream) : launch<T, DT, 2, 8, true>(a, paged, rows, stream);
  }
}

template <class T>
hipError_t launch_dim(const Tree &a, const Shape &s, bool paged, uint64_t rows, hipStream_t stream) {
  return s.dt == 64 ? launch_rows<T, 64>(a, s, paged, rows, stream) : s.dt == 128 ? launch_rows<T, 128>(a, s, paged, rows, stream)
                                                                                 : launch_rows<T, 256>(a, s, paged, rows, stream);
}

uint64_t rows_of(const ft_tree_call &t, uint32_t heads) {
  const uint64_t n = t.drafts < t.tokens ? t.drafts : t.tokens;
  return n * (t.heads / heads);
}

}  // namespace

uint64_t tree_workspace(const ft_kv_cache &c, const ft_tree_call &t, int cu_count) {
  const Shape s = shape_of(c.dim, rows_of(t, c.heads));
  return up16(((uint64_t)t.requests + 2) * 8) + waves_of(s, cu_count) * (sizeof(LeftOut) + 2ull * s.nr * (16 * s.dt + 32) * 4);
}

hipError_t launch_tree(const KvView &c, const ft_tree_call &t, int cu_count, hipStream_t stream) {
  const uint64_t rows = rows_of(t, c.heads);
  const Shape s = shape_of(c.dim, rows);
  Tree a{c, t};
  a.t.drafts = t.drafts < t.tokens ? t.drafts : t.tokens;
  // Pages of whole 16 keys, heads without padding, strides of 24 bits in bytes: one base address for 16 keys (57 us for 16 requests of 4096 tokens
  // and 64 rows, 66 without; 16 rows of 64 elements 34 both).
  const bool paged = c.dim == (uint32_t)s.dt && c.page_tokens.d % 16 == 0 && (c.token_stride | t.k_token_stride | t.v_token_stride) < 1u << 23;
  a.cluster = s.cluster;
  a.workers = workers_of(s, cu_count);
  a.group = t.heads / c.heads;
  a.by_group = Divisor(a.group);
  a.least = kSegment + 1;  // (17 requests of up to 1500 tokens: 16.3 us, with a step more 17.9, with four 19.3; 5 of up to 400 14.6, with three more 16.7)
  // Scores are scaled within the exponent's argument, so a scale of 0 must not make NaN of what is masked: the smallest number there is
  // does the same. Queries change their signs for one below 0, as the largest product is to be the largest score.
  a.scale = fabsf(t.scale * kLog2e);
  if (a.scale == 0) a.scale = 0x1p-149f;
  a.flip = t.scale < 0 ? 0x80008000u : 0;
  a.prefix = static_cast<uint64_t *>(t.workspace);
  a.left_out = reinterpret_cast<LeftOut *>(static_cast<char *>(t.workspace) + up16(((uint64_t)t.requests + 2) * 8));
  a.sums = reinterpret_cast<float *>(a.left_out + waves_of(s, cu_count));
  return c.type == FT_BF16 ? launch_dim<Bf16>(a, s, paged, rows, stream) : launch_dim<Fp16>(a, s, paged, rows, stream);
}

}  // namespace ft
