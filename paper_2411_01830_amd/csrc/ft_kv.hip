// Pages and slots of a step's tokens from the requests' lengths, pages given back, and tokens written to their slots.
#include <hip/hip_runtime.h>

#include "ft_operators.h"

namespace ft {

namespace {

constexpr int kThreads = 1024;  // and requests looked at together
constexpr int kWaves = kThreads / 64;

// Sums over the threads before this one, and all of them. Two quantities in one go: a launch of few requests is nothing but this.
struct Sums {
  uint64_t pages, items;  // (requests whose rows overlap, as starts that descend make them, have more of either than 32 bits count)
};

__device__ inline Sums scan(uint64_t pages, uint32_t items, Sums *before, Sums *lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t p = pages;
  uint32_t i = items;  // at most 2^25 a thread, so those of a wavefront have room
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t q = __shfl_up(p, d);
    const uint32_t j = __shfl_up(i, d);
    if (lane >= d) {
      p += q;
      i += j;
    }
  }
  if (lane == 63) lds[wave] = {p, i};
  __syncthreads();
  Sums all{0, 0}, front{0, 0};
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) front = all;
    all.pages += lds[w].pages;
    all.items += lds[w].items;
  }
  *before = {front.pages + p - pages, front.items + i - items};
  return all;
}

// The request whose items [at[r], at[r + 1]) contain i: the last r with at[r] <= i that has any. at ascends; n of them are looked at.
__device__ inline int owner(const uint64_t *at, int n, uint64_t i) {
  int lo = 0, hi = n;  // at[lo] <= i < at[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ inline int32_t clamped(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ inline uint32_t pages_of(int32_t tokens, const Divisor &page) { return tokens <= 0 ? 0 : page.of((uint32_t)tokens - 1) + 1; }

struct GrowLds {
  Sums wave[kWaves];
  uint64_t first[kThreads];  // pages taken by the requests before
  uint64_t item[kThreads];   // blocks of 64 rows of the requests before
  int32_t row[kThreads], count[kThreads], len[kThreads], added[kThreads];
  unsigned long long taken;
  uint32_t refused;
};

// A prefix sum over the requests of the pages that they lack, then 64 rows to a wavefront. Every workgroup does the whole sum for
// itself, which costs it a few microseconds of reads from the caches and saves a second launch; the rows are shared out. Latency bounds it:
// lengths, flags, two barriers of the sum, table, slot, each waited for. 7.6 us for 64 trees of 16 with flags, 6.7 for 256 prompts
// of up to 512 rows.
__global__ __launch_bounds__(kThreads) void ft_kv_grow_kernel(ft_kv_tables t, Divisor page, const int32_t *__restrict__ starts,
                                                              const uint8_t *__restrict__ keep, uint32_t tokens, int64_t *__restrict__ slots,
                                                              int32_t *__restrict__ lens_out, int32_t *__restrict__ state_out) {
  __shared__ GrowLds s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t top = clamped(t.state[0], 0, (int32_t)t.pages);
  const int32_t rows = (int32_t)tokens;
  uint64_t asked = 0;  // pages that the requests so far lack
  if (threadIdx.x == 0) {
    s.taken = 0;
    s.refused = 0;
  }
  for (uint32_t r0 = 0; r0 < t.requests; r0 += kThreads) {
    const uint32_t r = r0 + threadIdx.x;
    const bool mine = r < t.requests;
    __syncthreads();  // the tables of the requests before are no longer read
    int32_t row = 0, count = 0, len = 0;
    if (mine) {
      row = clamped(starts[r], 0, rows);
      count = clamped(starts[r + 1], row, rows) - row;
      len = t.lens[r];
    }
    s.row[threadIdx.x] = row;
    s.count[threadIdx.x] = count;
    if (keep != nullptr) {
      __syncthreads();
      const int n = (int)(t.requests - r0 < kThreads ? t.requests - r0 : kThreads);
      // four requests of a wavefront at a time, so that their flags are on their way together
      for (int q0 = wave; q0 < n; q0 += 4 * kWaves) {
        uint8_t flag[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int q = q0 + k * kWaves < n ? q0 + k * kWaves : q0;
          flag[k] = lane < s.count[q] ? keep[s.row[q] + lane] : 0;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int q = q0 + k * kWaves;
          if (q >= n) break;
          int32_t kept = __popcll(__ballot(flag[k] != 0));
          const uint32_t rows_of = (uint32_t)s.count[q];
          for (uint32_t i = 64; i < rows_of; i += 64) kept += __popcll(__ballot(i + lane < rows_of && keep[s.row[q] + i + lane] != 0));
          if (lane == 0) s.added[q] = kept;
        }
      }
      __syncthreads();
    }
    const int32_t added = keep != nullptr ? (mine ? s.added[threadIdx.x] : 0) : count;
    // a length below zero, or beyond what the table's rows name, is refused; sums of two such numbers need 33 bits
    const int64_t after = (int64_t)len + added;
    const bool fits = mine && len >= 0 && after <= 0x7fffffff && pages_of((int32_t)after, page) <= t.blocks;
    const uint32_t have = fits ? pages_of(len, page) : 0, want = fits ? pages_of((int32_t)after, page) : 0;
    Sums before;
    const Sums all = scan(want - have, ((uint32_t)count + 63) >> 6, &before, s.wave);
    const uint64_t first = asked + before.pages, end = first + (want - have);
    const bool served = fits && (want == have || end <= (uint64_t)top);
    s.first[threadIdx.x] = first;
    s.item[threadIdx.x] = before.items;
    s.len[threadIdx.x] = len;
    s.added[threadIdx.x] = served ? (int32_t)have : -1;
    if (blockIdx.x == 0 && mine) {
      lens_out[r] = served ? (int32_t)after : len;
      if (served && want != have) atomicMax(&s.taken, (unsigned long long)end);
      if (!served) atomicAdd(&s.refused, 1u);
    }
    asked += all.pages;
    __syncthreads();
    for (uint64_t i = blockIdx.x * kWaves + wave; i < all.items; i += gridDim.x * kWaves) {
      const int q = owner(s.item, kThreads, i);
      const int32_t begin = (int32_t)(i - s.item[q]) << 6, n = s.count[q], at = begin + lane, pages = s.added[q];
      const bool there = at < n;
      const int32_t token = s.row[q] + (there ? at : 0);
      int32_t rank = at;
      bool kept = there;
      if (keep != nullptr) {
        rank = 0;
        for (int32_t j = lane; j < begin; j += 64) rank += __popcll(__ballot(keep[s.row[q] + j] != 0));
        kept = there && keep[token] != 0;
        rank += __popcll(__ballot(kept) & ((1ull << lane) - 1));
      }
      int64_t slot = -1;
      if (kept && pages >= 0) {
        const uint32_t pos = (uint32_t)(s.len[q] + rank), block = page.of(pos), in_page = pos - block * page.d;
        int32_t *entry = t.table + (uint64_t)(r0 + q) * t.blocks + block;
        int32_t id;
        if ((int32_t)block < pages) {
          id = *entry;
        } else {
          id = t.free_pages[top - 1 - (int32_t)(s.first[q] + (block - (uint32_t)pages))];
          if (in_page == 0) *entry = id;  // the page's first token is one of these
        }
        slot = (int64_t)id * page.d + in_page;
      }
      if (there) slots[token] = slot;
    }
  }
  // rows of no request
  const int32_t lo = t.requests != 0 ? clamped(starts[0], 0, rows) : rows, hi = t.requests != 0 ? clamped(starts[t.requests], lo, rows) : rows;
  const uint32_t me = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
  for (uint32_t i = me; i < (uint32_t)lo; i += step) slots[i] = -1;
  for (uint32_t i = (uint32_t)hi + me; i < tokens; i += step) slots[i] = -1;
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    state_out[0] = top - (int32_t)s.taken;
    const uint64_t missing = asked > (uint64_t)top ? asked - (uint64_t)top : 0;
    state_out[1] = missing > 0x7fffffff ? 0x7fffffff : (int32_t)missing;
    state_out[2] = (int32_t)s.refused;
    state_out[3] = 0;
  }
}

struct ReleaseLds {
  Sums wave[kWaves];
  uint64_t first[kThreads];
  uint64_t item[kThreads];
  uint32_t count[kThreads];
};

// The same sum over the pages of the requests that are done, and their entries to the stack, 64 to a wavefront: 6.2 us for 64 of 256 requests of up to
// 4096 tokens, of which the launch and four dependent reads are nearly all.
__global__ __launch_bounds__(kThreads) void ft_kv_release_kernel(ft_kv_tables t, Divisor page, const uint8_t *__restrict__ done,
                                                                 int32_t *__restrict__ lens_out, int32_t *__restrict__ state_out) {
  __shared__ ReleaseLds s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t top = clamped(t.state[0], 0, (int32_t)t.pages);
  uint64_t given = 0;
  for (uint32_t r0 = 0; r0 < t.requests; r0 += kThreads) {
    const uint32_t r = r0 + threadIdx.x;
    __syncthreads();
    uint32_t pages = 0;
    if (r < t.requests) {
      const int32_t len = t.lens[r];
      const bool gone = done[r] != 0;
      if (gone) pages = pages_of(len, page);
      if (pages > t.blocks) pages = t.blocks;
      if (blockIdx.x == 0) lens_out[r] = gone ? 0 : len;
    }
    Sums before;
    const Sums all = scan(pages, (pages + 63) >> 6, &before, s.wave);
    s.first[threadIdx.x] = given + before.pages;
    s.item[threadIdx.x] = before.items;
    s.count[threadIdx.x] = pages;
    given += all.pages;
    __syncthreads();
    for (uint64_t i = blockIdx.x * kWaves + wave; i < all.items; i += gridDim.x * kWaves) {
      const int q = owner(s.item, kThreads, i);
      const uint32_t b = ((uint32_t)(i - s.item[q]) << 6) + lane;
      const uint64_t to = (uint64_t)top + s.first[q] + b;
      if (b < s.count[q] && to < t.pages) t.free_pages[to] = t.table[(uint64_t)(r0 + q) * t.blocks + b];
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const uint64_t now = (uint64_t)top + given;
    state_out[0] = now > t.pages ? (int32_t)t.pages : (int32_t)now;
    state_out[1] = state_out[2] = state_out[3] = 0;
  }
}

// 16 bytes at any element's address: the memory pipeline splits what straddles.
struct __attribute__((packed, aligned(2))) Vec {
  uint32_t w[4];
};

// Past the caches: what is appended is read by the next step at the earliest (269 MB read and written 52 -> 49 us, 2 MB the same).
__device__ inline void store_once(char *p, const Vec &v) {
  typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
  typedef __attribute__((address_space(1))) Words *Global;
  __builtin_nontemporal_store(Words{v.w[0], v.w[1], v.w[2], v.w[3]}, reinterpret_cast<Global>(reinterpret_cast<uintptr_t>(p)));
}

// A row's heads are cut into vectors of 8 elements, a vector of keys and one of values to a thread. Memory bounds it where there are many rows: 32773 rows
// of 8 heads of 128 elements in 49 us, 5.5 TB/s read and written (a large copy: 5.1); 1024 of which a fifth are kept take 4, the launch.
__global__ __launch_bounds__(256) void ft_kv_append_kernel(KvView c, const uint16_t *__restrict__ k, const uint16_t *__restrict__ v, uint64_t k_token,
                                                           uint64_t k_head, uint64_t v_token, uint64_t v_head, const int64_t *__restrict__ slots,
                                                           uint32_t tokens, Divisor row_vectors, Divisor head_vectors) {
  const uint64_t all = (uint64_t)tokens * row_vectors.d, slots_there = (uint64_t)c.pages * c.page_tokens.d;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256) {
    const uint32_t token = (uint32_t)(i / row_vectors.d), at = (uint32_t)(i - (uint64_t)token * row_vectors.d);
    const int64_t slot = slots[token];
    if (slot < 0 || (uint64_t)slot >= slots_there) continue;
    const uint32_t head = head_vectors.of(at), d = (at - head * head_vectors.d) * 8;
    const uint32_t p = c.page_tokens.of((uint32_t)slot), in_page = (uint32_t)slot - p * c.page_tokens.d;
    const uint64_t to = 2 * (p * c.page_stride + in_page * c.token_stride + head * c.head_stride + d);
    const Vec a = *reinterpret_cast<const Vec *>(k + token * k_token + head * k_head + d);
    const Vec b = *reinterpret_cast<const Vec *>(v + token * v_token + head * v_head + d);
    store_once(c.k + to, a);
    store_once(c.v + to, b);
  }
}

}  // namespace

hipError_t launch_kv_grow(const ft_kv_tables &t, const int32_t *starts, const uint8_t *keep, uint32_t tokens, int64_t *slots, int32_t *lens_out,
                          int32_t *state_out, hipStream_t stream) {
  const uint64_t items = tokens / 64 + (uint64_t)t.requests, each = (items + kWaves - 1) / kWaves;  // blocks of 64 rows, at most; one to a wavefront
  const uint32_t wg = each < 1 ? 1 : each > 256 ? 256 : (uint32_t)each;
  hipLaunchKernelGGL(ft_kv_grow_kernel, dim3(wg), dim3(kThreads), 0, stream, t, Divisor(t.page_tokens), starts, keep, tokens, slots, lens_out, state_out);
  return hipGetLastError();
}

hipError_t launch_kv_release(const ft_kv_tables &t, const uint8_t *done, int32_t *lens_out, int32_t *state_out, hipStream_t stream) {
  const uint32_t wg = t.requests / 64 < 1 ? 1 : t.requests / 64 > 64 ? 64 : t.requests / 64;
  hipLaunchKernelGGL(ft_kv_release_kernel, dim3(wg), dim3(kThreads), 0, stream, t, Divisor(t.page_tokens), done, lens_out, state_out);
  return hipGetLastError();
}

hipError_t launch_kv_append(const KvView &c, const void *k, const void *v, uint64_t k_token, uint64_t k_head, uint64_t v_token, uint64_t v_head,
                            const int64_t *slots, uint32_t tokens, hipStream_t stream) {
  const Divisor head(c.dim / 8), row(c.heads * (c.dim / 8));
  const uint64_t wg = ((uint64_t)tokens * row.d + 255) / 256;
  hipLaunchKernelGGL(ft_kv_append_kernel, dim3((uint32_t)(wg > 1u << 16 ? 1u << 16 : wg)), dim3(256), 0, stream, c, static_cast<const uint16_t *>(k),
                     static_cast<const uint16_t *>(v), k_token, k_head, v_token, v_head, slots, tokens, row, head);
  return hipGetLastError();
}

}  // namespace ft
