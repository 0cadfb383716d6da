// Launchers of the operators on pool memory (ft_kv.hip, ft_tree.hip, ft_adapters.hip), private to the library. Their callers
// (ft_operators.cpp) have checked the arguments.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "../../include/faastube.h"

namespace ft {

// n / d for n < 2^31 by a multiplication: with 2^(s-1) < d <= 2^s, m = floor(2^(31+s) / d) + 1 exceeds 2^(31+s) / d by e <= 1, and
// n * m / 2^(31+s) exceeds n / d by n * e / 2^(31+s) < 2^-s <= 1 / d: too little to reach the next whole number.
struct Divisor {
  uint32_t d = 1, m = 0, shift = 0;
  Divisor() = default;
  explicit Divisor(uint32_t by) : d(by) {
    uint32_t s = 0;
    while ((1ull << s) < by) ++s;
    if (by > 1) {
      m = (uint32_t)((1ull << (31 + s)) / by + 1);
      shift = s - 1;
    }
  }
  __host__ __device__ uint32_t of(uint32_t n) const { return d == 1 ? n : above_one(n); }
  __host__ __device__ uint32_t above_one(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> 32) >> shift; }  // where d > 1
  __host__ __device__ uint32_t rest(uint32_t n) const { return n - of(n) * d; }
};

// A cache with its pool offsets resolved.
struct KvView {
  char *k, *v;
  uint32_t type, pages, heads, dim;
  Divisor page_tokens;
  uint64_t page_stride, token_stride, head_stride;
};

hipError_t launch_kv_grow(const ft_kv_tables &t, const int32_t *starts, const uint8_t *keep, uint32_t tokens, int64_t *slots, int32_t *lens_out,
                          int32_t *state_out, hipStream_t stream);
hipError_t launch_kv_release(const ft_kv_tables &t, const uint8_t *done, int32_t *lens_out, int32_t *state_out, hipStream_t stream);
hipError_t launch_kv_append(const KvView &c, const void *k, const void *v, uint64_t k_token, uint64_t k_head, uint64_t v_token, uint64_t v_head,
                            const int64_t *slots, uint32_t tokens, hipStream_t stream);

uint64_t tree_workspace(const ft_kv_cache &c, const ft_tree_call &call, int cu_count);
hipError_t launch_tree(const KvView &c, const ft_tree_call &call, int cu_count, hipStream_t stream);

uint64_t adapter_tiles(uint32_t rows, uint32_t count);  // at most: workgroups of 256 threads along the first axis of the products' grids
uint64_t adapter_group_bytes(uint32_t rows, uint32_t count);
hipError_t launch_adapter_group(const int32_t *ids, uint32_t rows, uint32_t count, void *groups, hipStream_t stream);
uint64_t adapter_workspace(const ft_adapters_call &call);
hipError_t launch_adapters(const ft_adapters_call &call, hipStream_t stream);

}  // namespace ft
