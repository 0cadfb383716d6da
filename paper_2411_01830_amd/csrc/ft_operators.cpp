// C entry points of the operators on pool memory: argument checks, pool offsets to device addresses, launches on the
// caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>
#include <mutex>

#include "ft_guard.h"
#include "ft_internal.h"
#include "ft_operators.h"

using namespace ft;

namespace {

constexpr uint64_t kMostStride = 1ull << 40;

bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool there(const void *p, uintptr_t to) { return p != nullptr && aligned(p, to); }

// Bytes from the first element of either half of a cache to behind its last; 0: malformed.
uint64_t cache_extent(const ft_kv_cache &c) {
  if (c.type > FT_FP16 || c.pages == 0 || c.page_tokens == 0 || c.heads == 0) return 0;
  if (c.dim == 0 || c.dim > 256 || c.dim % 8 != 0 || c.k % 2 != 0 || c.v % 2 != 0) return 0;
  if ((uint64_t)c.pages * c.page_tokens >= 1ull << 31 || c.heads > 1u << 16) return 0;
  unsigned __int128 elements = c.dim;
  const uint64_t counts[3] = {c.pages, c.page_tokens, c.heads}, strides[3] = {c.page_stride, c.token_stride, c.head_stride};
  for (int i = 0; i < 3; ++i) {
    if (counts[i] == 1) continue;
    if (strides[i] < c.dim || strides[i] >= kMostStride) return 0;
    elements += (unsigned __int128)(counts[i] - 1) * strides[i];
  }
  return elements > (1ull << 60) ? 1ull << 61 : (uint64_t)elements * 2;
}

// Called with the pool's mutex held. Device address of [off, off + bytes), or null if it is not inside one live allocation.
char *resolve(ft_pool *p, uint64_t off, uint64_t bytes) {
  SlabPool::Place near = p->slabs.begin();
  const SlabPool::Entry *e = p->slabs.find(off, bytes, &near);
  return e == nullptr ? nullptr : reinterpret_cast<char *>(e->dev + (off - e->start));
}

// Called with the pool's mutex held.
int resolve_cache(ft_pool *p, const ft_kv_cache &c, KvView *out) {
  const uint64_t extent = cache_extent(c);
  if (extent == 0) return FT_EINVAL;
  out->k = resolve(p, c.k, extent);
  out->v = resolve(p, c.v, extent);
  if (out->k == nullptr || out->v == nullptr) return FT_ERANGE;
  out->type = c.type;
  out->pages = c.pages;
  out->heads = c.heads;
  out->dim = c.dim;
  out->page_tokens = Divisor(c.page_tokens);
  out->page_stride = c.page_stride;
  out->token_stride = c.token_stride;
  out->head_stride = c.head_stride;
  return FT_OK;
}

int compute_units(ft_pool *p, int *out) {
  static std::mutex mu;
  static std::unordered_map<int, int> known;
  std::lock_guard<std::mutex> lock(mu);
  auto it = known.find(p->device);
  if (it == known.end()) {
    int n = 0;
    FT_HIP(p, hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, p->device));
    if (n <= 0) {
      p->hip_error = "no compute units reported";
      return FT_EHIP;
    }
    it = known.emplace(p->device, n).first;
  }
  *out = it->second;
  return FT_OK;
}

// Without requests the state alone is read.
bool good_tables(const ft_kv_tables &t) {
  if (!there(t.state, 4) || t.pages >= 1u << 31 || t.page_tokens == 0 || (uint64_t)t.pages * t.page_tokens >= 1ull << 31) return false;
  if (t.requests == 0) return true;
  if (!there(t.lens, 4) || !there(t.table, 4) || !there(t.free_pages, 4)) return false;
  return t.blocks != 0 && t.pages != 0 && t.requests < 1u << 24;
}

bool good_strides(std::initializer_list<uint64_t> strides) {
  for (uint64_t s : strides)
    if (s >= kMostStride) return false;
  return true;
}

// A grid holds less than 2^32 threads along its first axis, and 2^16 workgroups along the others.
constexpr uint64_t kMostWorkgroups = (1ull << 32) / 256;

// What of a call is wrong whatever its pointers are.
bool good_numbers(const ft_kv_cache &c, const ft_tree_call &t) {
  if (t.drafts == 0 || t.requests > 1u << 24 || t.tokens >= 1u << 31 || t.drafts >= 1u << 31 || t.heads == 0 || t.heads % c.heads != 0) return false;
  if (t.heads > 1u << 16 || t.blocks > 1u << 31 || !std::isfinite(t.scale * 1.4426951f)) return false;  // (scores are kept in powers of two)
  const uint64_t drafts = t.drafts < t.tokens ? t.drafts : t.tokens;
  // the second launch has a workgroup to a request's key head, and 16 rows of them along the other axis
  return drafts * (t.heads / c.heads) < 1u << 20 && (uint64_t)t.requests * c.heads < kMostWorkgroups;
}

bool good_numbers(const ft_adapters_call &a) {
  if (a.type > FT_FP16 || a.count == 0 || a.count > 1u << 14 || a.width_in == 0 || a.width_out == 0 || a.rows >= 1u << 31) return false;
  if (a.width_in >= 1u << 24 || a.width_out >= 1u << 24) return false;
  if (a.rows != 0 && adapter_tiles(a.rows, a.count) >= kMostWorkgroups) return false;
  return a.max_rank >= 1 && a.max_rank <= 256;
}

}  // namespace

extern "C" {

int ft_kv_grow(ft_pool *p, const ft_kv_tables *t, const int32_t *starts, const uint8_t *keep, uint32_t tokens, int64_t *slots, int32_t *lens_out,
               int32_t *state_out, void *hip_stream) try {
  if (p == nullptr || t == nullptr) return FT_EINVAL;
  if (t->requests == 0 && tokens == 0 && state_out == nullptr) return FT_OK;
  if (!good_tables(*t)) return FT_EINVAL;
  if (t->requests != 0 && (!there(starts, 4) || !there(lens_out, 4) || lens_out == t->lens)) return FT_EINVAL;
  if (!there(state_out, 4) || state_out == t->state || tokens >= 1u << 31 || (tokens != 0 && !there(slots, 8))) return FT_EINVAL;
  std::lock_guard<std::mutex> lock(p->mu);
  DeviceGuard guard(p->device);
  FT_HIP(p, launch_kv_grow(*t, starts, keep, tokens, slots, lens_out, state_out, static_cast<hipStream_t>(hip_stream)));
  return FT_OK;
}
FT_CATCH_ALL

int ft_kv_release(ft_pool *p, const ft_kv_tables *t, const uint8_t *done, int32_t *lens_out, int32_t *state_out, void *hip_stream) try {
  if (p == nullptr || t == nullptr) return FT_EINVAL;
  if (t->requests == 0 && state_out == nullptr) return FT_OK;
  if (!good_tables(*t)) return FT_EINVAL;
  if (t->requests != 0 && (done == nullptr || !there(lens_out, 4) || lens_out == t->lens)) return FT_EINVAL;
  if (!there(state_out, 4) || state_out == t->state) return FT_EINVAL;
  std::lock_guard<std::mutex> lock(p->mu);
  DeviceGuard guard(p->device);
  FT_HIP(p, launch_kv_release(*t, done, lens_out, state_out, static_cast<hipStream_t>(hip_stream)));
  return FT_OK;
}
FT_CATCH_ALL

int ft_kv_append(ft_pool *p, const ft_kv_cache *c, const void *k, const void *v, uint64_t k_token_stride, uint64_t k_head_stride,
                 uint64_t v_token_stride, uint64_t v_head_stride, const int64_t *slots, uint32_t tokens, void *hip_stream) try {
  if (p == nullptr || c == nullptr || cache_extent(*c) == 0 || tokens >= 1u << 31) return FT_EINVAL;
  if (tokens != 0 && (!there(k, 2) || !there(v, 2) || !there(slots, 8))) return FT_EINVAL;
  if (!good_strides({k_token_stride, k_head_stride, v_token_stride, v_head_stride})) return FT_EINVAL;
  std::lock_guard<std::mutex> lock(p->mu);
  KvView view;
  const int rc = resolve_cache(p, *c, &view);
  if (rc != FT_OK) return rc;
  if (tokens == 0) return FT_OK;
  DeviceGuard guard(p->device);
  FT_HIP(p, launch_kv_append(view, k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots, tokens,
                             static_cast<hipStream_t>(hip_stream)));
  return FT_OK;
}
FT_CATCH_ALL

int ft_tree_workspace(ft_pool *p, const ft_kv_cache *c, const ft_tree_call *call, uint64_t *bytes_out) try {
  if (p == nullptr || c == nullptr || call == nullptr || bytes_out == nullptr || cache_extent(*c) == 0) return FT_EINVAL;
  if (call->tokens == 0 || call->requests == 0) {
    *bytes_out = 0;
    return FT_OK;
  }
  if (!good_numbers(*c, *call)) return FT_EINVAL;
  std::lock_guard<std::mutex> lock(p->mu);
  int cu_count = 0;
  const int rc = compute_units(p, &cu_count);
  if (rc != FT_OK) return rc;
  *bytes_out = tree_workspace(*c, *call, cu_count);
  return FT_OK;
}
FT_CATCH_ALL

int ft_tree_attention(ft_pool *p, const ft_kv_cache *c, const ft_tree_call *call, void *hip_stream) try {
  if (p == nullptr || c == nullptr || call == nullptr || cache_extent(*c) == 0) return FT_EINVAL;
  const ft_tree_call &t = *call;
  const bool any = t.tokens != 0 && t.requests != 0;
  if (any) {
    if (!good_numbers(*c, t)) return FT_EINVAL;
    if (!there(t.q, 2) || !there(t.k, 2) || !there(t.v, 2) || !there(t.out, 2) || !aligned(t.lse, 4) || !aligned(t.mask, 8)) return FT_EINVAL;
    if (!there(t.starts, 4) || !there(t.lens, 4) || (t.blocks != 0 && !there(t.table, 4))) return FT_EINVAL;
    if (t.mask != nullptr && 64ull * t.mask_words < t.drafts) return FT_EINVAL;
    if (!good_strides({t.q_token_stride, t.q_head_stride, t.k_token_stride, t.k_head_stride, t.v_token_stride, t.v_head_stride, t.out_token_stride,
                       t.out_head_stride}))
      return FT_EINVAL;
  }
  std::lock_guard<std::mutex> lock(p->mu);
  KvView view;
  int rc = resolve_cache(p, *c, &view);
  if (rc != FT_OK || !any) return rc;
  int cu_count = 0;
  rc = compute_units(p, &cu_count);
  if (rc != FT_OK) return rc;
  const uint64_t need = tree_workspace(*c, t, cu_count);
  if (need != 0 && (!there(t.workspace, 16) || t.workspace_bytes < need)) return FT_EINVAL;
  DeviceGuard guard(p->device);
  FT_HIP(p, launch_tree(view, t, cu_count, static_cast<hipStream_t>(hip_stream)));
  return FT_OK;
}
FT_CATCH_ALL

int ft_adapters_resolve(ft_pool *p, const ft_adapter *adapters, uint32_t count, uint32_t width_in, uint32_t width_out,
                        ft_adapter_record *records_out) try {
  if (p == nullptr || (count != 0 && (adapters == nullptr || records_out == nullptr))) return FT_EINVAL;
  if (width_in == 0 || width_out == 0 || width_in >= 1u << 24 || width_out >= 1u << 24) return FT_EINVAL;
  for (uint32_t i = 0; i < count; ++i) {
    const ft_adapter &a = adapters[i];
    if (a.rank == 0 || a.rank > 256 || !std::isfinite(a.scale) || a.a % 2 != 0 || a.b % 2 != 0) return FT_EINVAL;
  }
  std::lock_guard<std::mutex> lock(p->mu);
  for (int pass = 0; pass < 2; ++pass)  // nothing is written unless all of them are good
    for (uint32_t i = 0; i < count; ++i) {
      const ft_adapter &a = adapters[i];
      const char *da = resolve(p, a.a, 2ull * a.rank * width_in), *db = resolve(p, a.b, 2ull * a.rank * width_out);
      if (da == nullptr || db == nullptr) return FT_ERANGE;
      if (pass == 1) records_out[i] = {reinterpret_cast<uint64_t>(da), reinterpret_cast<uint64_t>(db), a.rank, a.scale};
    }
  return FT_OK;
}
FT_CATCH_ALL

int ft_adapters_group_bytes(uint32_t rows, uint32_t count, uint64_t *bytes_out) {
  if (bytes_out == nullptr || rows >= 1u << 31 || count == 0 || count > 1u << 14) return FT_EINVAL;
  *bytes_out = adapter_group_bytes(rows, count);
  return FT_OK;
}

int ft_adapters_group(ft_pool *p, const int32_t *ids, uint32_t rows, uint32_t count, void *groups, uint64_t groups_bytes, void *hip_stream) try {
  if (p == nullptr || rows >= 1u << 31 || count == 0 || count > 1u << 14) return FT_EINVAL;
  if (rows != 0 && !there(ids, 4)) return FT_EINVAL;
  if (!there(groups, 16) || groups_bytes < adapter_group_bytes(rows, count)) return FT_EINVAL;
  std::lock_guard<std::mutex> lock(p->mu);
  DeviceGuard guard(p->device);
  FT_HIP(p, launch_adapter_group(ids, rows, count, groups, static_cast<hipStream_t>(hip_stream)));
  return FT_OK;
}
FT_CATCH_ALL

int ft_adapters_workspace(ft_pool *p, const ft_adapters_call *call, uint64_t *bytes_out) try {
  if (p == nullptr || call == nullptr || bytes_out == nullptr || !good_numbers(*call)) return FT_EINVAL;
  *bytes_out = call->rows == 0 ? 0 : adapter_workspace(*call);
  return FT_OK;
}
FT_CATCH_ALL

int ft_adapters_apply(ft_pool *p, const ft_adapters_call *call, void *hip_stream) try {
  if (p == nullptr || call == nullptr || !good_numbers(*call)) return FT_EINVAL;
  const ft_adapters_call &a = *call;
  if (a.rows == 0) return FT_OK;
  if (!there(a.records, 8) || !there(a.groups, 16) || !there(a.x, 2) || !aligned(a.base, 2) || !there(a.out, 2)) return FT_EINVAL;
  if (a.x_stride < a.width_in || a.out_stride < a.width_out || (a.base != nullptr && a.base_stride < a.width_out)) return FT_EINVAL;
  if (!good_strides({a.x_stride, a.out_stride, a.base_stride})) return FT_EINVAL;
  if (a.out == a.base && a.out_stride != a.base_stride && a.rows > 1) return FT_EINVAL;  // a row's result would be another's base
  const uint64_t need = adapter_workspace(a);
  if (need != 0 && (!there(a.workspace, 16) || a.workspace_bytes < need)) return FT_EINVAL;
  std::lock_guard<std::mutex> lock(p->mu);
  DeviceGuard guard(p->device);
  FT_HIP(p, launch_adapters(a, static_cast<hipStream_t>(hip_stream)));
  return FT_OK;
}
FT_CATCH_ALL

}  // extern "C"
