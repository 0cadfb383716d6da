// Attention of drafted tokens over a paged cache and over each other.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

struct Tree {
  KvView c;
  ft_tree_call t;
};

// A workgroup per token and query head, 256 keys at a time.
template <class T>
__global__ __launch_bounds__(256) void ft_tree_kernel(Tree a) {
  const ft_tree_call &t = a.t;
  const KvView &c = a.c;
  __shared__ float q[256], p[256], part[4];
  __shared__ int64_t rows[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int token = blockIdx.x, head = blockIdx.y, kv_head = head / (t.heads / c.heads);
  int lo = 0, hi = (int)t.requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.starts[mid] <= token) lo = mid;
    else hi = mid;
  }
  while (lo > 0 && t.starts[lo] > token) --lo;
  const int start = t.starts[lo], end = t.starts[lo + 1] < (int)t.tokens ? t.starts[lo + 1] : (int)t.tokens;
  if (start < 0 || token < start || token >= end || token - start >= (int)t.drafts) return;
  int len = t.lens[lo];
  const int64_t room = (int64_t)t.blocks * c.page_tokens.d;
  if (len < 0) len = 0;
  if (len > room) len = (int)room;
  const int drafts = end - start;
  const int keys = len + drafts;
  const uint16_t *qp = static_cast<const uint16_t *>(t.q) + token * t.q_token_stride + head * t.q_head_stride;
  if (tid < (int)c.dim) q[tid] = T::to_float(qp[tid]);
  float m = -INFINITY, l = 0, acc = 0;
  for (int s0 = 0; s0 < keys; s0 += 256) {
    const int s = s0 + tid;
    bool sees = s < keys;
    const uint16_t *kp = nullptr;
    int64_t v_row = -1;
    if (s < len) {
      const uint32_t block = c.page_tokens.of((uint32_t)s);
      uint32_t page = (uint32_t)t.table[(uint64_t)lo * t.blocks + block];
      page = page < c.pages ? page : 0;
      const uint64_t at = page * c.page_stride + (s - block * c.page_tokens.d) * c.token_stride + kv_head * c.head_stride;
      kp = reinterpret_cast<const uint16_t *>(c.k) + at;
      v_row = (int64_t)at;
    } else if (sees) {
      const int j = s - len;
      sees = t.mask != nullptr ? (uint32_t)(j >> 6) < t.mask_words && (t.mask[(uint64_t)token * t.mask_words + (j >> 6)] >> (j & 63) & 1) != 0 : j <= token - start;
      kp = static_cast<const uint16_t *>(t.k) + (start + j) * t.k_token_stride + kv_head * t.k_head_stride;
      v_row = (int64_t)((start + j) * t.v_token_stride + kv_head * t.v_head_stride);
    }
    __syncthreads();
    float score = -INFINITY;
    if (sees) {
      float x = 0;
      for (uint32_t d = 0; d < c.dim; ++d) x += q[d] * T::to_float(kp[d]);
      score = x * (t.scale * kLog2e);
    }
    float top = score;
    bool nan = score != score;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) part[wave] = top;
    __syncthreads();
    for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w]);
    const float now = fmaxf(m, top), from = now == -INFINITY ? 0 : now;
    const float shrink = exp2f(m - from);
    const float weight = sees ? (nan ? score : exp2f(score - from)) : 0;
    float sum = weight;
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    __syncthreads();
    if (lane == 0) part[wave] = sum;
    p[tid] = weight;
    rows[tid] = sees ? v_row : -1;
    __syncthreads();
    l = l * shrink + part[0] + part[1] + part[2] + part[3];
    acc *= shrink;
    m = now;
    if (tid < (int)c.dim) {
      const int n = keys - s0 < 256 ? keys - s0 : 256;
      for (int j = 0; j < n; ++j) {
        if (rows[j] < 0) continue;
        const uint16_t *vp = s0 + j < len ? reinterpret_cast<const uint16_t *>(c.v) : static_cast<const uint16_t *>(t.v);
        acc += p[j] * T::to_float(vp[rows[j] + tid]);
      }
    }
  }
  if (tid < (int)c.dim)
    static_cast<uint16_t *>(t.out)[token * t.out_token_stride + head * t.out_head_stride + tid] = T::from_float(l == 0 ? 0 : acc / l);
  if (tid == 0 && t.lse != nullptr) t.lse[(uint64_t)token * t.heads + head] = l == 0 ? -INFINITY : (m + log2f(l)) / kLog2e;
}

}  // namespace

uint64_t tree_workspace(const ft_kv_cache &, const ft_tree_call &, int) { return 0; }

hipError_t launch_tree(const KvView &c, const ft_tree_call &call, int, hipStream_t stream) {
  const Tree a{c, call};
  const dim3 grid(call.tokens, call.heads);
  if (c.type == FT_BF16) hipLaunchKernelGGL(ft_tree_kernel<Bf16>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(ft_tree_kernel<Fp16>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ft
