// Norms of queries and keys, head by head, and their rotation by the token's position in the same pass.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

// sin and cos of position * freq: the product is taken in 64 bits, as turns, of which the fraction is what matters.
__device__ inline void angle(int32_t position, float freq, float *s, float *c) {
  constexpr double kTurn = 0.15915494309189533577;  // 1 / 2 pi
  const double turns = (double)position * ((double)freq * kTurn);
  const float part = (float)(turns - __builtin_rint(turns));  // within half a turn
  sincospif(2 * part, s, c);
}

// A wavefront to a head, any number of pairs. A lane has pairs l and l + 64, and elements behind the turned ones: what it writes it has read, so
// a head may be turned in place.
template <class T>
__global__ __launch_bounds__(256) void ft_rotate_any_kernel(ft_rotate_call r, Divisor by_heads, uint64_t all) {
  const uint32_t lane = threadIdx.x & 63, half = r.rot / 2;
  for (uint64_t i = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < all; i += (uint64_t)gridDim.x * 4) {
    const uint32_t token = (uint32_t)(i / by_heads.d);
    uint32_t head = (uint32_t)(i - (uint64_t)token * by_heads.d);
    const bool key = head >= r.heads;
    if (key) head -= r.heads;
    const uint16_t *in = static_cast<const uint16_t *>(key ? r.k : r.q) + token * (key ? r.k_token_stride : r.q_token_stride) +
                         head * (key ? r.k_head_stride : r.q_head_stride);
    uint16_t *out = static_cast<uint16_t *>(key ? r.k_out : r.q_out) + token * (key ? r.k_out_token_stride : r.q_out_token_stride) +
                    head * (key ? r.k_out_head_stride : r.q_out_head_stride);
    const uint16_t *weight = static_cast<const uint16_t *>(key ? r.k_weight : r.q_weight);
    float a[2], b[2], rest[4];
    uint32_t ia[2], ib[2];
    float squares = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t pair = lane + 64 * j;
      const bool there = pair < half;
      ia[j] = (r.flags & FT_ROTATE_NEIGHBOURS) != 0 ? 2 * pair : pair;
      ib[j] = (r.flags & FT_ROTATE_NEIGHBOURS) != 0 ? 2 * pair + 1 : pair + half;
      a[j] = there ? T::to_float(in[ia[j]]) : 0;
      b[j] = there ? T::to_float(in[ib[j]]) : 0;
      squares += a[j] * a[j] + b[j] * b[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t at = r.rot + lane + 64 * j;
      rest[j] = at < r.dim ? T::to_float(in[at]) : 0;
      squares += rest[j] * rest[j];
    }
    float by = 1;
    if ((r.flags & FT_ROTATE_NORM) != 0) {
      for (int d = 32; d > 0; d >>= 1) squares += __shfl_xor(squares, d);
      by = 1.0f / sqrtf(squares / (float)r.dim + r.eps);
    } else {
      weight = nullptr;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t pair = lane + 64 * j;
      if (pair >= half) break;
      uint32_t axis = r.axis == nullptr ? 0 : r.axis[pair];
      if (axis >= r.axes) axis = r.axes - 1;
      float s, c;
      angle(r.positions[(uint64_t)token * r.axes + axis], r.freqs[pair], &s, &c);
      float x = a[j] * by, y = b[j] * by;
      if (weight != nullptr) {
        x *= T::to_float(weight[ia[j]]);
        y *= T::to_float(weight[ib[j]]);
      }
      out[ia[j]] = T::from_float(x * c - y * s);
      out[ib[j]] = T::from_float(x * s + y * c);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t at = r.rot + lane + 64 * j;
      if (at >= r.dim) break;
      out[at] = T::from_float(rest[j] * by * (weight != nullptr ? T::to_float(weight[at]) : 1.0f));
    }
  }
}

}  // namespace

hipError_t launch_rotate(const ft_rotate_call &r, hipStream_t stream) {
  const uint64_t all = (uint64_t)r.tokens * (r.heads + r.kv_heads), wg = (all + 3) / 4;
  const dim3 grid((uint32_t)(wg > 1u << 20 ? 1u << 20 : wg));
  const Divisor heads(r.heads + r.kv_heads);
  if (r.type == FT_BF16) hipLaunchKernelGGL(ft_rotate_any_kernel<Bf16>, grid, dim3(256), 0, stream, r, heads, all);
  else hipLaunchKernelGGL(ft_rotate_any_kernel<Fp16>, grid, dim3(256), 0, stream, r, heads, all);
  return hipGetLastError();
}

}  // namespace ft
