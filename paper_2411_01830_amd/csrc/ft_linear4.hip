// Products of few rows with weights of 4 bits and group scales, read as they lie in the pool.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

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

hipError_t launch_linear4(const Linear4View &w, const ft_linear4_call &c, int, hipStream_t stream) {
  const uint32_t parts = (c.rows + 7) / 8;
  const dim3 grid((w.width_out + 3) / 4, parts < 1024 ? parts : 1024);
  if (w.type == FT_BF16) hipLaunchKernelGGL(ft_linear4_any_kernel<Bf16>, grid, dim3(256), 0, stream, w, c);
  else hipLaunchKernelGGL(ft_linear4_any_kernel<Fp16>, grid, dim3(256), 0, stream, w, c);
  return hipGetLastError();
}

}  // namespace ft
