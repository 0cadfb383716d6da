// Low-rank adapters of many requests beside a shared projection.
#include <hip/hip_runtime.h>

#include "ft_operators.h"
#include "ft_types.h"

namespace ft {

namespace {

// A wavefront per row and rank: the row's product with a row of A.
template <class T>
__global__ __launch_bounds__(256) void ft_adapter_shrink_kernel(ft_adapters_call c, float *h) {
  const int32_t *ids = static_cast<const int32_t *>(c.groups);
  const uint32_t row = blockIdx.x, lane = threadIdx.x & 63;
  const uint32_t id = (uint32_t)ids[row];
  if (id >= c.count) return;
  const ft_adapter_record rec = c.records[id];
  const uint32_t rank = rec.rank < c.max_rank ? rec.rank : c.max_rank;
  const uint16_t *x = static_cast<const uint16_t *>(c.x) + row * c.x_stride;
  for (uint32_t r = threadIdx.x >> 6; r < rank; r += 4) {
    const uint16_t *a = reinterpret_cast<const uint16_t *>(rec.a) + (uint64_t)r * c.width_in;
    float sum = 0;
    for (uint32_t i = lane; i < c.width_in; i += 64) sum += T::to_float(x[i]) * T::to_float(a[i]);
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) h[(uint64_t)row * c.max_rank + r] = sum * rec.scale;
  }
}

template <class T>
__global__ __launch_bounds__(256) void ft_adapter_expand_kernel(ft_adapters_call c, const float *h) {
  const int32_t *ids = static_cast<const int32_t *>(c.groups);
  const uint32_t row = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x;
  if (n >= c.width_out) return;
  const uint32_t id = (uint32_t)ids[row];
  float sum = 0;
  if (id < c.count) {
    const ft_adapter_record rec = c.records[id];
    const uint32_t rank = rec.rank < c.max_rank ? rec.rank : c.max_rank;
    const uint16_t *b = reinterpret_cast<const uint16_t *>(rec.b) + (uint64_t)n * rec.rank;
    for (uint32_t r = 0; r < rank; ++r) sum += h[(uint64_t)row * c.max_rank + r] * T::to_float(b[r]);
  }
  if (c.base != nullptr) sum += T::to_float(static_cast<const uint16_t *>(c.base)[row * c.base_stride + n]);
  static_cast<uint16_t *>(c.out)[row * c.out_stride + n] = T::from_float(sum);
}

}  // namespace

uint64_t adapter_group_bytes(uint32_t rows, uint32_t) { return ((uint64_t)rows * 4 + 15) / 16 * 16; }

hipError_t launch_adapter_group(const int32_t *ids, uint32_t rows, uint32_t, void *groups, hipStream_t stream) {
  return hipMemcpyAsync(groups, ids, (uint64_t)rows * 4, hipMemcpyDeviceToDevice, stream);
}

uint64_t adapter_workspace(const ft_adapters_call &call) { return ((uint64_t)call.rows * call.max_rank * 4 + 15) / 16 * 16; }

hipError_t launch_adapters(const ft_adapters_call &call, hipStream_t stream) {
  float *h = static_cast<float *>(call.workspace);
  const dim3 grid(call.rows, (call.width_out + 255) / 256);
  if (call.type == FT_BF16) {
    hipLaunchKernelGGL(ft_adapter_shrink_kernel<Bf16>, dim3(call.rows), dim3(256), 0, stream, call, h);
    hipLaunchKernelGGL(ft_adapter_expand_kernel<Bf16>, grid, dim3(256), 0, stream, call, h);
  } else {
    hipLaunchKernelGGL(ft_adapter_shrink_kernel<Fp16>, dim3(call.rows), dim3(256), 0, stream, call, h);
    hipLaunchKernelGGL(ft_adapter_expand_kernel<Fp16>, grid, dim3(256), 0, stream, call, h);
  }
  return hipGetLastError();
}

}  // namespace ft
