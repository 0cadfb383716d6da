// Norms of queries and keys, head by head, and their rotation by the token's position in the same pass.
//
// Every element is read once and written once, and memory is the bound: 32773 tokens of 40 heads of 128 elements, 671 MB, take 118 us (5.7 TB/s), 8192
// 35 (4.7). A token's angles are the same for all of its heads: a workgroup works out the sines and cosines of its tokens, a pair to a thread, in 64 bits
// up to the fraction of a turn, and has them in shared memory (worked out for every head again the same takes 467 us). Then a few neighbouring
// lanes have a head, 16 elements each - two loads and two stores of 16 bytes -: eight pairs, or what is not turned. One token of 40 heads takes 4.0 us, of
// which 2.8 are a launch that does next to nothing; the rest is its position, its angles and its elements, one after the other.
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

// For fewer pairs than a run of eight: a wavefront to a head. A lane has one pair or none, and elements behind the turned ones: what it writes it
// has read, so a head may be turned in place.
template <class T>
__global__ __launch_bounds__(256) void ft_rotate_few_kernel(ft_rotate_call r, Divisor by_heads, uint64_t all) {
  const uint32_t lane = threadIdx.x & 63, half = r.rot / 2;  // 1 .. 7
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
    const bool turned = lane < half;
    const float a = turned ? T::to_float(in[lane]) : 0, b = turned ? T::to_float(in[lane + half]) : 0;
    float rest[4], squares = a * a + b * b;
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
    if (turned) {
      uint32_t axis = r.axis == nullptr ? 0 : r.axis[lane];
      if (axis >= r.axes) axis = r.axes - 1;
      float s, c;
      angle(r.positions[(uint64_t)token * r.axes + axis], r.freqs[lane], &s, &c);
      float x = a * by, y = b * by;
      if (weight != nullptr) {
        x *= T::to_float(weight[lane]);
        y *= T::to_float(weight[lane + half]);
      }
      out[lane] = T::from_float(x * c - y * s);
      out[lane + half] = T::from_float(x * s + y * c);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t at = r.rot + lane + 64 * j;
      if (at >= r.dim) break;
      out[at] = T::from_float(rest[j] * by * (weight != nullptr ? T::to_float(weight[at]) : 1.0f));
    }
  }
}

constexpr uint32_t kMostPairs = 1024;  // of a workgroup's tokens

struct Eight {
  float v[8];
};

template <class T>
__device__ inline Eight eight(Words4 w) {
  Eight out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out.v[2 * i] = T::to_float((uint16_t)w[i]);
    out.v[2 * i + 1] = T::to_float((uint16_t)(w[i] >> 16));
  }
  return out;
}

// elements from `skip` on
template <class T>
__device__ inline void write(uint16_t *p, const Eight &e, uint32_t skip) {
  Loose4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) out.w[i] = T::pack(e.v[2 * i], e.v[2 * i + 1]);
  if (skip == 0) {
    *reinterpret_cast<Loose4 *>(p) = out;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i >= skip) p[i] = (uint16_t)(out.w[i / 2] >> 16 * (i % 2));
  }
}

// LP lanes to a head, each two runs of eight elements. Pairs of halves: the runs of a lane are the two sides of its pairs; the last one begins
// earlier than where the one before it ends if the pairs are not a multiple of eight, and does not count what that one has; both write it, the
// same. So do the last ones of what is not turned, where that is eight elements or more. Pairs of neighbours: a run has four of them.
template <class T, int LP, bool NEIGHBOURS, bool NORM>
__global__ __launch_bounds__(256) void ft_rotate_kernel(ft_rotate_call r, Divisor by_heads, Divisor by_pairs, uint32_t most_tokens) {
  __shared__ float cosine[kMostPairs], sine[kMostPairs];
  const uint32_t token0 = blockIdx.x * most_tokens, tokens = r.tokens - token0 < most_tokens ? r.tokens - token0 : most_tokens;
  const uint32_t half = r.rot / 2, pairs = by_pairs.d;  // turned ones, and those in shared memory: with NEIGHBOURS all of a head
  for (uint32_t i = threadIdx.x; i < tokens * pairs; i += 256) {
    const uint32_t token = by_pairs.of(i), pair = i - token * pairs;
    float s = 0, c = 1;
    if (pair < half) {
      uint32_t axis = r.axis == nullptr ? 0 : r.axis[pair];
      if (axis >= r.axes) axis = r.axes - 1;
      angle(r.positions[(uint64_t)(token0 + token) * r.axes + axis], r.freqs[pair], &s, &c);
    }
    cosine[i] = c;
    sine[i] = s;
  }

  // what of a head this lane has
  const uint32_t unit = threadIdx.x % LP, rest = r.dim - r.rot;
  uint32_t begin[2], skip[2] = {0, 0}, pair[2];
  bool there[2], turned = true;
  if (NEIGHBOURS) {
    const uint32_t runs = r.dim / 8, second = (runs + 1) / 2;
    there[0] = unit < second;
    there[1] = there[0] && unit + second < runs;
    begin[0] = 8 * unit;
    begin[1] = 8 * (unit + second);
  } else {
    const uint32_t units = (half + 7) / 8;
    turned = unit < units;
    if (turned) {
      there[0] = there[1] = true;
      begin[0] = 8 * unit + 8 <= half ? 8 * unit : half - 8;
      begin[1] = begin[0] + half;
      skip[0] = skip[1] = 8 * unit - begin[0];
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t at = 16 * (unit - units) + 8 * i;
        there[i] = at < rest;
        begin[i] = r.rot + at + 8 <= r.dim ? r.rot + at : r.dim - 8;
        skip[i] = r.rot + at - begin[i];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!there[i]) begin[i] = 0;
    pair[i] = NEIGHBOURS ? begin[i] / 2 : turned ? begin[0] : 0;
  }
  Words4 q_weight[2], k_weight[2];
  if (NORM) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t one = T::pack(1, 1);
      q_weight[i] = r.q_weight != nullptr ? load16(static_cast<const uint16_t *>(r.q_weight) + begin[i]) : Words4{one, one, one, one};
      k_weight[i] = r.k_weight != nullptr ? load16(static_cast<const uint16_t *>(r.k_weight) + begin[i]) : Words4{one, one, one, one};
    }
  }
  __syncthreads();

  for (uint32_t i = threadIdx.x / LP; i < tokens * by_heads.d; i += 256 / LP) {
    const uint32_t token = by_heads.of(i);
    uint32_t head = i - token * by_heads.d;
    const bool key = head >= r.heads;
    if (key) head -= r.heads;
    const uint16_t *in = static_cast<const uint16_t *>(key ? r.k : r.q) + (uint64_t)(token0 + token) * (key ? r.k_token_stride : r.q_token_stride) +
                         head * (key ? r.k_head_stride : r.q_head_stride);
    uint16_t *out = static_cast<uint16_t *>(key ? r.k_out : r.q_out) + (uint64_t)(token0 + token) * (key ? r.k_out_token_stride : r.q_out_token_stride) +
                    head * (key ? r.k_out_head_stride : r.q_out_head_stride);
    Eight x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) x[j] = eight<T>(load16(in + begin[j]));
    if (NORM) {
      float squares = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float sum = 0;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
          if (e >= skip[j]) sum = __builtin_fmaf(x[j].v[e], x[j].v[e], sum);
        if (there[j]) squares += sum;
      }
#pragma unroll
      for (int d = LP / 2; d > 0; d >>= 1) squares += __shfl_xor(squares, d);
      const float by = 1.0f / sqrtf(squares / (float)r.dim + r.eps);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        Words4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = key ? k_weight[j][e] : q_weight[j][e];
        const Eight weight = eight<T>(w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[j].v[e] *= by * weight.v[e];
      }
    }
    const float *c = cosine + token * pairs, *s = sine + token * pairs;
    if (NEIGHBOURS) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          const float a = x[j].v[2 * e], b = x[j].v[2 * e + 1], cos = c[pair[j] + e], sin = s[pair[j] + e];
          if (pair[j] + e < half) {
            x[j].v[2 * e] = a * cos - b * sin;
            x[j].v[2 * e + 1] = a * sin + b * cos;
          }
        }
    } else if (turned) {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        const float a = x[0].v[e], b = x[1].v[e], cos = c[pair[0] + e], sin = s[pair[0] + e];
        x[0].v[e] = a * cos - b * sin;
        x[1].v[e] = a * sin + b * cos;
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (there[j]) write<T>(out + begin[j], x[j], NEIGHBOURS || turned || rest >= 8 ? 0 : skip[j]);
  }
}

// Tokens to a workgroup: as many as its threads have at once, and twice that where the tokens are thousands. With 1, 2, 4 and 8 of them, heads of 128
// elements: 32773 tokens of 40 heads 117, 123, 128 and 135 us, 30000 of 5 heads 41, 32, 23 and 21; 4096 of 10 heads 9.9, 7.9, 7.2 and 8.1, 8192 of 10
// 18.9, 14.0, 13.3 and 12.8; 512 of 5 3.2, 3.3, 3.3 and 4.5; 1024 of 40 7.1, 7.8, 9.6 and 15.2.
template <class T, int LP, bool NEIGHBOURS, bool NORM>
void launch(const ft_rotate_call &r, hipStream_t stream) {
  const uint32_t pairs = NEIGHBOURS ? r.dim / 2 : r.rot / 2 == 0 ? 1 : r.rot / 2;
  const uint32_t lanes = LP * (r.heads + r.kv_heads);
  uint32_t once = 256 / (lanes > pairs ? lanes : pairs), twice = 512 / lanes;
  if (twice > r.tokens / 1024) twice = r.tokens / 1024;
  uint32_t most = once > twice ? once : twice;
  most = most < 1 ? 1 : most > kMostPairs / pairs ? kMostPairs / pairs : most;
  hipLaunchKernelGGL((ft_rotate_kernel<T, LP, NEIGHBOURS, NORM>), dim3((r.tokens + most - 1) / most), dim3(256), 0, stream, r, Divisor(r.heads + r.kv_heads),
                     Divisor(pairs), most);
}

template <class T, bool NEIGHBOURS, bool NORM>
void launch(const ft_rotate_call &r, hipStream_t stream) {
  const uint32_t lanes = NEIGHBOURS ? (r.dim / 8 + 1) / 2 : (r.rot / 2 + 7) / 8 + (r.dim - r.rot + 15) / 16;
  if (lanes <= 4) launch<T, 4, NEIGHBOURS, NORM>(r, stream);
  else if (lanes <= 8) launch<T, 8, NEIGHBOURS, NORM>(r, stream);
  else if (lanes <= 16) launch<T, 16, NEIGHBOURS, NORM>(r, stream);
  else launch<T, 32, NEIGHBOURS, NORM>(r, stream);
}

template <class T>
hipError_t launch(const ft_rotate_call &r, hipStream_t stream) {
  const bool neighbours = (r.flags & FT_ROTATE_NEIGHBOURS) != 0, norm = (r.flags & FT_ROTATE_NORM) != 0;
  if (!neighbours && r.rot != 0 && r.rot < 16) {  // fewer pairs than a run of eight has
    const uint64_t all = (uint64_t)r.tokens * (r.heads + r.kv_heads), wg = (all + 3) / 4;
    hipLaunchKernelGGL(ft_rotate_few_kernel<T>, dim3((uint32_t)(wg > 1u << 20 ? 1u << 20 : wg)), dim3(256), 0, stream, r, Divisor(r.heads + r.kv_heads), all);
  } else if (neighbours) {
    norm ? launch<T, true, true>(r, stream) : launch<T, true, false>(r, stream);
  } else {
    norm ? launch<T, false, true>(r, stream) : launch<T, false, false>(r, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const ft_rotate_call &r, hipStream_t stream) { return r.type == FT_BF16 ? launch<Bf16>(r, stream) : launch<Fp16>(r, stream); }

}  // namespace ft
