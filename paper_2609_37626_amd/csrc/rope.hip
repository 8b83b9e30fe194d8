// gfx950 kernel of splash_rope: rotary positions with several axes.
//
// A workgroup takes tokens one after the other.  Pair j's angle is the same for
// every head, so its sine and cosine are made once per token, into LDS, and the
// heads of both views turn by them.  The angle in turns, position * inv_freq /
// (2 pi), is formed and reduced to [-1/2, 1/2] in 64 bits: in 32 bits position
// 2^20 would leave 2^-4 rad of it.
//
// Bound: HBM (2 bytes read and 2 written per element).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "step.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float bf16_to_float(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }

__global__ __launch_bounds__(kThreads) void rope_kernel(RopeLaunch p) {
  __shared__ float cosine[kMaxRopePairs], sine[kMaxRopePairs];
  for (int n = blockIdx.x; n < p.num_tokens; n += gridDim.x) {
    __syncthreads();
    if ((int)threadIdx.x < p.pairs) {
      const int j = threadIdx.x;
      double turns = (double)p.positions[p.axis[j] * p.position_stride + n] * p.turns[j];
      turns -= __builtin_rint(turns);
      float s, c;
      sincospif(2.f * (float)turns, &s, &c);
      cosine[j] = c * p.scale;
      sine[j] = s * p.scale;
    }
    __syncthreads();
    for (int v = 0; v < p.num_views; ++v) {
      const RopeView& w = p.view[v];
      const uint16_t* x = w.x + n * w.x_token;
      uint16_t* y = w.y + n * w.y_token;
      for (int e = threadIdx.x; e < w.heads * p.pairs; e += kThreads) {
        const int h = e / p.pairs, j = e - h * p.pairs;
        const int ia = p.interleaved ? 2 * j : j, ib = p.interleaved ? 2 * j + 1 : j + p.pairs;
        const float a = bf16_to_float(x[h * w.x_head + ia]), b = bf16_to_float(x[h * w.x_head + ib]);
        const uint32_t r = pack_bf16x2(a * cosine[j] - b * sine[j], b * cosine[j] + a * sine[j]);
        y[h * w.y_head + ia] = (uint16_t)r;
        y[h * w.y_head + ib] = (uint16_t)(r >> 16);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeLaunch& p, hipStream_t s) {
  const int groups = p.num_tokens < 4096 ? p.num_tokens : 4096;
  hipLaunchKernelGGL(rope_kernel, dim3(groups), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace splash
