// gfx950 kernel of splash_rope: rotary positions with several axes.
//
// A wave takes a token and some of its heads.  Pair j's angle is the same for
// every head, so each sine and cosine is made once per wave, one pair a lane,
// and goes through LDS to the lanes that turn that pair: eight lanes of 16 bytes
// (rot_dim 128) hold a head, so a lane keeps its pairs' values for all of its
// heads, and two heads' loads are in flight a lane (four: 68 us instead of 65 for
// 16,384 tokens of 40 heads by 128).  The angle in turns,
// position * inv_freq / (2 pi), is formed and reduced to [-1/2, 1/2] in 64 bits:
// in 32 bits position 2^20 would leave 2^-4 rad of it.  What is left of it is
// rounded to fp32, by 2^-26 of a turn at most, for an fp32 sine and cosine: 2^-22
// or less of a pair beside the output's 2^-8.
//
// Bound: HBM (2 bytes read and 2 written per element); latency for a few tokens.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "step.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 2;           // heads' loads in flight
constexpr int kWavesWanted = 4096;

// Each wave's sines and cosines: lane j makes pairs j and j + 64.
__device__ __forceinline__ void make_turns(const RopeLaunch& p, int n, int lane, float* cosine, float* sine) {
  for (int j = lane; j < p.pairs; j += 64) {
    double turns = (double)p.positions[p.axis[j] * p.position_stride + n] * p.turns[j];
    turns -= __builtin_rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    cosine[j] = c * p.scale;
    sine[j] = s * p.scale;
  }
  __builtin_amdgcn_wave_barrier();  // (one wave's LDS is in order)
}

// Rows in pieces of 16 bytes: `INTERLEAVED` four pairs a lane, else eight.
template <bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeLaunch p, int32_t heads_per_wave) {
  __shared__ __align__(16) float cosine[kThreads / 64][kMaxRopePairs], sine[kThreads / 64][kMaxRopePairs];
  constexpr int kPairs = INTERLEAVED ? 4 : 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = blockIdx.x * (kThreads / 64) + wave;
  if (n >= p.num_tokens) return;
  make_turns(p, n, lane, cosine[wave], sine[wave]);
  const int lanes = p.pairs / kPairs, group = lane % lanes, side_by_side = 64 / lanes;  // lanes of a head; heads at a time
  if (lane >= lanes * side_by_side) return;
  float c[kPairs], s[kPairs];
#pragma unroll
  for (int j = 0; j < kPairs; j += 4) {
    const f32x4 a = *(const f32x4*)(cosine[wave] + group * kPairs + j), b = *(const f32x4*)(sine[wave] + group * kPairs + j);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[j + k] = a[k];
      s[j + k] = b[k];
    }
  }
  const int heads = p.view[0].heads + (p.num_views > 1 ? p.view[1].heads : 0);
  const int first = blockIdx.y * heads_per_wave, end = min(first + heads_per_wave, heads);
  const auto place = [&](int h, const uint16_t** x, uint16_t** y) {
    const bool second = h >= p.view[0].heads;
    const RopeView& w = p.view[second];
    const int at = second ? h - p.view[0].heads : h;
    *x = w.x + n * w.x_token + at * w.x_head + 8 * group;
    *y = w.y + n * w.y_token + at * w.y_head + 8 * group;
  };
  for (int h0 = first + lane / lanes; h0 < end; h0 += kAtOnce * side_by_side) {
    u32x4 lo[kAtOnce], hi[kAtOnce];
    uint16_t* y[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int h = h0 + k * side_by_side;
      const uint16_t* x;
      place(h < end ? h : h0, &x, &y[k]);
      lo[k] = *(const u32x4*)x;
      if constexpr (!INTERLEAVED) hi[k] = *(const u32x4*)(x + p.pairs);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (h0 + k * side_by_side >= end) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a0 = __builtin_bit_cast(float, lo[k][i] << 16), a1 = __builtin_bit_cast(float, lo[k][i] & 0xffff0000u);
        if constexpr (INTERLEAVED) {  // one pair a dword
          lo[k][i] = pack_bf16x2(a0 * c[i] - a1 * s[i], a1 * c[i] + a0 * s[i]);
        } else {
          const float b0 = __builtin_bit_cast(float, hi[k][i] << 16), b1 = __builtin_bit_cast(float, hi[k][i] & 0xffff0000u);
          lo[k][i] = pack_bf16x2(a0 * c[2 * i] - b0 * s[2 * i], a1 * c[2 * i + 1] - b1 * s[2 * i + 1]);
          hi[k][i] = pack_bf16x2(b0 * c[2 * i] + a0 * s[2 * i], b1 * c[2 * i + 1] + a1 * s[2 * i + 1]);
        }
      }
      *(u32x4*)y[k] = lo[k];
      if constexpr (!INTERLEAVED) *(u32x4*)(y[k] + p.pairs) = hi[k];
    }
  }
}

// Rows of any alignment and any even length, a pair a lane, in 2-byte pieces, all
// of a token's heads on one wave: 92 us for 16,384 tokens of 40 heads by 128 that
// start at an odd element (68 in 16-byte pieces), 11 for 256 tokens (4.1).
__global__ __launch_bounds__(kThreads) void rope_any_kernel(RopeLaunch p) {
  __shared__ float cosine[kThreads / 64][kMaxRopePairs], sine[kThreads / 64][kMaxRopePairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = blockIdx.x * (kThreads / 64) + wave;
  if (n >= p.num_tokens) return;
  make_turns(p, n, lane, cosine[wave], sine[wave]);
  for (int v = 0; v < p.num_views; ++v) {
    const RopeView& w = p.view[v];
    const uint16_t* x = w.x + n * w.x_token;
    uint16_t* y = w.y + n * w.y_token;
    for (int e = lane; e < w.heads * p.pairs; e += 64) {
      const int h = e / p.pairs, j = e - h * p.pairs;
      const int ia = p.interleaved ? 2 * j : j, ib = p.interleaved ? 2 * j + 1 : j + p.pairs;
      const float a = __builtin_bit_cast(float, (uint32_t)x[h * w.x_head + ia] << 16);
      const float b = __builtin_bit_cast(float, (uint32_t)x[h * w.x_head + ib] << 16);
      const float c = cosine[wave][j], s = sine[wave][j];
      const uint32_t r = pack_bf16x2(a * c - b * s, b * c + a * s);
      y[h * w.y_head + ia] = (uint16_t)r;
      y[h * w.y_head + ib] = (uint16_t)(r >> 16);
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeLaunch& p, hipStream_t s) {
  const unsigned groups = ((unsigned)p.num_tokens + kThreads / 64 - 1) / (kThreads / 64);
  // 16-byte pieces: four pairs a lane where they are interleaved, else eight
  bool pieces = p.pairs % (p.interleaved ? 4 : 8) == 0;
  int32_t heads = 0;
  for (int v = 0; v < p.num_views; ++v) {
    const RopeView& w = p.view[v];
    heads += w.heads;
    pieces = pieces && !(((uintptr_t)w.x | (uintptr_t)w.y) & 15) && !((w.x_token | w.x_head | w.y_token | w.y_head) & 7);
  }
  if (heads == 0) return hipSuccess;
  if (!pieces) {
    hipLaunchKernelGGL(rope_any_kernel, dim3(groups), dim3(kThreads), 0, s, p);
    return hipGetLastError();
  }
  // Enough waves for the chip where there are few tokens, each making its own
  // sines: kWavesWanted, or kAtOnce heads for every lane.
  const int32_t side_by_side = 64 / (p.pairs / (p.interleaved ? 4 : 8));
  const int32_t least = kAtOnce * side_by_side, most_chunks = (heads + least - 1) / least;
  int32_t chunks = kWavesWanted / p.num_tokens;
  chunks = chunks < 1 ? 1 : (chunks > most_chunks ? most_chunks : chunks);
  const int32_t per_wave = (heads + chunks - 1) / chunks;
  if (p.interleaved) hipLaunchKernelGGL((rope_kernel<true>), dim3(groups, chunks), dim3(kThreads), 0, s, p, per_wave);
  else hipLaunchKernelGGL((rope_kernel<false>), dim3(groups, chunks), dim3(kThreads), 0, s, p, per_wave);
  return hipGetLastError();
}

}  // namespace splash
