// gfx950 kernel of splash_mla_append: the norm of the latent, the turn of the
// shared key and the cache's format in one pass.
//
// A wave takes a token: a lane holds eight latent values (16 bytes) and one of
// the key's 64, so that every sine and cosine is made once, each store of the wave
// is one run of bytes, and maxima and the sum of squares are shuffles.
//
// y is formed in 64 bits and rounded to fp32 once (x and the weight are bf16, 64-bit
// products cost what 32-bit ones do here): a value next to 448 * 2^e then decides a
// scale the same way for everyone, where fp32 sums would leave it to their order.
//
// Bound: HBM for prompts, latency for a token a request.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"
#include "splash_attn.h"
#include "turn.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr float kTop = 448.f;

// A quotient by the scale, for the conversion: past the largest code, that code; NaN stays.
__device__ __forceinline__ float held(float x) { return x != x ? x : fminf(fmaxf(x, -kTop), kTop); }
__device__ __forceinline__ u32x2 codes_of(const float (&y)[8]) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(held(y[4 * i]), held(y[4 * i + 1]), 0, false);
    r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(held(y[4 * i + 2]), held(y[4 * i + 3]), lo, true);
  }
  return r;
}
__device__ __forceinline__ float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m <= 3.402823466e38f ? m : 0.f;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

template <int FORMAT>
__global__ __launch_bounds__(kThreads) void mla_append_kernel(MlaAppendLaunch a) {
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (n >= a.num_tokens) return;
  const int32_t slot = a.slots[n];
  if (slot < 0 || (slot >> 6) >= a.num_pages) return;
  const u32x4 raw = *(const u32x4*)(a.latent + n * a.latent_stride + 8 * lane);
  const float key = __builtin_bit_cast(float, (uint32_t)a.key[n * a.key_stride + lane] << 16);
  float x[8], y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xffff0000u);
  }
  float r = key;
  if (a.turn.positions) {
    float c, s;
    pair_turn(a.turn, n, pair_of(a.turn, lane), c, s);
    r = turn_element(a.turn, lane, key, c, s);
  }
  if (a.norm_weight) {
    const u32x4 w = *(const u32x4*)(a.norm_weight + 8 * lane);
    double squares = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) squares += (double)x[i] * (double)x[i];
    const double by = 1.0 / __builtin_sqrt(wave_sum(squares) * (1.0 / kDimV) + (double)a.norm_eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float wi = __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
      y[i] = (float)((double)x[i] * (double)wi * by);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
  }

  if constexpr (FORMAT == SPLASH_KV_BF16) {
    uint16_t* row = (uint16_t*)a.pages + (int64_t)slot * kDimQK;
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
    *(u32x4*)(row + 8 * lane) = q;
    row[kDimV + lane] = (uint16_t)pack_bf16x2(r, 0.f);
    return;
  }
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_magnitude(y[i]));
  if constexpr (FORMAT == SPLASH_KV_FP8_E4M3) {
    top = fmaxf(top, finite_magnitude(r));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float scale = top > 0.f ? fmaxf(top / kTop, 0x1p-126f) : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] / scale;
    uint8_t* row = a.pages + (int64_t)slot * kDimQK;
    *(u32x2*)(row + 8 * lane) = codes_of(y);
    row[kDimV + lane] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(held(r / scale), 0.f, 0, false);
    if (lane == 0) a.scales[slot] = scale;
  } else {
    // a quarter's 128 columns are 16 lanes
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    // the least e with top <= 1.75 * 2^(e + 8): by top's exponent and fraction
    const uint32_t bits = __builtin_bit_cast(uint32_t, top);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    e = top > 0.f ? min(max(e, -126), 63) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_ldexpf(y[i], -e);
    uint8_t* row = a.pages + (int64_t)slot * kLatentRowBytes;
    *(u32x2*)(row + 8 * lane) = codes_of(y);
    if ((lane & 15) == 0) *(float*)(row + kDimV + (lane >> 2)) = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
    *(uint16_t*)(row + kDimV + 16 + 2 * lane) = (uint16_t)pack_bf16x2(r, 0.f);
  }
}

}  // namespace

hipError_t launch_mla_append(const MlaAppendLaunch& a, hipStream_t s) {
  const dim3 groups(((unsigned)a.num_tokens + kThreads / 64 - 1) / (kThreads / 64));
  if (a.kv_dtype == SPLASH_KV_BF16) hipLaunchKernelGGL((mla_append_kernel<SPLASH_KV_BF16>), groups, dim3(kThreads), 0, s, a);
  else if (a.kv_dtype == SPLASH_KV_FP8_E4M3) hipLaunchKernelGGL((mla_append_kernel<SPLASH_KV_FP8_E4M3>), groups, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((mla_append_kernel<SPLASH_KV_FP8_LATENT>), groups, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace splash
