// gfx950 kernel of splash_mla_append: the norm of the latent, the turn of the
// shared key and the cache's format in one pass.
//
// A wave takes a token: a lane holds eight latent values (16 bytes) and one of
// the key's 64, so that every sine and cosine is made once, each store of the wave
// is one run of bytes, and maxima and the sum of squares are shuffles.
//
// y is formed in 64 bits and rounded to fp32 once (x and the weight are bf16; 64-bit
// products go at half the rate of 32-bit ones, and there are 32 a lane): a value next to
// 448 * 2^e then decides a scale the same way for everyone, where fp32 sums would leave
// it to their order.
//
// Bound: the instructions of a token, then HBM: 11.1k tokens into per-token E4M3 take
// 8.5 us for 19 MB (2.8 us at the rate of reads), into bf16 or latent rows 7.9 and 8.0.
// From 11.0 us: sums and maxima over lanes by row turns and lane reads rather than shuffles
// through LDS, 1 / sqrt by two Newton steps, quotients by one inverse and a correction,
// finite values on a path of their own (to 9.5), and every load of a token before the first
// wait (to 8.2).  A token for each of 256 requests is launch latency: 3.4 us, 2.8 after
// another kernel of a graph.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"
#include "quotient.hpp"
#include "splash_attn.h"
#include "turn.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr float kTop = 448.f;

template <bool FINITE>
__device__ __forceinline__ float held(float x) {  // past the largest code, that code; NaN stays
  return FINITE || x != x ? x : fminf(fmaxf(x, -kTop), kTop);
}
template <bool FINITE>
__device__ __forceinline__ u32x2 codes_of(const float (&y)[8]) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(held<FINITE>(y[4 * i]), held<FINITE>(y[4 * i + 1]), 0, false);
    r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(held<FINITE>(y[4 * i + 2]), held<FINITE>(y[4 * i + 3]), lo, true);
  }
  return r;
}

// Magnitudes as bits: they order like the numbers, with infinities and NaN above all.
constexpr uint32_t kInfinite = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t finite_magnitude(float x) { return magnitude(x) < kInfinite ? magnitude(x) : 0u; }

// The 16 lanes of a row of lanes together, in four turns of the row; then all 64.
template <int BY>
__device__ __forceinline__ uint32_t turned(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x120 | BY, 0xf, 0xf, true);
}
template <int BY>
__device__ __forceinline__ double turned(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)turned<BY>((uint32_t)(u >> 32)) << 32 | turned<BY>((uint32_t)u));
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, turned<8>(v));
  v = max(v, turned<4>(v));
  v = max(v, turned<2>(v));
  return max(v, turned<1>(v));
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)lane_of((uint32_t)(u >> 32), lane) << 32 | lane_of((uint32_t)u, lane));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = row_max(v);
  return max(max(lane_of(v, 0), lane_of(v, 16)), max(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ double wave_sum(double v) {
  v += turned<8>(v);
  v += turned<4>(v);
  v += turned<2>(v);
  v += turned<1>(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// 1 / sqrt(x): the hardware's 2^-26, then two steps of Newton's method (2^-52).
__device__ __forceinline__ double inverse_root(double x) {
  const double r = __builtin_amdgcn_rsq(x), h = 0.5 * x;
  double s = r * __builtin_fma(-h * r, r, 1.5);
  s = s * __builtin_fma(-h * s, s, 1.5);
  return r > 0.0 && r < __builtin_inf() ? s : r;  // (x infinite, zero or NaN: r itself)
}
// A token's row into the pool.  FINITE: no infinity and no NaN among its values.
template <int FORMAT, bool FINITE>
__device__ __forceinline__ void write_row(const MlaAppendLaunch& a, int32_t slot, int lane, float (&y)[8], float r, uint32_t top) {
  if constexpr (!FINITE) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(y[i]));
    if (FORMAT == SPLASH_KV_FP8_E4M3) top = max(top, finite_magnitude(r));
  }
  if constexpr (FORMAT == SPLASH_KV_FP8_E4M3) {
    const float largest = __builtin_bit_cast(float, wave_max(top));
    const float scale = largest > 0.f ? fmaxf(largest / kTop, 0x1p-126f) : 1.f;
    if (scale >= 0x1p-100f) {
      const float inverse = 1.f / scale;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = quotient<FINITE>(y[i], scale, inverse);
      r = quotient<FINITE>(r, scale, inverse);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] /= scale;
      r /= scale;
    }
    uint8_t* row = a.pages + (int64_t)slot * kDimQK;
    *(u32x2*)(row + 8 * lane) = codes_of<FINITE>(y);
    row[kDimV + lane] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(held<FINITE>(r), 0.f, 0, false);
    if (lane == 0) a.scales[slot] = scale;
  } else {
    // a quarter's 128 columns are 16 lanes; the least e with top <= 1.75 * 2^(e + 8), by
    // top's exponent and fraction
    top = row_max(top);
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
    e = top > 0 ? min(max(e, -126), 63) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_ldexpf(y[i], -e);
    uint8_t* row = a.pages + (int64_t)slot * kLatentRowBytes;
    *(u32x2*)(row + 8 * lane) = e < 63 ? codes_of<FINITE>(y) : codes_of<false>(y);
    if ((lane & 15) == 0) *(uint32_t*)(row + kDimV + (lane >> 2)) = (uint32_t)(e + 127) << 23;
    *(uint16_t*)(row + kDimV + 16 + 2 * lane) = (uint16_t)pack_bf16x2(r, 0.f);
  }
}

template <int FORMAT>
__global__ __launch_bounds__(kThreads) void mla_append_kernel(MlaAppendLaunch a) {
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (n >= a.num_tokens) return;
  // all of the token's loads before the first wait
  int none = 0;
  asm volatile("" : "+v"(none));  // (a vector load: a scalar one would be waited for with the arguments)
  int32_t slot = a.slots[n + none];
  const u32x4 raw = *(const u32x4*)(a.latent + n * a.latent_stride + 8 * lane);
  const uint32_t key_bits = a.key[n * a.key_stride + lane];
  u32x4 w = {0u, 0u, 0u, 0u};
  if (a.norm_weight) w = *(const u32x4*)(a.norm_weight + 8 * lane);
  PairAngle angle = {0, 0.0};
  if (a.turn.positions) angle = pair_angle(a.turn, n, pair_of(a.turn, lane));
  asm volatile("" ::"v"(slot), "v"(raw), "v"(key_bits), "v"(w), "v"(angle.position), "v"(angle.turns));
  slot = __builtin_amdgcn_readfirstlane(slot);
  if (slot < 0 || (slot >> 6) >= a.num_pages) return;
  const float key = __builtin_bit_cast(float, key_bits << 16);
  float x[8], y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xffff0000u);
  }
  float r = key;
  if (a.turn.positions) {
    float c, s;
    pair_turn(a.turn, angle, c, s);
    r = turn_element(a.turn, lane, key, c, s);
  }
  if (a.norm_weight) {
    double squares = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) squares = __builtin_fma((double)x[i], (double)x[i], squares);
    const double by = inverse_root(wave_sum(squares) * (1.0 / kDimV) + (double)a.norm_eps);
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
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude(y[i]));
    if (FORMAT == SPLASH_KV_FP8_E4M3) top = max(top, magnitude(r));
    if (!__any(top >= kInfinite)) write_row<FORMAT, true>(a, slot, lane, y, r, top);
    else write_row<FORMAT, false>(a, slot, lane, y, r, top);
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
