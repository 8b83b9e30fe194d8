// gfx950 kernel of splash_gqa_append: new K and V rows into their blocks of
// 8-bit codes, with one power-of-two scale per block.
//
// The rows of one page stand next to each other in the list; the wave of the
// first of them (the one whose predecessor lies in another page) writes the
// whole run, for one KV head and one of K and V: no two waves touch a block,
// and nothing is exchanged between them.  It finds the run's largest finite
// magnitude, from it the exponent (on bf16's bits, so without a rounding), and
// where the block's scale grows it brings the rows that were there to the new
// one.  A power of two moves an E4M3 code's exponent alone; only codes that
// reach its subnormals, and INT8 codes, are rounded again.
//
// Bound: HBM for prompts (2 bytes read, 1 written per element), latency for one
// new token per request (slot, row and scale, store).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "step.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float bf16_to_float(uint32_t x) { return __builtin_bit_cast(float, x << 16); }

// The least e >= -126 with the magnitude (15 bits of a finite bf16) <= TOP * 2^e:
// TOP is 1.75 * 2^8 (E4M3) or 127/64 * 2^6 (INT8).
template <int CODE>
__device__ __forceinline__ int32_t exponent_for(uint32_t mag) {
  const int32_t E = (int32_t)(mag >> 7) - 127;
  const uint32_t frac = mag & 127u;
  const int32_t e = CODE == 0 ? E - 8 + (frac > 96u) : E - 6 + (frac > 126u);
  return max(e, -126);
}

// Four values, already divided by the scale, to codes.
template <int CODE>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  float x[4] = {a, b, c, d};
  if constexpr (CODE == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.f), 448.f);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
  } else {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = x[i] != x[i] ? 0.f : fminf(fmaxf(__builtin_rintf(x[i]), -127.f), 127.f);
      r |= ((uint32_t)(int32_t)v & 255u) << (8 * i);
    }
    return r;
  }
}

// Four codes times 2^-d, rounded again.
template <int CODE>
__device__ __forceinline__ uint32_t rescale_codes(uint32_t q, int32_t d) {
  float x[4];
  if constexpr (CODE == 0) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(q >> (8 * i));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_ldexpf(x[i], -d);
  return to_codes<CODE>(x[0], x[1], x[2], x[3]);
}

template <int CODE>
__global__ __launch_bounds__(kThreads) void gqa_append_kernel(GqaAppendLaunch a) {
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t sides = 2 * a.Hk;
  const int32_t n = (int32_t)(task / sides), side = (int32_t)(task - (int64_t)n * sides);
  if (n >= a.num_tokens) return;
  const int32_t h = side >> 1;
  const bool is_v = side & 1;

  // the run of rows in this page
  const int32_t slot0 = a.slots[n], page = slot0 >> 6;
  if (slot0 < 0 || page >= a.num_pages) return;
  if (n > 0 && a.slots[n - 1] >> 6 == page) return;
  const int32_t slot = n + lane < a.num_tokens ? a.slots[n + lane] : -1;
  const uint64_t others = ~__ballot(slot >= 0 && slot >> 6 == page);
  const int32_t run = others ? __builtin_ctzll(others) : 64;
  uint64_t fresh = lane < run ? 1ull << (slot & 63) : 0;  // the places that get rows
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) fresh |= __shfl_xor(fresh, d);

  const uint16_t* x = (is_v ? a.v_new : a.k_new) + h * a.head_stride;
  const int64_t block = (int64_t)page * a.Hk + h;
  uint8_t* codes = (is_v ? a.v_pages : a.k_pages) + block * (int64_t)(kPage * a.D);
  float* scale = (is_v ? a.v_scales : a.k_scales) + block;

  const int32_t pieces = a.D / 8;  // 16-byte pieces of a row
  uint32_t top = 0;                // largest finite magnitude, as bf16 bits
  for (int32_t e = lane; e < run * pieces; e += 64) {
    const int32_t r = e / pieces, c = e - r * pieces;
    const u32x4 w = *(const u32x4*)(x + (n + r) * a.token_stride + 8 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
      if (lo < 0x7f80u) top = max(top, lo);
      if (hi < 0x7f80u) top = max(top, hi);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));

  int32_t e_new = exponent_for<CODE>(top);
  const bool goes_on = !(fresh & 1ull);  // no new row in place 0: the block has rows to keep
  if (goes_on) {
    const int32_t field = (int32_t)((__builtin_bit_cast(uint32_t, *scale) >> 23) & 255u);
    const int32_t e_old = min(max(field - 127, -126), 127);
    if (e_new > e_old) {
      const int32_t last = 63 - __builtin_clzll(fresh), words = a.D / 4;
      for (int32_t e = lane; e < last * words; e += 64) {
        if (fresh >> (e / words) & 1ull) continue;
        uint32_t* q = (uint32_t*)codes + e;
        *q = rescale_codes<CODE>(*q, e_new - e_old);
      }
    } else {
      e_new = e_old;
    }
  }
  for (int32_t e = lane; e < run * pieces; e += 64) {
    const int32_t r = e / pieces, c = e - r * pieces;
    const u32x4 w = *(const u32x4*)(x + (n + r) * a.token_stride + 8 * c);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __builtin_amdgcn_ldexpf(bf16_to_float(w[i] & 0xffffu), -e_new);
      f[2 * i + 1] = __builtin_amdgcn_ldexpf(__builtin_bit_cast(float, w[i] & 0xffff0000u), -e_new);
    }
    const int32_t to = a.slots[n + r] & 63;
    *(u32x2*)(codes + to * a.D + 8 * c) =
        (u32x2){to_codes<CODE>(f[0], f[1], f[2], f[3]), to_codes<CODE>(f[4], f[5], f[6], f[7])};
  }
  if (lane == 0) *scale = __builtin_bit_cast(float, (uint32_t)(e_new + 127) << 23);
}

}  // namespace

hipError_t launch_gqa_append(const GqaAppendLaunch& a, hipStream_t s) {
  const int64_t waves = (int64_t)a.num_tokens * 2 * a.Hk;
  const int64_t groups = (waves + kThreads / 64 - 1) / (kThreads / 64);
  if (groups > 0x7fffffff) return hipErrorInvalidConfiguration;
  if (a.code_type == 0) hipLaunchKernelGGL(gqa_append_kernel<0>, dim3((unsigned)groups), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(gqa_append_kernel<1>, dim3((unsigned)groups), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace splash
