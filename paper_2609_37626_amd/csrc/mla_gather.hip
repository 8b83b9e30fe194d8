// gfx950 kernel of splash_mla_gather: cached rows back as dense bf16.
//
// A wave takes kRows output rows: lane i finds row i's request (the wave's first
// row by 64 comparisons at a time, the others from there on) and its place in the
// pool; then the wave reads row after row, 16 bytes of bf16 a lane (8 of codes),
// all rows' loads in flight before the first store.
//
// Bound: HBM (1,152, 580 or 656 bytes read and 1,152 written a row): 67k rows of the
// latent format are 122 MB in 20 us, 6.0 TB/s.  It is rows in flight that carry the
// rate: bounds of six waves a SIMD took it from 32.6 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"
#include "splash_attn.h"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 8;

// 8 codes times a scale, each rounded once to bf16.
__device__ __forceinline__ u32x4 values_of(u32x2 codes, float scale) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], true);
    r[2 * i] = pack_bf16x2(lo[0] * scale, lo[1] * scale);
    r[2 * i + 1] = pack_bf16x2(hi[0] * scale, hi[1] * scale);
  }
  return r;
}

template <int FORMAT>
__global__ __launch_bounds__(kThreads, 6) void mla_gather_kernel(MlaGatherLaunch a) {
  constexpr int kRowBytes = FORMAT == SPLASH_KV_BF16 ? 2 * kDimQK : FORMAT == SPLASH_KV_FP8_E4M3 ? kDimQK : kLatentRowBytes;
  const int lane = threadIdx.x & 63;
  const int64_t r0 = ((int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kRows;
  if (r0 >= min((int64_t)a.max_rows, (int64_t)a.row_indptr[a.B]) || r0 + kRows <= a.row_indptr[0]) return;
  // requests whose rows end at or before r0
  int b = 0;
  while (b < a.B) {
    const bool behind = b + lane < a.B && a.row_indptr[b + lane + 1] <= r0;
    const uint64_t stays = ~__ballot(behind);
    const int skip = stays ? __builtin_ctzll(stays) : 64;
    b += skip;
    if (skip < 64) break;
  }
  // lane i: row r0 + i, its slot in the pool (-1: a row of zeros, -2: none)
  int64_t slot = -2;
  const int64_t row = r0 + (lane < kRows ? lane : 0);
  if (lane < kRows && row < a.max_rows && row >= a.row_indptr[0]) {
    while (b < a.B && a.row_indptr[b + 1] <= row) ++b;
    if (b < a.B) {
      const int64_t at = (a.key_begin ? (int64_t)a.key_begin[b] : 0) + row - a.row_indptr[b];
      slot = -1;
      if (at >= 0 && (at >> 6) < a.bt_stride) {
        const int32_t page = a.block_table[(int64_t)b * a.bt_stride + (at >> 6)];
        if (page >= 0 && page < a.num_pages) slot = (int64_t)page * kPage + (at & 63);
      }
    }
  }
  const float scale = FORMAT == SPLASH_KV_FP8_E4M3 && slot >= 0 ? a.scales[slot] : 0.f;
  int32_t slots[kRows];  // (64 * num_pages is below 2^31)
#pragma unroll
  for (int i = 0; i < kRows; ++i) slots[i] = __builtin_amdgcn_readlane((int32_t)slot, i);

  // the latent
  u32x4 value[kRows];
  float tile_scale[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    value[i] = (u32x4){0u, 0u, 0u, 0u};
    tile_scale[i] = 0.f;
    if (slots[i] < 0) continue;
    const uint8_t* from = a.pages + (int64_t)slots[i] * kRowBytes;
    if constexpr (FORMAT == SPLASH_KV_BF16) {
      value[i] = *(const u32x4*)(from + 16 * lane);
    } else {
      const u32x2 c = *(const u32x2*)(from + 8 * lane);
      value[i][0] = c[0];
      value[i][1] = c[1];
      if constexpr (FORMAT == SPLASH_KV_FP8_LATENT) tile_scale[i] = *(const float*)(from + kDimV + 4 * (lane >> 4));
    }
  }
  // the keys: eight lanes a row, eight rows at a time
  const int mine = lane >> 3, piece = lane & 7;
  const int32_t key_slot = __shfl((int32_t)slot, mine);
  u32x4 key = {0u, 0u, 0u, 0u};
  if (key_slot >= 0) {
    const uint8_t* from = a.pages + (int64_t)key_slot * kRowBytes;
    if constexpr (FORMAT == SPLASH_KV_BF16) key = *(const u32x4*)(from + 2 * kDimV + 16 * piece);
    else if constexpr (FORMAT == SPLASH_KV_FP8_LATENT) key = *(const u32x4*)(from + kDimV + 16 + 16 * piece);
    else key = values_of(*(const u32x2*)(from + kDimV + 8 * piece), a.scales[key_slot]);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (slots[i] == -2) continue;
    if constexpr (FORMAT != SPLASH_KV_BF16) {
      const float by = FORMAT == SPLASH_KV_FP8_E4M3 ? __shfl(scale, i) : tile_scale[i];
      if (slots[i] >= 0) value[i] = values_of((u32x2){value[i][0], value[i][1]}, by);
    }
    *(u32x4*)(a.latent + (r0 + i) * a.latent_stride + 8 * lane) = value[i];
  }
  if (key_slot != -2) *(u32x4*)(a.key + (r0 + mine) * a.key_stride + 8 * piece) = key;
}

}  // namespace

hipError_t launch_mla_gather(const MlaGatherLaunch& a, hipStream_t s) {
  const unsigned rows = kThreads / 64 * kRows;
  const dim3 groups(((unsigned)a.max_rows + rows - 1) / rows);
  if (a.kv_dtype == SPLASH_KV_BF16) hipLaunchKernelGGL((mla_gather_kernel<SPLASH_KV_BF16>), groups, dim3(kThreads), 0, s, a);
  else if (a.kv_dtype == SPLASH_KV_FP8_E4M3) hipLaunchKernelGGL((mla_gather_kernel<SPLASH_KV_FP8_E4M3>), groups, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((mla_gather_kernel<SPLASH_KV_FP8_LATENT>), groups, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace splash
