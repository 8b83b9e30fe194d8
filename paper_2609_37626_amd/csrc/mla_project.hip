// gfx950 kernels of splash_mla_absorb_q and splash_mla_expand_out: per head a
// product of the tokens' rows with a 128 x 512 weight.
//
// The weight stays: a wave keeps its piece of it in registers as the A operand of
// v_mfma_f32_16x16x32_bf16 (D^T = W^T X^T) and walks over tiles of 16 tokens, whose
// rows are the B operand straight from memory (lane (g, c): token c, eight values
// from 8 g).  D leaves lane (g, c) four rows 4 g .. of token c; a pair of tiles takes
// the weight's columns in the order that makes them eight neighbouring ones, so that
// a lane stores 16 bytes and four lanes 64 of a token.
//
// Bound: HBM (absorb: 384 bytes read and 1,152 written for 131,072 operations a row
// and head; expand: 1,024 and 256); for a few tokens the weight, 128 KiB a head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"
#include "turn.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 16;      // tokens of a tile
constexpr int kColumns = 128;  // latent columns of a workgroup of absorb

__device__ __forceinline__ bf16x8 load8(const uint16_t* p) { return __builtin_bit_cast(bf16x8, *(const u32x4*)p); }
__device__ __forceinline__ u32x4 round8(f32x4 lo, f32x4 hi) {
  return (u32x4){pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
}

// Grid: (token chunks, 4 column blocks and the rotary part, heads).
__global__ __launch_bounds__(kThreads, 2) void mla_absorb_kernel(MlaAbsorbLaunch a, int32_t chunk) {
  __shared__ __align__(16) uint16_t weight[kNope * kColumns];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int64_t begin = (int64_t)blockIdx.x * chunk, end = min(begin + chunk, (int64_t)a.num_tokens);
  const int h = blockIdx.z, block = blockIdx.y;
  const uint16_t* q = a.q + h * a.q_head;
  uint16_t* out = a.out + (int64_t)h * kDimQK;
  const int64_t out_token = (int64_t)a.heads * kDimQK;

  if (block == kDimV / kColumns) {  // the rotary part, a token a wave
    for (int64_t n = begin + wave; n < end; n += kThreads / 64) {
      float x = __builtin_bit_cast(float, (uint32_t)q[n * a.q_token + kNope + lane] << 16);
      if (a.turn.positions) {
        float cosine, sine;
        pair_turn(a.turn, n, pair_of(a.turn, lane), cosine, sine);
        x = turn_element(a.turn, lane, x, cosine, sine);
      }
      out[n * out_token + kDimV + lane] = (uint16_t)pack_bf16x2(x, 0.f);
    }
    return;
  }

  const uint16_t* w = a.w + h * a.w_head + block * kColumns;
#pragma unroll
  for (int i = 0; i < kNope * kColumns / 8 / kThreads; ++i) {
    const int piece = i * kThreads + threadIdx.x, d = piece / (kColumns / 8), at = piece % (kColumns / 8);
    *(u32x4*)(weight + d * kColumns + 8 * at) = *(const u32x4*)(w + d * a.w_row + 8 * at);
  }
  __syncthreads();
  // A operand of tile 2p + s: row m is column 32 p + 8 (m >> 2) + 4 s + (m & 3); lane (g, c)
  // takes rows d = 32 k + 8 g .. + 7 of the weight.  A transposing read gives lane c of each
  // 16 the column c of four rows that the lanes point at, four columns a lane.
  bf16x8 wf[4][8];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const uint16_t* at = weight + (32 * k + 8 * g + (c >> 2)) * kColumns + 32 * (t >> 1) + 8 * (c & 3) + 4 * (t & 1);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)(at + 4 * kColumns));
      wf[k][t] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  for (int64_t n0 = begin + kTile * wave; n0 < end; n0 += kTile * (kThreads / 64)) {
    const int64_t n = n0 + c;
    const uint16_t* row = q + min(n, end - 1) * a.q_token + 8 * g;
    bf16x8 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = load8(row + 32 * k);
    f32x4 d[8] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int t = 0; t < 8; ++t) d[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[k][t], x[k], d[t], 0, 0, 0);
    if (n < end) {
      uint16_t* to = out + n * out_token + block * kColumns + 8 * g;
#pragma unroll
      for (int p = 0; p < 4; ++p) *(u32x4*)(to + 32 * p) = round8(d[2 * p], d[2 * p + 1]);
    }
  }
}

// Grid: (token chunks, heads); a wave takes 32 of the head's 128 values.
__global__ __launch_bounds__(kThreads, 2) void mla_expand_kernel(MlaExpandLaunch a, int32_t chunk) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int64_t begin = (int64_t)blockIdx.x * chunk, end = min(begin + chunk, (int64_t)a.num_tokens);
  const int h = blockIdx.y;
  const uint16_t* w = a.w + h * a.w_head + 8 * g;
  bf16x8 wf[16][2];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int k = 0; k < 16; ++k) wf[k][s] = load8(w + (32 * wave + 8 * (c >> 2) + 4 * s + (c & 3)) * a.w_row + 32 * k);
  const uint16_t* x = a.x + (int64_t)h * kDimV + 8 * g;
  uint16_t* y = a.y + h * a.y_head + 32 * wave + 8 * g;
  for (int64_t n0 = begin; n0 < end; n0 += kTile) {
    const int64_t n = n0 + c;
    const uint16_t* row = x + min(n, end - 1) * a.heads * kDimV;
    f32x4 d[2] = {};
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const bf16x8 xf = load8(row + 32 * k);
#pragma unroll
      for (int s = 0; s < 2; ++s) d[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[k][s], xf, d[s], 0, 0, 0);
    }
    if (n < end) *(u32x4*)(y + n * a.y_token) = round8(d[0], d[1]);
  }
}

}  // namespace

hipError_t launch_mla_absorb(const MlaAbsorbLaunch& a, hipStream_t s) {
  const int32_t chunk = 64;
  const dim3 grid(((unsigned)a.num_tokens + chunk - 1) / chunk, kDimV / kColumns + 1, (unsigned)a.heads);
  hipLaunchKernelGGL(mla_absorb_kernel, grid, dim3(kThreads), 0, s, a, chunk);
  return hipGetLastError();
}

hipError_t launch_mla_expand(const MlaExpandLaunch& a, hipStream_t s) {
  const int32_t chunk = 64;
  const dim3 grid(((unsigned)a.num_tokens + chunk - 1) / chunk, (unsigned)a.heads);
  hipLaunchKernelGGL(mla_expand_kernel, grid, dim3(kThreads), 0, s, a, chunk);
  return hipGetLastError();
}

}  // namespace splash
