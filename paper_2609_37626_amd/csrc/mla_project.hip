// gfx950 kernels of splash_mla_absorb_q and splash_mla_expand_out: per head a
// product of the tokens' rows with a 128 x 512 weight.
//
// The weight stays: a wave keeps its piece of it in registers as the A operand of
// v_mfma_f32_16x16x32_bf16 (D^T = W^T X^T) and walks over tiles of 16 tokens, whose
// rows are the B operand (lane (g, c): token c, eight values from 8 g).  D leaves lane
// (g, c) four rows 4 g .. of token c; a pair of tiles takes the weight's columns in the
// order that makes them eight neighbouring ones, so that a lane stores 16 bytes and four
// lanes 64 of a token.  Operands read from memory as they are multiplied, 64 bytes of each
// of 16 rows, cost absorb 10 of 23 us (queries) and expand 8 of 17 (the weight) at 256
// tokens of 128 heads: they come in whole lines straight into LDS instead.
//
// Bound: HBM (absorb: 384 bytes read and 1,152 written for 131,072 operations a row
// and head; expand: 1,024 and 256); for a few tokens the weight, 128 KiB a head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"
#include "lds_loads.hpp"
#include "turn.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 16;      // tokens of a tile
constexpr int kColumns = 128;  // latent columns of a workgroup of absorb
constexpr int kHeads = 32;     // heads of a wave of the rotary part

__device__ __forceinline__ bf16x8 load8(const uint16_t* p) { return __builtin_bit_cast(bf16x8, *(const u32x4*)p); }
__device__ __forceinline__ u32x4 round8(f32x4 lo, f32x4 hi) {
  return (u32x4){pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
}

// Workgroups go round the 8 XCDs: `inner` neighbours of one item share one of them, one
// after the other; fewer than 8 items are spread over all.  The items' places; false past
// the last.
__device__ __forceinline__ bool place(uint32_t at, uint32_t items, uint32_t inner, uint32_t& item, uint32_t& part) {
  if (items < 8) {
    item = at % items;
    part = at / items;
    return part < inner;
  }
  const uint32_t xcd = at & 7, n = at >> 3;
  part = n % inner;
  item = n / inner * 8 + xcd;
  return item < items;
}

// The rotary part of a token, kHeads heads a wave: the lane's pairs' sines and cosines
// are made once, 16 bytes of a head a lane.
__device__ __forceinline__ void turn_heads(const MlaAbsorbLaunch& a, int64_t n, int32_t first, int lane, float (&cosine)[kRopePairs],
                                           float (&sine)[kRopePairs]) {
  const uint16_t* q = a.q + n * a.q_token + kNope;
  uint16_t* out = a.out + n * a.heads * kDimQK + kDimV;
  const int32_t end = min(first + kHeads, a.heads);
  const bool turned = a.turn.positions != nullptr;
  if (turned && lane < kRopePairs) pair_turn(a.turn, pair_angle(a.turn, n, lane), cosine[lane], sine[lane]);
  __builtin_amdgcn_wave_barrier();  // (one wave's LDS is in order)
  if (!turned || a.turn.interleaved) {
    const int piece = lane & 7;
    f32x4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
    if (turned) {
      c = *(const f32x4*)(cosine + 4 * piece);
      s = *(const f32x4*)(sine + 4 * piece);
    }
    u32x4 x[kHeads / 8];
#pragma unroll
    for (int i = 0; i < kHeads / 8; ++i) x[i] = *(const u32x4*)(q + min(first + 8 * i + (lane >> 3), end - 1) * a.q_head + 8 * piece);
#pragma unroll
    for (int i = 0; i < kHeads / 8; ++i) {
      const int32_t h = first + 8 * i + (lane >> 3);
      if (turned) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x0 = __builtin_bit_cast(float, x[i][j] << 16), x1 = __builtin_bit_cast(float, x[i][j] & 0xffff0000u);
          x[i][j] = pack_bf16x2(x0 * c[j] - x1 * s[j], x1 * c[j] + x0 * s[j]);
        }
      }
      if (h < end) *(u32x4*)(out + (int64_t)h * kDimQK + 8 * piece) = x[i];
    }
  } else {
    const int piece = lane & 3;  // of the first half, and of the second
    f32x4 c[2], s[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      c[k] = *(const f32x4*)(cosine + 8 * piece + 4 * k);
      s[k] = *(const f32x4*)(sine + 8 * piece + 4 * k);
    }
    u32x4 lo[kHeads / 16], hi[kHeads / 16];
#pragma unroll
    for (int i = 0; i < kHeads / 16; ++i) {
      const uint16_t* x = q + min(first + 16 * i + (lane >> 2), end - 1) * a.q_head + 8 * piece;
      lo[i] = *(const u32x4*)x;
      hi[i] = *(const u32x4*)(x + kRopePairs);
    }
#pragma unroll
    for (int i = 0; i < kHeads / 16; ++i) {
      const int32_t h = first + 16 * i + (lane >> 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float c0 = c[j >> 1][2 * (j & 1)], c1 = c[j >> 1][2 * (j & 1) + 1], s0 = s[j >> 1][2 * (j & 1)], s1 = s[j >> 1][2 * (j & 1) + 1];
        const float a0 = __builtin_bit_cast(float, lo[i][j] << 16), a1 = __builtin_bit_cast(float, lo[i][j] & 0xffff0000u);
        const float b0 = __builtin_bit_cast(float, hi[i][j] << 16), b1 = __builtin_bit_cast(float, hi[i][j] & 0xffff0000u);
        lo[i][j] = pack_bf16x2(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
        hi[i][j] = pack_bf16x2(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
      }
      if (h < end) {
        uint16_t* to = out + (int64_t)h * kDimQK + 8 * piece;
        *(u32x4*)to = lo[i];
        *(u32x4*)(to + kRopePairs) = hi[i];
      }
    }
  }
}

// The first `products` workgroups: a head's block of 128 columns for `chunk` tokens, 32
// columns a wave; the others: the rotary parts.  In LDS the weight and two batches of 64
// tokens' rows, 256 bytes a row, in chunks of 16 bytes at chunk ^ 4 (row & 3) (the weight:
// the transposing reads take four rows together) and at chunk ^ (row & 15).
constexpr int kBatch = 64;
constexpr int kRowBytes = 2 * kNope;
__global__ __launch_bounds__(kThreads, 2) void mla_absorb_kernel(MlaAbsorbLaunch a, int32_t chunk, uint32_t products) {
  __shared__ __align__(16) uint8_t lds[(kNope + 2 * kBatch) * kRowBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x >= products) {
    float(*trig)[2][kRopePairs] = (float(*)[2][kRopePairs])lds;
    const int32_t groups = (a.heads + kHeads - 1) / kHeads;
    const int64_t at = (int64_t)(blockIdx.x - products) * kWaves + wave, n = at / groups;
    if (n < a.num_tokens) turn_heads(a, n, (int32_t)(at % groups) * kHeads, lane, trig[wave][0], trig[wave][1]);
    return;
  }
  const uint32_t chunks = ((uint32_t)a.num_tokens + chunk - 1) / chunk;
  // A head's four blocks on one XCD, which then reads its queries once (256 tokens of 128
  // heads: 15.6 us, 17.0 with the blocks apart), where the heads fill the XCDs evenly.
  constexpr uint32_t kColumnBlocks = kDimV / kColumns;
  const bool even = a.heads % 8 == 0;
  uint32_t item, part;
  if (!place(blockIdx.x, even ? a.heads : a.heads * kColumnBlocks, even ? chunks * kColumnBlocks : chunks, item, part)) return;
  const int c = lane & 15, g = lane >> 4, h = even ? item : item / kColumnBlocks;
  const int block = (even ? part : item) % kColumnBlocks;
  if (even) part /= kColumnBlocks;
  const int64_t begin = (int64_t)part * chunk, end = min(begin + chunk, (int64_t)a.num_tokens);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_AS uint8_t*)lds;
  const int row = lane >> 4, slot = lane & 15;  // of a load's four rows
  const uint16_t* w = a.w + h * a.w_head + block * kColumns;
#pragma unroll
  for (int i = 0; i < kNope / 4 / kWaves; ++i) {
    const int d = 4 * (kNope / 4 / kWaves * wave + i) + row;
    load_lds_from(w + d * a.w_row + 8 * (slot ^ (4 * (d & 3))), lds0 + (d - row) * kRowBytes);
  }
  const uint16_t* q = a.q + h * a.q_head;
  const auto load = [&](int64_t n0) {  // (a row past the last token: that one)
    const uint32_t to = lds0 + (kNope + ((n0 - begin) & kBatch)) * kRowBytes;
#pragma unroll
    for (int i = 0; i < kBatch / 4 / kWaves; ++i) {
      const int t = 4 * (kBatch / 4 / kWaves * wave + i) + row;
      load_lds_from(q + min(n0 + t, end - 1) * a.q_token + 8 * (slot ^ (t & 15)), to + (t - row) * kRowBytes);
    }
  };
  constexpr int kLoads = kBatch / 4 / kWaves;  // of a batch, by each wave
  load(begin);
  load(begin + kBatch);
  wait_vmcnt<2 * kLoads>();
  lds_barrier();
  // A operand of tile s: row m is column 32 wave + 8 (m >> 2) + 4 s + (m & 3); lane (g, c)
  // takes rows d = 32 k + 8 g .. + 7 of the weight.  A transposing read gives lane c of each
  // 16 the column c of four rows that the lanes point at, four columns a lane.
  const LDS_AS uint8_t* buf = (const LDS_AS uint8_t*)lds;
  bf16x8 wf[4][2];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const LDS_AS uint8_t* at = buf + (32 * k + 8 * g + (c >> 2)) * kRowBytes + 16 * ((4 * wave + (c & 3)) ^ (4 * (c >> 2))) + 8 * s;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)(at + 4 * kRowBytes));
      wf[k][s] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  uint16_t* out = a.out + (int64_t)h * kDimQK + block * kColumns + 32 * wave + 8 * g;
  for (int64_t n0 = begin; n0 < end; n0 += kBatch) {
    wait_vmcnt<kLoads>();  // (loads come in order; the last batch's are younger)
    lds_barrier();
    const LDS_AS uint8_t* x = buf + (kNope + ((n0 - begin) & kBatch) + c) * kRowBytes;
#pragma unroll
    for (int t = 0; t < kBatch / kTile; ++t) {
      if (n0 + kTile * t >= end) break;
      f32x4 d[2] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bf16x8 xf = *(const LDS_AS bf16x8*)(x + kTile * kRowBytes * t + 16 * ((4 * k + g) ^ c));
#pragma unroll
        for (int s = 0; s < 2; ++s) d[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[k][s], xf, d[s], 0, 0, 0);
      }
      const int64_t n = n0 + kTile * t + c;
      if (n < end) *(u32x4*)(out + n * a.heads * kDimQK) = round8(d[0], d[1]);
    }
    lds_barrier();  // nobody reads these rows any more
    load(n0 + 2 * kBatch);  // (past the chunk: its last row, so that every batch counts as many)
  }
  wait_vmcnt<0>();
}

// A head for 32 TILES tokens.  Waves w and w + 4 take 128 of the 512 latent columns, half
// of the tokens each, so that each row is read by one wave once; the four slices' sums meet in LDS, 32
// values a wave.  The weight comes through LDS in whole lines, 256 bytes of a row to a
// slice, in chunks of 16 bytes at chunk ^ (row & 15).
constexpr int kSlices = 4;
constexpr int kSlice = kDimV / kSlices;
constexpr int kExpandWaves = 2 * kSlices;
template <int TILES>  // of a wave, all on their way at once
__global__ __launch_bounds__(64 * kExpandWaves, 2) void mla_expand_kernel(MlaExpandLaunch a) {
  typedef float Sums[kExpandWaves][kTile][kValue + 4];
  __shared__ __align__(16) uint8_t lds[2 * sizeof(Sums)];
  static_assert(sizeof(lds) >= kValue * kDimV * 2, "the weight");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4, slice = wave % kSlices, side = wave / kSlices;
  constexpr int kSide = kTile * TILES;
  uint32_t h, part;
  if (!place(blockIdx.x, a.heads, ((uint32_t)a.num_tokens + 2 * kSide - 1) / (2 * kSide), h, part)) return;
  const int64_t first = (int64_t)part * 2 * kSide;
  const int64_t begin = min(first + side * kSide, (int64_t)a.num_tokens);
  const int64_t end = min(begin + kSide, (int64_t)a.num_tokens);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_AS uint8_t*)lds;
  const uint16_t* w = a.w + h * a.w_head + kSlice * slice;
  const int row = lane >> 4, slot = lane & 15;  // of a load's four rows
#pragma unroll
  for (int i = 0; i < kValue / 8; ++i) {
    const int v = kValue / 2 * side + 4 * i + row;
    load_lds_from(w + v * a.w_row + 8 * (slot ^ (v & 15)), lds0 + (slice * kValue + v - row) * kRowBytes);
  }
  const uint16_t* x = a.x + (int64_t)h * kDimV + kSlice * slice + 8 * g;
  bf16x8 xf[TILES][4];
#pragma unroll
  for (int t = 0; t < TILES; ++t)
    if (begin + kTile * t < end)
#pragma unroll
      for (int k = 0; k < 4; ++k) xf[t][k] = load8(x + min(begin + kTile * t + c, end - 1) * a.heads * kDimV + 32 * k);
  wait_vmcnt<0>();
  lds_barrier();
  const LDS_AS uint8_t* buf = (const LDS_AS uint8_t*)lds + (slice * kValue + c) * kRowBytes;
  bf16x8 wf[8][4];
#pragma unroll
  for (int v = 0; v < 8; ++v)
#pragma unroll
    for (int k = 0; k < 4; ++k) wf[v][k] = *(const LDS_AS bf16x8*)(buf + 16 * kRowBytes * v + 16 * ((4 * k + g) ^ c));
  lds_barrier();  // the weight's place becomes the sums'
  Sums* sums = (Sums*)lds;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    if (first + kTile * t >= a.num_tokens) break;  // (of the first side: the same for all waves)
    const int64_t n0 = begin + kTile * t;
    if (n0 < end) {
      f32x4 d[8] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int v = 0; v < 8; ++v) d[v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[v][k], xf[t][k], d[v], 0, 0, 0);
#pragma unroll
      for (int v = 0; v < 8; ++v) *(f32x4*)(&sums[t & 1][wave][c][16 * v + 4 * g]) = d[v];  // (two buffers: one barrier a tile)
    }
    __syncthreads();
    const int64_t n = n0 + c;
    if (n < end) {
      // lane (g, c): values 32 slice + 8 g .. of token c
      f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll
      for (int i = 0; i < kSlices; ++i) {
        const float* from = &sums[t & 1][kSlices * side + i][c][32 * slice + 8 * g];
        lo += *(const f32x4*)from;
        hi += *(const f32x4*)(from + 4);
      }
      *(u32x4*)(a.y + n * a.y_token + h * a.y_head + 32 * slice + 8 * g) = round8(lo, hi);
    }
  }
}

}  // namespace

hipError_t launch_mla_absorb(const MlaAbsorbLaunch& a, hipStream_t s) {
  // Tokens of a workgroup: what leaves 512 of them, 64 to 256.
  const uint32_t items = (uint32_t)a.heads * (kDimV / kColumns);
  const int64_t each = ((int64_t)a.num_tokens * items / 512 + kBatch - 1) / kBatch * kBatch;
  const int32_t chunk = each < kBatch ? kBatch : each > 4 * kBatch ? 4 * kBatch : (int32_t)each;
  const uint32_t chunks = ((uint32_t)a.num_tokens + chunk - 1) / chunk;
  const uint64_t products = (uint64_t)(items + 7) / 8 * 8 * chunks;
  const uint64_t turns = ((uint64_t)a.num_tokens * ((a.heads + kHeads - 1) / kHeads) + kWaves - 1) / kWaves;
  hipLaunchKernelGGL(mla_absorb_kernel, dim3((unsigned)(products + turns)), dim3(kThreads), 0, s, a, chunk, (uint32_t)products);
  return hipGetLastError();
}

namespace {
template <int TILES>
hipError_t launch_expand(const MlaExpandLaunch& a, hipStream_t s) {
  const uint32_t chunks = ((uint32_t)a.num_tokens + 2 * kTile * TILES - 1) / (2 * kTile * TILES);
  hipLaunchKernelGGL((mla_expand_kernel<TILES>), dim3(((uint32_t)a.heads + 7) / 8 * 8 * chunks), dim3(64 * kExpandWaves), 0, s, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_mla_expand(const MlaExpandLaunch& a, hipStream_t s) {
  // The fewest tokens a workgroup (32, 64 or 128) with which all of them begin at once, one
  // a compute unit: 635 tokens of 8 heads take 5.6 us so, 10.8 at 128.
  const auto groups = [&](int64_t tokens) { return a.heads * ((a.num_tokens + tokens - 1) / tokens); };
  if (groups(32) <= 256) return launch_expand<1>(a, s);
  return groups(64) <= 256 ? launch_expand<2>(a, s) : launch_expand<4>(a, s);
}

}  // namespace splash
