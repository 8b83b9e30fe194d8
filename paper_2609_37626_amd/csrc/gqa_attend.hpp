// gfx950 kernel of splash_gqa_attend: grouped-query attention over a paged
// cache of 8-bit codes with one scale per block (64 tokens of one KV head).
//
// A tile is one request, one KV head and 16 to 128 of its query rows (q_chunk
// rows times the heads that share the KV head): every K and V byte is read once
// for all of them (by two groups of waves where the rows take two).  A step is
// the pages that a group's waves take side by side, one each: four, or two for
// the larger row counts.  The tiles' steps, one tile after the other with
// kGqaTileCost places in front of each for its fixed work, form one line, which is
// cut into equal spans, one for each workgroup: long and short histories load
// the chip alike without a plan, and only the tiles that a cut goes through
// leave partial results, at most two a workgroup, which a second kernel joins.
// The waves' results of a piece are joined through LDS; nothing else goes through
// it: each operand is loaded from the cache in the layout that its MFMA reads,
// because the contraction's order is free as long as both operands agree on it.
//   QK  S^T[key, row] = K Q^T, v_mfma_f32_16x16x32_bf16.  Lane (g, c), g =
//       lane / 16, c = lane % 16, holds dims [64 i + 16 g, + 16) of key c for
//       every i, so that the four lanes of a key read whole 64-byte pieces; Q is
//       held the same way.
//   PV  O^T[dim, row] = V^T P^T, v_mfma_f32_16x16x32_f16.  S^T leaves lane
//       (g, c) with row c's weights of keys 4g .. 4g+3 of each 16-key group, so
//       those are the keys it contracts; V^T's lane loads dims [c D/16,
//       (c+1) D/16) of the same keys, and a byte permutation pairs its keys.
// A page's weights 2^(z - peak + 15) are taken against the row's own largest score
// in it, `peak`, and go to fp16 for PV, in two terms (2^-22 relative) for tiles of
// 16 rows and in one (2^-11 relative, down to 2^-29 of the largest) for more; what
// is below fp16's subnormals, 2^-40 of the largest weight, is lost, whatever came
// before and whatever the scales of V are.  The page's products and the sum of its weights meet the
// accumulators in fp32, times 2^(peak - m - 9) and, the products, the block's V
// scale.  The reference m moves only when a row's score passes it by 2^8, so that
// the accumulators are seldom multiplied; they stay below 2^14 a key.  (Weights
// against m itself lose a page whose scores lie 2^-20 and more below it, however
// large its V scale is.  Against `peak` costs 1%: 64 rows of 256 dims 90 us, 89
// against m.)
//
// Bound: HBM for 16 and 32 rows (a page costs 128 D bytes against 4 D x 64 flops a
// row, RG x 16 MT rows a tile); for more the conversions and matrix instructions of
// one wave a SIMD.  Every block of a request's rows walks its whole history, what a
// prompt's earlier rows do not see among it: 2,048 rows of a 2,048-token prompt, 64
// heads over 8 by 128 dims, take 323 us, 213 TFLOP/s of what they see.
// (Times in this file are of a call's two launches, in a graph.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "step.hpp"

namespace splash {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

namespace gqa {

constexpr int kWaves = 4;
constexpr float kPageShift = 15.f;    // a page's weights are 2^(z - peak + 15) against its own largest score
constexpr float kWeightShift = 6.f;   // sums and outputs are of 2^(z - m + 6)
constexpr float kMoveAt = 8.f;        // the reference moves once a score passes it by this
// Scores past this are rounded before the peak is taken off them, as the peak is:
// in one operation, exactly, against the rounded peak - 15, a weight would be off
// by what those two roundings leave (at 2^24 powers of two, past fp16's end; up to
// here 2^-14 at most).
constexpr float kFar = 1024.f;
constexpr float kNegInf = -__builtin_inff();

// Places of a tile in the line: kGqaTileCost for its fixed work (two to three
// steps' time: first loads, queries, the join; a ragged batch of 64 takes 67.9 us
// with 2, 68.8 with 3 and 69.6 with 4, 256 short histories 238, 240 and 241, 64
// rows of 256 dims 92, 91.5 and 90.5; with no such places the ragged batch took
// half as long again), then its steps (cut between any two pages the ragged batch
// took 3% longer).  A span is at least kLeastSpan places long.
constexpr int kLeastSpan = 3;

// ---- codes to MFMA operands (exact) --------------------------------------

// Eight codes (two dwords) to bf16.
template <int CODE>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t a, uint32_t b) {
  u32x4 r;
  if constexpr (CODE == 0) {
    r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.0f, false));
    r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.0f, true));
    r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.0f, false));
    r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.0f, true));
  } else {
    r[0] = pack_bf16x2((float)(int8_t)a, (float)(int8_t)(a >> 8));
    r[1] = pack_bf16x2((float)(int8_t)(a >> 16), (float)(int8_t)(a >> 24));
    r[2] = pack_bf16x2((float)(int8_t)b, (float)(int8_t)(b >> 8));
    r[3] = pack_bf16x2((float)(int8_t)(b >> 16), (float)(int8_t)(b >> 24));
  }
  return __builtin_bit_cast(bf16x8, r);
}

// The codes of one dim (byte `byte` of each dword) of two tokens to fp16.
// pair holds [t0.b, t1.b, t0.b+1, t1.b+1]; hi selects the second dim.  INT8
// codes come with their sign bit flipped (code + 128).
template <int CODE, bool HI>
__device__ __forceinline__ uint32_t pair_to_f16(uint32_t pair) {
  if constexpr (CODE == 0) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)pair, 1.0f, HI));
  } else {
    // 0x6400 | u is the half 1024 + u, exactly
    const uint32_t u = __builtin_amdgcn_perm(0x64646464u, pair, HI ? 0x04030402u : 0x04010400u);
    const f16x2 v = __builtin_bit_cast(f16x2, u) - (f16x2){(_Float16)1152.0f, (_Float16)1152.0f};
    return __builtin_bit_cast(uint32_t, v);
  }
}

// A product rounded by itself, whatever it is added to.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// What brings a K block's products to base-2 scores: kept off 0 and infinity, so
// that masked products stay -inf and zeros stay 0 whatever the two scales are.
__device__ __forceinline__ float score_scale(float k_scale, float scale_log2) {
  return __builtin_amdgcn_fmed3f(k_scale * scale_log2, 0x1p-149f, 0x1.fffffep127f);
}

// The largest of lanes c, c + 16, c + 32 and c + 48, in all four.  (The swap of
// x's odd 16-lane rows with its own even ones leaves each row beside its
// neighbour; then the halves likewise.  No trip through LDS: once a page.)
__device__ __forceinline__ float xor_max(float x) {
  const uint32_t a = __builtin_bit_cast(uint32_t, x);
  const auto rows = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, (uint32_t)rows[0]), __builtin_bit_cast(float, (uint32_t)rows[1])));
  const auto halves = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)halves[0]), __builtin_bit_cast(float, (uint32_t)halves[1]));
}
__device__ __forceinline__ float xor_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A row's 1 / sum and LSE from its reference and sum (no key: 0 and -inf; NaN stays).
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }
__device__ __forceinline__ float row_lse(float top, float sum) {
  return sum == 0.f ? kNegInf : (top - kWeightShift + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

// (uniform: through the scalar cache, so that it waits for no vector load)
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// 4-byte pieces as wide as a lane's share of a row.
template <int N>
struct Dwords {
  uint32_t v[N];
};
// `at` is uniform and `lane` the lane's own offset, so that the address takes one register.
// Non-temporal for V up to 128 dims, whose lines no other wave reads (16 lanes
// take a row: a whole 128-byte line, or at 64 dims half of one, of which the next
// load takes the rest): 256 histories of 1,024 to 4,096 tokens 260 -> 238 us, at 64
// dims 140 -> 137 (but 19.5 -> 20.3 for 32 rows and 64 histories), four of 65,536 to
// 131,072 134 -> 122. Not for the 16-byte pieces, whose lines a later load or
// another wave reads again: with both non-temporal 247 us for the 256 (120.5 for
// the four), and 104 instead of 92 for 64 rows of 256 dims.
// Pieces of 16 bytes lie `step` bytes apart.
template <int N>
__device__ __forceinline__ Dwords<N> load_dwords(const uint8_t* at, uint32_t lane, int step = 16) {
  Dwords<N> r;
  const uint8_t* p = at + lane;
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 x = *(const u32x4*)(p + step * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) r.v[4 * i + j] = x[j];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = __builtin_nontemporal_load((const u32x2*)p);
    r.v[0] = x[0];
    r.v[1] = x[1];
  } else {
    r.v[0] = __builtin_nontemporal_load((const uint32_t*)p);
  }
  return r;
}

// D head dims, MT 16-row MFMA tiles a wave, RG groups of waves that take other
// rows of the same pages.
template <int D, int MT, int RG>
struct Shape {
  static constexpr int kWaveRows = 16 * MT;
  static constexpr int kRows = RG * kWaveRows;
  static constexpr int kLanes = kWaves / RG;  // waves that take a piece's pages in turn
  static constexpr int kSteps = D / 32;       // QK MFMAs per 16 keys and row tile
  static constexpr int kKDw = D / 16;         // dwords of a lane's share of a K row (D/4 bytes)
  static constexpr int kVDw = D / 64;         // dwords of a lane's share of a V row (D/16 bytes)
  static constexpr int kDims = D / 16;        // dims of a lane's share, = MFMA row groups of O^T
  // fp16 terms of a weight.  Two (2^-22) where the second's matrix instructions
  // hide behind HBM: 16 rows, 237 us with either for 256 histories of 1,024 to
  // 4,096, 73.3 and 73.5 for 64 of 2,048 to 8,192 at 256 dims; one (2^-11, beside
  // the output's 2^-8) where they would not: 32 rows of 128 dims 67.5 us with one
  // and 70 with two, 64 rows of 256 dims 90 and 102, 128 rows of 64 dims 41 and 49.
  static constexpr int kTerms = MT == 1 ? 2 : 1;
  // Workgroups on a CU: two with 256 registers a wave, or one with 512.  Two for 64
  // dims and up to 32 rows, whose waves have few bytes on the way (256 histories
  // of 1,024 to 4,096, 8 rows INT8: 137 us, with one 139 to 140; 64 of 2,048 to
  // 8,192: 16 rows 17.6 and 17.2, 32 rows 20.3 either way).  One for the rest,
  // which two do not hold without scratch or which have half the spans to begin
  // and join with one: 64 dims E4M3 with 64 rows 27.6 against 31.4 and with 128 rows
  // 39.4 against 48 (INT8 27.6 either way, 39.7 against 41.6); 128 dims with 16
  // rows and 256 histories 238 against 248; with 32 rows, a ragged batch, 68 against 92.
  static constexpr int kPerCu = D == 64 && MT < 4 ? 2 : 1;
  // the waves' results are joined kPass dims of each share at a time
  static constexpr int kJoinBytes = kPerCu == 2 ? 65536 : 131072;
  static constexpr int kPass = (kWaves * kWaveRows * D * 4 <= kJoinBytes) ? kDims : kJoinBytes / (kWaves * kWaveRows * 64);
  static constexpr int kRowStride = 16 * kPass + 4;  // floats, padded by a 16-byte bank group
};

// 1 in every byte that is an E4M3 NaN (0x7f, 0xff).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t d) { return (((d & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// NaN codes of a page that some rows see in part: each lane looks through V for
// its own outputs; bit 4 j + i of `hit` is dim group j, element i.  (Rare, so
// V is read again, byte by byte, and the loop takes few registers.)
template <int D, int MT>
__device__ __forceinline__ void nan_rows(const uint8_t* vb, int key0, int seq, const int (&sees)[MT], uint64_t (&hit)[MT]) {
  const int g = (threadIdx.x & 63) >> 4;
  const int end = min(kPage, seq - key0);
#pragma unroll 1
  for (int tok = 0; tok < end; ++tok)
#pragma unroll 1
    for (int e = 0; e < D / 4; ++e)
      if ((vb[tok * D + (4 * g + (e & 3)) * (D / 16) + (e >> 2)] & 0x7f) == 0x7f)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          if (key0 + tok < sees[mt]) hit[mt] |= 1ull << e;
}

__device__ __forceinline__ int history(const GqaAttendLaunch& a, int b) {
  const int seq = a.seq_lens[b], most = a.bt_stride * kPage;
  return seq < 0 ? 0 : (seq > most ? most : seq);
}
__device__ __forceinline__ int pages_of(int seq) { return (seq + kPage - 1) / kPage; }
template <int LANES>
__device__ __forceinline__ int places_of(int seq) { return kGqaTileCost + (pages_of(seq) + LANES - 1) / LANES; }

// A workgroup's share of one tile: pages [p0, p1) of request b's KV head hk for
// the query rows from row0 on.  slot: -1 for a whole tile, else the partial
// slot that takes the result.
struct Piece {
  int b, hk, row0, seq, p0, p1, slot;
};

// Walks the span's pieces, and notes the tile that begins in it and ends past it.
struct Walk {
  int at, hi, chunk, b, b_start;
  int4 joined;
};
// The workgroup's span of the line: every thread sums a few requests' places, a
// scan over the workgroup gives the line's length and with it the spans, and
// the thread whose requests hold the span's start finds the request.
template <int LANES>
__device__ __forceinline__ Walk find_span(const GqaAttendLaunch& a, int tiles, int* lds) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int per = (a.B + 64 * kWaves - 1) / (64 * kWaves);
  int mine = 0;
  for (int k = 0; k < per; ++k) {
    const int b = t * per + k;
    if (b < a.B) mine += tiles * places_of<LANES>(history(a, b));
  }
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 63) lds[wave] = upto;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) upto += lds[w];
    total += lds[w];
  }
  const int chunk = max((total + a.workers - 1) / a.workers, kLeastSpan);
  const int lo = min((int64_t)blockIdx.x * chunk, (int64_t)total), hi = min((int64_t)lo + chunk, (int64_t)total);
  if (lo < hi && lo >= upto - mine && lo < upto) {
    int start = upto - mine;
    for (int b = t * per;; ++b) {
      const int next = start + tiles * places_of<LANES>(history(a, b));
      if (lo < next) {
        lds[kWaves] = b;
        lds[kWaves + 1] = start;
        break;
      }
      start = next;
    }
  }
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(lo),
          __builtin_amdgcn_readfirstlane(hi),
          __builtin_amdgcn_readfirstlane(chunk),
          __builtin_amdgcn_readfirstlane(lds[kWaves]),
          __builtin_amdgcn_readfirstlane(lds[kWaves + 1]),
          {-1, 0, 0, 0}};
}

template <int LANES>
__device__ __forceinline__ bool next_piece(const GqaAttendLaunch& a, int row_blocks, int rows_per_tile, Walk& w, Piece* out) {
  const int tiles = a.Hk * row_blocks;
  while (w.at < w.hi) {
    const int seq = history(a, w.b), pages = pages_of(seq), cost = places_of<LANES>(seq);
    const int tile = __builtin_amdgcn_readfirstlane((w.at - w.b_start) / cost), start = w.b_start + tile * cost;
    const int hk = __builtin_amdgcn_readfirstlane(tile / row_blocks), rb = tile - hk * row_blocks;
    const bool begins = w.at == start;
    int p0 = max(w.at - start - kGqaTileCost, 0) * LANES, p1 = max(min((w.hi - start - kGqaTileCost) * LANES, pages), 0);
    if (a.whole_tiles) {
      p0 = begins ? 0 : pages;
      p1 = pages;
    }
    const Piece piece = {w.b, hk, rb * rows_per_tile, seq, p0, p1, p0 > 0 ? 2 * (int)blockIdx.x : p1 < pages ? 2 * (int)blockIdx.x + 1 : -1};
    w.at = start + cost;
    if (tile == tiles - 1) {
      ++w.b;
      w.b_start = w.at;
    }
    // (a tile without a page belongs to the span of its first place)
    if (p0 < p1 || (pages == 0 && begins)) {
      if (p0 == 0 && p1 < pages)
        w.joined = {piece.b, hk, rb, (start + cost - 1) / w.chunk - (int)blockIdx.x + 1};
      *out = piece;
      return true;
    }
  }
  return false;
}

// The four waves' results of a piece, joined through LDS: whole tiles give the
// normalised rows and their LSE, others the rows over their largest reference,
// that reference and the weights' sum.
template <int D, int MT, int RG>
__device__ __forceinline__ void join_waves(const GqaAttendLaunch& a, const Piece& t, f32x4 (&o)[D / 16][MT],
                                           const float (&m)[MT], const float (&l)[MT], float* lds_o, float* lds_m,
                                           float* lds_l) {
  using S = Shape<D, MT, RG>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.q_chunk * a.group, Hq = a.Hk * a.group;
  const int first = wave / S::kLanes * S::kLanes;  // of the waves with these rows
  const int slot = t.slot;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float sum = xor_sum(l[mt]);
    if (g == 0) {
      lds_m[wave * S::kWaveRows + 16 * mt + c] = m[mt];
      lds_l[wave * S::kWaveRows + 16 * mt + c] = sum;
    }
  }
  __syncthreads();
  float by[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = kNegInf;
    for (int w = 0; w < S::kLanes; ++w) top = fmaxf(top, lds_m[(first + w) * S::kWaveRows + 16 * mt + c]);
    by[mt] = m[mt] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m[mt] - top);
    float sum = 0.f;
    for (int w = 0; w < S::kLanes; ++w) {
      const int at = (first + w) * S::kWaveRows + 16 * mt + c;
      const float mw = lds_m[at];
      sum += mw == kNegInf ? lds_l[at] : lds_l[at] * __builtin_amdgcn_exp2f(mw - top);  // (0 there, or NaN)
    }
    const int rr = wave / S::kLanes * S::kWaveRows + 16 * mt + c, r = t.row0 + rr;
    if (slot >= 0) {
      if (wave == first && g == 0) {
        f32x2* ml = (f32x2*)a.part_ml + (int64_t)slot * S::kRows + rr;
        *ml = (f32x2){top, sum};
      }
    } else {
      if (wave == first && g == 0 && a.lse && r < rows) {
        const int i = r / a.group, h = t.hk * a.group + r - i * a.group;
        a.lse[((int64_t)t.b * a.q_chunk + i) * Hq + h] = row_lse(top, sum);
      }
      by[mt] *= inverse(sum);
    }
  }
#pragma unroll
  for (int pass = 0; pass < S::kDims / S::kPass; ++pass) {
    if (pass) __syncthreads();
    // the lane's dims [c' kDims + pass * kPass, + kPass) of shares c' = 4g + i
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < S::kPass; j += 4) {
          f32x4 x;
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = o[pass * S::kPass + j + k][mt][i] * by[mt];
          *(f32x4*)(lds_o + (wave * S::kWaveRows + 16 * mt + c) * S::kRowStride + (4 * g + i) * S::kPass + j) = x;
        }
    __syncthreads();
    constexpr int kQuads = 4 * S::kPass;  // 4-float pieces of a row in this pass
    static_assert(S::kRows * kQuads % (64 * kWaves) == 0, "whole turns");
#pragma unroll 8
    for (int turn = 0; turn < S::kRows * kQuads / (64 * kWaves); ++turn) {
      const int e = turn * 64 * kWaves + threadIdx.x;
      const int rr = e / kQuads, k4 = e - rr * kQuads;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < S::kLanes; ++w) {
        const int from = (rr / S::kWaveRows * S::kLanes + w) * S::kWaveRows + rr % S::kWaveRows;
        x += *(const f32x4*)(lds_o + from * S::kRowStride + 4 * k4);
      }
      const int r = t.row0 + rr;
      const int share = (4 * k4) / S::kPass, d = share * S::kDims + pass * S::kPass + (4 * k4 - share * S::kPass);
      if (slot >= 0) {
        *(f32x4*)(a.part_out + ((int64_t)slot * S::kRows + rr) * D + d) = x;
      } else if (r < rows) {
        const int i = r / a.group, h = t.hk * a.group + r - i * a.group;
        *(u32x2*)(a.out + (((int64_t)t.b * a.q_chunk + i) * Hq + h) * D + d) =
            (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      }
    }
  }
}

template <int D, int MT, int RG, int CODE>
__global__ __launch_bounds__(64 * kWaves, (Shape<D, MT, RG>::kPerCu)) void gqa_attend_kernel(GqaAttendLaunch a) {
  using S = Shape<D, MT, RG>;
  __shared__ __align__(16) float lds_o[kWaves * S::kWaveRows * S::kRowStride];
  __shared__ float lds_m[kWaves * S::kWaveRows];
  __shared__ float lds_l[kWaves * S::kWaveRows];
  __shared__ int lds_span[kWaves + 2];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int turn = wave % S::kLanes;                     // of the waves with the same rows
  const int wave_row = wave / S::kLanes * S::kWaveRows;  // first row in the tile
  const int rows = a.q_chunk * a.group, Hq = a.Hk * a.group;
  const int row_blocks = (rows + S::kRows - 1) / S::kRows;
  Walk walk = find_span<S::kLanes>(a, a.Hk * row_blocks, lds_span);
  Piece t, next_t;
  bool more = next_piece<S::kLanes>(a, row_blocks, S::kRows, walk, &t);
  if (!more) {
    if (threadIdx.x == 0) a.joined[blockIdx.x] = walk.joined;
    return;
  }

  // queries: dims 64 i + 16 g, + 16 of row c of each MFMA tile, eight a step
  bf16x8 q[MT][S::kSteps];
  const auto load_q = [&](const Piece& t) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int r = min(t.row0 + wave_row + 16 * mt + c, rows - 1);
      const int i = r / a.group, h = t.hk * a.group + r - i * a.group;
      const uint16_t* src = a.q + (((int64_t)t.b * a.q_chunk + i) * Hq + h) * D + 16 * g;
#pragma unroll
      for (int s = 0; s < S::kSteps; ++s) q[mt][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(src + 64 * (s >> 1) + 8 * (s & 1)));
    }
  };
  typedef Dwords<S::kKDw> KPage[4];
  typedef Dwords<S::kVDw> VPage[2][8];  // eight tokens a half page and lane
  KPage k;
  VPage v;
  const uint32_t k_lane = c * D + 16 * g, v_lane = 4 * g * D + c * (D / 16);
  const auto load_k = [&](int64_t block) {
    const uint8_t* kb = a.k_pages + block * (kPage * D);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) k[kt] = load_dwords<S::kKDw>(kb + 16 * kt * D, k_lane, 64);
  };
  const auto load_v = [&](int64_t block) {
    const uint8_t* vb = a.v_pages + block * (kPage * D);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int x = 0; x < 8; ++x) v[h][x] = load_dwords<S::kVDw>(vb + (32 * h + 16 * (x >> 2) + (x & 3)) * D, v_lane);
  };

  // The wave's pages of a piece are p0 + turn, + kLanes, ...  A page's V is
  // loaded before its QK and the next page's K after it, into the next piece at
  // the end of one; the block-table entry of the page after that is on its way.
  // An entry outside the pool reads page 0, all of it masked; past a piece's last
  // page that page is read again.
  const auto entry = [&](const Piece& t, int n) {
    const int p = max(min(t.p0 + turn + n * S::kLanes, t.p1 - 1), 0);
    return scalar_load(a.block_table + (int64_t)t.b * a.bt_stride + p);
  };
  const auto block_of = [&](int page, int hk) {
    return (int64_t)((unsigned)page < (unsigned)a.num_pages ? page : 0) * a.Hk + hk;
  };
  int page = entry(t, 0), next = entry(t, 1);
  int64_t block = block_of(page, t.hk);
  load_q(t);
  load_k(block);
  while (true) {
    more = next_piece<S::kLanes>(a, row_blocks, S::kRows, walk, &next_t);
    if (!more) next_t = t;
    const int pages = t.p0 + turn < t.p1 ? (t.p1 - t.p0 - turn + S::kLanes - 1) / S::kLanes : 0;  // of this wave
    if (pages == 1) next = entry(next_t, 0);
    const int row0 = t.row0 + wave_row;
    int sees[MT];  // keys that this lane's row sees
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sees[mt] = t.seq - a.q_chunk + min(row0 + 16 * mt + c, rows - 1) / a.group + 1;
    const int all_see = t.seq - a.q_chunk + min(row0, rows - 1) / a.group + 1;  // keys that every row of the wave sees

    f32x4 o[S::kDims][MT];
    float m[MT], l[MT];
    uint64_t hit[MT];  // NaN outputs, see nan_rows()
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      hit[mt] = 0;
      m[mt] = kNegInf;
      l[mt] = 0.f;
#pragma unroll
      for (int j = 0; j < S::kDims; ++j) o[j][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    float ks = score_scale(scalar_load(a.k_scales + block), a.scale_log2), vs = scalar_load(a.v_scales + block);
    for (int n = 0; n < pages; ++n) {
      const int p = t.p0 + turn + n * S::kLanes;
      const bool held = (unsigned)page < (unsigned)a.num_pages;
      const bool masked = !held || 64 * p + 64 > all_see;
      if (!held) ks = 1.f, vs = 0.f;  // (whatever the scales of page 0 are)
      const uint8_t* vb = a.v_pages + block * (kPage * D);
      const int after = n + 2 < pages ? entry(t, n + 2) : entry(next_t, n + 2 - pages);
      const int64_t next_block = block_of(next, n + 1 < pages ? t.hk : next_t.hk);
      const float next_ks = score_scale(scalar_load(a.k_scales + next_block), a.scale_log2), next_vs = scalar_load(a.v_scales + next_block);
      load_v(block);
      __builtin_amdgcn_sched_barrier(0);

      // scores
      f32x4 z[4][MT];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) z[kt][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
          const bf16x8 kf = codes_to_bf16<CODE>(k[kt].v[2 * s], k[kt].v[2 * s + 1]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            z[kt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[mt][s], z[kt][mt], 0, 0, 0);
        }
        if (kt & 1) __builtin_amdgcn_sched_barrier(0);  // (or all of K is converted ahead, in twice its registers)
      }
      load_k(next_block);
      __builtin_amdgcn_sched_barrier(0);

      if (masked) {
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!held || 64 * p + 16 * kt + 4 * g + i >= sees[mt]) z[kt][mt][i] = kNegInf;
      }

      // weights (ks brings the products to base-2 scores)
      uint32_t w[MT][S::kTerms][2][4];
      float v_by[MT];  // what brings a row's products to its reference: 2^(peak - m) and V's scale
      float peaks[MT];  // the rows' largest scores in this page
      bool far = false;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float top = kNegInf;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, z[kt][mt][i]);
        peaks[mt] = rounded_product(xor_max(top), ks);
        far |= __builtin_fabsf(peaks[mt]) > kFar && peaks[mt] != kNegInf;
      }
      // Far scores by their distances to the peak, each rounded like the peak itself.
      const bool distances = __any(far);
      if (distances)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[kt][mt][i] = rounded_product(z[kt][mt][i], ks) - (peaks[mt] == kNegInf ? 0.f : peaks[mt]);
      const float to_two = distances ? 1.f : ks;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const float peak = peaks[mt];
        if (__any(peak > m[mt] + kMoveAt)) {
          const float now = fmaxf(m[mt], peak);
          const float by = now == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m[mt] - now);
          m[mt] = now;
          l[mt] *= by;
#pragma unroll
          for (int j = 0; j < S::kDims; ++j) o[j][mt] *= by;
        }
        const float ref = distances ? -kPageShift : peak == kNegInf ? 0.f : peak - kPageShift;
        const float by = peak == kNegInf ? 0.f : __builtin_amdgcn_exp2f(peak - m[mt] + (kWeightShift - kPageShift));
        float sum = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[kt][mt][i], to_two, -ref));
            sum += e[i];
          }
#pragma unroll
          for (int term = 0; term < S::kTerms; ++term)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              const uint32_t pair = pack_f16x2(e[i], e[i + 1]);
              w[mt][term][kt >> 1][2 * (kt & 1) + i / 2] = pair;
              if (term + 1 < S::kTerms) {  // what is left of the weights, exactly
                e[i] -= (float)__builtin_bit_cast(f16x2, pair)[0];
                e[i + 1] -= (float)__builtin_bit_cast(f16x2, pair)[1];
              }
            }
        }
        l[mt] = __builtin_fmaf(sum, by, l[mt]);
        v_by[mt] = vs * by;
      }

      // Codes of places that no row sees count as 0, and so do NaN codes of a
      // page that some row sees in part; nan_rows() gives those to their rows.
      if (masked) {
        const int end = held ? t.seq - 64 * p : 0;
        uint32_t found = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int x = 0; x < S::kVDw; ++x) {
              uint32_t& d = v[h][t].v[x];
              if (32 * h + 16 * (t >> 2) + 4 * g + (t & 3) >= end) d = 0;
              if constexpr (CODE == 0) {
                const uint32_t bad = nan_bytes(d);
                d &= ~(bad * 255u);
                found |= bad;
              }
            }
        if constexpr (CODE == 0) {
          if (__any(found != 0)) nan_rows<D, MT>(vb, 64 * p, held ? t.seq : 0, sees, hit);
        }
      }
#pragma unroll
      for (int x = 0; x < S::kVDw; ++x)
#pragma unroll
        for (int pr = 0; pr < 2; ++pr) {  // dims 4x + 2 pr, 4x + 2 pr + 1
          u32x4 f[2][2];                  // [dim][half]
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              uint32_t pair = __builtin_amdgcn_perm(v[h][2 * t + 1].v[x], v[h][2 * t].v[x], pr ? 0x07030602u : 0x05010400u);
              if constexpr (CODE == 1) pair ^= 0x80808080u;
              f[0][h][t] = pair_to_f16<CODE, false>(pair);
              f[1][h][t] = pair_to_f16<CODE, true>(pair);
            }
#pragma unroll
          for (int dd = 0; dd < 2; ++dd) {
            const int j = 4 * x + 2 * pr + dd;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int term = 0; term < S::kTerms; ++term)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const uint32_t(&wf)[4] = w[mt][term][h];
                  t = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, f[dd][h]),
                                                             __builtin_bit_cast(f16x8, (u32x4){wf[0], wf[1], wf[2], wf[3]}), t, 0, 0, 0);
                }
#pragma unroll
              for (int i = 0; i < 4; ++i) o[j][mt][i] = __builtin_fmaf(v_by[mt], t[i], o[j][mt][i]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      page = next;
      next = after;
      block = next_block;
      ks = next_ks;
      vs = next_vs;
    }
    if (more) {
      if (pages == 0) {  // (the wave loaded a page of this piece that is not its own)
        page = entry(next_t, 0);
        next = entry(next_t, 1);
        block = block_of(page, next_t.hk);
        load_k(block);
      }
      load_q(next_t);
    }
    if constexpr (CODE == 0) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        if (__any(hit[mt] != 0))
#pragma unroll
          for (int j = 0; j < S::kDims; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (hit[mt] >> (4 * j + i) & 1) o[j][mt][i] = __builtin_nanf("");
    }

    join_waves<D, MT, RG>(a, t, o, m, l, lds_o, lds_m, lds_l);
    if (!more) break;
    __syncthreads();
    t = next_t;
  }
  if (threadIdx.x == 0) a.joined[blockIdx.x] = walk.joined;
}

// Joins the parts of the tile whose first part workgroup blockIdx.y of the
// attend kernel has, if any: one wave per row.  The parts lie in slots 2w + 1,
// 2(w + 1), 2(w + 2), ...; lanes take 4 dims each, 64 / (D / 4) parts at a time.
// (Rows along x: equal histories begin in every n-th workgroup, and along x those
// would all run on one XCD where n is a multiple of 8; the join alone of 32 tiles of
// 64 rows by 256 dims in eight parts 8.5 -> 7.0 us.)
template <int D, int ROWS>
__global__ __launch_bounds__(64 * kWaves) void gqa_join_kernel(GqaAttendLaunch a) {
  const int w = blockIdx.y, lane = threadIdx.x & 63;
  const int4 tile = a.joined[w];
  if (tile.x < 0) return;
  const int rr = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = tile.z * ROWS + rr;
  if (r >= a.q_chunk * a.group) return;
  const int parts = tile.w;
  const auto at = [&](int p) { return (int64_t)(p == 0 ? 2 * w + 1 : 2 * (w + p)) * ROWS + rr; };
  const f32x2* ml = (const f32x2*)a.part_ml;
  constexpr int kLanes = D / 4, kSide = 64 / kLanes;  // lanes of a row; parts side by side
  constexpr int kAhead = 8;                           // their loads, on the way before the weights are known
  const int side = lane / kLanes, d = 4 * (lane % kLanes);
  f32x4 x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int p = side + k * kSide;
    x[k] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (p < parts) x[k] = *(const f32x4*)(a.part_out + at(p) * D + d);
  }
  const f32x2 own = lane < parts ? ml[at(lane)] : (f32x2){kNegInf, 0.f};
  float top = own[0];
  for (int p = lane + 64; p < parts; p += 64) top = fmaxf(top, ml[at(p)][0]);
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
  const auto weight = [&](float m) { return m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - top); };
  const float by = weight(own[0]);
  float sum = own[1] * by;
  for (int p = lane + 64; p < parts; p += 64) {
    const f32x2 v = ml[at(p)];
    sum += v[1] * weight(v[0]);
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const float f = __shfl(by, side + k * kSide);  // (0 past the last part: x is 0 there)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(x[k][i], f, o[i]);
  }
  for (int p = side + kAhead * kSide; p < parts; p += kSide) {
    const float f = weight(ml[at(p)][0]);
    const f32x4 y = *(const f32x4*)(a.part_out + at(p) * D + d);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(y[i], f, o[i]);
  }
#pragma unroll
  for (int k = kLanes; k < 64; k <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], k);
  const int i = r / a.group, h = tile.y * a.group + r - i * a.group;
  const int64_t row = ((int64_t)tile.x * a.q_chunk + i) * (a.Hk * a.group) + h;
  if (lane < kLanes) {
    const float inv = inverse(sum);
    *(u32x2*)(a.out + row * D + d) = (u32x2){pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    if (lane == 0 && a.lse) a.lse[row] = row_lse(top, sum);
  }
}

template <int D, int MT, int RG, int CODE>
hipError_t launch_shape(GqaAttendLaunch a, hipStream_t s) {
  using S = Shape<D, MT, RG>;
  const int64_t row_blocks = ((int64_t)a.q_chunk * a.group + S::kRows - 1) / S::kRows;
  a.workers = a.workers * S::kPerCu < kGqaMaxWorkers ? a.workers * S::kPerCu : kGqaMaxWorkers;
  // no more workgroups than the longest histories would fill
  const int64_t most = ((int64_t)a.B * a.Hk * row_blocks * ((a.bt_stride + S::kLanes - 1) / S::kLanes + kGqaTileCost) + kLeastSpan - 1) / kLeastSpan;
  if (a.workers > most) a.workers = (int32_t)most;
  // Few short tiles are not cut: each goes to the span that it begins in, and
  // there is nothing to join (8 tiles of 2 to 8 pages: one launch of 7 us instead
  // of 7 and 4). At 16 pages a wave has four.
  a.whole_tiles = a.bt_stride <= 16 && (int64_t)a.B * a.Hk * row_blocks <= a.workers;
  hipLaunchKernelGGL((gqa_attend_kernel<D, MT, RG, CODE>), dim3(a.workers), dim3(64 * kWaves), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.whole_tiles) return e;
  hipLaunchKernelGGL((gqa_join_kernel<D, S::kRows>), dim3(S::kRows / kWaves, a.workers), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

template <int CODE>
hipError_t launch_code(const GqaAttendLaunch& a, hipStream_t s) {
  const int32_t rows = gqa_tile_rows(a.D, (int64_t)a.q_chunk * a.group);
  if (a.D == 64) {
    if (rows == 16) return launch_shape<64, 1, 1, CODE>(a, s);
    if (rows == 32) return launch_shape<64, 2, 1, CODE>(a, s);
    if (rows == 64) return launch_shape<64, 4, 1, CODE>(a, s);
    return launch_shape<64, 4, 2, CODE>(a, s);
  }
  if (a.D == 128) {
    if (rows == 16) return launch_shape<128, 1, 1, CODE>(a, s);
    if (rows == 32) return launch_shape<128, 2, 1, CODE>(a, s);
    if (rows == 64) return launch_shape<128, 4, 1, CODE>(a, s);
    return launch_shape<128, 4, 2, CODE>(a, s);
  }
  if (rows == 16) return launch_shape<256, 1, 1, CODE>(a, s);
  if (rows == 32) return launch_shape<256, 2, 1, CODE>(a, s);
  return launch_shape<256, 2, 2, CODE>(a, s);
}

}  // namespace gqa
}  // namespace splash
