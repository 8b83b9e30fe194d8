// gfx950 kernel of splash_gqa_attend: grouped-query attention over a paged
// cache of 8-bit codes with one scale per block (64 tokens of one KV head).
//
// A tile is one request, one KV head and up to 16*MT of its query rows
// (q_chunk rows times the heads that share the KV head): every K and V byte is
// read once for all of them.  The tiles' pages, one tile after the other with
// kTileCost places in front of each for its fixed work, form one line, which is
// cut into equal spans, one for each workgroup: long and short histories load
// the chip alike without a plan, and only the tiles that a cut goes through
// leave partial results, at most two a workgroup, which a second kernel joins.
// A workgroup's four waves take the pages of a span's tile in turn, one a step,
// and join their results through LDS.  Nothing else goes through LDS: each
// operand is loaded from the cache in the layout that its MFMA reads, because
// the contraction's order is free as long as both operands agree on it.
//   QK  S^T[key, row] = K Q^T, v_mfma_f32_16x16x32_bf16.  Lane (g, c), g =
//       lane / 16, c = lane % 16, holds key c's dims [g D/4, (g+1) D/4) as
//       contiguous bytes; Q is held the same way.
//   PV  O^T[dim, row] = V^T P^T, v_mfma_f32_16x16x32_f16.  S^T leaves lane
//       (g, c) with row c's weights of keys 4g .. 4g+3 of each 16-key group, so
//       those are the keys it contracts; V^T's lane loads dims [c D/16,
//       (c+1) D/16) of the same keys, and a byte permutation pairs its keys.
// The weights 2^(z - m + 6) are taken against a reference m that moves only
// when a row's maximum passes it by 2^8, so a weight stays below 2^14 and no
// exchange between lanes is needed on the other steps; 2^6 keeps the small ones
// off fp16's subnormals.  P is rounded to fp16 (2^-12 relative) for PV.  A
// block's V scale multiplies its product in fp32, never the weights.
//
// Bound: HBM.  A page costs 128 D bytes against 4 D x 64 x 16 MT flops.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "step.hpp"

namespace splash {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

namespace gqa {

constexpr int kWaves = 4;
constexpr float kWeightShift = 6.f;   // weights are 2^(z - m + 6)
constexpr float kMoveAt = 8.f;        // the reference moves once a score passes it by this
constexpr float kNegInf = -__builtin_inff();

// Places of a tile in the line: kTileCost for its fixed work, then its pages.
// A span is at least kLeastSpan places long: a page and a tile's fixed work
// for each wave.
constexpr int kTileCost = 2;
constexpr int kLeastSpan = 6;

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

__device__ __forceinline__ float xor_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
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
template <int N>
__device__ __forceinline__ Dwords<N> load_dwords(const uint8_t* at, uint32_t lane) {
  Dwords<N> r;
  const uint8_t* p = at + lane;
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 x = *(const u32x4*)(p + 16 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) r.v[4 * i + j] = x[j];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = *(const u32x2*)p;
    r.v[0] = x[0];
    r.v[1] = x[1];
  } else {
    r.v[0] = *(const uint32_t*)p;
  }
  return r;
}

template <int D, int MT>
struct Shape {
  static constexpr int kRows = 16 * MT;
  static constexpr int kSteps = D / 32;     // QK MFMAs per 16 keys and row tile
  static constexpr int kKDw = D / 16;       // dwords of a lane's share of a K row (D/4 bytes)
  static constexpr int kVDw = D / 64;       // dwords of a lane's share of a V row (D/16 bytes)
  static constexpr int kDims = D / 16;      // dims of a lane's share, = MFMA row groups of O^T
  static constexpr int kPerCu = D * MT <= 256 && D < 256 ? 2 : 1;  // workgroups on a CU: 256 registers a wave, or 512
  // the four waves' results are joined kPass dims of each share at a time, in at most 64 KB
  static constexpr int kPass = (kWaves * kRows * D * 4 <= 65536) ? kDims : 65536 / (kWaves * kRows * 64);
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

// One tile's pages [p0, p1) on the four waves.  Writes the normalised rows and
// their LSE, or, with a partial slot (>= 0), the rows over their largest
// reference, that reference and the weights' sum.
template <int D, int MT, int CODE>
__device__ __forceinline__ void attend_pages(const GqaAttendLaunch& a, int b, int hk, int row0, int seq, int p0, int p1,
                                             int slot, float* lds_o, float* lds_m, float* lds_l) {
  using S = Shape<D, MT>;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.q_chunk * a.group;
  const int Hq = a.Hk * a.group;

  // queries: row row0 + 16 mt + c, dims [g D/4, ...), eight a step
  bf16x8 q[MT][S::kSteps];
  int sees[MT];  // keys that this lane's row sees
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = row0 + 16 * mt + c;
    const int rr = r < rows ? r : rows - 1;
    const int i = rr / a.group, h = hk * a.group + rr - i * a.group;
    const uint16_t* src = a.q + (((int64_t)b * a.q_chunk + i) * Hq + h) * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) {
      u32x4 x = *(const u32x4*)(src + 8 * s);
      if (r >= rows) x = (u32x4){0, 0, 0, 0};
      q[mt][s] = __builtin_bit_cast(bf16x8, x);
    }
    sees[mt] = seq - a.q_chunk + i + 1;
  }
  // keys that every row of the tile sees (a page below it needs no mask), and
  // that the last row sees
  const int all_see = seq - a.q_chunk + row0 / a.group + 1;

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

  // The wave's pages p0 + wave, + kWaves, ...: while a page is worked on, its V
  // is in flight from before QK and the next page's K from after it, and the
  // block-table entry of the page after that is on its way.  A place whose entry
  // lies outside the pool reads page 0, all of it masked; past the last page the
  // last one is read again.
  const int32_t* bt = a.block_table + (int64_t)b * a.bt_stride;
  const auto entry = [&](int p) { return scalar_load(bt + min(p, p1 - 1)); };
  const auto block_of = [&](int page) {
    return (int64_t)((unsigned)page < (unsigned)a.num_pages ? page : 0) * a.Hk + hk;
  };
  const uint32_t k_lane = c * D + g * (D / 4), v_lane = 4 * g * D + c * (D / 16);
  Dwords<S::kKDw> k[4];
  const auto load_k = [&](int64_t block) {
    const uint8_t* kb = a.k_pages + block * (kPage * D);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) k[kt] = load_dwords<S::kKDw>(kb + 16 * kt * D, k_lane);
  };
  int p = p0 + wave, page = entry(p), next = entry(p + kWaves);
  int64_t block = block_of(page);
  float ks = scalar_load(a.k_scales + block) * a.scale_log2, vs = scalar_load(a.v_scales + block);
  if (p < p1) load_k(block);
  for (; p < p1; p += kWaves) {
    const bool held = (unsigned)page < (unsigned)a.num_pages;
    const bool masked = !held || 64 * p + 64 > all_see;

    // values: eight tokens a half page and lane
    const uint8_t* vb = a.v_pages + block * (kPage * D);
    Dwords<S::kVDw> v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < 8; ++t)
        v[h][t] = load_dwords<S::kVDw>(vb + (32 * h + 16 * (t >> 2) + (t & 3)) * D, v_lane);
    const int after = entry(p + 2 * kWaves);
    const int64_t next_block = block_of(next);
    const float next_ks = scalar_load(a.k_scales + next_block) * a.scale_log2, next_vs = scalar_load(a.v_scales + next_block);
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

#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) z[kt][mt] *= ks;
    if (masked) {
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!held || 64 * p + 16 * kt + 4 * g + i >= sees[mt]) z[kt][mt][i] = kNegInf;
    }

    // weights
    uint32_t w[MT][2][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float top = kNegInf;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, z[kt][mt][i]);
      if (__any(top > m[mt] + kMoveAt)) {
        const float now = fmaxf(m[mt], xor_max(top));
        const float by = now == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m[mt] - now);
        m[mt] = now;
        l[mt] *= by;
#pragma unroll
        for (int j = 0; j < S::kDims; ++j) o[j][mt] *= by;
      }
      const float ref = m[mt] == kNegInf ? 0.f : m[mt] - kWeightShift;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[i] = __builtin_amdgcn_exp2f(z[kt][mt][i] - ref);
          l[mt] += e[i];
        }
        w[mt][kt >> 1][2 * (kt & 1)] = pack_f16x2(e[0], e[1]);
        w[mt][kt >> 1][2 * (kt & 1) + 1] = pack_f16x2(e[2], e[3]);
      }
    }

    // Codes of places that no row sees count as 0, and so do NaN codes of a
    // page that some row sees in part; nan_rows() gives those to their rows.
    if (masked) {
      const int end = held ? seq - 64 * p : 0;
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
        if (__any(found != 0)) nan_rows<D, MT>(vb, 64 * p, held ? seq : 0, sees, hit);
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
            for (int h = 0; h < 2; ++h) {
              const u32x4 wf = {w[mt][h][0], w[mt][h][1], w[mt][h][2], w[mt][h][3]};
              t = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, f[dd][h]),
                                                         __builtin_bit_cast(f16x8, wf), t, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][mt][i] = __builtin_fmaf(vs, t[i], o[j][mt][i]);
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

  // join the four waves: every row's largest reference, then the waves' rows
  // brought to it
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float sum = xor_sum(l[mt]);
    if (g == 0) {
      lds_m[wave * S::kRows + 16 * mt + c] = m[mt];
      lds_l[wave * S::kRows + 16 * mt + c] = sum;
    }
  }
  __syncthreads();
  float by[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = kNegInf;
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_m[w * S::kRows + 16 * mt + c]);
    by[mt] = m[mt] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m[mt] - top);
    float sum = 0.f;
    for (int w = 0; w < kWaves; ++w) {
      const float mw = lds_m[w * S::kRows + 16 * mt + c];
      sum += mw == kNegInf ? 0.f : lds_l[w * S::kRows + 16 * mt + c] * __builtin_amdgcn_exp2f(mw - top);
    }
    const int r = row0 + 16 * mt + c;
    if (slot >= 0) {
      if (wave == 0 && g == 0) {
        f32x2* ml = (f32x2*)a.part_ml + (int64_t)slot * S::kRows + 16 * mt + c;
        *ml = (f32x2){top, sum};
      }
    } else {
      if (wave == 0 && g == 0 && a.lse && r < rows) {
        const int i = r / a.group, h = hk * a.group + r - i * a.group;
        a.lse[((int64_t)b * a.q_chunk + i) * Hq + h] = row_lse(top, sum);
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
          *(f32x4*)(lds_o + (wave * S::kRows + 16 * mt + c) * S::kRowStride + (4 * g + i) * S::kPass + j) = x;
        }
    __syncthreads();
    constexpr int kQuads = 4 * S::kPass;  // 4-float pieces of a row in this pass
    for (int e = threadIdx.x; e < S::kRows * kQuads; e += 64 * kWaves) {
      const int rr = e / kQuads, k4 = e - rr * kQuads;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) x += *(const f32x4*)(lds_o + (w * S::kRows + rr) * S::kRowStride + 4 * k4);
      const int r = row0 + rr;
      const int share = (4 * k4) / S::kPass, d = share * S::kDims + pass * S::kPass + (4 * k4 - share * S::kPass);
      if (slot >= 0) {
        *(f32x4*)(a.part_out + ((int64_t)slot * S::kRows + rr) * D + d) = x;
      } else if (r < rows) {
        const int i = r / a.group, h = hk * a.group + r - i * a.group;
        *(u32x2*)(a.out + (((int64_t)b * a.q_chunk + i) * Hq + h) * D + d) =
            (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      }
    }
  }
}

__device__ __forceinline__ int history(const GqaAttendLaunch& a, int b) {
  const int seq = a.seq_lens[b], most = a.bt_stride * kPage;
  return seq < 0 ? 0 : (seq > most ? most : seq);
}
__device__ __forceinline__ int pages_of(int seq) { return (seq + kPage - 1) / kPage; }

// The workgroup's span of the line: every thread sums a few requests' places, a
// scan over the workgroup gives the line's length and with it the spans, and
// the thread whose requests hold the span's start finds the request.
struct Span {
  int lo, hi;      // places
  int chunk;       // places of a span
  int b, b_start;  // the request at lo, and its first place
};
__device__ __forceinline__ Span find_span(const GqaAttendLaunch& a, int tiles, int* lds) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int per = (a.B + 64 * kWaves - 1) / (64 * kWaves);
  int mine = 0;
  for (int k = 0; k < per; ++k) {
    const int b = t * per + k;
    if (b < a.B) mine += tiles * (pages_of(history(a, b)) + kTileCost);
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
  Span s;
  s.chunk = max((total + a.workers - 1) / a.workers, kLeastSpan);
  s.lo = min((int64_t)blockIdx.x * s.chunk, (int64_t)total);
  s.hi = min((int64_t)s.lo + s.chunk, (int64_t)total);
  if (s.lo < s.hi && s.lo >= upto - mine && s.lo < upto) {
    int start = upto - mine;
    for (int b = t * per;; ++b) {
      const int next = start + tiles * (pages_of(history(a, b)) + kTileCost);
      if (s.lo < next) {
        lds[kWaves] = b;
        lds[kWaves + 1] = start;
        break;
      }
      start = next;
    }
  }
  __syncthreads();
  s.b = __builtin_amdgcn_readfirstlane(lds[kWaves]);
  s.b_start = __builtin_amdgcn_readfirstlane(lds[kWaves + 1]);
  s.lo = __builtin_amdgcn_readfirstlane(s.lo);
  s.hi = __builtin_amdgcn_readfirstlane(s.hi);
  s.chunk = __builtin_amdgcn_readfirstlane(s.chunk);
  return s;
}

template <int D, int MT, int CODE>
__global__ __launch_bounds__(64 * kWaves, (Shape<D, MT>::kPerCu)) void gqa_attend_kernel(GqaAttendLaunch a) {
  using S = Shape<D, MT>;
  __shared__ __align__(16) float lds_o[kWaves * S::kRows * S::kRowStride];
  __shared__ float lds_m[kWaves * S::kRows];
  __shared__ float lds_l[kWaves * S::kRows];
  __shared__ int lds_span[kWaves + 2];
  const int row_blocks = (a.q_chunk * a.group + S::kRows - 1) / S::kRows;
  const int tiles = a.Hk * row_blocks;  // of a request
  const Span span = find_span(a, tiles, lds_span);
  int4 joined = {-1, 0, 0, 0};  // the tile that this workgroup has the first part of
  int b = span.b, b_start = span.b_start;
  for (int at = span.lo; at < span.hi;) {
    const int seq = __builtin_amdgcn_readfirstlane(history(a, b)), pages = pages_of(seq), cost = pages + kTileCost;
    const int tile = (at - b_start) / cost, start = b_start + tile * cost;
    const int hk = tile / row_blocks, rb = tile - hk * row_blocks;
    const int p0 = max(at - start - kTileCost, 0), p1 = min(span.hi - start - kTileCost, pages);
    // (a tile without a page belongs to the span of its first place)
    if (p0 < p1 || (pages == 0 && at == start)) {
      int slot = -1;
      if (p0 > 0) {
        slot = 2 * blockIdx.x;
      } else if (p1 < pages) {
        slot = 2 * blockIdx.x + 1;
        joined = {b, hk, rb, (start + kTileCost + pages - 1) / span.chunk - (int)blockIdx.x + 1};
      }
      attend_pages<D, MT, CODE>(a, b, hk, rb * S::kRows, seq, p0, p1, slot, lds_o, lds_m, lds_l);
      __syncthreads();
    }
    at = start + cost;
    if (tile == tiles - 1) {
      ++b;
      b_start = at;
    }
  }
  if (threadIdx.x == 0) a.joined[blockIdx.x] = joined;
}

// Joins the parts of the tile whose first part workgroup blockIdx.x of the
// attend kernel has, if any: one wave per row.  The parts lie in slots 2w + 1,
// 2(w + 1), 2(w + 2), ...; lanes take 4 dims each, 64 / (D / 4) parts at a time.
template <int D, int MT>
__global__ __launch_bounds__(64 * kWaves) void gqa_join_kernel(GqaAttendLaunch a) {
  using S = Shape<D, MT>;
  const int w = blockIdx.x, lane = threadIdx.x & 63;
  const int4 tile = a.joined[w];
  if (tile.x < 0) return;
  const int rr = blockIdx.y * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = tile.z * S::kRows + rr;
  if (r >= a.q_chunk * a.group) return;
  const int parts = tile.w;
  const auto slot = [&](int p) { return (int64_t)(p == 0 ? 2 * w + 1 : 2 * (w + p)); };
  const f32x2* ml = (const f32x2*)a.part_ml;
  float top = kNegInf;
  for (int p = lane; p < parts; p += 64) top = fmaxf(top, ml[slot(p) * S::kRows + rr][0]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  constexpr int kLanes = D / 4, kSide = 64 / kLanes;  // lanes of a row; parts side by side
  const int d = 4 * (lane % kLanes);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
#pragma unroll 4
  for (int p = lane / kLanes; p < parts; p += kSide) {
    const int64_t at = slot(p) * S::kRows + rr;
    const f32x2 v = ml[at];
    const f32x4 x = *(const f32x4*)(a.part_out + at * D + d);
    if (v[0] != kNegInf) {
      const float by = __builtin_amdgcn_exp2f(v[0] - top);
      sum += v[1] * by;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(x[i], by, o[i]);
    }
  }
#pragma unroll
  for (int x = kLanes; x < 64; x <<= 1) {
    sum += __shfl_xor(sum, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], x);
  }
  const int i = r / a.group, h = tile.y * a.group + r - i * a.group;
  const int64_t row = ((int64_t)tile.x * a.q_chunk + i) * (a.Hk * a.group) + h;
  if (lane < kLanes) {
    const float inv = inverse(sum);
    *(u32x2*)(a.out + row * D + d) = (u32x2){pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    if (lane == 0 && a.lse) a.lse[row] = row_lse(top, sum);
  }
}

template <int D, int MT, int CODE>
hipError_t launch_shape(GqaAttendLaunch a, hipStream_t s) {
  using S = Shape<D, MT>;
  const int64_t row_blocks = ((int64_t)a.q_chunk * a.group + S::kRows - 1) / S::kRows;
  a.workers = a.workers * S::kPerCu < kGqaMaxWorkers ? a.workers * S::kPerCu : kGqaMaxWorkers;
  // no more workgroups than the longest histories would fill
  const int64_t most = ((int64_t)a.B * a.Hk * row_blocks * (a.bt_stride + kTileCost) + kLeastSpan - 1) / kLeastSpan;
  if (a.workers > most) a.workers = (int32_t)most;
  hipLaunchKernelGGL((gqa_attend_kernel<D, MT, CODE>), dim3(a.workers), dim3(64 * kWaves), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gqa_join_kernel<D, MT>), dim3(a.workers, S::kRows / kWaves), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

// Rows of a tile, by the rows that share a KV head: the fewest that hold them,
// at most 64 (32 at 256 dims, whose accumulators would not fit).
template <int CODE>
hipError_t launch_code(const GqaAttendLaunch& a, hipStream_t s) {
  const int mt = gqa_row_tiles(a.D, (int64_t)a.q_chunk * a.group);
  if (a.D == 64) return mt == 1 ? launch_shape<64, 1, CODE>(a, s) : mt == 2 ? launch_shape<64, 2, CODE>(a, s) : launch_shape<64, 4, CODE>(a, s);
  if (a.D == 128) return mt == 1 ? launch_shape<128, 1, CODE>(a, s) : mt == 2 ? launch_shape<128, 2, CODE>(a, s) : launch_shape<128, 4, CODE>(a, s);
  return mt == 1 ? launch_shape<256, 1, CODE>(a, s) : launch_shape<256, 2, CODE>(a, s);
}

}  // namespace gqa
}  // namespace splash
