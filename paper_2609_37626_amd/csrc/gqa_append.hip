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

// Tokens of a wave.
int32_t append_window(int32_t num_tokens) { return num_tokens <= 2048 ? 1 : 32; }

// The least e >= -126 with the magnitude (15 bits of a finite bf16) <= TOP * 2^e:
// TOP is 1.75 * 2^8 (E4M3) or 127/64 * 2^6 (INT8).
template <int CODE>
__device__ __forceinline__ int32_t exponent_for(uint32_t mag) {
  const int32_t E = (int32_t)(mag >> 7) - 127;
  const uint32_t frac = mag & 127u;
  const int32_t e = CODE == 0 ? E - 8 + (frac > 96u) : E - 6 + (frac > 126u);
  return max(e, -126);
}

// Four values, already divided by the scale, to codes: any values, or (FINITE)
// none past the largest code.  INT8: adding 1.5 * 2^23 leaves the nearest whole
// number (ties to even) in the low bits.
template <int CODE, bool FINITE>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  float x[4] = {a, b, c, d};
  constexpr float kTop = CODE == 0 ? 448.f : 127.f;
  if constexpr (!FINITE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = x[i] != x[i] ? (CODE == 0 ? x[i] : 0.f) : fminf(fmaxf(x[i], -kTop), kTop);
  }
  if constexpr (CODE == 0) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
  } else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_bit_cast(uint32_t, x[i] + 12582912.f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u), __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), 0x05040100u);
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
  return to_codes<CODE, false>(x[0], x[1], x[2], x[3]);
}

// A wave takes `window` tokens of the list (1 to 64), one KV head and one of K
// and V, and writes the runs that begin among them.
template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void gqa_append_kernel(GqaAppendLaunch a, int32_t window) {
  constexpr int kPieces = D / 8;         // 16-byte pieces of a row
  constexpr int kRowsAtOnce = 64 / kPieces;
  constexpr int kTurns = kPage / kRowsAtOnce;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t sides = 2 * a.Hk;
  const int64_t n0 = task / sides * window;
  const int32_t side = (int32_t)(task % sides), h = side >> 1;
  const bool is_v = side & 1;
  if (n0 >= a.num_tokens) return;
  const uint16_t* x = (is_v ? a.v_new : a.k_new) + h * a.head_stride + 8 * (lane % kPieces);
  const auto load_rows = [&](int64_t n, int turn) {
    const int64_t row = n + turn * kRowsAtOnce + lane / kPieces;
    return *(const u32x4*)(x + (row < a.num_tokens ? row : n) * a.token_stride);
  };
  u32x4 w[kTurns];
  if (window == 1) w[0] = load_rows(n0, 0);  // (its address needs no slot)

  // Where runs start: a slot in another page than the one before, or none.
  // Tokens n0 + lane and, for runs past the window's end, n0 + 64 + lane.
  const auto slot_at = [&](int64_t n) { return n >= 0 && n < a.num_tokens ? a.slots[n] : -1; };
  const auto valid = [&](int32_t slot) { return slot >= 0 && (slot >> 6) < a.num_pages; };
  const int32_t s0 = slot_at(n0 + lane), s1 = window > 1 ? slot_at(n0 + 64 + lane) : -1;
  const int32_t before = slot_at(n0 - 1), last0 = __shfl(s0, 63);
  int32_t p0 = __shfl_up(s0, 1), p1 = __shfl_up(s1, 1);
  if (lane == 0) {
    p0 = before;
    p1 = last0;
  }
  const uint64_t starts0 = __ballot(!valid(s0) || p0 >> 6 != s0 >> 6), starts1 = __ballot(!valid(s1) || p1 >> 6 != s1 >> 6);
  const uint64_t breaks0 = __ballot(s0 != p0 + 1), breaks1 = __ballot(s1 != p1 + 1);  // not the next place
  uint64_t leaders = starts0 & __ballot(valid(s0)) & (window == 64 ? ~0ull : (1ull << window) - 1);

  while (leaders) {
    const int32_t at = __builtin_ctzll(leaders);
    leaders &= leaders - 1;
    const int64_t n = n0 + at;
    // bit r of the two: token n + r starts a run, or is not in the next place
    const uint64_t starts = at ? starts0 >> at | starts1 << (64 - at) : starts0;
    const uint64_t breaks = at ? breaks0 >> at | breaks1 << (64 - at) : breaks0;
    const int32_t run = starts >> 1 ? __builtin_ctzll(starts >> 1) + 1 : 64;
    const uint64_t in_run = run == 64 ? ~0ull : (1ull << run) - 1;
    const int32_t slot = __builtin_amdgcn_readlane(s0, at), page = slot >> 6, place0 = slot & 63;
    const bool in_order = !(breaks & in_run & ~1ull);
    uint64_t fresh = in_run << place0;  // the places that get rows
    if (!in_order) {
      fresh = lane < run ? 1ull << (a.slots[n + lane] & 63) : 0;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) fresh |= __shfl_xor(fresh, d);
    }
    const int64_t block = (int64_t)page * a.Hk + h;
    uint8_t* codes = (is_v ? a.v_pages : a.k_pages) + block * (kPage * D);
    float* scale = (is_v ? a.v_scales : a.k_scales) + block;
    const uint32_t old_scale = *(const uint32_t*)scale;

#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (t * kRowsAtOnce < run && (t > 0 || window > 1)) w[t] = load_rows(n, t);
    uint32_t top = 0;  // largest finite magnitude, as bf16 bits
    bool odd = false;  // an infinity or NaN among the rows
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (t * kRowsAtOnce < run && t * kRowsAtOnce + lane / kPieces < run)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t lo = w[t][i] & 0x7fffu, hi = (w[t][i] >> 16) & 0x7fffu;
          const uint32_t more = max(lo, hi);
          if (more < 0x7f80u) {
            top = max(top, more);
          } else {
            odd = true;
            if (min(lo, hi) < 0x7f80u) top = max(top, min(lo, hi));
          }
        }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));

    int32_t e = exponent_for<CODE>(top);
    if (!(fresh & 1ull)) {  // no new row in place 0: the block has rows to keep
      const int32_t e_old = min(max((int32_t)((old_scale >> 23) & 255u) - 127, -126), 127);
      if (e > e_old) {
        const int32_t last = 63 - __builtin_clzll(fresh);
        for (int32_t j = lane; j < last * (D / 4); j += 64) {
          if (fresh >> (j / (D / 4)) & 1ull) continue;
          uint32_t* q = (uint32_t*)codes + j;
          *q = rescale_codes<CODE>(*q, e - e_old);
        }
      } else {
        e = e_old;
      }
    }
    const float by = __builtin_amdgcn_ldexpf(1.f, -e);
    const auto write = [&](auto finite) {
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int32_t r = t * kRowsAtOnce + lane / kPieces;
        if (t * kRowsAtOnce < run && r < run) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, w[t][i] << 16) * by;
            f[2 * i + 1] = __builtin_bit_cast(float, w[t][i] & 0xffff0000u) * by;
          }
          const int32_t to = in_order ? place0 + r : a.slots[n + r] & 63;
          *(u32x2*)(codes + to * D + 8 * (lane % kPieces)) =
              (u32x2){to_codes<CODE, finite>(f[0], f[1], f[2], f[3]), to_codes<CODE, finite>(f[4], f[5], f[6], f[7])};
        }
      }
    };
    if (__any(odd)) write(std::false_type{});
    else write(std::true_type{});
    if (lane == 0) *scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
  }
}

template <int D>
hipError_t launch_dim(const GqaAppendLaunch& a, hipStream_t s) {
  const int32_t window = append_window(a.num_tokens);
  const int64_t waves = ((int64_t)a.num_tokens + window - 1) / window * 2 * a.Hk;
  const int64_t groups = (waves + kThreads / 64 - 1) / (kThreads / 64);
  if (groups > 0x7fffffff) return hipErrorInvalidConfiguration;
  if (a.code_type == 0) hipLaunchKernelGGL((gqa_append_kernel<D, 0>), dim3((unsigned)groups), dim3(kThreads), 0, s, a, window);
  else hipLaunchKernelGGL((gqa_append_kernel<D, 1>), dim3((unsigned)groups), dim3(kThreads), 0, s, a, window);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gqa_append(const GqaAppendLaunch& a, hipStream_t s) {
  return a.D == 64 ? launch_dim<64>(a, s) : a.D == 128 ? launch_dim<128>(a, s) : launch_dim<256>(a, s);
}

}  // namespace splash
