// gfx950 kernels of splash_gqa_append: new K and V rows into their blocks of
// 8-bit codes, with one power-of-two scale per block.
//
// The rows of one page stand next to each other in the list: a run.  One wave,
// or a part of one, writes a whole run for one KV head and one of K and V: no
// two touch a block, and nothing is exchanged between waves.  It finds the run's
// largest finite magnitude, from it the exponent (on bf16's bits, so without a
// rounding), and where the block's scale grows it brings the rows that were
// there to the new one.  A power of two moves an E4M3 code's exponent alone;
// only codes that reach its subnormals, and INT8 codes, are rounded again.
//
// Runs of up to kShort rows (decode steps) take the D / 8 lanes that hold a row
// in 16-byte pieces, so that a wave writes 64 / (D / 8) of them at a time; longer
// ones (prompts) take the wave, with all of their rows in registers.  A wave of
// gqa_append_rows_kernel looks at one token, for several heads; one of
// gqa_append_prompts_kernel at kWindow tokens, for one, so that prompts do not
// pay for a wave per token that finds no run to write.
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

constexpr int32_t kShort = 8;
constexpr int32_t kWindow = 32;

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

// One of K and V of one head.
struct Side {
  const uint16_t* x;  // row 0 of the new rows
  uint8_t* codes;     // page 0
  float* scales;      // page 0
};
__device__ __forceinline__ Side side_of(const GqaAppendLaunch& a, int32_t side, int32_t D) {
  const bool is_v = side >= a.Hk;
  const int32_t h = is_v ? side - a.Hk : side;
  return {(is_v ? a.v_new : a.k_new) + h * a.head_stride, (is_v ? a.v_pages : a.k_pages) + (int64_t)h * (kPage * D),
          (is_v ? a.v_scales : a.k_scales) + h};
}
__device__ __forceinline__ int32_t exponent_of(uint32_t scale) { return min(max((int32_t)((scale >> 23) & 255u) - 127, -126), 127); }

// Largest finite magnitude of eight values (bf16 bits); `odd`: one that is not finite.
__device__ __forceinline__ void look(u32x4 w, uint32_t& top, bool& odd) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu, more = max(lo, hi), less = min(lo, hi);
    odd |= more >= 0x7f80u;
    top = max(top, more < 0x7f80u ? more : less < 0x7f80u ? less : 0u);
  }
}
template <int CODE, bool FINITE>
__device__ __forceinline__ u32x2 encode(u32x4 w, float by) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __builtin_bit_cast(float, w[i] << 16) * by;
    f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u) * by;
  }
  return (u32x2){to_codes<CODE, FINITE>(f[0], f[1], f[2], f[3]), to_codes<CODE, FINITE>(f[4], f[5], f[6], f[7])};
}
// Rows before place `last` that are not fresh, times 2^-d: `lanes` lanes, of which this is `lane`.
template <int D, int CODE>
__device__ __forceinline__ void rescale_rows(uint8_t* codes, uint64_t fresh, int32_t last, int32_t d, int lane, int lanes) {
  for (int32_t j = lane; j < last * (D / 16); j += lanes) {
    if (fresh >> (j / (D / 16)) & 1ull) continue;
    u32x4* q = (u32x4*)codes + j;
    u32x4 v = *q;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = rescale_codes<CODE>(v[i], d);
    *q = v;
  }
}

// A run of 1 to kShort rows n, n + 1, ... on the D / 8 lanes of this lane's
// group (run 0: none).  Groups work side by side on runs of their own.
template <int D, int CODE>
__device__ __forceinline__ void write_short(const GqaAppendLaunch& a, const Side& to, int64_t n, int32_t run, int32_t slot) {
  constexpr int kPieces = D / 8;
  const int piece = (threadIdx.x & 63) % kPieces;
  if (run == 0) return;
  const int64_t block = (int64_t)(slot >> 6) * a.Hk;
  uint8_t* codes = to.codes + block * (kPage * D);
  float* scale = to.scales + block;
  const uint32_t old_scale = *(const uint32_t*)scale;
  u32x4 w[kShort];
  int32_t place[kShort];
  uint64_t fresh = 0;
  uint32_t top = 0;
  bool odd = false;
#pragma unroll
  for (int r = 0; r < kShort; ++r)
    if (r < run) {
      w[r] = *(const u32x4*)(to.x + (n + r) * a.token_stride + 8 * piece);
      place[r] = (r == 0 ? slot : a.slots[n + r]) & 63;
    }
#pragma unroll
  for (int r = 0; r < kShort; ++r)
    if (r < run) {
      fresh |= 1ull << place[r];
      look(w[r], top, odd);
    }
#pragma unroll
  for (int d = 1; d < kPieces; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  int32_t e = exponent_for<CODE>(top);
  if (!(fresh & 1ull)) {  // no new row in place 0: the block has rows to keep
    const int32_t e_old = exponent_of(old_scale);
    if (e > e_old) rescale_rows<D, CODE>(codes, fresh, 63 - __builtin_clzll(fresh), e - e_old, piece, kPieces);
    else e = e_old;
  }
  const float by = __builtin_amdgcn_ldexpf(1.f, -e);
#pragma unroll
  for (int r = 0; r < kShort; ++r)
    if (r < run)
      *(u32x2*)(codes + place[r] * D + 8 * piece) = odd ? encode<CODE, false>(w[r], by) : encode<CODE, true>(w[r], by);
  if (piece == 0) *scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}

// A run of any length (at most 64) on the wave.  HELD: its rows stay in
// registers; else they are read twice.  in_order: its places follow each other.
template <int D, int CODE, bool HELD>
__device__ __forceinline__ void write_long(const GqaAppendLaunch& a, const Side& to, int64_t n, int32_t run, int32_t slot,
                                           bool in_order) {
  constexpr int kPieces = D / 8, kRowsAtOnce = 64 / kPieces, kTurns = kPage / kRowsAtOnce;
  const int lane = threadIdx.x & 63, piece = lane % kPieces, row = lane / kPieces;
  const int32_t place0 = slot & 63;
  uint64_t fresh = (run == 64 ? ~0ull : (1ull << run) - 1) << place0;  // the places that get rows
  if (!in_order) {
    fresh = lane < run ? 1ull << (a.slots[n + lane] & 63) : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) fresh |= __shfl_xor(fresh, d);
  }
  const int64_t block = (int64_t)(slot >> 6) * a.Hk;
  uint8_t* codes = to.codes + block * (kPage * D);
  float* scale = to.scales + block;
  const uint32_t old_scale = *(const uint32_t*)scale;
  const auto load = [&](int t) { return *(const u32x4*)(to.x + (n + min(t * kRowsAtOnce + row, run - 1)) * a.token_stride + 8 * piece); };
  u32x4 w[HELD ? kTurns : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (t * kRowsAtOnce < run) w[t] = load(t);
  }
  uint32_t top = 0;
  bool odd = false;
  const auto look_at = [&](int t) {
    if constexpr (!HELD) w[0] = load(t);
    look(w[HELD ? t : 0], top, odd);  // (past the run's end its last row again)
  };
  if constexpr (HELD) {
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (t * kRowsAtOnce < run) look_at(t);
  } else {
    for (int t = 0; t * kRowsAtOnce < run; ++t) look_at(t);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  int32_t e = exponent_for<CODE>(top);
  if (!(fresh & 1ull)) {
    const int32_t e_old = exponent_of(old_scale);
    if (e > e_old) rescale_rows<D, CODE>(codes, fresh, 63 - __builtin_clzll(fresh), e - e_old, lane, 64);
    else e = e_old;
  }
  const float by = __builtin_amdgcn_ldexpf(1.f, -e);
  const auto write = [&](int t, auto finite) {
    const int32_t r = t * kRowsAtOnce + row;
    if constexpr (!HELD) w[0] = load(t);
    if (r < run) *(u32x2*)(codes + (in_order ? place0 + r : a.slots[n + r] & 63) * D + 8 * piece) = encode<CODE, finite>(w[HELD ? t : 0], by);
  };
  const auto write_all = [&](auto finite) {
    if constexpr (HELD) {
#pragma unroll
      for (int t = 0; t < kTurns; ++t)
        if (t * kRowsAtOnce < run) write(t, finite);
    } else {
      for (int t = 0; t * kRowsAtOnce < run; ++t) write(t, finite);
    }
  };
  if (__any(odd)) write_all(std::false_type{});
  else write_all(std::true_type{});
  if (lane == 0) *scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}

__device__ __forceinline__ int32_t slot_at(const GqaAppendLaunch& a, int64_t n) { return n >= 0 && n < a.num_tokens ? a.slots[n] : -1; }
__device__ __forceinline__ bool in_pool(const GqaAppendLaunch& a, int32_t slot) { return slot >= 0 && (slot >> 6) < a.num_pages; }

// Token n's run, if one begins there, for the sides of one lane group each.
template <int D, int CODE>
__global__ __launch_bounds__(kThreads) void gqa_append_rows_kernel(GqaAppendLaunch a) {
  constexpr int kPieces = D / 8, kGroups = 64 / kPieces;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t sides = 2 * a.Hk, side_tasks = (sides + kGroups - 1) / kGroups;
  const int64_t n = task / side_tasks;
  const int32_t side0 = (int32_t)(task % side_tasks) * kGroups;
  if (n >= a.num_tokens) return;
  const int32_t before = slot_at(a, n - 1), s = slot_at(a, n + lane), prev = __shfl_up(s, 1);
  const int32_t slot = __builtin_amdgcn_readfirstlane(s), page = slot >> 6;
  if (!in_pool(a, slot) || before >> 6 == page) return;
  const uint64_t out = ~__ballot(s >= 0 && s >> 6 == page);  // tokens of other pages
  const int32_t run = out ? __builtin_ctzll(out) : 64;
  if (run <= kShort) {
    const int32_t side = side0 + lane / kPieces;
    write_short<D, CODE>(a, side_of(a, min(side, sides - 1), D), n, side < sides ? run : 0, slot);
  } else {
    const uint64_t in_run = run == 64 ? ~0ull : (1ull << run) - 1;
    const bool in_order = !(__ballot(lane > 0 && s != prev + 1) & in_run);
    for (int32_t side = side0; side < min(side0 + kGroups, sides); ++side)
      write_long<D, CODE, false>(a, side_of(a, side, D), n, run, slot, in_order);
  }
}

// The runs that begin among kWindow tokens, for one side: long ones one after
// the other, short ones one per lane group.  (Four waves a SIMD: with the
// registers of five it goes to memory for them, 38 us against 28 for 18,093 rows
// of 8 heads by 128 dims, floor 23.  At 256 dims the rows in registers leave two: as
// many bytes, 4 heads by 256, take a quarter longer.)
template <int D, int CODE>
__global__ __launch_bounds__(kThreads, (D == 256 ? 1 : 4)) void gqa_append_prompts_kernel(GqaAppendLaunch a) {
  constexpr int kPieces = D / 8, kGroups = 64 / kPieces;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t sides = 2 * a.Hk;
  const int64_t n0 = task / sides * kWindow;
  if (n0 >= a.num_tokens) return;
  const Side to = side_of(a, (int32_t)(task % sides), D);

  // Where runs begin, and where a slot is not the next place: tokens n0 + lane
  // and, for runs past the window's end, n0 + 64 + lane.
  const int32_t before = slot_at(a, n0 - 1), s0 = slot_at(a, n0 + lane), s1 = slot_at(a, n0 + 64 + lane);
  const int32_t last0 = __shfl(s0, 63);
  int32_t p0 = __shfl_up(s0, 1), p1 = __shfl_up(s1, 1);
  if (lane == 0) {
    p0 = before;
    p1 = last0;
  }
  const uint64_t starts0 = __ballot(!in_pool(a, s0) || p0 >> 6 != s0 >> 6), starts1 = __ballot(!in_pool(a, s1) || p1 >> 6 != s1 >> 6);
  const uint64_t breaks0 = __ballot(s0 != p0 + 1), breaks1 = __ballot(s1 != p1 + 1);
  const uint64_t leaders = starts0 & __ballot(in_pool(a, s0)) & ((1ull << kWindow) - 1);
  const auto run_at = [&](int at) {  // tokens from n0 + at to the next start
    const uint64_t next = at == 63 ? starts1 : (starts0 >> (at + 1) | starts1 << (63 - at));
    return next ? __builtin_ctzll(next) + 1 : 64;
  };

  uint64_t rest = 0;  // short runs
  for (uint64_t l = leaders; l; l &= l - 1) {
    const int at = __builtin_ctzll(l), run = min(run_at(at), 64);
    if (run <= kShort) {
      rest |= 1ull << at;
      continue;
    }
    const uint64_t breaks = at ? breaks0 >> at | breaks1 << (64 - at) : breaks0;
    const uint64_t in_run = run == 64 ? ~0ull : (1ull << run) - 1;
    write_long<D, CODE, true>(a, to, n0 + at, run, __builtin_amdgcn_readlane(s0, at), !(breaks & in_run & ~1ull));
  }
  while (rest) {
    int32_t mine = -1;  // this lane group's run
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
      if (rest) {
        if (lane / kPieces == k) mine = __builtin_ctzll(rest);
        rest &= rest - 1;
      }
    const int at = mine < 0 ? 0 : mine;
    const int32_t slot = __shfl(s0, at);
    write_short<D, CODE>(a, to, n0 + at, mine < 0 ? 0 : run_at(at), slot);
  }
}

template <int D, int CODE>
hipError_t launch_code(const GqaAppendLaunch& a, hipStream_t s) {
  constexpr int kGroups = 512 / D;
  // Tokens a request: 2,048 requests with one each take 6.7 us by rows (25 with
  // the wave's lanes on one head), a prompt of 2,000 takes 10 us by windows (22
  // by rows).  The host knows only the list's length, skipped slots among it: 256
  // one-token requests padded to fewer than 2,048 slots take 4.2 us, to 2,048 and
  // more 13.7 (22.5 at 256 dims), by windows.
  const bool prompts = a.num_tokens >= 8 * (int64_t)a.batch;
  const int64_t waves = prompts ? ((int64_t)a.num_tokens + kWindow - 1) / kWindow * 2 * a.Hk
                                : (int64_t)a.num_tokens * ((2 * a.Hk + kGroups - 1) / kGroups);
  const int64_t groups = (waves + kThreads / 64 - 1) / (kThreads / 64);
  if (prompts) hipLaunchKernelGGL((gqa_append_prompts_kernel<D, CODE>), dim3((unsigned)groups), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((gqa_append_rows_kernel<D, CODE>), dim3((unsigned)groups), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
template <int D>
hipError_t launch_dim(const GqaAppendLaunch& a, hipStream_t s) {
  return a.code_type == 0 ? launch_code<D, 0>(a, s) : launch_code<D, 1>(a, s);
}

}  // namespace

hipError_t launch_gqa_append(const GqaAppendLaunch& a, hipStream_t s) {
  return a.D == 64 ? launch_dim<64>(a, s) : a.D == 128 ? launch_dim<128>(a, s) : launch_dim<256>(a, s);
}

}  // namespace splash
