// gfx950 kernel of splash_mla_prefill: causal attention of ragged prompts over
// expanded keys (128 of a head's own dims, 64 shared rotary ones) and values.
//
// A workgroup takes 128 query rows of a request and head, 32 a wave, and walks over
// the keys 64 at a time; a step's keys and values come straight into LDS, the next
// step's while this one is multiplied.
//   QK  S^T[key, row] = K Q^T, v_mfma_f32_16x16x32_bf16.  Lane (g, c) holds keys
//       16 t + 4 g + i of row c: the weights of a row stay in its four lanes.
//   PV  O^T[value, row] = V^T P^T.  The product's slot (g, j) is key 4 g + j of tile
//       2 u (j < 4) or 4 g + j - 4 of tile 2 u + 1: P goes from QK's result to PV's
//       operand in the lane that has it, and V's transposing reads take the rows
//       in that order.
// The softmax runs over the steps once with a reference that moves only where a
// score passes it by 2^8: below that the weights' sums cannot overflow, and rows that
// do not move it need no exchange between lanes.
//
// LDS: two steps' keys, then two steps' values, in line groups of 128 bytes,
// [group][key][128], chunks of 16 bytes at chunk ^ swz(key); a step's keys are groups
// 0 and 1 for the head's own dims and 2 for the rotary ones, its values two more.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;              // query rows of a tile
constexpr int kWaveRows = 32;
constexpr int kKeys = 64;               // keys of a step
constexpr int kHalf = 32;
constexpr int kAhead = 4;
constexpr int kGroupBytes = kKeys * 128;
constexpr int kKeyBytes = 3 * kGroupBytes;    // a step's keys in LDS
constexpr int kValueBytes = 2 * kGroupBytes;  // and its values
constexpr float kSlack = 8.f;           // powers of two by which a score may pass the reference
constexpr float kLowest = -1e30f;       // the reference before any score
constexpr int32_t kTileCost = 1;        // a tile's fixed work, in steps
constexpr int32_t kNeverCut = 12;       // steps of the longest tile that is never cut
constexpr int32_t kLeast = 4;           // steps a worker of the line
constexpr int kSorted = 4;              // requests a lane that the order of the blocks looks at

__device__ __forceinline__ uint32_t swz(uint32_t r) {
  return ((r & 2u)) | ((((r >> 2) ^ (r >> 3)) & 1u) << 2) | ((r >> 3) & 1u);
}

// s_waitcnt with only vmcnt constrained.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
// Workgroup barrier that leaves loads to LDS in flight.
__device__ __forceinline__ void lds_barrier() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt((0x3F & 15) | (7 << 4) | (0 << 8) | ((0x3F >> 4) << 14));  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}
// 16 bytes a lane from base + offset + ADD straight to LDS at `lds` + 16 * lane.  Through
// asm, so that the compiler does not wait for it at every LDS read; the kernel does.  (The
// instruction's own offset moves the LDS address as well: M0 is set that much lower.)
template <int ADD>
__device__ __forceinline__ void load_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_sub_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" ::"s"(lds), "v"(offset), "s"(base), "n"(ADD) : "memory", "scc");
}

// A tile: 128 rows of a request, of the head `h`.
struct Tile {
  int32_t h;
  int32_t rows;        // of the request past the tile's first
  int64_t q0;          // the tile's first query row
  int64_t k0;          // the request's first key
  int32_t first_sees;  // keys that the tile's first row sees (may be negative)
  int32_t keys;        // keys that any row of the tile sees
};

struct Request {
  int32_t q0, nq, k0, nk;
};
__device__ __forceinline__ Request request(const MlaPrefillLaunch& a, int32_t b) {
  Request r;
  r.q0 = min(max(a.q_indptr[b], 0), a.num_rows);
  r.nq = min(max(a.q_indptr[b + 1], r.q0), a.num_rows) - r.q0;
  r.k0 = min(max(a.kv_indptr[b], 0), a.num_keys);
  r.nk = min(max(a.kv_indptr[b + 1], r.k0), a.num_keys) - r.k0;
  return r;
}
__device__ __forceinline__ Tile tile_of(const Request& r, int32_t h, int32_t i) {
  Tile t;
  t.h = h;
  t.q0 = r.q0 + (int64_t)i * kRows;
  t.rows = r.nq - i * kRows;
  t.k0 = r.k0;
  t.first_sees = r.nk - r.nq + i * kRows + 1;
  t.keys = max(0, t.first_sees - 1 + min(t.rows, kRows));
  return t;
}

__device__ __forceinline__ int32_t tiles_of(int32_t nq) { return (nq + kRows - 1) / kRows; }
// Steps that a request's tile i is counted as on the line: its own, at most as many
// as this, and one for its fixed work; 2 i + first(r).  The line's length up to tile i
// is i first + i (i - 1).
__device__ __forceinline__ int32_t line_first(const Request& r) { return max(0, (r.nk - r.nq + kKeys - 1) / kKeys) + 2 + kTileCost; }
__device__ __forceinline__ int64_t line_upto(int64_t i, int32_t first) { return i * (first + i - 1); }

__device__ __forceinline__ int32_t wave_prefix(int32_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t other = __shfl_up(v, d);
    v += lane >= d ? other : 0;
  }
  return v;
}
__device__ __forceinline__ int32_t uniform(int32_t v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int64_t uniform(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)(v >> 32), lane) << 32 | (uint32_t)uniform((int32_t)v, lane));
}
__device__ __forceinline__ Request uniform(const Request& r, int lane) {
  return {uniform(r.q0, lane), uniform(r.nq, lane), uniform(r.k0, lane), uniform(r.nk, lane)};
}

// What every workgroup finds out by itself about the whole call.
struct Call {
  int64_t line;     // a head's steps
  int32_t longest;  // the longest tile's
};
__device__ __forceinline__ Call look_at(const MlaPrefillLaunch& a) {
  const int lane = threadIdx.x & 63;
  int64_t line = 0;
  int32_t longest = 0;
  for (int32_t b = lane; b < a.B; b += 64) {
    const Request r = request(a, b);
    const int32_t n = tiles_of(r.nq);
    line += line_upto(n, line_first(r));
    longest = max(longest, n > 0 ? (r.nk + kKeys - 1) / kKeys : 0);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    line += __shfl_xor(line, d);
    longest = max(longest, __shfl_xor(longest, d));
  }
  return {uniform(line, 0), uniform(longest, 0)};
}

// Block `rank` of the requests' blocks of 2^shift tiles, counted from a request's last
// tile, the longest first: which of its request's and of which request (false: none).
// Block j counts as K - 2^(shift+1) j steps, K its request's last tile's: how many
// blocks are longer than a length is a sum over the requests, and the rank's length
// is found by halving.  Past 64 kSorted requests the blocks go in the requests' order.
__device__ __forceinline__ bool find_block(const MlaPrefillLaunch& a, int32_t rank, int shift, Request& r, int32_t& block) {
  const int lane = threadIdx.x & 63;
  if (a.B <= 64 * kSorted) {
    Request mine[kSorted];
    int32_t blocks[kSorted], top[kSorted], most = INT_MIN, least = INT_MAX;
#pragma unroll
    for (int k = 0; k < kSorted; ++k) {
      blocks[k] = top[k] = 0;
      mine[k] = Request{0, 0, 0, 0};
      if (64 * k < a.B) {
        const int32_t b = 64 * k + lane;
        mine[k] = request(a, min(b, a.B - 1));
        blocks[k] = b < a.B ? (tiles_of(mine[k].nq) + (1 << shift) - 1) >> shift : 0;
        top[k] = (mine[k].nk + kKeys - 1) / kKeys;
        if (blocks[k] > 0) {
          most = max(most, top[k]);
          least = min(least, top[k] - (blocks[k] - 1) * (2 << shift));
        }
      }
    }
    const auto longer = [&](int32_t than) {  // blocks of more steps
      int32_t n = 0;
#pragma unroll
      for (int k = 0; k < kSorted; ++k)
        if (64 * k < a.B) n += min(blocks[k], max(0, top[k] - than + (2 << shift) - 1) >> (shift + 1));
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
      return __builtin_amdgcn_readfirstlane(n);
    };
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      most = max(most, __shfl_xor(most, d));
      least = min(least, __shfl_xor(least, d));
    }
    // the least length that at most `rank` blocks pass: above it there are no more, and the
    // rank's block is one of this length
    int32_t lo = uniform(least, 0), hi = uniform(most, 0);
    if (lo > hi || rank >= longer(lo - 1)) return false;
    while (lo < hi) {
      const int32_t mid = lo + ((hi - lo) >> 1);
      if (longer(mid) <= rank) hi = mid;
      else lo = mid + 1;
    }
    rank -= longer(lo);
#pragma unroll
    for (int k = 0; k < kSorted; ++k) {
      if (64 * k >= a.B) break;
      const int32_t down = top[k] - lo, j = down >> (shift + 1);
      const uint64_t here = __ballot(down >= 0 && (down & ((2 << shift) - 1)) == 0 && j < blocks[k]);
      const int32_t count = __builtin_popcountll(here);
      if (rank < count) {
        uint64_t rest = here;
        for (; rank > 0; --rank) rest &= rest - 1;
        const int who = __builtin_ctzll(rest);
        r = uniform(mine[k], who);
        block = uniform(j, who);
        return true;
      }
      rank -= count;
    }
    return false;
  }
  for (int32_t b0 = 0; b0 < a.B; b0 += 64) {
    const Request mine = request(a, min(b0 + lane, a.B - 1));
    const int32_t blocks = b0 + lane < a.B ? (tiles_of(mine.nq) + (1 << shift) - 1) >> shift : 0, upto = wave_prefix(blocks);
    const uint64_t past = __ballot(upto > rank);
    if (!past) {
      rank -= uniform(upto, 63);
      continue;
    }
    const int who = __builtin_ctzll(past);
    r = uniform(mine, who);
    block = rank - uniform(upto - blocks, who);
    return true;
  }
  return false;
}

// The tile that holds place `at` of a head's line, and where it begins.
__device__ __forceinline__ bool find_place(const MlaPrefillLaunch& a, int32_t h, int64_t at, Tile& t, int64_t& begin, int32_t& count) {
  const int lane = threadIdx.x & 63;
  int64_t behind = 0;
  for (int32_t b0 = 0; b0 < a.B; b0 += 64) {
    const Request mine = request(a, min(b0 + lane, a.B - 1));
    const int32_t n = b0 + lane < a.B ? tiles_of(mine.nq) : 0;
    int64_t upto = line_upto(n, line_first(mine));
    const int64_t own = upto;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t other = __shfl_up(upto, d);
      upto += lane >= d ? other : 0;
    }
    const uint64_t past = __ballot(behind + upto > at);
    if (!past) {
      behind += uniform(upto, 63);
      continue;
    }
    const int who = __builtin_ctzll(past);
    const Request r = uniform(mine, who);
    behind += uniform(upto - own, who);
    // the last i with line_upto(i) <= at - behind
    const int32_t first = line_first(r);
    const int64_t x = at - behind;
    const double half = 0.5 * (first - 1);
    int64_t i = (int64_t)(__builtin_sqrt(half * half + (double)x) - half);
    i = min(max(i, (int64_t)0), (int64_t)tiles_of(r.nq) - 1);
    while (i > 0 && line_upto(i, first) > x) --i;
    while (i + 1 < tiles_of(r.nq) && line_upto(i + 1, first) <= x) ++i;
    const int32_t ti = __builtin_amdgcn_readfirstlane((int32_t)i);
    t = tile_of(r, h, ti);
    begin = behind + line_upto(ti, first);
    count = first + 2 * ti;
    return true;
  }
  return false;
}

// Softmax and products of a tile's steps [step0, step1) in this workgroup's waves.
struct Piece {
  f32x4 o[8][2];       // O^T: values 16 d + 4 g + i of rows 16 r + c, over exp2 of the reference
  float top[2], sum[2];
};
typedef f32x4 Scores[2][2];  // S^T of 32 keys: keys 16 t + 4 g + i of rows 16 r + c

__device__ __forceinline__ void attend(const MlaPrefillLaunch& a, const Tile& tile, int32_t step0, int32_t step1, uint8_t* lds, Piece& p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int32_t row0 = kWaveRows * wave;            // the wave's first row in the tile
  const int32_t sees0 = tile.first_sees + row0;     // keys that it sees
  // halves of steps up to which the wave sees a key
  const int32_t mine = row0 >= tile.rows ? 2 * step0 : min(2 * step1, max(sees0 + kWaveRows - 1 + kHalf - 1, 0) / kHalf);

  // Q as B operands: row c of a block of 16, eight dims from 8 g.
  bf16x8 qf[2][6];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int64_t row = tile.q0 + min(row0 + 16 * r + c, tile.rows - 1);
    const uint16_t* from = a.q + row * a.q_token + tile.h * a.q_head + 8 * g;
#pragma unroll
    for (int s = 0; s < 6; ++s) qf[r][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(from + 32 * s));
  }

  // A step's loads: its keys, and the values of the last step's second half and its own
  // first, as they are multiplied.  The wave brings rows 16 wave .. + 15, eight a load, of
  // each line group; a row outside the tile's keys is its first or last one, and past them
  // altogether there is none.
  const uint8_t* k_base = (const uint8_t*)(a.k + tile.k0 * a.k_token + tile.h * a.k_head);
  const uint8_t* key_base = (const uint8_t*)(a.key + tile.k0 * a.key_token);
  const uint8_t* v_base = (const uint8_t*)(a.v + tile.k0 * a.v_token + tile.h * a.v_head);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_AS uint8_t*)lds + 2048 * wave;
  const int32_t load_row = 16 * wave + (lane >> 3);
  const uint32_t chunk0 = 16 * ((lane & 7) ^ swz(load_row)), chunk1 = 16 * ((lane & 7) ^ swz(load_row + 8));
  const uint32_t k_off = load_row * (uint32_t)a.k_token * 2 + chunk0, key_off = load_row * (uint32_t)a.key_token * 2 + chunk0;
  const uint32_t v_off = load_row * (uint32_t)a.v_token * 2 + chunk0, next8 = chunk1 - chunk0;
  const auto load_rows = [&](const uint8_t* kb, const uint8_t* rb, const uint8_t* vb, int slot) {  // all of them there
    const uint32_t to = lds0 + slot * kKeyBytes, v_to = lds0 + 2 * kKeyBytes + slot * kValueBytes;
    load_lds<0>(kb, k_off, to);
    load_lds<128>(kb, k_off, to + kGroupBytes);
    load_lds<0>(rb, key_off, to + 2 * kGroupBytes);
    load_lds<0>(vb, v_off, v_to);
    load_lds<128>(vb, v_off, v_to + kGroupBytes);
    kb += 16 * a.k_token;
    rb += 16 * a.key_token;
    vb += 16 * a.v_token;
    load_lds<0>(kb, k_off + next8, to + 1024);
    load_lds<128>(kb, k_off + next8, to + 1024 + kGroupBytes);
    load_lds<0>(rb, key_off + next8, to + 1024 + 2 * kGroupBytes);
    load_lds<0>(vb, v_off + next8, v_to + 1024);
    load_lds<128>(vb, v_off + next8, v_to + 1024 + kGroupBytes);
  };
  const auto load_step = [&](int32_t step) {
    const int32_t first = step * kKeys, last = tile.keys - 1 - first;
    const int32_t v_first = max(first - kHalf, 0), v_last = tile.keys - 1 - v_first, v_skip = first - kHalf - v_first;
    const uint8_t* kb = k_base + (int64_t)first * a.k_token * 2;
    const uint8_t* rb = key_base + (int64_t)first * a.key_token * 2;
    const uint8_t* vb = v_base + (int64_t)v_first * a.v_token * 2;
    const int slot = (step - step0) & 1;
    if (last >= kKeys - 1 && v_skip == 0) {
      load_rows(kb, rb, vb, slot);
      return;
    }
    const uint32_t to = lds0 + slot * kKeyBytes, v_to = lds0 + 2 * kKeyBytes + slot * kValueBytes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t row = load_row + 8 * i;
      const uint32_t chunk = i ? chunk1 : chunk0;
      if (last >= 0) {
        const uint32_t from = min(row, last);
        const uint32_t k_at = from * (uint32_t)a.k_token * 2 + chunk, r_at = from * (uint32_t)a.key_token * 2 + chunk;
        load_lds<0>(kb, k_at, to + 1024 * i);
        load_lds<128>(kb, k_at, to + 1024 * i + kGroupBytes);
        load_lds<0>(rb, r_at, to + 1024 * i + 2 * kGroupBytes);
      }
      if (v_last >= 0) {
        const uint32_t v_at = (uint32_t)min(max(row + v_skip, 0), v_last) * (uint32_t)a.v_token * 2 + chunk;
        load_lds<0>(vb, v_at, v_to + 1024 * i);
        load_lds<128>(vb, v_at, v_to + 1024 * i + kGroupBytes);
      }
    }
  };

  // K operand of 32 dims: chunk g (or 4 + g) of row c; V: see the top.
  const uint32_t k_lane = 128 * c + 16 * (g ^ swz(c));
  const uint32_t v_row = 4 * g + (c >> 2);
  const uint32_t v_lane = 2 * kKeyBytes + 128 * v_row + 16 * (((c >> 1) & 1) ^ swz(v_row)) + 8 * (c & 1);
  const LDS_AS uint8_t* buf = (const LDS_AS uint8_t*)lds;

  f32x4 o[8][2];
  float top[2], sum[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    top[r] = kLowest;
    sum[r] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[d][r] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  const auto value_operand = [&](int at, int d) {
    const LDS_AS uint8_t* from = buf + (v_lane ^ (32 * (d & 3))) + kGroupBytes * (d >> 2) + at;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)from);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)(from + 2048));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const auto key_operand = [&](int at, int s, int t) {
    return *(const LDS_AS bf16x8*)(buf + (k_lane ^ (64 * (s & 1))) + kGroupBytes * (s >> 1) + 2048 * t + at);
  };
  const auto score_dims = [&](const bf16x8 (&kf)[2], int s, Scores& z) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r)
        z[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], qf[r][s], s == 0 ? (f32x4){0.f, 0.f, 0.f, 0.f} : z[t][r], 0, 0, 0);
  };
  // Scores of keys that a row does not see: -inf.
  const auto hide = [&](int32_t half, Scores& z) {
    if (half * kHalf + kHalf <= sees0) return;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int32_t sees = sees0 + 16 * r + c - half * kHalf - 4 * g;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) z[t][r][i] = 16 * t + i < sees ? z[t][r][i] : -INFINITY;
    }
  };
  const auto highest = [&](const Scores& z, int r) {
    float m = fmaxf(fmaxf(fmaxf(z[0][r][0], z[0][r][1]), z[0][r][2]), z[0][r][3]);
    return fmaxf(fmaxf(fmaxf(fmaxf(m, z[1][r][0]), z[1][r][1]), z[1][r][2]), z[1][r][3]) * a.scale_log2;
  };
  // Moves the reference of the rows whose scores pass it by 2^kSlack (a row by its
  // own scores alone).
  const auto move = [&](float m0, float m1) {
    if (!__any(m0 > top[0] + kSlack || m1 > top[1] + kSlack)) return;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float m = r ? m1 : m0;
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      m = m > top[r] + kSlack ? m : top[r];
      const float by = __builtin_amdgcn_exp2f(top[r] - m);
      top[r] = m;
      sum[r] *= by;
#pragma unroll
      for (int d = 0; d < 8; ++d) o[d][r] *= by;
    }
  };
  u32x4 pf[2];  // weights of a row block: pairs of keys 4 g .. of both tiles
  const auto weigh_pair = [&](const Scores& z, int n) {
    const int r = n >> 2, t = n >> 1 & 1, i = 2 * (n & 1);
    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][r][i], a.scale_log2, -top[r]));
    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][r][i + 1], a.scale_log2, -top[r]));
    pf[r][n & 3] = pack_bf16x2(p0, p1);
    sum[r] += p0;
    sum[r] += p1;
  };
  // Values that some rows do not see go into the product as 0 where they are not
  // finite (0 * NaN); the rows that see them get them at the end.
  bool odd = false;
  const auto only_finite = [&](bf16x8 v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // the exponent's field plus one of its units: the sign bit where it is all ones
      const u16x2 e = __builtin_bit_cast(u16x2, w[j] & 0x7f807f80u) + (u16x2){0x80, 0x80};
      const uint32_t bad = __builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, e) >> (s16x2){15, 15});
      odd |= bad != 0;
      w[j] &= ~bad;
    }
    return __builtin_bit_cast(bf16x8, w);
  };

  // Half by half: this half's scores beside the last one's weights, then its maxima
  // beside the last one's product.  k_at, v_at: where its keys and the last one's values are.
  const auto turn = [&](int32_t half, int k_at, int v_at, Scores& z, const Scores& last) {
    const bool now = half < mine, before = half > 2 * step0 && half - 1 < mine;  // (uniform in the wave)
    if (now) {
#pragma unroll
      for (int s = 0; s < 6; ++s) {
        const bf16x8 kf[2] = {key_operand(k_at, s, 0), key_operand(k_at, s, 1)};
        score_dims(kf, s, z);
      }
    }
    if (before) {
#pragma unroll
      for (int n = 0; n < 8; ++n) weigh_pair(last, n);
    }
    if (now) hide(half, z);
    if (before) {
      const auto product = [&](auto masked) {
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          bf16x8 vf = __builtin_bit_cast(bf16x8, value_operand(v_at, d));
          if constexpr (decltype(masked)::value) vf = only_finite(vf);
#pragma unroll
          for (int r = 0; r < 2; ++r) o[d][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pf[r]), o[d][r], 0, 0, 0);
        }
      };
      if (half * kHalf <= sees0) product(std::false_type{});
      else product(std::true_type{});
    }
    if (now) move(highest(z, 0), highest(z, 1));
  };

  // The same where every row sees every key and both halves have their part: 40 matrix
  // instructions in a row, the softmax dealt out between them, operands read kAhead
  // instructions' pairs before they are multiplied.  (In this order as written: left to
  // itself the compiler puts all of one kind together.)
  bf16x8 kf[12], vf[8];
  const auto full_turn = [&](int k_at, int v_at, int k_next, Scores& z, const Scores& last, auto first_half) {
    constexpr bool kFirst = decltype(first_half)::value;
    float p0 = 0.f, p1 = 0.f, m[2] = {-INFINITY, -INFINITY};
    // pair n's two exponentials, and what becomes of them
    const auto part = [&](auto at) {
      constexpr int n = decltype(at)::value >> 1, r = n >> 2, t = n >> 1 & 1, i = 2 * (n & 1);
      if constexpr ((decltype(at)::value & 1) == 0) {
        p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(last[t][r][i], a.scale_log2, -top[r]));
        p1 = __builtin_fmaf(last[t][r][i + 1], a.scale_log2, -top[r]);
      } else {
        p1 = __builtin_amdgcn_exp2f(p1);
        sum[r] += p0;
        pf[r][n & 3] = pack_bf16x2(p0, p1);
        sum[r] += p1;
      }
    };
    if constexpr (kFirst) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = key_operand(k_at, i >> 1, i & 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    static_for<24>([&](auto at) {
      constexpr int i = decltype(at)::value >> 1, r = decltype(at)::value & 1, s = i >> 1, t = i & 1;
      if constexpr (r == 0) {
        if constexpr (i + kAhead < 12) kf[i + kAhead] = key_operand(k_at, (i + kAhead) >> 1, (i + kAhead) & 1);
        else vf[i + kAhead - 12] = __builtin_bit_cast(bf16x8, value_operand(v_at, i + kAhead - 12));
      }
      z[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[r][s], s == 0 ? (f32x4){0.f, 0.f, 0.f, 0.f} : z[t][r], 0, 0, 0);
      if constexpr (decltype(at)::value % 3 != 2) part(std::integral_constant<int, decltype(at)::value / 3 * 2 + decltype(at)::value % 3>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    static_for<16>([&](auto at) {
      constexpr int d = decltype(at)::value >> 1, r = decltype(at)::value & 1;
      if constexpr (r == 0) {
        if constexpr (d + kAhead < 8) vf[d + kAhead] = __builtin_bit_cast(bf16x8, value_operand(v_at, d + kAhead));
        else if constexpr (kFirst) kf[d + kAhead - 8] = key_operand(k_next, (d + kAhead - 8) >> 1, (d + kAhead - 8) & 1);
      }
      o[d][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], __builtin_bit_cast(bf16x8, pf[r]), o[d][r], 0, 0, 0);
      m[d >> 2] = fmaxf(m[d >> 2], z[d >> 1 & 1][d >> 2][2 * (d & 1) + r]);
      __builtin_amdgcn_sched_barrier(0);
    });
    move(m[0] * a.scale_log2, m[1] * a.scale_log2);
  };

  Scores z0, z1;
  const auto arrive = [&]() {
    wait_vmcnt<0>();
    lds_barrier();  // this step's rows are there, and nobody reads the last one's
  };
  const auto general_step = [&](int32_t step) {
    arrive();
    if (step < step1) load_step(step + 1);
    const int slot = (step - step0) & 1;
    turn(2 * step, slot * kKeyBytes, slot * kValueBytes, z0, z1);
    turn(2 * step + 1, slot * kKeyBytes + 4096, slot * kValueBytes + 4096, z1, z0);
  };
  if (step0 < step1) {
    load_step(step0);
    general_step(step0);
    int32_t step = step0 + 1;
    // steps that all rows of the tile see, while a whole step follows them
    const int32_t full = min(min(step1, tile.keys / kKeys) - 1, tile.first_sees / kKeys);
    const bool idle = row0 >= tile.rows;
    if (step + 1 < full) {
      const uint8_t* kb = k_base + (int64_t)(step + 1) * kKeys * 2 * a.k_token;
      const uint8_t* rb = key_base + (int64_t)(step + 1) * kKeys * 2 * a.key_token;
      const uint8_t* vb = v_base + ((int64_t)(step + 1) * kKeys - kHalf) * 2 * a.v_token;
      for (; step + 1 < full; step += 2) {
        const auto one = [&](auto at) {
          constexpr int slot = decltype(at)::value;
          arrive();
          load_rows(kb, rb, vb, 1 - slot);
          kb += kKeys * 2 * a.k_token;
          rb += kKeys * 2 * a.key_token;
          vb += kKeys * 2 * a.v_token;
          if (idle) return;  // (uniform in the wave)
          full_turn(slot * kKeyBytes, slot * kValueBytes, slot * kKeyBytes + 4096, z0, z1, std::true_type{});
          full_turn(slot * kKeyBytes + 4096, slot * kValueBytes + 4096, 0, z1, z0, std::false_type{});
        };
        one(std::integral_constant<int, 1>{});
        one(std::integral_constant<int, 0>{});
      }
    }
    for (; step <= step1; ++step) general_step(step);
  }
  if (__any(odd)) {
    const int32_t from = max(sees0 / kHalf * kHalf, step0 * kKeys), to = min(mine * kHalf, tile.keys);
#pragma unroll 1
    for (int32_t j = max(from, 0); j < to; ++j)
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const u32x2 v = *(const u32x2*)(v_base + (int64_t)j * a.v_token * 2 + 32 * d + 8 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bits = i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16;
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if ((bits & 0x7f800000u) == 0x7f800000u && j < sees0 + 16 * r + c) o[d][r][i] += __builtin_bit_cast(float, bits);
        }
      }
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    p.top[r] = top[r];
    p.sum[r] = sum[r];
#pragma unroll
    for (int d = 0; d < 8; ++d) p.o[d][r] = o[d][r];
  }
}

// A row's sum over its four lanes.
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ void write_rows(const MlaPrefillLaunch& a, const Tile& tile, const Piece& p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int32_t row = kWaveRows * wave + 16 * r + c;
    const float l = row_sum(p.sum[r]);
    if (row >= min(tile.rows, kRows)) continue;
    const float by = 1.f / l;
    const int64_t n = (tile.q0 + row) * a.heads + tile.h;
    uint16_t* to = a.out + n * kValue + 4 * g;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const f32x4 v = l == 0.f ? (f32x4){0.f, 0.f, 0.f, 0.f} : p.o[d][r] * by;
      *(u32x2*)(to + 16 * d) = (u32x2){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
    if (a.lse && g == 0) a.lse[n] = l == 0.f ? -INFINITY : (p.top[r] + __log2f(l)) * 0.69314718055994530942f;
  }
}
__device__ __forceinline__ void write_part(const MlaPrefillLaunch& a, const Tile& tile, const Piece& p, int32_t slot) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int32_t row = kWaveRows * wave + 16 * r + c;
    const float l = row_sum(p.sum[r]);
    if (row >= min(tile.rows, kRows)) continue;
    float* to = a.part_out + ((int64_t)slot * kRows + row) * kValue + 4 * g;
#pragma unroll
    for (int d = 0; d < 8; ++d) *(f32x4*)(to + 16 * d) = p.o[d][r];
    if (g == 0) *(f32x2*)(a.part_ml + ((int64_t)slot * kRows + row) * 2) = (f32x2){p.top[r], l};
  }
}

// Workers of the line: all that fit on the chip, or as many as get kLeast steps.
__device__ __forceinline__ int32_t line_workers(const MlaPrefillLaunch& a, const Call& call) {
  const int64_t most = call.line * a.heads / kLeast / 8 * 8;
  return (int32_t)min(max(most, (int64_t)8), (int64_t)a.workers);
}
// Whether the tiles are cut: where the longest one takes longer than all of them over the chip.
__device__ __forceinline__ bool is_cut(const MlaPrefillLaunch& a, const Call& call) {
  return call.longest > kNeverCut && call.longest * (int64_t)a.workers > call.line * a.heads;
}

// A worker's piece of the line from `place` on.
struct Span {
  Tile tile;
  int32_t step0, step1;
  bool begins, ends;  // the piece begins or ends its tile
  int64_t first, tile_end, end;  // the worker's first place, the tile's end, the worker's
  int32_t workers;
  int64_t length;
};
__device__ __forceinline__ int64_t span_at(int64_t length, int32_t workers, int64_t k) {
  return length / workers * k + length % workers * k / workers;
}
__device__ __forceinline__ Span find_span(const MlaPrefillLaunch& a, const Call& call, int32_t w, int64_t place) {
  Span s;
  s.workers = line_workers(a, call);
  s.length = call.line * a.heads;
  s.first = span_at(s.length, s.workers, w);
  s.end = span_at(s.length, s.workers, w + 1);
  if (place < 0) place = s.first;
  const int32_t h = (int32_t)(place / call.line);
  int64_t begin = 0;
  int32_t count = 0;
  s.tile = Tile{h, 0, 0, 0, 0, 0};
  find_place(a, h, place - h * call.line, s.tile, begin, count);
  begin += h * call.line;
  s.tile_end = begin + count;
  // the tile's fixed work comes first on the line, and steps that it lacks last
  const int32_t steps = (s.tile.keys + kKeys - 1) / kKeys;
  s.begins = place == begin;
  s.ends = s.tile_end <= s.end;
  s.step0 = min(max((int32_t)(place - begin) - kTileCost, 0), steps);
  s.step1 = s.ends ? steps : min(max((int32_t)(s.end - begin) - kTileCost, 0), steps);
  return s;
}

// Whole tiles, a workgroup each, or the line of all tiles in equal spans.
__global__ __launch_bounds__(kThreads, 2) void mla_prefill_kernel(MlaPrefillLaunch a, int32_t shift) {
  __shared__ __align__(128) uint8_t lds[2 * (kKeyBytes + kValueBytes)];
  int32_t w = -1;             // the worker on the line (-1: a whole tile)
  int64_t place = -1;
  Tile tile;
  int32_t step0 = 0, step1;
  {
    const int32_t xcd = blockIdx.x & 7, at = blockIdx.x >> 3;   // (workgroups go round the 8 XCDs)
    if (a.joined) {
      const Call call = look_at(a);
      if (is_cut(a, call)) {
        const int32_t each = line_workers(a, call) / 8;
        if (at < each) w = xcd * each + at;  // neighbours on the line on one XCD
      }
      if (w < 0) {
        if (blockIdx.x < (uint32_t)a.workers && threadIdx.x == 0) a.joined[blockIdx.x] = make_int4(-1, 0, 0, 0);
        if (is_cut(a, call)) return;
      }
    }
    if (w < 0) {
      // Groups of 2^shift tiles of a head, neighbours of one XCD that begin together and
      // read the same keys; the longest groups first, of all heads.
      const int64_t group = (int64_t)(at >> shift) * 8 + xcd;
      Request r;
      int32_t block;
      if (!find_block(a, (int32_t)(group / a.heads), shift, r, block)) return;
      const int32_t i = tiles_of(r.nq) - 1 - (block << shift) - (at & ((1 << shift) - 1));
      if (i < 0) return;
      tile = tile_of(r, (int32_t)(group % a.heads), i);
      step1 = (tile.keys + kKeys - 1) / kKeys;
    }
  }
  int4 record = {-1, 0, 0, 0};
  Piece p;
  while (true) {
    if (w >= 0) {
      const Span s = find_span(a, look_at(a), w, place);
      if (place >= 0) lds_barrier();  // nobody reads the last piece's keys any more
      tile = s.tile;
      step0 = s.step0;
      step1 = s.step1;
    }
    attend(a, tile, step0, step1, lds, p);
    if (w < 0) {
      write_rows(a, tile, p);
      return;
    }
    // (found again: held beside the loop above, it would cost its registers)
    asm volatile("" : "+s"(place));
    const Span s = find_span(a, look_at(a), w, place);
    if (s.begins && s.ends) {
      write_rows(a, s.tile, p);
    } else {
      write_part(a, s.tile, p, 2 * w + (s.begins ? 1 : 0));
      if (s.begins) {
        // the parts of this tile: this one, and one of each worker up to its end
        int32_t last = w + 1;
        while (span_at(s.length, s.workers, last + 1) < s.tile_end) ++last;
        record = make_int4((int32_t)s.tile.q0, min(s.tile.rows, kRows), s.tile.h, last - w + 1);
      }
    }
    place = s.tile_end;
    if (place >= s.end) break;
  }
  if (threadIdx.x == 0) a.joined[w] = record;
}

// The parts of the tile that worker blockIdx.x begins, 16 rows a workgroup: sixteen
// lanes a row, eight values each.
__global__ __launch_bounds__(kThreads) void mla_prefill_join_kernel(MlaPrefillLaunch a) {
  const int32_t w = blockIdx.x;
  const int4 record = a.joined[w];
  const int32_t row = blockIdx.y * 16 + (threadIdx.x >> 4), lane = threadIdx.x & 15;
  if (record.x < 0 || row >= record.y) return;
  const auto slot = [&](int32_t k) { return ((int64_t)(k == 0 ? 2 * w + 1 : 2 * (w + k)) * kRows + row); };
  float top = kLowest;
  for (int32_t k = 0; k < record.w; ++k) {
    const float m = a.part_ml[slot(k) * 2];
    top = m > top || m != m ? m : top;
  }
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  float sum = 0.f;
  for (int32_t k = 0; k < record.w; ++k) {
    const f32x2 ml = *(const f32x2*)(a.part_ml + slot(k) * 2);
    if (ml[1] == 0.f) continue;  // no weight, and nothing in its output
    const float by = __builtin_amdgcn_exp2f(ml[0] - top);
    const f32x4* from = (const f32x4*)(a.part_out + slot(k) * kValue + 8 * lane);
    sum += by * ml[1];
    lo += by * from[0];
    hi += by * from[1];
  }
  const int64_t n = (int64_t)(record.x + row) * a.heads + record.z;
  const float by = sum == 0.f ? 0.f : 1.f / sum;
  lo *= by;
  hi *= by;
  *(u32x4*)(a.out + n * kValue + 8 * lane) =
      (u32x4){pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
  if (a.lse && lane == 0) a.lse[n] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * 0.69314718055994530942f;
}

}  // namespace

hipError_t launch_mla_prefill(const MlaPrefillLaunch& a, hipStream_t s) {
  // Tiles of a request that are placed together: as many as an average request has, at most 4.
  const int64_t rows_each = a.num_rows / a.B;
  const int shift = rows_each >= 4 * kRows ? 2 : rows_each >= 2 * kRows ? 1 : 0;
  // no request adds more than one block that is not full
  const int64_t blocks = min((int64_t)a.num_rows / (kRows << shift) + a.B, (int64_t)a.num_rows);
  int64_t groups = (blocks * a.heads + 7) / 8 * 8 << shift;
  MlaPrefillLaunch l = a;
  if (a.num_keys <= kNeverCut * kKeys) l.joined = nullptr;
  else groups = max(groups, (int64_t)a.workers);
  hipLaunchKernelGGL(mla_prefill_kernel, dim3((unsigned)groups), dim3(kThreads), 0, s, l, shift);
  if (l.joined) hipLaunchKernelGGL(mla_prefill_join_kernel, dim3((unsigned)a.workers, kRows / 16), dim3(kThreads), 0, s, l);
  return hipGetLastError();
}

}  // namespace splash
