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
// LDS: a step's rows in line groups of 128 bytes, [group][key][128], key chunks of 16
// bytes at chunk ^ swz(key); groups 0 and 1 are the head's key dims, 2 the rotary
// ones, 3 and 4 the value.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;              // query rows of a tile
constexpr int kWaveRows = 32;
constexpr int kKeys = 64;               // keys of a step
constexpr int kGroupBytes = kKeys * 128;
constexpr int kGroups = 5;
constexpr int kStepBytes = kGroups * kGroupBytes;
constexpr float kSlack = 8.f;           // powers of two by which a score may pass the reference
constexpr float kLowest = -1e30f;       // the reference before any score

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
// 16 bytes a lane from base + offset straight to LDS at `lds` + 16 * lane.  Through asm,
// so that the compiler does not wait for it at every LDS read; the kernel does.
__device__ __forceinline__ void load_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

struct Tile {
  int32_t rows;        // of the request past the tile's first
  int64_t q0;          // the tile's first query row
  int64_t k0;          // the request's first key
  int32_t first_sees;  // keys that the tile's first row sees (may be negative)
  int32_t keys;        // keys that any row of the tile sees
};

// Tile `at` of the requests' tiles in order (a request's last tile first), by 64
// requests at a time.
__device__ __forceinline__ bool find_tile(const MlaPrefillLaunch& a, int32_t at, Tile& t) {
  const int lane = threadIdx.x & 63;
  for (int32_t b0 = 0; b0 < a.B; b0 += 64) {
    const int32_t b = min(b0 + lane, a.B - 1);
    const int32_t q0 = min(max(a.q_indptr[b], 0), a.num_rows), q1 = min(max(a.q_indptr[b + 1], q0), a.num_rows);
    const int32_t tiles = b0 + lane < a.B ? (q1 - q0 + kRows - 1) / kRows : 0;
    int32_t upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t other = __shfl_up(upto, d);
      upto += lane >= d ? other : 0;
    }
    const uint64_t past = __ballot(upto > at);
    if (!past) {
      at -= __builtin_amdgcn_readlane(upto, 63);
      continue;
    }
    const int who = __builtin_ctzll(past);
    const int32_t i = __builtin_amdgcn_readlane(upto, who) - 1 - at;
    const int32_t first = __builtin_amdgcn_readlane(q0, who), nq = __builtin_amdgcn_readlane(q1, who) - first;
    const int32_t k0 = min(max(a.kv_indptr[b0 + who], 0), a.num_keys), k1 = min(max(a.kv_indptr[b0 + who + 1], k0), a.num_keys);
    const int32_t nk = k1 - k0;
    t.q0 = first + i * kRows;
    t.rows = nq - i * kRows;
    t.k0 = k0;
    t.first_sees = nk - nq + i * kRows + 1;
    t.keys = max(0, t.first_sees - 1 + min(t.rows, kRows));
    return true;
  }
  return false;
}

__global__ __launch_bounds__(kThreads, 2) void mla_prefill_kernel(MlaPrefillLaunch a, int32_t tiles, int32_t per_xcd) {
  __shared__ __align__(128) uint8_t lds[2 * kStepBytes];
  // Workgroups go round the 8 XCDs: each takes a run of the (head, tile) line, so
  // that the tiles of a head read its keys from one L2.
  const int64_t at = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (at >= (int64_t)tiles * a.heads) return;
  const int32_t h = (int32_t)(at / tiles);
  Tile tile;
  if (!find_tile(a, (int32_t)(at - (int64_t)h * tiles), tile)) return;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int32_t row0 = kWaveRows * wave;            // the wave's first row in the tile
  const int32_t sees0 = tile.first_sees + row0;     // keys that it sees
  const bool idle = row0 >= tile.rows;

  // Q as B operands: row c of a block of 16, eight dims from 8 g.
  bf16x8 qf[2][6];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int64_t row = tile.q0 + min(row0 + 16 * r + c, tile.rows - 1);
    const uint16_t* from = a.q + row * a.q_token + h * a.q_head + 8 * g;
#pragma unroll
    for (int s = 0; s < 6; ++s) qf[r][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(from + 32 * s));
  }

  // A step's loads: the wave brings keys 16 wave .. + 15, eight a load, of each line group.
  const int32_t steps = (tile.keys + kKeys - 1) / kKeys;
  const uint8_t* k_base = (const uint8_t*)(a.k + tile.k0 * a.k_token + h * a.k_head);
  const uint8_t* key_base = (const uint8_t*)(a.key + tile.k0 * a.key_token);
  const uint8_t* v_base = (const uint8_t*)(a.v + tile.k0 * a.v_token + h * a.v_head);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_AS uint8_t*)lds;
  const auto load_step = [&](int32_t step) {
    const int32_t first = step * kKeys, last = tile.keys - 1 - first;  // (a row past the last key: the last key again)
    const uint8_t* kb = k_base + (int64_t)first * a.k_token * 2;
    const uint8_t* rb = key_base + (int64_t)first * a.key_token * 2;
    const uint8_t* vb = v_base + (int64_t)first * a.v_token * 2;
    const uint32_t to = lds0 + (step & 1) * kStepBytes + 2048 * wave;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t row = 16 * wave + 8 * i + (lane >> 3), from = min((int32_t)row, last), chunk = 16 * ((lane & 7) ^ swz(row));
      const uint32_t k_at = from * (uint32_t)a.k_token * 2 + chunk, r_at = from * (uint32_t)a.key_token * 2 + chunk;
      const uint32_t v_at = from * (uint32_t)a.v_token * 2 + chunk;
      load_lds(kb, k_at, to + 1024 * i);
      load_lds(kb, k_at + 128, to + 1024 * i + kGroupBytes);
      load_lds(rb, r_at, to + 1024 * i + 2 * kGroupBytes);
      load_lds(vb, v_at, to + 1024 * i + 3 * kGroupBytes);
      load_lds(vb, v_at + 128, to + 1024 * i + 4 * kGroupBytes);
    }
  };

  // K operand of 32 dims: chunk g (or 4 + g) of row c; V: see the top.
  const uint32_t k_lane = 128 * c + 16 * (g ^ swz(c));
  const uint32_t v_row = 4 * g + (c >> 2);
  const uint32_t v_lane = 3 * kGroupBytes + 128 * v_row + 16 * (((c >> 1) & 1) ^ swz(v_row)) + 8 * (c & 1);

  f32x4 o[8][2] = {};
  float top[2] = {kLowest, kLowest}, sum[2] = {0.f, 0.f};
  if (steps > 0) load_step(0);
  for (int32_t step = 0; step < steps; ++step) {
    wait_vmcnt<0>();
    lds_barrier();  // this step is there, and nobody reads the other buffer
    if (step + 1 < steps) load_step(step + 1);
    const int32_t first = step * kKeys;
    if (idle || first >= sees0 + kWaveRows - 1) continue;  // (uniform in the wave; the barriers are outside)
    const LDS_AS uint8_t* buf = (const LDS_AS uint8_t*)lds + (step & 1) * kStepBytes;

    f32x4 z[4][2] = {};
#pragma unroll
    for (int s = 0; s < 6; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const bf16x8 kf = *(const LDS_AS bf16x8*)(buf + (k_lane ^ (64 * (s & 1))) + kGroupBytes * (s >> 1) + 2048 * t);
#pragma unroll
        for (int r = 0; r < 2; ++r) z[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][s], z[t][r], 0, 0, 0);
      }

    const bool masked = first + kKeys > sees0;
    uint32_t pf[2][2][4];  // [row block][32 keys][pairs]
    bool moves = false;
    float highest[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int32_t sees = sees0 + 16 * r + c - first;  // keys of this step that the row sees
      highest[r] = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          z[t][r][i] *= a.scale_log2;
          if (masked && 16 * t + 4 * g + i >= sees) z[t][r][i] = -INFINITY;
          highest[r] = fmaxf(highest[r], z[t][r][i]);
        }
      moves |= highest[r] > top[r] + kSlack;
    }
    if (__any(moves)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float m = fmaxf(highest[r], __shfl_xor(highest[r], 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        m = m > top[r] + kSlack ? m : top[r];  // (a row by its own scores alone)
        const float by = __builtin_amdgcn_exp2f(top[r] - m);
        top[r] = m;
        sum[r] *= by;
#pragma unroll
        for (int d = 0; d < 8; ++d) o[d][r] *= by;
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const float p0 = __builtin_amdgcn_exp2f(z[t][r][i] - top[r]), p1 = __builtin_amdgcn_exp2f(z[t][r][i + 1] - top[r]);
          pf[r][t >> 1][2 * (t & 1) + i / 2] = pack_bf16x2(p0, p1);
          sum[r] += p0;
          sum[r] += p1;
        }

    // Values that some rows do not see, where they are not finite: 0 * NaN.  They go
    // into the product as 0 and are added to the rows that see them.
    bool odd = false;
    if (masked) {
#pragma unroll 4
      for (int i = 0; i < 16; ++i) {
        const u32x4 w = *(const LDS_AS u32x4*)(buf + 3 * kGroupBytes + 1024 * i + 16 * lane);
#pragma unroll
        for (int j = 0; j < 4; ++j) odd |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
      }
      odd = __any(odd);
    }
    const auto multiply = [&](auto only_finite) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          const LDS_AS uint8_t* from = buf + (v_lane ^ (32 * (d & 3))) + kGroupBytes * (d >> 2) + 4096 * u;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)from);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)(from + 2048));
          auto vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          if constexpr (decltype(only_finite)::value) {
#pragma unroll
            for (int j = 0; j < 8; ++j) vf[j] = (vf[j] & 0x7f80) == 0x7f80 ? (short)0 : vf[j];
          }
#pragma unroll
          for (int r = 0; r < 2; ++r)
            o[d][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, vf),
                __builtin_bit_cast(bf16x8, (u32x4){pf[r][u][0], pf[r][u][1], pf[r][u][2], pf[r][u][3]}), o[d][r], 0, 0, 0);
        }
    };
    if (!odd) {
      multiply(std::false_type{});
    } else {
      multiply(std::true_type{});
      for (int32_t j = 0; j < kKeys; ++j)
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          const uint32_t chunk = (2 * (d & 3) + (g >> 1)) ^ swz(j);
          const u32x2 w = *(const LDS_AS u32x2*)(buf + (3 + (d >> 2)) * kGroupBytes + 128 * j + 16 * chunk + 8 * (g & 1));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bits = i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16;
#pragma unroll
            for (int r = 0; r < 2; ++r)
              if ((bits & 0x7f800000u) == 0x7f800000u && j < sees0 + 16 * r + c - first) o[d][r][i] += __builtin_bit_cast(float, bits);
          }
        }
    }
  }

#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int32_t row = row0 + 16 * r + c;
    float l = sum[r] + __shfl_xor(sum[r], 16);
    l += __shfl_xor(l, 32);
    if (row >= min(tile.rows, kRows)) continue;
    const float by = l == 0.f ? 0.f : 1.f / l;
    uint16_t* to = a.out + ((tile.q0 + row) * a.heads + h) * kValue + 4 * g;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const f32x4 v = l == 0.f ? (f32x4){0.f, 0.f, 0.f, 0.f} : o[d][r] * by;
      *(u32x2*)(to + 16 * d) = (u32x2){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
    if (a.lse && g == 0) a.lse[(tile.q0 + row) * a.heads + h] = l == 0.f ? -INFINITY : (top[r] + __log2f(l)) * 0.69314718055994530942f;
  }
}

}  // namespace

hipError_t launch_mla_prefill(const MlaPrefillLaunch& a, hipStream_t s) {
  // no request adds more than one tile that is not full
  const int32_t tiles = (int32_t)min((int64_t)a.num_rows / kRows + a.B, (int64_t)a.num_rows);
  const int64_t line = (int64_t)tiles * a.heads, per_xcd = (line + 7) / 8;
  hipLaunchKernelGGL(mla_prefill_kernel, dim3((unsigned)(8 * per_xcd)), dim3(kThreads), 0, s, a, tiles, (int32_t)per_xcd);
  return hipGetLastError();
}

}  // namespace splash
