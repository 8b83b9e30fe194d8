// gfx950 kernel of splash_mla_prefill: causal attention of ragged prompts over
// expanded keys (128 of a head's own dims, 64 shared rotary ones) and values.
//
// A workgroup of W waves takes a tile of 32 W query rows of a request and head, 32 a
// wave, and walks over the keys in steps of 64 whose keys and values come straight into
// LDS, the next steps' while this one is multiplied; a step is two turns of 32 keys.
//   QK  S^T[key, row] = K Q^T, v_mfma_f32_16x16x32_bf16.  Lane (g, c) holds keys
//       16 t + 4 g + i of row c: the weights of a row stay in its four lanes.
//   PV  O^T[value, row] = V^T P^T.  The product's slot (g, j) is key 4 g + j of tile 0
//       (j < 4) or 4 g + j - 4 of tile 1: P goes from QK's result to PV's operand in the
//       lane that has it, and V's transposing reads take the rows in that order.  P is
//       rounded to bf16, V's type, for it (outputs are off by 2.1e-3 of their norm, 1.6e-3
//       with exact weights); the weights' sum is of the unrounded ones.
// A turn multiplies QK of its keys while the exponentials of the last turn's scores are
// dealt out between the matrix instructions, then PV of the last turn: a step's values
// are the second half of the step before and the first of its own.
//
// The softmax runs over the keys once with a reference 2^10 above the largest score, which
// moves only where a lane's eight weights of a row pass 1: below that no sum of weights can
// overflow, and the lane needs no maximum and no exchange for it, only the sum that it makes
// anyway.  A row's nk weights are nk / 8 at most together (2^-5 of the first turn, 4 of each
// other one), so that values up to 2^129 / nk stay in fp32's range.  Each row decides by its own scores:
// other rows' values do not reach its result (their lengths do, where tiles are cut: the
// cuts' places are the whole call's, and the order of a row's sums with them).
//
// Bound: matrix instructions, 320 multiplications and additions each a row and key of a
// head (192 + 128), at 1.36 PFLOP/s of a large library product.  128 heads of one prompt
// of 4096 rows: 705 us, 975 TFLOP/s; 32 of 2 x 4096 rows over 4096 more: 907 us, 1,136.
// Of the first, the matrix instructions alone take 420 us, the loads into LDS 130, its
// reads 100 and the softmax 80 that two waves a SIMD do not hide (copies of the kernel
// with the rest left out); a tile costs 8 us beside its turns (by the clock: loads of its
// first step and queries 3.4, writing the last one's rows 3.6, the meeting of its waves
// 1.1), and a masked turn has 440 vector instructions, others 260.
//
// W = 8: one workgroup fills a compute unit, four steps in LDS, two of them on the way;
// W = 4: two do, two steps each.  The larger tile halves the loads a row and keeps long
// walks fed; the smaller one wastes less of the triangle at the end of the keys and of a
// last tile.
//
// LDS: a step's keys, then its values, in line groups of 128 bytes, [group][key][128],
// chunks of 16 bytes at chunk ^ swz(key); keys are groups 0 and 1 for the head's own dims
// and 2 for the rotary ones, values two more.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "device_types.hpp"
#include "layer.hpp"
#include "lds_loads.hpp"

namespace splash {

namespace {

constexpr int kThreads = 256;                 // of the join
constexpr int kKeys = 64;                     // keys of a step
constexpr int kHalf = 32;                     // keys of a turn
constexpr int kGroupBytes = kKeys * 128;
constexpr int kKeyBytes = 3 * kGroupBytes;    // a step's keys in LDS
constexpr int kStepBytes = 5 * kGroupBytes;   // and its values after them
constexpr int kLoads = 40;                    // loads to LDS a step, by all waves
constexpr int kAhead = 4;                     // operands read ahead
constexpr float kMost = 1.f;                  // a lane's eight weights of a row, before the reference moves
constexpr float kAbove = 10.f;                // powers of two from a row's largest score up to where it moves
constexpr float kLowest = -1e30f;             // the reference before any score
// A cut tile's parts pass through memory and a second launch joins them (6 us): tiles of
// at most kNeverCut steps, 768 keys, do not wait as long, and a worker of the line gets
// kLeast steps or more.  Places on the line count eighths of a step.  A piece costs 16 to
// 18 us beside its steps of 2.1 (first loads, the diagonal, writing its part), kTileCost,
// and a step of a tile of half the rows or less, a wave a SIMD instead of two, 0.65 of
// others (95 us against 145).  Counted so, 8 heads of 8192 rows take 186 us, 20 of 382 and
// 512 rows over 18k and 10k keys 181; with every step alike and a tile's cost of one 234
// and 194.  (Costs of 4 and 12 steps: 206 and 199, 185 and 187.)
constexpr int32_t kNeverCut = 12;
constexpr int32_t kLeast = 4;
constexpr int32_t kStep = 8, kHalfStep = 5;
constexpr int32_t kTileCost = 8 * kStep;
constexpr int64_t kLongest = (int64_t)1 << 50;  // a head's line (2^41 for any indptr that does not decrease)
constexpr int kSorted = 4;                    // requests a lane that the order of the blocks looks at

constexpr int kWaveRows = 32;
constexpr int kBlocks = 2;                    // row blocks of 16 a wave
constexpr int tile_rows(int W) { return kWaveRows * W; }
constexpr int steps_held(int W) { return W == 8 ? 4 : 2; }

__device__ __forceinline__ uint32_t swz(uint32_t r) {
  return ((r & 2u)) | ((((r >> 2) ^ (r >> 3)) & 1u) << 2) | ((r >> 3) & 1u);
}

// A tile: `ROWS` rows of a request, of the head `h`.
struct Tile {
  int32_t h;
  int32_t rows;        // at most ROWS
  int64_t q0;          // the tile's first query row
  int64_t k0;          // the request's first key
  int32_t first_sees;  // keys that the tile's first row sees (may be negative)
  int32_t keys;        // keys that any row of the tile sees
};

struct Request {
  int32_t q0, nq, k0, nk;
};
// The kernel's arguments, read again: scalar registers that hold them from one use to the
// next one far away are missed by the loop between.
__device__ __forceinline__ MlaPrefillLaunch arguments() {
  static_assert(sizeof(MlaPrefillLaunch) % 8 == 0, "words");
  constexpr int kWords = sizeof(MlaPrefillLaunch) / 8;
  const auto* from = (const __attribute__((address_space(4))) uint64_t*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(from));
  uint64_t word[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) word[i] = from[i];
  MlaPrefillLaunch a;
  __builtin_memcpy(&a, word, sizeof(a));
  return a;
}
__device__ __forceinline__ Request request(const MlaPrefillLaunch& a, int32_t b) {
  Request r;
  r.q0 = min(max(a.q_indptr[b], 0), a.num_rows);
  r.nq = min(max(a.q_indptr[b + 1], r.q0), a.num_rows) - r.q0;
  r.k0 = min(max(a.kv_indptr[b], 0), a.num_keys);
  r.nk = min(max(a.kv_indptr[b + 1], r.k0), a.num_keys) - r.k0;
  return r;
}
template <int ROWS>
__device__ __forceinline__ Tile tile_of(const Request& r, int32_t h, int32_t i) {
  Tile t;
  t.h = h;
  t.q0 = r.q0 + (int64_t)i * ROWS;
  t.rows = min(r.nq - i * ROWS, ROWS);
  t.k0 = r.k0;
  t.first_sees = r.nk - r.nq + i * ROWS + 1;
  t.keys = max(0, t.first_sees - 1 + t.rows);
  return t;
}

template <int ROWS>
__device__ __forceinline__ int32_t tiles_of(int32_t nq) {
  return (nq + ROWS - 1) / ROWS;
}
// A request's tile i on the line: a tile's cost, then base + D i steps, D = ROWS / 64, its
// own and at most D more.  The line's length up to tile i, of whole tiles all.
template <int ROWS>
__device__ __forceinline__ int32_t line_base(const Request& r) {
  return max(0, (r.nk - r.nq + kKeys - 1) / kKeys) + ROWS / kKeys;
}
template <int ROWS>
__device__ __forceinline__ int64_t line_upto(int64_t i, int32_t base, int32_t cost) {
  return i * ((int64_t)kStep * base + cost + kStep * (ROWS / kKeys) / 2 * (i - 1));
}
template <int ROWS>
__device__ __forceinline__ int32_t line_step(const Request& r, int32_t i) {
  return r.nq - i * ROWS <= ROWS / 2 ? kHalfStep : kStep;
}
template <int ROWS>
__device__ __forceinline__ int64_t line_tile(const Request& r, int32_t i, int32_t cost) {
  return (int64_t)line_step<ROWS>(r, i) * (line_base<ROWS>(r) + ROWS / kKeys * i) + cost;
}
template <int ROWS>
__device__ __forceinline__ int64_t line_request(const Request& r, int32_t cost) {
  const int32_t n = tiles_of<ROWS>(r.nq);
  return n > 0 ? line_upto<ROWS>(n - 1, line_base<ROWS>(r), cost) + line_tile<ROWS>(r, n - 1, cost) : 0;
}

__device__ __forceinline__ int32_t uniform(int32_t v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int64_t uniform(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)(v >> 32), lane) << 32 | (uint32_t)uniform((int32_t)v, lane));
}
__device__ __forceinline__ Request uniform(const Request& r, int lane) {
  return {uniform(r.q0, lane), uniform(r.nq, lane), uniform(r.k0, lane), uniform(r.nk, lane)};
}
// The lanes' running sum, maximum or minimum in six moves between registers (steps of
// 1, 2, 4 and 8 lanes of a row of 16, then the last lane of a row to the next row, and of
// two rows to the next two); `none` where a lane gets nothing.
template <int CONTROL, int ROWS>
__device__ __forceinline__ int32_t moved(int32_t v, int32_t none) {
  return __builtin_amdgcn_update_dpp(none, v, CONTROL, ROWS, 0xf, false);
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ int64_t moved(int64_t v, int64_t none) {
  return (int64_t)((uint64_t)(uint32_t)moved<CONTROL, ROWS>((int32_t)(v >> 32), (int32_t)(none >> 32)) << 32 |
                   (uint32_t)moved<CONTROL, ROWS>((int32_t)v, (int32_t)none));
}
template <typename T, typename F>
__device__ __forceinline__ T wave_run(T v, T none, F join) {
  v = join(v, moved<0x111, 0xf>(v, none));
  v = join(v, moved<0x112, 0xf>(v, none));
  v = join(v, moved<0x114, 0xf>(v, none));
  v = join(v, moved<0x118, 0xf>(v, none));
  v = join(v, moved<0x142, 0xa>(v, none));
  return join(v, moved<0x143, 0xc>(v, none));
}
template <typename T>
__device__ __forceinline__ T wave_prefix(T v) {
  return wave_run(v, (T)0, [](T a, T b) { return a + b; });
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
  return uniform(wave_prefix(v), 63);
}
__device__ __forceinline__ int32_t wave_max(int32_t v) {
  return uniform(wave_run(v, (int32_t)INT_MIN, [](int32_t a, int32_t b) { return max(a, b); }), 63);
}
__device__ __forceinline__ int32_t wave_min(int32_t v) {
  return uniform(wave_run(v, (int32_t)INT_MAX, [](int32_t a, int32_t b) { return min(a, b); }), 63);
}

// What every workgroup finds out by itself about the whole call.
struct Call {
  int64_t steps;    // a head's, in eighths
  int32_t tiles;    // a head's
  int32_t longest;  // the longest tile's steps
};
template <int ROWS>
__device__ __forceinline__ Call look_at(const MlaPrefillLaunch& a) {
  const int lane = threadIdx.x & 63;
  int64_t steps = 0, tiles = 0;
  int32_t longest = 0;
  for (int32_t b = lane; b < a.B; b += 64) {
    const Request r = request(a, b);
    const int32_t n = tiles_of<ROWS>(r.nq);
    steps += line_request<ROWS>(r, 0);
    tiles += n;
    longest = max(longest, n > 0 ? (r.nk + kKeys - 1) / kKeys : 0);
  }
  return {wave_sum(steps), (int32_t)min(wave_sum(tiles), (int64_t)INT_MAX), wave_max(longest)};
}

// Block number `rank` of the requests' blocks of 2^shift tiles, counted from a request's last
// tile, the longest first: which of its request's and of which request (false: none).
// Block j counts as K - D j steps, K its request's last tile's: how many
// blocks are longer than a length is a sum over the requests, and the rank's length
// is found by halving.  Past 64 kSorted requests, and where all tiles begin at once anyway
// (`sorted` false: 15.2 us for four short prompts, 16.1 sorted), the blocks go in the requests' order.
template <int ROWS>
__device__ __forceinline__ bool find_block(const MlaPrefillLaunch& a, bool sorted, int32_t rank, int shift, Request& r, int32_t& block) {
  const int lane = threadIdx.x & 63;
  constexpr int kLog = ROWS == 256 ? 2 : 1;  // of a tile's steps
  const int D = 1 << (kLog + shift);
  if (sorted && a.B <= 64 * kSorted) {
    Request mine[kSorted];
    int32_t blocks[kSorted], top[kSorted], most = INT_MIN, least = INT_MAX;
#pragma unroll
    for (int k = 0; k < kSorted; ++k) {
      blocks[k] = top[k] = 0;
      mine[k] = Request{0, 0, 0, 0};
      if (64 * k < a.B) {
        const int32_t b = 64 * k + lane;
        mine[k] = request(a, min(b, a.B - 1));
        blocks[k] = b < a.B ? (tiles_of<ROWS>(mine[k].nq) + (1 << shift) - 1) >> shift : 0;
        top[k] = (mine[k].nk + kKeys - 1) / kKeys;
        if (blocks[k] > 0) {
          most = max(most, top[k]);
          least = min(least, top[k] - (blocks[k] - 1) * D);
        }
      }
    }
    const auto longer = [&](int32_t than) {  // blocks of more steps
      int32_t n = 0;
#pragma unroll
      for (int k = 0; k < kSorted; ++k)
        if (64 * k < a.B) n += min(blocks[k], max(0, top[k] - than + D - 1) >> (kLog + shift));
      return wave_sum(n);
    };
    // the least length that at most `rank` blocks pass: above it there are no more, and the
    // rank's block is one of this length
    int32_t lo = wave_min(least), hi = wave_max(most);
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
      const int32_t down = top[k] - lo, j = down >> (kLog + shift);
      const uint64_t here = __ballot(down >= 0 && (down & (D - 1)) == 0 && j < blocks[k]);
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
    const int32_t blocks = b0 + lane < a.B ? (tiles_of<ROWS>(mine.nq) + (1 << shift) - 1) >> shift : 0, upto = wave_prefix(blocks);
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

// The tile that holds place `at` of a head's line: its request, which of it, and where it begins.
template <int ROWS>
__device__ __forceinline__ bool find_place(const MlaPrefillLaunch& a, int32_t cost, int64_t at, Request& r, int32_t& tile, int64_t& begin) {
  const int lane = threadIdx.x & 63;
  int64_t behind = 0;
  for (int32_t b0 = 0; b0 < a.B; b0 += 64) {
    const Request mine = request(a, min(b0 + lane, a.B - 1));
    const int64_t own = b0 + lane < a.B ? line_request<ROWS>(mine, cost) : 0, upto = wave_prefix(own);
    const uint64_t past = __ballot(behind + upto > at);
    if (!past) {
      behind += uniform(upto, 63);
      continue;
    }
    const int who = __builtin_ctzll(past);
    r = uniform(mine, who);
    behind += uniform(upto - own, who);
    // the last i with line_upto(i) <= at - behind
    const int32_t base = line_base<ROWS>(r);
    const int64_t x = at - behind;
    constexpr double kD = 0.5 * kStep * (ROWS / kKeys);
    const double half = 0.5 * ((double)kStep * base + cost - kD) / kD;
    int64_t i = (int64_t)(__builtin_sqrt(half * half + (double)x / kD) - half);
    i = min(max(i, (int64_t)0), (int64_t)tiles_of<ROWS>(r.nq) - 1);
    while (i > 0 && line_upto<ROWS>(i, base, cost) > x) --i;
    while (i + 1 < tiles_of<ROWS>(r.nq) && line_upto<ROWS>(i + 1, base, cost) <= x) ++i;
    tile = __builtin_amdgcn_readfirstlane((int32_t)i);
    begin = behind + line_upto<ROWS>(tile, base, cost);
    return true;
  }
  return false;
}

// A row's sum over its four lanes.
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A row's LSE from its reference and sum (both brought back by kAbove first: a logarithm near
// -10 would be off by more).
__device__ __forceinline__ float natural_lse(float top, float l) {
  return l == 0.f ? -INFINITY : (top - kAbove + __log2f(l * 1024.f)) * 0.69314718055994530942f;
}

// Softmax and products of a tile's steps [step0, step1) in this workgroup's waves;
// `before` runs once the first loads are on their way (p still holds the last tile),
// `after` once the wave has multiplied all that it sees, while others still do.
struct Piece {
  f32x4 o[8][kBlocks];  // O^T: values 16 d + 4 g + i of rows 16 r + c, over exp2 of the reference
  float top[kBlocks], sum[kBlocks];
};
typedef f32x4 Scores[2][kBlocks];  // S^T of a turn's keys: keys 16 t + 4 g + i of rows 16 r + c

template <int W, typename Before, typename After>
__device__ __forceinline__ void attend(const MlaPrefillLaunch& a, const Tile& tile, int32_t step0, int32_t step1, uint8_t* lds, Piece& p,
                                       Before before, After after) {
  constexpr int R = kBlocks, kHeld = steps_held(W);
  constexpr bool kEarly = W == 8;  // the next step arrives in the middle of a step's last turn
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // (its offsets are made for each tile, not held from one to the next)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int32_t row0 = kWaveRows * wave;            // the wave's first row in the tile
  const int32_t sees0 = tile.first_sees + row0;     // keys that it sees
  // turns up to which the wave sees a key
  const int32_t mine = row0 >= tile.rows ? 2 * step0 : max(2 * step0, min(2 * step1, (sees0 + kWaveRows - 1 + kHalf - 1) / kHalf));

  // A step's loads: its keys, and the values of the last step's second half and its own
  // first, as they are multiplied.  A wave brings 64 / W rows, eight a load, of each line
  // group; a row outside the tile's keys is its first or last one.
  constexpr int kEach = 8 / W;  // loads of a line group
  const uint8_t* k_base = (const uint8_t*)(a.k + tile.k0 * a.k_token + tile.h * a.k_head);
  const uint8_t* key_base = (const uint8_t*)(a.key + tile.k0 * a.key_token);
  const uint8_t* v_base = (const uint8_t*)(a.v + tile.k0 * a.v_token + tile.h * a.v_head);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_AS uint8_t*)lds + 1024 * kEach * wave;
  const int32_t load_row = 8 * kEach * wave + (lane >> 3);
  const uint32_t chunk0 = 16 * ((lane & 7) ^ swz(load_row)), chunk1 = 16 * ((lane & 7) ^ swz(load_row + 8));
  const uint32_t k_off = load_row * (uint32_t)a.k_token * 2 + chunk0, key_off = load_row * (uint32_t)a.key_token * 2 + chunk0;
  const uint32_t v_off = load_row * (uint32_t)a.v_token * 2 + chunk0, next8 = chunk1 - chunk0;
  const auto load_step = [&](int32_t step) {
    const int32_t first = step * kKeys;
    const uint32_t to = lds0 + ((step - step0) & (kHeld - 1)) * kStepBytes, v_to = to + kKeyBytes;
    if (first >= kHalf && first + kKeys <= tile.keys) {
      const uint8_t* kb = k_base + (int64_t)first * a.k_token * 2;
      const uint8_t* rb = key_base + (int64_t)first * a.key_token * 2;
      const uint8_t* vb = v_base + (int64_t)(first - kHalf) * a.v_token * 2;
      load_lds<0>(kb, k_off, to);
      load_lds<128>(kb, k_off, to + kGroupBytes);
      load_lds<0>(rb, key_off, to + 2 * kGroupBytes);
      load_lds<0>(vb, v_off, v_to);
      load_lds<128>(vb, v_off, v_to + kGroupBytes);
      if constexpr (kEach == 2) {
        kb += 16 * a.k_token;
        rb += 16 * a.key_token;
        vb += 16 * a.v_token;
        load_lds<0>(kb, k_off + next8, to + 1024);
        load_lds<128>(kb, k_off + next8, to + 1024 + kGroupBytes);
        load_lds<0>(rb, key_off + next8, to + 1024 + 2 * kGroupBytes);
        load_lds<0>(vb, v_off + next8, v_to + 1024);
        load_lds<128>(vb, v_off + next8, v_to + 1024 + kGroupBytes);
      }
      return;
    }
    // rows counted from a base that leaves them less than 64 apart (steps past the last
    // one load its rows again: every step counts as many)
    const int32_t most = max(tile.keys - kKeys, 0), k_from = min(first, most), v_from = min(max(first - kHalf, 0), most);
    const uint8_t* kb = k_base + (int64_t)k_from * a.k_token * 2;
    const uint8_t* rb = key_base + (int64_t)k_from * a.key_token * 2;
    const uint8_t* vb = v_base + (int64_t)v_from * a.v_token * 2;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int32_t row = load_row + 8 * i;
      const uint32_t chunk = i ? chunk1 : chunk0;
      const uint32_t k_row = min(first + row, tile.keys - 1) - k_from;
      const uint32_t v_row = min(max(first - kHalf + row, 0), tile.keys - 1) - v_from;
      const uint32_t k_at = k_row * (uint32_t)a.k_token * 2 + chunk, r_at = k_row * (uint32_t)a.key_token * 2 + chunk;
      const uint32_t v_at = v_row * (uint32_t)a.v_token * 2 + chunk;
      load_lds<0>(kb, k_at, to + 1024 * i);
      load_lds<128>(kb, k_at, to + 1024 * i + kGroupBytes);
      load_lds<0>(rb, r_at, to + 1024 * i + 2 * kGroupBytes);
      load_lds<0>(vb, v_at, v_to + 1024 * i);
      load_lds<128>(vb, v_at, v_to + 1024 * i + kGroupBytes);
    }
  };
  // Step `step` is there, nobody reads the one before the last, and another one is on its way.
  const auto arrive = [&](int32_t step) {
    wait_vmcnt<kEarly ? kLoads / W : 0>();
    lds_barrier();
    if (kEarly || step < step1) load_step(step + (kEarly ? 2 : 1));
  };

  // K operand of 32 dims: chunk g (or 4 + g) of row c; V: see the top.
  const uint32_t k_lane = 128 * c + 16 * (g ^ swz(c));
  const uint32_t v_row = 4 * g + (c >> 2);
  const uint32_t v_lane = kKeyBytes + 128 * v_row + 16 * (((c >> 1) & 1) ^ swz(v_row)) + 8 * (c & 1);

  // Q as B operands: row c of a block of 16, eight dims from 8 g.
  bf16x8 qf[R][6];
  if (step0 < step1) {
    load_step(step0);
    if constexpr (kEarly) load_step(step0 + 1);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = tile.q0 + min(row0 + 16 * r + c, tile.rows - 1);
      const uint16_t* from = a.q + row * a.q_token + tile.h * a.q_head + 8 * g;
#pragma unroll
      for (int s = 0; s < 6; ++s) qf[r][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(from + 32 * s));
    }
  }
  before();
  f32x4 o[8][R];
  float top[R], sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = kLowest;
    sum[r] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[d][r] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  typedef const LDS_AS uint8_t* Place;
  const auto place_of = [&](int32_t step) { return (Place)lds + ((step - step0) & (kHeld - 1)) * kStepBytes; };
  // (the turned chunks' bits are below those that a step's place changes: one lane offset
  // to hold, not four)
  const auto apart = [](Place p, uint32_t bits) { return (Place)(uintptr_t)((uint32_t)(uintptr_t)p ^ bits); };
  const auto key_operand = [&](Place buf, int at, int i) {
    return *(const LDS_AS bf16x8*)(apart(buf + k_lane, 64 * (i >> 1 & 1)) + kGroupBytes * (i >> 2) + 2048 * (i & 1) + at);
  };
  const auto value_operand = [&](Place buf, int at, int d) {
    Place from = apart(buf + v_lane, 32 * (d & 3)) + kGroupBytes * (d >> 2) + at;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)from);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 LDS_AS*)(from + 2048));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // Scores of keys that a row does not see: -inf.
  const auto hide = [&](int32_t half, Scores& z) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int32_t sees = sees0 + 16 * r + c - half * kHalf - 4 * g;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) z[t][r][i] = 16 * t + i < sees ? z[t][r][i] : -INFINITY;
    }
  };
  // The row's largest score, in powers of two.
  const auto highest = [&](const Scores& z, int r) {
    float m = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = fmaxf(m, z[t][r][i]);
    m = fmaxf(m, __shfl_xor(m, 16));
    return fmaxf(m, __shfl_xor(m, 32)) * a.scale_log2;
  };
  u32x4 pf[R];  // weights of a row block: pairs of keys 4 g .. of both tiles
  // The reference moves where a lane's weights of a row pass kMost, for that row alone;
  // the turn's weights are made again.
  const auto move = [&](const Scores& z, float (&s)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float most = fmaxf(s[r], __shfl_xor(s[r], 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const float m = highest(z, r), to = most > kMost ? m + kAbove : top[r], by = __builtin_amdgcn_exp2f(top[r] - to);
      top[r] = to;
      sum[r] *= by;
#pragma unroll
      for (int d = 0; d < 8; ++d) o[d][r] *= by;
      s[r] = 0.f;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[n >> 1][r][2 * (n & 1)], a.scale_log2, -to));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[n >> 1][r][2 * (n & 1) + 1], a.scale_log2, -to));
        pf[r][n] = pack_bf16x2(p0, p1);
        s[r] += p0;
        s[r] += p1;
      }
    }
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

  // A turn: the scores of 32 keys beside the last turn's weights, then the last one's
  // product.  40 matrix instructions in a row, the softmax dealt out between them,
  // operands read kAhead before they are multiplied, in this order as written: left to
  // itself the compiler puts all of one kind together.  MASKED: some rows do not see some
  // of the keys (all of them in the turns before the first and past the last one, whose
  // weights are 0).  SECOND of a step: its first operands are here, the next step arrives
  // (kEarly).
  bf16x8 kf[12], vf[8];
  const auto turn = [&](int32_t half, Scores& z, const Scores& last, auto masked_, auto second_) {
    constexpr bool MASKED = decltype(masked_)::value, SECOND = decltype(second_)::value;
    constexpr int at = SECOND ? 4096 : 0;
    const Place here = place_of(half >> 1);
    float p0 = 0.f, p1 = 0.f, s[R];
    // weights 2 n and 2 n + 1 of the lane's 16: their first exponential and the rest
    const auto part = [&](auto k) {
      constexpr int n = decltype(k)::value >> 1, r = n >> 2, t = n >> 1 & 1, i = 2 * (n & 1);
      if constexpr ((decltype(k)::value & 1) == 0) {
        p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(last[t][r][i], a.scale_log2, -top[r]));
        p1 = __builtin_fmaf(last[t][r][i + 1], a.scale_log2, -top[r]);
      } else {
        p1 = __builtin_amdgcn_exp2f(p1);
        s[r] = (n & 3) == 0 ? p0 : s[r] + p0;
        pf[r][n & 3] = pack_bf16x2(p0, p1);
        s[r] += p1;
      }
    };
    if constexpr (!SECOND && !kEarly) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = key_operand(here, at, i);
    }
    __builtin_amdgcn_sched_barrier(0);
    static_for<12 * R>([&](auto k) {
      constexpr int n = decltype(k)::value, i = n / R, r = n % R;
      if constexpr (r == 0) {
        if constexpr (i + kAhead < 12) kf[i + kAhead] = key_operand(here, at, i + kAhead);
        else vf[i + kAhead - 12] = value_operand(here, at, i + kAhead - 12);
      }
      z[i & 1][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[r][i >> 1], i < 2 ? (f32x4){0.f, 0.f, 0.f, 0.f} : z[i & 1][r], 0, 0, 0);
      if constexpr (n % 3 != 2) part(std::integral_constant<int, n / 3 * 2 + n % 3>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__any(s[0] > kMost || s[1] > kMost)) move(last, s);
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] += s[r];
    if constexpr (SECOND && kEarly) arrive((half >> 1) + 1);
    const Place there = place_of((half >> 1) + 1);
    __builtin_amdgcn_sched_barrier(0);
    static_for<8 * R>([&](auto k) {
      constexpr int d = decltype(k)::value / R, r = decltype(k)::value % R;
      if constexpr (r == 0) {
        if constexpr (d + kAhead < 8) vf[d + kAhead] = value_operand(here, at, d + kAhead);
        else if constexpr (!SECOND) kf[d + kAhead - 8] = key_operand(here, 4096, d + kAhead - 8);
        else if constexpr (kEarly) kf[d + kAhead - 8] = key_operand(there, 0, d + kAhead - 8);
        if constexpr (MASKED) vf[d] = only_finite(vf[d]);
      }
      o[d][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], __builtin_bit_cast(bf16x8, pf[r]), o[d][r], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (MASKED) hide(half, z);
  };

  // Steps that every row of the tile sees: no masks from the second one on.
  const int32_t full = min(step1, tile.first_sees / kKeys);
  if (step0 < step1) {
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    Scores z0, z1;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) z1[t][r] = (f32x4){-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if constexpr (kEarly) {
      arrive(step0);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = key_operand(place_of(step0), 0, i);
    }
    // (the compiler waits for the queries here, not at every turn)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < 6; ++i) asm volatile("" ::"v"(qf[r][i]));
    // (the wave's last step)
    const int32_t last = mine > 2 * step0 ? mine / 2 : step0 - 1;
    int32_t step = step0;
    while (step <= last) {
      if constexpr (!kEarly) arrive(step);
      turn(2 * step, z0, z1, yes, no);
      if (step == step1) break;
      turn(2 * step + 1, z1, z0, yes, yes);
      ++step;
      for (; step < full; ++step) {
        if constexpr (!kEarly) arrive(step);
        turn(2 * step, z0, z1, no, no);
        turn(2 * step + 1, z1, z0, no, yes);
      }
    }
    after();
    for (step = last + (kEarly ? 2 : 1); step <= step1; ++step) arrive(step);  // (the other waves' steps)
    wait_vmcnt<0>();  // (nothing of this piece's lands in the next one's)
  } else {
    after();
  }
  // Values that are not finite: the masked turns' products do not have them, and where an
  // infinity met a weight that is 0 in fp32 alone (a score far below the reference, or a
  // reference that moved far later on) the others' are NaN.  A sum that is not finite,
  // unless by its row's scores, is made anew of all such values that the row sees, as they
  // are: an infinity stays one, both signs or a NaN are NaN.  (With it four short prompts take
  // 15.6 us, 15.0 without, one of 4096 rows of 128 heads 673 and 667; 32 heads of 4096 rows
  // 202, and 693 where one value of the first key is infinite.)
  float beyond[R] = {};  // NaN: a sum of the row is not finite
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int d = 0; d < 8; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) beyond[r] = __builtin_fmaf(o[d][r][i], 0.f, beyond[r]);
  if (__any(odd || beyond[0] != beyond[0] || beyond[1] != beyond[1])) {
    constexpr float kMax = __FLT_MAX__;  // in place of a sum until its infinity is found
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float l = row_sum(sum[r]);
      odd |= beyond[r] != beyond[r] && l == l;
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][r][i] = __builtin_fabsf(o[d][r][i]) <= kMax ? o[d][r][i] : copysignf(kMax, o[d][r][i]);
    }
    const auto value = [&](int32_t j, int d) { return *(const u32x2*)(v_base + (int64_t)j * a.v_token * 2 + 32 * d + 8 * g); };
    const int32_t to = __any(odd) ? min(mine * kHalf, tile.keys) : 0;
    // sixteen keys at a time are looked at, one a lane c
#pragma unroll 1
    for (int32_t j0 = step0 * kKeys; j0 < to; j0 += 16) {
      bool has = false;
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const u32x2 v = value(min(j0 + c, to - 1), d);
#pragma unroll
        for (int i = 0; i < 2; ++i) has |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
      }
      const uint64_t lanes = __ballot(has);
      uint32_t keys = (uint32_t)(lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffffu;
#pragma unroll 1
      for (; keys; keys &= keys - 1) {
        const int32_t j = j0 + __builtin_ctz(keys);
        if (j >= to) break;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          const u32x2 v = value(j, d);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bits = i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16;
#pragma unroll
            for (int r = 0; r < R; ++r)
              if ((bits & 0x7f800000u) == 0x7f800000u && j < sees0 + 16 * r + c) o[d][r][i] += __builtin_bit_cast(float, bits);
          }
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)  // (no infinity: finite products past fp32's range)
          if (__builtin_fabsf(o[d][r][i]) == kMax) o[d][r][i] = copysignf(INFINITY, o[d][r][i]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    p.top[r] = top[r];
    p.sum[r] = sum[r];
#pragma unroll
    for (int d = 0; d < 8; ++d) p.o[d][r] = o[d][r];
  }
}

__device__ __forceinline__ void write_rows(const MlaPrefillLaunch& a, const Tile& tile, const Piece& p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int r = 0; r < kBlocks; ++r) {
    const int32_t row = kWaveRows * wave + 16 * r + c;
    const float l = row_sum(p.sum[r]);
    if (row >= tile.rows) continue;
    const float by = 1.f / l;
    const int64_t n = (tile.q0 + row) * a.heads + tile.h;
    // Lanes g = 0, 1 and 2, 3 exchange halves of two neighbouring blocks of 16 values:
    // eight in a row for each, 64 bytes of a row a store.
    uint16_t* to = a.out + n * kValue + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
    for (int d = 0; d < 8; d += 2) {
      u32x2 v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x4 x = l == 0.f ? (f32x4){0.f, 0.f, 0.f, 0.f} : p.o[d + k][r] * by;
        v[k] = (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      }
      const auto lo = __builtin_amdgcn_permlane16_swap(v[0][0], v[1][0], false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(v[0][1], v[1][1], false, false);
      *(u32x4*)(to + 16 * d) = (u32x4){lo[0], hi[0], lo[1], hi[1]};
    }
    if (a.lse && g == 0) a.lse[n] = natural_lse(p.top[r], l);
  }
}
template <int W>
__device__ __forceinline__ void write_part(const MlaPrefillLaunch& a, const Tile& tile, const Piece& p, int32_t slot) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int r = 0; r < kBlocks; ++r) {
    const int32_t row = kWaveRows * wave + 16 * r + c;
    const float l = row_sum(p.sum[r]);
    if (row >= tile.rows) continue;
    float* to = a.part_out + ((int64_t)slot * tile_rows(W) + row) * kValue + 4 * g;
#pragma unroll
    for (int d = 0; d < 8; ++d) *(f32x4*)(to + 16 * d) = p.o[d][r];
    if (g == 0) *(f32x2*)(a.part_ml + ((int64_t)slot * tile_rows(W) + row) * 2) = (f32x2){p.top[r], l};
  }
}

// Workers of the line: all that fit on the chip, or as many as get kLeast steps.
__device__ __forceinline__ int32_t line_workers(const MlaPrefillLaunch& a, const Call& call) {
  const int64_t most = call.steps * a.heads / (kStep * kLeast) / 8 * 8;
  return (int32_t)min(max(most, (int64_t)8), (int64_t)a.workers);
}
// Whether the tiles are cut: where the longest one takes longer than all of them over the chip.
__device__ __forceinline__ bool is_cut(const MlaPrefillLaunch& a, const Call& call) {
  return call.longest > kNeverCut && call.steps <= kLongest &&
         (int64_t)kStep * call.longest * a.workers > (call.steps + (int64_t)kStep * call.tiles) * a.heads;
}

// Worker w's piece of the line: of tile `i` of a request.
__device__ __forceinline__ int64_t span_at(int64_t length, int32_t workers, int64_t k) {
  return length / workers * k + length % workers * k / workers;
}
struct Span {
  Request r;
  int32_t i, h;
  int64_t begin, tile_end, end;  // the tile's place on the line, its end, the worker's end
  int64_t line;                  // a head's
  int32_t cost, workers;         // a tile's cost on it, and who shares it
  int32_t step0, step1;
  bool begins, ends;  // the piece begins or ends its tile
};
// From place on; tile and its begin are known.
template <int ROWS>
__device__ __forceinline__ void cut_piece(Span& s, int64_t place) {
  const Tile t = tile_of<ROWS>(s.r, s.h, s.i);
  s.tile_end = s.begin + line_tile<ROWS>(s.r, s.i, s.cost);
  // the tile's cost comes first on the line, and steps that it lacks last
  const int32_t steps = (t.keys + kKeys - 1) / kKeys, each = line_step<ROWS>(s.r, s.i);
  const auto step_at = [&](int64_t at) { return min(max((int32_t)(at - s.begin) - s.cost, 0) / each, steps); };
  s.begins = place == s.begin;
  s.ends = s.tile_end <= s.end;
  s.step0 = step_at(place);
  s.step1 = s.ends ? steps : step_at(s.end);
}
template <int ROWS>
__device__ __forceinline__ void find_piece(const MlaPrefillLaunch& a, Span& s, int64_t place) {
  s.h = (int32_t)(place / s.line);
  s.r = Request{0, 0, 0, 0};
  s.i = 0;
  s.begin = 0;
  find_place<ROWS>(a, s.cost, place - s.h * s.line, s.r, s.i, s.begin);
  s.begin += s.h * s.line;
  cut_piece<ROWS>(s, place);
}
// The worker's first piece, and the one after s: the request's next tile, as long as it has one.
template <int ROWS>
__device__ __forceinline__ Span first_piece(const MlaPrefillLaunch& a, int32_t w) {
  const Call call = look_at<ROWS>(a);
  Span s;
  s.workers = line_workers(a, call);
  // (not more than a quarter of a worker's steps)
  s.cost = (int32_t)min((int64_t)kTileCost, call.steps * a.heads / (4 * s.workers));
  s.line = call.steps + (int64_t)call.tiles * s.cost;
  s.end = span_at(s.line * a.heads, s.workers, w + 1);
  find_piece<ROWS>(a, s, span_at(s.line * a.heads, s.workers, w));
  return s;
}
template <int ROWS>
__device__ __forceinline__ void next_piece(const MlaPrefillLaunch& a, Span& s) {
  if (s.i + 1 < tiles_of<ROWS>(s.r.nq)) {
    ++s.i;
    s.begin = s.tile_end;
    cut_piece<ROWS>(s, s.begin);
  } else {
    find_piece<ROWS>(a, s, s.tile_end);
  }
}
// What is needed of it behind the loops, in the lanes of one register.
__device__ __forceinline__ int32_t in_lanes(const Span& s, int lane) {
  const int32_t told[15] = {s.r.q0, s.r.nq, s.r.k0, s.r.nk, s.i, s.h, (s.begins ? 1 : 0) | (s.ends ? 2 : 0),
                            (int32_t)s.tile_end, (int32_t)(s.tile_end >> 32), (int32_t)s.end, (int32_t)(s.end >> 32),
                            (int32_t)s.line, (int32_t)(s.line >> 32),
                            s.cost, s.workers};
  int32_t v = 0;
#pragma unroll
  for (int k = 0; k < 15; ++k) v = lane == k ? told[k] : v;
  return v;
}
__device__ __forceinline__ Span of_lanes(int32_t v) {
  const auto wide = [&](int k) { return (int64_t)((uint64_t)(uint32_t)uniform(v, k + 1) << 32 | (uint32_t)uniform(v, k)); };
  Span s = {};
  s.r = Request{uniform(v, 0), uniform(v, 1), uniform(v, 2), uniform(v, 3)};
  s.i = uniform(v, 4);
  s.h = uniform(v, 5);
  s.begins = uniform(v, 6) & 1;
  s.ends = uniform(v, 6) & 2;
  s.tile_end = wide(7);
  s.end = wide(9);
  s.line = wide(11);
  s.cost = uniform(v, 13);
  s.workers = uniform(v, 14);
  return s;
}

// What the tiles' order is looked up in: the block of every rank; `blocks` of them.
// a.tiles lies where a cut call's parts do.
struct Block {
  Request r;
  int32_t block;  // of its request, from the last one on
  int32_t none[3];
};
static_assert(sizeof(Block) == kPrefillBlock, "the workspace's");
// One wave a rank; past the requests that are ordered, one workgroup for all requests.
template <int ROWS>
__global__ __launch_bounds__(kThreads) void mla_prefill_order_kernel(MlaPrefillLaunch a, int32_t shift, int32_t blocks) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Block* to = (Block*)a.tiles;
  if (blockIdx.x == 0 && threadIdx.x < 8) a.tickets[32 * threadIdx.x] = 0;
  if (a.B <= 64 * kSorted) {
    const int32_t rank = (int32_t)blockIdx.x * (kThreads / 64) + wave;
    if (rank >= blocks) return;
    Block b = {};
    if (!find_block<ROWS>(a, true, rank, shift, b.r, b.block)) b.r.nq = 0;
    if (lane == 0) to[rank] = b;
    return;
  }
  __shared__ int32_t sums[kThreads / 64];
  int64_t behind = 0;
  for (int32_t b0 = 0; b0 < a.B && behind < blocks; b0 += kThreads) {
    const int32_t at = b0 + (int32_t)threadIdx.x;
    const Request r = request(a, min(at, a.B - 1));
    const int32_t own = at < a.B ? (tiles_of<ROWS>(r.nq) + (1 << shift) - 1) >> shift : 0, upto = wave_prefix(own);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int64_t first = behind + upto - own;
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) {
      if (k < wave) first += sums[k];
      behind += sums[k];
    }
    __syncthreads();
    for (int32_t k = 0; k < own && first + k < blocks; ++k) to[first + k] = Block{r, k, {}};
  }
  for (int64_t k = behind + threadIdx.x; k < blocks; k += kThreads) to[k] = Block{};
}

// Whole tiles, or the line of all tiles in equal spans.  A workgroup takes one tile, or
// (where there are more than the chip holds, with a.tickets) one after the other: a new
// workgroup would begin 10 us after the last one's end on its compute unit, with nothing
// on the way.  The first wave, whose rows see the fewest keys, finds the next tile while
// the others still multiply; its first step and queries are loaded before the last
// tile's rows are written.
template <int W>
__global__ __launch_bounds__(64 * W, 2) void mla_prefill_kernel(MlaPrefillLaunch a, int32_t shift, int32_t blocks) {
  __shared__ __align__(128) uint8_t lds[steps_held(W) * kStepBytes];
  constexpr int ROWS = tile_rows(W);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int32_t xcd = blockIdx.x & 7;  // (workgroups go round the 8 XCDs)
  int32_t w = -1;                      // the worker on the line (-1: whole tiles)
  Tile tile = {0, 0, 0, 0, 0, 0}, last = tile;
  if (a.joined) {
    const Call call = look_at<ROWS>(a);
    if (is_cut(a, call)) {
      const int32_t each = line_workers(a, call) / 8, at = blockIdx.x >> 3;
      if (at < each) w = xcd * each + at;  // neighbours on the line on one XCD
    }
    const uint32_t own = w < 0 ? blockIdx.x : w;
    if (own < (uint32_t)a.workers && threadIdx.x == 0) a.joined[own] = make_int4(-1, 0, 0, 0);
    if (w < 0 && is_cut(a, call)) return;
  }
  // Groups of 2^shift tiles of a head, neighbours of one XCD that begin together and
  // read the same keys; the longest groups first, of all heads.  False: there is no tile
  // at this place of the XCD's; rank: its block's.
  const auto tile_at = [&](int32_t at, const Request& r, int32_t block, Tile& t) {
    const int32_t i = tiles_of<ROWS>(r.nq) - 1 - (block << shift) - (at & ((1 << shift) - 1));
    if (i < 0) return false;
    t = tile_of<ROWS>(r, (int32_t)(((int64_t)(at >> shift) * 8 + xcd) % a.heads), i);
    return true;
  };
  const auto rank_of = [&](int32_t at) { return ((int64_t)(at >> shift) * 8 + xcd) / a.heads; };
  if (w < 0 && !a.tickets) {
    Request r;
    int32_t block;
    const int32_t at = blockIdx.x >> 3;
    if (!find_block<ROWS>(a, gridDim.x > (uint32_t)a.units, (int32_t)rank_of(at), shift, r, block) || !tile_at(at, r, block, tile)) return;
  }
  // The next tile, in lanes: rows (0: there are no more), q0, k0, first_sees, keys, h; or
  // the piece of the line that is worked on.
  volatile int32_t kept;  // (in memory: the loops have no register for it)
  bool first = true;
  const auto find = [&] {
    int32_t told[6] = {};
    while (true) {
      const MlaPrefillLaunch a = arguments();
      int32_t at = blockIdx.x >> 3;
      if (!first) {
        int32_t ticket = 0;
        if (lane == 0) ticket = __hip_atomic_fetch_add(a.tickets + 32 * xcd, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        at = (int32_t)(gridDim.x >> 3) + __builtin_amdgcn_readfirstlane(ticket);
      }
      first = false;
      const int64_t rank = rank_of(at);
      if (rank >= blocks) break;
      const Block b = ((const Block*)a.tiles)[rank];
      if (b.r.nq == 0) break;
      Tile t;
      if (!tile_at(at, b.r, b.block, t)) continue;
      told[0] = t.rows;
      told[1] = (int32_t)t.q0;
      told[2] = (int32_t)t.k0;
      told[3] = t.first_sees;
      told[4] = t.keys;
      told[5] = t.h;
      break;
    }
    int32_t found = 0;
#pragma unroll
    for (int k = 0; k < 6; ++k) found = lane == k ? told[k] : found;
    kept = found;
  };
  int32_t step0 = 0, step1 = (tile.keys + kKeys - 1) / kKeys;
  Span span = {};
  if (w >= 0) span = first_piece<ROWS>(arguments(), w);
  Piece p;
  while (true) {
    if (w >= 0) {
      kept = in_lanes(span, lane);
      tile = tile_of<ROWS>(span.r, span.h, span.i);
      step0 = span.step0;
      step1 = span.step1;
    }
    attend<W>(
        arguments(), tile, step0, step1, lds, p,
        [&] {
          if (last.rows > 0) write_rows(arguments(), last, p);
        },
        [&] {
          if (w < 0 && wave == 0 && a.tickets) find();
        });
    if (w < 0) {
      const MlaPrefillLaunch b = arguments();
      last = tile;
      if (b.tickets) {
        int32_t* told = (int32_t*)(lds + (steps_held(W) - 1) * kStepBytes);  // (the next first steps go elsewhere)
        lds_barrier();  // nobody reads keys any more
        if (wave == 0 && lane < 6) told[lane] = kept;
        lds_barrier();
        const int4 t0 = *(const int4*)told;
        const int2 t1 = *(const int2*)(told + 4);
        tile = Tile{uniform(t1.y, 0), uniform(t0.x, 0), uniform(t0.y, 0), uniform(t0.z, 0), uniform(t0.w, 0), uniform(t1.x, 0)};
        step1 = (tile.keys + kKeys - 1) / kKeys;
        if (tile.rows > 0) continue;
      }
      if (last.rows > 0) write_rows(b, last, p);
      return;
    }
    const MlaPrefillLaunch b = arguments();
    span = of_lanes(kept);
    const Tile t = tile_of<ROWS>(span.r, span.h, span.i);
    if (span.begins && span.ends) {
      write_rows(b, t, p);
    } else {
      write_part<W>(b, t, p, 2 * w + (span.begins ? 1 : 0));
      if (span.begins) {
        // the parts of this tile: this one, and one of each worker up to its end
        int32_t upto = w + 1;
        while (span_at(span.line * b.heads, span.workers, upto + 1) < span.tile_end) ++upto;
        if (threadIdx.x == 0) b.joined[w] = make_int4((int32_t)t.q0, t.rows, t.h, upto - w + 1);
      }
    }
    if (span.tile_end >= span.end) return;
    next_piece<ROWS>(b, span);
    lds_barrier();  // nobody reads this piece's keys any more
  }
}

// The parts of the tile that worker blockIdx.x begins, 16 rows a workgroup: sixteen
// lanes a row, eight values each.
template <int ROWS>
__global__ __launch_bounds__(kThreads) void mla_prefill_join_kernel(MlaPrefillLaunch a) {
  const int32_t w = blockIdx.x;
  const int4 record = a.joined[w];
  const int32_t row = blockIdx.y * 16 + (threadIdx.x >> 4), lane = threadIdx.x & 15;
  if (record.x < 0 || row >= record.y) return;
  const auto slot = [&](int32_t k) { return ((int64_t)(k == 0 ? 2 * w + 1 : 2 * (w + k)) * ROWS + row); };
  float top = kLowest, sum = 0.f;
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  // N parts, their loads at once (a part without a weight holds zeros)
  const auto join = [&](int32_t k0, auto n_) {
    constexpr int N = decltype(n_)::value;
    f32x2 ml[N];
    f32x4 v[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t at = slot(min(k0 + i, record.w - 1));
      ml[i] = *(const f32x2*)(a.part_ml + at * 2);
      v[i][0] = *(const f32x4*)(a.part_out + at * kValue + 8 * lane);
      v[i][1] = *(const f32x4*)(a.part_out + at * kValue + 8 * lane + 4);
    }
    float to = top;
#pragma unroll
    for (int i = 0; i < N; ++i) to = ml[i][0] > to || ml[i][0] != ml[i][0] ? ml[i][0] : to;
    const float old = __builtin_amdgcn_exp2f(top - to);
    top = to;
    sum *= old;
    lo *= old;
    hi *= old;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (k0 + i >= record.w) break;
      const float by = __builtin_amdgcn_exp2f(ml[i][0] - to);
      sum += by * ml[i][1];
      lo += by * v[i][0];
      hi += by * v[i][1];
    }
  };
  int32_t k = 0;
  for (; k + 8 < record.w; k += 16) join(k, std::integral_constant<int, 16>{});
  for (; k < record.w; k += 4) join(k, std::integral_constant<int, 4>{});
  const int64_t n = (int64_t)(record.x + row) * a.heads + record.z;
  float beyond = 0.f;  // NaN: a sum is not finite
#pragma unroll
  for (int i = 0; i < 4; ++i) beyond = __builtin_fmaf(lo[i], 0.f, __builtin_fmaf(hi[i], 0.f, beyond));
  if (beyond != beyond) {
    // those sums of the parts' own infinities, as they are: a part's weight may be 0 in fp32
    f32x4 of_lo = {0.f, 0.f, 0.f, 0.f}, of_hi = of_lo;
    const auto infinite = [](float x) { return !(__builtin_fabsf(x) < INFINITY); };
    for (k = 0; k < record.w; ++k) {
      const f32x4* from = (const f32x4*)(a.part_out + slot(k) * kValue + 8 * lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        of_lo[i] += infinite(from[0][i]) ? from[0][i] : 0.f;
        of_hi[i] += infinite(from[1][i]) ? from[1][i] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (infinite(lo[i]) && of_lo[i] != 0.f) lo[i] = of_lo[i];
      if (infinite(hi[i]) && of_hi[i] != 0.f) hi[i] = of_hi[i];
    }
  }
  if (sum == 0.f) lo = hi = (f32x4){0.f, 0.f, 0.f, 0.f};
  const float by = sum == 0.f ? 0.f : 1.f / sum;
  lo *= by;
  hi *= by;
  *(u32x4*)(a.out + n * kValue + 8 * lane) =
      (u32x4){pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
  if (a.lse && lane == 0) a.lse[n] = natural_lse(top, sum);
}

template <int W>
hipError_t launch_tiles(const MlaPrefillLaunch& a, bool small, hipStream_t s) {
  constexpr int kRows = tile_rows(W);
  MlaPrefillLaunch l = a;
  const int32_t workers = (W == 8 ? 1 : 2) * a.units / 8 * 8;
  l.workers = workers < 8 ? 8 : workers > kPrefillParts / kRows ? kPrefillParts / kRows : workers;
  // Tiles of a request that are placed together: as many as an average request has, at most 4.
  const int64_t rows_each = a.num_rows / a.B;
  const int shift = rows_each >= 4 * kRows ? 2 : rows_each >= 2 * kRows ? 1 : 0;
  // no request adds more than one block that is not full
  const int64_t blocks = min((int64_t)a.num_rows / (kRows << shift) + a.B, (int64_t)a.num_rows);
  int64_t groups = (blocks * a.heads + 7) / 8 * 8 << shift;
  if (a.num_keys <= kNeverCut * kKeys) l.joined = nullptr;
  else groups = max(groups, (int64_t)l.workers);
  if (groups > (small ? 4 : 1) * (int64_t)l.workers) {
    groups = l.workers;
    const int64_t waves = a.B <= 64 * kSorted ? blocks : 1;
    hipLaunchKernelGGL((mla_prefill_order_kernel<kRows>), dim3((unsigned)((waves + kThreads / 64 - 1) / (kThreads / 64))), dim3(kThreads), 0, s,
                       l, shift, (int32_t)blocks);
  } else {
    l.tickets = nullptr;
  }
  hipLaunchKernelGGL((mla_prefill_kernel<W>), dim3((unsigned)groups), dim3(64 * W), 0, s, l, shift, (int32_t)blocks);
  if (l.joined) hipLaunchKernelGGL((mla_prefill_join_kernel<kRows>), dim3((unsigned)l.workers, kRows / 16), dim3(kThreads), 0, s, l);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mla_prefill(const MlaPrefillLaunch& a, hipStream_t s) {
  // From the call's averages: W = 8 where tiles will be cut or see 40 steps or more on
  // average.  Measured (us, W = 4 / 8), cut: 8 heads of 16,384 rows 623 / 562, 20 of 2 x 512
  // rows over 8192 keys 161 / 141, of 8 x 200 over 4000 183 / 141; long: 128 of 6144 rows
  // 1,496 / 1,463, 32 of 8 x 1024 over 4096 777 / 709; else: 128 of 4096 rows 701 / 699, 32
  // of 4 x 1024 89 / 101, 16 of 64 x 200 95 / 108.
  const int64_t rows = max((int64_t)a.num_rows / a.B, (int64_t)1), keys = max((int64_t)a.num_keys / a.B, rows);
  const int64_t steps = (keys - rows / 2) / kKeys, tiles = (rows + 127) / 128 * a.B * a.heads;
  const bool cut = keys > kNeverCut * kKeys && keys / kKeys * 2 * a.units > tiles * steps;
  if (cut || steps >= 40) return launch_tiles<8>(a, false, s);
  // A workgroup each for a few short tiles: they are over before the order's launch is made
  // up for (us, a workgroup each / one after the other: 32 heads of 34 x 18 rows 28 / 32, 8 of
  // 100 x 60 34 / 38; but with more than four for each that stays 128 of 64 x 8 132 / 130, 64
  // of 10 x 500 153 / 150, 16 of 64 x 250 108 / 110).
  return launch_tiles<4>(a, keys < 384, s);
}

}  // namespace splash
