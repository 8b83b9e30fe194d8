// Internal launch interface of the serving step around grouped-query attention.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "splash_common.hpp"

namespace splash {

constexpr int32_t kMaxTableBatch = 8192;  // splash_step_tables keeps two offsets per request in LDS
constexpr int32_t kMaxRopePairs = 128;

struct TablesLaunch {
  const int32_t* seq_lens;
  const int32_t* new_lens;  // nullptr: q_chunk each
  int32_t q_chunk, B;
  const int32_t* free_pages;
  int32_t num_free;
  const int32_t* taken_in;
  int32_t* taken_out;
  int32_t* block_table;
  int32_t max_pages, num_pages, max_tokens;
  int32_t* new_indptr;
  int32_t* slots;
  int32_t* positions;
  int32_t* requests;
};

struct RopeView {
  const uint16_t* x;
  uint16_t* y;
  int64_t x_token, x_head, y_token, y_head;  // strides in elements
  int32_t heads;
};

// Travels by value: the frequencies and axes sit in the kernel's arguments.
struct RopeLaunch {
  RopeView view[2];
  const int32_t* positions;
  int64_t position_stride;
  int32_t num_views, num_tokens, pairs, interleaved;
  float scale;
  double turns[kMaxRopePairs];   // inv_freq / (2 pi): turns per position
  uint8_t axis[kMaxRopePairs];
};

struct GqaAppendLaunch {
  const uint16_t* k_new;
  const uint16_t* v_new;
  int64_t token_stride, head_stride;
  const int32_t* slots;
  int32_t num_tokens, batch, Hk, D, num_pages, code_type;
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;
  float* v_scales;
};

struct GqaAttendLaunch {
  const uint16_t* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  uint16_t* out;
  float* lse;
  int32_t B, Hk, group, D, q_chunk, bt_stride, num_pages, code_type;
  float scale_log2;  // softmax_scale * log2(e)
  bool whole_tiles;  // no tile is cut between workgroups
  int32_t workers;   // compute units; the launch makes it workgroups, at most kGqaMaxWorkers
  // workspace: two partial results per workgroup, of gqa_tile_rows() rows,
  // and {request, KV head, row block, parts} of the tile it begins (request -1: none)
  int4* joined;      // [workers]
  float* part_ml;    // [2 workers, rows, 2] reference and sum of a row
  float* part_out;   // [2 workers, rows, D]
};

constexpr int32_t kGqaMaxWorkers = 512;
constexpr int32_t kGqaTileCost = 2;  // a tile's fixed work, in steps of its waves

// Query rows of a tile, for `rows` of them per KV head: the fewest that hold
// them, at most 128 (64 at 256 dims, whose accumulators take twice the registers).
inline int32_t gqa_tile_rows(int32_t D, int64_t rows) {
  return rows <= 16 ? 16 : rows <= 32 ? 32 : (rows <= 64 || D == 256) ? 64 : 128;
}

hipError_t launch_step_tables(const TablesLaunch& p, hipStream_t s);
hipError_t launch_rope(const RopeLaunch& p, hipStream_t s);
hipError_t launch_gqa_append(const GqaAppendLaunch& p, hipStream_t s);
hipError_t launch_gqa_attend(const GqaAttendLaunch& p, hipStream_t s);

}  // namespace splash
