// Internal launch interface of the latent-attention layer around the cache.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "splash_common.hpp"

namespace splash {

constexpr int kNope = 128;            // no-position dims of a head's query and key
constexpr int kRope = 64;             // rotary dims
constexpr int kValue = 128;           // a head's value
constexpr int kRopePairs = kRope / 2;

// The rotary turn of 64 dims; travels by value.
struct TurnLaunch {
  const int32_t* positions;   // nullptr: rows are taken as they are
  int64_t position_stride;
  int32_t axes;               // 1: axis is all 0
  int32_t interleaved;
  float scale;
  double turns[kRopePairs];   // inv_freq / (2 pi): turns per position
  uint8_t axis[kRopePairs];
};

struct MlaAppendLaunch {
  const uint16_t* latent;
  const uint16_t* key;
  int64_t latent_stride, key_stride;
  const uint16_t* norm_weight;  // nullptr: no norm
  float norm_eps;
  const int32_t* slots;
  int32_t num_tokens, num_pages, kv_dtype;
  uint8_t* pages;
  float* scales;
  TurnLaunch turn;
};

struct MlaGatherLaunch {
  const uint8_t* pages;
  const float* scales;
  const int32_t* block_table;
  const int32_t* key_begin;  // nullptr: 0
  const int32_t* row_indptr;
  int32_t B, bt_stride, num_pages, max_rows, kv_dtype;
  uint16_t* latent;
  uint16_t* key;
  int64_t latent_stride, key_stride;
};

struct MlaAbsorbLaunch {
  const uint16_t* q;
  int64_t q_token, q_head;
  const uint16_t* w;
  int64_t w_head, w_row;
  int32_t num_tokens, heads;
  uint16_t* out;
  TurnLaunch turn;
};

struct MlaExpandLaunch {
  const uint16_t* x;
  const uint16_t* w;
  int64_t w_head, w_row;
  int32_t num_tokens, heads;
  uint16_t* y;
  int64_t y_token, y_head;
};

struct MlaPrefillLaunch {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* key;
  const uint16_t* v;
  int64_t q_token, q_head, k_token, k_head, key_token, v_token, v_head;
  const int32_t* q_indptr;
  const int32_t* kv_indptr;
  int32_t B, num_rows, num_keys, heads;
  float scale_log2;  // softmax_scale * log2(e)
  uint16_t* out;
  float* lse;
  int32_t units;     // compute units
  int32_t workers;   // (made by the launch) workgroups that the chip holds
  // workspace: the next place of each XCD's tiles (nullptr: a workgroup takes one tile),
  // two partial results per worker, and {first row, rows, head, parts} of
  // the tile that it begins and does not end (first row -1: none)
  int32_t* tickets;  // [8], 128 bytes apart
  int4* joined;      // [workers]
  float* part_ml;    // [2 workers, a tile's rows, 2] reference and sum of a row
  float* part_out;   // [2 workers, a tile's rows, 128]
  void* tiles;       // the tiles' order where none is cut: kPrefillBlock bytes a block, over the parts
};

constexpr int32_t kPrefillWorkers = 512;
constexpr int32_t kPrefillParts = 512 * 128;  // workers times a tile's rows, at most
constexpr int32_t kPrefillBlock = 32;

hipError_t launch_mla_append(const MlaAppendLaunch& a, hipStream_t s);
hipError_t launch_mla_gather(const MlaGatherLaunch& a, hipStream_t s);
hipError_t launch_mla_absorb(const MlaAbsorbLaunch& a, hipStream_t s);
hipError_t launch_mla_expand(const MlaExpandLaunch& a, hipStream_t s);
hipError_t launch_mla_prefill(const MlaPrefillLaunch& a, hipStream_t s);

}  // namespace splash
