// C-ABI of the serving step around grouped-query attention: argument checks
// and the entry points declared in include/splash_attn.h.  No C++ exception
// crosses this boundary.
#include "splash_attn.h"

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>

#include "errors.hpp"
#include "step.hpp"

using namespace splash;

namespace {

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int32_t kMaxPoolPages = 1 << 25;  // a slot (64 * page + place) fits int32
// A launch holds less than 2^32 lanes: 64 a token, or a token and KV head.
constexpr int32_t kMaxRopeTokens = 1 << 25;
constexpr int64_t kMaxAppendRows = 1 << 25;

int validate_gqa(const splash_gqa_desc* d) {
  if (!d) return fail(SPLASH_ERR_INVALID_ARGUMENT, "desc is NULL");
  if (d->batch < 0) return fail(SPLASH_ERR_INVALID_ARGUMENT, "batch < 0");
  if (d->page_size != kPage) return fail(SPLASH_ERR_UNSUPPORTED, "page_size must be 64 (got %d)", d->page_size);
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
    return fail(SPLASH_ERR_UNSUPPORTED, "head_dim must be 64, 128 or 256 (got %d)", d->head_dim);
  if (d->num_kv_heads < 1 || d->num_kv_heads > 128 || d->num_heads < 1 || d->num_heads > 1024 ||
      d->num_heads % d->num_kv_heads)
    return fail(SPLASH_ERR_UNSUPPORTED,
                "num_heads must be a multiple of num_kv_heads, at most 1024, with 1 <= num_kv_heads <= 128 (got %d, %d)",
                d->num_heads, d->num_kv_heads);
  if (d->code_type != SPLASH_GQA_E4M3 && d->code_type != SPLASH_GQA_INT8)
    return fail(SPLASH_ERR_UNSUPPORTED, "unknown code_type %d", d->code_type);
  if (d->max_pages_per_seq < 1 || d->num_pages < 1)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "max_pages_per_seq and num_pages must be >= 1");
  if (d->num_pages > kMaxPoolPages)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_pages must be at most 2^25 (got %d)", d->num_pages);
  if (d->max_pages_per_seq > INT32_MAX / kPage)  // (positions are int32)
    return fail(SPLASH_ERR_UNSUPPORTED, "max_pages_per_seq must be at most 2^25 - 1 (got %d)", d->max_pages_per_seq);
  if (!(std::isfinite(d->softmax_scale) && d->softmax_scale > 0.f))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "softmax_scale must be finite and > 0");
  return SPLASH_OK;
}

int check_gqa_cache(const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales) {
  if (!k_pages || !v_pages || !k_scales || !v_scales)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "k_pages, v_pages, k_scales and v_scales must be non-NULL");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16))
    return fail(SPLASH_ERR_MISALIGNED, "k_pages and v_pages must be 16-byte aligned");
  if (!aligned(k_scales, 4) || !aligned(v_scales, 4))
    return fail(SPLASH_ERR_MISALIGNED, "k_scales and v_scales must be 4-byte aligned");
  return SPLASH_OK;
}

// Whether two of a view's rows, `width` elements at n * token + h * head, share
// an element.  Rows n tokens apart in one direction and h heads in the other lie
// |h * head - n * token| apart; of each h the two nearest n decide.
bool rows_overlap(int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t width) {
  if ((tokens > 1 && token < width) || (heads > 1 && head < width)) return true;
  if (tokens < 2 || heads < 2) return false;
  typedef __int128 Wide;
  if ((Wide)token >= (Wide)(heads - 1) * head + width || (Wide)head >= (Wide)(tokens - 1) * token + width) return false;
  for (int64_t h = 1; h < heads; ++h) {
    const Wide at = (Wide)h * head, n = at / token, past = at - n * token;
    if (n >= tokens) return false;
    if (past < width || (n + 1 < tokens && token - past < width)) return true;
  }
  return false;
}

struct GqaLayout {
  size_t part_ml, part_out, total;  // the joined tiles' records come first
};

GqaLayout gqa_layout(const splash_gqa_desc* d, int32_t q_chunk) {
  const int64_t rows = gqa_tile_rows(d->head_dim, (int64_t)q_chunk * (d->num_heads / d->num_kv_heads));
  const size_t slots = 2 * (size_t)kGqaMaxWorkers * rows;
  GqaLayout l;
  l.part_ml = sizeof(int4) * kGqaMaxWorkers;
  l.part_out = l.part_ml + slots * 2 * sizeof(float);
  l.total = l.part_out + slots * d->head_dim * sizeof(float);
  return l;
}

}  // namespace

extern "C" {

int splash_step_tables(const int32_t* seq_lens, const int32_t* new_lens, int32_t q_chunk, int32_t batch,
                       const int32_t* free_pages, int32_t num_free, const int32_t* taken_in, int32_t* taken_out,
                       int32_t* block_table, int32_t max_pages_per_seq, int32_t num_pages, int32_t max_tokens,
                       int32_t* new_indptr, int32_t* slots, int32_t* positions, int32_t* requests, void* stream) {
  if (batch < 0 || max_tokens < 0 || num_free < 0 || q_chunk < 0 || max_pages_per_seq < 1 || num_pages < 1)
    return fail(SPLASH_ERR_INVALID_ARGUMENT,
                "need batch, max_tokens, num_free and q_chunk >= 0, max_pages_per_seq and num_pages >= 1");
  if (batch > kMaxTableBatch) return fail(SPLASH_ERR_UNSUPPORTED, "batch must be at most %d (got %d)", kMaxTableBatch, batch);
  if (num_pages > kMaxPoolPages)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_pages must be at most 2^25 (got %d)", num_pages);
  if ((int64_t)max_pages_per_seq * kPage * (batch > 0 ? batch : 1) > INT32_MAX)
    return fail(SPLASH_ERR_UNSUPPORTED, "64 * max_pages_per_seq * batch passes 2^31 - 1");
  if (!taken_in || !taken_out || !new_indptr || (batch > 0 && (!seq_lens || !block_table)) ||
      (num_free > 0 && !free_pages) || (max_tokens > 0 && (!slots || !positions || !requests)))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "NULL buffer");
  const void* ints[] = {seq_lens, new_lens, free_pages, taken_in, taken_out, block_table, new_indptr, slots, positions, requests};
  for (const void* p : ints)
    if (!aligned(p, 4)) return fail(SPLASH_ERR_MISALIGNED, "int32 buffers must be 4-byte aligned");
  const uintptr_t in = reinterpret_cast<uintptr_t>(taken_in), out = reinterpret_cast<uintptr_t>(taken_out);
  if ((in < out ? out - in : in - out) < 2 * sizeof(int32_t))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "taken_out must not overlap taken_in");
  const TablesLaunch t = {seq_lens,  new_lens,    q_chunk,           batch,     free_pages, num_free,   taken_in,  taken_out,
                          block_table, max_pages_per_seq, num_pages, max_tokens, new_indptr, slots,     positions, requests};
  const hipError_t e = launch_step_tables(t, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "step tables launch");
}

int splash_rope(const splash_rope_view* views, int32_t num_views, const int32_t* positions, int64_t position_stride,
                int32_t num_tokens, const splash_rope_desc* desc, void* stream) {
  if (!views || !desc || !desc->inv_freq) return fail(SPLASH_ERR_INVALID_ARGUMENT, "views, desc and inv_freq must be non-NULL");
  if (num_views < 1 || num_views > 2) return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_views must be 1 or 2 (got %d)", num_views);
  if (num_tokens < 0) return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_tokens < 0");
  if (num_tokens > kMaxRopeTokens) return fail(SPLASH_ERR_UNSUPPORTED, "num_tokens must be at most 2^25 (got %d)", num_tokens);
  if (desc->rot_dim < 2 || desc->rot_dim > 2 * kMaxRopePairs || desc->rot_dim % 2)
    return fail(SPLASH_ERR_UNSUPPORTED, "rot_dim must be even, 2 .. %d (got %d)", 2 * kMaxRopePairs, desc->rot_dim);
  if (desc->num_axes < 1 || desc->num_axes > 4)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_axes must be 1 .. 4 (got %d)", desc->num_axes);
  if (!std::isfinite(desc->scale)) return fail(SPLASH_ERR_INVALID_ARGUMENT, "scale is not finite");
  RopeLaunch r = {};
  r.positions = positions;
  r.position_stride = position_stride;
  r.num_views = num_views;
  r.num_tokens = num_tokens;
  r.pairs = desc->rot_dim / 2;
  r.interleaved = desc->interleaved ? 1 : 0;
  r.scale = desc->scale;
  for (int32_t j = 0; j < r.pairs; ++j) {
    if (!std::isfinite(desc->inv_freq[j])) return fail(SPLASH_ERR_INVALID_ARGUMENT, "inv_freq[%d] is not finite", j);
    r.turns[j] = desc->inv_freq[j] * 0.15915494309189533577;  // 1 / (2 pi)
    r.axis[j] = desc->pair_axis ? desc->pair_axis[j] : 0;
    if (r.axis[j] >= desc->num_axes)
      return fail(SPLASH_ERR_INVALID_ARGUMENT, "pair_axis[%d] = %d is outside [0, %d)", j, r.axis[j], desc->num_axes);
  }
  for (int32_t v = 0; v < num_views; ++v) {
    const splash_rope_view& w = views[v];
    if (w.num_heads < 0) return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_heads < 0");
    if (w.num_heads > 65536) return fail(SPLASH_ERR_UNSUPPORTED, "num_heads must be at most 65536 (got %d)", w.num_heads);
    if (w.x_token_stride < 0 || w.x_head_stride < 0 || w.y_token_stride < 0 || w.y_head_stride < 0)
      return fail(SPLASH_ERR_INVALID_ARGUMENT, "negative stride");
    if (num_tokens > 0 && w.num_heads > 0) {
      if (!w.x || !w.y) return fail(SPLASH_ERR_INVALID_ARGUMENT, "x and y must be non-NULL");
      if (!aligned(w.x, 2) || !aligned(w.y, 2)) return fail(SPLASH_ERR_MISALIGNED, "x and y must be 2-byte aligned");
      if (rows_overlap(num_tokens, w.y_token_stride, w.num_heads, w.y_head_stride, desc->rot_dim))
        return fail(SPLASH_ERR_INVALID_ARGUMENT, "rows of y overlap");
      if (w.x == w.y && (w.x_token_stride != w.y_token_stride || w.x_head_stride != w.y_head_stride))
        return fail(SPLASH_ERR_INVALID_ARGUMENT, "rotating in place needs equal strides");
    }
    r.view[v] = {static_cast<const uint16_t*>(w.x), static_cast<uint16_t*>(w.y), w.x_token_stride, w.x_head_stride,
                 w.y_token_stride, w.y_head_stride, w.num_heads};
  }
  if (num_tokens == 0) return SPLASH_OK;
  if (num_views == 2 && views[0].num_heads > 0 && views[1].num_heads > 0 &&
      (views[0].y == views[1].y || views[0].y == views[1].x || views[1].y == views[0].x))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "a view's y is the other view's x or y");
  if (!positions) return fail(SPLASH_ERR_INVALID_ARGUMENT, "positions is NULL");
  if (!aligned(positions, 4)) return fail(SPLASH_ERR_MISALIGNED, "positions not 4-byte aligned");
  if (desc->num_axes > 1 && position_stride < num_tokens && position_stride != 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "position_stride must be 0 or at least num_tokens");
  const hipError_t e = launch_rope(r, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "rope launch");
}

int splash_gqa_append(const void* k_new, const void* v_new, int64_t token_stride, int64_t head_stride,
                      const int32_t* slots, int32_t num_tokens, void* k_pages, void* v_pages, float* k_scales,
                      float* v_scales, const splash_gqa_desc* desc, void* stream) {
  int st = validate_gqa(desc);
  if (st != SPLASH_OK) return st;
  if (num_tokens < 0 || token_stride < 0 || head_stride < 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_tokens and strides must be >= 0");
  if (num_tokens == 0 || desc->batch == 0) return SPLASH_OK;
  if ((int64_t)num_tokens * desc->num_kv_heads > kMaxAppendRows)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_tokens * num_kv_heads passes 2^25");
  if (!k_new || !v_new || !slots) return fail(SPLASH_ERR_INVALID_ARGUMENT, "k_new, v_new and slots must be non-NULL");
  if ((st = check_gqa_cache(k_pages, v_pages, k_scales, v_scales)) != SPLASH_OK) return st;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || token_stride % 8 || head_stride % 8)
    return fail(SPLASH_ERR_MISALIGNED, "k_new and v_new must be 16-byte aligned, with strides of whole 8 elements");
  if (!aligned(slots, 4)) return fail(SPLASH_ERR_MISALIGNED, "slots not 4-byte aligned");
  const GqaAppendLaunch a = {static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new), token_stride,
                             head_stride, slots, num_tokens, desc->batch, desc->num_kv_heads, desc->head_dim, desc->num_pages,
                             desc->code_type, static_cast<uint8_t*>(k_pages), static_cast<uint8_t*>(v_pages),
                             k_scales, v_scales};
  const hipError_t e = launch_gqa_append(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "gqa append launch");
}

size_t splash_gqa_workspace_size(const splash_gqa_desc* desc, int32_t q_chunk) {
  if (validate_gqa(desc) != SPLASH_OK) return 0;
  if (q_chunk < 1) {
    fail(SPLASH_ERR_INVALID_ARGUMENT, "q_chunk must be >= 1 (got %d)", q_chunk);
    return 0;
  }
  return gqa_layout(desc, q_chunk).total;
}

int splash_gqa_attend(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                      const float* v_scales, const int32_t* block_table, const int32_t* seq_lens, int32_t q_chunk,
                      void* out, float* lse, const splash_gqa_desc* desc, void* workspace, size_t ws_bytes,
                      void* stream) {
  int st = validate_gqa(desc);
  if (st != SPLASH_OK) return st;
  if (q_chunk < 1) return fail(SPLASH_ERR_INVALID_ARGUMENT, "q_chunk must be >= 1 (got %d)", q_chunk);
  if (desc->batch == 0) return SPLASH_OK;
  if (!q || !block_table || !seq_lens || !out || !workspace)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "q, block_table, seq_lens, out and workspace must be non-NULL");
  if ((st = check_gqa_cache(k_pages, v_pages, k_scales, v_scales)) != SPLASH_OK) return st;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
    return fail(SPLASH_ERR_MISALIGNED, "q, out and workspace must be 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(lse, 4))
    return fail(SPLASH_ERR_MISALIGNED, "block_table, seq_lens and lse must be 4-byte aligned");
  const int32_t group = desc->num_heads / desc->num_kv_heads;
  // tiles (request, KV head, block of at least 16 query rows) and the pages
  // and per-tile shares that their positions count stay below 2^30
  const int64_t row_blocks = ((int64_t)q_chunk * group + 15) / 16;
  const int64_t tiles = row_blocks > (1 << 20) ? INT64_MAX : (int64_t)desc->batch * desc->num_kv_heads * row_blocks;
  if (tiles > (1 << 30) || tiles * ((int64_t)desc->max_pages_per_seq + kGqaTileCost) > (1 << 30))
    return fail(SPLASH_ERR_UNSUPPORTED, "batch * num_kv_heads * row blocks * pages passes 2^30");
  const GqaLayout layout = gqa_layout(desc, q_chunk);
  if (ws_bytes < layout.total)
    return fail(SPLASH_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, need %zu", ws_bytes, layout.total);
  GqaAttendLaunch a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.k_pages = static_cast<const uint8_t*>(k_pages);
  a.v_pages = static_cast<const uint8_t*>(v_pages);
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.B = desc->batch;
  a.Hk = desc->num_kv_heads;
  a.group = group;
  a.D = desc->head_dim;
  a.q_chunk = q_chunk;
  a.bt_stride = desc->max_pages_per_seq;
  a.num_pages = desc->num_pages;
  a.code_type = desc->code_type;
  char* ws = static_cast<char*>(workspace);
  a.joined = reinterpret_cast<int4*>(ws);
  a.part_ml = reinterpret_cast<float*>(ws + layout.part_ml);
  a.part_out = reinterpret_cast<float*>(ws + layout.part_out);
  a.workers = splash_device_workers();
  a.scale_log2 = desc->softmax_scale * 1.44269504088896340736f;
  const hipError_t e = launch_gqa_attend(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "gqa attend launch");
}

}  // extern "C"
