// C-ABI of the latent-attention layer around the cache: argument checks and the
// entry points declared in include/splash_attn.h.  No C++ exception crosses this
// boundary.
#include "splash_attn.h"

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>

#include "errors.hpp"
#include "layer.hpp"

using namespace splash;

namespace {

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int32_t kMaxPoolPages = 1 << 25;  // a slot (64 * page + place) fits int32
constexpr int32_t kMaxRows = 1 << 25;       // a launch holds less than 2^32 lanes: 64 a row
constexpr int32_t kMaxProjected = 1 << 24;  // tokens, 16 of them a tile
constexpr int32_t kMaxLayerHeads = 1024;
// A launch holds less than 2^32 lanes: at most 8 a row and head of a projection.
constexpr int64_t kMaxProjectedRows = 1 << 28;
// Tiles of a prompt, of all heads.  Its launches take no more workgroups than stay on the
// chip (a few each where tiles are short), so that two smaller things have to fit: a block of
// the order for the tiles of one head, in the parts' place, and an int32 for each place on an
// XCD.  The limit leaves room for both.
constexpr int64_t kMaxTiles = 1 << 21;
static_assert(kMaxTiles * kPrefillBlock <= 2 * (int64_t)kPrefillParts * kValue * 4, "every block's place in the workspace");
constexpr int64_t kMaxTokenStride = 1 << 24;  // 64 rows' byte offsets fit 32 bits

// A stride over `count` items; over one, which nothing walks (a view may report anything
// there), `none`.
int64_t walked(int32_t count, int64_t stride, int64_t none = 0) { return count > 1 ? stride : none; }

// The pool's limits beyond validate_mla_desc, and its pages.
int check_pool(const splash_mla_desc* d, const void* kv_pages) {
  if (d->num_pages > kMaxPoolPages)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_pages must be at most 2^25 (got %d)", d->num_pages);
  if (!kv_pages) return fail(SPLASH_ERR_INVALID_ARGUMENT, "kv_pages is NULL");
  if (!aligned(kv_pages, 16)) return fail(SPLASH_ERR_MISALIGNED, "kv_pages not 16-byte aligned");
  return SPLASH_OK;
}

// The turn of 64 rotary dims; rope NULL: none.
int read_turn(const splash_rope_desc* rope, const int32_t* positions, int64_t position_stride, int32_t num_tokens,
              TurnLaunch* t) {
  if (!rope) return SPLASH_OK;
  if (!rope->inv_freq) return fail(SPLASH_ERR_INVALID_ARGUMENT, "rope's inv_freq is NULL");
  if (rope->rot_dim != kRope) return fail(SPLASH_ERR_INVALID_ARGUMENT, "rope's rot_dim must be 64 (got %d)", rope->rot_dim);
  if (rope->num_axes < 1 || rope->num_axes > 4)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_axes must be 1 .. 4 (got %d)", rope->num_axes);
  if (!std::isfinite(rope->scale)) return fail(SPLASH_ERR_INVALID_ARGUMENT, "rope's scale is not finite");
  for (int j = 0; j < kRopePairs; ++j) {
    if (!std::isfinite(rope->inv_freq[j])) return fail(SPLASH_ERR_INVALID_ARGUMENT, "inv_freq[%d] is not finite", j);
    t->turns[j] = rope->inv_freq[j] * 0.15915494309189533577;  // 1 / (2 pi)
    t->axis[j] = rope->pair_axis ? rope->pair_axis[j] : 0;
    if (t->axis[j] >= rope->num_axes)
      return fail(SPLASH_ERR_INVALID_ARGUMENT, "pair_axis[%d] = %d is outside [0, %d)", j, t->axis[j], rope->num_axes);
  }
  if (!positions) return fail(SPLASH_ERR_INVALID_ARGUMENT, "positions is NULL");
  if (!aligned(positions, 4)) return fail(SPLASH_ERR_MISALIGNED, "positions not 4-byte aligned");
  if (rope->num_axes > 1 && position_stride < num_tokens && position_stride != 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "position_stride must be 0 or at least num_tokens");
  t->positions = positions;
  t->position_stride = position_stride;
  t->axes = rope->num_axes;
  t->interleaved = rope->interleaved ? 1 : 0;
  t->scale = rope->scale;
  return SPLASH_OK;
}

int check_projection(int32_t num_tokens, int32_t num_heads, const void* w, int64_t w_head_stride, int64_t w_row_stride) {
  if (num_tokens > kMaxProjected) return fail(SPLASH_ERR_UNSUPPORTED, "num_tokens must be at most 2^24 (got %d)", num_tokens);
  if (num_heads > kMaxLayerHeads)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_heads must be at most %d (got %d)", kMaxLayerHeads, num_heads);
  if ((int64_t)num_tokens * num_heads > kMaxProjectedRows)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_tokens * num_heads passes 2^28");
  if (w_head_stride < 0 || w_row_stride < 0) return fail(SPLASH_ERR_INVALID_ARGUMENT, "negative stride");
  if (!w) return fail(SPLASH_ERR_INVALID_ARGUMENT, "the weight is NULL");
  if (!aligned(w, 16) || w_head_stride % 8 || w_row_stride % 8)
    return fail(SPLASH_ERR_MISALIGNED, "the weight must be 16-byte aligned, with strides of whole 8 elements");
  return SPLASH_OK;
}

// The same for every call: parts of all workers (whose number is the chip's), 68 MB.
struct PrefillLayout {
  size_t joined, part_ml, part_out, total;  // the tickets come first
};
PrefillLayout prefill_layout() {
  const size_t slots = 2 * (size_t)kPrefillParts;
  PrefillLayout l;
  l.joined = 8 * 128;
  l.part_ml = l.joined + sizeof(int4) * kPrefillWorkers;
  l.part_out = l.part_ml + slots * 2 * sizeof(float);
  l.total = l.part_out + slots * kValue * sizeof(float);
  return l;
}

}  // namespace

extern "C" {

int splash_mla_append(const void* latent, int64_t latent_stride, const void* key, int64_t key_stride,
                      const void* norm_weight, float norm_eps, const int32_t* positions, int64_t position_stride,
                      const splash_rope_desc* rope, const int32_t* slots, int32_t num_tokens, void* kv_pages,
                      float* kv_scales, const splash_mla_desc* desc, void* stream) {
  int st = validate_mla_desc(desc, 1);
  if (st != SPLASH_OK) return st;
  latent_stride = walked(num_tokens, latent_stride);
  key_stride = walked(num_tokens, key_stride);
  if (num_tokens < 0 || latent_stride < 0 || key_stride < 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "num_tokens and strides must be >= 0");
  if (num_tokens > kMaxRows) return fail(SPLASH_ERR_UNSUPPORTED, "num_tokens must be at most 2^25 (got %d)", num_tokens);
  if (norm_weight && !(std::isfinite(norm_eps) && norm_eps >= 0.f))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "norm_eps must be finite and >= 0");
  if (num_tokens == 0 || desc->batch == 0) return SPLASH_OK;
  if (!latent || !key || !slots) return fail(SPLASH_ERR_INVALID_ARGUMENT, "latent, key and slots must be non-NULL");
  if ((st = check_pool(desc, kv_pages)) != SPLASH_OK) return st;
  if (!aligned(latent, 16) || !aligned(key, 16) || !aligned(norm_weight, 16) || latent_stride % 8 || key_stride % 8)
    return fail(SPLASH_ERR_MISALIGNED, "latent, key and norm_weight must be 16-byte aligned, with strides of whole 8 elements");
  if (!aligned(slots, 4)) return fail(SPLASH_ERR_MISALIGNED, "slots not 4-byte aligned");
  if (desc->kv_dtype == SPLASH_KV_FP8_E4M3) {
    if (kv_scales != desc->kv_scales) return fail(SPLASH_ERR_INVALID_ARGUMENT, "kv_scales is not desc's");
    if (!aligned(kv_scales, 4)) return fail(SPLASH_ERR_MISALIGNED, "kv_scales not 4-byte aligned");
  }
  MlaAppendLaunch a = {};
  if ((st = read_turn(rope, positions, position_stride, num_tokens, &a.turn)) != SPLASH_OK) return st;
  a.latent = static_cast<const uint16_t*>(latent);
  a.key = static_cast<const uint16_t*>(key);
  a.latent_stride = latent_stride;
  a.key_stride = key_stride;
  a.norm_weight = static_cast<const uint16_t*>(norm_weight);
  a.norm_eps = norm_eps;
  a.slots = slots;
  a.num_tokens = num_tokens;
  a.num_pages = desc->num_pages;
  a.kv_dtype = desc->kv_dtype;
  a.pages = static_cast<uint8_t*>(kv_pages);
  a.scales = kv_scales;
  const hipError_t e = launch_mla_append(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "mla append launch");
}

int splash_mla_gather(const void* kv_pages, const int32_t* block_table, const int32_t* key_begin,
                      const int32_t* row_indptr, int32_t max_rows, void* latent_out, int64_t latent_stride,
                      void* key_out, int64_t key_stride, const splash_mla_desc* desc, void* stream) {
  int st = validate_mla_desc(desc, 1);
  if (st != SPLASH_OK) return st;
  latent_stride = walked(max_rows, latent_stride, kDimV);
  key_stride = walked(max_rows, key_stride, kRope);
  if (max_rows < 0) return fail(SPLASH_ERR_INVALID_ARGUMENT, "max_rows < 0");
  if (max_rows > kMaxRows) return fail(SPLASH_ERR_UNSUPPORTED, "max_rows must be at most 2^25 (got %d)", max_rows);
  if (desc->max_pages_per_seq > INT32_MAX / kPage)
    return fail(SPLASH_ERR_UNSUPPORTED, "max_pages_per_seq must be at most 2^25 - 1 (got %d)", desc->max_pages_per_seq);
  if (latent_stride < kDimV || key_stride < kRope)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "latent_stride must be at least 512 and key_stride at least 64");
  if (max_rows == 0 || desc->batch == 0) return SPLASH_OK;
  if ((st = check_pool(desc, kv_pages)) != SPLASH_OK) return st;
  if (!block_table || !row_indptr || !latent_out || !key_out)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "block_table, row_indptr, latent_out and key_out must be non-NULL");
  if (!aligned(latent_out, 16) || !aligned(key_out, 16) || latent_stride % 8 || key_stride % 8)
    return fail(SPLASH_ERR_MISALIGNED, "outputs must be 16-byte aligned, with strides of whole 8 elements");
  if (!aligned(block_table, 4) || !aligned(key_begin, 4) || !aligned(row_indptr, 4) || !aligned(desc->kv_scales, 4))
    return fail(SPLASH_ERR_MISALIGNED, "block_table, key_begin, row_indptr and kv_scales must be 4-byte aligned");
  const MlaGatherLaunch g = {static_cast<const uint8_t*>(kv_pages), desc->kv_scales, block_table, key_begin, row_indptr,
                             desc->batch, desc->max_pages_per_seq, desc->num_pages, max_rows, desc->kv_dtype,
                             static_cast<uint16_t*>(latent_out), static_cast<uint16_t*>(key_out), latent_stride, key_stride};
  const hipError_t e = launch_mla_gather(g, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "mla gather launch");
}

int splash_mla_absorb_q(const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* w_uk,
                        int64_t w_head_stride, int64_t w_row_stride, const int32_t* positions, int64_t position_stride,
                        const splash_rope_desc* rope, int32_t num_tokens, int32_t num_heads, void* q_out, void* stream) {
  q_token_stride = walked(num_tokens, q_token_stride);
  q_head_stride = walked(num_heads, q_head_stride);
  w_head_stride = walked(num_heads, w_head_stride);
  if (num_tokens < 0 || num_heads < 0 || q_token_stride < 0 || q_head_stride < 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "counts and strides must be >= 0");
  if (num_tokens == 0 || num_heads == 0) return SPLASH_OK;
  int st = check_projection(num_tokens, num_heads, w_uk, w_head_stride, w_row_stride);
  if (st != SPLASH_OK) return st;
  if (!q || !q_out) return fail(SPLASH_ERR_INVALID_ARGUMENT, "q and q_out must be non-NULL");
  if (!aligned(q, 16) || !aligned(q_out, 16) || q_token_stride % 8 || q_head_stride % 8)
    return fail(SPLASH_ERR_MISALIGNED, "q and q_out must be 16-byte aligned, with strides of whole 8 elements");
  if (q == q_out) return fail(SPLASH_ERR_INVALID_ARGUMENT, "q_out is q");
  MlaAbsorbLaunch a = {};
  if ((st = read_turn(rope, positions, position_stride, num_tokens, &a.turn)) != SPLASH_OK) return st;
  a.q = static_cast<const uint16_t*>(q);
  a.q_token = q_token_stride;
  a.q_head = q_head_stride;
  a.w = static_cast<const uint16_t*>(w_uk);
  a.w_head = w_head_stride;
  a.w_row = w_row_stride;
  a.num_tokens = num_tokens;
  a.heads = num_heads;
  a.out = static_cast<uint16_t*>(q_out);
  const hipError_t e = launch_mla_absorb(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "mla absorb launch");
}

int splash_mla_expand_out(const void* out, const void* w_uv, int64_t w_head_stride, int64_t w_row_stride,
                          int32_t num_tokens, int32_t num_heads, void* y, int64_t y_token_stride, int64_t y_head_stride,
                          void* stream) {
  w_head_stride = walked(num_heads, w_head_stride);
  y_token_stride = walked(num_tokens, y_token_stride);
  y_head_stride = walked(num_heads, y_head_stride);
  if (num_tokens < 0 || num_heads < 0 || y_token_stride < 0 || y_head_stride < 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "counts and strides must be >= 0");
  if (num_tokens == 0 || num_heads == 0) return SPLASH_OK;
  const int st = check_projection(num_tokens, num_heads, w_uv, w_head_stride, w_row_stride);
  if (st != SPLASH_OK) return st;
  if (!out || !y) return fail(SPLASH_ERR_INVALID_ARGUMENT, "out and y must be non-NULL");
  if (!aligned(out, 16) || !aligned(y, 16) || y_token_stride % 8 || y_head_stride % 8)
    return fail(SPLASH_ERR_MISALIGNED, "out and y must be 16-byte aligned, with strides of whole 8 elements");
  // a token's heads side by side and tokens past each other, or the other way round
  typedef __int128 Wide;
  const Wide token = num_tokens > 1 ? y_token_stride : INT64_MAX, head = num_heads > 1 ? y_head_stride : INT64_MAX;
  const Wide heads_width = num_heads > 1 ? (num_heads - 1) * head + kValue : kValue;
  const Wide tokens_width = num_tokens > 1 ? (num_tokens - 1) * token + kValue : kValue;
  if (!((head >= kValue && token >= heads_width) || (token >= kValue && head >= tokens_width)))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "rows of y overlap, or lie among each other");
  if (out == y) return fail(SPLASH_ERR_INVALID_ARGUMENT, "y is out");
  const MlaExpandLaunch a = {static_cast<const uint16_t*>(out), static_cast<const uint16_t*>(w_uv), w_head_stride, w_row_stride,
                             num_tokens, num_heads, static_cast<uint16_t*>(y), y_token_stride, y_head_stride};
  const hipError_t e = launch_mla_expand(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "mla expand launch");
}

size_t splash_mla_prefill_workspace_size(int32_t batch, int32_t num_rows, int32_t num_heads) {
  if (batch < 0 || num_rows < 0 || num_heads < 0) return 0;
  return prefill_layout().total;
}

int splash_mla_prefill(const splash_mla_rows* q, const splash_mla_rows* k, const void* key, int64_t key_stride,
                       const splash_mla_rows* v, const int32_t* q_indptr, const int32_t* kv_indptr, int32_t batch,
                       int32_t num_rows, int32_t num_keys, int32_t num_heads, float softmax_scale, void* out, float* lse,
                       void* workspace, size_t ws_bytes, void* stream) {
  if (!q || !k || !v) return fail(SPLASH_ERR_INVALID_ARGUMENT, "q, k and v must be non-NULL");
  const auto view = [&](const splash_mla_rows* r, int32_t count) {
    return splash_mla_rows{r->x, walked(count, r->token_stride), walked(num_heads, r->head_stride)};
  };
  const splash_mla_rows views[] = {view(q, num_rows), view(k, num_keys), view(v, num_keys)};
  key_stride = walked(num_keys, key_stride);
  if (batch < 0 || num_rows < 0 || num_keys < 0 || num_heads < 0 || key_stride < 0)
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "counts and strides must be >= 0");
  for (const splash_mla_rows& r : views) {
    if (r.token_stride < 0 || r.head_stride < 0) return fail(SPLASH_ERR_INVALID_ARGUMENT, "negative stride");
    if (r.token_stride % 8 || r.head_stride % 8 || !aligned(r.x, 16))
      return fail(SPLASH_ERR_MISALIGNED, "q, k and v must be 16-byte aligned, with strides of whole 8 elements");
    if (r.token_stride > kMaxTokenStride) return fail(SPLASH_ERR_UNSUPPORTED, "a token stride past 2^24");
  }
  if (key_stride > kMaxTokenStride) return fail(SPLASH_ERR_UNSUPPORTED, "a token stride past 2^24");
  if (key_stride % 8 || !aligned(key, 16) || !aligned(out, 16) || !aligned(workspace, 16))
    return fail(SPLASH_ERR_MISALIGNED, "key, out and workspace must be 16-byte aligned, key_stride whole 8 elements");
  if (!aligned(q_indptr, 4) || !aligned(kv_indptr, 4) || !aligned(lse, 4))
    return fail(SPLASH_ERR_MISALIGNED, "q_indptr, kv_indptr and lse must be 4-byte aligned");
  if (!(std::isfinite(softmax_scale) && softmax_scale > 0.f))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "softmax_scale must be finite and > 0");
  if (num_heads > kMaxLayerHeads)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_heads must be at most %d (got %d)", kMaxLayerHeads, num_heads);
  if (num_rows > kMaxRows || num_keys > kMaxRows || batch > 1 << 20)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_rows and num_keys must be at most 2^25, batch at most 2^20");
  if ((int64_t)num_rows * num_heads > INT32_MAX)
    return fail(SPLASH_ERR_UNSUPPORTED, "num_rows * num_heads passes 2^31 - 1");
  if ((num_rows / 128 + (int64_t)(batch < num_rows ? batch : num_rows)) * num_heads > kMaxTiles)
    return fail(SPLASH_ERR_UNSUPPORTED, "(num_rows / 128 + batch) * num_heads passes 2^21");
  if (num_rows == 0 || num_heads == 0 || batch == 0) return SPLASH_OK;
  if (!q->x || !q_indptr || !kv_indptr || !out || !workspace || (num_keys > 0 && (!k->x || !key || !v->x)))
    return fail(SPLASH_ERR_INVALID_ARGUMENT, "NULL buffer");
  const size_t need = splash_mla_prefill_workspace_size(batch, num_rows, num_heads);
  if (ws_bytes < need)
    return fail(SPLASH_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, need %zu", ws_bytes, need);
  MlaPrefillLaunch a = {};
  a.q = static_cast<const uint16_t*>(q->x);
  a.k = static_cast<const uint16_t*>(k->x);
  a.key = static_cast<const uint16_t*>(key);
  a.v = static_cast<const uint16_t*>(v->x);
  a.q_token = views[0].token_stride;
  a.q_head = views[0].head_stride;
  a.k_token = views[1].token_stride;
  a.k_head = views[1].head_stride;
  a.key_token = key_stride;
  a.v_token = views[2].token_stride;
  a.v_head = views[2].head_stride;
  a.q_indptr = q_indptr;
  a.kv_indptr = kv_indptr;
  a.B = batch;
  a.num_rows = num_rows;
  a.num_keys = num_keys;
  a.heads = num_heads;
  a.scale_log2 = softmax_scale * 1.44269504088896340736f;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  char* ws = static_cast<char*>(workspace);
  const PrefillLayout layout = prefill_layout();
  a.tickets = reinterpret_cast<int32_t*>(ws);
  a.joined = reinterpret_cast<int4*>(ws + layout.joined);
  a.part_ml = reinterpret_cast<float*>(ws + layout.part_ml);
  a.part_out = reinterpret_cast<float*>(ws + layout.part_out);
  a.tiles = a.part_out;
  a.units = splash_device_workers();
  if (!std::isfinite(a.scale_log2)) return fail(SPLASH_ERR_INVALID_ARGUMENT, "softmax_scale * log2(e) passes fp32");
  const hipError_t e = launch_mla_prefill(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SPLASH_OK : hip_fail(e, "mla prefill launch");
}

}  // extern "C"
