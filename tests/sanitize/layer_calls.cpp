// Host driver of single calls around the latent cache, on addresses that are never
// read: the launchers' stand-ins keep what they get.  Prints "ok" and the number of
// calls looked at, or what failed.
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "layer.hpp"
#include "splash_attn.h"

namespace {
int launches = 0, calls = 0;
splash::MlaAppendLaunch append_;
splash::MlaGatherLaunch gather_;
splash::MlaAbsorbLaunch absorb_;
splash::MlaExpandLaunch expand_;
splash::MlaPrefillLaunch prefill_;
void* const kAt = reinterpret_cast<void*>(1 << 20);
void* const kTo = reinterpret_cast<void*>(2 << 20);
}  // namespace

namespace splash {
hipError_t launch_mla_append(const MlaAppendLaunch& a, hipStream_t) { return append_ = a, ++launches, hipSuccess; }
hipError_t launch_mla_gather(const MlaGatherLaunch& a, hipStream_t) { return gather_ = a, ++launches, hipSuccess; }
hipError_t launch_mla_absorb(const MlaAbsorbLaunch& a, hipStream_t) { return absorb_ = a, ++launches, hipSuccess; }
hipError_t launch_mla_expand(const MlaExpandLaunch& a, hipStream_t) { return expand_ = a, ++launches, hipSuccess; }
hipError_t launch_mla_prefill(const MlaPrefillLaunch& a, hipStream_t) { return prefill_ = a, ++launches, hipSuccess; }
}  // namespace splash

namespace {
void need(bool c, const char* what) {
  if (!c) {
    std::printf("FAILED %s: %s\n", what, splash_last_error());
    std::exit(1);
  }
}
// The call is taken, or refused before any launch.
void taken(int status, const char* what) {
  ++calls;
  need(status == SPLASH_OK && launches == 1, what);
  launches = 0;
}
void refused(int status, int as, const char* what) {
  ++calls;
  need(status == as && launches == 0, what);
}

splash_mla_desc pool() {
  splash_mla_desc d = {};
  d.batch = 1;
  d.num_heads = 128;
  d.page_size = 64;
  d.max_pages_per_seq = d.num_pages = 4;
  d.dim_qk = 576;
  d.dim_v = 512;
  d.kv_dtype = SPLASH_KV_BF16;
  d.softmax_scale = 0.1f;
  return d;
}
int append(int32_t n, int64_t latent, int64_t key) {
  const splash_mla_desc d = pool();
  return splash_mla_append(kAt, latent, kAt, key, nullptr, 0.f, nullptr, 0, nullptr, (int32_t*)kAt, n, kTo, nullptr, &d, nullptr);
}
int gather(int32_t rows, int64_t latent, int64_t key) {
  const splash_mla_desc d = pool();
  return splash_mla_gather(kAt, (int32_t*)kAt, nullptr, (int32_t*)kAt, rows, kTo, latent, kTo, key, &d, nullptr);
}
int absorb(int32_t n, int32_t heads, int64_t token, int64_t head, int64_t w) {
  return splash_mla_absorb_q(kAt, token, head, kAt, w, 512, nullptr, 0, nullptr, n, heads, kTo, nullptr);
}
int expand(int32_t n, int32_t heads, int64_t w, int64_t token, int64_t head) {
  return splash_mla_expand_out(kAt, kAt, w, 512, n, heads, kTo, token, head, nullptr);
}
int prefill(int32_t rows, int32_t keys, int32_t heads, splash_mla_rows q, splash_mla_rows k, int64_t key, splash_mla_rows v) {
  q.x = k.x = v.x = kAt;
  return splash_mla_prefill(&q, &k, kAt, key, &v, (int32_t*)kAt, (int32_t*)kAt, 1, rows, keys, heads, 0.1f, kTo, nullptr, kTo,
                            splash_mla_prefill_workspace_size(1, rows, heads), nullptr);
}

// A stride over a dimension of one is whatever a view happens to report.
void strides() {
  const int64_t odd[] = {577, 1, 0, -8, (int64_t)1 << 40, INT64_MAX, INT64_MIN};
  for (const int64_t s : odd) {
    taken(append(1, s, s), "append of one row");
    need(append_.latent_stride >= 0 && append_.key_stride >= 0, "append's strides");
    taken(gather(1, s, s), "gather of one row");
    need(gather_.latent_stride >= 0 && gather_.key_stride >= 0, "gather's strides");
    taken(absorb(1, 4, s, 192, 65536), "absorb of one token");
    taken(absorb(4, 1, 192, s, s), "absorb of one head");
    need(absorb_.q_token == 192 && absorb_.q_head >= 0 && absorb_.w_head >= 0 && absorb_.w_row == 512, "absorb's strides");
    taken(expand(1, 4, 65536, s, 128), "expand of one token");
    need(expand_.y_head == 128 && expand_.y_token >= 0 && expand_.w_head == 65536, "expand's strides");
    taken(expand(4, 1, s, 128, s), "expand of one head");
    need(expand_.y_token == 128 && expand_.y_head >= 0 && expand_.w_head >= 0, "expand's strides");
    taken(expand(1, 1, s, s, s), "expand of one row");
    taken(prefill(1, 2, 2, {0, s, 192}, {0, 256, 128}, 64, {0, 256, 128}), "prefill of one row");
    need(prefill_.q_token >= 0 && prefill_.q_head == 192 && prefill_.k_token == 256 && prefill_.key_token == 64, "prefill's strides");
    taken(prefill(2, 1, 2, {0, 384, 192}, {0, s, 128}, s, {0, s, 128}), "prefill over one key");
    need(prefill_.q_token == 384 && prefill_.k_token >= 0 && prefill_.key_token >= 0 && prefill_.v_token >= 0, "prefill's strides");
    taken(prefill(2, 2, 1, {0, 192, s}, {0, 128, s}, 64, {0, 128, s}), "prefill of one head");
    need(prefill_.q_head >= 0 && prefill_.k_head >= 0 && prefill_.v_head >= 0 && prefill_.v_token == 128, "prefill's strides");
    taken(prefill(1, 1, 1, {0, s, s}, {0, s, s}, s, {0, s, s}), "prefill of one row, key and head");
  }
  // over two they are walked
  refused(append(2, 577, 64), SPLASH_ERR_MISALIGNED, "latent");
  refused(append(2, 512, -8), SPLASH_ERR_INVALID_ARGUMENT, "key");
  refused(gather(2, 504, 64), SPLASH_ERR_INVALID_ARGUMENT, "latent");
  refused(gather(2, 512, 65), SPLASH_ERR_MISALIGNED, "key");
  refused(absorb(2, 1, 193, 192, 65536), SPLASH_ERR_MISALIGNED, "tokens");
  refused(absorb(1, 2, 384, 193, 65536), SPLASH_ERR_MISALIGNED, "heads");
  refused(absorb(1, 2, 384, 192, 65537), SPLASH_ERR_MISALIGNED, "the weight's heads");
  refused(expand(2, 1, 65536, 129, 128), SPLASH_ERR_MISALIGNED, "tokens");
  refused(expand(2, 1, 65536, 120, 128), SPLASH_ERR_INVALID_ARGUMENT, "tokens that overlap");
  refused(expand(1, 2, 65536, 256, 120), SPLASH_ERR_INVALID_ARGUMENT, "heads that overlap");
  refused(prefill(2, 1, 1, {0, 193, 0}, {0, 0, 0}, 0, {0, 0, 0}), SPLASH_ERR_MISALIGNED, "q");
  refused(prefill(1, 2, 1, {0, 0, 0}, {0, 128, 0}, (int64_t)1 << 25, {0, 128, 0}), SPLASH_ERR_UNSUPPORTED, "key");
  refused(prefill(1, 2, 1, {0, 0, 0}, {0, 128, 0}, 64, {0, -128, 0}), SPLASH_ERR_INVALID_ARGUMENT, "v");
  refused(prefill(1, 1, 2, {0, 0, 192}, {0, 0, 132}, 0, {0, 0, 128}), SPLASH_ERR_MISALIGNED, "k's heads");
}
}  // namespace

int main(int argc, char** argv) {
  if (argc > 1 && !std::strcmp(argv[1], "strides")) strides();
  std::printf("ok %d\n", calls);
  return 0;
}
