// Host sanitizer driver of the calls around the latent cache: random and extreme
// arguments on addresses that are never read (the rope's host arrays apart, which
// have exactly their documented length).  The launchers' stand-ins check what the
// kernels rely on.  Prints "ok <launches of each call>".
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <memory>
#include <random>

#include "layer.hpp"
#include "splash_attn.h"

namespace {
long launches[5] = {};
void need(bool c, const char* what) {
  if (!c) {
    std::fprintf(stderr, "FAILED %s\n", what);
    std::abort();
  }
}
bool wide(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 16 == 0; }
void check_turn(const splash::TurnLaunch& t) {
  for (int j = 0; t.positions && j < splash::kRopePairs; ++j) need(t.axis[j] < 4, "axis");
}
}  // namespace

namespace splash {
hipError_t launch_mla_append(const MlaAppendLaunch& a, hipStream_t) {
  ++launches[0];
  need(wide(a.latent) && wide(a.key) && wide(a.pages) && a.slots && a.latent_stride % 8 == 0 && a.key_stride >= 0, "rows");
  need(a.num_tokens >= 1 && a.num_tokens <= 1 << 25 && a.num_pages <= 1 << 25, "append");
  need(a.kv_dtype != SPLASH_KV_FP8_E4M3 || a.scales, "scales");
  check_turn(a.turn);
  return hipSuccess;
}
hipError_t launch_mla_gather(const MlaGatherLaunch& a, hipStream_t) {
  ++launches[1];
  need(wide(a.pages) && wide(a.latent) && wide(a.key) && a.block_table && a.row_indptr, "buffers");
  need(a.B >= 1 && a.max_rows >= 1 && a.max_rows <= 1 << 25 && a.num_pages <= 1 << 25, "gather");
  need(a.bt_stride >= 1 && (int64_t)a.bt_stride * kPage <= INT32_MAX && a.latent_stride >= 512 && a.key_stride >= 64, "table");
  need(a.kv_dtype != SPLASH_KV_FP8_E4M3 || a.scales, "scales");
  return hipSuccess;
}
hipError_t launch_mla_absorb(const MlaAbsorbLaunch& a, hipStream_t) {
  ++launches[2];
  need(wide(a.q) && wide(a.w) && wide(a.out) && a.num_tokens >= 1 && a.heads >= 1 && a.heads <= 1024, "absorb");
  need((int64_t)a.num_tokens * a.heads <= 1 << 28 && a.num_tokens <= 1 << 24 && a.w_row % 8 == 0 && a.q_head % 8 == 0, "sizes");
  check_turn(a.turn);
  return hipSuccess;
}
hipError_t launch_mla_expand(const MlaExpandLaunch& a, hipStream_t) {
  ++launches[3];
  need(wide(a.x) && wide(a.w) && wide(a.y) && a.num_tokens >= 1 && a.heads >= 1 && a.heads <= 1024, "expand");
  need((int64_t)a.num_tokens * a.heads <= 1 << 28 && a.w_head % 8 == 0 && a.y_token % 8 == 0, "sizes");
  need(a.num_tokens == 1 || a.y_token >= kValue, "rows of y by token");
  need(a.heads == 1 || a.y_head >= kValue, "rows of y by head");
  return hipSuccess;
}
hipError_t launch_mla_prefill(const MlaPrefillLaunch& a, hipStream_t) {
  ++launches[4];
  need(wide(a.q) && wide(a.out) && wide(a.joined) && wide(a.part_out) && (a.num_keys == 0 || (wide(a.k) && wide(a.key) && wide(a.v))),
       "buffers");
  need(a.B >= 1 && a.num_rows >= 1 && a.heads >= 1 && a.units >= 1 && a.scale_log2 > 0.f, "prefill");
  need((int64_t)a.num_rows * a.heads <= INT32_MAX && a.num_rows <= 1 << 25 && a.num_keys <= 1 << 25, "sizes");
  need((a.num_rows / 128 + (int64_t)(a.B < a.num_rows ? a.B : a.num_rows)) * a.heads <= 1 << 21, "tiles");
  need(a.q_token <= 1 << 24 && a.k_token <= 1 << 24 && a.key_token <= 1 << 24 && a.v_token <= 1 << 24, "strides");
  return hipSuccess;
}
}  // namespace splash

int main(int argc, char** argv) {
  const int calls = argc > 1 ? std::atoi(argv[1]) : 100000;
  std::mt19937 rng(11);
  auto uni = [&](int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); };
  // small numbers mostly, the extremes of the type now and then
  auto num = [&](int64_t hi) -> int32_t {
    switch (uni(0, 15)) {
      case 0: return INT32_MAX;
      case 1: return (int32_t)(INT32_MAX >> uni(0, 30));
      case 2: return uni(0, 20) ? 0 : INT32_MIN;
      default: return (int32_t)uni(1, hi);
    }
  };
  auto stride = [&](int64_t hi) -> int64_t {
    switch (uni(0, 20)) {
      case 0: return INT64_MAX >> uni(0, 40);
      case 1: return uni(0, 9) ? 0 : INT64_MIN;
      default: return 8 * uni(1, hi);
    }
  };
  auto p = [&]() -> int32_t* { return reinterpret_cast<int32_t*>(uni(0, 60) ? (1 << 20) + 256 * uni(0, 100) : uni(0, 1)); };
  for (int i = 0; i < calls; ++i) {
    const int32_t pairs = 32;
    std::unique_ptr<double[]> freq(new double[pairs]);
    std::unique_ptr<uint8_t[]> axis(new uint8_t[pairs]);
    const int axes = (int)uni(0, 5);
    for (int j = 0; j < pairs; ++j) {
      freq[j] = 0.5;
      axis[j] = (uint8_t)uni(0, axes > 1 ? axes - 1 : 0);
    }
    splash_rope_desc rope = {uni(0, 9) ? 64 : num(300), (int)uni(0, 1), axes, 1.f, freq.get(), uni(0, 3) ? axis.get() : nullptr};
    const splash_rope_desc* turn = uni(0, 1) ? &rope : nullptr;
    splash_mla_desc d = {};
    d.dim_qk = 576;
    d.dim_v = 512;
    d.batch = num(300);
    d.num_heads = 128;
    d.page_size = 64;
    d.max_pages_per_seq = num(300);
    d.num_pages = num(3000);
    d.kv_dtype = (int32_t)uni(0, uni(0, 9) ? 2 : 4);
    float* scales = (float*)p();
    d.kv_scales = scales;
    d.softmax_scale = 0.1f;
    switch (i % 5) {
      case 0:
        splash_mla_append(p(), stride(1000), p(), stride(1000), uni(0, 1) ? p() : nullptr, 1e-6f, p(), num(1000), turn, p(),
                          num(1000), p(), uni(0, 9) ? scales : (float*)p(), &d, nullptr);
        break;
      case 1:
        splash_mla_gather(p(), p(), uni(0, 1) ? p() : nullptr, p(), num(1000), p(), uni(0, 9) ? 504 + 8 * uni(0, 100) : stride(100), p(),
                          uni(0, 9) ? 56 + 8 * uni(0, 100) : stride(100), &d, nullptr);
        break;
      case 2:
        splash_mla_absorb_q(p(), stride(1000), stride(100), p(), stride(1000), stride(100), p(), num(1000), turn, num(1000),
                            num(128), p(), nullptr);
        break;
      case 3: {
        const int32_t n = num(100), heads = num(64);
        const int64_t head = uni(0, 9) ? 128 + 8 * uni(0, 9) : stride(100);
        const int64_t token = uni(0, 9) && head >= 0 && head < 1 << 20 ? head * (heads > 0 ? heads : 1) : stride(5000);
        const bool swap = uni(0, 3) == 0;
        splash_mla_expand_out(p(), p(), stride(1000), stride(100), swap ? heads : n, swap ? n : heads, p(), swap ? head : token,
                              swap ? token : head, nullptr);
        break;
      }
      default: {
        splash_mla_rows q = {p(), stride(1000), stride(100)}, k = {p(), stride(1000), stride(100)}, v = {p(), stride(1000), stride(100)};
        const int32_t b = num(100), rows = num(5000), heads = num(128);
        splash_mla_prefill(uni(0, 99) ? &q : nullptr, &k, p(), stride(100), &v, p(), p(), b, rows, num(5000), heads,
                           uni(0, 20) ? 0.1f : -1.f, p(), (float*)p(), p(),
                           uni(0, 9) ? splash_mla_prefill_workspace_size(b, rows, heads) : uni(0, 1000), nullptr);
      }
    }
  }
  std::printf("ok");
  for (long n : launches) std::printf(" %ld", n);
  std::printf("\n");
  return 0;
}
