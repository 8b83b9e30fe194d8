// Host sanitizer driver of the serving-step calls: random and extreme arguments
// on addresses that are never read (the host arrays of splash_rope apart, which
// have exactly their documented length).  The launchers' stand-ins check what
// the kernels rely on.  Prints "ok <launches>".
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <memory>
#include <random>

#include "splash_attn.h"
#include "step.hpp"

namespace {
long launches = 0;
void need(bool c, const char* what) {
  if (!c) {
    std::fprintf(stderr, "FAILED %s\n", what);
    std::abort();
  }
}
}  // namespace

namespace splash {
hipError_t launch_step_tables(const TablesLaunch& p, hipStream_t) {
  ++launches;
  need(p.B >= 0 && p.B <= kMaxTableBatch && (int64_t)p.max_pages * kPage * p.B <= INT32_MAX && p.num_pages <= 1 << 25, "tables");
  return hipSuccess;
}
hipError_t launch_rope(const RopeLaunch& p, hipStream_t) {
  ++launches;
  need(p.pairs >= 1 && p.pairs <= kMaxRopePairs && p.num_tokens >= 1 && p.num_tokens <= 1 << 25, "rope");
  for (int j = 0; j < p.pairs; ++j) need(p.axis[j] < 4, "axis");
  return hipSuccess;
}
hipError_t launch_gqa_append(const GqaAppendLaunch& p, hipStream_t) {
  ++launches;
  need(p.num_tokens >= 1 && (int64_t)p.num_tokens * p.Hk <= 1 << 25 && p.num_pages <= 1 << 25 && p.Hk >= 1 && p.token_stride % 8 == 0, "append");
  return hipSuccess;
}
hipError_t launch_gqa_attend(const GqaAttendLaunch& p, hipStream_t) {
  ++launches;
  const int64_t rows = (int64_t)p.q_chunk * p.group;
  need(rows <= 1 << 24 && (int64_t)p.bt_stride * kPage <= INT32_MAX, "rows");
  need((int64_t)p.B * p.Hk * ((rows + 15) / 16) * (p.bt_stride + kGqaTileCost) <= 1 << 30, "places");
  return hipSuccess;
}
}  // namespace splash

int main(int argc, char** argv) {
  const int calls = argc > 1 ? std::atoi(argv[1]) : 100000;
  std::mt19937 rng(7);
  auto uni = [&](int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); };
  // small numbers mostly, the extremes of the type now and then
  auto num = [&](int64_t hi) -> int32_t {
    switch (uni(0, 9)) {
      case 0: return INT32_MAX;
      case 1: return (int32_t)(INT32_MAX >> uni(0, 30));
      case 2: return uni(0, 20) ? 0 : INT32_MIN;
      default: return (int32_t)uni(1, hi);
    }
  };
  auto p = [&]() -> int32_t* { return reinterpret_cast<int32_t*>(uni(0, 60) ? (1 << 20) + 256 * uni(0, 100) : uni(0, 1)); };
  for (int i = 0; i < calls; ++i) {
    const int kv = (int)uni(1, 8);
    splash_gqa_desc d = {num(300), uni(0, 9) ? kv * (int)uni(1, 40) : num(9), kv, 64 << uni(0, 2), uni(0, 30) ? 64 : num(64),
                         num(300), num(3000), (int)uni(0, uni(0, 9) ? 1 : 3), uni(0, 20) ? 0.1f : -1.f};
    const int32_t q = num(9);
    switch (i % 4) {
      case 0:
        splash_gqa_attend(p(), p(), p(), (float*)p(), (float*)p(), p(), p(), q, p(), (float*)p(), &d, p(),
                          uni(0, 9) ? splash_gqa_workspace_size(&d, q) : uni(0, 1000), nullptr);
        break;
      case 1:
        splash_gqa_append(p(), p(), 8 * (int64_t)num(1000), 8 * (int64_t)num(100), p(), num(1000), p(), p(), (float*)p(),
                          (float*)p(), &d, nullptr);
        break;
      case 2:
        splash_step_tables(p(), uni(0, 1) ? p() : nullptr, num(9), num(9000), p(), num(1000), p(), p(), p(), num(300),
                           num(3000), num(9000), p(), p(), p(), p(), nullptr);
        break;
      default: {
        const int32_t rot = uni(0, 5) ? 2 * (int)uni(1, 128) : (int)uni(-4, 300), half = rot > 1 ? rot / 2 : 1;
        std::unique_ptr<double[]> freq(new double[half]);
        std::unique_ptr<uint8_t[]> axis(new uint8_t[half]);
        const int axes = (int)uni(0, 5);
        for (int j = 0; j < half; ++j) {
          freq[j] = 0.5;
          axis[j] = (uint8_t)uni(0, axes > 1 && uni(0, 99) ? axes - 1 : axes ? axes - 1 : 0);
        }
        splash_rope_desc r = {rot, (int)uni(0, 1), axes, 1.f, freq.get(), uni(0, 3) ? axis.get() : nullptr};
        splash_rope_view v[2];
        for (auto& w : v) w = {p(), p(), num(1000), num(1000), num(1000), num(1000), uni(0, 4) ? num(64) : num(100000)};
        splash_rope(v, (int)uni(0, 3), p(), num(5000), num(1000), &r, nullptr);
      }
    }
  }
  std::printf("ok %ld\n", launches);
  return 0;
}
