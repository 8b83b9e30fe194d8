// splash_rope's refusal of overlapping rows, against every element of small
// layouts: on addresses that are never read, with a stand-in for the launch.
// Prints "ok <accepted> <refused>".
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "splash_attn.h"
#include "step.hpp"

namespace {
long launches = 0;

// Whether two of the view's rows share an element of y.
bool overlap(int tokens, int64_t token, int heads, int64_t head, int rot) {
  std::vector<char> seen((size_t)((tokens - 1) * token + (heads - 1) * head + rot), 0);
  for (int n = 0; n < tokens; ++n)
    for (int h = 0; h < heads; ++h)
      for (int d = 0; d < rot; ++d) {
        char& s = seen[(size_t)(n * token + h * head + d)];
        if (s) return true;
        s = 1;
      }
  return false;
}
}  // namespace

namespace splash {
hipError_t launch_step_tables(const TablesLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_rope(const RopeLaunch&, hipStream_t) {
  ++launches;
  return hipSuccess;
}
hipError_t launch_gqa_append(const GqaAppendLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_gqa_attend(const GqaAttendLaunch&, hipStream_t) { return hipSuccess; }
}  // namespace splash

int main() {
  const double freq[4] = {1., 1., 1., 1.};
  char* const x = reinterpret_cast<char*>(1 << 20);
  char* const far = reinterpret_cast<char*>(1 << 24);
  const int32_t* const pos = reinterpret_cast<const int32_t*>(1 << 26);
  long accepted = 0, refused = 0;
  for (int rot = 2; rot <= 4; rot += 2)
    for (int tokens = 1; tokens <= 5; ++tokens)
      for (int heads = 1; heads <= 5; ++heads)
        for (int64_t token = 0; token <= 24; ++token)
          for (int64_t head = 0; head <= 24; ++head)
            for (int in_place = 0; in_place <= 1; ++in_place) {
              const splash_rope_desc desc = {rot, 0, 1, 1.f, freq, nullptr};
              const splash_rope_view view = {x, in_place ? x : far, token, head, token, head, heads};
              const long before = launches;
              const int st = splash_rope(&view, 1, pos, tokens, tokens, &desc, nullptr);
              const bool bad = overlap(tokens, token, heads, head, rot);
              if (bad ? (st != SPLASH_ERR_INVALID_ARGUMENT || launches != before) : (st != SPLASH_OK || launches != before + 1)) {
                std::fprintf(stderr, "rot %d tokens %d heads %d strides %d %d in place %d: overlap %d, status %d\n", rot, tokens,
                             heads, (int)token, (int)head, in_place, bad, st);
                return 1;
              }
              (bad ? refused : accepted) += 1;
            }
  // strides and counts at the ends of their types
  const int64_t most = INT64_MAX;
  const splash_rope_desc desc = {4, 0, 1, 1.f, freq, nullptr};
  for (int64_t token : {most, most / 2, (int64_t)4})
    for (int64_t head : {most, most / 2, (int64_t)4}) {
      const splash_rope_view view = {x, x, token, head, token, head, 65536};
      const int st = splash_rope(&view, 1, pos, 1 << 25, 1 << 25, &desc, nullptr);
      if (st != (token == head || (token != 4 && head != 4) ? SPLASH_ERR_INVALID_ARGUMENT : SPLASH_OK)) {
        std::fprintf(stderr, "strides %lld %lld: status %d\n", (long long)token, (long long)head, st);
        return 1;
      }
    }
  // two views of one tensor, and one's result in the place of the other's input
  const splash_rope_view a = {x, x, 16, 4, 16, 4, 4}, b = {far, far, 16, 4, 16, 4, 4}, c = {far, x, 16, 4, 16, 4, 4},
                         none = {x, x, 16, 4, 16, 4, 0};
  const struct {
    splash_rope_view v[2];
    int want;
  } pairs[] = {{{a, b}, SPLASH_OK}, {{a, a}, SPLASH_ERR_INVALID_ARGUMENT}, {{b, c}, SPLASH_ERR_INVALID_ARGUMENT},
               {{c, a}, SPLASH_ERR_INVALID_ARGUMENT}, {{a, none}, SPLASH_OK}};
  for (const auto& p : pairs)
    if (splash_rope(p.v, 2, pos, 3, 3, &desc, nullptr) != p.want) {
      std::fprintf(stderr, "pair %d\n", (int)(&p - pairs));
      return 1;
    }
  std::printf("ok %ld %ld\n", accepted, refused);
  return 0;
}
