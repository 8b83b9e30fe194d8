// The rotary turn of a 64-dim row, an element a lane (gfx950 device code).
#pragma once

#include "layer.hpp"

namespace splash {

// What pair j's angle at token n is made of.
struct PairAngle {
  int32_t position;
  double turns;  // a position
};
__device__ __forceinline__ PairAngle pair_angle(const TurnLaunch& t, int64_t n, int j) {
  const int64_t axis = t.axes > 1 ? t.axis[j] * t.position_stride : 0;
  return {t.positions[axis + n], t.turns[j]};
}

// Its sine and cosine, times the turn's scale.  The angle in turns, position *
// inv_freq / (2 pi), is formed and reduced to [-1/2, 1/2] in 64 bits (in 32, position
// 2^20 would leave 2^-4 rad of it); what is left goes through fp32, 2^-22 or less of a
// pair.
__device__ __forceinline__ void pair_turn(const TurnLaunch& t, PairAngle angle, float& cosine, float& sine) {
  double turns = (double)angle.position * angle.turns;
  turns -= __builtin_rint(turns);
  float s, c;
  sincospif(2.f * (float)turns, &s, &c);
  cosine = c * t.scale;
  sine = s * t.scale;
}

// The pair of element `lane`, and of its row's value the turned one: (a, b) ->
// (a cos - b sin, b cos + a sin) with the pair (2j, 2j + 1) or (j, j + 32).
__device__ __forceinline__ int pair_of(const TurnLaunch& t, int lane) { return t.interleaved ? lane >> 1 : lane & (kRopePairs - 1); }
__device__ __forceinline__ float turn_element(const TurnLaunch& t, int lane, float x, float cosine, float sine) {
  const int apart = t.interleaved ? 1 : kRopePairs;
  const float other = __shfl_xor(x, apart);
  return lane & apart ? x * cosine + other * sine : x * cosine - other * sine;
}

}  // namespace splash
