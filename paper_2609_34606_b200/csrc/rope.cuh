// Rotary positions on the device: the angle of a pair and its sine and cosine.
#pragma once
#include <stdint.h>

#include "hsa_internal.h"

namespace hsa {

struct RopeDev {
  const uint64_t* turns;  // [half] turns per position, as a 64-bit fraction of a turn
  const int32_t* pos;     // [n_axes][tokens] or null: position = token index given by the caller
  int64_t axis_stride;
  int half;               // pairs
  int interleaved;
  int end0, end1;         // pairs before end0 belong to axis 0, before end1 to axis 1, the others to axis 2
  float amplitude;
  float sign;             // +1, or -1 for the transposed rotation
};

// Checks a call's arguments and fills `out`; false where they do not fit.
bool rope_args(const hsa_rope_args* r, int head_dim, int64_t tokens, bool transpose, RopeDev* out);

// Sine and cosine of a fraction of a turn, a / 2^32 (signed or not: whole turns do not matter), each off by little more
// than half a step of fp32.  The nearest quarter turn is taken off in whole numbers, which leaves an eighth of a turn on
// either side, exact to 2^-32 of a turn, as a float x and what x is short of (r and 2 pi / 2^32 both have more than 24
// bits).  The two series are cut behind x^9 and x^10: |x| <= pi/4 leaves x^11 / 11! < 1.8e-9 and x^12 / 12! < 1.2e-10.
__device__ __forceinline__ void sincos_turn(uint32_t a, float* s, float* c) {
  constexpr float kUnit = 1.4629180268e-09f;                                          // 2 pi / 2^32 to 24 bits, and the rest
  constexpr float kRest = static_cast<float>(1.46291807926715968105e-09 - static_cast<double>(kUnit));
  const uint32_t k = (a + 0x20000000u) >> 30;
  const int32_t r = static_cast<int32_t>(a - (k << 30));
  const float rf = static_cast<float>(r);
  const float x = rf * kUnit;
  const float more = fmaf(static_cast<float>(r - static_cast<int32_t>(rf)), kUnit, fmaf(rf, kRest, fmaf(rf, kUnit, -x)));
  const float x2 = x * x;
  float p = 1.f / 362880.f;
  p = fmaf(p, x2, -1.f / 5040.f);
  p = fmaf(p, x2, 1.f / 120.f);
  p = fmaf(p, x2, -1.f / 6.f);
  float q = -1.f / 3628800.f;
  q = fmaf(q, x2, 1.f / 40320.f);
  q = fmaf(q, x2, -1.f / 720.f);
  q = fmaf(q, x2, 1.f / 24.f);
  // sin(x + m) = x + (x^3 p + m (1 - x^2 / 2)),  cos(x + m) = (1 - x^2 / 2) + (x^4 q - x m)
  const float half = 0.5f * x2, w = 1.f - half;
  const float sn = x + fmaf(p * x2, x, more * w);
  const float cs = w + (((1.f - w) - half) + fmaf(q * x2, x2, -x * more) + 0.5f * -fmaf(x, x, -x2));
  const float s0 = (k & 1u) ? cs : sn, c0 = (k & 1u) ? sn : cs;
  *s = (k & 2u) ? -s0 : s0;
  *c = ((k + 1u) & 2u) ? -c0 : c0;
}

// The top 32 bits of position * turns modulo a turn.  Two 32-bit products: the high word of turns times the position
// counts from its low half only.
__device__ __forceinline__ uint32_t turn_of(int32_t pos, uint64_t turns) {
  return static_cast<uint32_t>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * turns) >> 32);
}

__device__ __forceinline__ int rope_axis(const RopeDev& r, int pair) { return pair < r.end0 ? 0 : pair < r.end1 ? 1 : 2; }

// cos and sin of a pair, amplitude and sign included.  `token`: column of pos; `place`: its position where pos is null.
__device__ __forceinline__ float2 rope_cos_sin(const RopeDev& r, int pair, int64_t token, int32_t place) {
  const int32_t at = r.pos ? __ldg(r.pos + rope_axis(r, pair) * r.axis_stride + token) : place;
  float s, c;
  sincos_turn(turn_of(at, __ldg(r.turns + pair)), &s, &c);
  return make_float2(c * r.amplitude, s * (r.amplitude * r.sign));
}

}  // namespace hsa
