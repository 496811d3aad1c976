// Angles of rotary positions, for the kernels that turn channels.
#pragma once
#include "common.h"
#include <math.h>

namespace cd {

// The angle in turns, in [-1/2, 1/2).  A frequency is a 64-bit fraction of a turn, so that whole turns fall out of the integer product; what is lost at any
// position is the rounding to fp32, 2^-25 of a turn, and less than 2^-31 of cut bits.  A single fp32 product is a thousandth of a radian off at 30000 and half
// a turn at 2^24.
__device__ static inline float turns(int32_t pos, uint64_t freq) { return (float)(int32_t)(((uint64_t)(int64_t)pos * freq) >> 32) * 0x1p-32f; }

template <typename T> __device__ static inline void cos_sin(float r, float* c, float* s) {
  if (sizeof(T) == 2) {   // the instructions take turns; their error, 1e-6, is far below a bf16 rounding
    *c = __builtin_amdgcn_cosf(r);
    *s = __builtin_amdgcn_sinf(r);
  } else {
    *c = cospif(2.f * r);
    *s = sinpif(2.f * r);
  }
}

// freq / (2 pi) without its whole turns, in units of 2^-64, cut: the number's 53 bits times 1 / (2 pi) to 128 bits, in integers.  (A quotient of doubles is off by
// 2^-53 of itself, at position 2^31 and a thousand radians a position by 4e-5 of a turn.)  |freq| < 2^20.
static inline uint64_t fraction_of_turn(double freq) {
  int e = 0;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(freq), &e), 53);   // |freq| = m 2^(e - 53)
  const unsigned __int128 low = (unsigned __int128)m * 0x7f09d5f47d4d3770ull, high = (unsigned __int128)m * 0x28be60db9391054aull + (uint64_t)(low >> 64);
  const int shift = 53 - e;   // at least 33: `high` is m / (2 pi) in units of 2^-64
  const uint64_t f = shift < 128 ? (uint64_t)(high >> shift) : 0;
  return freq < 0 ? 0 - f : f;
}

static inline int check_rope(const char* what, const cd_rotary* rope, const int32_t* positions, int64_t tokens, int64_t n_tensors) {
  CD_REQUIRE(rope->dtype == CD_F32 || rope->dtype == CD_BF16, "%s: unknown dtype %d", what, rope->dtype);
  CD_REQUIRE(rope->dim >= 2 && rope->dim % 2 == 0 && rope->dim <= 2 * CD_ROPE_MAX_PAIRS, "%s: dim=%d must be even and in 2..%d", what, rope->dim,
             2 * CD_ROPE_MAX_PAIRS);
  CD_REQUIRE(rope->n_pairs >= 0 && rope->n_pairs <= rope->dim / 2, "%s: n_pairs=%d of %d", what, rope->n_pairs, rope->dim / 2);
  CD_REQUIRE(rope->layout == CD_ROPE_HALVES || rope->layout == CD_ROPE_PAIRS, "%s: unknown layout %d", what, rope->layout);
  CD_REQUIRE(n_tensors >= 1 && n_tensors <= CD_ROPE_MAX_TENSORS, "%s: n_tensors=%lld outside 1..%d", what, (long long)n_tensors, CD_ROPE_MAX_TENSORS);
  CD_REQUIRE(tokens >= 0 && tokens <= INT32_MAX, "%s: tokens=%lld out of range", what, (long long)tokens);
  CD_REQUIRE((reinterpret_cast<uintptr_t>(positions) & 3) == 0, "%s: positions must be 4-byte aligned", what);
  return CD_OK;
}
// frequencies and axes of the pairs, as the kernels take them
static inline int fill_pairs(const char* what, const cd_rotary* rope, uint64_t* freq, uint8_t* axis) {
  for (int p = 0; p < rope->n_pairs; p++) {
    CD_REQUIRE(rope->axis[p] >= 0 && rope->axis[p] < rope->axes && rope->axis[p] < 256, "%s: axis %d of pair %d outside 0..%d", what, rope->axis[p], p, rope->axes - 1);
    CD_REQUIRE(isfinite(rope->freq[p]) && fabs(rope->freq[p]) < 1e6, "%s: frequency of pair %d", what, p);
    freq[p] = fraction_of_turn(rope->freq[p]);
    axis[p] = (uint8_t)rope->axis[p];
  }
  return CD_OK;
}

}  // namespace cd
