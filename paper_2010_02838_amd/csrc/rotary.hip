// Rotary positions with several axes, queries and keys in one launch.
//
//     y1 = x1 cos a - x2 sin a,  y2 = x2 cos a + x1 sin a,  a = position of the pair's axis * frequency of the pair
//
// HBM-bound: every element is read and written once, 3 flops each.  A workgroup takes a few tokens: it first computes the cosines and sines of
// their pairs (once for all heads of all tensors, into LDS), then streams the heads past them in 16-byte vectors.  8192 tokens of 32 heads of 64 in bf16 (67 MB
// moved): 13.0 us, 5.2 TB/s; 16 tokens: 3.8, a launch and its latencies.
#include "common.h"
#include <math.h>

namespace cd {
namespace {

constexpr int RT_MAX_TOKENS = 8;   // tokens of a workgroup

struct RopeArgs {
  const void* x[CD_ROPE_MAX_TENSORS];
  void* y[CD_ROPE_MAX_TENSORS];
  int64_t x_token[CD_ROPE_MAX_TENSORS], y_token[CD_ROPE_MAX_TENSORS];
  int32_t heads_end[CD_ROPE_MAX_TENSORS];   // heads of the tensors up to and including this one
  int32_t n_tensors, dim, n_pairs, block_tokens;
  int64_t tokens;
  const int32_t* pos;
  float sign;
  uint64_t freq[CD_ROPE_MAX_PAIRS];   // turns a position, as a fraction of 2^64
  uint8_t axis[CD_ROPE_MAX_PAIRS];
};
static_assert(sizeof(RopeArgs) <= 4096, "kernel arguments");

// The angle in turns, in [-1/2, 1/2).  A frequency is a 64-bit fraction of a turn, so that whole turns fall out of the integer product; what is lost at any
// position is the rounding to fp32, 2^-25 of a turn, and less than 2^-31 of cut bits.  A single fp32 product is a thousandth of a radian off at 30000 and half
// a turn at 2^24.
__device__ inline float turns(int32_t pos, uint64_t freq) { return (float)(int32_t)(((uint64_t)(int64_t)pos * freq) >> 32) * 0x1p-32f; }

template <typename T, int N> struct Vec { T e[N]; };
template <typename T, int N> __device__ inline Vec<T, N> load_vec(const T* p) {
  Vec<T, N> v;
  if constexpr (N * sizeof(T) == 16) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    __builtin_memcpy(&v, &u, 16);
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) v.e[i] = p[i];
  }
  return v;
}
template <typename T, int N> __device__ inline void store_vec(T* p, const Vec<T, N>& v) {
  if constexpr (N * sizeof(T) == 16) {
    uint4 u;
    __builtin_memcpy(&u, &v, 16);
    *reinterpret_cast<uint4*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = v.e[i];
  }
}

// VEC: elements a load; one pair an item where the tensors do not lie in whole vectors
template <typename T, bool PAIRS, bool VECTOR>
__global__ void __launch_bounds__(256) rotary_kernel(RopeArgs a) {
  constexpr int N = VECTOR ? 16 / (int)sizeof(T) : 1;       // HALVES: pairs an item (two loads of N); PAIRS: N elements an item (or one pair)
  constexpr int P = !VECTOR ? 1 : PAIRS ? N / 2 : N;        // pairs an item
  __shared__ float cs[RT_MAX_TOKENS * CD_ROPE_MAX_PAIRS], sn[RT_MAX_TOKENS * CD_ROPE_MAX_PAIRS];
  const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
  const int nt = (int)min((int64_t)a.block_tokens, a.tokens - t0);
  for (int i = threadIdx.x; i < nt * a.n_pairs; i += 256) {
    const int t = i / a.n_pairs, p = i % a.n_pairs;
    const float r = turns(a.pos[(int64_t)a.axis[p] * a.tokens + t0 + t], a.freq[p]);
    if (sizeof(T) == 2) {   // the instructions take turns; their error, 1e-6, is far below a bf16 rounding
      cs[t * CD_ROPE_MAX_PAIRS + p] = __builtin_amdgcn_cosf(r);
      sn[t * CD_ROPE_MAX_PAIRS + p] = a.sign * __builtin_amdgcn_sinf(r);
    } else {
      cs[t * CD_ROPE_MAX_PAIRS + p] = cospif(2.f * r);
      sn[t * CD_ROPE_MAX_PAIRS + p] = a.sign * sinpif(2.f * r);
    }
  }
  __syncthreads();
  const int half = a.dim >> 1, per_head = half / P, per_token = a.heads_end[a.n_tensors - 1] * per_head;
  for (int i = threadIdx.x; i < nt * per_token; i += 256) {
    const int t = i / per_token, j = i - t * per_token;
    int h = j / per_head;
    const int p = (j - h * per_head) * P;
    int n = 0;
    while (h >= a.heads_end[n]) n++;
    if (n) h -= a.heads_end[n - 1];
    const T* x = static_cast<const T*>(a.x[n]) + (t0 + t) * a.x_token[n] + (int64_t)h * a.dim;
    T* y = static_cast<T*>(a.y[n]) + (t0 + t) * a.y_token[n] + (int64_t)h * a.dim;
    const float* c = cs + t * CD_ROPE_MAX_PAIRS + p;
    const float* s = sn + t * CD_ROPE_MAX_PAIRS + p;
    if constexpr (PAIRS) {
      auto v = load_vec<T, 2 * P>(x + 2 * p);
#pragma unroll
      for (int e = 0; e < P; e++) {
        const float u = Cvt<T>::ld(v.e[2 * e]), w = Cvt<T>::ld(v.e[2 * e + 1]);
        if (p + e < a.n_pairs) {   // (the others are copied: zero times an infinity is no copy)
          v.e[2 * e] = Cvt<T>::st(u * c[e] - w * s[e]);
          v.e[2 * e + 1] = Cvt<T>::st(w * c[e] + u * s[e]);
        }
      }
      store_vec<T, 2 * P>(y + 2 * p, v);
    } else {
      auto v = load_vec<T, P>(x + p), z = load_vec<T, P>(x + half + p);
#pragma unroll
      for (int e = 0; e < P; e++) {
        const float u = Cvt<T>::ld(v.e[e]), w = Cvt<T>::ld(z.e[e]);
        if (p + e < a.n_pairs) {
          v.e[e] = Cvt<T>::st(u * c[e] - w * s[e]);
          z.e[e] = Cvt<T>::st(w * c[e] + u * s[e]);
        }
      }
      store_vec<T, P>(y + p, v);
      store_vec<T, P>(y + half + p, z);
    }
  }
}

// freq / (2 pi) without its whole turns, in units of 2^-64, cut: the number's 53 bits times 1 / (2 pi) to 128 bits, in integers.  (A quotient of doubles is off by
// 2^-53 of itself, at position 2^31 and a thousand radians a position by 4e-5 of a turn.)  |freq| < 2^20.
static uint64_t fraction_of_turn(double freq) {
  int e = 0;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(freq), &e), 53);   // |freq| = m 2^(e - 53)
  const unsigned __int128 low = (unsigned __int128)m * 0x7f09d5f47d4d3770ull, high = (unsigned __int128)m * 0x28be60db9391054aull + (uint64_t)(low >> 64);
  const int shift = 53 - e;   // at least 33: `high` is m / (2 pi) in units of 2^-64
  const uint64_t f = shift < 128 ? (uint64_t)(high >> shift) : 0;
  return freq < 0 ? 0 - f : f;
}

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_rotary(const cd_rotary* rope, const int32_t* positions, int64_t tokens, const cd_rotary_tensor* tensors,
                                int64_t n_tensors, int inverse, void* stream) {
  CD_REQUIRE(rope && tensors && (positions || tokens == 0), "rotary: NULL pointer argument");
  CD_REQUIRE(rope->dtype == CD_F32 || rope->dtype == CD_BF16, "rotary: unknown dtype %d", rope->dtype);
  CD_REQUIRE(rope->dim >= 2 && rope->dim % 2 == 0 && rope->dim <= 2 * CD_ROPE_MAX_PAIRS, "rotary: dim=%d must be even and in 2..%d", rope->dim,
             2 * CD_ROPE_MAX_PAIRS);
  CD_REQUIRE(rope->n_pairs >= 0 && rope->n_pairs <= rope->dim / 2, "rotary: n_pairs=%d of %d", rope->n_pairs, rope->dim / 2);
  CD_REQUIRE(rope->layout == CD_ROPE_HALVES || rope->layout == CD_ROPE_PAIRS, "rotary: unknown layout %d", rope->layout);
  CD_REQUIRE(n_tensors >= 1 && n_tensors <= CD_ROPE_MAX_TENSORS, "rotary: n_tensors=%lld outside 1..%d", (long long)n_tensors, CD_ROPE_MAX_TENSORS);
  CD_REQUIRE(tokens >= 0 && tokens <= INT32_MAX, "rotary: tokens=%lld out of range", (long long)tokens);
  CD_REQUIRE((reinterpret_cast<uintptr_t>(positions) & 3) == 0, "rotary: positions must be 4-byte aligned");
  const int elem = rope->dtype == CD_BF16 ? 2 : 4, vec = 16 / elem;
  RopeArgs a = {};
  // whole vectors: both halves of a head (or the head) are vectors, and so is where every head begins
  bool vector = rope->layout == CD_ROPE_HALVES ? (rope->dim / 2) % vec == 0 : rope->dim % vec == 0;
  int64_t heads = 0, moved = 0;
  for (int64_t i = 0; i < n_tensors; i++) {
    const cd_rotary_tensor& t = tensors[i];
    CD_REQUIRE((t.x && t.y) || tokens == 0, "rotary: NULL pointer in tensor %lld", (long long)i);
    CD_REQUIRE(t.heads >= 1 && t.heads <= 65536, "rotary: heads=%lld of tensor %lld out of range", (long long)t.heads, (long long)i);
    CD_REQUIRE((t.x_token >= t.heads * rope->dim && t.y_token >= t.heads * rope->dim) || tokens <= 1, "rotary: a token of tensor %lld is longer than its stride",
               (long long)i);
    CD_REQUIRE(reinterpret_cast<uintptr_t>(t.x) % elem == 0 && reinterpret_cast<uintptr_t>(t.y) % elem == 0, "rotary: misaligned pointer in tensor %lld", (long long)i);
    vector = vector && aligned16(t.x) && aligned16(t.y) && t.x_token % vec == 0 && t.y_token % vec == 0;
    a.x[i] = t.x; a.y[i] = t.y; a.x_token[i] = t.x_token; a.y_token[i] = t.y_token;
    heads += t.heads;
    a.heads_end[i] = (int32_t)heads;
    moved += 2 * tokens * t.heads * rope->dim * elem;
  }
  for (int p = 0; p < rope->n_pairs; p++) {
    CD_REQUIRE(rope->axis[p] >= 0 && rope->axis[p] < rope->axes && rope->axis[p] < 256, "rotary: axis %d of pair %d outside 0..%d", rope->axis[p], p, rope->axes - 1);
    CD_REQUIRE(isfinite(rope->freq[p]) && fabs(rope->freq[p]) < 1e6, "rotary: frequency of pair %d", p);
    a.freq[p] = fraction_of_turn(rope->freq[p]);
    a.axis[p] = (uint8_t)rope->axis[p];
  }
  if (tokens == 0) return CD_OK;
  a.n_tensors = (int32_t)n_tensors; a.dim = rope->dim; a.n_pairs = rope->n_pairs; a.tokens = tokens; a.pos = positions;
  a.sign = inverse ? -1.f : 1.f;
  // enough workgroups for two rounds of the chip before a workgroup takes several tokens
  a.block_tokens = (int32_t)(tokens >= 512 * RT_MAX_TOKENS ? RT_MAX_TOKENS : tokens <= 512 ? 1 : tokens / 512);
  const dim3 grid((unsigned)cdiv(tokens, a.block_tokens));
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_GLUE, s, 1.5 * moved / elem, (double)moved);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
  const bool pairs = rope->layout == CD_ROPE_PAIRS;
  if (rope->dtype == CD_BF16) {
    if (pairs) { if (vector) run(rotary_kernel<bf16_t, true, true>); else run(rotary_kernel<bf16_t, true, false>); }
    else { if (vector) run(rotary_kernel<bf16_t, false, true>); else run(rotary_kernel<bf16_t, false, false>); }
  } else {
    if (pairs) { if (vector) run(rotary_kernel<float, true, true>); else run(rotary_kernel<float, true, false>); }
    else { if (vector) run(rotary_kernel<float, false, true>); else run(rotary_kernel<float, false, false>); }
  }
  return check_launch("rotary");
}
