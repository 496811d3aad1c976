// Norm of every head's channels with a rotary position behind it, queries and keys in one launch; forward and backward.
//
//     r = 1 / sqrt(mean(x^2) + eps),  xhat = x r,  n = g xhat:    y1 = n1 cos a - n2 sin a,  y2 = n2 cos a + n1 sin a
//     dn = dy turned by -a,  h = g dn:    dx = r (h - xhat mean(h xhat)),    dg = sum over all heads and tokens of dn xhat
//
// HBM-bound: every element is read and written once (backward: two reads, one write), where a norm and a rotation behind each other move twice
// that and round in between.  A head belongs to the fewest lanes (a power of two) that hold it as two runs of V channels, one of its first
// half and one of its second, so that a pair of channels meets in one lane and the head's sum takes a few exchanges inside a wave.  A
// workgroup computes the cosines and sines of its tokens once, into LDS, for all heads of its tensor (queries and keys: twice in all).  dg is summed in registers (a lane meets the same
// channels in every head that it walks), over the workgroup's lanes, and over the workgroups by a second launch, always in the same order.
//
// A workgroup works on one tensor, so that its lanes hold their channels' gains in registers: read again for every head they are as many loads as the heads
// themselves (21.0 us where 17.2 are taken now), from LDS 19.5.
//
// 8192 tokens of 16 + 16 heads of 64 in bf16 (33.6 MB a tensor), tensors that come from memory: forward 17.2 us (3.9 TB/s), backward 25.4 (4.0), the sum over its
// workgroups 4.0; tensors that the caches hold 15 and 23.  Norms and rotation apart take 30.9 and 43.2.  16 tokens of 32 + 8 heads: 4.5, a launch and its latencies.
// The same 8192 tokens in fp32 (134 MB forward, 201 backward), from the caches in part: 27.7 and, with the sum, 45.0.
#include "common.h"
#include "conv_rules.h"
#include "kernels.h"
#include "rotary.h"
#include "vec.h"

namespace cd {
namespace {

constexpr int NR_TOKENS = 8;        // tokens whose angles are in LDS together
constexpr int NR_BLOCKS = 1024;     // most workgroups of the backward pass (and one more for each tensor): rows of partial sums of dg
constexpr int NR_ROWS = NR_BLOCKS + CD_ROPE_MAX_TENSORS;

struct NormRopeTensor {
  const void* x; const void* gain; const void* dy;
  void* out;                        // y, or dx
  float* dgain;
  int64_t x_token, dy_token, out_token;
};
struct NormRopeArgs {
  NormRopeTensor t[CD_ROPE_MAX_TENSORS];
  int32_t heads_end[CD_ROPE_MAX_TENSORS];    // heads of the tensors up to and including this one
  int32_t blocks_end[CD_ROPE_MAX_TENSORS];   // backward: workgroups, likewise
  int32_t n_tensors, dim, n_pairs, block_tokens, lanes;
  int64_t tokens;
  const int32_t* pos;
  float* partial;                            // backward: [workgroups][dim]
  FastDiv by_heads[CD_ROPE_MAX_TENSORS];
  float eps;
  uint64_t freq[CD_ROPE_MAX_PAIRS];          // turns a position, as a fraction of 2^64
  uint8_t axis[CD_ROPE_MAX_PAIRS];
};
static_assert(sizeof(NormRopeArgs) <= 4096, "kernel arguments");

// n / d for n below 2^31
__device__ inline int quotient(int n, FastDiv d) { return (int)div_by((unsigned)n, d); }

struct Angles { float c[NR_TOKENS * CD_ROPE_MAX_PAIRS], s[NR_TOKENS * CD_ROPE_MAX_PAIRS]; };

template <typename T> __device__ inline void fill_angles(const NormRopeArgs& a, Angles& at, int64_t t0, int nt) {
  for (int i = threadIdx.x; i < nt * a.n_pairs; i += 256) {
    const int t = i / a.n_pairs, p = i % a.n_pairs;
    cos_sin<T>(turns(a.pos[(int64_t)a.axis[p] * a.tokens + t0 + t], a.freq[p]), &at.c[t * CD_ROPE_MAX_PAIRS + p], &at.s[t * CD_ROPE_MAX_PAIRS + p]);
  }
}
__device__ inline float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// where run k of lane `sub` lies: two runs of V channels, the second one half a head behind the first (single neighbours: the next channel)
template <int V, bool PAIRS> struct Place {
  int first, second;
  bool live;
  __device__ inline Place(int sub, int k, int lanes, int half) {
    const int s = sub + k * lanes;
    live = s * V < half;
    first = PAIRS && V == 1 ? 2 * s : s * V;
    second = PAIRS && V == 1 ? 2 * s + 1 : half + s * V;
  }
};

// turns the pairs of two runs; channels behind the last pair stay (they are not multiplied by one and zero: zero times an infinity is not zero)
template <int V, bool PAIRS> __device__ inline void turn(float (&u)[V], float (&w)[V], const float* c, const float* s, const Place<V, PAIRS>& at, int n_pairs, float sign) {
  if constexpr (PAIRS && V > 1) {
    auto inside = [&](float (&x)[V], int from) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const int p = (from + e) >> 1;
        if (p < n_pairs) {
          const float x1 = x[e], x2 = x[e + 1], sn = sign * s[p];
          x[e] = x1 * c[p] - x2 * sn;
          x[e + 1] = x2 * c[p] + x1 * sn;
        }
      }
    };
    inside(u, at.first);
    inside(w, at.second);
  } else {
    const int from = PAIRS ? at.first >> 1 : at.first;
#pragma unroll
    for (int e = 0; e < V; e++) {
      const int p = from + e;
      if (p < n_pairs) {
        const float x1 = u[e], x2 = w[e], sn = sign * s[p];
        u[e] = x1 * c[p] - x2 * sn;
        w[e] = x2 * c[p] + x1 * sn;
      }
    }
  }
}

template <typename T, int V> __device__ inline void load_floats(const T* p, float (&out)[V]) {
  T t[V];
  load_run<T, V>(p, t);
#pragma unroll
  for (int e = 0; e < V; e++) out[e] = Cvt<T>::ld(t[e]);
}
template <typename T, int V> __device__ inline void load_gain(const void* gain, int at, float (&out)[V]) {
  if (gain) {
    load_floats<T, V>(static_cast<const T*>(gain) + at, out);
  } else {
#pragma unroll
    for (int e = 0; e < V; e++) out[e] = 1.f;
  }
}

// blockIdx.y: the tensor; x and z: tokens (a launch holds fewer than 2^32 threads along x)
// NV: runs a lane holds of each half (single channels of wide heads: two)
template <typename T, int V, bool PAIRS, int NV>
__global__ void __launch_bounds__(256) norm_rotary_kernel(NormRopeArgs a) {
  __shared__ Angles angles;
  const int64_t t0 = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * a.block_tokens;
  if (t0 >= a.tokens) return;
  const int nt = (int)min((int64_t)a.block_tokens, a.tokens - t0);
  const int sub = threadIdx.x % a.lanes, per_wg = 256 / a.lanes, half = a.dim >> 1, n = blockIdx.y;
  const int heads = a.heads_end[n] - (n ? a.heads_end[n - 1] : 0), all = nt * heads;
  const NormRopeTensor me = a.t[n];
  T x[NV][2][V];
  int t = 0, h = 0;
  // a head is on its way while the one before it is turned, the first one while the angles are computed
  auto fetch = [&](int i) {
    t = quotient(i, a.by_heads[n]);
    h = i - t * heads;
    const T* from = static_cast<const T*>(me.x) + (t0 + t) * me.x_token + (int64_t)h * a.dim;
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const Place<V, PAIRS> at(sub, k, a.lanes, half);
      if (at.live) {
        load_run<T, V>(from + at.first, x[k][0]);
        load_run<T, V>(from + at.second, x[k][1]);
      }
    }
  };
  int i = threadIdx.x / a.lanes;
  if (i < all) fetch(i);
  float gu[NV][V], gw[NV][V];
#pragma unroll
  for (int k = 0; k < NV; k++) {
    const Place<V, PAIRS> at(sub, k, a.lanes, half);
    if (at.live) {
      load_gain<T, V>(me.gain, at.first, gu[k]);
      load_gain<T, V>(me.gain, at.second, gw[k]);
    }
  }
  fill_angles<T>(a, angles, t0, nt);
  __syncthreads();
  while (i < all) {
    float u[NV][V], w[NV][V], sq = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const bool live = Place<V, PAIRS>(sub, k, a.lanes, half).live;
#pragma unroll
      for (int e = 0; e < V; e++) {
        u[k][e] = live ? Cvt<T>::ld(x[k][0][e]) : 0.f;
        w[k][e] = live ? Cvt<T>::ld(x[k][1][e]) : 0.f;
        sq += u[k][e] * u[k][e] + w[k][e] * w[k][e];
      }
    }
    T* const y = static_cast<T*>(me.out) + (t0 + t) * me.out_token + (int64_t)h * a.dim;
    const float *c = angles.c + t * CD_ROPE_MAX_PAIRS, *s = angles.s + t * CD_ROPE_MAX_PAIRS;
    i += per_wg;
    if (i < all) fetch(i);
    const float r = 1.f / sqrtf(lanes_sum(sq, a.lanes) / a.dim + a.eps);
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const Place<V, PAIRS> at(sub, k, a.lanes, half);
      if (!at.live) continue;
#pragma unroll
      for (int e = 0; e < V; e++) {
        u[k][e] *= r * gu[k][e];
        w[k][e] *= r * gw[k][e];
      }
      turn<V, PAIRS>(u[k], w[k], c, s, at, a.n_pairs, 1.f);
      store_run<T, V>(y + at.first, u[k]);
      store_run<T, V>(y + at.second, w[k]);
    }
  }
}

// A workgroup works on one tensor, so that its sums of dg are one gain's.
template <typename T, int V, bool PAIRS, int NV>
__global__ void __launch_bounds__(256) norm_rotary_backward_kernel(NormRopeArgs a) {
  __shared__ Angles angles;
  __shared__ float red[4][2 * CD_ROPE_MAX_PAIRS];
  const int sub = threadIdx.x % a.lanes, per_wg = 256 / a.lanes, half = a.dim >> 1;
  int n = 0;
  while ((int)blockIdx.x >= a.blocks_end[n]) n++;
  const int first_block = n ? a.blocks_end[n - 1] : 0, blocks = a.blocks_end[n] - first_block, heads = a.heads_end[n] - (n ? a.heads_end[n - 1] : 0);
  const NormRopeTensor me = a.t[n];
  float gu[NV][V], gw[NV][V], du[NV][V], dw[NV][V];
#pragma unroll
  for (int k = 0; k < NV; k++) {
    const Place<V, PAIRS> at(sub, k, a.lanes, half);
#pragma unroll
    for (int e = 0; e < V; e++) gu[k][e] = gw[k][e] = du[k][e] = dw[k][e] = 0.f;
    if (at.live) {
      load_gain<T, V>(me.gain, at.first, gu[k]);
      load_gain<T, V>(me.gain, at.second, gw[k]);
    }
  }
  for (int64_t t0 = (int64_t)(blockIdx.x - first_block) * a.block_tokens; t0 < a.tokens; t0 += (int64_t)blocks * a.block_tokens) {
    const int nt = (int)min((int64_t)a.block_tokens, a.tokens - t0);
    __syncthreads();
    fill_angles<T>(a, angles, t0, nt);
    __syncthreads();
    for (int i = threadIdx.x / a.lanes; i < nt * heads; i += per_wg) {
      const int t = i / heads, h = i - t * heads;
      const T* x = static_cast<const T*>(me.x) + (t0 + t) * me.x_token + (int64_t)h * a.dim;
      const T* dy = static_cast<const T*>(me.dy) + (t0 + t) * me.dy_token + (int64_t)h * a.dim;
      T* dx = static_cast<T*>(me.out) + (t0 + t) * me.out_token + (int64_t)h * a.dim;
      float u[NV][V], w[NV][V], p[NV][V], q[NV][V], sq = 0.f, dot = 0.f;
#pragma unroll
      for (int k = 0; k < NV; k++) {
        const Place<V, PAIRS> at(sub, k, a.lanes, half);
#pragma unroll
        for (int e = 0; e < V; e++) u[k][e] = w[k][e] = p[k][e] = q[k][e] = 0.f;
        if (at.live) {
          load_floats<T, V>(x + at.first, u[k]);
          load_floats<T, V>(x + at.second, w[k]);
          load_floats<T, V>(dy + at.first, p[k]);
          load_floats<T, V>(dy + at.second, q[k]);
          turn<V, PAIRS>(p[k], q[k], angles.c + t * CD_ROPE_MAX_PAIRS, angles.s + t * CD_ROPE_MAX_PAIRS, at, a.n_pairs, -1.f);
        }
#pragma unroll
        for (int e = 0; e < V; e++) {
          sq += u[k][e] * u[k][e] + w[k][e] * w[k][e];
          dot += gu[k][e] * p[k][e] * u[k][e] + gw[k][e] * q[k][e] * w[k][e];
        }
      }
      const float r = 1.f / sqrtf(lanes_sum(sq, a.lanes) / a.dim + a.eps);
      const float mean = lanes_sum(dot, a.lanes) * r / a.dim;   // mean(h xhat)
#pragma unroll
      for (int k = 0; k < NV; k++) {
        const Place<V, PAIRS> at(sub, k, a.lanes, half);
#pragma unroll
        for (int e = 0; e < V; e++) {
          const float xu = u[k][e] * r, xw = w[k][e] * r;
          u[k][e] = r * (gu[k][e] * p[k][e] - xu * mean);
          w[k][e] = r * (gw[k][e] * q[k][e] - xw * mean);
          du[k][e] += p[k][e] * xu;
          dw[k][e] += q[k][e] * xw;
        }
        if (at.live) {
          store_run<T, V>(dx + at.first, u[k]);
          store_run<T, V>(dx + at.second, w[k]);
        }
      }
    }
  }
  if (!me.dgain) return;
  // the lanes of a wave that hold the same channels, then the four waves
#pragma unroll
  for (int k = 0; k < NV; k++) {
    const Place<V, PAIRS> at(sub, k, a.lanes, half);
#pragma unroll
    for (int e = 0; e < V; e++) {
      for (int o = a.lanes; o < 64; o *= 2) {
        du[k][e] += __shfl_xor(du[k][e], o, 64);
        dw[k][e] += __shfl_xor(dw[k][e], o, 64);
      }
      if (at.live && (threadIdx.x & 63) < a.lanes) {
        red[threadIdx.x >> 6][at.first + e] = du[k][e];
        red[threadIdx.x >> 6][at.second + e] = dw[k][e];
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < a.dim) a.partial[(int64_t)blockIdx.x * a.dim + threadIdx.x] = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
}

// dg of a tensor: the sum of its workgroups' rows.  A workgroup takes 8 channels, 128 threads each, all loads of a thread in flight at once
constexpr int NR_EACH = (NR_ROWS + 127) / 128;
__global__ void __launch_bounds__(1024) norm_rotary_gain_kernel(NormRopeArgs a) {
  __shared__ float red[16][8];
  const int n = blockIdx.y;
  float* const dgain = a.t[n].dgain;
  if (!dgain) return;
  const int first = n ? a.blocks_end[n - 1] : 0, rows = a.blocks_end[n] - first;
  const int at = threadIdx.x & 7, col = blockIdx.x * 8 + at, part = threadIdx.x >> 3;
  const float* partial = a.partial + (int64_t)first * a.dim;
  float t[NR_EACH], sum = 0.f;
#pragma unroll
  for (int e = 0; e < NR_EACH; e++) t[e] = col < a.dim && part + 128 * e < rows ? partial[(int64_t)(part + 128 * e) * a.dim + col] : 0.f;
#pragma unroll
  for (int e = 0; e < NR_EACH; e++) sum += t[e];
#pragma unroll
  for (int o = 8; o < 64; o *= 2) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][at] = sum;
  __syncthreads();
  if (threadIdx.x < 8 && col < a.dim) {
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 16; q++) s += red[q][at];
    dgain[col] = s;
  }
}

// The longest runs that all heads' halves, pointers and strides are whole in: 16 bytes, 8, or single channels.
struct Runs {
  int64_t mask = 0;   // bytes of all offsets, or-ed
  void add(const void* p, int64_t token, int elem) { mask |= (int64_t)reinterpret_cast<uintptr_t>(p) | token * elem; }
  int bytes(int dim, int elem) const {
    const int64_t m = mask | (int64_t)dim / 2 * elem;
    return m % 16 == 0 ? 16 : m % 8 == 0 ? 8 : elem;
  }
};

template <typename T, bool PAIRS, typename F> static void pick_runs(int bytes, F f) {
  if (bytes == 16) f(std::integral_constant<int, 16 / (int)sizeof(T)>(), std::integral_constant<int, 1>());
  else if (bytes == 8) f(std::integral_constant<int, 8 / (int)sizeof(T)>(), std::integral_constant<int, 1>());
  else f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
}
static int lanes_of(int dim, int elem, int bytes) {
  const int runs = (int)cdiv(dim / 2, bytes / elem);
  int lanes = 1;
  while (lanes < 64 && lanes < runs) lanes *= 2;
  return lanes;
}
static bool whole(const void* p, int elem) { return reinterpret_cast<uintptr_t>(p) % elem == 0; }

static int fill(const char* what, NormRopeArgs& a, const cd_rotary* rope, const int32_t* positions, int64_t tokens, const cd_norm_rotary_tensor* tensors,
                int64_t n_tensors, float eps, bool backward, int* bytes) {
  const int elem = rope->dtype == CD_BF16 ? 2 : 4;
  CD_REQUIRE(eps >= 0.f && eps < __builtin_inff(), "%s: eps must be finite and not negative", what);
  int64_t heads = 0;
  Runs runs;
  for (int64_t i = 0; i < n_tensors; i++) {
    const cd_norm_rotary_tensor& t = tensors[i];
    const void* out = backward ? t.dx : t.y;
    const int64_t out_token = backward ? t.dx_token : t.y_token, dy_token = backward ? t.dy_token : t.x_token;
    CD_REQUIRE((t.x && out && (t.dy || !backward)) || tokens == 0, "%s: NULL pointer in tensor %lld", what, (long long)i);
    CD_REQUIRE(!backward || (t.gain != nullptr) == (t.dgain != nullptr), "%s: tensor %lld has a gain without its gradient, or the gradient alone", what, (long long)i);
    CD_REQUIRE(t.heads >= 1 && t.heads <= 65536, "%s: heads=%lld of tensor %lld out of range", what, (long long)t.heads, (long long)i);
    const int64_t least = t.heads * rope->dim;
    CD_REQUIRE((t.x_token >= least && out_token >= least && dy_token >= least) || tokens <= 1, "%s: a token of tensor %lld is longer than its stride", what, (long long)i);
    CD_REQUIRE(whole(t.x, elem) && whole(out, elem) && whole(t.gain, elem) && (!backward || (whole(t.dy, elem) && whole(t.dgain, 4))),
               "%s: misaligned pointer in tensor %lld", what, (long long)i);
    // a gain may be several tensors', the sums of its gradient are one tensor's each
    for (int64_t j = 0; backward && t.dgain && j < i; j++) {
      const uintptr_t here = reinterpret_cast<uintptr_t>(t.dgain), other = reinterpret_cast<uintptr_t>(tensors[j].dgain), bytes = (uintptr_t)rope->dim * 4;
      CD_REQUIRE(!other || (here < other ? other - here : here - other) >= bytes, "%s: the gains' gradients of tensors %lld and %lld share memory", what, (long long)j, (long long)i);
    }
    // (the stride of a single token is not gone by)
    runs.add(t.x, tokens > 1 ? t.x_token : 0, elem);
    runs.add(out, tokens > 1 ? out_token : 0, elem);
    runs.add(t.gain, 0, elem);
    if (backward) runs.add(t.dy, tokens > 1 ? dy_token : 0, elem);
    heads += t.heads;
    a.heads_end[i] = (int32_t)heads;
    a.t[i] = {t.x, t.gain, backward ? t.dy : nullptr, const_cast<void*>(out), backward ? t.dgain : nullptr, t.x_token, dy_token, out_token};
  }
  if (const int rc = fill_pairs(what, rope, a.freq, a.axis)) return rc;
  *bytes = runs.bytes(rope->dim, elem);
  a.n_tensors = (int32_t)n_tensors; a.dim = rope->dim; a.n_pairs = rope->n_pairs; a.tokens = tokens; a.pos = positions; a.eps = eps;
  a.lanes = lanes_of(rope->dim, elem, *bytes);
  return CD_OK;
}

template <typename F> static void dispatch(const cd_rotary* rope, int bytes, F f) {
  const bool pairs = rope->layout == CD_ROPE_PAIRS;
  auto with = [&](auto type) {
    typedef decltype(type) T;
    if (pairs) pick_runs<T, true>(bytes, [&](auto v, auto nv) { f(type, v, std::true_type(), nv); });
    else pick_runs<T, false>(bytes, [&](auto v, auto nv) { f(type, v, std::false_type(), nv); });
  };
  if (rope->dtype == CD_BF16) with(bf16_t()); else with(float());
}

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_norm_rotary(const cd_rotary* rope, const int32_t* positions, int64_t tokens, const cd_norm_rotary_tensor* tensors, int64_t n_tensors,
                                     float eps, void* stream) {
  CD_REQUIRE(rope && tensors && (positions || tokens == 0), "norm_rotary: NULL pointer argument");
  if (const int rc = check_rope("norm_rotary", rope, positions, tokens, n_tensors)) return rc;
  NormRopeArgs a = {};
  int bytes = 0;
  if (const int rc = fill("norm_rotary", a, rope, positions, tokens, tensors, n_tensors, eps, false, &bytes)) return rc;
  if (tokens == 0) return CD_OK;
  // enough workgroups for two rounds of the chip before a workgroup takes several tokens
  a.block_tokens = (int32_t)(tokens >= 512 * NR_TOKENS ? NR_TOKENS : tokens <= 512 ? 1 : tokens / 512);
  for (int64_t i = 0; i < n_tensors; i++) a.by_heads[i] = fast_div((unsigned)tensors[i].heads);
  const double n = (double)tokens * a.heads_end[n_tensors - 1] * a.dim, elem = rope->dtype == CD_BF16 ? 2 : 4;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_NORM, s, 8 * n, 2 * elem * n);
  const int64_t blocks = cdiv(tokens, a.block_tokens), across = blocks < (1 << 22) ? blocks : 1 << 22;
  const dim3 grid((unsigned)across, (unsigned)n_tensors, (unsigned)cdiv(blocks, across));
  dispatch(rope, bytes, [&](auto type, auto v, auto pairs, auto nv) {
    hipLaunchKernelGGL((norm_rotary_kernel<decltype(type), decltype(v)::value, decltype(pairs)::value, decltype(nv)::value>), grid, dim3(256), 0, s, a);
  });
  return check_launch("norm_rotary");
}

extern "C" int codistill_norm_rotary_workspace_bytes(const cd_rotary* rope, int64_t tokens, int64_t n_tensors, size_t* bytes) {
  CD_REQUIRE(rope && bytes, "norm_rotary_workspace_bytes: NULL pointer argument");
  if (const int rc = check_rope("norm_rotary_workspace_bytes", rope, nullptr, tokens, n_tensors)) return rc;
  *bytes = align_up((size_t)NR_ROWS * rope->dim * 4, 16);
  return CD_OK;
}

extern "C" int codistill_norm_rotary_backward(const cd_rotary* rope, const int32_t* positions, int64_t tokens, const cd_norm_rotary_tensor* tensors,
                                              int64_t n_tensors, float eps, void* workspace, size_t workspace_bytes, void* stream) {
  CD_REQUIRE(rope && tensors && workspace && (positions || tokens == 0), "norm_rotary_backward: NULL pointer argument");
  if (const int rc = check_rope("norm_rotary_backward", rope, positions, tokens, n_tensors)) return rc;
  NormRopeArgs a = {};
  int bytes = 0;
  if (const int rc = fill("norm_rotary_backward", a, rope, positions, tokens, tensors, n_tensors, eps, true, &bytes)) return rc;
  CD_REQUIRE(aligned16(workspace), "norm_rotary_backward: the workspace must be 16-byte aligned");
  size_t need = 0;
  codistill_norm_rotary_workspace_bytes(rope, tokens, n_tensors, &need);
  if (workspace_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "norm_rotary_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  a.partial = static_cast<float*>(workspace);
  // workgroups go to the tensors by their heads
  const int64_t heads = a.heads_end[n_tensors - 1];
  a.block_tokens = (int32_t)(tokens >= 512 * NR_TOKENS ? NR_TOKENS : tokens <= 512 ? 1 : tokens / 512);
  int32_t blocks = 0;
  bool gains = false;
  for (int64_t i = 0; i < n_tensors; i++) {
    const int64_t share = 1 + (int64_t)(NR_BLOCKS) * tensors[i].heads / heads, all = cdiv(tokens, a.block_tokens);
    blocks += (int32_t)(share < all ? share : all);
    a.blocks_end[i] = blocks;
    gains = gains || tensors[i].dgain;
  }
  const double n = (double)tokens * heads * a.dim, elem = rope->dtype == CD_BF16 ? 2 : 4;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_NORM, s, 16 * n, 3 * elem * n);
  if (tokens > 0)
    dispatch(rope, bytes, [&](auto type, auto v, auto pairs, auto nv) {
      hipLaunchKernelGGL((norm_rotary_backward_kernel<decltype(type), decltype(v)::value, decltype(pairs)::value, decltype(nv)::value>), dim3((unsigned)blocks),
                         dim3(256), 0, s, a);
    });
  if (gains) hipLaunchKernelGGL(norm_rotary_gain_kernel, dim3((unsigned)cdiv(a.dim, 8), (unsigned)n_tensors), dim3(1024), 0, s, a);
  return check_launch("norm_rotary_backward");
}
