// Norm of every head's channels behind differential attention, forward and backward.
//
//     y = post g x r,  r = 1 / sqrt(mean(x^2) + eps)
//     h = post g dy,  xhat = x r:   dx = r (h - xhat mean(h xhat)),   dg = post sum over all groups of dy xhat
//
// HBM-bound: the forward pass reads and writes every element once, the backward pass reads two tensors and writes one.  A group of `width`
// channels belongs to the fewest lanes (a power of two) that hold it in registers as 16-byte vectors, so its sums are a few exchanges inside a
// wave.  In the backward pass a lane meets the same channels in every group it walks, so dg is summed in registers, once per workgroup in
// LDS, and over the workgroups by a second launch, always in the same order.
//
// 65536 groups of 128 bf16 channels (16.8 MB a tensor): forward 9.3 us, backward 13.2, the sum over its workgroups 3.9, of which some 3 us each are
// a launch's own (300 rows of 3 groups of 80 take 3.1).
#include "common.h"

namespace cd {
namespace {

constexpr int HN_MAX_WIDTH = 1024;
constexpr int HN_BLOCKS = 1024;   // most workgroups of the backward pass, rows of partial sums of dg: four a compute unit (two: 15.6 us for the groups above)

struct HeadNormArgs {
  const void* x; const void* gain; const void* dy; void* y; void* dx;
  int64_t x_row, y_row, dy_row, dx_row, groups;
  int32_t heads, width, lanes;   // lanes of a group: a power of two up to 64
  float eps, post;
  float* partial;                // backward: [workgroups][width]
};

template <typename T, int N> __device__ inline void load_raw(const T* p, T (&out)[N]) {
  if constexpr (N * sizeof(T) == 16) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    __builtin_memcpy(out, &u, 16);
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) out[i] = p[i];
  }
}
template <typename T, int N> __device__ inline void load_n(const T* p, float (&out)[N]) {
  T t[N];
  load_raw<T, N>(p, t);
#pragma unroll
  for (int i = 0; i < N; i++) out[i] = Cvt<T>::ld(t[i]);
}
template <typename T, int N> __device__ inline void store_n(T* p, const float (&in)[N]) {
  T t[N];
#pragma unroll
  for (int i = 0; i < N; i++) t[i] = Cvt<T>::st(in[i]);
  if constexpr (N * sizeof(T) == 16) {
    uint4 u;
    __builtin_memcpy(&u, t, 16);
    *reinterpret_cast<uint4*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = t[i];
  }
}
// the row of a group (a division of 64 bits is many times one of 32)
__device__ inline int64_t row_of(const HeadNormArgs& a, int64_t i) { return a.groups <= 0xffffffffll ? (uint32_t)i / (uint32_t)a.heads : i / a.heads; }
__device__ inline float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// V: elements a vector (1: element by element), NV: vectors a lane
template <typename T, int V, int NV>
__global__ void __launch_bounds__(256) head_norm_kernel(HeadNormArgs a) {
  const int sub = threadIdx.x % a.lanes, per_wg = 256 / a.lanes;
  float g[NV][V];
#pragma unroll
  for (int k = 0; k < NV; k++) {
    const int c = (sub + k * a.lanes) * V;
#pragma unroll
    for (int e = 0; e < V; e++) g[k][e] = 0.f;
    if (c < a.width) load_n<T, V>(static_cast<const T*>(a.gain) + c, g[k]);
  }
  for (int64_t i = (int64_t)blockIdx.x * per_wg + threadIdx.x / a.lanes; i < a.groups; i += (int64_t)gridDim.x * per_wg) {
    const int64_t row = row_of(a, i), at = (i - row * a.heads) * a.width;
    const T* x = static_cast<const T*>(a.x) + row * a.x_row + at;
    T* y = static_cast<T*>(a.y) + row * a.y_row + at;
    float v[NV][V], sq = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int c = (sub + k * a.lanes) * V;
#pragma unroll
      for (int e = 0; e < V; e++) v[k][e] = 0.f;
      if (c < a.width) load_n<T, V>(x + c, v[k]);
#pragma unroll
      for (int e = 0; e < V; e++) sq += v[k][e] * v[k][e];
    }
    const float r = a.post / sqrtf(lanes_sum(sq, a.lanes) / a.width + a.eps);
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int c = (sub + k * a.lanes) * V;
#pragma unroll
      for (int e = 0; e < V; e++) v[k][e] *= r * g[k][e];
      if (c < a.width) store_n<T, V>(y + c, v[k]);
    }
  }
}

template <typename T, int V, int NV>
__global__ void __launch_bounds__(256) head_norm_backward_kernel(HeadNormArgs a) {
  __shared__ float red[256 * V];
  const int sub = threadIdx.x % a.lanes, per_wg = 256 / a.lanes;
  float g[NV][V], dg[NV][V];
#pragma unroll
  for (int k = 0; k < NV; k++) {
    const int c = (sub + k * a.lanes) * V;
#pragma unroll
    for (int e = 0; e < V; e++) { g[k][e] = 0.f; dg[k][e] = 0.f; }
    if (c < a.width) load_n<T, V>(static_cast<const T*>(a.gain) + c, g[k]);
  }
  const int64_t step = (int64_t)gridDim.x * per_wg;
  // a group's elements are on their way while the one before is worked on
  T xs[NV][V], ds[NV][V];
  T* dx = nullptr;
  auto fetch = [&](int64_t i) {
    const int64_t row = row_of(a, i), at = (i - row * a.heads) * a.width;
    const T* x = static_cast<const T*>(a.x) + row * a.x_row + at;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_row + at;
    dx = static_cast<T*>(a.dx) + row * a.dx_row + at;
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int c = (sub + k * a.lanes) * V;
      if (c < a.width) {
        load_raw<T, V>(x + c, xs[k]);
        load_raw<T, V>(dy + c, ds[k]);
      }
    }
  };
  int64_t i = (int64_t)blockIdx.x * per_wg + threadIdx.x / a.lanes;
  if (i < a.groups) fetch(i);
  for (; i < a.groups; i += step) {
    T* const to = dx;
    float v[NV][V], d[NV][V], sq = 0.f, dot = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const bool live = (sub + k * a.lanes) * V < a.width;
#pragma unroll
      for (int e = 0; e < V; e++) {
        v[k][e] = live ? Cvt<T>::ld(xs[k][e]) : 0.f;
        d[k][e] = live ? Cvt<T>::ld(ds[k][e]) : 0.f;
        sq += v[k][e] * v[k][e];
        dot += g[k][e] * d[k][e] * v[k][e];
      }
    }
    if (i + step < a.groups) fetch(i + step);
    const float r = 1.f / sqrtf(lanes_sum(sq, a.lanes) / a.width + a.eps);
    const float mean = lanes_sum(dot, a.lanes) * r / a.width;   // mean(g dy xhat)
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int c = (sub + k * a.lanes) * V;
      float o[V];
#pragma unroll
      for (int e = 0; e < V; e++) {
        const float xhat = v[k][e] * r;
        o[e] = a.post * r * (g[k][e] * d[k][e] - xhat * mean);
        dg[k][e] += d[k][e] * xhat;
      }
      if (c < a.width) store_n<T, V>(to + c, o);
    }
  }
  // the workgroup's sums: the lanes that hold the same channels, in their order
#pragma unroll
  for (int k = 0; k < NV; k++) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; e++) red[threadIdx.x * V + e] = dg[k][e];
    __syncthreads();
    for (int c = threadIdx.x; c < a.lanes * V; c += 256) {
      float t = 0.f;
      for (int q = 0; q < per_wg; q++) t += red[q * a.lanes * V + c];
      const int col = k * a.lanes * V + c;
      if (col < a.width) a.partial[(int64_t)blockIdx.x * a.width + col] = t;
    }
  }
}

// dg = post * sum of the workgroups' rows: a workgroup takes 8 channels, 128 threads each, all loads of a thread in flight at once
constexpr int HN_EACH = HN_BLOCKS / 128;
__global__ void __launch_bounds__(1024) head_norm_gain_kernel(const float* __restrict__ partial, float* __restrict__ dgain, int rows, int width, float post) {
  __shared__ float red[16][8];
  const int at = threadIdx.x & 7, col = blockIdx.x * 8 + at, part = threadIdx.x >> 3;
  float t[HN_EACH], sum = 0.f;
#pragma unroll
  for (int e = 0; e < HN_EACH; e++) t[e] = col < width && part + 128 * e < rows ? partial[(int64_t)(part + 128 * e) * width + col] : 0.f;
#pragma unroll
  for (int e = 0; e < HN_EACH; e++) sum += t[e];
#pragma unroll
  for (int o = 8; o < 64; o *= 2) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][at] = sum;
  __syncthreads();
  if (threadIdx.x < 8 && col < width) {
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 16; q++) s += red[q][at];
    dgain[col] = post * s;
  }
}

struct Shape { bool vector; int lanes, nv; };
static Shape shape_of(int dtype, int64_t width, bool aligned) {
  Shape s;
  const int v = dtype == CD_BF16 ? 8 : 4;
  s.vector = aligned && width % v == 0;
  const int64_t n = s.vector ? width / v : width;
  s.lanes = 1;
  while (s.lanes < 64 && s.lanes < n) s.lanes *= 2;
  s.nv = (int)cdiv(n, s.lanes);
  return s;
}
static int64_t workgroups(int64_t groups, int lanes, int64_t most) {
  const int64_t n = cdiv(groups, 256 / lanes);
  return n < 1 ? 1 : n < most ? n : most;
}

template <typename T, int V> struct Kernels {
  template <typename F> static void pick(int nv, F f) {   // nv: at most 4 whole vectors (width 1024 of fp32), or 16 single elements
    if constexpr (V > 1) {
      if (nv <= 1) f(std::integral_constant<int, 1>()); else if (nv <= 2) f(std::integral_constant<int, 2>()); else f(std::integral_constant<int, 4>());
    } else {
      if (nv <= 2) f(std::integral_constant<int, 2>()); else f(std::integral_constant<int, 16>());
    }
  }
  static void forward(int nv, dim3 grid, hipStream_t s, const HeadNormArgs& a) {
    pick(nv, [&](auto n) { hipLaunchKernelGGL((head_norm_kernel<T, V, decltype(n)::value>), grid, dim3(256), 0, s, a); });
  }
  static void backward(int nv, dim3 grid, hipStream_t s, const HeadNormArgs& a) {
    pick(nv, [&](auto n) { hipLaunchKernelGGL((head_norm_backward_kernel<T, V, decltype(n)::value>), grid, dim3(256), 0, s, a); });
  }
};

static int check(const char* what, int dtype, int64_t rows, int64_t heads, int64_t width, float eps, float post) {
  CD_REQUIRE(dtype == CD_F32 || dtype == CD_BF16, "%s: unknown dtype %d", what, dtype);
  CD_REQUIRE(rows >= 0 && heads >= 1 && heads <= INT32_MAX && rows <= INT64_MAX / 4096 / heads, "%s: rows=%lld heads=%lld out of range", what, (long long)rows,
             (long long)heads);
  CD_REQUIRE(width >= 1 && width <= HN_MAX_WIDTH, "%s: width=%lld outside 1..%d", what, (long long)width, HN_MAX_WIDTH);
  CD_REQUIRE(eps >= 0.f && eps < __builtin_inff() && post == post, "%s: eps must be finite and not negative, post no NaN", what);
  return CD_OK;
}
static bool fits(const void* p, int elem) { return reinterpret_cast<uintptr_t>(p) % elem == 0; }

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_head_norm(int dtype, const void* x, int64_t x_row, const void* gain, void* y, int64_t y_row, int64_t rows, int64_t heads,
                                   int64_t width, float eps, float post, void* stream) {
  CD_REQUIRE(gain && (rows == 0 || (x && y)), "head_norm: NULL pointer argument");
  if (const int rc = check("head_norm", dtype, rows, heads, width, eps, post)) return rc;
  const int elem = dtype == CD_BF16 ? 2 : 4;
  CD_REQUIRE(fits(x, elem) && fits(gain, elem) && fits(y, elem), "head_norm: misaligned pointer");
  CD_REQUIRE((x_row >= heads * width && y_row >= heads * width) || rows <= 1, "head_norm: a row is longer than its stride");
  if (rows == 0) return CD_OK;
  const bool aligned = aligned16(x) && aligned16(gain) && aligned16(y) && x_row * elem % 16 == 0 && y_row * elem % 16 == 0;
  const Shape sh = shape_of(dtype, width, aligned);
  HeadNormArgs a = {};
  a.x = x; a.gain = gain; a.y = y; a.x_row = x_row; a.y_row = y_row; a.groups = rows * heads;
  a.heads = (int32_t)heads; a.width = (int32_t)width; a.lanes = sh.lanes; a.eps = eps; a.post = post;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_NORM, s, 4.0 * rows * heads * width, 2.0 * elem * rows * heads * width);
  const dim3 grid((unsigned)workgroups(a.groups, sh.lanes, 8192));
  if (dtype == CD_BF16) { if (sh.vector) Kernels<bf16_t, 8>::forward(sh.nv, grid, s, a); else Kernels<bf16_t, 1>::forward(sh.nv, grid, s, a); }
  else { if (sh.vector) Kernels<float, 4>::forward(sh.nv, grid, s, a); else Kernels<float, 1>::forward(sh.nv, grid, s, a); }
  return check_launch("head_norm");
}

extern "C" int codistill_head_norm_workspace_bytes(int64_t rows, int64_t heads, int64_t width, size_t* bytes) {
  CD_REQUIRE(bytes != nullptr, "head_norm_workspace_bytes: output pointer is NULL");
  if (const int rc = check("head_norm_workspace_bytes", CD_F32, rows, heads, width, 0.f, 1.f)) return rc;
  *bytes = (size_t)HN_BLOCKS * width * 4;
  return CD_OK;
}

extern "C" int codistill_head_norm_backward(int dtype, const void* x, int64_t x_row, const void* gain, const void* dy, int64_t dy_row, void* dx,
                                            int64_t dx_row, float* dgain, int64_t rows, int64_t heads, int64_t width, float eps, float post,
                                            void* workspace, size_t workspace_bytes, void* stream) {
  CD_REQUIRE(gain && dgain && workspace && (rows == 0 || (x && dy && dx)), "head_norm_backward: NULL pointer argument");
  if (const int rc = check("head_norm_backward", dtype, rows, heads, width, eps, post)) return rc;
  const int elem = dtype == CD_BF16 ? 2 : 4;
  CD_REQUIRE(fits(x, elem) && fits(gain, elem) && fits(dy, elem) && fits(dx, elem) && fits(dgain, 4) && aligned16(workspace), "head_norm_backward: misaligned pointer");
  CD_REQUIRE((x_row >= heads * width && dy_row >= heads * width && dx_row >= heads * width) || rows <= 1, "head_norm_backward: a row is longer than its stride");
  size_t need = 0;
  codistill_head_norm_workspace_bytes(rows, heads, width, &need);
  if (workspace_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "head_norm_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  const bool aligned = aligned16(x) && aligned16(gain) && aligned16(dy) && aligned16(dx) && x_row * elem % 16 == 0 && dy_row * elem % 16 == 0 &&
                       dx_row * elem % 16 == 0;
  const Shape sh = shape_of(dtype, width, aligned);
  HeadNormArgs a = {};
  a.x = x; a.gain = gain; a.dy = dy; a.dx = dx; a.x_row = x_row; a.dy_row = dy_row; a.dx_row = dx_row; a.groups = rows * heads;
  a.heads = (int32_t)heads; a.width = (int32_t)width; a.lanes = sh.lanes; a.eps = eps; a.post = post;
  a.partial = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_NORM, s, 12.0 * rows * heads * width, 3.0 * elem * rows * heads * width);
  const dim3 grid((unsigned)workgroups(a.groups, sh.lanes, HN_BLOCKS));
  if (dtype == CD_BF16) { if (sh.vector) Kernels<bf16_t, 8>::backward(sh.nv, grid, s, a); else Kernels<bf16_t, 1>::backward(sh.nv, grid, s, a); }
  else { if (sh.vector) Kernels<float, 4>::backward(sh.nv, grid, s, a); else Kernels<float, 1>::backward(sh.nv, grid, s, a); }
  hipLaunchKernelGGL(head_norm_gain_kernel, dim3((unsigned)cdiv(width, 8)), dim3(1024), 0, s, a.partial, dgain, (int)grid.x, (int)width, post);
  return check_launch("head_norm");
}
