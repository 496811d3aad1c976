// AdamW over many tensors in one launch, moments in 32 or in 8 bits.
//
//     g = grad_scale grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g g;  w = w (1 - lr wd) - step m / (sqrt(v) rs + eps)
//
// with step = lr / (1 - b1^t) and rs = 1 / sqrt(1 - b2^t) from the host, in double.  HBM-bound: 28 bytes a parameter with 32-bit moments, 16
// with 8-bit ones, 2 more for the bf16 copy.  One launch whatever the number of tensors: a workgroup takes 1024 elements of one tensor and
// finds which in a table in device memory, so that 180 tensors of a Transformer are not 180 launches that each fill part of the chip.
//
// 8-bit moments.  A block of 256 elements (four a lane of one wave) shares a power of two, 2^E, with E the smallest for which no value exceeds
// 1.875 2^E; a value x is stored as the float y = |x| 2^-E with three mantissa bits and exponents from 0 down to -14 (m, beside its sign) or -30 (v), equally
// spaced below.  Scaling by powers of two is exact, so the only rounding is that of the code: the bits of y, moved so that the code's lowest bit is
// bit 20, plus 20 random bits, cut.  Products and sums of m and v are kept unfused: the code then depends on the formula alone, not on
// which products a compiler fuses.
#include "common.h"
#include <math.h>
#include <new>

namespace cd {
namespace {

constexpr int AW_BLOCK = 256;   // elements that share an exponent
constexpr int AW_CHUNK = 1024;  // elements of a workgroup: four blocks
constexpr int M_TOP = 15, V_TOP = 31;   // exponent fields of the top binade
constexpr int E_MIN = 40;       // smallest exponent field of a block: 2^-87
constexpr int E_NAN = 255;      // a block with a value that is not finite

// What the device needs of a tensor, and behind all of them one word a workgroup: the tensor it belongs to.
struct Entry {
  float* w; const void* grad; bf16_t* lowp; void* m; void* v; uint8_t* exps; bf16_t* m_out; bf16_t* v_out;
  int64_t n;
  int64_t first_block;    // blocks of the tensors before this one
  uint32_t first_wg;      // workgroups of the tensors before this one
  float decay, lr_scale;
  uint32_t pad;
};
static_assert(sizeof(Entry) == 96, "table layout");

struct StepArgs {
  const Entry* entries; const uint32_t* owner;
  const float* grad_scale;
  float b1, c1, b2, c2;   // beta, 1 - beta (of the double)
  float rs, eps;
  double lr, bias1;       // 1 - beta1^t
  uint32_t seed;
};

__device__ inline float pow2(int e) { return __uint_as_float((uint32_t)e << 23); }   // 2^(e - 127), 1 <= e <= 254; 0 for the fresh state's 0
__device__ inline float block_scale(int e) { return e == E_NAN ? __uint_as_float(0x7fc00000u) : pow2(e); }

__device__ inline float decode_m(uint32_t code, float scale) {
  const float y = __uint_as_float((code & 127u) << 20) * pow2(254 - M_TOP) * scale;
  return code & 128u ? -y : y;
}
__device__ inline float decode_v(uint32_t code, float scale) { return __uint_as_float(code << 20) * pow2(254 - V_TOP) * scale; }

// exponent field of a block whose largest magnitude has these bits (2^127 and more counts as not finite: its reciprocal is no normal float)
__device__ inline int block_exponent(uint32_t bits) {
  const int e = (int)((bits + 0xfffffu) >> 23);   // (a mantissa above 1.875 carries)
  return bits >= 0x7f800000u || e >= 254 ? E_NAN : e < E_MIN ? E_MIN : e;
}
__device__ inline uint32_t encode(float x, int e, int top, uint32_t rnd) {
  const float y = fabsf(x) * pow2(254 - e) * pow2(top);
  return (__float_as_uint(y) + rnd) >> 20;
}

__device__ inline uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// 32 bits for an element, from its place among all blocks and the step's seed
__device__ inline uint32_t random_bits(uint32_t at, uint32_t seed) {
  uint32_t x = at + seed * 0x9E3779B9u;
  x = (x ^ (x >> 16)) * 0x6C8E9CF5u;
  x = (x ^ (x >> 15)) * 0x52DCE729u;
  return x ^ (x >> 16);
}

template <typename T> __device__ inline void load4(const T* p, int count, float (&out)[4]) {
  if (count == 4) {
    if constexpr (sizeof(T) == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p);
      out[0] = v.x; out[1] = v.y; out[2] = v.z; out[3] = v.w;
    } else {
      const ushort4 v = *reinterpret_cast<const ushort4*>(p);
      out[0] = bf16_to_f32(v.x); out[1] = bf16_to_f32(v.y); out[2] = bf16_to_f32(v.z); out[3] = bf16_to_f32(v.w);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++) out[k] = k < count ? Cvt<T>::ld(p[k]) : 0.f;
  }
}
__device__ inline void store4(float* p, int count, const float (&in)[4]) {
  if (count == 4) *reinterpret_cast<float4*>(p) = make_float4(in[0], in[1], in[2], in[3]);
  else
    for (int k = 0; k < count; k++) p[k] = in[k];
}
__device__ inline void store4(bf16_t* p, int count, const float (&in)[4]) {
  if (count == 4) *reinterpret_cast<ushort4*>(p) = make_ushort4(f32_to_bf16(in[0]), f32_to_bf16(in[1]), f32_to_bf16(in[2]), f32_to_bf16(in[3]));
  else
    for (int k = 0; k < count; k++) p[k] = f32_to_bf16(in[k]);
}
__device__ inline uint32_t load_codes(const uint8_t* p, int count) {
  if (count == 4) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t u = 0;
  for (int k = 0; k < count; k++) u |= (uint32_t)p[k] << (8 * k);
  return u;
}
__device__ inline void store_codes(uint8_t* p, int count, uint32_t u) {
  if (count == 4) *reinterpret_cast<uint32_t*>(p) = u;
  else
    for (int k = 0; k < count; k++) p[k] = (uint8_t)(u >> (8 * k));
}

template <typename G, int BITS>
__global__ void __launch_bounds__(256) adamw_kernel(StepArgs a) {
  const Entry& t = a.entries[a.owner[blockIdx.x]];
  const int64_t i = (int64_t)(blockIdx.x - t.first_wg) * AW_CHUNK + 4 * (int)threadIdx.x;
  // (a wave whose block lies behind the tensor's end leaves whole: i of its first lane is a multiple of the block)
  if (i - 4 * (int)(threadIdx.x & 63) >= t.n) return;
  const int count = (int)max((int64_t)0, min((int64_t)4, t.n - i));
  float w[4], g[4], m[4], v[4];
  load4(t.w + i, count, w);
  load4(static_cast<const G*>(t.grad) + i, count, g);
  uint8_t* mc = static_cast<uint8_t*>(t.m) + i;
  uint8_t* vc = static_cast<uint8_t*>(t.v) + i;
  uint8_t* ex = BITS == 8 ? t.exps + 2 * (i / AW_BLOCK) : nullptr;
  if constexpr (BITS == 8) {
    const uint32_t cm = load_codes(mc, count), cv = load_codes(vc, count);
    const float sm = block_scale(ex[0]), sv = block_scale(ex[1]);   // 0 in a fresh state: zeros
#pragma unroll
    for (int k = 0; k < 4; k++) {
      m[k] = decode_m((cm >> (8 * k)) & 255u, sm);
      v[k] = decode_v((cv >> (8 * k)) & 255u, sv);
    }
  } else {
    load4(static_cast<const float*>(t.m) + i, count, m);
    load4(static_cast<const float*>(t.v) + i, count, v);
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const double lr = a.lr * t.lr_scale;
  const float keep = (float)(1.0 - lr * t.decay), step = (float)(lr / a.bias1);
#pragma unroll
  for (int k = 0; k < 4; k++) {
#pragma clang fp contract(off)
    const float gg = a.grad_scale ? g[k] * gs : g[k];
    m[k] = a.b1 * m[k] + a.c1 * gg;
    v[k] = a.b2 * v[k] + a.c2 * gg * gg;
    w[k] = w[k] * keep - step * m[k] / (sqrtf(v[k]) * a.rs + a.eps);
  }
  store4(t.w + i, count, w);
  if (t.lowp) store4(t.lowp + i, count, w);
  if constexpr (BITS == 8) {
    uint32_t tm = 0, tv = 0;
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (k < count) {   // (magnitudes compared as integers: NaN above infinity above the finite ones)
        tm = max(tm, __float_as_uint(m[k]) & 0x7fffffffu);
        tv = max(tv, __float_as_uint(v[k]) & 0x7fffffffu);
      }
    const int em = block_exponent(wave_max_u32(tm)), ev = block_exponent(wave_max_u32(tv));
    const uint32_t at = (uint32_t)((t.first_block + i / AW_BLOCK) * AW_BLOCK + i % AW_BLOCK);
    uint32_t cm = 0, cv = 0;
    if (em != E_NAN) {
#pragma unroll
      for (int k = 0; k < 4; k++) cm |= (encode(m[k], em, M_TOP, ((random_bits(at + k, a.seed) & 0xffffu) << 4) | 8u) | (m[k] < 0.f ? 128u : 0u)) << (8 * k);
    }
    if (ev != E_NAN) {
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const uint32_t c = encode(v[k], ev, V_TOP, ((random_bits(at + k, a.seed) >> 16) << 4) | 8u);
        cv |= (c == 0 && v[k] > 0.f ? 1u : c) << (8 * k);
      }
    }
    store_codes(mc, count, cm);
    store_codes(vc, count, cv);
    if ((threadIdx.x & 63) == 0) { ex[0] = (uint8_t)em; ex[1] = (uint8_t)ev; }
  } else {
    store4(static_cast<float*>(t.m) + i, count, m);
    store4(static_cast<float*>(t.v) + i, count, v);
  }
}

// the values that 8-bit moments stand for: four significant bits times a power of two, so bf16 holds them exactly
__global__ void __launch_bounds__(256) adamw_unpack_kernel(const Entry* __restrict__ entries, const uint32_t* __restrict__ owner) {
  const Entry& t = entries[owner[blockIdx.x]];
  const int64_t i = (int64_t)(blockIdx.x - t.first_wg) * AW_CHUNK + 4 * (int)threadIdx.x;
  if (i >= t.n) return;
  const int count = (int)min((int64_t)4, t.n - i);
  const uint8_t* ex = t.exps + 2 * (i / AW_BLOCK);
  float x[4];
  if (t.m_out) {
    const uint32_t c = load_codes(static_cast<const uint8_t*>(t.m) + i, count);
    const float s = block_scale(ex[0]);
#pragma unroll
    for (int k = 0; k < 4; k++) x[k] = decode_m((c >> (8 * k)) & 255u, s);
    store4(t.m_out + i, count, x);
  }
  if (t.v_out) {
    const uint32_t c = load_codes(static_cast<const uint8_t*>(t.v) + i, count);
    const float s = block_scale(ex[1]);
#pragma unroll
    for (int k = 0; k < 4; k++) x[k] = decode_v((c >> (8 * k)) & 255u, s);
    store4(t.v_out + i, count, x);
  }
}

static int count(const char* what, const cd_adamw_tensor* t, int64_t n_tensors, int64_t* workgroups) {
  CD_REQUIRE(t != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE(n_tensors >= 1 && n_tensors <= INT32_MAX, "%s: n_tensors=%lld out of range", what, (long long)n_tensors);
  int64_t wg = 0;
  for (int64_t i = 0; i < n_tensors; i++) {
    CD_REQUIRE(t[i].n >= 1 && t[i].n <= INT64_MAX / 64, "%s: n=%lld of tensor %lld must be positive", what, (long long)t[i].n, (long long)i);
    wg += cdiv(t[i].n, AW_CHUNK);
    CD_REQUIRE(wg <= INT32_MAX, "%s: more than 2^31 chunks of %d elements", what, AW_CHUNK);
  }
  *workgroups = wg;
  return CD_OK;
}
static bool aligned(const void* p, int a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_adamw_table_bytes(const cd_adamw_tensor* tensors, int64_t n_tensors, size_t* bytes) {
  CD_REQUIRE(bytes != nullptr, "adamw_table_bytes: output pointer is NULL");
  int64_t wg = 0;
  if (const int rc = count("adamw_table_bytes", tensors, n_tensors, &wg)) return rc;
  *bytes = align_up(sizeof(Entry) * (size_t)n_tensors + 4 * (size_t)wg, 16);
  return CD_OK;
}

extern "C" int codistill_adamw_table(const cd_adamw_tensor* tensors, int64_t n_tensors, int state_bits, int grad_dtype, void* table, size_t table_bytes,
                                     cd_adamw_plan* plan) {
  CD_REQUIRE(table && plan, "adamw_table: NULL pointer argument");
  CD_REQUIRE(state_bits == 8 || state_bits == 32, "adamw_table: state_bits=%d must be 8 or 32", state_bits);
  CD_REQUIRE(grad_dtype == CD_F32 || grad_dtype == CD_BF16, "adamw_table: unknown grad_dtype %d", grad_dtype);
  int64_t wg = 0;
  if (const int rc = count("adamw_table", tensors, n_tensors, &wg)) return rc;
  size_t need = 0;
  codistill_adamw_table_bytes(tensors, n_tensors, &need);
  if (table_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "adamw_table: buffer of %zu bytes, %zu needed", table_bytes, need);
  for (int64_t i = 0; i < n_tensors; i++) {
    const cd_adamw_tensor& t = tensors[i];
    CD_REQUIRE(t.w && t.grad && t.m && t.v && (state_bits == 32 || t.exps), "adamw_table: NULL pointer in tensor %lld", (long long)i);
    const int s = state_bits == 32 ? 16 : 4;
    CD_REQUIRE(aligned16(t.w) && aligned(t.grad, grad_dtype == CD_F32 ? 16 : 8) && aligned(t.lowp, 8) && aligned(t.m, s) && aligned(t.v, s) &&
                   aligned(t.m_out, 8) && aligned(t.v_out, 8),
               "adamw_table: tensor %lld: fp32 pointers must be 16-byte aligned, bf16 ones 8, 8-bit moments 4", (long long)i);
    CD_REQUIRE(t.weight_decay == t.weight_decay && t.lr_scale == t.lr_scale, "adamw_table: NaN weight_decay or lr_scale of tensor %lld", (long long)i);
  }
  Entry* e = static_cast<Entry*>(table);
  uint32_t* owner = reinterpret_cast<uint32_t*>(e + n_tensors);
  cd_adamw_plan p = {};
  int64_t block = 0, first = 0;
  for (int64_t i = 0; i < n_tensors; i++) {
    const cd_adamw_tensor& t = tensors[i];
    e[i] = {t.w, t.grad, static_cast<bf16_t*>(t.lowp), t.m, t.v, t.exps, static_cast<bf16_t*>(t.m_out), static_cast<bf16_t*>(t.v_out), t.n, block,
            (uint32_t)first, t.weight_decay, t.lr_scale, 0};
    block += cdiv(t.n, AW_BLOCK);
    const int64_t end = first + cdiv(t.n, AW_CHUNK);
    for (; first < end; first++) owner[first] = (uint32_t)i;
    p.elements += t.n;
    p.has_out |= t.m_out != nullptr || t.v_out != nullptr;
  }
  p.tensors = n_tensors; p.workgroups = wg; p.state_bits = state_bits; p.grad_dtype = grad_dtype;
  *plan = p;
  return CD_OK;
}

static int check_plan(const char* what, const cd_adamw_plan* p, const void* table) {
  CD_REQUIRE(p && table, "%s: NULL pointer argument", what);
  CD_REQUIRE(p->tensors >= 1 && p->workgroups >= 1 && p->workgroups <= INT32_MAX && (p->state_bits == 8 || p->state_bits == 32) &&
                 (p->grad_dtype == CD_F32 || p->grad_dtype == CD_BF16),
             "%s: the plan was not filled by adamw_table", what);
  CD_REQUIRE(aligned16(table), "%s: the table must be 16-byte aligned", what);
  return CD_OK;
}

extern "C" int codistill_adamw_step(const cd_adamw_plan* plan, const void* device_table, const cd_adamw_cfg* cfg, const float* grad_scale, void* stream) {
  if (const int rc = check_plan("adamw_step", plan, device_table)) return rc;
  CD_REQUIRE(cfg != nullptr, "adamw_step: NULL pointer argument");
  CD_REQUIRE(cfg->t >= 1, "adamw_step: the update counter t=%lld starts at 1", (long long)cfg->t);
  CD_REQUIRE(cfg->lr == cfg->lr && cfg->beta1 >= 0 && cfg->beta1 < 1 && cfg->beta2 >= 0 && cfg->beta2 < 1 && cfg->eps > 0,
             "adamw_step: need 0 <= beta1, beta2 < 1, eps > 0 and no NaN hyper-parameter");
  CD_REQUIRE(aligned(grad_scale, 4), "adamw_step: grad_scale must be 4-byte aligned");
  StepArgs a = {};
  a.entries = static_cast<const Entry*>(device_table);
  a.owner = reinterpret_cast<const uint32_t*>(a.entries + plan->tensors);
  a.grad_scale = grad_scale;
  a.b1 = (float)cfg->beta1; a.c1 = (float)(1.0 - cfg->beta1); a.b2 = (float)cfg->beta2; a.c2 = (float)(1.0 - cfg->beta2);
  a.lr = cfg->lr; a.bias1 = 1.0 - pow(cfg->beta1, (double)cfg->t);
  a.rs = (float)(1.0 / sqrt(1.0 - pow(cfg->beta2, (double)cfg->t)));
  a.eps = (float)cfg->eps;
  a.seed = cfg->seed;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double state = plan->state_bits == 32 ? 16 : 4;
  ProfScope prof(CD_K_SGD, s, 14.0 * plan->elements, (10.0 + (plan->grad_dtype == CD_F32 ? 4 : 2) + state) * plan->elements);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)plan->workgroups), dim3(256), 0, s, a); };
  if (plan->grad_dtype == CD_F32) { if (plan->state_bits == 32) run(adamw_kernel<float, 32>); else run(adamw_kernel<float, 8>); }
  else { if (plan->state_bits == 32) run(adamw_kernel<bf16_t, 32>); else run(adamw_kernel<bf16_t, 8>); }
  return check_launch("adamw_step");
}

extern "C" int codistill_adamw_unpack(const cd_adamw_plan* plan, const void* device_table, void* stream) {
  if (const int rc = check_plan("adamw_unpack", plan, device_table)) return rc;
  CD_REQUIRE(plan->state_bits == 8 && plan->has_out, "adamw_unpack: needs 8-bit moments and somewhere to write their values");
  const Entry* e = static_cast<const Entry*>(device_table);
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_SGD, s, 0, 6.0 * plan->elements);
  hipLaunchKernelGGL(adamw_unpack_kernel, dim3((unsigned)plan->workgroups), dim3(256), 0, s, e, reinterpret_cast<const uint32_t*>(e + plan->tensors));
  return check_launch("adamw_unpack");
}
