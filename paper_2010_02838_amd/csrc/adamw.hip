// AdamW over many tensors in one launch, moments in 32 or in 8 bits.
//
//     g = grad_scale grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g g;  w = w (1 - lr wd) - step m / (sqrt(v) rs + eps)
//
// with step = lr / (1 - b1^t) and rs = 1 / sqrt(1 - b2^t) from the host, in double.  HBM-bound: 28 bytes a parameter with 32-bit moments, 16
// with 8-bit ones, 2 more for the bf16 copy.  One launch whatever the number of tensors: a workgroup takes 1024 or 2048 elements of one tensor and
// finds which in a table in device memory, so that 180 tensors of a Transformer are not 180 launches that each fill part of the chip.  60.9 M parameters:
// 315 to 330 us with 32-bit moments (1.83 GB, 5.5 to 5.8 TB/s), 195 to 205 with 8-bit ones (1.1 GB, 5.3 to 5.6), 65 to 70 to unpack those.
//
// 8-bit moments.  A block of 256 elements (four a lane of one wave) shares a power of two, 2^E, with E the smallest for which no value exceeds
// 1.875 2^E; a value x is stored as the float y = |x| 2^-E with three mantissa bits and exponents from 0 down to -14 (m, beside its sign) or -30 (v), equally
// spaced below.  Scaling by powers of two is exact, so the only rounding is that of the code: the bits of y, moved so that the code's lowest bit is
// bit 20, plus 20 random bits, cut.  Products and sums of m and v are kept unfused: the code then depends on the formula alone, not on
// which products a compiler fuses.
#include "common.h"
#include <math.h>
#include <type_traits>

namespace cd {
namespace {

constexpr int AW_BLOCK = 256;   // elements that share an exponent
constexpr int chunk(int bits) { return bits == 8 ? 2048 : 1024; }   // elements of a workgroup (8 bits: 206 us with 1024, 198 with 2048; 32 bits: 323 and 340)
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

// 32 bits for an element, from its place among all blocks and the step's seed (times 2^32 over the golden ratio, so that seeds in a row begin far apart).  Shifts,
// exclusive ors and products with odd numbers can be undone, so no two places of a step share their bits.  The two multipliers have nothing to them but what was
// measured: over 2^20 numbers every bit of the place flips every bit of the result with a probability of 0.495 to 0.505, and neighbouring places, steps in a row
// and the two halves that m and v are rounded with are correlated by less than 2e-3.
__device__ inline uint32_t random_bits(uint32_t at, uint32_t seed) {
  uint32_t x = at + seed * 0x9E3779B9u;
  x = (x ^ (x >> 16)) * 0x6C8E9CF5u;
  x = (x ^ (x >> 15)) * 0x52DCE729u;
  return x ^ (x >> 16);
}

// STREAM: loads and stores of w, the gradient and the moments bypass the caches, in updates that move more than twice the 256 MB of the memory-side
// cache (as the other updates of this library do).  The bf16 copy, which the next forward pass reads, is stored through them always.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <bool STREAM, typename V> __device__ inline V load_as(const void* p) {
  return STREAM ? __builtin_nontemporal_load(static_cast<const V*>(p)) : *static_cast<const V*>(p);
}
template <bool STREAM, typename V> __device__ inline void store_as(void* p, V v) {
  if (STREAM) __builtin_nontemporal_store(v, static_cast<V*>(p)); else *static_cast<V*>(p) = v;
}
template <bool STREAM> __device__ inline void load4(const float* p, int count, float (&out)[4]) {
  if (count == 4) {
    const u32x4 v = load_as<STREAM, u32x4>(p);
#pragma unroll
    for (int k = 0; k < 4; k++) out[k] = __uint_as_float(v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++) out[k] = k < count ? p[k] : 0.f;
  }
}
template <bool STREAM> __device__ inline void load4(const bf16_t* p, int count, float (&out)[4]) {
  if (count == 4) {
    const u32x2 v = load_as<STREAM, u32x2>(p);
#pragma unroll
    for (int k = 0; k < 4; k++) out[k] = __uint_as_float(k & 1 ? v[k / 2] & 0xffff0000u : v[k / 2] << 16);
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++) out[k] = k < count ? bf16_to_f32(p[k]) : 0.f;
  }
}
template <bool STREAM> __device__ inline void store4(float* p, int count, const float (&in)[4]) {
  if (count == 4) store_as<STREAM, u32x4>(p, u32x4{__float_as_uint(in[0]), __float_as_uint(in[1]), __float_as_uint(in[2]), __float_as_uint(in[3])});
  else
    for (int k = 0; k < count; k++) p[k] = in[k];
}
template <bool STREAM> __device__ inline void store4(bf16_t* p, int count, const float (&in)[4]) {
  if (count == 4)
    store_as<STREAM, u32x2>(p, u32x2{(uint32_t)f32_to_bf16(in[0]) | (uint32_t)f32_to_bf16(in[1]) << 16, (uint32_t)f32_to_bf16(in[2]) | (uint32_t)f32_to_bf16(in[3]) << 16});
  else
    for (int k = 0; k < count; k++) p[k] = f32_to_bf16(in[k]);
}
template <bool STREAM> __device__ inline uint32_t load_codes(const uint8_t* p, int count) {
  if (count == 4) return load_as<STREAM, uint32_t>(p);
  uint32_t u = 0;
  for (int k = 0; k < count; k++) u |= (uint32_t)p[k] << (8 * k);
  return u;
}
template <bool STREAM> __device__ inline void store_codes(uint8_t* p, int count, uint32_t u) {
  if (count == 4) store_as<STREAM, uint32_t>(p, u);
  else
    for (int k = 0; k < count; k++) p[k] = (uint8_t)(u >> (8 * k));
}

// Four elements of a thread: what it loads, and the update of it.
template <typename G, int BITS, bool STREAM> struct Four {
  float w[4], g[4], m[4], v[4];
  uint32_t cm, cv;
  float sm, sv;
  __device__ inline void load(const Entry& t, int64_t i, int count) {
    load4<STREAM>(t.w + i, count, w);
    load4<STREAM>(static_cast<const G*>(t.grad) + i, count, g);
    if constexpr (BITS == 8) {
      cm = load_codes<STREAM>(static_cast<const uint8_t*>(t.m) + i, count);
      cv = load_codes<STREAM>(static_cast<const uint8_t*>(t.v) + i, count);
      const uint8_t* ex = t.exps + 2 * (i / AW_BLOCK);
      sm = block_scale(ex[0]);
      sv = block_scale(ex[1]);   // 0 in a fresh state: zeros
    } else {
      load4<STREAM>(static_cast<const float*>(t.m) + i, count, m);
      load4<STREAM>(static_cast<const float*>(t.v) + i, count, v);
    }
  }
  __device__ inline void update(const StepArgs& a, const Entry& t, int64_t i, int count, float gs, float keep, float step) {
    if constexpr (BITS == 8) {
#pragma unroll
      for (int k = 0; k < 4; k++) {
        m[k] = decode_m((cm >> (8 * k)) & 255u, sm);
        v[k] = decode_v((cv >> (8 * k)) & 255u, sv);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; k++) {
#pragma clang fp contract(off)
      const float gg = a.grad_scale ? g[k] * gs : g[k];
      m[k] = a.b1 * m[k] + a.c1 * gg;
      v[k] = a.b2 * v[k] + a.c2 * gg * gg;
      w[k] = w[k] * keep - step * m[k] / (sqrtf(v[k]) * a.rs + a.eps);
    }
    store4<STREAM>(t.w + i, count, w);
    if (t.lowp) store4<false>(t.lowp + i, count, w);
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
      cm = 0;
      cv = 0;
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const uint32_t rnd = random_bits(at + k, a.seed);
        cm |= (encode(m[k], em, M_TOP, (rnd & 0xffffu) << 4 | 8u) | (m[k] < 0.f ? 128u : 0u)) << (8 * k);
        const uint32_t c = encode(v[k], ev, V_TOP, (rnd >> 16) << 4 | 8u);
        cv |= (c == 0 && v[k] > 0.f ? 1u : c) << (8 * k);
      }
      store_codes<STREAM>(static_cast<uint8_t*>(t.m) + i, count, em == E_NAN ? 0 : cm);
      store_codes<STREAM>(static_cast<uint8_t*>(t.v) + i, count, ev == E_NAN ? 0 : cv);
      uint8_t* ex = t.exps + 2 * (i / AW_BLOCK);
      if ((threadIdx.x & 63) == 0) { ex[0] = (uint8_t)em; ex[1] = (uint8_t)ev; }
    } else {
      store4<STREAM>(static_cast<float*>(t.m) + i, count, m);
      store4<STREAM>(static_cast<float*>(t.v) + i, count, v);
    }
  }
};

// A thread's elements: chunk(BITS) / 1024 groups of four, 1024 apart, so that a wave always has whole blocks.  FULL: all of a wave's are there, so that no
// load waits behind a branch (with a branch for every load the 8-bit update of 60.9 M parameters took 250 us, without 206).  Everything is sent for
// before anything is computed from the table: a workgroup is a chain of latencies, its tensor's number, its tensor, the elements.
template <typename G, int BITS, bool STREAM, bool FULL> __device__ inline void update_chunk(const StepArgs& a, const Entry& t, int64_t i, int64_t block) {
  constexpr int EACH = chunk(BITS) / 1024;
  Four<G, BITS, STREAM> x[EACH];
  int count[EACH];
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    count[e] = FULL ? 4 : (int)max((int64_t)0, min((int64_t)4, t.n - i - 1024 * e));
    if (FULL || block + 1024 * e < t.n) x[e].load(t, i + 1024 * e, count[e]);
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const double lr = a.lr * t.lr_scale;
  const float keep = (float)(1.0 - lr * t.decay), step = (float)(lr / a.bias1);
#pragma unroll
  for (int e = 0; e < EACH; e++)
    if (FULL || block + 1024 * e < t.n) x[e].update(a, t, i + 1024 * e, count[e], gs, keep, step);
}

template <typename G, int BITS, bool STREAM>
__global__ void __launch_bounds__(256) adamw_kernel(StepArgs a) {
  const Entry& t = a.entries[a.owner[blockIdx.x]];
  const int64_t block = (int64_t)(blockIdx.x - t.first_wg) * chunk(BITS) + AW_BLOCK * __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);   // the wave's first
  const int64_t i = block + 4 * (int)(threadIdx.x & 63);
  if (block + chunk(BITS) - 1024 + AW_BLOCK <= t.n) update_chunk<G, BITS, STREAM, true>(a, t, i, block);
  else if (block < t.n) update_chunk<G, BITS, STREAM, false>(a, t, i, block);
}

// The values that 8-bit moments stand for: four significant bits times a power of two, so bf16 holds them exactly.  One half of a workgroup takes m, the
// other v, two times eight elements a thread.
__global__ void __launch_bounds__(256) adamw_unpack_kernel(const Entry* __restrict__ entries, const uint32_t* __restrict__ owner) {
  const Entry& t = entries[owner[blockIdx.x]];
  const int second = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 7);
  const int64_t first = (int64_t)(blockIdx.x - t.first_wg) * chunk(8), i = first + 8 * (int)(threadIdx.x & 127);
  bf16_t* out = second ? t.v_out : t.m_out;
  if (!out) return;
  const uint8_t* codes = static_cast<const uint8_t*>(second ? t.v : t.m);
  auto value = [&](uint32_t c, float scale) { return f32_to_bf16(second ? decode_v(c, scale) : decode_m(c, scale)); };
  auto write = [&](int64_t at, u32x2 u, float scale) {
    u32x4 o;
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const uint32_t two = u[k / 2] >> (16 * (k & 1));
      o[k] = (uint32_t)value(two & 255u, scale) | (uint32_t)value(two >> 8 & 255u, scale) << 16;
    }
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(out + at));
  };
  auto scale_at = [&](int64_t at) { return t.exps[2 * (at / AW_BLOCK) + second]; };
  if (first + chunk(8) <= t.n) {
    const u32x2 u = *reinterpret_cast<const u32x2*>(codes + i), v = *reinterpret_cast<const u32x2*>(codes + i + 1024);
    const int eu = scale_at(i), ev = scale_at(i + 1024);
    write(i, u, block_scale(eu));
    write(i + 1024, v, block_scale(ev));
    return;
  }
  for (int64_t at = i; at < t.n; at += 1024) {
    const float scale = block_scale(scale_at(at));
    if (at + 8 <= t.n) write(at, *reinterpret_cast<const u32x2*>(codes + at), scale);
    else
      for (int k = 0; k < t.n - at; k++) out[at + k] = value(codes[at + k], scale);
    if (at + 1024 >= first + chunk(8)) break;
  }
}

static int count(const char* what, const cd_adamw_tensor* t, int64_t n_tensors, int bits, int64_t* workgroups) {
  CD_REQUIRE(t != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE(n_tensors >= 1 && n_tensors <= INT32_MAX, "%s: n_tensors=%lld out of range", what, (long long)n_tensors);
  int64_t wg = 0;
  for (int64_t i = 0; i < n_tensors; i++) {
    CD_REQUIRE(t[i].n >= 1 && t[i].n <= INT64_MAX / 64, "%s: n=%lld of tensor %lld must be positive", what, (long long)t[i].n, (long long)i);
    wg += cdiv(t[i].n, chunk(bits));
    CD_REQUIRE(wg <= INT32_MAX, "%s: more than 2^31 chunks of %d elements", what, chunk(bits));
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
  if (const int rc = count("adamw_table_bytes", tensors, n_tensors, 32, &wg)) return rc;
  *bytes = align_up(sizeof(Entry) * (size_t)n_tensors + 4 * (size_t)wg, 16);
  return CD_OK;
}

extern "C" int codistill_adamw_table(const cd_adamw_tensor* tensors, int64_t n_tensors, int state_bits, int grad_dtype, void* table, size_t table_bytes,
                                     cd_adamw_plan* plan) {
  CD_REQUIRE(table && plan, "adamw_table: NULL pointer argument");
  CD_REQUIRE(state_bits == 8 || state_bits == 32, "adamw_table: state_bits=%d must be 8 or 32", state_bits);
  CD_REQUIRE(grad_dtype == CD_F32 || grad_dtype == CD_BF16, "adamw_table: unknown grad_dtype %d", grad_dtype);
  int64_t wg = 0;
  if (const int rc = count("adamw_table", tensors, n_tensors, state_bits, &wg)) return rc;
  size_t need = 0;
  codistill_adamw_table_bytes(tensors, n_tensors, &need);
  if (table_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "adamw_table: buffer of %zu bytes, %zu needed", table_bytes, need);
  for (int64_t i = 0; i < n_tensors; i++) {
    const cd_adamw_tensor& t = tensors[i];
    CD_REQUIRE(t.w && t.grad && t.m && t.v && (state_bits == 32 || t.exps), "adamw_table: NULL pointer in tensor %lld", (long long)i);
    const int s = state_bits == 32 ? 16 : 8;
    CD_REQUIRE(aligned16(t.w) && aligned(t.grad, grad_dtype == CD_F32 ? 16 : 8) && aligned(t.lowp, 8) && aligned(t.m, s) && aligned(t.v, s) &&
                   aligned16(t.m_out) && aligned16(t.v_out),
               "adamw_table: tensor %lld: fp32 pointers must be 16-byte aligned, bf16 ones 8 (m_out and v_out 16), 8-bit moments 8", (long long)i);
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
    const int64_t end = first + cdiv(t.n, chunk(state_bits));
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
  const double moved = (10.0 + (plan->grad_dtype == CD_F32 ? 4 : 2) + (plan->state_bits == 32 ? 16 : 4)) * plan->elements;
  ProfScope prof(CD_K_SGD, s, 14.0 * plan->elements, moved);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)plan->workgroups), dim3(256), 0, s, a); };
  auto pick = [&](auto stream_all) {
    constexpr bool S = decltype(stream_all)::value;
    if (plan->grad_dtype == CD_F32) { if (plan->state_bits == 32) run(adamw_kernel<float, 32, S>); else run(adamw_kernel<float, 8, S>); }
    else { if (plan->state_bits == 32) run(adamw_kernel<bf16_t, 32, S>); else run(adamw_kernel<bf16_t, 8, S>); }
  };
  if (moved > (512 << 20)) pick(std::true_type()); else pick(std::false_type());
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
