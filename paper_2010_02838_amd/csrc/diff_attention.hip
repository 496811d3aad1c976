// Differential attention, forward and backward.
//
//     P_m = softmax over the visible keys of scale q_m . k_m  (m = 1, 2),   out = (P_1 - lambda P_2) v
//
// One pass over the keys, with a running maximum and sum for each of the two maps and two accumulators: both maps are weights of the same
// values, so every fragment of v that leaves LDS feeds two products, and nothing of size queries x keys is stored.  Backward, from the kept
// log-sums of both maps:
//
//     dP = dO v^T (one product for both maps),  delta_m = rowsum(P_m dP),  dS_1 = P_1 (dP - delta_1),  dS_2 = -lambda P_2 (dP - delta_2)
//     dq_m = scale dS_m k_m,  dk_m = scale dS_m^T q_m,  dv = (P_1 - lambda P_2)^T dO,  dlambda = -delta_2
//
// in two kernels, one that owns queries (dq, delta, dlambda) and one that owns keys (dk, dv); neither adds into memory that another
// workgroup writes, so the same inputs give the same bits.
//
// Rows.  The queries of all heads that share a key head are rows of one product: row r of a sequence is query r / group of head
// r % group.  A gradient of a shared key head is then one sum over rows, and a single new token of a decoder still fills a tile with
// its heads.
//
// Tiles.  32x32 products (v_mfma_f32_32x32x16_bf16, or eight v_mfma_f32_32x32x2_f32 on the same fragments): lane l holds row or column l % 32
// and the contraction elements 8 (l / 32) .. + 7 of 16, and of the result column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 in register i.  A
// wave owns 32 rows (or keys) on its lanes as the second operand, so that whatever belongs to a row is one value a lane, and a score
// tile, rounded, is the second operand of the next product as it lies: its contraction order 8 (e / 4) + 4 (l / 32) + e % 4 is the order
// in which the first operand, the streamed tensor transposed, is read from LDS.
#include "common.h"
#include "kernels.h"
#include <math.h>

namespace cd {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct DiffArgs {
  const void* q; const void* k; const void* v; const float* lam;
  void* out; void* o2; float* lse;
  const void* dout; void* dq; void* dk; void* dv; float* dlam;
  float* delta;                                   // backward: [2][heads][q rows]
  float* part; float* part_ml;                    // forward over parts of the keys: unnormalised sums and (maximum, sum) of a part
  int64_t q_token, q_batch, k_token, k_batch, v_token, v_batch, o_token, o_batch, o2_token;
  const int32_t* q_lens; const int32_t* k_lens; const int32_t* q_starts; const int32_t* k_starts;
  int64_t q_rows, k_rows;                         // rows of the q and k tensors (batch * tq when padded)
  int32_t batch, tq, tk, heads, kv_heads, group, dim, causal, lam_token, parts, tiles, units;
  uint32_t group_inv;                             // floor(2^32 / group) + 1 (group > 1)
  float scale, c;                                 // c = scale log2(e)
};

// ---- fragments ----------------------------------------------------------------------------------------------------------
template <typename T> struct Ops;
template <> struct Ops<bf16_t> {
  typedef v8bf Frag;
  static constexpr int VE = 8;   // elements of 16 bytes
  static __device__ inline Frag load(const bf16_t* p) { return __builtin_bit_cast(v8bf, *reinterpret_cast<const uint4*>(p)); }
  static __device__ inline Frag zero() { return __builtin_bit_cast(v8bf, make_uint4(0, 0, 0, 0)); }
  static __device__ inline v16f mma(const Frag& a, const Frag& b, const v16f& c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ inline float get(const Frag& f, int i) { return (float)f[i]; }
  // registers 8 u .. 8 u + 7 of a tile as a second operand
  static __device__ inline Frag operand(const v16f& d, int u) {
    v8bf f;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const v2f two = {d[8 * u + 2 * e], d[8 * u + 2 * e + 1]};
      const v2bf r = __builtin_convertvector(two, v2bf);
      f[2 * e] = r[0];
      f[2 * e + 1] = r[1];
    }
    return f;
  }
  // rows row0 .. row0 + 15 of a row-major copy as contraction, columns col0 .. col0 + 31 on the lanes.  In a group of 16 lanes, lane i of a
  // transposing load receives element i & 3 of the four 8-byte pieces that lanes i >> 2, 4 + (i >> 2), ... address.
  template <int PITCH> static __device__ inline Frag transposed(const bf16_t* t, int col0, int row0, int lane) {
    const int grp = lane >> 4, li = lane & 15;
    typedef __attribute__((address_space(3))) v4bf lds4;
    const bf16_t* p = t + (row0 + 4 * (grp >> 1) + (li >> 2)) * PITCH + col0 + 16 * (grp & 1) + 4 * (li & 3);
    const v4bf lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)p);
    const v4bf hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p + 8 * PITCH));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ inline void store4(bf16_t* p, float a, float b, float c, float d) {
    const v2f lo = {a, b}, hi = {c, d};
    uint2 u;
    u.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, v2bf));
    u.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, v2bf));
    *reinterpret_cast<uint2*>(p) = u;
  }
};
template <> struct Ops<float> {
  typedef v8f Frag;
  static constexpr int VE = 4;
  static __device__ inline Frag load(const float* p) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    return Frag{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  }
  static __device__ inline Frag zero() { return Frag{0, 0, 0, 0, 0, 0, 0, 0}; }
  static __device__ inline v16f mma(const Frag& a, const Frag& b, v16f c) {
#pragma unroll
    for (int j = 0; j < 8; j++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ inline float get(const Frag& f, int i) { return f[i]; }
  static __device__ inline Frag operand(const v16f& d, int u) {
    Frag f;
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = d[8 * u + e];
    return f;
  }
  template <int PITCH> static __device__ inline Frag transposed(const float* t, int col0, int row0, int lane) {
    const float* p = t + (row0 + 4 * (lane >> 5)) * PITCH + col0 + (lane & 31);
    Frag f;
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = p[(8 * (e >> 2) + (e & 3)) * PITCH];
    return f;
  }
  static __device__ inline void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
};

// Sizes of an instance: DT = head_dim rounded up to 32, 64 or 128, rows of 2 DT elements in LDS (both maps, or the values), KC streamed rows at
// a time, 16 bytes of padding a row so that 16-byte reads of many rows spread over the banks.
template <typename T, int DT> struct Sizes {
  static constexpr int W = 2 * DT, PITCH = W + Ops<T>::VE, KC = 32;
  static constexpr int KS = DT / 16, VT = W / 32, DTT = DT / 32;
};
constexpr int EXACT_KEYS = 128;   // rows that reach no more keys than this get their deltas in a pass of their own
constexpr int ROWS = 128;   // rows (or keys) of a workgroup: four waves of 32

// ---- sequences and rows ---------------------------------------------------------------------------------------------------
struct Seq { int nq, nk; int64_t q0, k0; };   // lengths; rows of the sequence's first query and key in their tensors
__device__ inline Seq sequence(const DiffArgs& a, int b) {
  Seq s;
  if (a.q_starts) {
    const int64_t qs = min(max((int64_t)a.q_starts[b], (int64_t)0), a.q_rows), ks = min(max((int64_t)a.k_starts[b], (int64_t)0), a.k_rows);
    s.q0 = qs; s.k0 = ks;
    s.nq = (int)min(min((int64_t)a.q_starts[b + 1], a.q_rows) - qs, (int64_t)a.tq);
    s.nk = (int)min(min((int64_t)a.k_starts[b + 1], a.k_rows) - ks, (int64_t)a.tk);
    s.nq = max(s.nq, 0);
    s.nk = max(s.nk, 0);
  } else {
    s.q0 = (int64_t)b * a.tq; s.k0 = (int64_t)b * a.tk;
    s.nq = a.q_lens ? min(max(a.q_lens[b], 0), a.tq) : a.tq;
    s.nk = a.k_lens ? min(max(a.k_lens[b], 0), a.tk) : a.tk;
  }
  return s;
}
// first element of a sequence's rows
template <typename T> __device__ inline T* rows_of(const DiffArgs& a, T* p, int b, int64_t first, int64_t token, int64_t batch) {
  return p + (a.q_starts ? first * token : b * batch);
}
__device__ inline int query_of(const DiffArgs& a, int r) { return a.group == 1 ? r : (int)__umulhi((uint32_t)r, a.group_inv); }

// Workgroups go to the eight L2 caches in turn; each cache gets a run of neighbours in the order (unit, tile), which share their keys.  Under a
// causal mask the run's units are taken in turns, so that the long tiles of all of them start before the short ones.
__device__ inline int work_index(int n, int per_unit, bool turns) {
  const int per = (n + 7) >> 3, at = (int)(blockIdx.x >> 3);
  int x = at;
  if (turns) {
    const int units = per / per_unit;
    if (units > 1 && units * per_unit == per) x = at % units * per_unit + at / units;
  }
  return (int)(blockIdx.x & 7) * per + x;
}
static unsigned work_blocks(int64_t n) { return (unsigned)(cdiv(n, 8) * 8); }

// Up to KC rows of 2 dim elements (two ranges of dim for the maps, MAPS, or one of 2 dim) on their way into LDS; what lies beyond the rows and the
// channels becomes zero.  `at(r)` is the address of row r < n.
template <typename T, int DT, bool MAPS, int THREADS = 256> struct Stage {
  typedef Sizes<T, DT> S;
  static constexpr int VE = Ops<T>::VE, VPR = S::W / VE, IT = S::KC * VPR / THREADS;
  uint4 u[IT];
  template <typename At> __device__ inline void load(int n, int dim, At at) {
#pragma unroll
    for (int i = 0; i < IT; i++) {
      const int x = threadIdx.x + THREADS * i, r = x / VPR, c = (x % VPR) * VE;
      u[i] = make_uint4(0, 0, 0, 0);
      const int cc = MAPS ? (c >= DT ? c - DT : c) : c;
      const bool in = r < n && cc < (MAPS ? dim : 2 * dim);
      if (in) u[i] = *reinterpret_cast<const uint4*>(at(r) + (MAPS && c >= DT ? dim + cc : cc));
    }
  }
  __device__ inline void store(T* dst) const {
#pragma unroll
    for (int i = 0; i < IT; i++) {
      const int x = threadIdx.x + THREADS * i, r = x / VPR, c = (x % VPR) * VE;
      *reinterpret_cast<uint4*>(dst + r * S::PITCH + c) = u[i];
    }
  }
};

// The fragments of a row of 2 dim elements that a lane owns.
template <typename T, int DT> using RowFrags = typename Ops<T>::Frag[Sizes<T, DT>::W / 16];
template <typename T, int DT, bool MAPS>
__device__ inline void own_row(RowFrags<T, DT>& f, const T* row, bool live, int dim, int hh) {
#pragma unroll
  for (int t = 0; t < Sizes<T, DT>::W / 16; t++) {
    const int c = 16 * t + 8 * hh, cc = MAPS && c >= DT ? c - DT : c;
    f[t] = Ops<T>::zero();
    if (live && cc < (MAPS ? dim : 2 * dim)) f[t] = Ops<T>::load(row + (MAPS && c >= DT ? dim + cc : cc));
  }
}

__device__ inline void clear(v16f& t) {
#pragma unroll
  for (int i = 0; i < 16; i++) t[i] = 0.f;
}
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float other_half(float v) { return __shfl_xor(v, 32, 64); }
__device__ inline float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// ---- forward -------------------------------------------------------------------------------------------------------------------
// A wave owns 32 rows of one of the two maps; the waves of a pair exchange their results at the end.  (Both maps in one wave share the fragments of
// v, but need 256 accumulators for the widest heads, which spill, and 128 for heads of 64, which leave two waves a SIMD and nothing in
// flight beside them.)
constexpr int F_GROUPS = 2, F_ROWS = 32 * F_GROUPS, F_THREADS = 128 * F_GROUPS;

template <typename T, int DT>
__global__ void __launch_bounds__(F_THREADS, sizeof(T) == 4 ? (DT == 128 ? 1 : 2) : DT == 128 ? 2 : 3) diff_forward_kernel(DiffArgs a) {
  typedef Ops<T> O;
  typedef Sizes<T, DT> S;
  __shared__ __attribute__((aligned(16))) T lds[4 * S::KC * S::PITCH];   // keys and values, two buffers each
  constexpr int BUF = S::KC * S::PITCH;
  const int total = a.units * a.tiles * a.parts;
  const int w = work_index(total, a.tiles * a.parts, a.causal);
  if (w >= total) return;
  const int part = w % a.parts, ut = w / a.parts, unit = ut / a.tiles;
  const int tile = a.tiles - 1 - ut % a.tiles;   // under a causal mask the last rows see the most keys: they go first
  const int b = unit / a.kv_heads, hk = unit % a.kv_heads;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.group, r0 = tile * F_ROWS, room = a.q_starts ? R : a.tq * a.group;
  if (r0 >= room) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 31, hh = lane >> 5, m = wave & 1, rg = wave >> 1;
  const int wr0 = r0 + 32 * rg, r = wr0 + c;
  const bool live = r < R;
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group);
  const T* kp = rows_of(a, static_cast<const T*>(a.k), b, s.k0, a.k_token, a.k_batch) + (int64_t)hk * 2 * a.dim;
  const T* vp = rows_of(a, static_cast<const T*>(a.v), b, s.k0, a.v_token, a.v_batch) + (int64_t)hk * 2 * a.dim;
  typename O::Frag qf[S::KS];
  {
    const T* qp = rows_of(a, static_cast<const T*>(a.q), b, s.q0, a.q_token, a.q_batch) + i * a.q_token + (int64_t)h * 2 * a.dim + m * a.dim;
#pragma unroll
    for (int t = 0; t < S::KS; t++) {
      qf[t] = O::zero();
      if (live && 16 * t + 8 * hh < a.dim) qf[t] = O::load(qp + 16 * t + 8 * hh);
    }
  }
  // keys this row sees, and those that the rows of the wave and of the workgroup reach
  const int off = s.nk - s.nq;
  auto limit = [&](int row) { return a.causal ? min(s.nk, query_of(a, row) + off + 1) : s.nk; };
  // (the keys of a part: whole tiles of 32)
  const int per = a.parts == 1 ? s.nk : (((s.nk + 31) / 32 + a.parts - 1) / a.parts) * 32;
  const int begin = part * per, last = r0 < R ? min(limit(min(r0 + F_ROWS, R) - 1), begin + per) : 0;
  const int see = min(live ? limit(r) : s.nk, last), least = min(limit(wr0), last), reach = wr0 < R ? min(limit(min(wr0 + 31, R - 1)), last) : 0;
  v16f o[S::VT];
#pragma unroll
  for (int t = 0; t < S::VT; t++) clear(o[t]);
  float mx = -INFINITY, sum = 0.f;
  // One barrier a tile: while a tile of keys and values is worked on, the next one is written to the other buffer and the one after it is
  // on its way into registers.
  Stage<T, DT, true, F_THREADS> ks;
  Stage<T, DT, false, F_THREADS> vs;
  auto fetch = [&](int j) {
    ks.load(min(S::KC, s.nk - j), a.dim, [&](int row) { return kp + (int64_t)(j + row) * a.k_token; });
    vs.load(min(S::KC, s.nk - j), a.dim, [&](int row) { return vp + (int64_t)(j + row) * a.v_token; });
  };
  if (begin < last) {
    fetch(begin);
    ks.store(lds);
    vs.store(lds + 2 * BUF);
    if (begin + S::KC < last) fetch(begin + S::KC);
  }
  __syncthreads();
  for (int j0 = begin, buf = 0; j0 < last; j0 += S::KC, buf ^= 1) {
    const T* Ks = lds + buf * BUF;
    const T* Vs = lds + (2 + buf) * BUF;
    if (j0 < reach) {
      v16f sc;
      clear(sc);
#pragma unroll
      for (int t = 0; t < S::KS; t++) sc = O::mma(O::load(Ks + c * S::PITCH + m * DT + 16 * t + 8 * hh), qf[t], sc);
      if (j0 + 32 > least) {   // some row of the wave does not see all of the tile
#pragma unroll
        for (int v = 0; v < 16; v++)
          if (j0 + 8 * (v >> 2) + 4 * hh + (v & 3) >= see) sc[v] = -INFINITY;
      }
      float top = sc[0];
#pragma unroll
      for (int v = 1; v < 16; v++) top = fmaxf(top, sc[v]);
      top *= a.c;
      // The maximum is only raised, and what has been summed only rescaled, when a score exceeds it by 2^8: weights up to 256 round as well
      // as weights up to 1, and after the first tiles this is rare.
      if (__any(top > mx + 8.f)) {
        const float now = fmaxf(mx, fmaxf(top, other_half(top)));
        const float f = exp2_fast(mx - finite_or_zero(now));
        mx = now;
        sum *= f;
#pragma unroll
        for (int t = 0; t < S::VT; t++) o[t] *= f;
      }
      const float base = finite_or_zero(mx);   // (a row that has seen no key: exp2(-inf) = 0)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        sc[v] = exp2_fast(fmaf(sc[v], a.c, -base));
        sum += sc[v];
      }
#pragma unroll
      for (int u = 0; u < 2; u++) {
        const typename O::Frag p = O::operand(sc, u);
#pragma unroll
        for (int t = 0; t < S::VT; t++) o[t] = O::mma(O::template transposed<S::PITCH>(Vs, 32 * t, 16 * u, lane), p, o[t]);
      }
    }
    if (j0 + S::KC < last) {
      ks.store(lds + (buf ^ 1) * BUF);
      vs.store(lds + (2 + (buf ^ 1)) * BUF);
      if (j0 + 2 * S::KC < last) fetch(j0 + 2 * S::KC);
    }
    __syncthreads();
  }
  sum += other_half(sum);
  if (a.parts > 1) {   // a part's sums, joined by diff_join_kernel
    if (!live) return;
    const int64_t at = (((int64_t)part * a.units + unit) * (a.tq * a.group) + r) * 2 + m;
    float* p = a.part + at * 2 * a.dim + 4 * hh;
#pragma unroll
    for (int t = 0; t < S::VT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        if (32 * t + 8 * g < 2 * a.dim) *reinterpret_cast<float4*>(p + 32 * t + 8 * g) = make_float4(o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]);
    if (hh == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(mx, sum);
    return;
  }
  const int64_t row = s.q0 + i;
  const float norm = sum > 0.f || sum != sum ? 1.f / sum : 0.f;   // (NaN stays NaN)
#pragma unroll
  for (int t = 0; t < S::VT; t++) o[t] *= norm;
  if (a.lse && live && hh == 0) a.lse[(int64_t)(m * a.heads + h) * a.q_rows + row] = sum > 0.f ? mx + __log2f(sum) : sum;
  // P_2 v to the wave that holds P_1 v: [row group][4 channels][row], 16 bytes a lane
  static_assert(F_GROUPS * S::VT * 4096 <= (int)sizeof(lds), "exchange");
  float4* ex = reinterpret_cast<float4*>(lds) + (rg * S::VT * 8) * 32;
  T* second = a.o2 ? static_cast<T*>(a.o2) + row * a.o2_token + (int64_t)h * 2 * a.dim + 4 * hh : nullptr;
  if (m == 1) {
#pragma unroll
    for (int t = 0; t < S::VT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        ex[(t * 8 + 2 * g + hh) * 32 + c] = make_float4(o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]);
        if (second && live && 32 * t + 8 * g < 2 * a.dim) O::store4(second + 32 * t + 8 * g, o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]);
      }
  }
  __syncthreads();
  if (m == 1 || r >= room) return;
  const float lam = live ? a.lam[a.lam_token ? row * a.heads + h : h] : 0.f;
  T* op = rows_of(a, static_cast<T*>(a.out), b, s.q0, a.o_token, a.o_batch) + i * a.o_token + (int64_t)h * 2 * a.dim + 4 * hh;
#pragma unroll
  for (int t = 0; t < S::VT; t++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      if (32 * t + 8 * g >= 2 * a.dim) continue;
      const float4 y = ex[(t * 8 + 2 * g + hh) * 32 + c];
      O::store4(op + 32 * t + 8 * g, live ? o[t][4 * g] - lam * y.x : 0.f, live ? o[t][4 * g + 1] - lam * y.y : 0.f, live ? o[t][4 * g + 2] - lam * y.z : 0.f,
                live ? o[t][4 * g + 3] - lam * y.w : 0.f);
    }
}

// Joins the parts of a row: one wave a row.  Lane p holds the maximum and the sum of part p (at most 64 parts), so that the weights of all parts are
// known before the sums are read.
template <typename T>
__global__ void __launch_bounds__(256) diff_join_kernel(DiffArgs a) {
  const int room = a.tq * a.group;
  const int64_t x = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, unit = (int)(x / room), r = (int)(x - (int64_t)unit * room);
  if (unit >= a.units) return;
  const int b = unit / a.kv_heads, hk = unit % a.kv_heads;
  const Seq s = sequence(a, b);
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group);
  const bool live = r < s.nq * a.group;
  if (!live && a.q_starts) return;
  const int64_t row = s.q0 + i, step = (int64_t)a.units * room, at = (int64_t)unit * room + r;
  float f[2] = {0.f, 0.f}, acc[2][4] = {};
  if (live) {
    float lse[2];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < a.parts) ml = *reinterpret_cast<const float2*>(a.part_ml + ((at + lane * step) * 2 + k) * 2);
      const float top = wave_max(ml.x), e = exp2_fast(ml.x - finite_or_zero(top)), sum = wave_sum(e * ml.y);
      f[k] = sum > 0.f || sum != sum ? e / sum : 0.f;   // (NaN stays NaN)
      lse[k] = sum > 0.f ? top + __log2f(sum) : sum;
    }
    if (a.lse && lane < 2) a.lse[(int64_t)(lane * a.heads + h) * a.q_rows + row] = lane ? lse[1] : lse[0];
    for (int p0 = 0; p0 < a.parts; p0 += 4) {   // (four parts' loads in flight)
      float g[2][4], v[2][4][4];
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int p = min(p0 + q, a.parts - 1);
        const float* o = a.part + (at + p * step) * 4 * a.dim;
#pragma unroll
        for (int k = 0; k < 2; k++) {
          g[k][q] = p0 + q < a.parts ? __shfl(f[k], p, 64) : 0.f;
#pragma unroll
          for (int e = 0; e < 4; e++) v[k][q][e] = lane + 64 * e < 2 * a.dim && p0 + q < a.parts ? o[k * 2 * a.dim + lane + 64 * e] : 0.f;
        }
      }
#pragma unroll
      for (int q = 0; q < 4; q++)
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
          for (int e = 0; e < 4; e++) acc[k][e] += g[k][q] * v[k][q][e];
    }
  }
  const float lam = live ? a.lam[a.lam_token ? row * a.heads + h : h] : 0.f;
  T* op = rows_of(a, static_cast<T*>(a.out), b, s.q0, a.o_token, a.o_batch) + i * a.o_token + (int64_t)h * 2 * a.dim;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const int d = lane + 64 * e;
    if (d >= 2 * a.dim) continue;
    op[d] = Cvt<T>::st(acc[0][e] - lam * acc[1][e]);
    if (a.o2 && live) static_cast<T*>(a.o2)[row * a.o2_token + (int64_t)h * 2 * a.dim + d] = Cvt<T>::st(acc[1][e]);
  }
}

// ---- backward: queries ------------------------------------------------------------------------------------------------------------
// dq, delta and dlambda.  delta first comes from the kept outputs, delta_2 = dO . (P_2 v), delta_1 = dO . out + lambda delta_2, which were rounded;
// the pass over the keys gives what is missing, rowsum(P_m (dP - delta_m)) in fp32, so that dlambda and the deltas that the other kernel
// reads are exact to fp32 rounding (with the kept bf16 outputs alone dlambda is off by their rounding, a thousandth).
template <typename T, int DT>
__global__ void __launch_bounds__(256, sizeof(T) == 2 && DT <= 64 ? 2 : 1) diff_backward_q_kernel(DiffArgs a) {
  typedef Ops<T> O;
  typedef Sizes<T, DT> S;
  __shared__ __attribute__((aligned(16))) T Ks[S::KC * S::PITCH];
  __shared__ __attribute__((aligned(16))) T Vs[S::KC * S::PITCH];
  const int w = work_index(a.units * a.tiles, a.tiles, a.causal);
  if (w >= a.units * a.tiles) return;
  const int unit = w / a.tiles, tile = a.tiles - 1 - w % a.tiles;
  const int b = unit / a.kv_heads, hk = unit % a.kv_heads;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.group, r0 = tile * ROWS, room = a.q_starts ? R : a.tq * a.group;
  if (r0 >= room) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 31, hh = lane >> 5;
  const int r = r0 + 32 * wave + c;
  const bool live = r < R;
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group);
  const int64_t row = s.q0 + i;
  const T* kp = rows_of(a, static_cast<const T*>(a.k), b, s.k0, a.k_token, a.k_batch) + (int64_t)hk * 2 * a.dim;
  const T* vp = rows_of(a, static_cast<const T*>(a.v), b, s.k0, a.v_token, a.v_batch) + (int64_t)hk * 2 * a.dim;
  typename O::Frag qf[2 * S::KS], gf[2 * S::KS];
  own_row<T, DT, true>(qf, rows_of(a, static_cast<const T*>(a.q), b, s.q0, a.q_token, a.q_batch) + i * a.q_token + (int64_t)h * 2 * a.dim, live, a.dim, hh);
  const int64_t o_at = i * a.o_token + (int64_t)h * 2 * a.dim;
  own_row<T, DT, false>(gf, rows_of(a, static_cast<const T*>(a.dout), b, s.q0, a.o_token, a.o_batch) + o_at, live, a.dim, hh);
  float lam = 0.f, lse[2] = {0.f, 0.f}, delta[2] = {0.f, 0.f}, rest[2] = {0.f, 0.f};
  if (live) {
    lam = a.lam[a.lam_token ? row * a.heads + h : h];
    lse[0] = a.lse[(int64_t)h * a.q_rows + row];
    lse[1] = a.lse[(int64_t)(a.heads + h) * a.q_rows + row];
  }
  {
    typename O::Frag f[2 * S::KS];
    own_row<T, DT, false>(f, rows_of(a, static_cast<const T*>(a.out), b, s.q0, a.o_token, a.o_batch) + o_at, live, a.dim, hh);
#pragma unroll
    for (int t = 0; t < 2 * S::KS; t++)
#pragma unroll
      for (int e = 0; e < 8; e++) delta[0] += O::get(f[t], e) * O::get(gf[t], e);
    own_row<T, DT, false>(f, static_cast<const T*>(a.o2) + row * a.o2_token + (int64_t)h * 2 * a.dim, live, a.dim, hh);
#pragma unroll
    for (int t = 0; t < 2 * S::KS; t++)
#pragma unroll
      for (int e = 0; e < 8; e++) delta[1] += O::get(f[t], e) * O::get(gf[t], e);
    delta[0] += other_half(delta[0]);
    delta[1] += other_half(delta[1]);
    delta[0] += lam * delta[1];
  }
  const int off = s.nk - s.nq;
  auto limit = [&](int x) { return a.causal ? min(s.nk, query_of(a, x) + off + 1) : s.nk; };
  const int see = live ? limit(r) : s.nk;
  const int wr0 = r0 + 32 * wave, least = limit(wr0), reach = wr0 < R ? limit(min(wr0 + 31, R - 1)) : 0;
  const int last = r0 < R ? limit(min(r0 + ROWS, R) - 1) : 0;
  v16f dq[2][S::DTT];
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int t = 0; t < S::DTT; t++) clear(dq[m][t]);
  // Rows with few keys: a rounding of the kept outputs is as large as their small dS (two keys: dq off by 5e-3 where its own rounding is 1.7e-3,
  // 128 keys 2.8e-3, 700 keys 2.5e-3 as without it), so delta is completed by a pass of its own first.
  const bool two = last <= EXACT_KEYS;
  for (int pass = two ? 0 : 1; pass < 2; pass++) {
  if (two && pass == 1) {
#pragma unroll
    for (int m = 0; m < 2; m++) {
      delta[m] += rest[m] + other_half(rest[m]);
      rest[m] = 0.f;
    }
  }
  for (int j0 = 0; j0 < last; j0 += S::KC) {
    if (pass == 0 || !two || last > S::KC) {   // (else the first pass has staged all keys)
      Stage<T, DT, true> ks;
      Stage<T, DT, false> vs;
      const int n = min(S::KC, s.nk - j0);
      ks.load(n, a.dim, [&](int x) { return kp + (int64_t)(j0 + x) * a.k_token; });
      vs.load(n, a.dim, [&](int x) { return vp + (int64_t)(j0 + x) * a.v_token; });
      __syncthreads();
      ks.store(Ks);
      vs.store(Vs);
      __syncthreads();
    }
#pragma unroll
    for (int kt = 0; kt < S::KC / 32; kt++) {
      const int jt = j0 + 32 * kt;
      if (jt >= reach) break;
      v16f sc[2], dp;
#pragma unroll
      for (int m = 0; m < 2; m++) {
        clear(sc[m]);
#pragma unroll
        for (int t = 0; t < S::KS; t++)
          sc[m] = O::mma(O::load(Ks + (32 * kt + c) * S::PITCH + m * DT + 16 * t + 8 * hh), qf[m * S::KS + t], sc[m]);
      }
      clear(dp);
#pragma unroll
      for (int t = 0; t < 2 * S::KS; t++) dp = O::mma(O::load(Vs + (32 * kt + c) * S::PITCH + 16 * t + 8 * hh), gf[t], dp);
      if (jt + 32 > least) {
#pragma unroll
        for (int v = 0; v < 16; v++)
          if (jt + 8 * (v >> 2) + 4 * hh + (v & 3) >= see) { sc[0][v] = -INFINITY; sc[1][v] = -INFINITY; }
      }
#pragma unroll
      for (int m = 0; m < 2; m++)
#pragma unroll
        for (int v = 0; v < 16; v++) {
          sc[m][v] = exp2_fast(fmaf(sc[m][v], a.c, -lse[m])) * (dp[v] - delta[m]);
          rest[m] += sc[m][v];
        }
      if (pass == 0) continue;
#pragma unroll
      for (int u = 0; u < 2; u++)
#pragma unroll
        for (int m = 0; m < 2; m++) {
          const typename O::Frag p = O::operand(sc[m], u);
#pragma unroll
          for (int t = 0; t < S::DTT; t++)
            dq[m][t] = O::mma(O::template transposed<S::PITCH>(Ks, m * DT + 32 * t, 32 * kt + 16 * u, lane), p, dq[m][t]);
        }
    }
  }
  }
  if (r >= room) return;
#pragma unroll
  for (int m = 0; m < 2; m++) delta[m] += rest[m] + other_half(rest[m]);
  T* dqp = rows_of(a, static_cast<T*>(a.dq), b, s.q0, a.q_token, a.q_batch) + i * a.q_token + (int64_t)h * 2 * a.dim + 4 * hh;
#pragma unroll
  for (int m = 0; m < 2; m++) {
    const float f = live ? (m ? -lam * a.scale : a.scale) : 0.f;
#pragma unroll
    for (int t = 0; t < S::DTT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        if (32 * t + 8 * g < a.dim)
          O::store4(dqp + m * a.dim + 32 * t + 8 * g, f * dq[m][t][4 * g], f * dq[m][t][4 * g + 1], f * dq[m][t][4 * g + 2], f * dq[m][t][4 * g + 3]);
  }
  if (hh == 0) {
    a.delta[(int64_t)h * a.q_rows + row] = live ? delta[0] : 0.f;
    a.delta[(int64_t)(a.heads + h) * a.q_rows + row] = live ? delta[1] : 0.f;
    if (a.lam_token) a.dlam[row * a.heads + h] = live ? -delta[1] : 0.f;
  }
}

// dlambda of a head: minus the sum of delta_2 over the sequences' rows, always in the same order.  One workgroup a head.
__global__ void __launch_bounds__(1024) diff_lambda_kernel(DiffArgs a) {
  __shared__ float red[16];
  const int h = blockIdx.x;
  const float* d = a.delta + (int64_t)(a.heads + h) * a.q_rows;
  float t = 0.f;
  if (!a.q_starts) {   // (rows behind a sequence's queries hold zeros)
    for (int64_t x = threadIdx.x; x < a.q_rows; x += 1024) t += d[x];
  } else {
    for (int b = threadIdx.x >> 6; b < a.batch; b += 16) {
      const Seq s = sequence(a, b);
      for (int x = threadIdx.x & 63; x < s.nq; x += 64) t += d[s.q0 + x];
    }
  }
  t = wave_sum(t);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    float z = 0.f;
#pragma unroll
    for (int k = 0; k < 16; k++) z += red[k];
    a.dlam[h] = -z;
  }
}

// ---- backward: keys ------------------------------------------------------------------------------------------------------------------
template <typename T, int DT>
__global__ void __launch_bounds__(256, 1) diff_backward_kv_kernel(DiffArgs a) {
  typedef Ops<T> O;
  typedef Sizes<T, DT> S;
  __shared__ __attribute__((aligned(16))) T Qs[S::KC * S::PITCH];
  __shared__ __attribute__((aligned(16))) T Gs[S::KC * S::PITCH];
  __shared__ __attribute__((aligned(16))) float st[5][S::KC];   // log-sums, deltas and lambda of the rows
  const int w = work_index(a.units * a.tiles, a.tiles, a.causal);
  if (w >= a.units * a.tiles) return;
  const int unit = w / a.tiles, tile = w % a.tiles;   // (under a causal mask the first keys are seen by the most rows)
  const int b = unit / a.kv_heads, hk = unit % a.kv_heads;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.group, j0 = tile * ROWS, room = a.q_starts ? s.nk : a.tk;
  if (j0 >= room) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 31, hh = lane >> 5;
  const int j = j0 + 32 * wave + c;
  const bool live = j < s.nk;
  const T* qp = rows_of(a, static_cast<const T*>(a.q), b, s.q0, a.q_token, a.q_batch) + (int64_t)hk * a.group * 2 * a.dim;
  const T* gp = rows_of(a, static_cast<const T*>(a.dout), b, s.q0, a.o_token, a.o_batch) + (int64_t)hk * a.group * 2 * a.dim;
  typename O::Frag kf[2 * S::KS], vf[2 * S::KS];
  const int64_t k_at = (int64_t)j * a.k_token + (int64_t)hk * 2 * a.dim, v_at = (int64_t)j * a.v_token + (int64_t)hk * 2 * a.dim;
  own_row<T, DT, true>(kf, rows_of(a, static_cast<const T*>(a.k), b, s.k0, a.k_token, a.k_batch) + k_at, live, a.dim, hh);
  own_row<T, DT, false>(vf, rows_of(a, static_cast<const T*>(a.v), b, s.k0, a.v_token, a.v_batch) + v_at, live, a.dim, hh);
  // the first row that sees key j, and those of the wave's first and last key
  const int off = s.nk - s.nq;
  auto from = [&](int key) { return a.causal ? max(0, key - off) * a.group : 0; };
  const int first = live ? from(j) : 0;
  const int wfirst = j0 + 32 * wave < s.nk ? from(j0 + 32 * wave) : R, wlast = from(min(j0 + 32 * wave + 31, s.nk - 1));
  v16f dk[2][S::DTT], dv[S::VT];
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int t = 0; t < S::DTT; t++) clear(dk[m][t]);
#pragma unroll
  for (int t = 0; t < S::VT; t++) clear(dv[t]);
  for (int r0 = j0 < s.nk ? from(j0) / S::KC * S::KC : R; r0 < R; r0 += S::KC) {
    Stage<T, DT, true> qs;
    Stage<T, DT, false> gs;
    const int n = min(S::KC, R - r0);
    auto place = [&](int x, int64_t token) { const int r = r0 + x, i = query_of(a, r); return i * token + (int64_t)(r - i * a.group) * 2 * a.dim; };
    qs.load(n, a.dim, [&](int x) { return qp + place(x, a.q_token); });
    gs.load(n, a.dim, [&](int x) { return gp + place(x, a.o_token); });
    float sv[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
    if ((int)threadIdx.x < n) {
      const int r = r0 + threadIdx.x, i = query_of(a, r), h = hk * a.group + (r - i * a.group);
      const int64_t row = s.q0 + i, at = (int64_t)h * a.q_rows + row, two = (int64_t)a.heads * a.q_rows;
      sv[0] = a.lse[at]; sv[1] = a.lse[at + two]; sv[2] = a.delta[at]; sv[3] = a.delta[at + two];
      sv[4] = a.lam[a.lam_token ? row * a.heads + h : h];
    }
    __syncthreads();
    qs.store(Qs);
    gs.store(Gs);
    if ((int)threadIdx.x < S::KC)
#pragma unroll
      for (int e = 0; e < 5; e++) st[e][threadIdx.x] = sv[e];
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < S::KC / 32; rt++) {
      const int rr = r0 + 32 * rt;
      if (rr + 32 <= wfirst || rr >= R) continue;   // no key of the wave is seen by these rows
      v16f sc[2], dp;
#pragma unroll
      for (int m = 0; m < 2; m++) {
        clear(sc[m]);
#pragma unroll
        for (int t = 0; t < S::KS; t++)
          sc[m] = O::mma(O::load(Qs + (32 * rt + c) * S::PITCH + m * DT + 16 * t + 8 * hh), kf[m * S::KS + t], sc[m]);
      }
      clear(dp);
#pragma unroll
      for (int t = 0; t < 2 * S::KS; t++) dp = O::mma(O::load(Gs + (32 * rt + c) * S::PITCH + 16 * t + 8 * hh), vf[t], dp);
      if (rr < wlast) {
#pragma unroll
        for (int v = 0; v < 16; v++)
          if (rr + 8 * (v >> 2) + 4 * hh + (v & 3) < first) { sc[0][v] = -INFINITY; sc[1][v] = -INFINITY; }
      }
      v16f wt;
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const int at = 32 * rt + 8 * g + 4 * hh;
        float x[5][4];
#pragma unroll
        for (int e = 0; e < 5; e++) {
          const float4 f = *reinterpret_cast<const float4*>(&st[e][at]);
          x[e][0] = f.x; x[e][1] = f.y; x[e][2] = f.z; x[e][3] = f.w;
        }
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const int v = 4 * g + e;
          const float p0 = exp2_fast(fmaf(sc[0][v], a.c, -x[0][e])), p1 = x[4][e] * exp2_fast(fmaf(sc[1][v], a.c, -x[1][e]));
          wt[v] = p0 - p1;
          sc[0][v] = p0 * (dp[v] - x[2][e]);
          sc[1][v] = p1 * (x[3][e] - dp[v]);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; u++) {
        const typename O::Frag pw = O::operand(wt, u);
#pragma unroll
        for (int t = 0; t < S::VT; t++) dv[t] = O::mma(O::template transposed<S::PITCH>(Gs, 32 * t, 32 * rt + 16 * u, lane), pw, dv[t]);
#pragma unroll
        for (int m = 0; m < 2; m++) {
          const typename O::Frag p = O::operand(sc[m], u);
#pragma unroll
          for (int t = 0; t < S::DTT; t++)
            dk[m][t] = O::mma(O::template transposed<S::PITCH>(Qs, m * DT + 32 * t, 32 * rt + 16 * u, lane), p, dk[m][t]);
        }
      }
    }
  }
  if (j >= room) return;
  T* dkp = rows_of(a, static_cast<T*>(a.dk), b, s.k0, a.k_token, a.k_batch) + k_at + 4 * hh;
  T* dvp = rows_of(a, static_cast<T*>(a.dv), b, s.k0, a.v_token, a.v_batch) + v_at + 4 * hh;
  const float f = live ? a.scale : 0.f;
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int t = 0; t < S::DTT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        if (32 * t + 8 * g < a.dim)
          O::store4(dkp + m * a.dim + 32 * t + 8 * g, live ? f * dk[m][t][4 * g] : 0.f, live ? f * dk[m][t][4 * g + 1] : 0.f,
                    live ? f * dk[m][t][4 * g + 2] : 0.f, live ? f * dk[m][t][4 * g + 3] : 0.f);
#pragma unroll
  for (int t = 0; t < S::VT; t++)
#pragma unroll
    for (int g = 0; g < 4; g++)
      if (32 * t + 8 * g < 2 * a.dim)
        O::store4(dvp + 32 * t + 8 * g, live ? dv[t][4 * g] : 0.f, live ? dv[t][4 * g + 1] : 0.f, live ? dv[t][4 * g + 2] : 0.f,
                  live ? dv[t][4 * g + 3] : 0.f);
}

// ---- host ----------------------------------------------------------------------------------------------------------------------------
static int elem_of(const cd_diff_attn* d) { return d->dtype == CD_BF16 ? 2 : 4; }
static int64_t rows_q(const cd_diff_attn* d) { return d->q_starts ? d->q_rows : (int64_t)d->batch * d->tq; }

static int check(const char* what, const cd_diff_attn* d) {
  CD_REQUIRE(d != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE(d->dtype == CD_F32 || d->dtype == CD_BF16, "%s: unknown dtype %d", what, d->dtype);
  CD_REQUIRE(d->lambda_kind == CD_LAMBDA_HEAD || d->lambda_kind == CD_LAMBDA_TOKEN, "%s: unknown lambda_kind %d", what, d->lambda_kind);
  CD_REQUIRE(d->batch >= 1 && d->heads >= 1 && d->kv_heads >= 1 && d->heads % d->kv_heads == 0, "%s: batch=%d heads=%d kv_heads=%d", what, d->batch, d->heads,
             d->kv_heads);
  CD_REQUIRE(d->scale >= 0.f && d->scale < INFINITY, "%s: scale must be finite and not negative", what);
  CD_REQUIRE((d->q_starts != nullptr) == (d->k_starts != nullptr), "%s: one of q_starts and k_starts without the other", what);
  CD_REQUIRE(!d->q_starts || (!d->q_lens && !d->k_lens), "%s: starts and lens together", what);
  CD_REQUIRE(!d->q_starts || (d->q_rows >= 0 && d->k_rows >= 0 && d->q_rows <= INT32_MAX && d->k_rows <= INT32_MAX), "%s: q_rows=%lld k_rows=%lld", what,
             (long long)d->q_rows, (long long)d->k_rows);
  CD_REQUIRE(d->tq >= 0 && d->tk >= 0, "%s: tq=%d tk=%d", what, d->tq, d->tk);
  const int64_t group = d->heads / d->kv_heads;
  CD_REQUIRE(group <= 1024 && d->tq * group <= (1 << 30) / group, "%s: tq=%d with %lld heads a key head is too long", what, d->tq, (long long)group);
  CD_REQUIRE((int64_t)d->batch * d->kv_heads * (cdiv(d->tq * group, F_ROWS) + cdiv(d->tk, ROWS) + 1) < (1 << 30) && (int64_t)d->batch * d->tq <= INT32_MAX,
             "%s: too many rows", what);
  for (const void* p : {(const void*)d->q_lens, (const void*)d->k_lens, (const void*)d->q_starts, (const void*)d->k_starts})
    CD_REQUIRE((reinterpret_cast<uintptr_t>(p) & 3) == 0, "%s: length and start tables must be 4-byte aligned", what);
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8 != 0)
    return set_error(CD_ERR_UNSUPPORTED, "%s: head_dim=%d must be a multiple of 8 up to 128", what, d->head_dim);
  const int ve = 16 / elem_of(d);
  const int64_t w = 2LL * d->head_dim, tokens[4] = {d->q_token, d->k_token, d->v_token, d->o_token}, batches[4] = {d->q_batch, d->k_batch, d->v_batch, d->o_batch};
  for (int t = 0; t < 4; t++) {
    const int64_t heads = t == 1 || t == 2 ? d->kv_heads : d->heads;
    CD_REQUIRE(tokens[t] >= heads * w && tokens[t] % ve == 0, "%s: token stride %lld of %s", what, (long long)tokens[t], t == 0 ? "q" : t == 1 ? "k" : t == 2 ? "v" : "out");
    CD_REQUIRE(batches[t] >= 0 && batches[t] % ve == 0, "%s: batch stride %lld of %s", what, (long long)batches[t], t == 0 ? "q" : t == 1 ? "k" : t == 2 ? "v" : "out");
  }
  return CD_OK;
}

// sequences that lie apart: a batch stride of at least their rows
static int check_apart(const char* what, const cd_diff_attn* d, bool out_only) {
  if (d->q_starts || d->batch == 1) return CD_OK;
  const int64_t batches[4] = {d->o_batch, d->q_batch, d->k_batch, d->v_batch}, tokens[4] = {d->o_token, d->q_token, d->k_token, d->v_token};
  for (int t = 0; t < (out_only ? 1 : 4); t++) {
    const int64_t rows = t < 2 ? d->tq : d->tk;
    CD_REQUIRE(batches[t] >= rows * tokens[t] || rows == 0, "%s: the sequences that are written share memory (batch stride %lld)", what, (long long)batches[t]);
  }
  return CD_OK;
}

// Parts of the keys that get a workgroup of their own: few rows against many keys would leave most of the chip without work.
static int parts_of(const cd_diff_attn* d) {
  const int64_t groups = (int64_t)d->batch * d->kv_heads * cdiv((int64_t)d->tq * (d->heads / d->kv_heads), F_ROWS);
  int64_t p = groups ? 768 / groups : 1;
  if (p > cdiv(d->tk, 128)) p = cdiv(d->tk, 128);
  if (p > 64) p = 64;
  return p < 2 || groups > 128 ? 1 : (int)p;
}

static DiffArgs args_of(const cd_diff_attn* d) {
  DiffArgs a = {};
  a.q_token = d->q_token; a.q_batch = d->q_batch; a.k_token = d->k_token; a.k_batch = d->k_batch;
  a.v_token = d->v_token; a.v_batch = d->v_batch; a.o_token = d->o_token; a.o_batch = d->o_batch; a.o2_token = 2LL * d->heads * d->head_dim;
  a.q_lens = d->q_lens; a.k_lens = d->k_lens; a.q_starts = d->q_starts; a.k_starts = d->k_starts;
  a.q_rows = rows_q(d); a.k_rows = d->q_starts ? d->k_rows : (int64_t)d->batch * d->tk;
  a.batch = d->batch; a.tq = d->tq; a.tk = d->tk; a.heads = d->heads; a.kv_heads = d->kv_heads; a.group = d->heads / d->kv_heads; a.dim = d->head_dim;
  a.causal = d->causal != 0; a.lam_token = d->lambda_kind == CD_LAMBDA_TOKEN; a.parts = 1;
  a.units = d->batch * d->kv_heads;
  a.group_inv = a.group > 1 ? (uint32_t)((1ull << 32) / a.group) + 1 : 0;
  a.scale = d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->head_dim);
  a.c = a.scale * 1.44269504088896340736f;
  return a;
}

// f<T, DT>() of this dtype and head_dim
#define CD_DIFF_DISPATCH(d, KERNEL, THREADS, BLOCKS, s, a)                                                                                  \
  do {                                                                                                                             \
    const dim3 grid_(BLOCKS), block_(THREADS);                                                                                                      \
    if ((d)->dtype == CD_BF16) {                                                                                                   \
      if ((d)->head_dim <= 32) hipLaunchKernelGGL((KERNEL<bf16_t, 32>), grid_, block_, 0, s, a);                                \
      else if ((d)->head_dim <= 64) hipLaunchKernelGGL((KERNEL<bf16_t, 64>), grid_, block_, 0, s, a);                           \
      else hipLaunchKernelGGL((KERNEL<bf16_t, 128>), grid_, block_, 0, s, a);                                                   \
    } else {                                                                                                                       \
      if ((d)->head_dim <= 32) hipLaunchKernelGGL((KERNEL<float, 32>), grid_, block_, 0, s, a);                                 \
      else if ((d)->head_dim <= 64) hipLaunchKernelGGL((KERNEL<float, 64>), grid_, block_, 0, s, a);                            \
      else hipLaunchKernelGGL((KERNEL<float, 128>), grid_, block_, 0, s, a);                                                    \
    }                                                                                                                              \
  } while (0)

static double pairs(const cd_diff_attn* d) { return (double)d->batch * d->heads * d->tq * d->tk * (d->causal ? 0.5 : 1.0); }

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_diff_attention_workspace_bytes(const cd_diff_attn* desc, int backward, size_t* bytes) {
  if (const int rc = check("diff_attention_workspace_bytes", desc)) return rc;
  CD_REQUIRE(bytes != nullptr, "diff_attention_workspace_bytes: output pointer is NULL");
  const int parts = parts_of(desc);
  size_t n = parts > 1 ? (size_t)parts * desc->batch * desc->kv_heads * desc->tq * (desc->heads / desc->kv_heads) * 2 * (2 * desc->head_dim + 2) * 4 : 0;
  if (backward) {
    const size_t deltas = (size_t)2 * desc->heads * rows_q(desc) * 4;
    n = n > deltas ? n : deltas;
  }
  *bytes = align_up(n, 16);
  return CD_OK;
}

extern "C" int codistill_diff_attention(const cd_diff_attn* desc, const void* q, const void* k, const void* v, const float* lambda, void* out,
                                        void* o_second, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check("diff_attention", desc)) return rc;
  CD_REQUIRE(q && k && v && lambda && out, "diff_attention: NULL pointer argument");
  CD_REQUIRE((o_second != nullptr) == (lse != nullptr), "diff_attention: o_second and lse are kept together or not at all");
  CD_REQUIRE(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out) && aligned16(o_second) && aligned16(lse) && aligned16(workspace) &&
                 (reinterpret_cast<uintptr_t>(lambda) & 3) == 0,
             "diff_attention: pointers must be 16-byte aligned, lambda 4-byte aligned");
  if (const int rc = check_apart("diff_attention", desc, true)) return rc;
  size_t need = 0;
  codistill_diff_attention_workspace_bytes(desc, 0, &need);
  if (workspace_bytes < need || (need && !workspace)) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "diff_attention: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (desc->tq == 0) return CD_OK;
  DiffArgs a = args_of(desc);
  a.q = q; a.k = k; a.v = v; a.lam = lambda; a.out = out; a.o2 = o_second; a.lse = lse;
  a.tiles = (int)cdiv((int64_t)a.tq * a.group, F_ROWS);
  a.parts = parts_of(desc);
  a.part_ml = static_cast<float*>(workspace);
  a.part = a.part_ml + (size_t)a.parts * a.units * a.tq * a.group * 4;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double e = elem_of(desc), qe = 2.0 * a.q_rows * a.heads * 2 * a.dim, ke = 2.0 * a.k_rows * a.kv_heads * 2 * a.dim;
  ProfScope prof(CD_K_ATTN, s, 12.0 * a.dim * pairs(desc), e * (qe + ke));
  CD_DIFF_DISPATCH(desc, diff_forward_kernel, F_THREADS, work_blocks((int64_t)a.units * a.tiles * a.parts), s, a);
  if (a.parts > 1) {
    const dim3 grid((unsigned)cdiv((int64_t)a.units * a.tq * a.group, 4));
    if (desc->dtype == CD_BF16) hipLaunchKernelGGL((diff_join_kernel<bf16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((diff_join_kernel<float>), grid, dim3(256), 0, s, a);
  }
  return check_launch("diff_attention");
}

extern "C" int codistill_diff_attention_backward(const cd_diff_attn* desc, const void* q, const void* k, const void* v, const float* lambda, const void* out,
                                                 const void* o_second, const float* lse, const void* dout, void* dq, void* dk, void* dv, float* dlambda,
                                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check("diff_attention_backward", desc)) return rc;
  CD_REQUIRE(q && k && v && lambda && out && o_second && lse && dout && dq && dk && dv && dlambda && (workspace || rows_q(desc) == 0),
             "diff_attention_backward: NULL pointer argument");
  CD_REQUIRE(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out) && aligned16(o_second) && aligned16(lse) && aligned16(dout) && aligned16(dq) &&
                 aligned16(dk) && aligned16(dv) && aligned16(workspace) && ((reinterpret_cast<uintptr_t>(lambda) | reinterpret_cast<uintptr_t>(dlambda)) & 3) == 0,
             "diff_attention_backward: pointers must be 16-byte aligned, lambda and dlambda 4-byte aligned");
  if (const int rc = check_apart("diff_attention_backward", desc, false)) return rc;
  size_t need = 0;
  codistill_diff_attention_workspace_bytes(desc, 1, &need);
  if (workspace_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "diff_attention_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  DiffArgs a = args_of(desc);
  a.q = q; a.k = k; a.v = v; a.lam = lambda; a.out = const_cast<void*>(out); a.o2 = const_cast<void*>(o_second); a.lse = const_cast<float*>(lse);
  a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv; a.dlam = dlambda;
  a.delta = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double e = elem_of(desc), qe = 4.0 * a.q_rows * a.heads * 2 * a.dim, ke = 4.0 * a.k_rows * a.kv_heads * 2 * a.dim;
  ProfScope prof(CD_K_ATTN, s, 20.0 * a.dim * pairs(desc), e * (qe + ke));
  if (a.tq > 0) {
    a.tiles = (int)cdiv((int64_t)a.tq * a.group, ROWS);
    CD_DIFF_DISPATCH(desc, diff_backward_q_kernel, 256, work_blocks((int64_t)a.units * a.tiles), s, a);
  }
  if (!a.lam_token) hipLaunchKernelGGL(diff_lambda_kernel, dim3((unsigned)a.heads), dim3(1024), 0, s, a);
  if (a.tk > 0) {
    a.tiles = (int)cdiv(a.tk, ROWS);
    CD_DIFF_DISPATCH(desc, diff_backward_kv_kernel, 256, work_blocks((int64_t)a.units * a.tiles), s, a);
  }
  return check_launch("diff_attention_backward");
}
