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
//
// What bounds them.  Long sequences: neither memory nor LDS, but the matrix instructions (43 % of the forward kernel's cycles) and the vector ones (63 %,
// exponentials and what surrounds them) of few waves taking turns; two causal sequences of 4096 tokens, 8 heads of 64: forward 128 us (806 TFLOP/s),
// queries' gradients 164, keys' 182 (497 TFLOP/s together, which repeat scores and dP: 696 with those).  One query a sequence: the cache's bytes, 178 MB in
// 41 us (4.4 TB/s).  Short sequences: the latency of a workgroup's few tiles, one after the other, and the second walk over few keys (EXACT_KEYS).
//
// Roundings to bf16 (fp32 has none of them).  P where it multiplies v, P_m (dP - delta_m) where it multiplies k or q, P_1 - lambda P_2 where it multiplies dO: the
// matrix instructions take bf16, at sixteen times the rate of fp32.  Each is off by 1.7e-3 (2-norm), as the rounding of a result is, so that results are off by
// 2.3e-3 to 2.6e-3 where 32-bit arithmetic rounded once has 1.7e-3.  out and P_2 v are kept as they are returned, rounded: deltas begin from them (below).
#include "common.h"
#include "conv_rules.h"
#include "kernels.h"
#include "lds_load.h"
#include <math.h>

namespace cd {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// What the pass that owns keys needs of a row, in the form it uses it: the pass that owns queries leaves it in the workspace.
struct RowValues {
  uint2 lse[2];    // minus the log-sums over c, each fp32 value in three bf16 parts (all of its bits); the second one with the logarithm of |lambda|
  uint2 delta[2];  // minus the deltas
  uint32_t lam_negative, unused[3];
};
static_assert(sizeof(RowValues) == 48, "three pieces of 16 bytes");
__device__ inline uint2 three_parts(float x) {
  const bf16_t hi = f32_to_bf16(x), mid = f32_to_bf16(x - bf16_to_f32(hi)), lo = f32_to_bf16(x - bf16_to_f32(hi) - bf16_to_f32(mid));
  return make_uint2((uint32_t)hi | (uint32_t)mid << 16, lo);
}

struct DiffArgs {
  const void* q; const void* k; const void* v; const float* lam;
  void* out; void* o2; float* lse;
  const void* dout; void* dq; void* dk; void* dv; float* dlam;
  RowValues* rows;                                // backward: [q rows][heads]
  float* second;                                  // backward, a lambda for each head: delta_2 [heads][q rows]
  float* part; float* part_ml;                    // forward over parts of the keys: unnormalised sums and (maximum, sum, rounded sum, -) of a part
  int64_t q_token, q_batch, k_token, k_batch, v_token, v_batch, o_token, o_batch, o2_token;
  const int32_t* q_lens; const int32_t* k_lens; const int32_t* q_starts; const int32_t* k_starts;
  int64_t q_rows, k_rows;                         // rows of the q and k tensors (batch * tq when padded)
  int32_t batch, tq, tk, heads, kv_heads, group, dim, causal, lam_token, parts, tiles, units, work, run, turns, uneven;
  FastDiv by_run, by_turns, by_unit, by_parts, by_tiles, by_heads, by_dim, by_quads;   // by run, turns, tiles * parts, parts, tiles, kv_heads, dim, dim / 2
  uint32_t group_inv;                             // floor(2^32 / group) + 1 (group > 1)
  float scale, c;                                 // c = scale log2(e)
};

// A copy in LDS: rows of W elements, the 16-byte pieces of a row exchanged among themselves so that both kinds of reads meet all banks.  Sixteen rows
// read at the same column (row by row) differ in four bits of the row, four consecutive rows read over 64 bytes (transposed) in bits 2 and 3 of
// the piece.  Padded rows serve one of the two: with 16 bytes a row the transposing loads met each bank four times.
template <typename T, int W> __host__ __device__ constexpr int lds_swap(int row) {
  return W * (int)sizeof(T) == 128 ? ((row >> 1 & 1) << 2) | (row >> 2 & 3) : ((row & 3) << 2) | (row >> 2 & 3);   // (rows of 128 bytes: bit 0 changes banks by itself)
}
template <typename T, int W> __host__ __device__ constexpr int lds_at(int row, int col) {
  constexpr int VE = 16 / (int)sizeof(T);
  return row * W + ((col / VE) ^ lds_swap<T, W>(row)) * VE + col % VE;
}

// Where a lane's reads begin: the pieces are exchanged by exclusive or, so a constant column is one more exclusive or.
struct LaneAt {
  int row, lo, hi;
  // forgets what the compiler knows of them, so that it does not keep the address of every read of a loop in a register of its own
  __device__ inline void fresh() { asm volatile("" : "+v"(row), "+v"(lo), "+v"(hi)); }
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
  // rows row0 .. row0 + 15 (row0 a multiple of 16) of a copy as contraction, columns col0 .. col0 + 31 on the lanes.  In a group of 16 lanes, lane i
  // of a transposing load receives element i & 3 of the four 8-byte pieces that lanes i >> 2, 4 + (i >> 2), ... address.
  template <int W> static __device__ inline Frag transposed(const bf16_t* t, int col0, int row0, const LaneAt& at) {
    typedef __attribute__((address_space(3))) v4bf lds4;
    const v4bf lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(t + row0 * W + (at.lo ^ col0)));
    const v4bf hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(t + row0 * W + (at.hi ^ col0)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  // columns col + 8 (l / 32) .. + 7 of row row0 + l % 32 (col a multiple of 16, row0 of 32)
  template <int W> static __device__ inline Frag rowwise(const bf16_t* t, int row0, int col, const LaneAt& at) { return load(t + row0 * W + (at.row ^ col)); }
  template <int W> static __device__ inline LaneAt lane_at(int lane) {
    const int grp = lane >> 4, li = lane & 15, row = 4 * (grp >> 1) + (li >> 2), col = 16 * (grp & 1) + 4 * (li & 3);
    return {lds_at<bf16_t, W>(lane & 31, 8 * (lane >> 5)), lds_at<bf16_t, W>(row, col), lds_at<bf16_t, W>(row + 8, col)};
  }
  // c and the sum of a fragment's elements (products with ones: two elements an instruction)
  static __device__ inline float add_up(const Frag& f, float c) {
    const v2bf one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int e = 0; e < 4; e++) c = __builtin_amdgcn_fdot2_f32_bf16(v2bf{f[2 * e], f[2 * e + 1]}, one, c, false);
    return c;
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
  template <int W> static __device__ inline Frag transposed(const float* t, int col0, int row0, const LaneAt& at) {
    Frag f;
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = t[(row0 + 8 * (e >> 2) + (e & 3)) * W + (at.lo ^ col0 ^ (16 * (e & 3) + 8 * (e >> 2)))];
    return f;
  }
  template <int W> static __device__ inline Frag rowwise(const float* t, int row0, int col, const LaneAt& at) {
    const float4 a = *reinterpret_cast<const float4*>(t + row0 * W + (at.row ^ col)), b = *reinterpret_cast<const float4*>(t + row0 * W + (at.row ^ (col + 4)));
    return Frag{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  }
  template <int W> static __device__ inline LaneAt lane_at(int lane) {
    static_assert(W * sizeof(float) >= 256, "rows of 16 pieces");
    return {lds_at<float, W>(lane & 31, 8 * (lane >> 5)), lds_at<float, W>(4 * (lane >> 5), lane & 31), 0};
  }
  static __device__ inline float add_up(const Frag& f, float c) {
#pragma unroll
    for (int e = 0; e < 8; e++) c += f[e];
    return c;
  }
  static __device__ inline void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
};

// Sizes of an instance: DT = head_dim rounded up to 32, 64 or 128, rows of 2 DT elements in LDS (both maps, or the values), KC streamed rows at a time.
template <typename T, int DT> struct Sizes {
  static constexpr int W = 2 * DT, KC = 32;
  static constexpr int KS = DT / 16, VT = W / 32, DTT = DT / 32;
};
// Waves whose first row sees no more keys than this get their deltas in a pass over them of its own (bf16; why: at the pass over the queries).  What the pass
// takes of forward and backward: 4.0 of 72.2 us for 113 packed sentences of up to 126 tokens with 4 heads of 64, 7 of 107 for 64 x 128 tokens with 8, 4.4 of 54.6
// for 16 x 130 causal queries on 230 keys.
constexpr int EXACT_KEYS = 128;

// ---- sequences and rows ---------------------------------------------------------------------------------------------------
struct Seq { int nq, nk; int64_t q0, k0; };   // lengths; rows of the sequence's first query and key in their tensors
__device__ inline Seq sequence(const DiffArgs& a, int b) {
  Seq s;
  if (a.q_starts) {
    const int64_t qs = min(max((int64_t)a.q_starts[b], (int64_t)0), a.q_rows), ks = min(max((int64_t)a.k_starts[b], (int64_t)0), a.k_rows);
    s.q0 = qs; s.k0 = ks;
    // (cut in 64 bits: the difference of two table entries may pass 32)
    s.nq = (int)max(min(min((int64_t)a.q_starts[b + 1], a.q_rows) - qs, (int64_t)a.tq), (int64_t)0);
    s.nk = (int)max(min(min((int64_t)a.k_starts[b + 1], a.k_rows) - ks, (int64_t)a.tk), (int64_t)0);
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

// Workgroups go to the eight L2 caches in turn; each cache gets runs of neighbours in the order (unit, tile, part), which share their keys.  Under a
// causal mask its run is one, and the run's units are taken in turns, so that the long tiles of all of them start before the short ones.
struct Work { int unit, part, tile, b, hk; };
__device__ inline int quotient(int n, FastDiv d) { return (int)div_by((unsigned)n, d); }
// KEYS: the workgroups that read the same rows, those of a part, are neighbours
template <bool KEYS = false> __device__ inline bool work_of(const DiffArgs& a, Work& w) {
  const int at = (int)(blockIdx.x >> 3), per_unit = a.tiles * a.parts, run = quotient(at, a.by_run);
  int x = at - run * a.run;
  if (a.turns > 1) {
    const int turn = quotient(x, a.by_turns);
    x = (x - turn * a.turns) * per_unit + turn;
  }
  x += (run * 8 + (int)(blockIdx.x & 7)) * a.run;
  w.unit = quotient(x, a.by_unit);
  if (w.unit >= a.units) return false;
  x -= w.unit * per_unit;
  if (KEYS && !a.causal) {
    w.part = quotient(x, a.by_tiles);
    w.tile = x - w.part * a.tiles;
  } else {
    w.tile = quotient(x, a.by_parts);
    w.part = x - w.tile * a.parts;
  }
  w.b = quotient(w.unit, a.by_heads);
  w.hk = w.unit - w.b * a.kv_heads;
  return true;
}
// The number of workgroups.  Where sequences differ in length (and nothing else does), a cache that got whole units would have the short ones or the
// long ones: every cache gets a part of every unit.  Five sequences of up to 777 tokens, 8 heads of 128 on 2: 53 instead of 55 us forward and 60 instead of 64
// for the queries' gradients; the keys' gradients, whose rows are split over workgroups of their own, deal those parts out (110 -> 64 us).
static unsigned work_blocks(DiffArgs& a, bool keys = false) {
  const int64_t per_unit = (int64_t)a.tiles * a.parts, n = a.units * per_unit;
  a.run = (int)cdiv(n, 8);
  if (a.uneven && !a.causal) a.run = (int)(per_unit <= 8 ? per_unit : keys && a.parts > 1 ? a.tiles : cdiv(per_unit, 8));
  if (a.run < 1) a.run = 1;
  const int64_t units = a.causal && per_unit ? a.run / per_unit : 0;
  a.turns = units * per_unit == a.run ? (int)units : 1;
  a.by_run = fast_div(a.run); a.by_turns = fast_div(a.turns > 1 ? a.turns : 1); a.by_unit = fast_div(per_unit > 1 ? (uint32_t)per_unit : 1);
  a.by_parts = fast_div(a.parts); a.by_tiles = fast_div(a.tiles > 1 ? a.tiles : 1);
  return (unsigned)(cdiv(n, 8 * (int64_t)a.run) * 8 * a.run);
}

// A buffer that is the same in all lanes, and known to be (nothing is left of this where the compiler has seen it by itself).
__device__ inline rsrc_words_t buffer_of(const void* p, int64_t bytes) {
  rsrc_words_t w = make_rsrc_words(p, (uint32_t)min(bytes, (int64_t)0xfffffff0));
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
  return w;
}

// KC rows of 2 dim elements (two ranges of dim for the maps, MAPS, or one of 2 dim) from memory straight into LDS: no registers hold them on the way
// and no branch asks for their end, since what lies beyond the bytes of the last row reads as zeros.  A lane's pieces are where its LDS places
// want them from; their offsets from the tile's first row stay the same from tile to tile.  (With loads into registers the compiler turned the
// addresses into running pointers, spilled those and waited for all loads to have them back.)
template <typename T, int DT, bool MAPS, int THREADS> struct Loader {
  typedef Sizes<T, DT> S;
  static constexpr int VE = Ops<T>::VE, VPR = S::W / VE, IT = S::KC * VPR / THREADS;
  uint32_t off[IT];   // bytes
  static __device__ inline int row(int i) { return ((int)threadIdx.x + THREADS * i) / VPR; }
  // at(r): elements from the tile's first row to row r
  template <typename At> __device__ inline void plan(int dim, At at) {
#pragma unroll
    for (int i = 0; i < IT; i++) {
      const int r = row(i), c = (((int)threadIdx.x % VPR) ^ lds_swap<T, S::W>(r)) * VE, cc = MAPS && c >= DT ? c - DT : c;
      off[i] = cc < (MAPS ? dim : 2 * dim) ? (uint32_t)((at(r) + (MAPS && c >= DT ? dim + cc : cc)) * sizeof(T)) : ~0u;   // (~0: beyond any buffer)
    }
  }
  // first: the tile's first row; elements: from there to the end of the last row.  The same in all lanes.
  __device__ inline void load(const T* first, int64_t elements, uint32_t lds) const {
    const rsrc_words_t w = buffer_of(first, elements * (int64_t)sizeof(T));
#pragma unroll
    for (int i = 0; i < IT; i++) load_lds16(w, (uint32_t)__builtin_amdgcn_readfirstlane((int)lds + THREADS * 16 * i), off[i]);
  }
};
__device__ inline uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

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

// Everything loaded so far has arrived: a value that is first used inside a loop would otherwise make every turn of it wait for all loads, those
// of the tile after next among them.
template <typename V> __device__ inline void arrived(V& v) { asm volatile("" : "+v"(v)); }
__device__ inline void arrived(v8bf& v) {
  typedef int v4i __attribute__((ext_vector_type(4)));
  v4i u = __builtin_bit_cast(v4i, v);
  asm volatile("" : "+v"(u));
  v = __builtin_bit_cast(v8bf, u);
}
__device__ inline int wave_of_thread() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }   // (the same value in all lanes, and known to be)

// N fragments, used in order, G of them on their way from LDS while the G before are used.  (Left alone, the compiler reads a fragment, waits for it and
// uses it, a fragment at a time.)  The first G can be sent for earlier, in front of work that needs none of them.
template <typename F, int G, typename Load> __device__ inline void stream_first(F (&f)[G], Load load) {
#pragma unroll
  for (int e = 0; e < G; e++) f[e] = load(e);
  __builtin_amdgcn_sched_barrier(0);
}
template <typename F, int N, int G, typename Load, typename Use> __device__ inline void stream_rest(F (&first)[G], Load load, Use use) {
  static_assert(N % G == 0, "groups");
  F f[2][G];
#pragma unroll
  for (int e = 0; e < G; e++) f[0][e] = first[e];
#pragma unroll
  for (int g = 0; g < N / G; g++) {
    if (g + 1 < N / G) {
#pragma unroll
      for (int e = 0; e < G; e++) f[(g + 1) & 1][e] = load((g + 1) * G + e);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < G; e++) use(g * G + e, f[g & 1][e]);
  }
}
template <typename F, int N, int G, typename Load, typename Use> __device__ inline void stream(Load load, Use use) {
  F first[G];
#pragma unroll
  for (int e = 0; e < G; e++) first[e] = load(e);
  stream_rest<F, N, G>(first, load, use);
}

__device__ inline void clear(v16f& t) {
#pragma unroll
  for (int i = 0; i < 16; i++) t[i] = 0.f;
}
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float other_half(float v) { return __shfl_xor(v, 32, 64); }
__device__ inline float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// ---- forward -------------------------------------------------------------------------------------------------------------------
// Bound by its instructions (above).  A wave owns 32 rows of one of the two maps; the waves of a pair exchange their results at the end.  (Both maps in one wave share the fragments of
// v, but need 256 accumulators for the widest heads, which spill, and 128 for heads of 64, which leave two waves a SIMD and nothing in
// flight beside them.)
constexpr int F_GROUPS = 2, F_ROWS = 32 * F_GROUPS, F_THREADS = 128 * F_GROUPS;

template <typename T, int DT>
__global__ void __launch_bounds__(F_THREADS, sizeof(T) == 4 ? (DT == 128 ? 1 : 2) : DT == 128 ? 2 : 3) diff_forward_kernel(DiffArgs a) {
  typedef Ops<T> O;
  typedef Sizes<T, DT> S;
  __shared__ __attribute__((aligned(16))) T lds[4 * S::KC * S::W];   // keys and values, two buffers each
  constexpr int BUF = S::KC * S::W, G = sizeof(T) == 2 ? 4 : 2, GK = G < S::KS ? G : S::KS;
  constexpr bool EARLY = sizeof(T) == 2 && DT <= 64;
  Work w;
  if (!work_of(a, w)) return;
  const int part = w.part, unit = w.unit, b = w.b, hk = w.hk;
  const int tile = a.tiles - 1 - w.tile;   // under a causal mask the last rows see the most keys: they go first
  const Seq s = sequence(a, b);
  const int R = s.nq * a.group, r0 = tile * F_ROWS, room = a.q_starts ? R : a.tq * a.group;
  if (r0 >= room) return;
  const int lane = threadIdx.x & 63, wave = wave_of_thread(), c = lane & 31, hh = lane >> 5, m = wave & 1, rg = wave >> 1;
  const int wr0 = r0 + 32 * rg, r = wr0 + c;
  const bool live = r < R;
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group);
  const T* kp = rows_of(a, static_cast<const T*>(a.k), b, s.k0, a.k_token, a.k_batch) + (int64_t)hk * 2 * a.dim;
  const T* vp = rows_of(a, static_cast<const T*>(a.v), b, s.k0, a.v_token, a.v_batch) + (int64_t)hk * 2 * a.dim;
  typename O::Frag qf[S::KS];
  float lam = live ? a.lam[a.lam_token ? (s.q0 + i) * a.heads + h : h] : 0.f;
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
  // (the keys of a part: whole tiles of 32; the same number in long and short sequences, which then have fewer parts)
  const int per = a.parts == 1 ? s.nk : (((a.tk + 31) / 32 + a.parts - 1) / a.parts) * 32;
  const int begin = part * per, last = r0 < R ? min(limit(min(r0 + F_ROWS, R) - 1), begin + per) : 0;
  const int see = min(live ? limit(r) : s.nk, last), least = min(limit(wr0), last), reach = wr0 < R ? min(limit(min(wr0 + 31, R - 1)), last) : 0;
  v16f o[S::VT];
#pragma unroll
  for (int t = 0; t < S::VT; t++) clear(o[t]);
  // The log-sum comes from the weights before they are rounded, the values' divisor from the rounded ones: those then add up to one, so that what the
  // values of all keys have in common, which the difference of the maps reduces to 1 - lambda of itself, is not touched by the rounding.
  float mx = -INFINITY, sum = 0.f, weight = 0.f;
  LaneAt at = O::template lane_at<S::W>(lane);
  // One barrier a tile: behind it the tile has arrived, and nobody reads the other buffer any more, into which the next tile is sent for.
  Loader<T, DT, true, F_THREADS> ks;
  Loader<T, DT, false, F_THREADS> vs;
  ks.plan(a.dim, [&](int row) { return row * a.k_token; });
  vs.plan(a.dim, [&](int row) { return row * a.v_token; });
  const uint32_t to = lds_address(lds) + wave * 1024;
  auto fetch = [&](int j, int buf) {
    ks.load(kp + j * a.k_token, (s.nk - 1 - j) * a.k_token + 2 * a.dim, to + buf * (BUF * (int)sizeof(T)));
    vs.load(vp + j * a.v_token, (s.nk - 1 - j) * a.v_token + 2 * a.dim, to + (2 + buf) * (BUF * (int)sizeof(T)));
  };
#pragma unroll
  for (int t = 0; t < S::KS; t++) arrived(qf[t]);
  arrived(lam);
  if (begin < last) fetch(begin, 0);
  for (int j0 = begin, buf = 0; j0 < last; j0 += S::KC, buf ^= 1) {
    wait_step<0>();
    if (j0 + S::KC < last) fetch(j0 + S::KC, buf ^ 1);
    const T* Ks = lds + buf * BUF;
    const T* Vs = lds + (2 + buf) * BUF;
    if (j0 < reach) {
      at.fresh();
      v16f sc;
      clear(sc);
      typename O::Frag kf[GK], vf[G];
      auto key = [&](int t) { return O::template rowwise<S::W>(Ks, 0, m * DT + 16 * t, at); };
      auto value = [&](int x) { return O::template transposed<S::W>(Vs, 32 * (x % S::VT), 16 * (x / S::VT), at); };
      stream_first(kf, key);
      if (EARLY) stream_first(vf, value);   // (they arrive while the scores are worked on)
      stream_rest<typename O::Frag, S::KS, GK>(kf, key, [&](int t, const typename O::Frag& f) { sc = O::mma(f, qf[t], sc); });
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
        weight *= f;
#pragma unroll
        for (int t = 0; t < S::VT; t++) o[t] *= f;
      }
      const float base = finite_or_zero(mx);   // (a row that has seen no key: exp2(-inf) = 0)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        sc[v] = exp2_fast(fmaf(sc[v], a.c, -base));
        sum += sc[v];
      }
      const typename O::Frag p[2] = {O::operand(sc, 0), O::operand(sc, 1)};
      weight = O::add_up(p[1], O::add_up(p[0], weight));
      if (!EARLY) stream_first(vf, value);
      stream_rest<typename O::Frag, 2 * S::VT, G>(vf, value, [&](int x, const typename O::Frag& f) { o[x % S::VT] = O::mma(f, p[x / S::VT], o[x % S::VT]); });
    }
  }
  __syncthreads();   // (the exchange below writes where the last tile was read)
  sum += other_half(sum);
  weight += other_half(weight);
  if (a.parts > 1) {   // a part's sums, joined by diff_join_kernel
    if (!live) return;
    const int64_t place = (((int64_t)part * a.units + unit) * (a.tq * a.group) + r) * 2 + m;
    float* p = a.part + place * 2 * a.dim + 4 * hh;
#pragma unroll
    for (int t = 0; t < S::VT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        if (32 * t + 8 * g < 2 * a.dim) *reinterpret_cast<float4*>(p + 32 * t + 8 * g) = make_float4(o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]);
    if (hh == 0) *reinterpret_cast<float4*>(a.part_ml + place * 4) = make_float4(mx, sum, weight, 0.f);
    return;
  }
  const int64_t row = s.q0 + i;
  const float norm = weight > 0.f || weight != weight ? 1.f / weight : 0.f;   // (NaN stays NaN)
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

// Joins the parts of a row: one wave a row, bound by the latency of its code and of two rounds of loads (6 us for 256 rows of 12 parts).  Lane p holds the maximum and the sums of part p (at
// most 64 parts), so that the weights of all parts are known before the sums are read.  Then a lane has four channels, and with heads of up to 64 the halves
// of a wave take a part each.
template <typename T>
__global__ void __launch_bounds__(256) diff_join_kernel(DiffArgs a) {
  const int room = a.tq * a.group, unit = blockIdx.y, r = (int)blockIdx.x * 4 + wave_of_thread(), lane = threadIdx.x & 63;
  if (r >= room) return;
  const int b = quotient(unit, a.by_heads), hk = unit - b * a.kv_heads;
  const Seq s = sequence(a, b);
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group);
  const bool live = r < s.nq * a.group;
  if (!live && a.q_starts) return;
  const int64_t row = s.q0 + i, step = (int64_t)a.units * room, at = (int64_t)unit * room + r;
  const bool both = a.dim <= 64;
  const int half = both ? lane >> 5 : 0, col = 4 * (both ? lane & 31 : lane), each = both ? 2 : 1;
  const bool in = col < 2 * a.dim;
  float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
  if (live) {
    float f[2], lse[2];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      float4 ml = make_float4(-INFINITY, 0.f, 0.f, 0.f);
      if (lane < a.parts) ml = *reinterpret_cast<const float4*>(a.part_ml + ((at + lane * step) * 2 + k) * 4);
      const float top = wave_max(ml.x), e = exp2_fast(ml.x - finite_or_zero(top)), sum = wave_sum(e * ml.y), weight = wave_sum(e * ml.z);
      f[k] = weight > 0.f || weight != weight ? e / weight : 0.f;   // (NaN stays NaN)
      lse[k] = sum > 0.f ? top + __log2f(sum) : sum;
    }
    if (a.lse && lane < 2) a.lse[(int64_t)(lane * a.heads + h) * a.q_rows + row] = lane ? lse[1] : lse[0];
    const float* from = a.part + (at + half * step) * 4 * a.dim + col;
    for (int p0 = 0; p0 < a.parts; p0 += 4 * each) {   // (the loads of four or eight parts in flight)
      float4 v[2][4];
#pragma unroll
      for (int q = 0; q < 4; q++)
#pragma unroll
        for (int k = 0; k < 2; k++)
          v[k][q] = in && p0 + q * each + half < a.parts ? *reinterpret_cast<const float4*>(from + (p0 + q * each) * step * 4 * a.dim + k * 2 * a.dim) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int q = 0; q < 4; q++)
#pragma unroll
        for (int k = 0; k < 2; k++) {
          const int p = p0 + q * each + half;
          const float g = __shfl(f[k], min(p, 63), 64);   // (zero in the lanes behind the parts)
          o[k].x += g * v[k][q].x; o[k].y += g * v[k][q].y; o[k].z += g * v[k][q].z; o[k].w += g * v[k][q].w;
        }
    }
    if (both)
#pragma unroll
      for (int k = 0; k < 2; k++) { o[k].x += other_half(o[k].x); o[k].y += other_half(o[k].y); o[k].z += other_half(o[k].z); o[k].w += other_half(o[k].w); }
  }
  if (!in || half) return;
  const float lam = live ? a.lam[a.lam_token ? row * a.heads + h : h] : 0.f;
  T* op = rows_of(a, static_cast<T*>(a.out), b, s.q0, a.o_token, a.o_batch) + i * a.o_token + (int64_t)h * 2 * a.dim + col;
  Ops<T>::store4(op, o[0].x - lam * o[1].x, o[0].y - lam * o[1].y, o[0].z - lam * o[1].z, o[0].w - lam * o[1].w);
  if (a.o2 && live) Ops<T>::store4(static_cast<T*>(a.o2) + row * a.o2_token + (int64_t)h * 2 * a.dim + col, o[1].x, o[1].y, o[1].z, o[1].w);
}

// What the pass over the keys takes of a row is divided by the scale: below this one the gradients are refused.
constexpr float LEAST_SCALE = 0x1p-100f;

// What the pass over the queries leaves of a row's map m for the pass over the keys, and dlambda.
__device__ inline void leave_row(const DiffArgs& a, int64_t row, int h, int m, bool live, float lse, float delta, float lam) {
  RowValues* v = a.rows + row * a.heads + h;
  // The parts have to be finite.  A weight P_2 is at most one, so 2^-1000 of it is zero: a lambda of zero, and those below the normal numbers, which the logarithm's
  // instruction takes for zero.  Over the least scale of this pass (LEAST_SCALE) a thousand is still far below the largest number.
  const float weight = m == 0 ? 0.f : fabsf(lam) < 0x1p-126f ? -1000.f : __log2f(fabsf(lam));
  v->lse[m] = three_parts(live ? (weight - lse) / a.c : 0.f);
  v->delta[m] = three_parts(live ? -delta : 0.f);
  if (m == 1) {
    v->lam_negative = live && lam < 0.f;
    if (a.lam_token) a.dlam[row * a.heads + h] = live ? -delta : 0.f;
    else a.second[(int64_t)h * a.q_rows + row] = live ? delta : 0.f;
  }
}

// whether the weights of a row that sees so many keys depend on its scores
__device__ inline bool moves(int keys) { return keys != 1; }

// ---- backward: queries ------------------------------------------------------------------------------------------------------------
// dq, delta and dlambda.  delta first comes from the kept outputs, delta_2 = dO . (P_2 v), delta_1 = dO . out + lambda delta_2, which were rounded;
// the pass over the keys gives what is missing, rowsum(P_m (dP - delta_m)) in fp32, so that dlambda and the deltas that the other kernel
// reads are exact to fp32 rounding (with the kept bf16 outputs alone dlambda is off by their rounding, a thousandth).
// Bound by its instructions, as the forward kernel is.  Both maps of 32 rows in a wave share dP; where that needs more registers than two waves a SIMD have (the widest heads, fp32), a wave takes one
// map and computes dP for itself.
template <typename T, int DT> struct QSizes {
  static constexpr bool SPLIT = DT * sizeof(T) >= 256;
  static constexpr int MAPS = SPLIT ? 1 : 2, ROWS = SPLIT ? 64 : 128;
};

template <typename T, int DT>
__global__ void __launch_bounds__(256, DT * sizeof(T) <= 256 ? 2 : 1) diff_backward_q_kernel(DiffArgs a) {
  typedef Ops<T> O;
  typedef Sizes<T, DT> S;
  typedef QSizes<T, DT> Z;
  __shared__ __attribute__((aligned(16))) T lds[4 * S::KC * S::W];   // keys and values, two buffers each
  constexpr int BUF = S::KC * S::W, G = sizeof(T) == 2 && DT == 64 ? 4 : 2, MAPS = Z::MAPS;
  Work w;
  if (!work_of(a, w)) return;
  const int part = w.part, unit = w.unit, b = w.b, hk = w.hk, tile = a.tiles - 1 - w.tile;
  const Seq s = sequence(a, b);
  const int R = s.nq * a.group, r0 = tile * Z::ROWS, room = a.q_starts ? R : a.tq * a.group;
  if (r0 >= room) return;
  const int lane = threadIdx.x & 63, wave = wave_of_thread(), c = lane & 31, hh = lane >> 5;
  const int m0 = Z::SPLIT ? wave & 1 : 0, wr0 = r0 + 32 * (Z::SPLIT ? wave >> 1 : wave), r = wr0 + c;   // the wave's first map, its first row
  const bool live = r < R;
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group);
  const int64_t row = s.q0 + i;
  const T* kp = rows_of(a, static_cast<const T*>(a.k), b, s.k0, a.k_token, a.k_batch) + (int64_t)hk * 2 * a.dim;
  const T* vp = rows_of(a, static_cast<const T*>(a.v), b, s.k0, a.v_token, a.v_batch) + (int64_t)hk * 2 * a.dim;
  typename O::Frag qf[MAPS * S::KS];
  RowFrags<T, DT> gf;
  {
    const T* qp = rows_of(a, static_cast<const T*>(a.q), b, s.q0, a.q_token, a.q_batch) + i * a.q_token + (int64_t)h * 2 * a.dim + m0 * a.dim;
#pragma unroll
    for (int t = 0; t < MAPS * S::KS; t++) {
      const int d = 16 * (t % S::KS) + 8 * hh;
      qf[t] = O::zero();
      if (live && d < a.dim) qf[t] = O::load(qp + t / S::KS * a.dim + d);
    }
  }
  const int64_t o_at = i * a.o_token + (int64_t)h * 2 * a.dim;
  own_row<T, DT, false>(gf, rows_of(a, static_cast<const T*>(a.dout), b, s.q0, a.o_token, a.o_batch) + o_at, live, a.dim, hh);
  float lam = 0.f, lse[MAPS], delta[MAPS], rest[MAPS];
  if (live) lam = a.lam[a.lam_token ? row * a.heads + h : h];
#pragma unroll
  for (int m = 0; m < MAPS; m++) {
    lse[m] = live ? a.lse[(int64_t)((m0 + m) * a.heads + h) * a.q_rows + row] : 0.f;
    rest[m] = 0.f;
  }
  {
    const T* kept[2] = {rows_of(a, static_cast<const T*>(a.out), b, s.q0, a.o_token, a.o_batch) + o_at,
                        static_cast<const T*>(a.o2) + row * a.o2_token + (int64_t)h * 2 * a.dim};
    float dot[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
      for (int t = 0; t < 2 * S::KS; t++)
        if (live && 16 * t + 8 * hh < 2 * a.dim) {
          const typename O::Frag f = O::load(kept[k] + 16 * t + 8 * hh);
#pragma unroll
          for (int e = 0; e < 8; e++) dot[k] += O::get(f, e) * O::get(gf[t], e);
        }
    dot[0] += other_half(dot[0]);
    dot[1] += other_half(dot[1]);
    dot[0] += lam * dot[1];
#pragma unroll
    for (int m = 0; m < MAPS; m++) delta[m] = m0 + m ? dot[1] : dot[0];
  }
  const int off = s.nk - s.nq;
  auto limit = [&](int x) { return a.causal ? min(s.nk, query_of(a, x) + off + 1) : s.nk; };
  const int see = live ? limit(r) : s.nk;
  const int least = limit(wr0), reach = wr0 < R ? limit(min(wr0 + 31, R - 1)) : 0;
  int begin = 0, last = r0 < R ? limit(min(r0 + Z::ROWS, R) - 1) : 0;
  // The workgroup walks its keys twice where its first row sees few (the waves whose first row does work in the first pass, which ends where the
  // last of their rows ends).
  const bool two = sizeof(T) == 2 && min(limit(r0), last) <= EXACT_KEYS, few = least <= EXACT_KEYS;
  if (a.parts > 1) {   // (the keys of rows with few are one part's, so that the two passes below see all of them)
    const int per = (((a.tk + 31) / 32 + a.parts - 1) / a.parts) * 32;
    if (two) begin = part ? last : 0;
    else { begin = part * per; last = min(last, begin + per); }
  }
  v16f dq[MAPS][S::DTT];
#pragma unroll
  for (int m = 0; m < MAPS; m++)
#pragma unroll
    for (int t = 0; t < S::DTT; t++) clear(dq[m][t]);
  // Rows with few keys: a rounding of the kept outputs is as large as their small dS (two keys: dq off by 5e-3 where its own rounding is 1.7e-3 and that of dS
  // as much, 128 keys 2.8e-3, 700 keys 2.5e-3 as without it), so delta is completed by a pass of its own first.  fp32 outputs are as exact as the products; there
  // one pass does, and a row of one key, whose gradient is zero to the last bit, gets it by name (`moves`).
  LaneAt at = O::template lane_at<S::W>(lane);
  Loader<T, DT, true, 256> ks;
  Loader<T, DT, false, 256> vs;
  ks.plan(a.dim, [&](int row) { return row * a.k_token; });
  vs.plan(a.dim, [&](int row) { return row * a.v_token; });
  const uint32_t to = lds_address(lds) + wave * 1024;
  auto fetch = [&](int j, int buf) {
    ks.load(kp + j * a.k_token, (s.nk - 1 - j) * a.k_token + 2 * a.dim, to + buf * (BUF * (int)sizeof(T)));
    vs.load(vp + j * a.v_token, (s.nk - 1 - j) * a.v_token + 2 * a.dim, to + (2 + buf) * (BUF * (int)sizeof(T)));
  };
#pragma unroll
  for (int t = 0; t < 2 * S::KS; t++) arrived(gf[t]);
#pragma unroll
  for (int t = 0; t < MAPS * S::KS; t++) arrived(qf[t]);
#pragma unroll
  for (int m = 0; m < MAPS; m++) { arrived(lse[m]); arrived(delta[m]); }
  for (int pass = two ? 0 : 1; pass < 2; pass++) {
    if (two && pass == 1) {
#pragma unroll
      for (int m = 0; m < MAPS; m++) {
        delta[m] += rest[m] + other_half(rest[m]);
        rest[m] = 0.f;
      }
    }
    const int end = pass ? last : min(last, EXACT_KEYS + 31);   // (32 rows of a wave see up to 31 keys more than its first)
    __syncthreads();   // (the first pass may still read what is fetched anew)
    if (begin < end) fetch(begin, 0);
    for (int j0 = begin, buf = 0; j0 < end; j0 += S::KC, buf ^= 1) {
      wait_step<0>();
      if (j0 + S::KC < end) fetch(j0 + S::KC, buf ^ 1);
      const T* Ks = lds + buf * BUF;
      const T* Vs = lds + (2 + buf) * BUF;
      if (j0 < reach && (pass || few)) {
        at.fresh();
        v16f sc[MAPS], dp;
        clear(dp);
#pragma unroll
        for (int m = 0; m < MAPS; m++) clear(sc[m]);
        const int base = m0 * DT;   // the first map's columns
        stream<typename O::Frag, (2 + MAPS) * S::KS, G>(
            [&](int x) { return x < MAPS * S::KS ? O::template rowwise<S::W>(Ks, 0, base + 16 * x, at) : O::template rowwise<S::W>(Vs, 0, 16 * (x - MAPS * S::KS), at); },
            [&](int x, const typename O::Frag& f) {
              if (x < MAPS * S::KS) sc[x / S::KS] = O::mma(f, qf[x], sc[x / S::KS]);
              else dp = O::mma(f, gf[x - MAPS * S::KS], dp);
            });
        if (j0 + 32 > least) {
#pragma unroll
          for (int v = 0; v < 16; v++)
            if (j0 + 8 * (v >> 2) + 4 * hh + (v & 3) >= see) {
#pragma unroll
              for (int m = 0; m < MAPS; m++) sc[m][v] = -INFINITY;
            }
        }
#pragma unroll
        for (int m = 0; m < MAPS; m++) {
#pragma unroll
          for (int v = 0; v < 16; v++) {
            sc[m][v] = exp2_fast(fmaf(sc[m][v], a.c, -lse[m])) * (dp[v] - delta[m]);
            rest[m] += sc[m][v];
          }
          if (pass == 1) {
            const typename O::Frag p[2] = {O::operand(sc[m], 0), O::operand(sc[m], 1)};
            constexpr int GT = 2 * S::DTT < G ? 2 * S::DTT : G;
            stream<typename O::Frag, 2 * S::DTT, GT>([&](int x) { return O::template transposed<S::W>(Ks, base + m * DT + 32 * (x % S::DTT), 16 * (x / S::DTT), at); },
                                                     [&](int x, const typename O::Frag& f) { dq[m][x % S::DTT] = O::mma(f, p[x / S::DTT], dq[m][x % S::DTT]); });
          }
        }
      }
    }
  }
  if (a.parts > 1) {   // a part's sums, joined by diff_join_q_kernel
    if (!live) return;
    const int64_t rows = (int64_t)a.tq * a.group, place = ((int64_t)part * a.units + unit) * rows + r;
#pragma unroll
    for (int m = 0; m < MAPS; m++) {
      float* p = a.part + place * 2 * a.dim + (m0 + m) * a.dim + 4 * hh;
#pragma unroll
      for (int t = 0; t < S::DTT; t++)
#pragma unroll
        for (int g = 0; g < 4; g++)
          if (32 * t + 8 * g < a.dim)
            *reinterpret_cast<float4*>(p + 32 * t + 8 * g) = make_float4(dq[m][t][4 * g], dq[m][t][4 * g + 1], dq[m][t][4 * g + 2], dq[m][t][4 * g + 3]);
      rest[m] += other_half(rest[m]);
      if (hh == 0) a.part_ml[place * 2 + m0 + m] = rest[m] + (part == 0 ? delta[m] : 0.f);   // (their sum is delta)
    }
    return;
  }
  if (r >= room) return;
  T* dqp = rows_of(a, static_cast<T*>(a.dq), b, s.q0, a.q_token, a.q_batch) + i * a.q_token + (int64_t)h * 2 * a.dim + 4 * hh;
#pragma unroll
  for (int m = 0; m < MAPS; m++) {
    delta[m] += rest[m] + other_half(rest[m]);
    const float f = live && moves(see) ? (m0 + m ? -lam * a.scale : a.scale) : 0.f;
#pragma unroll
    for (int t = 0; t < S::DTT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        if (32 * t + 8 * g < a.dim)
          O::store4(dqp + (m0 + m) * a.dim + 32 * t + 8 * g, f * dq[m][t][4 * g], f * dq[m][t][4 * g + 1], f * dq[m][t][4 * g + 2], f * dq[m][t][4 * g + 3]);
    if (hh == 0) leave_row(a, row, h, m0 + m, live, lse[m], delta[m], lam);
  }
}

// Adds the parts of a row's dq and delta, always in the same order: a thread takes four channels.
template <typename T>
__global__ void __launch_bounds__(256) diff_join_q_kernel(DiffArgs a) {
  const int64_t rows = (int64_t)a.tq * a.group;
  const int x = (int)blockIdx.x * 256 + threadIdx.x, unit = blockIdx.y, r = quotient(x, a.by_quads), col = (x - r * (a.dim / 2)) * 4;
  if (r >= rows) return;
  const int b = quotient(unit, a.by_heads), hk = unit - b * a.kv_heads;
  const Seq s = sequence(a, b);
  const bool live = r < s.nq * a.group;
  if (!live && a.q_starts) return;
  const int i = query_of(a, r), h = hk * a.group + (r - i * a.group), m = col / a.dim;
  const int64_t row = s.q0 + i, step = a.units * rows, at = unit * rows + r;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  float delta = 0.f;
  if (live)
    for (int p = 0; p < a.parts; p++) {
      const float4 y = *reinterpret_cast<const float4*>(a.part + (at + p * step) * 2 * a.dim + col);
      t.x += y.x; t.y += y.y; t.z += y.z; t.w += y.w;
      delta += a.part_ml[(at + p * step) * 2 + m];
    }
  const float lam = live ? a.lam[a.lam_token ? row * a.heads + h : h] : 0.f, f = !moves(a.causal ? min(s.nk, i + s.nk - s.nq + 1) : s.nk) ? 0.f : m ? -lam * a.scale : a.scale;
  T* dq = rows_of(a, static_cast<T*>(a.dq), b, s.q0, a.q_token, a.q_batch) + i * a.q_token + (int64_t)h * 2 * a.dim + col;
  Ops<T>::store4(dq, f * t.x, f * t.y, f * t.z, f * t.w);
  if (col == m * a.dim) leave_row(a, row, h, m, live, live ? a.lse[(int64_t)(m * a.heads + h) * a.q_rows + row] : 0.f, delta, lam);
}

// dlambda of a head: minus the sum of delta_2 over the sequences' rows, always in the same order.  One workgroup a head, beside the workgroups that own keys.
template <int THREADS> __device__ inline void sum_lambda(const DiffArgs& a, int h) {
  __shared__ float red[THREADS / 64];
  const float* d = a.second + (int64_t)h * a.q_rows;
  float t = 0.f;
  if (!a.q_starts) {   // (rows behind a sequence's queries hold zeros)
    for (int64_t x = threadIdx.x; x < a.q_rows; x += THREADS) t += d[x];
  } else {
    for (int b = threadIdx.x >> 6; b < a.batch; b += THREADS / 64) {
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
    for (int k = 0; k < THREADS / 64; k++) z += red[k];
    a.dlam[h] = -z;
  }
}

// ---- backward: keys ------------------------------------------------------------------------------------------------------------------
// Bound by the longer half of a pair.  A pair of waves owns 32 keys: one computes P and dS of a tile of rows and leaves them in LDS as operands, the other multiplies the tile before
// it into dk and dv.  In one wave the accumulators (128 registers for heads of 64) beside the keys' and values' fragments (64) and three tiles
// need more than 256 registers: one wave a SIMD, and most of its time went into copies to and from accumulation registers.
//
// What belongs to a row (log-sums, deltas, lambda) is a register index here, not a lane.  It comes to all lanes as a product: the fp32 value in
// three bf16 parts, which hold all of its bits, times ones; as the initial accumulator of the scores it costs no vector instruction, and an eighth of the LDS
// traffic of reading it for every register.
template <typename T, int DT> struct KvSizes {
  static constexpr int PAIRS = DT * sizeof(T) <= 128 && DT > 32 ? 4 : DT * sizeof(T) <= 256 ? 2 : 1;   // pairs of waves of a workgroup
  static constexpr int BUFFERS = DT * sizeof(T) <= 256 ? 3 : 2;   // of a tile of rows (two, and one more barrier a tile, where three exceed LDS)
  static constexpr int KEYS = 32 * PAIRS, THREADS = 128 * PAIRS;
};
// adds a row's value, held by the row's lane of the lower half, to a tile's rows
__device__ inline v16f add_rows(uint2 parts, int hh, const v16f& c) {
  const uint4 a = hh ? make_uint4(0, 0, 0, 0) : make_uint4(parts.x, parts.y, 0, 0), one = make_uint4(0x3f803f80u, 0x3f80u, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, one), c, 0, 0, 0);
}

template <typename T, int DT>
__global__ void __launch_bounds__((KvSizes<T, DT>::THREADS), sizeof(T) == 2 && DT <= 64 ? 2 : 1) diff_backward_kv_kernel(DiffArgs a) {
  typedef Ops<T> O;
  typedef Sizes<T, DT> S;
  typedef KvSizes<T, DT> Z;
  constexpr int BUF = S::KC * S::W, G = sizeof(T) == 2 ? 4 : 2, NB = Z::BUFFERS, FRAG = sizeof(typename O::Frag);
  __shared__ __attribute__((aligned(16))) T lds[2 * NB * BUF];                         // queries and dO
  __shared__ __attribute__((aligned(16))) RowValues st[NB][43];                        // the rows' values: 32, and room for the 2048 bytes that two waves write
  __shared__ __attribute__((aligned(16))) char ex[2][Z::PAIRS][6 * 64 * FRAG];         // P_1 - lambda P_2, dS_1, dS_2 of a tile, two operands each
  if ((int)blockIdx.x >= a.work) {   // the workgroups behind those of the keys
    sum_lambda<Z::THREADS>(a, (int)blockIdx.x - a.work);
    return;
  }
  Work w;
  if (!work_of<true>(a, w)) return;
  const int part = w.part, unit = w.unit, b = w.b, hk = w.hk, tile = w.tile;   // under a causal mask the first keys are seen by the most rows
  const Seq s = sequence(a, b);
  const int R = s.nq * a.group, j0 = tile * Z::KEYS, room = a.q_starts ? s.nk : a.tk;
  if (j0 >= room) return;
  const int lane = threadIdx.x & 63, wave = wave_of_thread(), c = lane & 31, hh = lane >> 5;
  const int pair = wave % Z::PAIRS;
  const bool producer = wave < Z::PAIRS;   // (waves go to the four SIMDs in turn: one of each kind on a SIMD)
  const int wj0 = j0 + 32 * pair, j = wj0 + c;
  const bool live = j < s.nk;
  const T* qp = rows_of(a, static_cast<const T*>(a.q), b, s.q0, a.q_token, a.q_batch) + (int64_t)hk * a.group * 2 * a.dim;
  const T* gp = rows_of(a, static_cast<const T*>(a.dout), b, s.q0, a.o_token, a.o_batch) + (int64_t)hk * a.group * 2 * a.dim;
  const int64_t k_at = (int64_t)j * a.k_token + (int64_t)hk * 2 * a.dim, v_at = (int64_t)j * a.v_token + (int64_t)hk * 2 * a.dim;
  // the first row that sees key j, and those of the pair's first and last key
  const int off = s.nk - s.nq;
  auto from = [&](int key) { return a.causal ? max(0, key - off) * a.group : 0; };
  const int first = live ? from(j) : 0;
  const int wfirst = wj0 < s.nk ? from(wj0) : R, wlast = from(min(wj0 + 31, s.nk - 1));
  LaneAt at = O::template lane_at<S::W>(lane);
  Loader<T, DT, true, Z::THREADS> qs;
  Loader<T, DT, false, Z::THREADS> gs;
  // row r0 + x of a tile, from the token of its first row
  auto plan = [&](int r0) {
    auto place = [&](int x, int64_t token) { const int i = query_of(a, r0 + x); return (i - query_of(a, r0)) * token + (int64_t)(r0 + x - i * a.group) * 2 * a.dim; };
    qs.plan(a.dim, [&](int x) { return place(x, a.q_token); });
    gs.plan(a.dim, [&](int x) { return place(x, a.o_token); });
  };
  plan(0);
  const bool alike = 32 % a.group == 0;   // the rows of all tiles lie alike
  const int piece = wave * 64 + lane, value_row = piece / 3;
  const uint32_t to = lds_address(lds) + wave * 1024;
  auto fetch = [&](int r0, int buf) {
    const int i0 = query_of(a, r0);
    if (!alike) plan(r0);
    qs.load(qp + i0 * a.q_token, (s.nq - 1 - i0) * a.q_token + a.group * 2 * a.dim, to + buf * (BUF * (int)sizeof(T)));
    gs.load(gp + i0 * a.o_token, (s.nq - 1 - i0) * a.o_token + a.group * 2 * a.dim, to + (NB + buf) * (BUF * (int)sizeof(T)));
    if (wave < 2) {   // 96 pieces of row values
      const int r = r0 + value_row, i = query_of(a, r);
      const rsrc_words_t w = buffer_of(a.rows + (s.q0 + i0) * a.heads + hk * a.group, 0xfffffff0);
      load_lds16(w, (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_address(st[buf]) + wave * 1024), value_row < 32 && r < R ? (uint32_t)(((i - i0) * a.heads + r - i * a.group) * 48 + piece % 3 * 16) : ~0u);
    }
  };
  int begin = j0 < s.nk ? from(j0) / S::KC : (R + S::KC - 1) / S::KC, end = (R + S::KC - 1) / S::KC;   // tiles of rows
  if (a.parts > 1) {
    const int per = (max(end - begin, 0) + a.parts - 1) / a.parts;
    begin += part * per;
    end = min(end, begin + per);
  }
  // The last tile first: under a causal mask all workgroups of a unit reach the last rows, few the first ones, and those that begin together find
  // each other's tiles in the cache.
  const int tiles = max(end - begin, 0);
  auto row_of = [&](int t) { return (end - 1 - t) * S::KC; };
  auto seen = [&](int t) { return row_of(t) + 32 > wfirst; };   // some key of the pair is seen by the tile's rows
  // Tile t is worked on from buffer t mod NB by the first wave of a pair while the second one has the tile before it and the tile after it
  // is on its way.
  auto next = [](int x) { return x == NB - 1 ? 0 : x + 1; };
  if (tiles > 0) fetch(row_of(0), 0);
  auto stage = [&](int t, int buf) {
    wait_step<0>();   // tile t has arrived, the pairs are done with tile t - 2, and what the first waves left of tile t - 1 is there
    if (NB > 2 && t + 1 < tiles) fetch(row_of(t + 1), next(buf));
  };
  auto stage_behind = [&](int t, int buf) {
    if (NB == 2) {   // the next tile goes where the one before was read
      wait_step<0>();
      if (t + 1 < tiles) fetch(row_of(t + 1), next(buf));
    }
  };
  if (producer) {
    __builtin_amdgcn_s_setprio(1);   // (the longer half of a pair)
    RowFrags<T, DT> kf, vf;
    own_row<T, DT, true>(kf, rows_of(a, static_cast<const T*>(a.k), b, s.k0, a.k_token, a.k_batch) + k_at, live, a.dim, hh);
    own_row<T, DT, false>(vf, rows_of(a, static_cast<const T*>(a.v), b, s.k0, a.v_token, a.v_batch) + v_at, live, a.dim, hh);
#pragma unroll
    for (int t = 0; t < 2 * S::KS; t++) { arrived(kf[t]); arrived(vf[t]); }
    for (int t = 0, buf = 0; t <= tiles; t++, buf = next(buf)) {
      stage(t, buf);
      if (t < tiles && seen(t)) {
        const T* Qs = lds + buf * BUF;
        const T* Gs = lds + (NB + buf) * BUF;
        typename O::Frag* x = reinterpret_cast<typename O::Frag*>(ex[t & 1][pair]) + lane;
        at.fresh();
        v16f dp, wt, scores[2];
        clear(dp);
        const uint32_t negative = (uint32_t)__ballot(st[buf][c].lam_negative != 0);   // the rows whose lambda is below zero
#pragma unroll
        for (int m = 0; m < 2; m++) {
          clear(scores[m]);
          scores[m] = add_rows(st[buf][c].lse[m], hh, scores[m]);
        }
        stream<typename O::Frag, 4 * S::KS, G>([&](int e) { return O::template rowwise<S::W>(e < 2 * S::KS ? Qs : Gs, 0, 16 * (e % (2 * S::KS)), at); },
                                               [&](int e, const typename O::Frag& f) {
                                                 if (e < 2 * S::KS) scores[e / S::KS] = O::mma(f, kf[e], scores[e / S::KS]);
                                                 else dp = O::mma(f, vf[e - 2 * S::KS], dp);
                                               });
        const int r0 = row_of(t);
        if (r0 < wlast) {
#pragma unroll
          for (int v = 0; v < 16; v++)
            if (r0 + 8 * (v >> 2) + 4 * hh + (v & 3) < first) { scores[0][v] = -INFINITY; scores[1][v] = -INFINITY; }
        }
#pragma unroll
        for (int m = 0; m < 2; m++) {
          v16f& sc = scores[m];
          // (delta is subtracted from the finished dP: a softmax over one key has dP = delta to the last bit, and a gradient of zero)
          const v16f ds = add_rows(st[buf][c].delta[m], hh, dp);
          if (m == 0) {
#pragma unroll
            for (int v = 0; v < 16; v++) {
              wt[v] = exp2_fast(a.c * sc[v]);
              sc[v] = wt[v] * ds[v];
            }
          } else {
#pragma unroll
            for (int v = 0; v < 16; v++) sc[v] = exp2_fast(a.c * sc[v]);   // |lambda| P_2
            if (negative) {
#pragma unroll
              for (int v = 0; v < 16; v++)
                if (negative >> (8 * (v >> 2) + 4 * hh + (v & 3)) & 1) sc[v] = -sc[v];
            }
#pragma unroll
            for (int v = 0; v < 16; v++) {
              wt[v] -= sc[v];
              sc[v] = -sc[v] * ds[v];
            }
          }
#pragma unroll
          for (int u = 0; u < 2; u++) x[(2 + 2 * m + u) * 64] = O::operand(sc, u);
        }
#pragma unroll
        for (int u = 0; u < 2; u++) x[u * 64] = O::operand(wt, u);
      }
      stage_behind(t, buf);
    }
    return;
  }
  v16f dv[S::VT], dk[2][S::DTT];
#pragma unroll
  for (int t = 0; t < S::VT; t++) { clear(dv[t]); clear(dk[t / S::DTT][t % S::DTT]); }
  for (int t = 0, buf = 0, before = NB - 1; t <= tiles; t++, before = buf, buf = next(buf)) {
    stage(t, buf);
    if (t > 0 && seen(t - 1)) {
      const T* Qs = lds + before * BUF;
      const T* Gs = lds + (NB + before) * BUF;
      const typename O::Frag* x = reinterpret_cast<const typename O::Frag*>(ex[(t - 1) & 1][pair]) + lane;
      at.fresh();
      typename O::Frag p[6];
#pragma unroll
      for (int e = 0; e < 6; e++) p[e] = x[e * 64];
      // columns of dO and of the two maps' queries, 2 W in all, for either half of the rows
      stream<typename O::Frag, 4 * S::VT, G>(
          [&](int e) { return O::template transposed<S::W>(e % (2 * S::VT) < S::VT ? Gs : Qs, 32 * (e % S::VT), 16 * (e / (2 * S::VT)), at); },
          [&](int e, const typename O::Frag& f) {
            const int u = e / (2 * S::VT), z = e % (2 * S::VT), m = z / S::DTT & 1;
            if (z < S::VT) dv[z] = O::mma(f, p[u], dv[z]);
            else dk[m][z % S::DTT] = O::mma(f, p[2 + 2 * m + u], dk[m][z % S::DTT]);
          });
    }
    stage_behind(t, buf);
  }
  if (a.parts > 1) {   // a part's sums, joined by diff_join_kv_kernel
    if (!live) return;
    float* q = a.part + ((((int64_t)part * a.units + unit) * a.tk) + j) * 4 * a.dim + 4 * hh;
#pragma unroll
    for (int t = 0; t < S::VT; t++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        if (32 * t + 8 * g < 2 * a.dim) *reinterpret_cast<float4*>(q + 32 * t + 8 * g) = make_float4(dv[t][4 * g], dv[t][4 * g + 1], dv[t][4 * g + 2], dv[t][4 * g + 3]);
        const v16f& d = dk[t / S::DTT][t % S::DTT];
        const int col = 32 * (t % S::DTT) + 8 * g;
        if (col < a.dim) *reinterpret_cast<float4*>(q + (2 + t / S::DTT) * a.dim + col) = make_float4(d[4 * g], d[4 * g + 1], d[4 * g + 2], d[4 * g + 3]);
      }
    return;
  }
  if (j >= room) return;
  T* dkp = rows_of(a, static_cast<T*>(a.dk), b, s.k0, a.k_token, a.k_batch) + k_at + 4 * hh;
  T* dvp = rows_of(a, static_cast<T*>(a.dv), b, s.k0, a.v_token, a.v_batch) + v_at + 4 * hh;
#pragma unroll
  for (int t = 0; t < S::VT; t++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      float y[4], z[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        y[e] = live ? dv[t][4 * g + e] : 0.f;
        z[e] = live ? a.scale * dk[t / S::DTT][t % S::DTT][4 * g + e] : 0.f;
      }
      if (32 * t + 8 * g < 2 * a.dim) O::store4(dvp + 32 * t + 8 * g, y[0], y[1], y[2], y[3]);
      const int col = 32 * (t % S::DTT) + 8 * g;
      if (col < a.dim) O::store4(dkp + t / S::DTT * a.dim + col, z[0], z[1], z[2], z[3]);
    }
}

// Adds the parts of a key's gradients, always in the same order: a thread takes four channels.
template <typename T>
__global__ void __launch_bounds__(256) diff_join_kv_kernel(DiffArgs a) {
  const int x = (int)blockIdx.x * 256 + threadIdx.x, unit = blockIdx.y, j = quotient(x, a.by_dim), col = (x - j * a.dim) * 4;
  if (j >= a.tk) return;
  const int b = quotient(unit, a.by_heads), hk = unit - b * a.kv_heads;
  const Seq s = sequence(a, b);
  const bool live = j < s.nk;
  if (!live && a.q_starts) return;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  if (live)
    for (int p = 0; p < a.parts; p++) {
      const float4 y = *reinterpret_cast<const float4*>(a.part + (((int64_t)p * a.units + unit) * a.tk + j) * 4 * a.dim + col);
      t.x += y.x; t.y += y.y; t.z += y.z; t.w += y.w;
    }
  if (col < 2 * a.dim) {
    T* dv = rows_of(a, static_cast<T*>(a.dv), b, s.k0, a.v_token, a.v_batch) + j * a.v_token + (int64_t)hk * 2 * a.dim + col;
    Ops<T>::store4(dv, t.x, t.y, t.z, t.w);
  } else {
    T* dk = rows_of(a, static_cast<T*>(a.dk), b, s.k0, a.k_token, a.k_batch) + j * a.k_token + (int64_t)hk * 2 * a.dim + col - 2 * a.dim;
    Ops<T>::store4(dk, a.scale * t.x, a.scale * t.y, a.scale * t.z, a.scale * t.w);
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------------------
static int elem_of(const cd_diff_attn* d) { return d->dtype == CD_BF16 ? 2 : 4; }
static int64_t rows_q(const cd_diff_attn* d) { return d->q_starts ? d->q_rows : (int64_t)d->batch * d->tq; }
static int64_t rows_k(const cd_diff_attn* d) { return d->k_starts ? d->k_rows : (int64_t)d->batch * d->tk; }
// whether lambda (or its gradient) has an element
static bool has_lambda(const cd_diff_attn* d) { return d->lambda_kind == CD_LAMBDA_HEAD || rows_q(d) > 0; }

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
  CD_REQUIRE(!d->q_starts || ((d->tq >= 1 || d->q_rows == 0) && (d->tk >= 1 || d->k_rows == 0)), "%s: packed rows and no longest sequence (tq=%d tk=%d)", what, d->tq,
             d->tk);
  CD_REQUIRE(d->heads <= 65536, "%s: heads=%d above 65536", what, d->heads);   // (the row values of a tile, 31 rows of all heads apart, are addressed with 32 bits)
  const int64_t group = d->heads / d->kv_heads;
  CD_REQUIRE(group <= 1024 && d->tq * group <= (1 << 30) / group, "%s: tq=%d with %lld heads a key head is too long", what, d->tq, (long long)group);
  CD_REQUIRE((int64_t)d->batch * d->kv_heads * (cdiv(d->tq * group, F_ROWS) + cdiv(d->tk, 64) + 1) < (1 << 30) && (int64_t)d->batch * d->tq <= INT32_MAX,
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
    if (tokens[t] * elem_of(d) > 1 << 27)   // (32 rows of a tile are addressed with 32 bits)
      return set_error(CD_ERR_UNSUPPORTED, "%s: token stride %lld is above 2^27 bytes", what, (long long)tokens[t]);
    CD_REQUIRE(batches[t] >= 0 && batches[t] % ve == 0, "%s: batch stride %lld of %s", what, (long long)batches[t], t == 0 ? "q" : t == 1 ? "k" : t == 2 ? "v" : "out");
  }
  return CD_OK;
}

// Sequences that lie apart: one behind the other, or all of a token's sequences inside its stride (time-major).
static int check_apart(const char* what, const cd_diff_attn* d, bool out_only) {
  if (d->q_starts || d->batch == 1) return CD_OK;
  const int64_t batches[4] = {d->o_batch, d->q_batch, d->k_batch, d->v_batch}, tokens[4] = {d->o_token, d->q_token, d->k_token, d->v_token};
  for (int t = 0; t < (out_only ? 1 : 4); t++) {
    const int64_t rows = t < 2 ? d->tq : d->tk, width = 2LL * d->head_dim * (t < 2 ? d->heads : d->kv_heads);
    const bool apart = batches[t] >= width && (batches[t] - width >= (rows - 1) * tokens[t] || (tokens[t] - width) / (d->batch - 1) >= batches[t]);
    CD_REQUIRE(apart || rows == 0, "%s: the sequences that are written share memory (batch stride %lld, token stride %lld)", what, (long long)batches[t],
               (long long)tokens[t]);
  }
  return CD_OK;
}

// Parts of the keys that get a workgroup of their own: few rows against many keys would leave most of the chip without work.  Heads of 64, one part against
// this rule: one query of 16 sequences and 4 key heads on up to 8192 keys 187 against 41 + 6 us (the join); 16 queries of 8 heads on 4096 keys 88
// against 16; 4096 causal tokens of 4 heads 104 against 77; where there are rows enough (512 causal tokens of 8 heads) the rule leaves one part: 19.
// All three rules at once in fp32, heads of 64, forward and backward: 1024 causal tokens of 8 heads 415 against 231, of 2 heads 412 against 167; 16 queries of 8 heads
// on 4096 keys 987 against 111; 300 causal tokens of 8 heads on one key head 444 against 151; 3 x 77 on 130 keys, where they leave one part, 47.  Single queries of 4
// sequences on 4096 keys 412 against 25.  A loss: 4 x 512 causal queries on 600 keys, 8 heads of 64 in bf16, 81 against 97 (two parts in every pass).
static int parts_of(const cd_diff_attn* d) {
  const int64_t groups = (int64_t)d->batch * d->kv_heads * cdiv((int64_t)d->tq * (d->heads / d->kv_heads), F_ROWS);
  int64_t p = groups ? 768 / groups : 1;   // (three workgroups a compute unit: all parts at once)
  // (a single tile of rows is split down to 128 keys; where the rows fill more, what the parts write and read again is worth it from 512 keys on)
  const int64_t least = (int64_t)d->tq * (d->heads / d->kv_heads) > F_ROWS ? 512 : 128;
  if (p > cdiv(d->tk, least)) p = cdiv(d->tk, least);
  if (p > 64) p = 64;
  return p < 2 ? 1 : (int)p;
}

static DiffArgs args_of(const cd_diff_attn* d) {
  DiffArgs a = {};
  a.q_token = d->q_token; a.q_batch = d->q_batch; a.k_token = d->k_token; a.k_batch = d->k_batch;
  a.v_token = d->v_token; a.v_batch = d->v_batch; a.o_token = d->o_token; a.o_batch = d->o_batch; a.o2_token = 2LL * d->heads * d->head_dim;
  a.q_lens = d->q_lens; a.k_lens = d->k_lens; a.q_starts = d->q_starts; a.k_starts = d->k_starts;
  a.q_rows = rows_q(d); a.k_rows = rows_k(d);
  a.batch = d->batch; a.tq = d->tq; a.tk = d->tk; a.heads = d->heads; a.kv_heads = d->kv_heads; a.group = d->heads / d->kv_heads; a.dim = d->head_dim;
  a.causal = d->causal != 0; a.lam_token = d->lambda_kind == CD_LAMBDA_TOKEN; a.parts = 1;
  a.units = d->batch * d->kv_heads;
  a.uneven = d->q_lens || d->k_lens;
  a.by_heads = fast_div(a.kv_heads); a.by_dim = fast_div(a.dim); a.by_quads = fast_div(a.dim / 2);
  a.group_inv = a.group > 1 ? (uint32_t)((1ull << 32) / a.group) + 1 : 0;
  a.scale = d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->head_dim);
  a.c = a.scale * 1.44269504088896340736f;
  return a;
}

// f<T, DT>() of this dtype and head_dim
// f(instance) for the dtype and the head dimension of a descriptor: instance holds T and DT
template <typename T_, int DT_> struct Instance { typedef T_ T; static constexpr int DT = DT_; };
template <typename F> static void dispatch(const cd_diff_attn* d, F f) {
  if (d->dtype == CD_BF16) {
    if (d->head_dim <= 32) f(Instance<bf16_t, 32>()); else if (d->head_dim <= 64) f(Instance<bf16_t, 64>()); else f(Instance<bf16_t, 128>());
  } else {
    if (d->head_dim <= 32) f(Instance<float, 32>()); else if (d->head_dim <= 64) f(Instance<float, 64>()); else f(Instance<float, 128>());
  }
}
static int64_t keys_of(const cd_diff_attn* d) {
  int64_t n = 0;
  dispatch(d, [&](auto x) { n = KvSizes<typename decltype(x)::T, decltype(x)::DT>::KEYS; });
  return n;
}
// Parts of the rows that get a workgroup of their own in the pass that owns keys: few keys under many rows (shared key heads) leave compute units without
// work.  Five sequences of up to 777 tokens, 8 heads of 128 on 2: one part 144 us, this rule 63 and a join of 8; both passes of 4 x 1024 causal tokens, 8
// heads of 64 on 2: 203 against 102.
static int kv_parts_of(const cd_diff_attn* d) {
  const int64_t groups = (int64_t)d->batch * d->kv_heads * cdiv(d->tk, keys_of(d)), tiles = cdiv((int64_t)d->tq * (d->heads / d->kv_heads), 32);
  int64_t p = groups && groups < 256 ? 512 / groups : 1;
  if (p > tiles / 8) p = tiles / 8;
  if (p > 16) p = 16;
  return p < 2 ? 1 : (int)p;
}

// The same of the keys in the pass that owns queries: a few queries against many keys (both passes of 16 queries, 8 heads of 64 on 4096 keys: one part 146 us,
// this rule 37).
static int q_parts_of(const cd_diff_attn* d) {
  int64_t rows = 0;
  dispatch(d, [&](auto x) { rows = QSizes<typename decltype(x)::T, decltype(x)::DT>::ROWS; });
  const int64_t groups = (int64_t)d->batch * d->kv_heads * cdiv((int64_t)d->tq * (d->heads / d->kv_heads), rows);
  int64_t p = groups && groups < 256 ? 512 / groups : 1;
  if (p > d->tk / 256) p = d->tk / 256;
  if (p > 64) p = 64;
  return p < 2 ? 1 : (int)p;
}

// Workspace of the backward pass: what the pass over the queries leaves of every row, delta_2 once more where it is summed, and the parts' sums.
struct Layout { size_t second, sums, bytes; };
static Layout layout_of(const cd_diff_attn* d) {
  const size_t rows = (size_t)d->heads * rows_q(d), parts = (size_t)kv_parts_of(d);
  Layout l;
  l.second = rows * sizeof(RowValues);
  l.sums = l.second + (d->lambda_kind == CD_LAMBDA_HEAD ? align_up(rows * 4, 16) : 0);
  const size_t keys = parts > 1 ? parts * d->batch * d->kv_heads * d->tk * 4 * d->head_dim * 4 : 0, q_parts = (size_t)q_parts_of(d);
  const size_t queries = q_parts > 1 ? q_parts * d->batch * d->tq * d->heads * (2 * d->head_dim + 2) * 4 : 0;
  l.bytes = l.sums + (keys > queries ? keys : queries);   // (the one pass has joined its parts before the other writes its own)
  return l;
}

static double pairs(const cd_diff_attn* d) { return (double)d->batch * d->heads * d->tq * d->tk * (d->causal ? 0.5 : 1.0); }

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_diff_attention_workspace_bytes(const cd_diff_attn* desc, int backward, size_t* bytes) {
  if (const int rc = check("diff_attention_workspace_bytes", desc)) return rc;
  CD_REQUIRE(bytes != nullptr, "diff_attention_workspace_bytes: output pointer is NULL");
  const int parts = parts_of(desc);
  size_t n = parts > 1 ? (size_t)parts * desc->batch * desc->kv_heads * desc->tq * (desc->heads / desc->kv_heads) * 2 * (2 * desc->head_dim + 4) * 4 : 0;
  if (backward) {
    const size_t back = layout_of(desc).bytes;
    n = n > back ? n : back;
  }
  *bytes = align_up(n, 16);
  return CD_OK;
}

extern "C" int codistill_diff_attention(const cd_diff_attn* desc, const void* q, const void* k, const void* v, const float* lambda, void* out,
                                        void* o_second, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check("diff_attention", desc)) return rc;
  CD_REQUIRE(((q && out) || rows_q(desc) == 0) && ((k && v) || rows_k(desc) == 0) && (lambda || !has_lambda(desc)), "diff_attention: NULL pointer argument");
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
  a.part = a.part_ml + (size_t)a.parts * a.units * a.tq * a.group * 8;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double e = elem_of(desc), qe = 2.0 * a.q_rows * a.heads * 2 * a.dim, ke = 2.0 * a.k_rows * a.kv_heads * 2 * a.dim;
  ProfScope prof(CD_K_ATTN, s, 12.0 * a.dim * pairs(desc), e * (qe + ke));
  const unsigned blocks = work_blocks(a);
  dispatch(desc, [&](auto x) {
    hipLaunchKernelGGL((diff_forward_kernel<typename decltype(x)::T, decltype(x)::DT>), dim3(blocks), dim3(F_THREADS), 0, s, a);
  });
  if (a.parts > 1) {
    const dim3 grid((unsigned)cdiv((int64_t)a.tq * a.group, 4), (unsigned)a.units);   // (units of few workgroups: parts_of)
    if (desc->dtype == CD_BF16) hipLaunchKernelGGL((diff_join_kernel<bf16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((diff_join_kernel<float>), grid, dim3(256), 0, s, a);
  }
  return check_launch("diff_attention");
}

extern "C" int codistill_diff_attention_backward(const cd_diff_attn* desc, const void* q, const void* k, const void* v, const float* lambda, const void* out,
                                                 const void* o_second, const float* lse, const void* dout, void* dq, void* dk, void* dv, float* dlambda,
                                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check("diff_attention_backward", desc)) return rc;
  CD_REQUIRE(((q && out && o_second && lse && dout && dq) || rows_q(desc) == 0) && ((k && v && dk && dv) || rows_k(desc) == 0) &&
                 ((lambda && dlambda) || !has_lambda(desc)),
             "diff_attention_backward: NULL pointer argument");
  CD_REQUIRE(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out) && aligned16(o_second) && aligned16(lse) && aligned16(dout) && aligned16(dq) &&
                 aligned16(dk) && aligned16(dv) && aligned16(workspace) && ((reinterpret_cast<uintptr_t>(lambda) | reinterpret_cast<uintptr_t>(dlambda)) & 3) == 0,
             "diff_attention_backward: pointers must be 16-byte aligned, lambda and dlambda 4-byte aligned");
  if (const int rc = check_apart("diff_attention_backward", desc, false)) return rc;
  if (desc->scale > 0.f && desc->scale < LEAST_SCALE) return set_error(CD_ERR_UNSUPPORTED, "diff_attention_backward: scale %g is below 2^-100", desc->scale);
  size_t need = 0;
  codistill_diff_attention_workspace_bytes(desc, 1, &need);
  CD_REQUIRE(workspace || need == 0, "diff_attention_backward: NULL pointer argument");
  if (workspace_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "diff_attention_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  DiffArgs a = args_of(desc);
  a.q = q; a.k = k; a.v = v; a.lam = lambda; a.out = const_cast<void*>(out); a.o2 = const_cast<void*>(o_second); a.lse = const_cast<float*>(lse);
  a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv; a.dlam = dlambda;
  const Layout lay = layout_of(desc);
  a.rows = static_cast<RowValues*>(workspace);
  a.second = reinterpret_cast<float*>(static_cast<char*>(workspace) + lay.second);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double e = elem_of(desc), qe = 4.0 * a.q_rows * a.heads * 2 * a.dim, ke = 4.0 * a.k_rows * a.kv_heads * 2 * a.dim;
  ProfScope prof(CD_K_ATTN, s, 20.0 * a.dim * pairs(desc), e * (qe + ke));
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + lay.sums);
  if (a.tq > 0) {
    a.parts = q_parts_of(desc);
    a.part_ml = a.part + (size_t)a.parts * a.units * a.tq * a.group * 2 * a.dim;
    dispatch(desc, [&](auto x) {
      a.tiles = (int)cdiv((int64_t)a.tq * a.group, QSizes<typename decltype(x)::T, decltype(x)::DT>::ROWS);
      const unsigned blocks = work_blocks(a);
      hipLaunchKernelGGL((diff_backward_q_kernel<typename decltype(x)::T, decltype(x)::DT>), dim3(blocks), dim3(256), 0, s, a);
    });
    if (a.parts > 1) {
      const dim3 grid((unsigned)cdiv((int64_t)a.tq * a.group * (a.dim / 2), 256), (unsigned)a.units);
      if (desc->dtype == CD_BF16) hipLaunchKernelGGL((diff_join_q_kernel<bf16_t>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((diff_join_q_kernel<float>), grid, dim3(256), 0, s, a);
    }
  }
  a.parts = kv_parts_of(desc);
  const int heads = a.lam_token ? 0 : a.heads;   // workgroups that add up a head's dlambda
  if (a.tk > 0 || heads)
    dispatch(desc, [&](auto x) {
      typedef KvSizes<typename decltype(x)::T, decltype(x)::DT> Z;
      a.tiles = (int)cdiv(a.tk, Z::KEYS);
      a.work = (int)work_blocks(a, true);
      hipLaunchKernelGGL((diff_backward_kv_kernel<typename decltype(x)::T, decltype(x)::DT>), dim3((unsigned)(a.work + heads)), dim3(Z::THREADS), 0, s, a);
    });
  if (a.tk > 0) {
    if (a.parts > 1) {
      const dim3 grid((unsigned)cdiv((int64_t)a.tk * a.dim, 256), (unsigned)a.units);
      if (desc->dtype == CD_BF16) hipLaunchKernelGGL((diff_join_kv_kernel<bf16_t>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((diff_join_kv_kernel<float>), grid, dim3(256), 0, s, a);
    }
  }
  return check_launch("diff_attention_backward");
}
