// A cache of keys and values in 8 bits for differential attention: written as codes, read back, and attended from.
//
// Codes.  The two keys and the value of a token and key head each have a scale, the smallest bf16 number s >= max|x| / 127 (and >= 2^-100), and codes
// rint(x / s) in -127 .. 127.  A code times its scale is what the cache holds.  (An 8-bit float is off by 2^-4 of every element, a code by 2^-8 of the largest: for
// elements of a normal distribution four times less.)
//
// Layout.  Keys [page][key head][token][2][dim padded to 32], values [page][key head][2 dim][token], scales bf16 [page][key head][3][token].  64 tokens of a
// key head, whatever the page, are what a wave takes at a time, and both products read them from memory straight into the registers of the matrix
// instructions: of the keys a lane takes a run of one token's channels, of the values 16 tokens of one channel, which is why values are
// stored with the tokens side by side.  No copy in LDS, no exchange between lanes.
//
// Writing and reading move bytes: 14510 tokens of 24 packed prompts, 4 key heads of 64 in bf16 (45 MB each way, 9.4 us at the copy rate), 16.0 and 13.1 us (prompts that the caches hold 15.0 and 12.7;
// without the arithmetic of the codes 2 less); a workgroup's rows are all asked for at once, so that the chip loads, computes and stores in turns.  14496 tokens in fp32 (75 MB each way, 15.6): 15.7 and 19.6, from the caches in
// part.  One token of each of 16 sequences: 4.8 and 2.9, a launch and its latencies.
#include "common.h"
#include "conv_rules.h"
#include "kernels.h"
#include "vec.h"
#include <math.h>

namespace cd {
namespace {

constexpr int KV_TILE = 64;           // tokens that are worked on together: pages are whole tiles
constexpr float KV_LEAST = 0x1p-100f;
constexpr int KV_WAVES = 4;           // waves of a workgroup of the attention
constexpr int KV_CUS = 256;
constexpr int KV_MOST_PARTS = 512;
constexpr float LOG2E = 1.4426950408889634f;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct KvArgs {
  int8_t* k; int8_t* v; uint16_t* scales;
  const int32_t* table;
  int64_t pages;
  int32_t sequences, kv_heads, dim, padded, page_tokens, seq_pages;
  FastDiv by_page, by_heads;   // by page_tokens, kv_heads
};
// n / d for n below 2^31
__device__ inline int quotient(int n, FastDiv d) { return (int)div_by((unsigned)n, d); }

// The page of a sequence's tokens from `pos` on, and the place in it; or -1 where the sequence has none (the table may hold anything).
__device__ inline int64_t page_of(const KvArgs& c, int b, int64_t pos, int* slot) {
  *slot = 0;
  if (pos < 0 || pos > INT32_MAX) return -1;
  const int p = quotient((int)pos, c.by_page);
  if (p >= c.seq_pages) return -1;
  *slot = (int)pos - p * c.page_tokens;
  const int64_t at = (int64_t)b * c.seq_pages + p, page = c.table ? c.table[at] : at;
  return page >= 0 && page < c.pages ? page : -1;
}

// ---- codes --------------------------------------------------------------------------------------------------------------
// magnitudes as integers: larger numbers are larger, infinities and NaN largest
__device__ inline uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
// the largest of `lanes` neighbours (a power of two up to 32), each of which receives it: exchanges inside rows of 16 lanes, which need no LDS
__device__ inline uint32_t lanes_max(uint32_t v, int lanes) {
  auto with = [&](uint32_t u) { v = v > u ? v : u; };
  if (lanes > 1) with(__builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true));    // lane ^ 1
  if (lanes > 2) with(__builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true));    // lane ^ 2
  if (lanes > 4) with(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true));   // the other four of eight
  if (lanes > 8) with(__builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, true));   // the other eight of sixteen
  if (lanes > 16) with(__shfl_xor(v, 16, 64));
  return v;
}
// the smallest bf16 number that is at least top / 127 (127 times a bf16 number is exact in fp32); NaN where an element is not finite.  The product with
// 1 / 127, cut to bf16, is at most two below.
__device__ inline uint16_t scale_of(uint32_t top) {
  const float t = __builtin_bit_cast(float, top);
  uint32_t s = __builtin_bit_cast(uint32_t, fmaxf(t * (1.f / 127.f), KV_LEAST)) >> 16;
  s += 127.f * bf16_to_f32((bf16_t)s) < t;
  s += 127.f * bf16_to_f32((bf16_t)s) < t;
  return top >= 0x7f800000u ? 0x7fc0 : (uint16_t)s;
}
// rint(x / s) in the lowest byte, exactly.  t is the quotient rounded once (a product and a correction by what it leaves, which fp32 holds exactly), and a quotient that
// is not halfway between two codes does not round to there: s has 8 bits, so it lies at least half a step of fp32 and 2^-32 of itself away.  Adding 1.5 2^23 rounds
// to nearest even.
__device__ inline uint32_t code_of(float x, float s, float inverse) {
  float t = x * inverse;
  t = fmaf(fmaf(-t, s, x), inverse, t);
  return __builtin_bit_cast(uint32_t, t + 0x1.8p23f);
}
__device__ inline uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {   // the lowest bytes of four
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// eight codes and their scale: `lanes` neighbours share it
__device__ inline uint2 quantise(const float (&x)[8], int lanes, uint16_t* scale) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; e++) top = max(top, magnitude(x[e]));
  top = lanes_max(top, lanes);
  *scale = scale_of(top);
  if (top >= 0x7f800000u) return make_uint2(0, 0);
  const float s = bf16_to_f32(*scale), inverse = __builtin_amdgcn_rcpf(s);   // (off by 2^-23: the correction's error is 2^-45)
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; e++) w[e] = code_of(x[e], s, inverse);
  return make_uint2(bytes_of(w[0], w[1], w[2], w[3]), bytes_of(w[4], w[5], w[6], w[7]));
}
// four words of four bytes, rows for columns
__device__ inline void transpose4(uint32_t (&w)[4]) {
  const uint32_t lo01 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t lo23 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
}
template <typename T> __device__ inline void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    T t[8];
    load_run<T, 8>(p, t);
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = Cvt<T>::ld(t[e]);
  } else {
    float lo[4], hi[4];
    load_run<float, 4>(p, lo);
    load_run<float, 4>(p + 4, hi);
#pragma unroll
    for (int e = 0; e < 4; e++) { x[e] = lo[e]; x[4 + e] = hi[e]; }
  }
}
template <typename T> __device__ inline void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    store_run<T, 8>(p, x);
  } else {
    float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    store_run<float, 4>(p, lo);
    store_run<float, 4>(p + 4, hi);
  }
}

struct KvRowArgs {
  KvArgs c;
  const void* k_in; const void* v_in; void* k_out; void* v_out;
  const int32_t* first; const int32_t* counts; const int32_t* starts;
  int64_t rows, k_token, k_batch, v_token, v_batch;
  int32_t max_new, tiles, k_lanes, v_lanes;   // lanes of a key, of a value (powers of two)
  uint32_t all;                               // tiles of all sequences and key heads, below 2^31
  FastDiv by_tiles;
};

// What a workgroup of the writing or reading kernel works on: the tokens of one sequence that lie in one tile of the cache.
struct KvTile {
  int b, h, lo, hi;        // sequence, key head, slots lo .. hi - 1 of the tile
  int64_t row0;            // row of the tile's first slot, which may lie in front of the first row
  int64_t i0;              // the same counted in the sequence
  int64_t page;
  int slot0;               // the tile's place in its page
};
__device__ inline KvTile tile_of(const KvRowArgs& a) {
  KvTile t;
  const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;   // (a launch holds fewer than 2^32 threads along x)
  if (id >= a.all) {
    t.lo = t.hi = 0;
    return t;
  }
  const int unit = quotient((int)id, a.by_tiles), n_tile = (int)id - unit * a.tiles;
  t.b = quotient(unit, a.c.by_heads);
  t.h = unit - t.b * a.c.kv_heads;
  const int64_t first = a.first ? a.first[t.b] : 0;
  int64_t from = 0, n = a.max_new;
  if (a.starts) {      // rows of the tensors only, whatever the table says
    from = a.starts[t.b];
    const int64_t end = a.starts[t.b + 1];
    n = end - from;
    if (from < 0 || end > a.rows) n = 0;
  } else if (a.counts) {
    n = a.counts[t.b];
  }
  n = n < 0 ? 0 : n < a.max_new ? n : a.max_new;
  const int64_t base = ((first >> 6) + n_tile) * KV_TILE;   // position of the tile's first slot
  t.i0 = base - first;
  t.row0 = from + t.i0;
  const int64_t lo = -t.i0, hi = n - t.i0;
  t.lo = (int)(lo > 0 ? lo : 0);
  t.hi = (int)(hi < KV_TILE ? hi : KV_TILE);
  t.page = page_of(a.c, t.b, base, &t.slot0);
  return t;
}

// Two waves of a workgroup take the keys, two the values (as much work), 8 channels a lane.  Values go through LDS as they are quantised, token by token, and
// leave it channel by channel, 8 tokens of 4 channels a thread; rows of 4 bytes more than the channels keep both sides off each other's banks.
constexpr int KV_AHEAD = 4;   // tokens of a lane whose loads are in flight together (2, 4, 8: 16.6, 15.0 and 15.2 us for the prompts below)
constexpr int V_PAD = 4, V_WORDS = (256 + V_PAD) / 4;   // words of a token's row, widest heads

template <typename T>
__global__ void __launch_bounds__(256) kv_write_kernel(KvRowArgs a) {
  __shared__ uint32_t tile[KV_TILE * V_WORDS];
  const KvTile t = tile_of(a);
  if (t.lo >= t.hi || t.page < 0) return;
  const KvArgs& c = a.c;
  const int64_t head = t.page * c.kv_heads + t.h;
  uint16_t* const scales = c.scales + head * 3 * c.page_tokens + t.slot0;
  const int lane = threadIdx.x & 127, words = (2 * c.dim + V_PAD) / 4;
  if (threadIdx.x < 128) {
    const int sub = lane % a.k_lanes, per_wg = 128 / a.k_lanes, ch = sub * 8, all = 2 * (t.hi - t.lo);
    const T* const in = static_cast<const T*>(a.k_in) + (a.starts ? 0 : t.b * a.k_batch) + (int64_t)2 * t.h * c.dim + ch;
    const int64_t row = a.starts ? t.row0 : t.i0;
    for (int g0 = lane / a.k_lanes; g0 < all; g0 += KV_AHEAD * per_wg) {
      float x[KV_AHEAD][8];
#pragma unroll
      for (int u = 0; u < KV_AHEAD; u++) {
        const int g = g0 + u * per_wg;
#pragma unroll
        for (int e = 0; e < 8; e++) x[u][e] = 0.f;
        if (ch < c.dim && g < all) load8<T>(in + (row + t.lo + (g >> 1)) * a.k_token + (g & 1) * c.dim, x[u]);
      }
#pragma unroll
      for (int u = 0; u < KV_AHEAD; u++) {
        const int g = g0 + u * per_wg, slot = t.lo + (g >> 1), m = g & 1;
        if (g >= all) break;   // (for all lanes that share a scale)
        uint16_t s;
        const uint2 w = quantise(x[u], a.k_lanes, &s);
        if (sub == 0) scales[(int64_t)m * c.page_tokens + slot] = s;
        if (ch < c.dim) *reinterpret_cast<uint2*>(c.k + ((head * c.page_tokens + t.slot0 + slot) * 2 + m) * c.padded + ch) = w;
      }
    }
  } else {
    const int sub = lane % a.v_lanes, per_wg = 128 / a.v_lanes, ch = sub * 8, all = t.hi - t.lo;
    const T* const in = static_cast<const T*>(a.v_in) + (a.starts ? 0 : t.b * a.v_batch) + (int64_t)2 * t.h * c.dim + ch;
    const int64_t row = a.starts ? t.row0 : t.i0;
    for (int g0 = lane / a.v_lanes; g0 < all; g0 += KV_AHEAD * per_wg) {
      float x[KV_AHEAD][8];
#pragma unroll
      for (int u = 0; u < KV_AHEAD; u++) {
        const int g = g0 + u * per_wg;
#pragma unroll
        for (int e = 0; e < 8; e++) x[u][e] = 0.f;
        if (ch < 2 * c.dim && g < all) load8<T>(in + (row + t.lo + g) * a.v_token, x[u]);
      }
#pragma unroll
      for (int u = 0; u < KV_AHEAD; u++) {
        const int g = g0 + u * per_wg, slot = t.lo + g;
        if (g >= all) break;   // (for all lanes that share a scale)
        uint16_t s;
        const uint2 w = quantise(x[u], a.v_lanes, &s);
        if (sub == 0) scales[(int64_t)2 * c.page_tokens + slot] = s;
        if (ch < 2 * c.dim) {
          tile[slot * words + ch / 4] = w.x;
          tile[slot * words + ch / 4 + 1] = w.y;
        }
      }
    }
  }
  __syncthreads();
  int8_t* const v = c.v + head * 2 * c.dim * c.page_tokens + t.slot0;
  const int o0 = t.lo >> 3, octets = ((t.hi + 7) >> 3) - o0;   // (rows in front of and behind the tokens hold anything: they are not written)
  for (int i = threadIdx.x; i < c.dim / 2 * octets; i += 256) {
    const int q = i / octets, s0 = 8 * (o0 + i - q * octets);
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      lo[e] = tile[(s0 + e) * words + q];
      hi[e] = tile[(s0 + 4 + e) * words + q];
    }
    transpose4(lo);
    transpose4(hi);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      int8_t* const to = v + (int64_t)(4 * q + e) * c.page_tokens + s0;
      if (s0 >= t.lo && s0 + 8 <= t.hi) {
        *reinterpret_cast<uint2*>(to) = make_uint2(lo[e], hi[e]);
      } else {
        for (int j = 0; j < 8; j++)
          if (s0 + j >= t.lo && s0 + j < t.hi) to[j] = (int8_t)((j < 4 ? lo[e] : hi[e]) >> 8 * (j & 3));
      }
    }
  }
}

template <typename T> __device__ inline void store_values(T* to, uint2 w, float s) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> 8 * (e & 3)) * s;
  store8<T>(to, x);
}
template <typename T>
__global__ void __launch_bounds__(256) kv_read_kernel(KvRowArgs a) {
  __shared__ uint32_t tile[KV_TILE * V_WORDS];
  const KvTile t = tile_of(a);
  if (t.lo >= t.hi) return;
  const KvArgs& c = a.c;
  const bool there = t.page >= 0;
  const int64_t head = there ? t.page * c.kv_heads + t.h : 0;
  const uint16_t* const scales = c.scales + head * 3 * c.page_tokens + t.slot0;
  const int words = (2 * c.dim + V_PAD) / 4;
  if (there) {
    const int8_t* const v = c.v + head * 2 * c.dim * c.page_tokens + t.slot0;
    const int o0 = t.lo >> 3, octets = ((t.hi + 7) >> 3) - o0;
    for (int i = threadIdx.x; i < c.dim / 2 * octets; i += 256) {
      const int q = i / octets, s0 = 8 * (o0 + i - q * octets);
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const uint2 w = *reinterpret_cast<const uint2*>(v + (int64_t)(4 * q + e) * c.page_tokens + s0);
        lo[e] = w.x;
        hi[e] = w.y;
      }
      transpose4(lo);
      transpose4(hi);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        tile[(s0 + e) * words + q] = lo[e];
        tile[(s0 + 4 + e) * words + q] = hi[e];
      }
    }
  }
  {
    const int sub = threadIdx.x % a.k_lanes, per_wg = 256 / a.k_lanes, ch = sub * 8;
    for (int g = threadIdx.x / a.k_lanes; g < 2 * (t.hi - t.lo); g += per_wg) {
      const int slot = t.lo + (g >> 1), m = g & 1;
      if (ch >= c.dim) continue;
      const int64_t to = a.starts ? (t.row0 + slot) * a.k_token : t.b * a.k_batch + (t.i0 + slot) * a.k_token;
      uint2 w = make_uint2(0, 0);
      if (there) w = *reinterpret_cast<const uint2*>(c.k + ((head * c.page_tokens + t.slot0 + slot) * 2 + m) * c.padded + ch);
      store_values<T>(static_cast<T*>(a.k_out) + to + (int64_t)(2 * t.h + m) * c.dim + ch, w, there ? bf16_to_f32(scales[(int64_t)m * c.page_tokens + slot]) : 0.f);
    }
  }
  __syncthreads();
  {
    const int sub = threadIdx.x % a.v_lanes, per_wg = 256 / a.v_lanes, ch = sub * 8;
    for (int g = threadIdx.x / a.v_lanes; g < t.hi - t.lo; g += per_wg) {
      const int slot = t.lo + g;
      if (ch >= 2 * c.dim) continue;
      const int64_t to = a.starts ? (t.row0 + slot) * a.v_token : t.b * a.v_batch + (t.i0 + slot) * a.v_token;
      const uint2 w = there ? make_uint2(tile[slot * words + ch / 4], tile[slot * words + ch / 4 + 1]) : make_uint2(0, 0);
      store_values<T>(static_cast<T*>(a.v_out) + to + (int64_t)t.h * 2 * c.dim + ch, w, there ? bf16_to_f32(scales[(int64_t)2 * c.page_tokens + slot]) : 0.f);
    }
  }
}

// ---- attention -----------------------------------------------------------------------------------------------------------
//
//     P_m = softmax over the visible keys of scale q_m . k_m  (m = 1, 2),   out = (P_1 - lambda P_2) v
//
// Memory-bound where few queries share a key head: a key and its value, 4 dim + 6 bytes, are read once for a tile of 8 rows (two tiles where `row_tiles` says so).  Every further tile is a
// workgroup that reads and converts them again, through the caches: 16 sequences of 8092 tokens, 4 key heads of 64, take 30.5 us for 4 rows a key head and 73 for 32 (fp32, tiles of
// 8: 31.2 and 101); 4 of 3996, 2 key heads of 128, 36.7 for 64 rows, where the bytes alone are 3.5.
//
// Rows.  Row r of a sequence is query r / group of head r % group.  A 16x16x32 product has 16 columns: 8 rows, each once for either map.  Both keys of a token are
// multiplied with all columns and a column keeps its own map's score; from there on a map is a row like any other, with its own running maximum, and both maps
// are weights of one read of the values.
//
// Tiles.  64 keys are four products, and row 4 g + i of product t is key 16 g + 4 t + i, so that lane l (g = l / 16), which holds the scores of
// column l % 16 for those rows, has the keys 16 g .. 16 g + 15: their values of one channel are the 16 bytes that it loads, and its weights
// are the second product's operand as they lie.
//
// Roundings.  Codes are exact in bf16.  fp32 queries, and the weights times the values' scales, are sums of three bf16 numbers (all 24 bits), bf16 models'
// weights of two (16 bits): results are then off by their own rounding alone, 1.7e-3 as a 2-norm, and the second product costs 5 to 9 %.
//
// 16 sequences of 2000 to 8000 tokens, one query each, 16 heads of 64 on 4 (80 MB): 22.3 us (3.6 TB/s; 17 are the copy rate), and 4.1 for the join; the same on bf16 keys and
// values takes 41 and 6.  One of 124000 on 2 key heads (47 MB): 15.2 and 5.1.  Five of up to 4096, four queries, heads of 128: 14.9 and 4.6, of which the bytes are 2.5: a launch, the chain
// from the lengths to the first keys, and one or two blocks a wave, one wave a SIMD.
struct KvAttnArgs {
  KvArgs c;
  const void* q; const float* lam; void* out;
  const int32_t* q_lens; const int32_t* k_lens;
  float* part; float* part_ml;            // sums of a part [unit][row][part][2][2 dim], maxima and sums [unit][row][part][2][2]
  int64_t q_token, q_batch, o_token, o_batch;
  int32_t tq, heads, group, rows, causal, lam_token, parts, tiles;
  FastDiv by_tiles, by_parts, by_group, by_quads;   // by tiles, parts, group, dim / 2
  float factor;                           // scale log2(e)
};

template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int Q = 1, P = 2; };
template <> struct Terms<float> { static constexpr int Q = 3, P = 3; };

__device__ inline v8bf codes_as_bf16(uint2 w) {
  v8bf f;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const uint32_t word = e < 2 ? w.x : w.y;
    const int shift = 16 * (e & 1);
    const v2f two = {(float)(int8_t)(word >> shift), (float)(int8_t)(word >> (shift + 8))};
    const v2bf r = __builtin_convertvector(two, v2bf);
    f[2 * e] = r[0];
    f[2 * e + 1] = r[1];
  }
  return f;
}
// x as a sum of N bf16 numbers
template <int N> __device__ inline void split8(const float (&x)[8], v8bf (&out)[N]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; e++) rest[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const v2f two = {rest[e], rest[e + 1]};
      const v2bf r = __builtin_convertvector(two, v2bf);
      out[n][e] = r[0];
      out[n][e + 1] = r[1];
      if (n + 1 < N) {
        rest[e] -= (float)r[0];
        rest[e + 1] -= (float)r[1];
      }
    }
}

struct KvRow { int query, head; bool real; };

// NK: 32-channel steps of a map's key; RT: tiles of 8 rows
template <typename T, int NK, int RT>
__global__ void __launch_bounds__(64 * KV_WAVES, NK <= 2 && RT == 1 ? 2 : 1) kv_attention_kernel(KvAttnArgs a) {
  constexpr int NC = 4 * NK, TQ = Terms<T>::Q, TP = Terms<T>::P, COLS = 16 * RT;
  __shared__ float sums[KV_WAVES][COLS][64 * NK + 4];
  __shared__ float tops[KV_WAVES][COLS], totals[KV_WAVES][COLS];
  const KvArgs& c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4, map = col >> 3;
  int id = blockIdx.x, next = quotient(id, a.by_tiles);
  const int tile = id - next * a.tiles;
  id = next;
  next = quotient(id, a.by_parts);
  const int part = id - next * a.parts, b = quotient(next, c.by_heads), h = next - b * c.kv_heads;
  const int nk = min(max(a.k_lens[b], 0), c.seq_pages * c.page_tokens), nq = a.q_lens ? min(max(a.q_lens[b], 0), a.tq) : a.tq;
  auto seen_by = [&](int query) { return a.causal ? max(0, min(nk, query - nq + nk + 1)) : nk; };
  auto row_of = [&](int r) {
    KvRow w;
    w.query = quotient(r, a.by_group);
    w.head = h * a.group + r - w.query * a.group;
    w.real = r < a.rows && w.query < nq;
    return w;
  };
  // all real rows of the tile see at least `least` keys, none more than `most`; the others are computed like the last one and not written
  const int row0 = tile * 8 * RT, first_query = quotient(row0, a.by_group), last_query = min(quotient(row0 + 8 * RT - 1, a.by_group), nq - 1);
  const int least = first_query < nq ? seen_by(first_query) : 0, most = first_query < nq ? seen_by(last_query) : 0;
  int sees[RT];
  v8bf q[RT][NK][TQ];      // the lane's row and map
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const KvRow w = row_of(row0 + 8 * rt + (col & 7));
    sees[rt] = w.real ? seen_by(w.query) : most;
    const T* from = static_cast<const T*>(a.q) + b * a.q_batch + w.query * a.q_token + (int64_t)(2 * w.head + map) * c.dim;
#pragma unroll
    for (int s = 0; s < NK; s++) {
      const int ch = grp * 8 * NK + 8 * s;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] = 0.f;
      if (w.real && ch < c.dim) load8<T>(from + ch, x);
      split8<TQ>(x, q[rt][s]);
    }
  }
  const int blocks = (most + KV_TILE - 1) / KV_TILE, whole = least / KV_TILE;   // whole: blocks that all rows see to their ends
  // a run of blocks for each part, the first `more` of them one longer
  const int each = quotient(blocks, a.by_parts), more = blocks - each * a.parts;
  const int from = part * each + min(part, more), to = from + each + (part < more);

  v4f acc[RT][NC];
  float top[RT], total[RT];
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    top[rt] = -INFINITY;
    total[rt] = 0.f;
#pragma unroll
    for (int n = 0; n < NC; n++) acc[rt][n] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  uint2 kc[4][2][NK];
  uint4 vc[NC];
  uint4 ks[2], vs[2];     // bf16 scales of the lane's 16 keys: its own map's, the values'
  const int last_ch = 2 * c.dim - 16;
  auto load_keys = [&](int64_t page, int slot) {
    const int64_t head = page * c.kv_heads + h;
    const int8_t* const base = c.k + (head * c.page_tokens + slot) * 2 * c.padded;
    const uint16_t* const sc = c.scales + head * 3 * c.page_tokens + slot;
#pragma unroll
    for (int t = 0; t < 4; t++)
#pragma unroll
      for (int m = 0; m < 2; m++) {
        const int8_t* const p = base + ((16 * (col >> 2) + 4 * t + (col & 3)) * 2 + m) * (32 * NK) + grp * 8 * NK;
        if constexpr (NK % 2 == 0) {
#pragma unroll
          for (int s = 0; s < NK; s += 2) {
            const uint4 w = *reinterpret_cast<const uint4*>(p + 8 * s);
            kc[t][m][s] = make_uint2(w.x, w.y);
            kc[t][m][s + 1] = make_uint2(w.z, w.w);
          }
        } else {
#pragma unroll
          for (int s = 0; s < NK; s++) kc[t][m][s] = *reinterpret_cast<const uint2*>(p + 8 * s);
        }
      }
#pragma unroll
    for (int u = 0; u < 2; u++) {
      ks[u] = *reinterpret_cast<const uint4*>(sc + map * c.page_tokens + 16 * grp + 8 * u);
      vs[u] = *reinterpret_cast<const uint4*>(sc + 2 * c.page_tokens + 16 * grp + 8 * u);
    }
  };
  auto scale_at = [&](const uint4 (&w)[2], int i) {
    const uint32_t word = (&w[i >> 3].x)[(i & 7) >> 1];
    return __builtin_bit_cast(float, i & 1 ? word & 0xffff0000u : word << 16);
  };
  int blk = from + wave, slot = 0;
  int64_t page = -1;
  // the next block of this wave that has a page
  auto seek = [&]() {
    for (; blk < to; blk += KV_WAVES) {
      page = page_of(c, b, (int64_t)blk * KV_TILE, &slot);
      if (page >= 0) return;
    }
  };
  seek();
  if (blk < to) load_keys(page, slot);
  while (blk < to) {
    {
      const int8_t* const base = c.v + (page * c.kv_heads + h) * 2 * c.dim * c.page_tokens + slot;
#pragma unroll
      for (int n = 0; n < NC; n++)   // (channels behind the last one: the last ones again, which nobody reads)
        vc[n] = *reinterpret_cast<const uint4*>(base + (int64_t)(min(16 * n, last_ch) + col) * c.page_tokens + 16 * grp);
    }
    v4f sc[RT][4];
#pragma unroll
    for (int t = 0; t < 4; t++) {
      v4f both[RT][2];
#pragma unroll
      for (int m = 0; m < 2; m++) {
#pragma unroll
        for (int rt = 0; rt < RT; rt++) both[rt][m] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NK; s++) {
          const v8bf key = codes_as_bf16(kc[t][m][s]);
#pragma unroll
          for (int rt = 0; rt < RT; rt++)
#pragma unroll
            for (int n = TQ - 1; n >= 0; n--) both[rt][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[rt][s][n], both[rt][m], 0, 0, 0);
        }
      }
#pragma unroll
      for (int rt = 0; rt < RT; rt++)
#pragma unroll
        for (int i = 0; i < 4; i++) sc[rt][t][i] = map ? both[rt][1][i] : both[rt][0][i];
    }
    float kf[16], vf[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
      kf[i] = scale_at(ks, i) * a.factor;
      vf[i] = scale_at(vs, i);
    }
    const int now = blk;
    blk += KV_WAVES;
    seek();
    if (blk < to) load_keys(page, slot);
    v8bf w[RT][2][TP];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      float p[16], high = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; i++) p[i] = sc[rt][i >> 2][i & 3] * kf[i];
      const int left = sees[rt] - now * KV_TILE - 16 * grp;   // visible ones of the lane's 16 keys
      if (now >= whole) {
#pragma unroll
        for (int i = 0; i < 16; i++) p[i] = i < left ? p[i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 16; i++) high = fmaxf(high, p[i]);
      high = fmaxf(high, __shfl_xor(high, 16, 64));
      high = fmaxf(high, __shfl_xor(high, 32, 64));
      high = fmaxf(high, top[rt]);
      const float at = high == -INFINITY ? 0.f : high;
      if (__any(high > top[rt])) {
        const float f = __builtin_amdgcn_exp2f(top[rt] - at);
        total[rt] *= f;
#pragma unroll
        for (int n = 0; n < NC; n++) acc[rt][n] *= f;
        top[rt] = high;
      }
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; i++) {
        p[i] = __builtin_amdgcn_exp2f(p[i] - at);
        sum += p[i];
      }
      total[rt] += sum;
      if (now >= whole) {   // (the scale of a key that the row does not see may be anything: it is not multiplied by a weight of zero)
#pragma unroll
        for (int i = 0; i < 16; i++) p[i] = i < left ? p[i] * vf[i] : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < 16; i++) p[i] *= vf[i];
      }
      split8<TP>(*reinterpret_cast<float(*)[8]>(p), w[rt][0]);
      split8<TP>(*reinterpret_cast<float(*)[8]>(p + 8), w[rt][1]);
    }
#pragma unroll
    for (int n = 0; n < NC; n++) {
      const v8bf lo = codes_as_bf16(make_uint2(vc[n].x, vc[n].y)), hi = codes_as_bf16(make_uint2(vc[n].z, vc[n].w));
#pragma unroll
      for (int rt = 0; rt < RT; rt++)
#pragma unroll
        for (int e = TP - 1; e >= 0; e--) {
          acc[rt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, w[rt][0][e], acc[rt][n], 0, 0, 0);
          acc[rt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, w[rt][1][e], acc[rt][n], 0, 0, 0);
        }
    }
  }

  // the waves' sums, brought to the largest maximum
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    total[rt] += __shfl_xor(total[rt], 16, 64);
    total[rt] += __shfl_xor(total[rt], 32, 64);
    if (grp == 0) tops[wave][16 * rt + col] = top[rt];
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    float high = tops[0][16 * rt + col];
#pragma unroll
    for (int w = 1; w < KV_WAVES; w++) high = fmaxf(high, tops[w][16 * rt + col]);
    const float f = top[rt] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[rt] - high);   // (a wave without keys has zeros)
    if (grp == 0) totals[wave][16 * rt + col] = total[rt] * f;
#pragma unroll
    for (int n = 0; n < NC; n++)
      *reinterpret_cast<float4*>(&sums[wave][16 * rt + col][16 * n + 4 * grp]) = make_float4(acc[rt][n][0] * f, acc[rt][n][1] * f, acc[rt][n][2] * f, acc[rt][n][3] * f);
  }
  __syncthreads();
  const int width = 2 * c.dim, quads = width / 4;
  for (int i = threadIdx.x; i < 8 * RT * quads; i += 64 * KV_WAVES) {
    const int r = quotient(i, a.by_quads), ch = 4 * (i - r * quads), at = 16 * (r >> 3) + (r & 7);
    if (row0 + r >= a.rows) break;
    float o[2][4], t[2];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      t[k] = ((totals[0][at + 8 * k] + totals[1][at + 8 * k]) + totals[2][at + 8 * k]) + totals[3][at + 8 * k];
#pragma unroll
      for (int w = 0; w < KV_WAVES; w++) {
        const float4 v = *reinterpret_cast<const float4*>(&sums[w][at + 8 * k][ch]);
        const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; e++) o[k][e] = w ? o[k][e] + x[e] : x[e];
      }
    }
    if (a.parts > 1) {
      const int64_t to_part = (((int64_t)b * c.kv_heads + h) * a.rows + row0 + r) * a.parts + part;
#pragma unroll
      for (int k = 0; k < 2; k++) {
        *reinterpret_cast<float4*>(a.part + (to_part * 2 + k) * width + ch) = make_float4(o[k][0], o[k][1], o[k][2], o[k][3]);
        if (ch == 0) {
          const int to = at + 8 * k;
          a.part_ml[(to_part * 2 + k) * 2] = fmaxf(fmaxf(tops[0][to], tops[1][to]), fmaxf(tops[2][to], tops[3][to]));
          a.part_ml[(to_part * 2 + k) * 2 + 1] = t[k];
        }
      }
    } else {
      const KvRow w = row_of(row0 + r);
      const float lam = a.lam[a.lam_token ? ((int64_t)b * a.tq + w.query) * a.heads + w.head : w.head];
      const bool seen = w.real && seen_by(w.query) > 0;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] = seen ? (t[0] == 0.f ? 0.f : o[0][e] / t[0]) - (t[1] == 0.f ? 0.f : lam * (o[1][e] / t[1])) : 0.f;
      store_run<T, 4>(static_cast<T*>(a.out) + b * a.o_batch + w.query * a.o_token + (int64_t)w.head * width + ch, v);
    }
  }
}

// The parts of a row: a workgroup takes 32 channels, 8 of its threads every eighth part of one.
template <typename T>
__global__ void __launch_bounds__(256) kv_join_kernel(KvAttnArgs a) {
  __shared__ float factor[2][KV_MOST_PARTS], red[8][2][32], most[4][2], totals[4][2];
  const KvArgs& c = a.c;
  const int width = 2 * c.dim, chunks = (width + 31) / 32, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x / chunks;
  const int ch = (int)(blockIdx.x % chunks) * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
  const int unit = (int)(row / a.rows), r = (int)(row % a.rows), b = unit / c.kv_heads, h = unit % c.kv_heads;
  const float* const sums = a.part + row * a.parts * 2 * width + min(ch, width - 1);
  const float4* const ml = reinterpret_cast<const float4*>(a.part_ml) + row * a.parts;   // maximum and sum of the first map, of the second
  constexpr int EACH = KV_MOST_PARTS / 256;
  float4 mine[EACH];
  float high[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    const int p = threadIdx.x + 256 * e;
    mine[e] = p < a.parts ? ml[p] : make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
    high[0] = fmaxf(high[0], mine[e].x);
    high[1] = fmaxf(high[1], mine[e].z);
  }
#pragma unroll
  for (int k = 0; k < 2; k++) {
    high[k] = wave_max(high[k]);
    if ((threadIdx.x & 63) == 0) most[wave][k] = high[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; k++) high[k] = fmaxf(fmaxf(most[0][k], most[1][k]), fmaxf(most[2][k], most[3][k]));
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    const int p = threadIdx.x + 256 * e;
    if (p < a.parts) {   // (a part without keys has zeros)
      factor[0][p] = mine[e].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mine[e].x - high[0]);
      factor[1][p] = mine[e].z == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mine[e].z - high[1]);
      total[0] += mine[e].y * factor[0][p];
      total[1] += mine[e].w * factor[1][p];
    }
  }
#pragma unroll
  for (int k = 0; k < 2; k++) {
    total[k] = wave_sum(total[k]);
    if ((threadIdx.x & 63) == 0) totals[wave][k] = total[k];
  }
  __syncthreads();
  float sum[2] = {0.f, 0.f};
#pragma unroll 8
  for (int p = run; p < a.parts; p += 8) {
    sum[0] += sums[(int64_t)p * 2 * width] * factor[0][p];
    sum[1] += sums[((int64_t)p * 2 + 1) * width] * factor[1][p];
  }
  red[run][0][threadIdx.x & 31] = sum[0];
  red[run][1][threadIdx.x & 31] = sum[1];
  __syncthreads();
  if (threadIdx.x >= 32 || ch >= width) return;
#pragma unroll
  for (int k = 0; k < 2; k++) {
    total[k] = ((totals[0][k] + totals[1][k]) + totals[2][k]) + totals[3][k];
    sum[k] = 0.f;
#pragma unroll
    for (int q = 0; q < 8; q++) sum[k] += red[q][k][threadIdx.x];
  }
  const int query = r / a.group, head = h * a.group + r % a.group;
  const float lam = a.lam[a.lam_token ? ((int64_t)b * a.tq + query) * a.heads + head : head];
  const float v = (total[0] == 0.f ? 0.f : sum[0] / total[0]) - (total[1] == 0.f ? 0.f : lam * (sum[1] / total[1]));
  const int nq = a.q_lens ? min(max(a.q_lens[b], 0), a.tq) : a.tq;
  static_cast<T*>(a.out)[b * a.o_batch + query * a.o_token + (int64_t)head * width + ch] = Cvt<T>::st(query < nq ? v : 0.f);
}

// ---- host -------------------------------------------------------------------------------------------------------------------
static int elem_of(const cd_kv_cache* c) { return c->dtype == CD_BF16 ? 2 : 4; }
constexpr int64_t KV_FAR = 1ll << 31;   // largest stride of a token (of a sequence: 128 times that), so that no offset passes 63 bits
static int padded_dim(int dim) { return (dim + 31) / 32 * 32; }

static int check_cache(const char* what, const cd_kv_cache* c, bool pointers) {
  CD_REQUIRE(c != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE(c->dtype == CD_F32 || c->dtype == CD_BF16, "%s: unknown dtype %d", what, c->dtype);
  CD_REQUIRE(c->kv_heads >= 1 && c->kv_heads <= 65536, "%s: kv_heads=%d out of range", what, c->kv_heads);
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return set_error(CD_ERR_UNSUPPORTED, "%s: head_dim=%d is no multiple of 8 up to 128", what, c->head_dim);
  CD_REQUIRE(c->page_tokens >= KV_TILE && c->page_tokens % KV_TILE == 0 && c->page_tokens <= (1 << 21), "%s: page_tokens=%d is no multiple of 64 up to 2^21", what, c->page_tokens);
  CD_REQUIRE(c->sequences >= 1 && c->seq_pages >= 1 && c->pages >= 1 && c->pages <= INT32_MAX, "%s: sequences=%d, seq_pages=%d, pages=%lld must be positive", what,
             c->sequences, c->seq_pages, (long long)c->pages);
  CD_REQUIRE((int64_t)c->seq_pages * c->page_tokens <= INT32_MAX - KV_TILE, "%s: a sequence of %lld tokens", what, (long long)c->seq_pages * c->page_tokens);
  CD_REQUIRE((int64_t)c->sequences * c->kv_heads <= (1 << 24), "%s: %d sequences of %d key heads", what, c->sequences, c->kv_heads);
  if (!pointers) return CD_OK;
  CD_REQUIRE(c->k && c->v && c->scales, "%s: NULL pointer in the cache", what);
  CD_REQUIRE(aligned16(c->k) && aligned16(c->v) && aligned16(c->scales) && (reinterpret_cast<uintptr_t>(c->table) & 3) == 0,
             "%s: the cache's buffers must be 16-byte aligned, its table 4-byte aligned", what);
  CD_REQUIRE(c->table || c->pages >= (int64_t)c->sequences * c->seq_pages, "%s: %lld pages without a table for %d sequences of %d", what, (long long)c->pages, c->sequences,
             c->seq_pages);
  return CD_OK;
}
static KvArgs cache_args(const cd_kv_cache* c) {
  return {c->k, c->v, c->scales, c->table, c->pages, c->sequences, c->kv_heads, c->head_dim, padded_dim(c->head_dim), c->page_tokens, c->seq_pages,
          fast_div(c->page_tokens), fast_div(c->kv_heads)};
}
static int lanes_for(int runs) {
  int lanes = 1;
  while (lanes < runs) lanes *= 2;
  return lanes;
}

static int check_rows(const char* what, const cd_kv_cache* c, const cd_kv_rows* r, const void* k, const void* v, bool written) {
  if (const int rc = check_cache(what, c, true)) return rc;
  CD_REQUIRE(r != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE(r->max_new >= 0, "%s: max_new=%d must not be negative", what, r->max_new);
  CD_REQUIRE(!(r->starts && r->counts), "%s: starts together with counts", what);
  CD_REQUIRE(!r->starts || (r->rows >= 0 && r->rows <= INT32_MAX), "%s: rows=%lld out of range", what, (long long)r->rows);
  CD_REQUIRE(!r->starts || r->rows == 0 || r->max_new > 0, "%s: packed sequences without their longest one", what);
  CD_REQUIRE(((reinterpret_cast<uintptr_t>(r->first) | reinterpret_cast<uintptr_t>(r->counts) | reinterpret_cast<uintptr_t>(r->starts)) & 3) == 0, "%s: misaligned table", what);
  if (r->max_new == 0) return CD_OK;
  CD_REQUIRE((k && v) || (r->starts && r->rows == 0), "%s: NULL pointer argument", what);
  CD_REQUIRE(r->k_token <= KV_FAR && r->v_token <= KV_FAR && r->k_batch <= 128 * KV_FAR && r->v_batch <= 128 * KV_FAR, "%s: strides out of range", what);
  const int vec = 16 / elem_of(c);
  const int64_t least = (int64_t)c->kv_heads * 2 * c->head_dim;
  CD_REQUIRE(aligned16(k) && aligned16(v), "%s: pointers must be 16-byte aligned", what);
  const bool several = r->starts ? r->rows > 1 : r->max_new > 1, sequences = !r->starts && c->sequences > 1;
  CD_REQUIRE(!several || (r->k_token >= least && r->v_token >= least && r->k_token % vec == 0 && r->v_token % vec == 0),
             "%s: token strides must be multiples of 16 bytes and hold a token", what);
  CD_REQUIRE(!sequences || (r->k_batch % vec == 0 && r->v_batch % vec == 0 && r->k_batch >= 0 && r->v_batch >= 0), "%s: batch strides must be multiples of 16 bytes", what);
  // rows that are written lie apart: sequences one behind the other, or all of a token's inside its stride
  auto apart = [&](int64_t token, int64_t batch) {
    return (batch >= least && batch >= (int64_t)(r->max_new - 1) * token + least) ||
           (batch >= least && (r->max_new == 1 || token >= (int64_t)(c->sequences - 1) * batch + least));
  };
  CD_REQUIRE(!written || !sequences || (apart(r->k_token, r->k_batch) && apart(r->v_token, r->v_batch)), "%s: sequences of the rows share memory", what);
  CD_REQUIRE((int64_t)c->sequences * c->kv_heads * ((r->max_new + 126ll) / KV_TILE) <= INT32_MAX, "%s: too many tiles", what);
  return CD_OK;
}
static dim3 row_grid(const KvRowArgs& a) {
  const unsigned across = a.all < (1u << 22) ? a.all : 1u << 22;
  return dim3(across, (unsigned)cdiv((int64_t)a.all, (int64_t)across));
}
static KvRowArgs row_args(const cd_kv_cache* c, const cd_kv_rows* r) {
  KvRowArgs a = {};
  a.c = cache_args(c);
  a.first = r->first; a.counts = r->counts; a.starts = r->starts; a.rows = r->rows;
  a.k_token = r->k_token; a.k_batch = r->k_batch; a.v_token = r->v_token; a.v_batch = r->v_batch;
  a.max_new = r->max_new;
  a.tiles = (int32_t)((r->max_new + 126ll) / KV_TILE);   // (the first token may be the last of its tile)
  a.all = (uint32_t)((int64_t)a.tiles * c->sequences * c->kv_heads);
  a.by_tiles = fast_div(a.tiles);
  a.k_lanes = lanes_for(c->head_dim / 8);
  a.v_lanes = lanes_for(c->head_dim / 4);
  return a;
}

static int check_attention(const char* what, const cd_kv_cache* c, const cd_kv_attn* d) {
  if (const int rc = check_cache(what, c, false)) return rc;
  CD_REQUIRE(d != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE(d->tq >= 0 && d->heads >= 1 && d->heads <= 65536 && d->heads % c->kv_heads == 0, "%s: tq=%d, heads=%d for %d key heads", what, d->tq, d->heads, c->kv_heads);
  CD_REQUIRE(d->lambda_kind == CD_LAMBDA_HEAD || d->lambda_kind == CD_LAMBDA_TOKEN, "%s: unknown lambda kind %d", what, d->lambda_kind);
  CD_REQUIRE(d->scale >= 0.f && d->scale < __builtin_inff(), "%s: scale must be finite and not negative", what);
  CD_REQUIRE(d->q_token <= KV_FAR && d->o_token <= KV_FAR && d->q_batch <= 128 * KV_FAR && d->o_batch <= 128 * KV_FAR, "%s: strides out of range", what);
  const int vec = 16 / elem_of(c);
  const int64_t least = (int64_t)d->heads * 2 * c->head_dim;
  CD_REQUIRE(d->tq <= 1 || (d->q_token >= least && d->o_token >= least && d->q_token % vec == 0 && d->o_token % vec == 0),
             "%s: token strides must be multiples of 16 bytes and hold a token", what);
  CD_REQUIRE(c->sequences == 1 || (d->q_batch >= 0 && d->q_batch % vec == 0 && d->o_batch % vec == 0), "%s: batch strides must be multiples of 16 bytes", what);
  CD_REQUIRE(c->sequences == 1 || d->tq == 0 ||
                 (d->o_batch >= least && (d->o_batch >= (int64_t)(d->tq - 1) * d->o_token + least || d->tq == 1 || d->o_token >= (int64_t)(c->sequences - 1) * d->o_batch + least)),
             "%s: sequences of out share memory", what);
  CD_REQUIRE((int64_t)d->tq * (d->heads / c->kv_heads) * c->sequences * c->kv_heads < (1 << 24), "%s: %d queries of %d heads in %d sequences", what, d->tq, d->heads, c->sequences);
  CD_REQUIRE((reinterpret_cast<uintptr_t>(d->q_lens) & 3) == 0 && (reinterpret_cast<uintptr_t>(d->k_lens) & 3) == 0, "%s: misaligned table", what);
  return CD_OK;
}
static int rows_of(const cd_kv_cache* c, const cd_kv_attn* d) { return d->tq * (d->heads / c->kv_heads); }
// Two tiles of rows share what is read, where there are registers for their sums (fp32 queries take three times a tile's registers) and enough blocks to read
// (of at most so many tokens: the lengths are on the device).  Two tiles and one, us: 16 queries of a key head on 16 x 4 caches of 8192 tokens, heads of 64, 39.9 and
// 46.7; on 2 caches of 131072 34.0 and 45.2; but on 16 of 8192 16.7 and 16.4, on 4 of 600 12.3 and 9.6.
constexpr int KV_SHARED_BLOCKS = 2560;
static int row_tiles(const cd_kv_cache* c, const cd_kv_attn* d) {
  const int64_t blocks = (int64_t)c->sequences * c->kv_heads * ((int64_t)c->seq_pages * c->page_tokens / KV_TILE);
  return rows_of(c, d) > 8 && c->dtype == CD_BF16 && c->head_dim <= 64 && blocks >= KV_SHARED_BLOCKS ? 2 : 1;
}
// Workgroups of a sequence and key head: as many as run at once (two a compute unit, wide heads and double tiles one), each with at least a block for every wave.
// Half as many, as many and twice as many, with the join, us: 16 x 4 caches of up to 8192 tokens, heads of 64, 28.9, 26.4 and 27.9; 2 of 131072 18.3, 19.8 and 24.4; 10 of up to
// 4096, heads of 128, 22.4, 20.1 and 23.0.
static int parts_of(const cd_kv_cache* c, const cd_kv_attn* d) {
  const int64_t groups = (int64_t)c->sequences * c->kv_heads * cdiv(rows_of(c, d), 8 * row_tiles(c, d));
  const int64_t blocks = (int64_t)c->seq_pages * c->page_tokens / KV_TILE, most = blocks / KV_WAVES < KV_MOST_PARTS ? blocks / KV_WAVES : KV_MOST_PARTS;
  const int64_t want = KV_CUS * (c->head_dim <= 64 && row_tiles(c, d) == 1 ? 2 : 1) / (groups > 0 ? groups : 1);
  const int64_t parts = want < most ? want : most;
  return parts < 1 ? 1 : (int)parts;
}

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_kv_cache_bytes(const cd_kv_cache* cache, size_t* k_bytes, size_t* v_bytes, size_t* scale_bytes) {
  if (const int rc = check_cache("kv_cache_bytes", cache, false)) return rc;
  CD_REQUIRE(k_bytes && v_bytes && scale_bytes, "kv_cache_bytes: output pointer is NULL");
  const size_t tokens = (size_t)cache->pages * cache->kv_heads * cache->page_tokens;
  *k_bytes = tokens * 2 * padded_dim(cache->head_dim);
  *v_bytes = tokens * 2 * cache->head_dim;
  *scale_bytes = tokens * 3 * 2;
  return CD_OK;
}

extern "C" int codistill_kv_write(const cd_kv_cache* cache, const cd_kv_rows* rows, const void* k, const void* v, void* stream) {
  if (const int rc = check_rows("kv_write", cache, rows, k, v, false)) return rc;
  if (rows->max_new == 0 || (rows->starts && rows->rows == 0)) return CD_OK;
  KvRowArgs a = row_args(cache, rows);
  a.k_in = k; a.v_in = v;
  const double n = (rows->starts ? (double)rows->rows : (double)cache->sequences * rows->max_new) * cache->kv_heads * 4 * cache->head_dim;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_GLUE, s, 6 * n, n * (elem_of(cache) + 1));
  const dim3 grid = row_grid(a);
  if (cache->dtype == CD_BF16) hipLaunchKernelGGL((kv_write_kernel<bf16_t>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_write_kernel<float>), grid, dim3(256), 0, s, a);
  return check_launch("kv_write");
}

extern "C" int codistill_kv_read(const cd_kv_cache* cache, const cd_kv_rows* rows, void* k, void* v, void* stream) {
  if (const int rc = check_rows("kv_read", cache, rows, k, v, true)) return rc;
  if (rows->max_new == 0 || (rows->starts && rows->rows == 0)) return CD_OK;
  KvRowArgs a = row_args(cache, rows);
  a.k_out = k; a.v_out = v;
  const double n = (rows->starts ? (double)rows->rows : (double)cache->sequences * rows->max_new) * cache->kv_heads * 4 * cache->head_dim;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_GLUE, s, n, n * (elem_of(cache) + 1));
  const dim3 grid = row_grid(a);
  if (cache->dtype == CD_BF16) hipLaunchKernelGGL((kv_read_kernel<bf16_t>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_read_kernel<float>), grid, dim3(256), 0, s, a);
  return check_launch("kv_read");
}

extern "C" int codistill_kv_diff_attention_workspace_bytes(const cd_kv_cache* cache, const cd_kv_attn* desc, size_t* bytes) {
  if (const int rc = check_attention("kv_diff_attention_workspace_bytes", cache, desc)) return rc;
  CD_REQUIRE(bytes != nullptr, "kv_diff_attention_workspace_bytes: output pointer is NULL");
  const int parts = parts_of(cache, desc);
  *bytes = parts > 1 ? align_up((size_t)parts * cache->sequences * cache->kv_heads * rows_of(cache, desc) * (4 * cache->head_dim + 4) * 4, 16) : 0;
  return CD_OK;
}

extern "C" int codistill_kv_diff_attention(const cd_kv_cache* cache, const cd_kv_attn* desc, const void* q, const float* lambda, void* out, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  if (const int rc = check_attention("kv_diff_attention", cache, desc)) return rc;
  if (const int rc = check_cache("kv_diff_attention", cache, true)) return rc;
  CD_REQUIRE(desc->k_lens && ((q && out) || desc->tq == 0) && lambda, "kv_diff_attention: NULL pointer argument");
  CD_REQUIRE(aligned16(q) && aligned16(out) && aligned16(workspace) && (reinterpret_cast<uintptr_t>(lambda) & 3) == 0,
             "kv_diff_attention: pointers must be 16-byte aligned, lambda 4-byte aligned");
  size_t need = 0;
  codistill_kv_diff_attention_workspace_bytes(cache, desc, &need);
  if (workspace_bytes < need || (need && !workspace))
    return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "kv_diff_attention: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (desc->tq == 0) return CD_OK;
  KvAttnArgs a = {};
  a.c = cache_args(cache);
  a.q = q; a.lam = lambda; a.out = out; a.q_lens = desc->q_lens; a.k_lens = desc->k_lens;
  a.q_token = desc->q_token; a.q_batch = desc->q_batch; a.o_token = desc->o_token; a.o_batch = desc->o_batch;
  a.tq = desc->tq; a.heads = desc->heads; a.group = desc->heads / cache->kv_heads; a.rows = rows_of(cache, desc);
  a.causal = desc->causal != 0; a.lam_token = desc->lambda_kind == CD_LAMBDA_TOKEN;
  a.parts = parts_of(cache, desc);
  const int rt = row_tiles(cache, desc);
  a.tiles = (int)cdiv(a.rows, 8 * rt);
  a.by_tiles = fast_div(a.tiles); a.by_parts = fast_div(a.parts); a.by_group = fast_div(a.group); a.by_quads = fast_div(cache->head_dim / 2);
  a.factor = (desc->scale > 0.f ? desc->scale : 1.f / sqrtf((float)cache->head_dim)) * LOG2E;
  a.part_ml = static_cast<float*>(workspace);
  a.part = a.part_ml + (size_t)a.parts * cache->sequences * cache->kv_heads * a.rows * 4;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double keys = (double)cache->sequences * cache->seq_pages * cache->page_tokens;   // (at most: the lengths are on the device)
  ProfScope prof(CD_K_ATTN, s, 12.0 * cache->head_dim * desc->heads * desc->tq * keys, keys * cache->kv_heads * (4 * cache->head_dim + 6));
  const dim3 grid((unsigned)(a.tiles * a.parts * cache->sequences * cache->kv_heads));
  auto with = [&](auto type) {
    typedef decltype(type) T;
    auto run = [&](auto nk) {
      constexpr int NK = decltype(nk)::value;
      if constexpr (sizeof(T) == 2 && NK <= 2) {
        if (rt == 2) {
          hipLaunchKernelGGL((kv_attention_kernel<T, NK, 2>), grid, dim3(64 * KV_WAVES), 0, s, a);
          return;
        }
      }
      hipLaunchKernelGGL((kv_attention_kernel<T, NK, 1>), grid, dim3(64 * KV_WAVES), 0, s, a);
    };
    switch (a.c.padded / 32) {
      case 1: run(std::integral_constant<int, 1>()); break;
      case 2: run(std::integral_constant<int, 2>()); break;
      case 3: run(std::integral_constant<int, 3>()); break;
      default: run(std::integral_constant<int, 4>());
    }
    if (a.parts > 1) {
      const dim3 joins((unsigned)(cache->sequences * cache->kv_heads * a.rows * cdiv(2 * cache->head_dim, 32)));
      hipLaunchKernelGGL((kv_join_kernel<T>), joins, dim3(256), 0, s, a);
    }
  };
  if (cache->dtype == CD_BF16) with(bf16_t()); else with(float());
  return check_launch("kv_diff_attention");
}
