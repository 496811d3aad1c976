// Embedding lookup with a factor, and the gradient of its table by sorted tokens.
//
//     y[i] = scale table[token[i]],        dtable[w] (+)= scale * sum of dy[i] over the rows i with token[i] == w, in the rows' order
//
// Both move bytes and compute nothing to speak of.  The gradient: the rows are put in the order of their words (stable: rows of a word stay in their
// order), then a workgroup adds up a block of neighbours in that order, whatever their words, so that a word of half the text costs as much as a
// thousand rare ones; sums of a word that goes on in the next block are left as partial rows and added, first to last, by a second launch.  Nothing is
// added into memory by two workgroups: the same inputs give the same bits.  Words that do not occur are zeroed by workgroups beside the
// first launch of the sort.
//
// The order.  Up to 512 rows: in LDS, by every workgroup for itself.  Few rows: a row's place is the number of rows in front of it, counted by comparing it with all of
// them in one launch (8192 rows: 12.1 us, of which the comparisons, two and a half instructions for 64 of them, are 7).  Many rows: a radix sort, two launches for each digit
// of up to 10 bits (65536 rows 4.8 + 9.6 us a digit): digits of a chunk are counted, then every chunk knows where its own begin.
//
// 8192 rows of 512 bf16 channels among 32768 words, beside what the table's gradient holds: lookup 5.1 us, order 12.1, sums 9.6, parts 4.6: latency, 26 MB are 5.  65536 rows of 1024
// among as many words, all written: lookup 45 (169 MB, 3.7 TB/s; 30 where the caches still hold much of the table), order 28.8, sums and zeros 74 (402 MB, 5.4 TB/s), parts 5.5.
// 300 rows of 256 fp32 channels: 2.6 and 10.1.  fp32 rows, three sets in turn, lookup and whole gradient added to another: 8192 rows of 512 from a bf16 table 6.8 and 25.4, from an fp32 one 6.6 and 25.1
// (bf16 rows 5.3 and 24.8); 65536 of 1024 100 and 106, 60 and 106 (bf16 rows 30 and 93).  The 100 are a lane's two stores of 16 bytes, 32 apart, past the caches.
#include "common.h"
#include "vec.h"

namespace cd {
namespace {

constexpr uint32_t NO_WORD = 0x7fffffffu;   // sorted behind all words
// Most rows that a workgroup puts in order for itself, and places it takes of them.  One launch and three, us: 64 rows of 512 bf16 channels 7.2 and 11.9, 300 10.0 and 12.4,
// 512 of 1024 12.0 and 12.1, 500 of two words 13.1 and 12.3.
constexpr int SMALL_ROWS = 512, SMALL_BLOCK = 32;
// Most rows whose places are counted, for each launch of two that the radix sort would take and one more.  Gradients of 64 channels, counted and sorted, us: vocabularies
// below 1024 (one digit) 4096 rows 15.7 and 19.1, 8192 20.7 and 19.7; up to 2^20 (two) 8192 21.6 and 27.7, 10240 27.9 and 29.4, 12288 30.4 and 29.1, 16384 40 and 30.
constexpr int RANK_ROWS = 3840;
constexpr int RANK_EACH = 16, RANK_AHEAD = 8;   // rows of a workgroup there, loads in flight
constexpr int DIGIT_BITS = 10, SORT_CHUNKS = 256, SORT_LEAST = 1024, SORT_WAVES = 8;
constexpr int SUM_WAVES = 8;                // waves of a block of rows
constexpr int FILL_BLOCKS = 1024;
// From here on what is read once (rows of dy) or written and not read again here (rows of y, zeros) bypasses the caches, which the table's rows are left to: 65536 rows of
// 1024 bf16 channels on as many words (134 MB of rows, 268 MB of gradients): lookup 51 -> 30 us where the table is looked up again and again, 50 -> 45 where it comes from memory, sums 93 -> 73.  Rows of 8.4 MB, which the operator in front
// has left in the caches: sums 8.8 -> 9.4.  Between them, rows of 1024 bf16 channels on 32768 words, three sets in turn, through the caches and past them: lookup 16 MiB 7.0 and 6.2 us, 32 MiB 10.9 and 10.0, 64 MiB 21.6 and 17.2, 96 MiB
// 36 and 23 (fp32 rows of 512 from bf16: 7.0 and 5.8, 10.4 and 10.0, 64 MiB 16.9 and 18.8); gradient with its zeros 48.6 and 45.7, 66 and 57, 78 and 64, 87 and 73: what the operator in front has left decides below 64 MiB.  2000 rows on a gradient of
// 16, 64 and 256 MiB: 29.6 and 27.2, 30.9 and 28.7, 58.5 and 55.8.
constexpr int64_t STREAM_BYTES = 64 << 20;

struct EmbedArgs {
  const void* tokens; const void* table; const void* dy; void* y; float* dtable;
  int32_t *order, *words, *order2, *words2, *counts;   // rows and words in sorted order; the same between passes of the radix sort; counts [digits][chunks]
  float* partial;                                      // [blocks][2][width]: sums of a block's first and last words, where others have parts of them
  int64_t rows, vocabulary, width, row_stride, sums;   // sums: workgroups that add up; the others write zeros
  int32_t token_bytes, accumulate, zero_stream, each, blocks, slabs, chunk, chunks, shift, digits, from_tokens;
  int32_t from_end;            // tokens are an index: those below zero count from the vocabulary's end
  float scale, absent;         // absent: elements of a row without a word
};

// (halves of 32 bits: a token whose upper half is not zero, or whose lower half is no word, is none)
__device__ inline uint32_t word_from(const EmbedArgs& a, int64_t token) {
  const uint32_t low = (uint32_t)token < (uint32_t)a.vocabulary ? (uint32_t)token : NO_WORD;
  return (uint32_t)(token >> 32) == 0 ? low : NO_WORD;
}
__device__ inline uint32_t word_from(const EmbedArgs& a, int32_t token) { return (uint32_t)token < (uint32_t)a.vocabulary ? (uint32_t)token : NO_WORD; }
// INDEX: tokens are an index
template <bool INDEX, typename TOK> __device__ inline uint32_t word_from(const EmbedArgs& a, TOK token) {
  return word_from(a, INDEX && token < 0 ? (TOK)(token + (TOK)a.vocabulary) : token);
}
template <bool INDEX, typename TOK> __device__ inline uint32_t word_of(const EmbedArgs& a, int64_t i) { return word_from<INDEX>(a, static_cast<const TOK*>(a.tokens)[i]); }
__device__ inline uint32_t word_of(const EmbedArgs& a, int64_t i) {
  uint32_t w = a.token_bytes == 8 ? word_of<false, int64_t>(a, i) : word_of<false, int32_t>(a, i);
  if (a.from_end && w == NO_WORD) w = a.token_bytes == 8 ? word_of<true, int64_t>(a, i) : word_of<true, int32_t>(a, i);   // (looked at again, so that others do not wait for it)
  return w;
}

// ---- lookup ---------------------------------------------------------------------------------------------------------------
// TT: the table's type, RT: the rows'; V: elements of a run; STREAM: rows bypass the caches
template <typename RT, int V, bool STREAM> __device__ inline void put_run(RT* p, const float (&x)[V]) {
  if constexpr (STREAM) store_run_stream<RT, V>(p, x); else store_run<RT, V>(p, x);
}
template <typename TT, typename RT, int V, bool STREAM>
__global__ void __launch_bounds__(256) embedding_kernel(EmbedArgs a, int lanes) {
  const int64_t per_wg = 256 / lanes;
  for (int64_t i = blockIdx.x * per_wg + threadIdx.x / lanes; i < a.rows; i += gridDim.x * per_wg) {
    const uint32_t w = word_of(a, i);
    const TT* from = static_cast<const TT*>(a.table) + (int64_t)w * a.width;
    RT* to = static_cast<RT*>(a.y) + i * a.row_stride;
    for (int64_t c = (int64_t)(threadIdx.x % lanes) * V; c < a.width; c += (int64_t)lanes * V) {
      float out[V];
      if (w == NO_WORD) {
#pragma unroll
        for (int e = 0; e < V; e++) out[e] = a.absent;
      } else {
        TT t[V];
        load_run<TT, V>(from + c, t);
#pragma unroll
        for (int e = 0; e < V; e++) out[e] = a.scale * Cvt<TT>::ld(t[e]);
      }
      // (runs of 8 floats are two stores)
      if constexpr (sizeof(RT) * V == 32) {
        float lo[4] = {out[0], out[1], out[2], out[3]}, hi[4] = {out[4], out[5], out[6], out[7]};
        put_run<RT, 4, STREAM>(to + c, lo);
        put_run<RT, 4, STREAM>(to + c + 4, hi);
      } else {
        put_run<RT, V, STREAM>(to + c, out);
      }
    }
  }
}

// ---- the order of the rows --------------------------------------------------------------------------------------------------
// 1 where a < b (-1 <= a < 2^31, 0 <= b <= 2^31): the sign of their difference, which is faster than a comparison, whose result travels through a mask
__device__ inline uint32_t below(uint32_t a, uint32_t b) { return (a - b) >> 31; }
// Few rows: place of row i = rows with a smaller word + rows in front of it with the same.  A lane compares its row with each of the workgroup's; the lanes'
// counts are added up at the end.  (Comparisons and the addition of their carries, or counts of their masks in scalar registers: 15 us for 8192 rows.)
// the sum over a wave, in lane 63
__device__ inline int sum_of_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // one, two, four and eight lanes up inside rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // a row's last lane to the next row
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // the first half's last lane to the second half
  return x;
}
template <typename TOK, bool INDEX>
__global__ void __launch_bounds__(256) embedding_rank_kernel(EmbedArgs a) {
  __shared__ uint32_t mine[RANK_EACH];
  __shared__ int found[4][RANK_EACH];
  const int i0 = blockIdx.x * RANK_EACH, rows = (int)a.rows, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (threadIdx.x < RANK_EACH) mine[threadIdx.x] = i0 + (int)threadIdx.x < rows ? word_of<INDEX, TOK>(a, i0 + threadIdx.x) : 0;
  TOK others[RANK_AHEAD];
  auto fetch = [&](int k0) {   // rows k0 .. + 63 and every 256 from there
#pragma unroll
    for (int u = 0; u < RANK_AHEAD; u++)
      if (k0 + 256 * u < rows) others[u] = static_cast<const TOK*>(a.tokens)[min(k0 + 256 * u + lane, rows - 1)];
  };
  fetch(wave * 64);
  __syncthreads();
  uint32_t w[RANK_EACH];
  int count[RANK_EACH];
#pragma unroll
  for (int r = 0; r < RANK_EACH; r++) {
    w[r] = __builtin_amdgcn_readfirstlane(mine[r]);
    count[r] = 0;
  }
  for (int k0 = wave * 64; k0 < rows; k0 += 256 * RANK_AHEAD) {
    uint32_t now[RANK_AHEAD];
#pragma unroll
    for (int u = 0; u < RANK_AHEAD; u++) now[u] = k0 + 256 * u + lane < rows ? word_from<INDEX>(a, others[u]) : NO_WORD;
    if (k0 + 256 * RANK_AHEAD < rows) fetch(k0 + 256 * RANK_AHEAD);
#pragma unroll
    for (int u = 0; u < RANK_AHEAD; u += 2) {
      const int j0 = k0 + 256 * u, j1 = j0 + 256;
      if (j0 >= rows) break;
      const bool among = (j0 < i0 + RANK_EACH && j0 + 64 > i0) || (j1 < i0 + RANK_EACH && j1 + 64 > i0);
      if (!among) {   // all 64 rows in front of the workgroup's rows, or all behind
        const uint32_t x = now[u] - (j0 < i0), y = now[u + 1] - (j1 < i0);
#pragma unroll
        for (int r = 0; r < RANK_EACH; r++) count[r] += below(x, w[r]) + below(y, w[r]);
      } else {
#pragma unroll
        for (int r = 0; r < RANK_EACH; r++) count[r] += below(now[u], w[r] + below(j0 + lane, i0 + r)) + below(now[u + 1], w[r] + below(j1 + lane, i0 + r));
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RANK_EACH; r++) {
    const int all = sum_of_wave(count[r]);
    if (lane == 63) found[wave][r] = all;
  }
  __syncthreads();
  if (threadIdx.x < RANK_EACH && i0 + (int)threadIdx.x < rows) {
    const int r = threadIdx.x, at = found[0][r] + found[1][r] + found[2][r] + found[3][r];
    a.order[at] = i0 + r;
    a.words[at] = (int32_t)mine[r];
  }
}

// Many rows: a pass of the radix sort.  Words that are none sort as the vocabulary's size does: behind all others.
__device__ inline uint32_t sort_key(const EmbedArgs& a, int64_t i) {
  const uint32_t w = a.from_tokens ? word_of(a, i) : (uint32_t)a.words2[i];
  return w == NO_WORD ? (uint32_t)a.vocabulary : w;
}
__global__ void __launch_bounds__(512) embedding_count_kernel(EmbedArgs a) {
  __shared__ int count[1 << DIGIT_BITS];
  for (int d = threadIdx.x; d < a.digits; d += 512) count[d] = 0;
  __syncthreads();
  const int64_t from = (int64_t)blockIdx.x * a.chunk, to = min(from + a.chunk, a.rows);
  for (int64_t i = from + threadIdx.x; i < to; i += 512) atomicAdd(&count[sort_key(a, i) >> a.shift & (a.digits - 1)], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < a.digits; d += 512) a.counts[d * a.chunks + blockIdx.x] = count[d];
}
__global__ void __launch_bounds__(512) embedding_scatter_kernel(EmbedArgs a) {
  __shared__ int at[SORT_WAVES][1 << DIGIT_BITS];
  __shared__ int sums[2][8];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, me = blockIdx.x;
  for (int d = lane; d < a.digits; d += 64) at[wave][d] = 0;
  // a thread's digits (one, and one 512 behind it): rows of them in chunks in front, and in all
  int before[2] = {0, 0}, all[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const int d = threadIdx.x + 512 * k;
    if (d < a.digits) {
#pragma unroll 16
      for (int c = 0; c < a.chunks; c += 4) {   // (rows of whole vectors: what lies behind the chunks is zero)
        const int4 n = *reinterpret_cast<const int4*>(a.counts + d * a.chunks + c);
        before[k] += (c < me ? n.x : 0) + (c + 1 < me ? n.y : 0) + (c + 2 < me ? n.z : 0) + (c + 3 < me ? n.w : 0);
        all[k] += (n.x + n.y) + (n.z + n.w);
      }
    }
  }
  // rows of smaller digits
  int base[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; k++) {
    int sum = all[k];
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int up = __shfl_up(sum, o, 64);
      if (lane >= o) sum += up;
    }
    if (lane == 63) sums[k][wave] = sum;
    base[k] = sum - all[k];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 8; q++) {
    base[0] += q < wave ? sums[0][q] : 0;
    base[1] += sums[0][q] + (q < wave ? sums[1][q] : 0);
  }
  // each wave counts its own run of the chunk
  const int64_t from = (int64_t)me * a.chunk, to = min(from + a.chunk, a.rows);
  const int64_t run = a.chunk / SORT_WAVES, mine = min(from + wave * run, to), end = min(mine + run, to);
  for (int64_t i = mine + lane; i < end; i += 64) atomicAdd(&at[wave][sort_key(a, i) >> a.shift & (a.digits - 1)], 1);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const int d = threadIdx.x + 512 * k;
    if (d < a.digits) {
      int place = base[k] + before[k];
      for (int q = 0; q < SORT_WAVES; q++) {
        const int n = at[q][d];
        at[q][d] = place;
        place += n;
      }
    }
  }
  __syncthreads();
  volatile int* const place = at[wave];
  for (int64_t i0 = mine; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool live = i < end;
    const uint32_t key = live ? sort_key(a, i) : 0;
    const int d = key >> a.shift & (a.digits - 1);
    uint64_t same = __ballot(live);
    for (int b = 1; b < a.digits; b *= 2) {
      const uint64_t set = __ballot((d & b) != 0);
      same &= d & b ? set : ~set;
    }
    if (live) {
      const int rank = __popcll(same & ((1ull << lane) - 1)), to_place = place[d] + rank;
      a.order[to_place] = a.from_tokens ? (int32_t)i : a.order2[i];
      a.words[to_place] = (int32_t)(key == (uint32_t)a.vocabulary ? NO_WORD : key);
      __builtin_amdgcn_wave_barrier();   // every lane has read its digit's place; the last of each digit moves it
      if (same >> lane == 1) place[d] = to_place + 1;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- sums -------------------------------------------------------------------------------------------------------------------
typedef float float4_anywhere_t __attribute__((ext_vector_type(4), aligned(4)));   // (the gradient may begin inside a vector)
template <int V> __device__ inline void load_floats(const float* p, float (&x)[V]) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const float4_anywhere_t t = *reinterpret_cast<const float4_anywhere_t*>(p + e);
      x[e] = t.x; x[e + 1] = t.y; x[e + 2] = t.z; x[e + 3] = t.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; e++) x[e] = p[e];
  }
}
// to = old + scale sum, old being zero or what is there
template <int V> __device__ inline void put_row(float* to, const float (&old)[V], const float (&sum)[V], float scale) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int e = 0; e < V; e += 4)
      *reinterpret_cast<float4_anywhere_t*>(to + e) =
          float4_anywhere_t{old[e] + scale * sum[e], old[e + 1] + scale * sum[e + 1], old[e + 2] + scale * sum[e + 2], old[e + 3] + scale * sum[e + 3]};
  } else {
#pragma unroll
    for (int e = 0; e < V; e++) to[e] = old[e] + scale * sum[e];
  }
}

// The first place in from .. to - 1 of the sorted words that is not below w (or `to`): a wave looks at 64 places at a time.
__device__ inline int64_t lower_bound(const int32_t* words, uint32_t w, int64_t from, int64_t to) {
  const int lane = threadIdx.x & 63;
  while (from < to) {
    const int64_t step = (to - from + 63) / 64, at = from + lane * step;
    const uint64_t below = __ballot(at < to && (uint32_t)words[at] < w);
    const int n = __popcll(below);   // places 0 .. n - 1 are below
    if (n == 0) return from;
    const int64_t next = from + (n - 1) * step + 1;
    to = min(to, from + n * step);
    from = next;
  }
  return from;
}
// Zeros in the rows of words that do not occur: a workgroup takes 512 words at a time.
template <bool SMALL> __device__ inline void zero_absent(const EmbedArgs& a, int me, int all) {
  __shared__ uint8_t there[64 * SUM_WAVES];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool vector = a.width % 4 == 0 && (reinterpret_cast<uintptr_t>(a.dtable) & 15) == 0;
  for (int64_t w0 = (int64_t)me * 64 * SUM_WAVES; w0 < a.vocabulary; w0 += (int64_t)all * 64 * SUM_WAVES) {
    __syncthreads();
    if constexpr (SMALL) {   // (the rows are not in order yet)
      there[threadIdx.x] = 0;
      __syncthreads();
      const int64_t at = (int64_t)threadIdx.x < a.rows ? (int64_t)word_of(a, threadIdx.x) - w0 : -1;
      if (at >= 0 && at < 64 * SUM_WAVES) there[at] = 1;
    } else {
      const int64_t first = lower_bound(a.words, (uint32_t)w0, 0, a.rows), last = lower_bound(a.words, (uint32_t)w0 + 64 * SUM_WAVES, first, a.rows);
      const uint32_t mine = (uint32_t)w0 + threadIdx.x;
      int64_t from = first, to = last;
      while (from < to) {
        const int64_t middle = (from + to) / 2;
        if ((uint32_t)a.words[middle] < mine) from = middle + 1; else to = middle;
      }
      there[threadIdx.x] = from < last && (uint32_t)a.words[from] == mine;
    }
    __syncthreads();
    const int n = (int)min((int64_t)64 * SUM_WAVES, a.vocabulary - w0);
    for (int i = wave; i < n; i += SUM_WAVES) {
      if (there[i]) continue;
      float* const row = a.dtable + (w0 + i) * a.width;
      if (vector && a.zero_stream) {
        for (int64_t col = 4 * lane; col < a.width; col += 256) __builtin_nontemporal_store(run4_t{0, 0, 0, 0}, reinterpret_cast<run4_t*>(row + col));
      } else if (vector) {
        for (int64_t col = 4 * lane; col < a.width; col += 256) *reinterpret_cast<uint4*>(row + col) = make_uint4(0, 0, 0, 0);
      } else {
        for (int64_t col = lane; col < a.width; col += 64) row[col] = 0.f;
      }
    }
  }
}

// A block of SUM_WAVES * each rows in sorted order, 64 V columns.  A wave adds up `each` of them, writes the words that are its alone and leaves its first and
// its last word's sum in LDS; the waves' ends are then put together, column by column, in their order.
// SMALL: up to SMALL_ROWS rows.  Every workgroup puts all of them in order itself, in LDS, and takes the words that begin among its SMALL_BLOCK places, whole:
// nothing is left to join, and the gradient is one launch.
template <typename T, int V, bool SMALL, bool STREAM>
__global__ void __launch_bounds__(64 * SUM_WAVES) embedding_sum_kernel(EmbedArgs a) {
  static_assert(SMALL_ROWS == 64 * SUM_WAVES, "a row for each thread");
  if ((int64_t)blockIdx.x >= a.sums) return zero_absent<SMALL>(a, (int)(blockIdx.x - a.sums), (int)(gridDim.x - a.sums));
  __shared__ float ends[2][SUM_WAVES][64 * V];
  __shared__ uint32_t word[2][SUM_WAVES];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, block = blockIdx.x / a.slabs, slab = blockIdx.x % a.slabs;
  const int64_t col = (int64_t)slab * 64 * V + lane * V;
  const bool mine = col < a.width;     // (a width of whole runs)
  int64_t from = (int64_t)block * SUM_WAVES * a.each + (int64_t)wave * a.each;
  int n = (int)max((int64_t)0, min((int64_t)a.each, a.rows - from));
  // this wave's rows and words: one a lane
  int row_here = 0;
  uint32_t word_here = NO_WORD;
  if constexpr (SMALL) {
    __shared__ __align__(16) uint32_t unsorted[SMALL_ROWS];
    __shared__ uint32_t in_order[2][SMALL_ROWS];
    const uint32_t me = (int64_t)threadIdx.x < a.rows ? word_of(a, threadIdx.x) : NO_WORD;
    unsorted[threadIdx.x] = me;
    __syncthreads();
    // rows in front of the wave's, among them, and behind them (behind the last one: no word, which is below none)
    int place = 0;
    const int from_wave = 64 * wave, rows = (int)a.rows;
    auto count = [&](int j, uint32_t limit) {
      const uint4 other = *reinterpret_cast<const uint4*>(unsorted + j);
      place += below(other.x, limit) + below(other.y, limit);
      place += below(other.z, limit) + below(other.w, limit);
    };
    if (from_wave < rows) {
#pragma unroll 4
      for (int j = 0; j < from_wave; j += 4) count(j, me + 1);
#pragma unroll 4
      for (int j = from_wave; j < from_wave + 64; j++) place += below(unsorted[j], me + below(j, threadIdx.x));
#pragma unroll 4
      for (int j = from_wave + 64; j < rows; j += 4) count(j, me);
    }
    __shared__ int limits[2];    // where the block's words begin and end
    in_order[1][threadIdx.x] = NO_WORD;
    if (threadIdx.x < 2) limits[threadIdx.x] = SMALL_ROWS;
    __syncthreads();
    if ((int64_t)threadIdx.x < a.rows) {
      in_order[0][place] = threadIdx.x;
      in_order[1][place] = me;
    }
    __syncthreads();
    const uint32_t here = in_order[1][threadIdx.x], in_front = threadIdx.x ? in_order[1][threadIdx.x - 1] : 0xffffffffu;
    const bool begins = here != in_front;    // a word, or the rows without one
#pragma unroll
    for (int k = 0; k < 2; k++) {
      const uint64_t set = __ballot(begins && (int)threadIdx.x >= SMALL_BLOCK * (block + k));
      if (set && lane == 0) atomicMin(&limits[k], 64 * wave + __ffsll((unsigned long long)set) - 1);
    }
    __syncthreads();
    const int begin = limits[0], end = limits[1], each = (end - begin + SUM_WAVES - 1) / SUM_WAVES;
    from = begin + wave * each;
    n = max(0, min(each, end - (int)from));
    if (lane < n) {
      row_here = in_order[0][from + lane];
      word_here = in_order[1][from + lane];
    }
  } else if (lane < n) {
    row_here = a.order[from + lane];
    word_here = (uint32_t)a.words[from + lane];
  }
  // Real rows come first.  What the loop needs of a row is one bit (whether its word ends with it, and is not the wave's last) and an offset.
  const int real = __popcll(__ballot(word_here != NO_WORD));
  const uint32_t after = __shfl_down(word_here, 1, 64);
  const uint64_t last_of_word = __ballot(lane + 1 < real && word_here != after);
  const uint32_t first = __builtin_amdgcn_readfirstlane(word_here), final = __builtin_amdgcn_readlane(word_here, max(real - 1, 0));
  const int64_t offset = (int64_t)row_here * a.row_stride;
  const uint32_t offset_low = (uint32_t)offset, offset_high = (uint32_t)(offset >> 32);
  const T* const rows_here = static_cast<const T*>(a.dy) + (mine ? col : 0);   // (lanes behind the width read the first columns, and write nothing)
  float* const table_here = a.dtable + (mine ? col : 0);
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; e++) sum[e] = 0.f;
  bool one = true;     // the wave's first word has not ended
  constexpr int AHEAD = SMALL ? 8 : 4;
  for (int i0 = 0; i0 < real; i0 += AHEAD) {
    T t[AHEAD][V];
    float old[AHEAD][V];
    // rows, and what the table's gradient holds for words that end with them, on their way together
#pragma unroll
    for (int k = 0; k < AHEAD; k++) {
      const int i = min(i0 + k, real - 1);
      const int64_t from = (int64_t)(((uint64_t)__builtin_amdgcn_readlane(offset_high, i) << 32) | __builtin_amdgcn_readlane(offset_low, i));
      if constexpr (STREAM) load_run_stream<T, V>(rows_here + from, t[k]); else load_run_anywhere<T, V>(rows_here + from, t[k]);
    }
    if (a.accumulate) {
#pragma unroll
      for (int k = 0; k < AHEAD; k++)
        if (last_of_word >> (i0 + k) & 1) load_floats<V>(table_here + (int64_t)__builtin_amdgcn_readlane(word_here, i0 + k) * a.width, old[k]);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; k++) {
      const int i = i0 + k;
      if (i >= real) break;
#pragma unroll
      for (int e = 0; e < V; e++) sum[e] += Cvt<T>::ld(t[k][e]);
      if (!(last_of_word >> i & 1)) continue;
      if (one) {
        one = false;
#pragma unroll
        for (int e = 0; e < V; e++) ends[0][wave][lane * V + e] = sum[e];
      } else if (mine) {
        if (!a.accumulate) {
#pragma unroll
          for (int e = 0; e < V; e++) old[k][e] = 0.f;
        }
        put_row<V>(table_here + (int64_t)__builtin_amdgcn_readlane(word_here, i) * a.width, old[k], sum, a.scale);
      }
#pragma unroll
      for (int e = 0; e < V; e++) sum[e] = 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < V; e++) ends[one ? 0 : 1][wave][lane * V + e] = sum[e];
  if (lane == 0) {
    word[0][wave] = first;
    word[1][wave] = final;     // (the same word: one sum)
  }
  const int64_t begin = (int64_t)block * SUM_WAVES * a.each, end = min(begin + (int64_t)SUM_WAVES * a.each, a.rows);
  const uint32_t in_front = !SMALL && begin > 0 ? (uint32_t)a.words[begin - 1] : NO_WORD, behind = !SMALL && end < a.rows ? (uint32_t)a.words[end] : NO_WORD;
  __syncthreads();
  uint32_t words[2][SUM_WAVES];
#pragma unroll
  for (int q = 0; q < SUM_WAVES; q++)
#pragma unroll
    for (int k = 0; k < 2; k++) words[k][q] = word[k][q];
#pragma unroll
  for (int q = 0; q < SUM_WAVES; q++)
#pragma unroll
    for (int k = 0; k < 2; k++) words[k][q] = __builtin_amdgcn_readfirstlane(words[k][q]);
  for (int c = threadIdx.x; c < 64 * V; c += 64 * SUM_WAVES) {
    const int64_t to = (int64_t)slab * 64 * V + c;
    if (to >= a.width) break;
    float old[2][SUM_WAVES], part[2][SUM_WAVES];
#pragma unroll
    for (int q = 0; q < SUM_WAVES; q++)
#pragma unroll
      for (int k = 0; k < 2; k++) {
        part[k][q] = ends[k][q][c];
        old[k][q] = a.accumulate && words[k][q] != NO_WORD ? a.dtable[(int64_t)words[k][q] * a.width + to] : 0.f;
      }
    uint32_t w = words[0][0];
    float s = part[0][0], was = old[0][0];
    bool started = w != in_front;     // here, not in an earlier block
    auto put = [&](bool goes_on) {
      if (w == NO_WORD) return;
      if (started && !goes_on) a.dtable[(int64_t)w * a.width + to] = was + a.scale * s;
      else a.partial[((int64_t)block * 2 + (started ? 1 : 0)) * a.width + to] = s;
    };
#pragma unroll
    for (int q = 0; q < SUM_WAVES; q++) {
      if (q > 0) {
        if (words[0][q] == w) {
          s += part[0][q];
        } else {
          put(false);
          w = words[0][q];
          s = part[0][q];
          was = old[0][q];
          started = true;
        }
      }
      if (words[1][q] != words[0][q]) {
        put(false);
        w = words[1][q];
        s = part[1][q];
        was = old[1][q];
        started = true;
      }
    }
    put(w == behind);
  }
}

// A word that goes on behind the block where it begins: its parts, first to last.  One workgroup for every block and 64 V columns, a quarter of the parts a wave; most have
// nothing to do.
template <int V>
__global__ void __launch_bounds__(256) embedding_join_kernel(EmbedArgs a) {
  __shared__ float red[4][64 * V];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, per = (int)((a.width + 64 * V - 1) / (64 * V)), block = blockIdx.x / per;
  const int64_t size = (int64_t)SUM_WAVES * a.each, begin = block * size, end = begin + size;
  if (end >= a.rows) return;
  const uint32_t w = (uint32_t)a.words[end - 1], next = (uint32_t)a.words[end], first = (uint32_t)a.words[begin], in_front = begin > 0 ? (uint32_t)a.words[begin - 1] : NO_WORD;
  if (w == NO_WORD || next != w || (first == w && in_front == w)) return;
  // the last block that begins with it: the words are sorted
  int last = block + 1, beyond = a.blocks;
  while (beyond - last > 1) {
    const int middle = (last + beyond) / 2;
    if ((uint32_t)a.words[middle * size] == w) last = middle; else beyond = middle;
  }
  const int64_t col = (int64_t)(blockIdx.x % per) * 64 * V + lane * V;
  float s[V];
#pragma unroll
  for (int e = 0; e < V; e++) s[e] = 0.f;
  if (col < a.width) {
    const int n = last - block + 1, run = (n + 3) / 4, lo = min(wave * run, n), hi = min(lo + run, n);
#pragma unroll 8
    for (int i = lo; i < hi; i++) {
      float x[V];
      load_floats<V>(a.partial + ((int64_t)(block + i) * 2 + (i ? 0 : 1)) * a.width + col, x);
#pragma unroll
      for (int e = 0; e < V; e++) s[e] += x[e];
    }
  }
#pragma unroll
  for (int e = 0; e < V; e++) red[wave][lane * V + e] = s[e];
  __syncthreads();
  if (wave == 0 && col < a.width) {
#pragma unroll
    for (int e = 0; e < V; e++) s[e] = ((red[0][lane * V + e] + red[1][lane * V + e]) + red[2][lane * V + e]) + red[3][lane * V + e];
    float* const to = a.dtable + (int64_t)w * a.width + col;
    float old[V] = {};
    if (a.accumulate) load_floats<V>(to, old);
    put_row<V>(to, old, s, a.scale);
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------------
static int bits_of(int64_t n) {
  int b = 0;
  while (b < 62 && (int64_t(1) << b) <= n) b++;
  return b;
}
// Elements that a lane adds up.  They follow from the sizes and the type, not from where the tensors lie, and so do the rows of a wave, the order of a word's sum and its bits.  Rows
// and gradients that begin inside a vector are moved by the same instructions (8192 rows of 1024 bf16 channels, the whole gradient: 24.1 us, from odd addresses 24.5; by single elements,
// 4 rows a wave as well, 34).
static int run_of(int dtype, int64_t rows, int64_t width) {
  if (rows <= SMALL_ROWS) return dtype == CD_BF16 && width % 2 == 0 ? 2 : 1;   // (the columns are what workgroups are there for)
  return dtype == CD_BF16 && width % 8 == 0 ? 8 : width % 4 == 0 ? 4 : 1;
}

struct EmbedLayout {
  int run;                       // elements a lane adds up
  int32_t slabs, each, blocks, chunk, chunks, passes, digit_bits;
  size_t order, words, order2, words2, counts, partial, bytes;
};
static int passes_of(int64_t vocabulary) { return (int)cdiv(bits_of(vocabulary), DIGIT_BITS); }
static bool counted(int64_t rows, int64_t vocabulary) { return rows <= RANK_ROWS * (passes_of(vocabulary) + 1); }
static EmbedLayout layout_of(const cd_embedding* d) {
  const int64_t rows = d->rows, vocabulary = d->vocabulary, width = d->width;
  EmbedLayout l = {};
  l.run = run_of(d->row_dtype, rows, width);
  l.slabs = (int32_t)cdiv(width, 64 * l.run);
  if (rows <= SMALL_ROWS) {   // (no workspace)
    l.blocks = (int32_t)cdiv(rows, SMALL_BLOCK);
    return l;
  }
  l.each = 4;
  while (l.each < 64 && rows * l.slabs > (int64_t)l.each * SUM_WAVES * 1024) l.each *= 2;
  l.blocks = (int32_t)cdiv(rows, (int64_t)SUM_WAVES * l.each);
  const int64_t chunk = cdiv(rows, SORT_CHUNKS);
  l.chunk = (int32_t)(cdiv(chunk > SORT_LEAST ? chunk : SORT_LEAST, 64 * SORT_WAVES) * 64 * SORT_WAVES);
  l.chunks = (int32_t)(cdiv(cdiv(rows, l.chunk), 4) * 4);   // (the last ones may be empty)
  l.passes = passes_of(vocabulary);
  l.digit_bits = (int32_t)cdiv(bits_of(vocabulary), l.passes);
  size_t at = 0;
  auto room = [&](size_t n) { const size_t was = at; at += align_up(n, 256); return was; };
  l.order = room(rows * 4);
  l.words = room(rows * 4);
  if (!counted(rows, vocabulary)) {
    l.order2 = room(rows * 4);
    l.words2 = room(rows * 4);
    l.counts = room(((size_t)l.chunks << l.digit_bits) * 4);
  }
  l.partial = room((size_t)l.blocks * 2 * width * 4);
  l.bytes = at;
  return l;
}

static int32_t token_size(const cd_embedding* d) { return d->token_bytes & ~CD_TOKENS_AS_INDEX; }
static int check(const char* what, const cd_embedding* d) {
  CD_REQUIRE(d != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE((d->table_dtype == CD_F32 || d->table_dtype == CD_BF16) && (d->row_dtype == CD_F32 || d->row_dtype == CD_BF16), "%s: unknown dtype", what);
  const int32_t size = token_size(d);
  CD_REQUIRE(size == 4 || size == 8, "%s: token_bytes=%d must be 4 or 8, or with CD_TOKENS_AS_INDEX", what, d->token_bytes);
  CD_REQUIRE(d->rows >= 0 && d->rows <= (1ll << 30), "%s: rows=%lld out of range", what, (long long)d->rows);
  CD_REQUIRE(d->vocabulary >= 1 && d->vocabulary < (int64_t)NO_WORD, "%s: vocabulary=%lld out of range", what, (long long)d->vocabulary);
  CD_REQUIRE(d->width >= 1 && d->width <= 65536, "%s: width=%lld outside 1..65536", what, (long long)d->width);
  CD_REQUIRE(d->row_stride >= d->width || d->rows <= 1, "%s: a row is longer than its stride", what);
  CD_REQUIRE(d->row_stride <= (1ll << 32), "%s: row_stride=%lld out of range", what, (long long)d->row_stride);
  CD_REQUIRE(d->scale - d->scale == 0.f, "%s: scale must be finite", what);
  if (d->rows * cdiv(d->width, 64) >= (1ll << 32)) return set_error(CD_ERR_UNSUPPORTED, "%s: %lld rows of %lld", what, (long long)d->rows, (long long)d->width);
  return CD_OK;
}
static void set_tokens(EmbedArgs& a, const cd_embedding* d) {
  const bool index = d->token_bytes & CD_TOKENS_AS_INDEX;
  a.token_bytes = token_size(d);
  a.from_end = index;
  a.absent = index ? __builtin_nanf("") : 0.f;
}
static bool whole(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
static int size_of(int dtype) { return dtype == CD_BF16 ? 2 : 4; }

}  // namespace
}  // namespace cd

using namespace cd;

extern "C" int codistill_embedding(const cd_embedding* desc, const void* tokens, const void* table, void* y, void* stream) {
  if (const int rc = check("embedding", desc)) return rc;
  CD_REQUIRE(table && ((tokens && y) || desc->rows == 0), "embedding: NULL pointer argument");
  const int te = size_of(desc->table_dtype), re = size_of(desc->row_dtype);
  CD_REQUIRE(whole(tokens, token_size(desc)) && whole(table, te) && whole(y, re), "embedding: misaligned pointer");
  if (desc->rows == 0) return CD_OK;
  EmbedArgs a = {};
  a.tokens = tokens; a.table = table; a.y = y; a.rows = desc->rows; a.vocabulary = desc->vocabulary; a.width = desc->width;
  a.row_stride = desc->row_stride; a.scale = desc->scale;
  set_tokens(a, desc);
  // runs of 8 where both sides move 16 bytes or more a lane, of 4 where 8 or more, single elements otherwise
  auto fits = [&](int v) {
    const int64_t tb = (int64_t)v * te < 16 ? v * te : 16, rb = (int64_t)v * re < 16 ? v * re : 16;
    return desc->width % v == 0 && whole(table, tb) && whole(y, rb) && (desc->rows <= 1 || desc->row_stride * re % rb == 0);
  };
  const int v = te == 2 && fits(8) ? 8 : fits(4) ? 4 : 1;
  int lanes = 1;
  while (lanes < 256 && lanes * v < desc->width) lanes *= 2;
  const int64_t groups = cdiv(desc->rows, 256 / lanes);
  const dim3 grid((unsigned)(groups < 16384 ? groups : 16384));
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_GLUE, s, (double)a.rows * a.width, (double)a.rows * a.width * (te + re));
  auto with = [&](auto table_type, auto row_type, auto run) {
    typedef decltype(table_type) TT;
    typedef decltype(row_type) RT;
    constexpr int V = decltype(run)::value;
    if (V > 1 && desc->rows * desc->width * re >= STREAM_BYTES) hipLaunchKernelGGL((embedding_kernel<TT, RT, V, (V > 1)>), grid, dim3(256), 0, s, a, lanes);
    else hipLaunchKernelGGL((embedding_kernel<TT, RT, V, false>), grid, dim3(256), 0, s, a, lanes);
  };
  auto rows = [&](auto table_type, auto run) { if (re == 2) with(table_type, bf16_t(), run); else with(table_type, float(), run); };
  if (te == 2 && v == 8) rows(bf16_t(), std::integral_constant<int, 8>());
  else if (te == 2 && v == 4) rows(bf16_t(), std::integral_constant<int, 4>());
  else if (te == 2) rows(bf16_t(), std::integral_constant<int, 1>());
  else if (v == 4) rows(float(), std::integral_constant<int, 4>());
  else rows(float(), std::integral_constant<int, 1>());
  return check_launch("embedding");
}

extern "C" int codistill_embedding_workspace_bytes(const cd_embedding* desc, size_t* bytes) {
  if (const int rc = check("embedding_workspace_bytes", desc)) return rc;
  CD_REQUIRE(bytes != nullptr, "embedding_workspace_bytes: output pointer is NULL");
  *bytes = layout_of(desc).bytes;
  return CD_OK;
}

extern "C" int codistill_embedding_backward(const cd_embedding* desc, const void* tokens, const void* dy, float* dtable, int accumulate, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  if (const int rc = check("embedding_backward", desc)) return rc;
  CD_REQUIRE(dtable && ((tokens && dy) || desc->rows == 0), "embedding_backward: NULL pointer argument");
  const int re = size_of(desc->row_dtype);
  CD_REQUIRE(whole(tokens, token_size(desc)) && whole(dy, re) && whole(dtable, 4) && whole(workspace, 16), "embedding_backward: misaligned pointer");
  const bool small = desc->rows <= SMALL_ROWS;
  const EmbedLayout l = layout_of(desc);
  const size_t need = l.bytes;
  const int run = l.run;
  CD_REQUIRE(workspace || need == 0, "embedding_backward: NULL pointer argument");
  if (workspace_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "embedding_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (desc->rows == 0 && accumulate) return CD_OK;
  char* const ws = static_cast<char*>(workspace);
  EmbedArgs a = {};
  a.tokens = tokens; a.dy = dy; a.dtable = dtable; a.rows = desc->rows; a.vocabulary = desc->vocabulary; a.width = desc->width; a.row_stride = desc->row_stride;
  a.scale = desc->scale; a.accumulate = accumulate != 0;
  set_tokens(a, desc);
  const bool past = desc->rows * desc->width * re >= STREAM_BYTES;
  a.zero_stream = desc->vocabulary * desc->width * 4 >= STREAM_BYTES;
  a.order = reinterpret_cast<int32_t*>(ws + l.order); a.words = reinterpret_cast<int32_t*>(ws + l.words); a.partial = reinterpret_cast<float*>(ws + l.partial);
  a.each = l.each; a.blocks = l.blocks; a.slabs = l.slabs;
  const int64_t zeros = accumulate ? 0 : cdiv(desc->vocabulary, 64 * SUM_WAVES), fill = zeros < FILL_BLOCKS ? zeros : FILL_BLOCKS;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_GLUE, s, (double)a.rows * a.width, (double)a.rows * a.width * re + 4.0 * a.vocabulary * a.width);
  if (!small && counted(desc->rows, desc->vocabulary)) {
    const dim3 ranks((unsigned)cdiv(desc->rows, RANK_EACH));
    auto rank = [&](auto kernel) { hipLaunchKernelGGL(kernel, ranks, dim3(256), 0, s, a); };
    if (a.token_bytes == 8) { if (a.from_end) rank(embedding_rank_kernel<int64_t, true>); else rank(embedding_rank_kernel<int64_t, false>); }
    else if (a.from_end) rank(embedding_rank_kernel<int32_t, true>);
    else rank(embedding_rank_kernel<int32_t, false>);
  } else if (!small) {
    int32_t *order = a.order, *words = a.words, *order2 = reinterpret_cast<int32_t*>(ws + l.order2), *words2 = reinterpret_cast<int32_t*>(ws + l.words2);
    a.counts = reinterpret_cast<int32_t*>(ws + l.counts);
    a.chunk = l.chunk; a.chunks = l.chunks; a.digits = 1 << l.digit_bits;
    for (int pass = 0; pass < l.passes; pass++) {
      const bool here = (l.passes - 1 - pass) % 2 == 0;   // the last pass leaves its result in order and words
      a.order = here ? order : order2; a.words = here ? words : words2;
      a.order2 = here ? order2 : order; a.words2 = here ? words2 : words;
      a.from_tokens = pass == 0; a.shift = pass * l.digit_bits;
      hipLaunchKernelGGL(embedding_count_kernel, dim3(a.chunks), dim3(512), 0, s, a);
      hipLaunchKernelGGL(embedding_scatter_kernel, dim3(a.chunks), dim3(512), 0, s, a);
    }
  }
  a.sums = (int64_t)l.blocks * l.slabs;
  const dim3 blocks((unsigned)(a.sums + fill));
  auto sum = [&](auto kernel) { hipLaunchKernelGGL(kernel, blocks, dim3(64 * SUM_WAVES), 0, s, a); };
  if (small) {
    if (re == 2) { if (run == 2) sum(embedding_sum_kernel<bf16_t, 2, true, false>); else sum(embedding_sum_kernel<bf16_t, 1, true, false>); }
    else sum(embedding_sum_kernel<float, 1, true, false>);
  } else if (re == 2) {
    if (run == 8) { if (past) sum(embedding_sum_kernel<bf16_t, 8, false, true>); else sum(embedding_sum_kernel<bf16_t, 8, false, false>); }
    else if (run == 4) sum(embedding_sum_kernel<bf16_t, 4, false, false>);
    else sum(embedding_sum_kernel<bf16_t, 1, false, false>);
  } else {
    if (run == 4) { if (past) sum(embedding_sum_kernel<float, 4, false, true>); else sum(embedding_sum_kernel<float, 4, false, false>); }
    else sum(embedding_sum_kernel<float, 1, false, false>);
  }
  if (l.blocks > 1 && !small) {
    const int64_t joins = l.blocks - 1;
    if (run > 1) hipLaunchKernelGGL((embedding_join_kernel<4>), dim3((unsigned)(joins * cdiv(desc->width, 256))), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((embedding_join_kernel<1>), dim3((unsigned)(joins * cdiv(desc->width, 64))), dim3(256), 0, s, a);
  }
  return check_launch("embedding_backward");
}
