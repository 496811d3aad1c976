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
// The order.  Few rows: a row's place is the number of rows in front of it, counted by comparing it with all of them (64 comparisons are one
// vector instruction and two scalar ones: 8192 rows are 2^20 of those, a few microseconds of the chip, and one launch).  Many rows: a radix sort, two
// launches for each digit of up to 10 bits: digits of a chunk are counted, then every chunk knows where its own begin.
#include "common.h"
#include "vec.h"

namespace cd {
namespace {

constexpr uint32_t NO_WORD = 0x7fffffffu;   // sorted behind all words
constexpr int RANK_ROWS = 16384;            // most rows whose places are counted
constexpr int RANK_EACH = 16, RANK_AHEAD = 8;   // rows of a workgroup there, loads in flight
constexpr int DIGIT_BITS = 10, SORT_CHUNKS = 256, SORT_LEAST = 1024, SORT_WAVES = 8;
constexpr int SUM_WAVES = 8;                // waves of a block of rows
constexpr int FILL_BLOCKS = 1024;

struct EmbedArgs {
  const void* tokens; const void* table; const void* dy; void* y; float* dtable;
  int32_t *order, *words, *order2, *words2, *counts;   // rows and words in sorted order; the same between passes of the radix sort; counts [digits][chunks]
  float* partial;                                      // [blocks][2][width]: sums of a block's first and last words, where others have parts of them
  int64_t rows, vocabulary, width, row_stride, sums;   // sums: workgroups that add up; the others write zeros
  int32_t token_bytes, accumulate, each, blocks, slabs, chunk, chunks, shift, digits, from_tokens;
  float scale;
};

__device__ inline uint32_t word_of(const EmbedArgs& a, int64_t i) {
  const int64_t w = a.token_bytes == 8 ? static_cast<const int64_t*>(a.tokens)[i] : static_cast<const int32_t*>(a.tokens)[i];
  return w >= 0 && w < a.vocabulary ? (uint32_t)w : NO_WORD;
}

// ---- lookup ---------------------------------------------------------------------------------------------------------------
// TT: the table's type, RT: the rows'; V: elements of a run
template <typename TT, typename RT, int V>
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
        for (int e = 0; e < V; e++) out[e] = 0.f;
      } else {
        TT t[V];
        load_run<TT, V>(from + c, t);
#pragma unroll
        for (int e = 0; e < V; e++) out[e] = a.scale * Cvt<TT>::ld(t[e]);
      }
      // (runs of 8 floats are two stores)
      if constexpr (sizeof(RT) * V == 32) {
        float lo[4] = {out[0], out[1], out[2], out[3]}, hi[4] = {out[4], out[5], out[6], out[7]};
        store_run<RT, 4>(to + c, lo);
        store_run<RT, 4>(to + c + 4, hi);
      } else {
        store_run<RT, V>(to + c, out);
      }
    }
  }
}

// ---- the order of the rows --------------------------------------------------------------------------------------------------
// Few rows: place of row i = rows with a smaller word + rows in front of it with the same.  A wave compares 64 rows with one of the
// workgroup's at a time; what it counts is scalar.
__global__ void __launch_bounds__(256) embedding_rank_kernel(EmbedArgs a) {
  __shared__ uint32_t mine[RANK_EACH];
  __shared__ int found[4][RANK_EACH];
  const int i0 = blockIdx.x * RANK_EACH, rows = (int)a.rows, wave = threadIdx.x >> 6;
  if (threadIdx.x < RANK_EACH) mine[threadIdx.x] = i0 + (int)threadIdx.x < rows ? word_of(a, i0 + threadIdx.x) : 0;
  __syncthreads();
  uint32_t w[RANK_EACH];
  int count[RANK_EACH];
#pragma unroll
  for (int r = 0; r < RANK_EACH; r++) {
    w[r] = __builtin_amdgcn_readfirstlane(mine[r]);
    count[r] = 0;
  }
  for (int k0 = wave * 64; k0 < rows; k0 += 256 * RANK_AHEAD) {
    uint32_t others[RANK_AHEAD];
#pragma unroll
    for (int u = 0; u < RANK_AHEAD; u++) {
      const int j = k0 + 256 * u + (threadIdx.x & 63);
      others[u] = j < rows ? word_of(a, j) : 0xffffffffu;
    }
#pragma unroll
    for (int u = 0; u < RANK_AHEAD; u++) {
      const int j0 = k0 + 256 * u;
      const uint32_t other = others[u];
      if (j0 + 64 <= i0 || j0 >= i0 + RANK_EACH) {   // all 64 in front of the workgroup's rows, or all behind
        const uint32_t same = j0 < i0;
#pragma unroll
        for (int r = 0; r < RANK_EACH; r++) count[r] += __popcll(__ballot(other < w[r] + same));
      } else {
        const int j = j0 + (threadIdx.x & 63);
#pragma unroll
        for (int r = 0; r < RANK_EACH; r++) count[r] += __popcll(__ballot(other < w[r] + (j < i0 + r ? 1u : 0u)));
      }
    }
  }
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int r = 0; r < RANK_EACH; r++) found[wave][r] = count[r];
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
  __shared__ int sums[8];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, me = blockIdx.x;
  for (int d = lane; d < a.digits; d += 64) at[wave][d] = 0;
  // a thread's two digits: rows of them in chunks in front, and in all
  int before[2] = {0, 0}, all[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const int d = 2 * threadIdx.x + k;
    if (d < a.digits) {
#pragma unroll 8
      for (int c = 0; c < a.chunks; c += 4) {   // (rows of whole vectors: what lies behind the chunks is zero)
        const int4 n = *reinterpret_cast<const int4*>(a.counts + d * a.chunks + c);
        before[k] += (c < me ? n.x : 0) + (c + 1 < me ? n.y : 0) + (c + 2 < me ? n.z : 0) + (c + 3 < me ? n.w : 0);
        all[k] += (n.x + n.y) + (n.z + n.w);
      }
    }
  }
  // exclusive sum of `all` over the digits
  int sum = all[0] + all[1];
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int up = __shfl_up(sum, o, 64);
    if (lane >= o) sum += up;
  }
  if (lane == 63) sums[wave] = sum;
  __syncthreads();
  int base = sum - all[0] - all[1];
  for (int q = 0; q < wave; q++) base += sums[q];
  // each wave counts its own run of the chunk
  const int64_t from = (int64_t)me * a.chunk, to = min(from + a.chunk, a.rows);
  const int64_t run = a.chunk / SORT_WAVES, mine = min(from + wave * run, to), end = min(mine + run, to);
  for (int64_t i = mine + lane; i < end; i += 64) atomicAdd(&at[wave][sort_key(a, i) >> a.shift & (a.digits - 1)], 1);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const int d = 2 * threadIdx.x + k;
    if (d < a.digits) {
      int place = base + (k ? all[0] : 0) + before[k];
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
template <int V> __device__ inline void add_row(float* to, const float (&sum)[V], float scale, bool accumulate, bool vector) {
  if (V >= 4 && vector) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      float4 t = make_float4(scale * sum[e], scale * sum[e + 1], scale * sum[e + 2], scale * sum[e + 3]);
      if (accumulate) {
        const float4 old = *reinterpret_cast<const float4*>(to + e);
        t = make_float4(old.x + t.x, old.y + t.y, old.z + t.z, old.w + t.w);
      }
      *reinterpret_cast<float4*>(to + e) = t;
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; e++) to[e] = accumulate ? to[e] + scale * sum[e] : scale * sum[e];
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
__device__ inline void zero_absent(const EmbedArgs& a, int me, int all) {
  __shared__ uint8_t there[64 * SUM_WAVES];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool vector = a.width % 4 == 0 && (reinterpret_cast<uintptr_t>(a.dtable) & 15) == 0;
  for (int64_t w0 = (int64_t)me * 64 * SUM_WAVES; w0 < a.vocabulary; w0 += (int64_t)all * 64 * SUM_WAVES) {
    const int64_t first = lower_bound(a.words, (uint32_t)w0, 0, a.rows), last = lower_bound(a.words, (uint32_t)w0 + 64 * SUM_WAVES, first, a.rows);
    const uint32_t mine = (uint32_t)w0 + threadIdx.x;
    int64_t from = first, to = last;
    while (from < to) {
      const int64_t middle = (from + to) / 2;
      if ((uint32_t)a.words[middle] < mine) from = middle + 1; else to = middle;
    }
    __syncthreads();
    there[threadIdx.x] = from < last && (uint32_t)a.words[from] == mine;
    __syncthreads();
    const int n = (int)min((int64_t)64 * SUM_WAVES, a.vocabulary - w0);
    for (int i = wave; i < n; i += SUM_WAVES) {
      if (there[i]) continue;
      float* const row = a.dtable + (w0 + i) * a.width;
      if (vector) {
        for (int64_t col = 4 * lane; col < a.width; col += 256) *reinterpret_cast<uint4*>(row + col) = make_uint4(0, 0, 0, 0);
      } else {
        for (int64_t col = lane; col < a.width; col += 64) row[col] = 0.f;
      }
    }
  }
}

// A block of SUM_WAVES * each rows in sorted order, 64 V columns.  A wave adds up `each` of them, writes the words that are its alone and leaves its first and
// its last word's sum in LDS; the waves' ends are then put together, column by column, in their order.
template <typename T, int V>
__global__ void __launch_bounds__(64 * SUM_WAVES) embedding_sum_kernel(EmbedArgs a) {
  if ((int64_t)blockIdx.x >= a.sums) return zero_absent(a, (int)(blockIdx.x - a.sums), (int)(gridDim.x - a.sums));
  __shared__ float ends[2][SUM_WAVES][64 * V];
  __shared__ uint32_t word[2][SUM_WAVES];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, block = blockIdx.x / a.slabs, slab = blockIdx.x % a.slabs;
  const int64_t col = (int64_t)slab * 64 * V + lane * V;
  const bool mine = col < a.width;     // (a width of whole runs)
  const int64_t from = (int64_t)block * SUM_WAVES * a.each + (int64_t)wave * a.each;
  const int n = (int)max((int64_t)0, min((int64_t)a.each, a.rows - from));
  // this wave's rows and words: one a lane
  const int row_here = lane < n ? a.order[from + lane] : 0;
  const uint32_t word_here = lane < n ? (uint32_t)a.words[from + lane] : NO_WORD;
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; e++) sum[e] = 0.f;
  uint32_t first = __builtin_amdgcn_readlane(word_here, 0), open = first;
  bool one = true;     // no word has ended yet
  auto close = [&]() {   // `open` has ended inside this wave's rows
    if (one) {
#pragma unroll
      for (int e = 0; e < V; e++) ends[0][wave][lane * V + e] = sum[e];
    } else if (mine) {
      add_row<V>(a.dtable + (int64_t)open * a.width + col, sum, a.scale, a.accumulate, V >= 4);
    }
    one = false;
#pragma unroll
    for (int e = 0; e < V; e++) sum[e] = 0.f;
  };
  constexpr int AHEAD = 4;
  for (int i0 = 0; i0 < n; i0 += AHEAD) {
    T t[AHEAD][V];
#pragma unroll
    for (int k = 0; k < AHEAD; k++) {
      const int i = i0 + k;
#pragma unroll
      for (int e = 0; e < V; e++) t[k][e] = T(0);
      if (i < n && __builtin_amdgcn_readlane(word_here, i) != NO_WORD && mine)
        load_run<T, V>(static_cast<const T*>(a.dy) + (int64_t)__builtin_amdgcn_readlane(row_here, i) * a.row_stride + col, t[k]);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; k++) {
      const int i = i0 + k;
      if (i >= n) break;
      const uint32_t w = __builtin_amdgcn_readlane(word_here, i);
      if (w != open) {
        close();
        open = w;
      }
#pragma unroll
      for (int e = 0; e < V; e++) sum[e] += Cvt<T>::ld(t[k][e]);
    }
  }
#pragma unroll
  for (int e = 0; e < V; e++) ends[one ? 0 : 1][wave][lane * V + e] = sum[e];
  if (lane == 0) {
    word[0][wave] = first;
    word[1][wave] = one ? first : open;     // (the same word: one sum)
  }
  __syncthreads();
  const int64_t begin = (int64_t)block * SUM_WAVES * a.each, end = min(begin + (int64_t)SUM_WAVES * a.each, a.rows);
  const uint32_t in_front = begin > 0 ? (uint32_t)a.words[begin - 1] : NO_WORD, behind = end < a.rows ? (uint32_t)a.words[end] : NO_WORD;
  for (int c = threadIdx.x; c < 64 * V; c += 64 * SUM_WAVES) {
    const int64_t to = (int64_t)slab * 64 * V + c;
    if (to >= a.width) break;
    uint32_t w = word[0][0];
    float s = ends[0][0][c];
    bool started = w != in_front;     // here, not in an earlier block
    auto put = [&](bool goes_on) {
      if (w == NO_WORD) return;
      if (started && !goes_on) {
        float* const p = a.dtable + (int64_t)w * a.width + to;
        *p = a.accumulate ? *p + a.scale * s : a.scale * s;
      } else {
        a.partial[((int64_t)block * 2 + (started ? 1 : 0)) * a.width + to] = s;
      }
    };
    for (int q = 0; q < SUM_WAVES; q++) {
      if (q > 0) {
        if (word[0][q] == w) {
          s += ends[0][q][c];
        } else {
          put(false);
          w = word[0][q];
          s = ends[0][q][c];
          started = true;
        }
      }
      if (word[1][q] != word[0][q]) {
        put(false);
        w = word[1][q];
        s = ends[1][q][c];
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
      load_run<float, V>(a.partial + ((int64_t)(block + i) * 2 + (i ? 0 : 1)) * a.width + col, x);
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
    add_row<V>(a.dtable + (int64_t)w * a.width + col, s, a.scale, a.accumulate, V >= 4);
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------------
static int bits_of(int64_t n) {
  int b = 0;
  while (b < 62 && (int64_t(1) << b) <= n) b++;
  return b;
}
static int run_of(int dtype, int64_t width) { return dtype == CD_BF16 && width % 8 == 0 ? 8 : width % 4 == 0 ? 4 : 1; }

struct EmbedLayout {
  int run;                       // elements a lane adds up
  int32_t slabs, each, blocks, chunk, chunks, passes, digit_bits;
  size_t order, words, order2, words2, counts, partial, bytes;
};
static EmbedLayout layout_of(int dtype, int64_t rows, int64_t vocabulary, int64_t width, int run) {
  EmbedLayout l = {};
  l.run = run;
  l.slabs = (int32_t)cdiv(width, 64 * run);
  l.each = 4;
  while (l.each < 64 && rows * l.slabs > (int64_t)l.each * SUM_WAVES * 1024) l.each *= 2;
  l.blocks = (int32_t)cdiv(rows, (int64_t)SUM_WAVES * l.each);
  const int64_t chunk = cdiv(rows, SORT_CHUNKS);
  l.chunk = (int32_t)(cdiv(chunk > SORT_LEAST ? chunk : SORT_LEAST, 64 * SORT_WAVES) * 64 * SORT_WAVES);
  l.chunks = (int32_t)(cdiv(cdiv(rows, l.chunk), 4) * 4);   // (the last ones may be empty)
  const int bits = bits_of(vocabulary);
  l.passes = (int32_t)cdiv(bits, DIGIT_BITS);
  l.digit_bits = (int32_t)cdiv(bits, l.passes);
  size_t at = 0;
  auto room = [&](size_t n) { const size_t was = at; at += align_up(n, 256); return was; };
  l.order = room(rows * 4);
  l.words = room(rows * 4);
  if (rows > RANK_ROWS) {
    l.order2 = room(rows * 4);
    l.words2 = room(rows * 4);
    l.counts = room(((size_t)l.chunks << l.digit_bits) * 4);
  }
  l.partial = room((size_t)l.blocks * 2 * width * 4);
  l.bytes = at;
  return l;
}

static int check(const char* what, const cd_embedding* d) {
  CD_REQUIRE(d != nullptr, "%s: NULL pointer argument", what);
  CD_REQUIRE((d->table_dtype == CD_F32 || d->table_dtype == CD_BF16) && (d->row_dtype == CD_F32 || d->row_dtype == CD_BF16), "%s: unknown dtype", what);
  CD_REQUIRE(d->token_bytes == 4 || d->token_bytes == 8, "%s: token_bytes=%d must be 4 or 8", what, d->token_bytes);
  CD_REQUIRE(d->rows >= 0 && d->rows <= (1ll << 30), "%s: rows=%lld out of range", what, (long long)d->rows);
  CD_REQUIRE(d->vocabulary >= 1 && d->vocabulary < (int64_t)NO_WORD, "%s: vocabulary=%lld out of range", what, (long long)d->vocabulary);
  CD_REQUIRE(d->width >= 1 && d->width <= 65536, "%s: width=%lld outside 1..65536", what, (long long)d->width);
  CD_REQUIRE(d->row_stride >= d->width || d->rows <= 1, "%s: a row is longer than its stride", what);
  CD_REQUIRE(d->row_stride <= (1ll << 32), "%s: row_stride=%lld out of range", what, (long long)d->row_stride);
  CD_REQUIRE(d->scale - d->scale == 0.f, "%s: scale must be finite", what);
  if (d->rows * d->width > (1ll << 40)) return set_error(CD_ERR_UNSUPPORTED, "%s: %lld rows of %lld", what, (long long)d->rows, (long long)d->width);
  return CD_OK;
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
  CD_REQUIRE(whole(tokens, desc->token_bytes) && whole(table, te) && whole(y, re), "embedding: misaligned pointer");
  if (desc->rows == 0) return CD_OK;
  EmbedArgs a = {};
  a.tokens = tokens; a.table = table; a.y = y; a.rows = desc->rows; a.vocabulary = desc->vocabulary; a.width = desc->width;
  a.row_stride = desc->row_stride; a.token_bytes = desc->token_bytes; a.scale = desc->scale;
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
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, lanes); };
  if (te == 2 && re == 2) { if (v == 8) run(embedding_kernel<bf16_t, bf16_t, 8>); else if (v == 4) run(embedding_kernel<bf16_t, bf16_t, 4>); else run(embedding_kernel<bf16_t, bf16_t, 1>); }
  else if (te == 2) { if (v == 8) run(embedding_kernel<bf16_t, float, 8>); else if (v == 4) run(embedding_kernel<bf16_t, float, 4>); else run(embedding_kernel<bf16_t, float, 1>); }
  else if (re == 2) { if (v == 4) run(embedding_kernel<float, bf16_t, 4>); else run(embedding_kernel<float, bf16_t, 1>); }
  else { if (v == 4) run(embedding_kernel<float, float, 4>); else run(embedding_kernel<float, float, 1>); }
  return check_launch("embedding");
}

extern "C" int codistill_embedding_workspace_bytes(const cd_embedding* desc, size_t* bytes) {
  if (const int rc = check("embedding_workspace_bytes", desc)) return rc;
  CD_REQUIRE(bytes != nullptr, "embedding_workspace_bytes: output pointer is NULL");
  // (which runs a call takes depends on its pointers: room for any of them)
  size_t most = 0;
  for (int run : {8, 4, 1}) {
    const EmbedLayout l = layout_of(desc->row_dtype, desc->rows, desc->vocabulary, desc->width, run);
    most = l.bytes > most ? l.bytes : most;
  }
  *bytes = most;
  return CD_OK;
}

extern "C" int codistill_embedding_backward(const cd_embedding* desc, const void* tokens, const void* dy, float* dtable, int accumulate, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  if (const int rc = check("embedding_backward", desc)) return rc;
  CD_REQUIRE(dtable && ((tokens && dy && workspace) || desc->rows == 0), "embedding_backward: NULL pointer argument");
  const int re = size_of(desc->row_dtype);
  CD_REQUIRE(whole(tokens, desc->token_bytes) && whole(dy, re) && whole(dtable, 4) && whole(workspace, 16), "embedding_backward: misaligned pointer");
  int run = run_of(desc->row_dtype, desc->width);
  if (run > 1 && !(whole(dtable, 16) && whole(dy, run * re) && (desc->rows <= 1 || desc->row_stride % run == 0))) run = 1;
  size_t need = 0;
  codistill_embedding_workspace_bytes(desc, &need);
  if (workspace_bytes < need) return set_error(CD_ERR_WORKSPACE_TOO_SMALL, "embedding_backward: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (desc->rows == 0 && accumulate) return CD_OK;
  const EmbedLayout l = layout_of(desc->row_dtype, desc->rows, desc->vocabulary, desc->width, run);
  char* const ws = static_cast<char*>(workspace);
  EmbedArgs a = {};
  a.tokens = tokens; a.dy = dy; a.dtable = dtable; a.rows = desc->rows; a.vocabulary = desc->vocabulary; a.width = desc->width; a.row_stride = desc->row_stride;
  a.token_bytes = desc->token_bytes; a.scale = desc->scale; a.accumulate = accumulate != 0;
  a.order = reinterpret_cast<int32_t*>(ws + l.order); a.words = reinterpret_cast<int32_t*>(ws + l.words); a.partial = reinterpret_cast<float*>(ws + l.partial);
  a.each = l.each; a.blocks = l.blocks; a.slabs = l.slabs;
  const int64_t zeros = accumulate ? 0 : cdiv(desc->vocabulary, 64 * SUM_WAVES), fill = zeros < FILL_BLOCKS ? zeros : FILL_BLOCKS;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope prof(CD_K_GLUE, s, (double)a.rows * a.width, (double)a.rows * a.width * re + 4.0 * a.vocabulary * a.width);
  if (desc->rows <= RANK_ROWS) {
    if (desc->rows) hipLaunchKernelGGL(embedding_rank_kernel, dim3((unsigned)cdiv(desc->rows, RANK_EACH)), dim3(256), 0, s, a);
  } else {
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
  if (re == 2) { if (run == 8) sum(embedding_sum_kernel<bf16_t, 8>); else if (run == 4) sum(embedding_sum_kernel<bf16_t, 4>); else sum(embedding_sum_kernel<bf16_t, 1>); }
  else { if (run == 4) sum(embedding_sum_kernel<float, 4>); else sum(embedding_sum_kernel<float, 1>); }
  if (l.blocks > 1) {
    const int64_t joins = l.blocks - 1;
    if (run > 1) hipLaunchKernelGGL((embedding_join_kernel<4>), dim3((unsigned)(joins * cdiv(desc->width, 256))), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((embedding_join_kernel<1>), dim3((unsigned)(joins * cdiv(desc->width, 64))), dim3(256), 0, s, a);
  }
  return check_launch("embedding_backward");
}
