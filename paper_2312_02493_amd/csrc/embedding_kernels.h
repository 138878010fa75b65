// Embedding lookup and its gradient, for gfx950.
//
//   y[i] = scale table[token[i]]
//   dtable[v] = scale (sum over the places i with token[i] = v of dy[i])  (added to what is there, or in its place)
//
// Both are bound by memory.  The gradient's places are sorted by token first (stable: a token's places stay in order), so that
// every row of the table has one owner that sums its places in a fixed order: no atomics on sums, the same bits every time.  Most
// of what the gradient writes are zeros, rows of tokens that do not occur; they are written beside the sort.
//
// Measured: gradient of 32768 places x 2048 bfloat16 into 64000 rows of float32 (658 MB) 136 us = 4.8 TB/s, of which the sort's four
// launches 35 (with 190 MB of zeros), the sums 96 (with the other 250 MB), heavy tokens' shares 5; lookup of 32768 x 4096, float32 to
// bfloat16, 87 us (results through the caches 95).
#pragma once

#include "elements.h"

namespace artopk {

// Token numbers of 32 or 64 bits.
struct Tokens {
  const void* at;
  int32_t wide;
  __device__ __forceinline__ int64_t operator[](int64_t i) const {
    return wide ? static_cast<const int64_t*>(at)[i] : static_cast<int64_t>(static_cast<const int32_t*>(at)[i]);
  }
};

// Sixteen bytes at a place of four, or of two.
typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t Words2 __attribute__((ext_vector_type(4), aligned(2)));

// V elements at any place of their type, as they lie.
template <class T, int V>
struct Some {
  T e[V];
  using Words = std::conditional_t<sizeof(T) == 4, Words4, Words2>;
  // sixteen bytes at a time (as such: of single elements the compiler may make single loads), or all there is; with ONCE past
  // the caches
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(e) % 16 == 0) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(e) / 16; ++i) {
        const Words* at = reinterpret_cast<const Words*>(p) + i;
        Words w;
        if constexpr (ONCE) w = __builtin_nontemporal_load(at); else w = *at;
        __builtin_memcpy(reinterpret_cast<char*>(e) + 16 * i, &w, 16);
      }
    } else {
      __builtin_memcpy(e, p, sizeof(e));
    }
  }
  template <bool ONCE = false>
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (sizeof(e) % 16 == 0) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(e) / 16; ++i) {
        Words w;
        __builtin_memcpy(&w, reinterpret_cast<const char*>(e) + 16 * i, 16);
        if constexpr (ONCE) __builtin_nontemporal_store(w, reinterpret_cast<Words*>(p) + i);
        else reinterpret_cast<Words*>(p)[i] = w;
      }
    } else {
      __builtin_memcpy(p, e, sizeof(e));
    }
  }
};

constexpr int kEmbedPieces = 4;  // a lane has under way

// A wave takes 64 >> lg tokens at a time (one where a row has at least 64 pieces of V elements) and kEmbedPieces << lg pieces
// of each.  Columns are at least V.
template <class TT, class TY, int V>
__global__ __launch_bounds__(256) void k_embed(const TT* __restrict__ table, int64_t table_stride, int64_t vocab, Tokens tokens,
                                               int64_t count, int64_t cols, float scale, TY* __restrict__ y, int64_t y_stride,
                                               int lg, int64_t units, int64_t tiles, int* __restrict__ error) {
  const int lane = threadIdx.x & 63;
  const int sub = lane >> lg, at = lane & ((1 << lg) - 1);
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t group = unit / tiles, tile = unit % tiles;
    const int64_t i = group * (64 >> lg) + sub;
    const int64_t tok = tokens[i < count ? i : count - 1];
    const bool good = tok >= 0 && tok < vocab;
    const TT* row = table + (good ? tok : 0) * table_stride;
    int64_t c[kEmbedPieces];
    Some<TT, V> in[kEmbedPieces];
#pragma unroll
    for (int u = 0; u < kEmbedPieces; ++u) {
      c[u] = (tile * (kEmbedPieces << lg) + (u << lg) + at) * V;
      in[u].load(row + (c[u] + V <= cols ? c[u] : cols - V));  // (places behind the row's end: its last ones, not stored)
    }
    if (i >= count) continue;
    if (tok >= vocab && at == 0) *error = 1;
    const float other = tok < 0 ? 0.0f : __builtin_nanf("");
    TY* out = y + i * y_stride;
#pragma unroll
    for (int u = 0; u < kEmbedPieces; ++u) {
      if (c[u] >= cols) continue;
      Some<TY, V> o;
      if (c[u] + V <= cols) {
#pragma unroll
        for (int j = 0; j < V; ++j) o.e[j] = static_cast<TY>(good ? static_cast<float>(in[u].e[j]) * scale : other);
        o.template store<true>(out + c[u]);
      } else {
        for (int64_t j = c[u]; j < cols; ++j) out[j] = static_cast<TY>(good ? static_cast<float>(row[j]) * scale : other);
      }
    }
  }
}

// ---- rows of zeros --------------------------------------------------------------------------------
// Rows of a table that no token names, in bytes (zero is all bits zero in every type).  They are most of what a gradient has to
// write, so the launches that sort, which fill a few compute units, write them beside it: blocks from a launch's own on call
// zero_rows.  Which rows are named says a byte each (`marks`), or, once they are sorted, the keys.
struct ZeroRows {
  uint8_t* at;  // NULL: none
  int64_t pitch;
  int32_t bytes, lg;  // of a row; lanes a row, as a power of two
  int64_t begin, end;  // the rows of this launch
  const uint8_t* marks;
  const uint32_t* key;  // where marks is NULL: `count` sorted keys
  int64_t count;
};

__device__ __forceinline__ bool row_named(const ZeroRows& z, int64_t r) {
  if (z.marks) return z.marks[r] != 0;
  int64_t a = 0, b = z.count;
  while (a < b) {
    const int64_t m = (a + b) >> 1;
    if (z.key[m] < r) a = m + 1; else b = m;
  }
  return a < z.count && z.key[a] == r;
}

__device__ __forceinline__ void zero_rows(const ZeroRows& z, int64_t wave, int64_t waves) {
  const int lane = threadIdx.x & 63, sub = lane >> z.lg, at = lane & ((1 << z.lg) - 1), per = 64 >> z.lg;
  for (int64_t r0 = z.begin + wave * per; r0 < z.end; r0 += waves * per) {
    const int64_t r = r0 + sub;
    if (r >= z.end || row_named(z, r)) continue;
    uint8_t* row = z.at + r * z.pitch;
    const int lead = (int)(-reinterpret_cast<uintptr_t>(row) & 15), head = lead < z.bytes ? lead : z.bytes;
    const int pieces = (z.bytes - head) / 16, tail = head + pieces * 16;
    for (int j = at * 2; j < head; j += 2 << z.lg) *reinterpret_cast<uint16_t*>(row + j) = 0;
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words* p = reinterpret_cast<words*>(row + head);
#pragma unroll 4
    for (int j = at; j < pieces; j += 1 << z.lg) __builtin_nontemporal_store((words)(0), p + j);
    for (int j = tail + at * 2; j < z.bytes; j += 2 << z.lg) *reinterpret_cast<uint16_t*>(row + j) = 0;
  }
}

// ---- places sorted by token ----------------------------------------------------------------------
// One pass of a radix sort takes `bits` bits of the keys, from `shift` on: how often each tile has each digit, then every key
// to its place.  A tile is a run of tokens of one block, `per` of them; keys of the first pass are the tokens themselves, places
// without a token (or with one that is not in the table) get the key `vocab` and so come last.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortBits = 11, kSortDigits = 1 << kSortBits;
constexpr int kSortTiles = 64;  // at most

struct SortKeys {
  Tokens tokens;  // of the first pass
  const uint32_t *key, *pos;
  uint32_t vocab;
  int first;
  uint32_t* heavy_count;  // the first pass's first thread makes it zero
  uint8_t* marks;  // NULL, or where the first pass marks the rows that are named
  __device__ __forceinline__ void get(int64_t i, uint32_t& k, uint32_t& p) const {
    if (first) {
      const int64_t t = tokens[i];
      k = t < 0 || t >= (int64_t)vocab ? vocab : (uint32_t)t;
      p = (uint32_t)i;
    } else {
      k = key[i];
      p = pos[i];
    }
  }
};

// Lanes of a wave see what the others wrote to LDS before.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The lanes among `live` that have the same digit.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, bool live) {
  uint64_t same = __ballot(live);
  for (int b = 0; b < bits; ++b) {
    const uint64_t one = __ballot((d >> b) & 1);
    same &= (d >> b) & 1 ? one : ~one;
  }
  return same;
}

// Sums over the block of the values before each thread's own; `room` holds one value a wave.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(s, off, 64);
    if (lane >= off) s += o;
  }
  if (lane == 63) room[wave] = s;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) before += w < wave ? room[w] : 0;
  return before + s - v;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_count(SortKeys in, int64_t count, int64_t per, int shift, int bits, int tiles,
                                                             uint32_t* __restrict__ counts, int* __restrict__ error, ZeroRows zero) {
  __shared__ uint32_t hist[kSortDigits];
  if ((int)blockIdx.x >= tiles) {
    zero_rows(zero, (int64_t)(blockIdx.x - tiles) * kSortWaves + (threadIdx.x >> 6), (int64_t)(gridDim.x - tiles) * kSortWaves);
    return;
  }
  const uint32_t mask = (1u << bits) - 1;
  if (in.first && blockIdx.x == 0 && threadIdx.x == 0) *in.heavy_count = 0;
  for (int d = threadIdx.x; d <= (int)mask; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * per, hi = lo + per < count ? lo + per : count;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads) {
    uint32_t k, p;
    in.get(i, k, p);
    if (in.first) {
      if (k < in.vocab) {
        if (in.marks) in.marks[k] = 1;
      } else if (in.tokens[i] >= 0) {
        *error = 1;
      }
    }
    atomicAdd(&hist[(k >> shift) & mask], 1u);  // (whole numbers: the order does not matter)
  }
  __syncthreads();
  for (int d = threadIdx.x; d <= (int)mask; d += kSortThreads) counts[(size_t)blockIdx.x * (mask + 1) + d] = hist[d];
}

// R keys a thread in a round.
template <int R>
__global__ __launch_bounds__(kSortThreads) void k_sort_place(SortKeys in, int64_t count, int64_t per, int shift, int bits,
                                                             const uint32_t* __restrict__ counts, int tiles,
                                                             uint32_t* __restrict__ key_out, uint32_t* __restrict__ pos_out,
                                                             ZeroRows zero) {
  __shared__ uint32_t base[kSortDigits];           // where the tile's next key of each digit goes
  __shared__ alignas(8) uint16_t seen[kSortWaves * kSortDigits];  // keys of each digit that a wave has in this round
  __shared__ uint32_t room[kSortWaves];
  if ((int)blockIdx.x >= tiles) {
    zero_rows(zero, (int64_t)(blockIdx.x - tiles) * kSortWaves + (threadIdx.x >> 6), (int64_t)(gridDim.x - tiles) * kSortWaves);
    return;
  }
  const int digits = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t mask = digits - 1;
  uint16_t* mine = seen + wave * digits;
  {
    // Two digits a thread, side by side, so that the sum over threads runs over the digits in order; up to sixteen groups of
    // threads share the tiles (one alone waits 5 us for 64 tiles' counts).
    const int pairs = digits / 2, groups = kSortThreads / pairs < 16 ? kSortThreads / pairs : 16;
    const int group = threadIdx.x / pairs, d = threadIdx.x % pairs * 2;
    uint2* sums = reinterpret_cast<uint2*>(seen);  // [group][digit]: keys of all tiles, and of those before this one
    if (group < groups) {
      uint2 s[2] = {{0, 0}, {0, 0}};
#pragma unroll 8
      for (int t = group; t < tiles; t += groups) {
        const uint2 n = *reinterpret_cast<const uint2*>(counts + (size_t)t * digits + d);
        s[0].x += n.x;
        s[1].x += n.y;
        s[0].y += t < (int)blockIdx.x ? n.x : 0;
        s[1].y += t < (int)blockIdx.x ? n.y : 0;
      }
      sums[group * digits + d] = s[0];
      sums[group * digits + d + 1] = s[1];
    }
    __syncthreads();
    uint2 s[2] = {{0, 0}, {0, 0}};
    if (group == 0)
      for (int g = 0; g < groups; ++g)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint2 one = sums[g * digits + d + j];
          s[j].x += one.x;
          s[j].y += one.y;
        }
    const uint32_t lower = block_before(s[0].x + s[1].x, room);
    if (group == 0) {
      base[d] = lower + s[0].y;
      base[d + 1] = lower + s[0].x + s[1].y;
    }
    // (block_before has a barrier behind the reads of sums)
  }
  const int64_t lo = (int64_t)blockIdx.x * per, hi = lo + per < count ? lo + per : count;
  // A round: each wave has R times 64 keys side by side, in order.
  for (int64_t at = lo; at < hi; at += kSortThreads * R) {
    for (int d = threadIdx.x; d < kSortWaves * digits / 2; d += kSortThreads) reinterpret_cast<uint32_t*>(seen)[d] = 0;
    uint32_t key[R], pos[R], rank[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t i = at + wave * (64 * R) + r * 64 + lane;
      in.get(i < hi ? i : hi - 1, key[r], pos[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool live = at + wave * (64 * R) + r * 64 + lane < hi;
      const uint32_t d = (key[r] >> shift) & mask;
      const uint64_t same = same_digit(d, bits, live);
      const uint32_t before = __popcll(same & ((1ull << lane) - 1));
      if (live) rank[r] = mine[d] + before;
      wave_fence();
      if (live && before == 0) mine[d] += (uint16_t)__popcll(same);
      wave_fence();
    }
    __syncthreads();
    // where each wave's keys of a digit begin
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
      uint32_t n[kSortWaves], next = 0;
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) n[w] = seen[w * digits + d];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        seen[w * digits + d] = (uint16_t)next;
        next += n[w];
      }
      seen[d] = (uint16_t)next;  // (wave 0 begins at 0 anyway: in its place how far base moves on behind this round)
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (at + wave * (64 * R) + r * 64 + lane < hi) {
        const uint32_t d = (key[r] >> shift) & mask;
        const uint32_t to = base[d] + (wave ? mine[d] : 0) + rank[r];
        key_out[to] = key[r];
        pos_out[to] = pos[r];
      }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) base[d] += seen[d];
    __syncthreads();
  }
}

// Few tokens: each one's place is the number of smaller keys and of equal ones before it.  A block has B tokens, and 1024 / B
// threads for each, which compare it with as many shares of all keys, read from LDS (4099 tokens 7.7 us; two passes over their
// digits by one block 19, by several in four launches 20).
template <int B>
__global__ __launch_bounds__(kSortThreads) void k_sort_few(SortKeys in, int count, uint32_t* __restrict__ key_out,
                                                           uint32_t* __restrict__ pos_out, int* __restrict__ error) {
  constexpr int kParts = kSortThreads / B;
  extern __shared__ uint4 keys4[];  // count keys, filled up with the largest number to a multiple of 4 kParts
  __shared__ uint32_t below[kParts][B];
  uint32_t* keys = reinterpret_cast<uint32_t*>(keys4);
  const int each = (count + 4 * kParts - 1) / (4 * kParts) * 4;  // of a share
  if (blockIdx.x == 0 && threadIdx.x == 0) *in.heavy_count = 0;
#pragma unroll 8
  for (int i = threadIdx.x; i < each * kParts; i += kSortThreads) {
    uint32_t k, p;
    in.get(i < count ? i : count - 1, k, p);
    keys[i] = i < count ? k : 0xffffffffu;
  }
  __syncthreads();
  const int t = threadIdx.x % B, part = threadIdx.x / B, i = blockIdx.x * B + t;
  const uint32_t mine = keys[i < count ? i : count - 1];
  // keys before the block's tokens count up to equality, those behind only below it; beside them places decide
  const int first = blockIdx.x * B, lo = part * each, hi = lo + each;
  const int mid = first < lo ? lo : first < hi ? first : hi, end = first + B < lo ? lo : first + B < hi ? first + B : hi;
  uint32_t n = 0;
  auto all = [&](int from, int to, uint32_t limit) {
#pragma unroll 4
    for (int j = from; j < to; j += 4) {
      const uint4 k = keys4[j >> 2];
      n += (k.x < limit) + (k.y < limit) + (k.z < limit) + (k.w < limit);
    }
  };
  all(lo, mid, mine + 1);  // (keys are below 2^31)
  for (int j = mid; j < end; ++j) n += keys[j] < mine || (keys[j] == mine && j < i);
  all(end, hi, mine);
  below[part][t] = n;
  __syncthreads();
  if (threadIdx.x < B && i < count) {
    uint32_t to = 0;
#pragma unroll
    for (int q = 0; q < kParts; ++q) to += below[q][t];
    key_out[to] = mine;
    pos_out[to] = i;
    if (mine >= in.vocab && in.tokens[i] >= 0) *error = 1;
  }
}

// ---- sums over the sorted places -------------------------------------------------------------------
// A block takes the tokens that begin in its run of kSumRun sorted places.  One of at most kSumMost places is summed there and
// written; a heavier one is summed run by run, and k_embed_join adds the runs' shares up: part[run][1] of the run that it begins in
// (its places in that run), part[run][0] of the others, float32, rows of part_pitch(cols); its first run is put on the list `heavy`
// (whose order does not matter).  Waves take a token and 64 V columns at a time; `split` blocks share a run.  `zero_blocks` more
// write zeros, spread among the others, so that both kinds are under way at any time.
//
// Measured on 32768 places x 2048 bfloat16 into 64000 rows of float32: zeros through the caches leave 256 MB behind that the sums then
// wait for (171 us in all, past them 157), dy through them 157 (past them 151; only where its rows lie at sixteen bytes: neighbours
// share lines otherwise, 4099 x 1111 float32 14 us and past them 17), more blocks than 4096 or sixteen waves a block 166 to 169.
__host__ __device__ constexpr int64_t part_pitch(int64_t cols) { return (cols + 3) / 4 * 4; }  // rows at sixteen bytes
constexpr int kSumRun = 32, kSumMost = 32, kSumWaves = 8;

// A heavy token: the run that it begins in, the first one without a share of it, itself.
struct HeavyToken {
  uint32_t run, stop, token;
};

// What run `lo / kSumRun` has to do, the same in every lane.
struct RunItems {
  uint32_t starts;  // bit e: a token begins at place lo + e
  int live;         // places of the run that hold a token
  bool heavy;       // the run begins inside a heavy token
};

__device__ __forceinline__ RunItems run_items(const uint32_t* key, int64_t count, uint32_t vocab, int64_t lo, uint32_t& my_key) {
  const int lane = threadIdx.x & 63;
  // (a lane beyond the run has the places after it)
  my_key = lo + lane < count ? key[lo + lane] : 0xffffffffu;
  const uint32_t prev = lo + lane > 0 && lo + lane - 1 < count ? key[lo + lane - 1] : 0xffffffffu;
  const uint32_t back = lo - 1 - lane >= 0 ? key[lo - 1 - lane] : 0xffffffffu;
  RunItems it;
  const uint64_t live = __ballot(lane < kSumRun && my_key < vocab);
  it.live = __popcll(live);
  it.starts = (uint32_t)__ballot(lane < kSumRun && my_key < vocab && my_key != prev);
  const uint32_t first = __builtin_amdgcn_readfirstlane(my_key);
  // places of the first token from here on, and before, up to 64 each
  const int on = __popcll(__ballot(my_key == first)), before = __popcll(__ballot(back == first));
  it.heavy = it.live > 0 && !(it.starts & 1) && on + before > kSumMost;
  return it;
}

// dtable's row `v`, columns from c on: scale times the sums, added or not.
template <class TG, int V>
__device__ __forceinline__ void put_sums(TG* row, int64_t c, int64_t cols, const float (&s)[V], float scale, bool add,
                                         const Some<TG, V>& old) {
  Some<TG, V> o;
#pragma unroll
  for (int j = 0; j < V; ++j) o.e[j] = static_cast<TG>(add ? static_cast<float>(old.e[j]) + s[j] * scale : s[j] * scale);
  if (c + V <= cols) {
    o.store(row + c);
  } else {  // (o's elements are those of the row's last V columns)
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (cols - V + j >= c) row[cols - V + j] = o.e[j];
  }
}

template <class TD, class TG, int V, bool ONCE>  // ONCE: rows of dy lie at 16-byte boundaries and go past the caches
__global__ __launch_bounds__(kSumWaves * 64) void k_embed_sum(const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                                              int64_t count, uint32_t vocab, const TD* __restrict__ dy,
                                                              int64_t dy_stride, int64_t cols, float scale, TG* __restrict__ dtable,
                                                              int64_t grad_stride, int add, float* __restrict__ part, int64_t runs,
                                                              int split, int tiles, HeavyToken* __restrict__ heavy,
                                                              uint32_t* __restrict__ heavy_count, int zero_blocks,
                                                              ZeroRows zero) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int mine = blockIdx.x;
  if (zero_blocks > 0) {
    // zero_blocks of all blocks, evenly: those where the share of the blocks up to here passes a whole number
    const int turn = (int)((uint64_t)blockIdx.x * zero_blocks / gridDim.x);
    if ((int)((uint64_t)(blockIdx.x + 1) * zero_blocks / gridDim.x) > turn) {
      zero_rows(zero, (int64_t)turn * kSumWaves + wave, (int64_t)zero_blocks * kSumWaves);
      return;
    }
    mine -= turn;
  }
  const int share = mine % split;
  const int64_t step = (gridDim.x - zero_blocks) / split;
  for (int64_t run = mine / split; run < runs; run += step) {
    const int64_t lo = run * kSumRun;
    uint32_t my_key;
    const RunItems it = run_items(key, count, vocab, lo, my_key);
    if (it.live == 0) return;  // (nor have the runs behind it)
    // the run's places, and those behind that its last token may have (it begins at most 31 places on and has at most 32)
    const uint32_t my_pos = pos[lo + lane < count ? lo + lane : count - 1];
    const int items = __popc(it.starts) + it.heavy;
    for (int w = share * kSumWaves + wave; w < items * tiles; w += kSumWaves * split) {
      const int item = w / tiles, tile = w % tiles;
      int e0, e1;         // places lo + e0 .. lo + e1 - 1
      int slot = -1;      // of part, or the table itself
      if (it.heavy && item == 0) {
        e0 = 0;
        e1 = it.starts ? __ffs(it.starts) - 1 : it.live;
        slot = 0;
      } else {
        uint32_t m = it.starts;
        for (int j = it.heavy; j < item; ++j) m &= m - 1;
        e0 = __ffs(m) - 1;
        m &= m - 1;
        if (m) {
          e1 = __ffs(m) - 1;
        } else {
          // the run's last token: how far it goes on
          const uint32_t k = __builtin_amdgcn_readlane(my_key, e0);
          const int n = __popcll(__ballot(my_key == k));
          e1 = e0 + n;
          if (n > kSumMost) {
            e1 = it.live;
            slot = 1;
            if (tile == 0) {
              // the first place with another token: 64 places are looked at at a time, ever closer ones
              int64_t a = lo + kSumRun, b = count;
              while (a < b) {
                const int64_t apart = (b - a + 63) / 64, look = a + lane * apart;
                const int same = __popcll(__ballot(look < b && key[look < b ? look : a] == k));
                if (same == 0) break;
                b = a + same * apart < b ? a + same * apart : b;
                a += (same - 1) * apart + 1;
              }
              if (lane == 0)
                heavy[atomicAdd(heavy_count, 1u)] = {(uint32_t)run, (uint32_t)((a + kSumRun - 1) / kSumRun), k};
            }
          }
        }
      }
      const uint32_t tok = __builtin_amdgcn_readlane(my_key, e0);
      const int64_t c = ((int64_t)tile * 64 + lane) * V;
      const int64_t from = c + V <= cols ? c : cols - V;  // (behind the row's end its last elements)
      TG* row = dtable + (int64_t)tok * grad_stride;
      Some<TG, V> old;
      if (add && slot < 0) old.load(row + from);
      float s[V];
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] = 0.0f;
      // sixteen rows under way at a time; of those left over up to eight, four, two and one, so 15 take four rounds of loads
      int e = e0;
      auto rows = [&](auto N, bool all) {
        Some<TD, V> in[N()];
#pragma unroll
        for (int i = 0; i < N(); ++i) {
          const uint32_t p = __builtin_amdgcn_readlane(my_pos, all || e + i < e1 ? e + i : e1 - 1);
          const TD* at = dy + (int64_t)p * dy_stride + from;
          in[i].template load<ONCE>(at);
        }
#pragma unroll
        for (int i = 0; i < N(); ++i)
          if (all || e + i < e1) {
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] += static_cast<float>(in[i].e[j]);
          }
        e += N();
      };
      while (e1 - e >= 16) rows(std::integral_constant<int, 16>(), true);
      if (e1 - e > 4) rows(std::integral_constant<int, 8>(), false);
      if (e1 - e > 2) rows(std::integral_constant<int, 4>(), false);
      if (e1 - e > 1) rows(std::integral_constant<int, 2>(), true);
      if (e1 - e > 0) rows(std::integral_constant<int, 1>(), true);
      if (c < cols && slot < 0) {
        put_sums<TG, V>(row, c, cols, s, scale, add, old);
      } else if (c < cols) {
        float* to = part + (run * 2 + slot) * part_pitch(cols);
        Some<float, V> one;
#pragma unroll
        for (int j = 0; j < V; ++j) one.e[j] = s[j];
        put_sums<float, V>(to, c, cols, s, 1.0f, false, one);
      }
    }
  }
}

// Heavy tokens from their list: blockIdx.y 256 columns, sixteen waves that take every sixteenth share.  Clears the marks, too.
template <class TG>
__global__ __launch_bounds__(1024) void k_embed_join(const float* __restrict__ part, int64_t vocab, int64_t cols, float scale,
                                                     TG* __restrict__ dtable, int64_t grad_stride, int add,
                                                     const HeavyToken* __restrict__ heavy, const uint32_t* __restrict__ heavy_count,
                                                     uint8_t* __restrict__ marks) {
  __shared__ float room[16][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (marks && blockIdx.y == 0)
    for (int64_t v = (int64_t)blockIdx.x * 1024 + threadIdx.x; v < vocab; v += (int64_t)gridDim.x * 1024) marks[v] = 0;
  const uint32_t n = *heavy_count;
  for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
    const HeavyToken token = heavy[i];
    const int64_t run = token.run, stop = token.stop;  // runs run + 1 .. stop - 1 hold shares
    const int64_t c = (int64_t)blockIdx.y * 256 + lane * 4, pitch = part_pitch(cols);
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < cols) {
      if (wave == 0)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < cols) s[j] = part[(run * 2 + 1) * pitch + c + j];
      if (c + 4 <= cols) {
#pragma unroll 4
        for (int64_t r = run + 1 + wave; r < stop; r += 16) {
          Some<float, 4> v;
          v.load(part + (r * 2) * pitch + c);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[j] += v.e[j];
        }
      } else {
        for (int64_t r = run + 1 + wave; r < stop; r += 16)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c + j < cols) s[j] += part[(r * 2) * pitch + c + j];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) room[wave][lane * 4 + j] = s[j];
    __syncthreads();
    const int64_t mine_c = (int64_t)blockIdx.y * 256 + threadIdx.x;
    if (threadIdx.x < 256 && mine_c < cols) {
      float t = room[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < 16; ++w) t += room[w][threadIdx.x];
      TG* to = dtable + (int64_t)token.token * grad_stride + mine_c;
      *to = static_cast<TG>(add ? static_cast<float>(*to) + t * scale : t * scale);
    }
    __syncthreads();
  }
}

}  // namespace artopk
