// Embedding lookup and its gradient, for gfx950.
//
//   y[i] = scale table[token[i]]
//   dtable[v] = scale (sum over the places i with token[i] = v of dy[i])  (added to what is there, or in its place)
//
// Both are bound by memory.  The gradient's places are sorted by token first (a stable radix sort of the places), so that
// every row of the table is summed by one owner in the order of its places: no atomics, the same bits every time.
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

// V elements at any place of their type, as they lie.
template <class T, int V>
struct Some {
  T e[V];
  __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(e, p, sizeof(e)); }
  __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, e, sizeof(e)); }
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
        o.store(out + c[u]);
      } else {
        for (int64_t j = c[u]; j < cols; ++j) out[j] = static_cast<TY>(good ? static_cast<float>(row[j]) * scale : other);
      }
    }
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

__global__ __launch_bounds__(kSortThreads) void k_sort_count(SortKeys in, int64_t count, int64_t per, int shift, int bits,
                                                             uint32_t* __restrict__ counts, int* __restrict__ error) {
  __shared__ uint32_t hist[kSortDigits];
  const uint32_t mask = (1u << bits) - 1;
  for (int d = threadIdx.x; d <= (int)mask; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * per, hi = lo + per < count ? lo + per : count;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads) {
    uint32_t k, p;
    in.get(i, k, p);
    if (in.first && in.tokens[i] >= (int64_t)in.vocab) *error = 1;
    atomicAdd(&hist[(k >> shift) & mask], 1u);  // (whole numbers: the order does not matter)
  }
  __syncthreads();
  for (int d = threadIdx.x; d <= (int)mask; d += kSortThreads) counts[(size_t)blockIdx.x * (mask + 1) + d] = hist[d];
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
  for (int w = 0; w < wave; ++w) before += room[w];
  return before + s - v;
}

// Lanes of a wave see what the others wrote to LDS before.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(kSortThreads) void k_sort_place(SortKeys in, int64_t count, int64_t per, int shift, int bits,
                                                             const uint32_t* __restrict__ counts, int tiles,
                                                             uint32_t* __restrict__ key_out, uint32_t* __restrict__ pos_out) {
  __shared__ uint32_t base[kSortDigits];              // where the tile's next key of each digit goes
  __shared__ uint16_t seen[kSortWaves][kSortDigits];  // keys of each digit that a wave has in this round
  __shared__ uint32_t room[kSortWaves];
  const int digits = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t mask = digits - 1;
  {
    // two digits a thread, side by side, so that the sum over threads runs over the digits in order
    const int d = threadIdx.x * 2;
    uint32_t all[2] = {0, 0}, before[2] = {0, 0};
    for (int t = 0; t < tiles; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t n = d + j < digits ? counts[(size_t)t * digits + d + j] : 0;
        all[j] += n;
        if (t < (int)blockIdx.x) before[j] += n;
      }
    const uint32_t lower = block_before(all[0] + all[1], room);
    if (d < digits) base[d] = lower + before[0];
    if (d + 1 < digits) base[d + 1] = lower + all[0] + before[1];
  }
  const int64_t lo = (int64_t)blockIdx.x * per, hi = lo + per < count ? lo + per : count;
  // A round: each wave has four times 64 keys side by side, in order.
  for (int64_t at = lo; at < hi; at += kSortThreads * 4) {
    for (int d = threadIdx.x; d < kSortWaves * kSortDigits / 2; d += kSortThreads)
      if ((d * 2) % kSortDigits < digits) reinterpret_cast<uint32_t*>(seen)[d] = 0;
    __syncthreads();
    uint32_t key[4], pos[4], rank[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t i = at + wave * 256 + r * 64 + lane;
      const bool live = i < hi;
      in.get(live ? i : hi - 1, key[r], pos[r]);
      const uint32_t d = (key[r] >> shift) & mask;
      // lanes with the same digit
      uint64_t same = __ballot(live);
      for (int b = 0; b < bits; ++b) {
        const uint64_t one = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? one : ~one;
      }
      const uint32_t mine = __popcll(same & ((1ull << lane) - 1));
      if (live) rank[r] = seen[wave][d] + mine;
      wave_fence();
      if (live && mine == 0) seen[wave][d] += (uint16_t)__popcll(same);
      wave_fence();
    }
    __syncthreads();
    // where each wave's keys of a digit begin
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
      uint32_t next = 0;
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = seen[w][d];
        seen[w][d] = (uint16_t)next;
        next += n;
      }
      seen[0][d] = (uint16_t)next;  // (wave 0 begins at 0 anyway: in its place how far base moves on behind this round)
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t i = at + wave * 256 + r * 64 + lane;
      if (i < hi) {
        const uint32_t d = (key[r] >> shift) & mask;
        const uint32_t to = base[d] + (wave ? seen[wave][d] : 0) + rank[r];
        key_out[to] = key[r];
        pos_out[to] = pos[r];
      }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) base[d] += seen[0][d];
    __syncthreads();
  }
}

// ---- sums over the sorted places -------------------------------------------------------------------
// A wave takes kSumRun places side by side, and 64 V columns of their rows.  A token whose places all lie in the run is summed
// and written by it.  Of one that reaches beyond, the run's share goes to part[run][0] (it began before the run) or
// part[run][1] (it begins in it), float32, and k_embed_join adds the shares up, run by run.
constexpr int kSumRun = 32, kSumAhead = 8;

// dtable's row `v`, columns from c on: scale times the sums, added or not.
template <class TG, int V>
__device__ __forceinline__ void put_sums(TG* row, int64_t c, int64_t cols, const float (&s)[V], float scale, bool add) {
  Some<TG, V> o;
  if (c + V <= cols) {
    if (add) o.load(row + c);
#pragma unroll
    for (int j = 0; j < V; ++j) o.e[j] = static_cast<TG>(add ? static_cast<float>(o.e[j]) + s[j] * scale : s[j] * scale);
    o.store(row + c);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (c + j < cols) row[c + j] = static_cast<TG>(add ? static_cast<float>(row[c + j]) + s[j] * scale : s[j] * scale);
  }
}

template <int V>
__device__ __forceinline__ void put_part(float* row, int64_t c, int64_t cols, const float (&s)[V]) {
  if (c + V <= cols) {
    Some<float, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.e[j] = s[j];
    o.store(row + c);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (c + j < cols) row[c + j] = s[j];
  }
}

template <class TD, class TG, int V>
__global__ __launch_bounds__(256) void k_embed_sum(const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                                   int64_t count, uint32_t vocab, const TD* __restrict__ dy, int64_t dy_stride,
                                                   int64_t cols, float scale, TG* __restrict__ dtable, int64_t grad_stride,
                                                   int add, float* __restrict__ part, int64_t units, int64_t tiles) {
  const int lane = threadIdx.x & 63;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t run = unit / tiles, c = (unit % tiles * 64 + lane) * V;
    const int64_t from = c + V <= cols ? c : cols - V;  // behind the row's end its last elements, shifted into place below
    const int64_t lo = run * kSumRun;
    const int n = count - lo < kSumRun ? (int)(count - lo) : kSumRun;
    const uint32_t my_key = key[lo + (lane < n ? lane : n - 1)], my_pos = pos[lo + (lane < n ? lane : n - 1)];
    const uint32_t first = __builtin_amdgcn_readfirstlane(my_key);
    if (first >= vocab) continue;  // (nothing but places without a token from here on)
    const bool head = lo > 0 && key[lo - 1] == first;
    const uint32_t last = __shfl(my_key, n - 1, 64);
    const bool tail = lo + n < count && key[lo + n] == last;
    float s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.0f;
    uint32_t now = first;
    bool began = !head;  // whether the token being summed begins in this run
    for (int e0 = 0; e0 < n; e0 += kSumAhead) {
      Some<TD, V> in[kSumAhead];
#pragma unroll
      for (int e = 0; e < kSumAhead; ++e) {
        const uint32_t p = __builtin_amdgcn_readlane(my_pos, e0 + e < n ? e0 + e : n - 1);
        in[e].load(dy + (int64_t)p * dy_stride + from);
      }
#pragma unroll
      for (int e = 0; e < kSumAhead; ++e) {
        if (e0 + e >= n) break;
        const uint32_t k = __builtin_amdgcn_readlane(my_key, e0 + e);
        if (k != now) {
          if (began)
            put_sums<TG, V>(dtable + (int64_t)now * grad_stride, c, cols, s, scale, add);
          else
            put_part<V>(part + (run * 2) * cols, c, cols, s);
          began = true;
          now = k;
#pragma unroll
          for (int j = 0; j < V; ++j) s[j] = 0.0f;
          if (k >= vocab) break;
        }
        if (c + V <= cols) {
#pragma unroll
          for (int j = 0; j < V; ++j) s[j] += static_cast<float>(in[e].e[j]);
        } else {
          // (the loaded piece begins at `from`: element j of ours is element c - from + j of it)
#pragma unroll
          for (int j = 0; j < V; ++j)
#pragma unroll
            for (int q = 0; q < V; ++q)
              if (c + j < cols && c - from + j == q) s[j] += static_cast<float>(in[e].e[q]);
        }
      }
      if (now >= vocab) break;
    }
    if (now >= vocab) continue;
    if (!began)
      put_part<V>(part + (run * 2) * cols, c, cols, s);
    else if (tail)
      put_part<V>(part + (run * 2 + 1) * cols, c, cols, s);
    else
      put_sums<TG, V>(dtable + (int64_t)now * grad_stride, c, cols, s, scale, add);
  }
}

// Tokens that reach over several runs, each by the block of the run that it begins in: blockIdx.x the run, blockIdx.y 64
// columns, sixteen waves that take every sixteenth share.
template <class TG>
__global__ __launch_bounds__(1024) void k_embed_join(const uint32_t* __restrict__ key, int64_t count, uint32_t vocab,
                                                     const float* __restrict__ part, int64_t cols, float scale,
                                                     TG* __restrict__ dtable, int64_t grad_stride, int add, int64_t runs) {
  __shared__ float room[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t run = blockIdx.x; run < runs; run += gridDim.x) {
    const int64_t end = (run + 1) * kSumRun;
    if (end >= count) return;
    const uint32_t k = key[end - 1];
    if (k >= vocab) return;
    if (key[end] != k) continue;
    if (key[run * kSumRun] == k && run > 0 && key[run * kSumRun - 1] == k) continue;  // it began before
    // the first place behind `end` with another token
    int64_t a = end, b = count;
    while (a < b) {
      const int64_t m = (a + b) >> 1;
      if (key[m] == k) a = m + 1; else b = m;
    }
    const int64_t stop = (a + kSumRun - 1) / kSumRun;  // runs run + 1 .. stop - 1 hold shares
    const int64_t c = (int64_t)blockIdx.y * 64 + lane;
    float s = 0.0f;
    if (c < cols) {
      if (wave == 0) s = part[(run * 2 + 1) * cols + c];
#pragma unroll 8
      for (int64_t r = run + 1 + wave; r < stop; r += 16) s += part[(r * 2) * cols + c];
    }
    room[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
      for (int w = 1; w < 16; ++w) s += room[w][lane];
      const float one[1] = {s};
      put_sums<TG, 1>(dtable + (int64_t)k * grad_stride, c, cols, one, scale, add);
    }
    __syncthreads();
  }
}

// Rows of zeros.
template <class TG>
__global__ __launch_bounds__(256) void k_embed_zero(TG* __restrict__ dtable, int64_t grad_stride, int64_t rows, int64_t cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < cols; c += 256) dtable[r * grad_stride + c] = static_cast<TG>(0.0f);
}

}  // namespace artopk
