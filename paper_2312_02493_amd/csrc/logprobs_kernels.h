// Log probabilities of given tokens, with entropy and top alternatives, and their gradient, for gfx950.
//
//   peak = max x,  logsum = log(sum e^(scale (x - peak))),  log p = scale (x - peak) - logsum,  logp = log p[token],
//   entropy = -sum p log p,  lse = scale peak + logsum
//   dx = scale (dlogp (delta - p) + dlse p - dentropy p (log p + entropy))
//
// Both are bound by memory: forward reads a row once, backward reads and writes it once.  Two numbers of a row are kept for the
// backward pass, not lse alone: beside a large peak (a row that is masked with the type's lowest value) lse would hold nothing of
// logsum.  Exponentials are powers of two of c (x - ..), c = scale log2(e).  The largest element stays out of the sum
// r = sum over the others of 2^(c (x - peak)): then log(1 + r) loses nothing where one token is nearly sure, as it would beside
// the largest element's own 1.
//
// Forward has to stay below some twelve instruction slots an element (64 lanes a cycle and compute unit, an exponential takes
// four) to be bound by memory in 16-bit types.  A wave keeps one largest element for all its lanes: 16 elements a lane at a time are
// added with nothing but their own maximum besides, and only where some lane has a larger one (once, then ever more rarely)
// the sums move to it: 10.1 slots, counted in the compiled loop (11.1 in rows far from zero, which are scaled by differences).
#pragma once

#include "embedding_kernels.h"
#include "lanes.h"

namespace artopk {

constexpr int kMostTop = 64;
constexpr int kGroupTop = 32;    // alternatives, at most, that are bounded by groups of four threads
// Candidates for a row's alternatives that are held on chip.  In a row of equal elements (or one with fewer than `top` others left) the
// bound is an element of the last of `top` keys' pieces, so all before it are candidates, and the larger ones: up to 128 pieces of 8
// and 64 more with four waves, 56 pieces with one.
constexpr int kListRoom = 128 * 8 + 64, kWaveRoom = 56 * 8 + 64;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float pow2(float v) { return __builtin_amdgcn_exp2f(v); }  // (0 below the normal range)

// Whole numbers in the order of the floats; -0 counts as +0.
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t b = __float_as_uint(f + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// The largest element m, r = sum over the others of 2^(c (x - m)), u = the same sum with each term times its exponent.
struct RowSum {
  float m, r, u;
};

__device__ __forceinline__ RowSum join(const RowSum& a, const RowSum& b, float c) {
  const bool first = a.m >= b.m;
  const RowSum &hi = first ? a : b, &lo = first ? b : a;
  const float d = fminf((hi.m - lo.m) * c, 200.0f);  // (2^-200 is 0; also where one or both have no element above -inf)
  const float f = pow2(-d), more = lo.r + 1.0f;
  return {hi.m, hi.r + more * f, hi.u + (lo.u - more * d) * f};
}

// The largest of N values; NaN counts for nothing.
template <int N>
__device__ __forceinline__ float largest(const float* x) {
  float m = x[0];
  if constexpr (N % 2 == 0) m = fmaxf(x[0], x[1]);
#pragma unroll
  for (int i = N % 2 == 0 ? 2 : 1; i < N; i += 2) m = fmaxf(fmaxf(x[i], x[i + 1]), m);
  return m;
}

__device__ __forceinline__ float wave_largest(float v) {
  return over_wave(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_total(float v) {
  return over_wave(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ uint64_t larger(uint64_t a, uint64_t b) { return a > b ? a : b; }

// A wave's share of a row: m is the largest element so far, the same in all lanes, r and u a lane's sums over its other ones
// with exponents c x - ref.  ref is c m rounded (the same for all, so it costs nothing but its distance from c m in the end).  That
// distance is half a step of float32 at c m: at most 1/2 below kNear, but it grows with c m, and from 2^31 on two to its power is
// no float32 any more.  So from kNear on exponents are c (x - m), one more operation an element.
struct Gather {
  static constexpr float kNear = 0x1p24f;
  float m = -INFINITY, ref = 0.0f, r = 0.0f, u = 0.0f;
  bool far = false;
  // c m less what exponents are relative to, exact
  __device__ __forceinline__ float apart(float c) const { return far ? 0.0f : fmaf(m, c, -ref); }
  __device__ __forceinline__ float exponent(float x, float c) const { return far ? (x - m) * c : fmaf(x, c, -ref); }
  // N elements a lane, `top` their largest; all lanes of the wave call it together
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], float top, float c) {
    if (__any(top > m)) {
      move(x, top, c);
    } else if (far) {
      sum<N>(x, [&](float v) { return (v - m) * c; });
    } else {
      sum<N>(x, [&](float v) { return fmaf(v, c, -ref); });
    }
  }
  template <int N, class F>
  __device__ __forceinline__ void sum(const float (&x)[N], F&& f) {
    constexpr int S = N % 4 == 0 ? 4 : 1;  // sums side by side
    float a[S], b[S];
#pragma unroll
    for (int i = 0; i < S; ++i) a[i] = b[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = f(x[i]), e = pow2(d);  // (NaN stays NaN and ends up in r)
      a[i % S] += e;
      b[i % S] = fmaf(e, fmaxf(d, -200.0f), b[i % S]);
    }
#pragma unroll
    for (int i = 1; i < S; ++i) {
      a[0] += a[i];
      b[0] += b[i];
    }
    r += a[0];
    u += b[0];
  }
  // the same where some lane has a larger element: the first lane that has the largest leaves it out, and adds the one before
  template <int N>
  __device__ __forceinline__ void move(const float (&x)[N], float top, float c) {
    const float to = wave_largest(top), before = m, next = to * c;
    const int owner = __ffsll((unsigned long long)__ballot(top == to)) - 1;
    bool mine = (int)(threadIdx.x & 63) == owner;
    const bool was_far = far;
    const float step = next - ref, was_apart = apart(c);
    far = !(fabsf(next) < kNear);
    m = to;
    ref = next;
    if (before > -INFINITY) {
      const float d = fminf(far || was_far ? (to - before) * c + (was_apart - apart(c)) : step, 200.0f), f = pow2(-d);
      u = (u - r * d) * f;
      r *= f;
    }
    if (mine && before > -INFINITY) {
      const float d = fmaxf(exponent(before, c), -200.0f), e = pow2(d);
      r += e;
      u = fmaf(e, d, u);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool out = mine && x[i] == to;
      mine = mine && !out;
      const float d = exponent(x[i], c), e = out ? 0.0f : pow2(d);
      r += e;
      u = fmaf(e, fmaxf(d, -200.0f), u);
    }
  }
  // over the wave
  __device__ __forceinline__ RowSum total(float c) const {
    if (!(m > -INFINITY)) return {m, wave_total(r), 0.0f};  // (r may be NaN)
    const float d = apart(c), f = pow2(-d);
    return {m, wave_total(r * f), wave_total((u - r * d) * f)};
  }
};

// A row in pieces of sixteen bytes from its first element on, wherever that lies.  The last one may be part of one: it is read as
// the row's last V elements, of which those that belong to the piece before it count as -infinity.
template <class T>
struct RowRun {
  static constexpr int V = 16 / sizeof(T);
  const T* row;
  int cols, count;
  __device__ __forceinline__ RowRun(const T* r, int c) : row(r), cols(c), count((int)(((int64_t)c + V - 1) / V)) {}
  // (a row shorter than a piece is read element by element)
  __device__ __forceinline__ int64_t begin(int j) const {
    const int64_t at = (int64_t)j * V;
    return cols < V ? 0 : at + V <= cols ? at : cols - V;
  }
  // of rows of V elements or more; ONCE: nothing reads it again, so past the caches (16384 x 64000 bfloat16 355 us, so 337)
  template <bool ONCE>
  __device__ __forceinline__ void ask(Some<T, V>& raw, int j, bool whole) const {
    raw.template load<ONCE>(row + (whole ? (int64_t)j * V : begin(j)));
  }
  // `all`: the piece is there and whole
  __device__ __forceinline__ void take(float* x, const Some<T, V>& raw, int j, bool all) const {
    const int skip = all ? 0 : (int)((int64_t)j * V - begin(j));
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = all || (j < count && k >= skip) ? static_cast<float>(raw.e[k]) : -INFINITY;
  }
  __device__ __forceinline__ void take_short(float* x, bool there) const {
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = there && k < cols ? static_cast<float>(row[k]) : -INFINITY;
  }
};

// A row in pieces of sixteen bytes that begin at aligned places; the first and the last may be part of one.  Piece j holds the
// elements from V j - shift on.
template <class T>
struct RowPieces {
  static constexpr int V = 16 / sizeof(T);
  const T* row;
  int cols, shift, count, whole0, whole1;  // pieces whole0 .. whole1 - 1 are whole
  __device__ __forceinline__ RowPieces(const T* r, int c) : row(r), cols(c) {
    shift = (int)((reinterpret_cast<uintptr_t>(r) & 15) / sizeof(T));
    count = (int)(((int64_t)cols + shift + V - 1) / V);
    whole0 = shift ? 1 : 0;
    whole1 = (int)(((int64_t)cols + shift) / V);
    if (whole1 < whole0) whole1 = whole0;
  }
  __device__ __forceinline__ void load_whole(float (&x)[V], int j) const { load_elems<V>(x, row + ((int64_t)j * V - shift)); }
  // a piece of which there is only a part, `other` in the places outside the row
  __device__ __forceinline__ void load_part(float (&x)[V], int j, float other) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t e = (int64_t)j * V - shift + i;
      x[i] = e >= 0 && e < cols ? static_cast<float>(row[e]) : other;
    }
  }
  __device__ __forceinline__ bool is_whole(int j) const { return j >= whole0 && j < whole1; }
};

struct LogpOut {
  float *logp, *peak, *logsum, *entropy;
  int32_t* top_ids;
  float* top_logp;
};

// What a row's outputs come from, once its sums are known.
struct RowEnd {
  RowSum s;
  float scale, log;
  bool broken, none;  // NaN or infinity in the row; nothing left in it
  __device__ __forceinline__ RowEnd(const RowSum& sum, float by) : s(sum), scale(by) {
    broken = s.r != s.r || s.m == INFINITY;
    none = s.m == -INFINITY;
    log = log1pf(s.r);
  }
  __device__ __forceinline__ float logp(float x) const {
    const float apart = x - s.m;  // (or beyond float32, where its product with scale may not be)
    const float d = apart == -INFINITY && x > -INFINITY ? x * scale - s.m * scale : apart * scale;
    return broken ? __builtin_nanf("") : none ? -INFINITY : d - log;
  }
  __device__ __forceinline__ void put(const LogpOut& out, int64_t row, int64_t tok, int cols, float xt) const {
    const float nan = __builtin_nanf("");
    if (out.peak) out.peak[row] = broken ? nan : s.m;
    if (out.logsum) out.logsum[row] = broken ? nan : log;
    if (out.entropy) out.entropy[row] = broken ? nan : none ? 0.0f : log - s.u * kLn2 / (1.0f + s.r);
    if (out.logp) out.logp[row] = tok >= cols ? nan : tok < 0 ? (broken ? nan : 0.0f) : logp(xt);
  }
  // one of the alternatives; its key is its value's order and the complement of its place
  __device__ __forceinline__ void put_top(const LogpOut& out, int64_t at, uint64_t key) const {
    out.top_ids[at] = broken ? -1 : (int32_t)~(uint32_t)key;
    out.top_logp[at] = logp(from_ordered((uint32_t)(key >> 32)));
  }
};

// A team of WAVES waves (4, or 1: four teams a block) has a row, or with `split` > 1 one of as many parts of it, whose sums and
// alternatives then go to parts and part_keys for k_logp_join.  Thread t has the part's pieces t, t + 64 WAVES, ..
//
// Alternatives.  Every thread notes its largest element (the first among equal ones), groups of threads the largest of theirs.  The
// `top`-th largest of these n keys is a bound: the row's alternatives are not below it, and all lie with the threads whose
// largest element reaches it (some 24 for 20).  So those threads' elements are read once more, those that reach the bound listed
// (n ln(n / (n - top)) of them in a row without an order), and a listed one's place is the number of larger ones.  n is 64 for up to
// kGroupTop alternatives; more are bounded by 128, of which a comparison costs more but leaves fewer (32768 x 8000 bfloat16, 64
// alternatives: 64 keys 632 us, 128 326).  Should there be more than there is room for, the alternatives are found one
// after the other.  Columns are at least V (k_logp_narrow has up to 256).
struct LogpPart {
  RowSum s;
  float unused;
};

template <class T, int WAVES, bool TOP>
__global__ __launch_bounds__(256) void k_logp(
    const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols, Tokens tokens, int has_tokens, float scale, float c, int top,
    LogpOut out, int split, LogpPart* __restrict__ parts, uint64_t* __restrict__ part_keys, int* __restrict__ error) {
  constexpr int V = RowPieces<T>::V, kTeams = 4 / WAVES, NT = 64 * WAVES, kBatch = 16 / V;
  using Full = std::integral_constant<int, kBatch>;
  using One = std::integral_constant<int, 1>;
  constexpr int kRoom = WAVES == 1 ? kWaveRoom : kListRoom;
  __shared__ RowSum sums[4];
  __shared__ uint64_t keys[TOP ? 256 : 1], lists[TOP ? kTeams * kRoom : 1], bests[4];
  __shared__ uint8_t chosens[TOP ? 256 : 1];
  __shared__ uint64_t bounds[kTeams];
  __shared__ int list_counts[kTeams], chosen_counts[kTeams];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int team = wave / WAVES, t = threadIdx.x % NT, team_wave = wave % WAVES;
  auto meet = [] {
    if constexpr (WAVES == 1) wave_fence(); else __syncthreads();
  };
  const int64_t units = rows * split;
  for (int64_t unit = (int64_t)blockIdx.x * kTeams + team; unit < units; unit += (int64_t)gridDim.x * kTeams) {
    const int64_t row = split == 1 ? unit : unit / split;
    const int part = split == 1 ? 0 : (int)(unit % split);
    const RowRun<T> p(x + row * x_stride, cols);
    const int q0 = split == 1 ? 0 : (int)((int64_t)p.count * part / split);
    const int q1 = split == 1 ? p.count : (int)((int64_t)p.count * (part + 1) / split);
    const int64_t tok = has_tokens && split == 1 ? tokens[row] : -1;
    const int group = WAVES == 1 ? 0 : top <= kGroupTop ? 2 : q1 - q0 >= NT ? 1 : 0;  // of so many threads' logarithm
    Gather g;
    // the thread's largest element, and the first piece that has it: to begin with its first piece
    float own = -INFINITY;
    int where = q0 + t < q1 ? q0 + t : -1;
    auto note = [&](float v, int j) {
      if (TOP && v > own) {
        own = v;
        where = j;
      }
    };
    auto batch = [&](auto pieces, int j, bool all) {  // pieces j, j + NT, ..; with `all` they are all there and whole
      constexpr int N = pieces();
      Some<T, V> raw[N];
#pragma unroll
      for (int i = 0; i < N; ++i) p.template ask<!TOP>(raw[i], all || j + i * NT < q1 ? j + i * NT : q1 - 1, all);
      __builtin_amdgcn_sched_barrier(0);  // (all loads go out before one is waited for)
      float v[N * V], most[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const bool there = all || j + i * NT < q1;
        p.take(v + i * V, raw[i], there ? j + i * NT : p.count, all);
        most[i] = largest<V>(v + i * V);
        if (there) note(most[i], j + i * NT);
      }
      g.add<N * V>(v, largest<N>(most), c);
    };
    // (the same for all lanes: full batches of whole pieces begin up to here)
    const int last = (q1 * (int64_t)V <= cols ? q1 : q1 - 1) - kBatch * NT;
    int j = q0 + t, base = q0;
    for (; base <= last; base += kBatch * NT, j += kBatch * NT) batch(Full(), j, true);
    for (; base + NT < q1; base += kBatch * NT, j += kBatch * NT) batch(Full(), j, false);
    if (base + team_wave * 64 < q1) batch(One(), j, false);
    // (read behind the row, of which it is a part, and needed behind the sums)
    const float xt = tok >= 0 && tok < cols ? static_cast<float>(p.row[tok]) : 0.0f;
    RowSum s = g.total(c);
    // a thread's key: its largest element, the lower place first; 0 where it has none
    const uint64_t own_key = where < 0 ? 0 : (uint64_t)ordered(own) << 32 | (uint32_t)~where;
    if (TOP) {
      uint64_t key = own_key;
      if (group >= 1) key = larger(key, moved<0xb1>(key, key));  // of the neighbour
      if (group == 2) key = larger(key, moved<0x4e>(key, key));  // of the other pair
      if ((t & ((1 << group) - 1)) == 0) keys[team * NT + (t >> group)] = key;
      if (t == 0) {
        list_counts[team] = chosen_counts[team] = 0;
        bounds[team] = 0;
      }
    }
    if constexpr (WAVES > 1) {
      if (lane == 0) sums[wave] = s;
      meet();
      s = sums[0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s = join(s, sums[w], c);
    } else if (TOP) {
      meet();
    }
    const RowEnd end(s, scale);
    if (t == 0) {
      if (split == 1) end.put(out, row, tok, cols, xt);
      else parts[unit].s = s;
      if (tok >= cols) *error = 1;
    }
    if constexpr (TOP) {
      auto put = [&](int at, uint64_t key) {
        if (split == 1) end.put_top(out, row * top + at, key);
        else part_keys[unit * top + at] = key;
      };
      uint64_t* list = lists + team * kRoom;
      uint8_t* chosen = chosens + team * NT;
      const int some = group ? NT >> group : q1 - q0 < NT ? q1 - q0 : NT;  // keys
      if (team_wave * 64 < some) {  // the bound; 0 where there are fewer keys
        const uint64_t* all = keys + team * NT;
        const uint64_t key = all[t];
        int rank = 0;
        int i = 0;
        for (; i + 64 <= some; i += 64) {
#pragma unroll 16
          for (int k = 0; k < 64; ++k) rank += all[i + k] > key;
        }
        for (; i < some; i += 16) {  // (keys behind the last are 0)
#pragma unroll
          for (int k = 0; k < 16; ++k) rank += all[i + k] > key;
        }
        if (key != 0 && rank == top - 1) bounds[team] = key;
      }
      if (end.broken || split > 1)
        for (int i = t; i < top; i += NT) put(i, 0);  // (a part may have fewer elements)
      meet();
      const uint64_t least = bounds[team];
      const float least_value = from_ordered((uint32_t)(least >> 32));
      if (own_key && own_key >= least && !end.broken) chosen[atomicAdd(&chosen_counts[team], 1)] = (uint8_t)t;
      meet();
      const int count = chosen_counts[team], pieces = (q1 - q0 + NT - 1) / NT;  // of a thread
      // lanes side by side have a thread's pieces, and where these are few several threads'
      int lg = 6;
      while (lg > 0 && pieces << 1 <= 1 << lg) --lg;
      const int with = lane & ((1 << lg) - 1);
      auto each = [&](auto&& f) {
        for (int i = team_wave * (64 >> lg) + (lane >> lg); i < count; i += WAVES * (64 >> lg)) {
          for (int j = q0 + chosen[i] + with * NT; j < q1; j += NT << lg) {
            float v[V];
            Some<T, V> raw;
            p.template ask<false>(raw, j, false);
            p.take(v, raw, j, false);
            if (!(largest<V>(v) >= least_value) && least) continue;
            const int64_t begin = p.begin(j);
#pragma unroll
            for (int k = 0; k < V; ++k) {
              if (begin + k < (int64_t)j * V) continue;  // (the piece's before it)
              const uint64_t o = (uint64_t)ordered(v[k]) << 32;
              if ((o | (uint32_t)~j) >= least) f(o | (uint32_t)~(uint32_t)(begin + k));
            }
          }
        }
      };
      each([&](uint64_t k) {
        const int at = atomicAdd(&list_counts[team], 1);
        if (at < kRoom) list[at] = k;
      });
      meet();
      const int n = list_counts[team];
      if (n <= kRoom) {
        for (int i = t; i < n; i += NT) {
          const uint64_t k = list[i];
          int above = 0;
#pragma unroll 4
          for (int q = 0; q < n; ++q) above += list[q] > k;
          if (above < top) put(above, k);
        }
      } else {
        uint64_t bound = ~0ull;
        for (int a = 0; a < top; ++a) {
          uint64_t b = 0;
          each([&](uint64_t k) { b = k < bound && k > b ? k : b; });
          b = wave_max(b);
          if (lane == 0) bests[wave] = b;
          meet();
          bound = 0;
          for (int i = 0; i < WAVES; ++i) bound = bests[team * WAVES + i] > bound ? bests[team * WAVES + i] : bound;
          if (t == 0 && bound) put(a, bound);
          meet();
        }
      }
    }
    meet();  // read before the next row's
  }
}

// Narrow rows: sixteen lanes have a row, each of them N of its pieces, which stay in registers.  All elements equal to the largest
// are counted, one of them stays out of the sum.  Alternatives are found one after the other.  What bounds it is a row's own
// instructions, reductions and ends, which four rows share: 32768 x 130 bfloat16 9.1 us (a wave a row 26.4), 5 alternatives 17.9
// (53.2), 32768 x 512 float32 16.6 (27.7); 32768 x 1000 bfloat16 25.3 (28.1), x 1024 float32 31.6 (28.6).
template <class T, int N, bool TOP>
__global__ __launch_bounds__(256) void k_logp_narrow(const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols, Tokens tokens,
                                                     int has_tokens, float scale, float c, int top, LogpOut out,
                                                     int* __restrict__ error) {
  constexpr int V = RowRun<T>::V, E = N * V;
  const int lane = threadIdx.x & 15;
  for (int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); row < rows; row += (int64_t)gridDim.x * 16) {
    const RowRun<T> p(x + row * x_stride, cols);
    const int64_t tok = has_tokens ? tokens[row] : -1;
    float v[E];
    if (cols < V) {
#pragma unroll
      for (int i = 1; i < N; ++i) p.take_short(v + i * V, false);
      p.take_short(v, lane == 0);
    } else {
      Some<T, V> raw[N];
#pragma unroll
      for (int i = 0; i < N; ++i) p.template ask<true>(raw[i], lane + i * 16 < p.count ? lane + i * 16 : p.count - 1, false);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < N; ++i) p.take(v + i * V, raw[i], lane + i * 16, false);
    }
    const float xt = tok >= 0 && tok < cols ? static_cast<float>(p.row[tok]) : 0.0f;
    RowSum s;
    s.m = over_sixteen(largest<E>(v), [](float a, float b) { return fmaxf(a, b); });
    const float peak = s.m > -INFINITY ? s.m : 0.0f;
    float r[4] = {}, u[4] = {}, equal = 0.0f;  // (sums side by side)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = (v[e] - peak) * c;
      const bool same = v[e] == s.m;
      const float f = same ? 0.0f : pow2(d);  // (NaN stays NaN)
      r[e % 4] += f;
      u[e % 4] = fmaf(f, fmaxf(d, -200.0f), u[e % 4]);
      equal += same ? 1.0f : 0.0f;
    }
    auto plus = [](float a, float b) { return a + b; };
    s.r = over_sixteen((r[0] + r[1]) + (r[2] + r[3]), plus);
    s.u = over_sixteen((u[0] + u[1]) + (u[2] + u[3]), plus);
    if (s.m > -INFINITY) s.r += over_sixteen(equal, plus) - 1.0f;
    const RowEnd end(s, scale);
    if (lane == 0) {
      end.put(out, row, tok, cols, xt);
      if (tok >= cols) *error = 1;
    }
    if constexpr (TOP) {
      uint32_t o[E];  // 0: not there, or taken
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int j = lane + e / V * 16;
        const int64_t at = p.begin(j) + e % V;
        o[e] = j < p.count && at >= (int64_t)j * V && at < cols ? ordered(v[e]) : 0;
      }
      uint64_t kept = 0;
      for (int a = 0; a < top; ++a) {
        uint32_t most = o[0];
#pragma unroll
        for (int e = 1; e < E; ++e) most = o[e] > most ? o[e] : most;
        most = over_sixteen(most, [](uint32_t f, uint32_t g) { return f > g ? f : g; });
        int own = E;  // the lane's first one
#pragma unroll
        for (int e = E - 1; e >= 0; --e) own = o[e] == most ? e : own;
        const uint32_t at = own < E ? (uint32_t)p.begin(lane + own / V * 16) + own % V : 0xffffffffu;
        const uint32_t first = over_sixteen(at, [](uint32_t f, uint32_t g) { return f < g ? f : g; });
        if (at != first) own = E;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = e == own ? 0 : o[e];
        if ((a & 15) == lane) kept = (uint64_t)most << 32 | (uint32_t)~first;
        if ((a & 15) == 15 || a == top - 1) {
          if (lane <= (a & 15)) end.put_top(out, row * top + (a & ~15) + lane, kept);
        }
      }
    }
  }
}

// Parts of rows put together: sums by lane, alternatives from the parts' lists, which are in order, one after the other.  One wave
// works, the others help it to read the lists.
__global__ __launch_bounds__(1024) void k_logp_join(const LogpPart* __restrict__ parts, const uint64_t* __restrict__ part_keys, int split,
                                                  int64_t x_stride, const void* __restrict__ x, int type, int cols, Tokens tokens,
                                                  int has_tokens, float scale, float c, int top, LogpOut out,
                                                    int* __restrict__ error) {
  __shared__ uint64_t lists[64 * (kMostTop + 1)];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  // (a list ends with 0, below every key)
  for (int i = threadIdx.x; i < split * top; i += 1024)
    lists[i / top * (kMostTop + 1) + i % top] = part_keys[row * split * top + i];
  if (lane < split) lists[lane * (kMostTop + 1) + top] = 0;
  const bool live = lane < split;
  RowSum s = live ? parts[row * split + lane].s : RowSum{-INFINITY, 0.0f, 0.0f};
  int64_t tok = -1;
  float xt = 0.0f;
  if (lane == 0 && has_tokens) {
    tok = tokens[row];
    if (tok >= cols) *error = 1;
    if (tok >= 0 && tok < cols) {
      const int64_t at = row * x_stride + tok;
      xt = type == kTypeF32 ? static_cast<const float*>(x)[at]
           : type == kTypeBf16 ? static_cast<float>(static_cast<const __bf16*>(x)[at])
                               : static_cast<float>(static_cast<const _Float16*>(x)[at]);
    }
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
    s = join(s, RowSum{__shfl_xor(s.m, off, 64), __shfl_xor(s.r, off, 64), __shfl_xor(s.u, off, 64)}, c);
  const RowEnd end(s, scale);
  if (lane == 0) end.put(out, row, tok, cols, xt);
  const uint64_t* list = lists + (live ? lane : 0) * (kMostTop + 1);
  uint64_t head = live ? list[0] : 0, ahead = live && top ? list[1] : 0;
  int next = 2;
  uint64_t kept = 0;  // the lane's own alternative
  for (int a = 0; a < top; ++a) {
    // the upper halves (values) first: two lists' first values are rarely the same
    const uint32_t value = (uint32_t)(head >> 32), place = (uint32_t)head, top_value = wave_max(value);
    uint64_t who = __ballot(value == top_value);
    if (__popcll(who) > 1) {
      const uint32_t top_place = wave_max(value == top_value ? place : 0u);
      who = __ballot(value == top_value && place == top_place);
    }
    const uint64_t most = lane_value(head, __ffsll((unsigned long long)who) - 1);
    if (lane == a) kept = most;
    if (head == most && most) {
      head = ahead;
      ahead = next <= top ? list[next] : 0;
      ++next;
    }
  }
  if (lane < top) end.put_top(out, row * top + lane, kept);
}

struct LogpGrads {
  const float *peak, *logsum, *entropy, *dlogp, *dlse, *dentropy;  // rows each; dlogp, dlse, and entropy with dentropy may be NULL
};

// Four pieces of a row a thread: of one row a block (a row has `tiles` blocks), or for short rows of one row a wave or
// sixteen lanes (32768 x 130 bfloat16 a wave a row 27.5 us, so 15.1).  dx may be x itself: a thread reads its elements before it
// writes them.  It goes past the caches, which it would only fill (8192 x 128000 bfloat16 722 us, so 707); x is better left to them
// (2047 x 10007 float16 26 us past them, so 19).
template <class T, bool SAME, int LANES>  // SAME: dx's rows lie within sixteen bytes as x's do
__global__ __launch_bounds__(256) void k_logp_backward(const T* x, int64_t x_stride, int64_t rows, int cols, Tokens tokens,
                                                       int has_tokens, float scale, float c, LogpGrads in, T* dx,
                                                       int64_t dx_stride, int64_t units, int tiles, int* error) {
  constexpr int V = RowPieces<T>::V, kTeams = 256 / LANES;
  const int t = threadIdx.x % LANES;
  const int team = LANES == 256 ? 0 : LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / LANES;
  for (int64_t unit = (int64_t)blockIdx.x * kTeams + team; unit < units; unit += (int64_t)gridDim.x * kTeams) {
    const int64_t row = LANES < 256 ? unit : unit / tiles;
    const int tile = LANES < 256 ? 0 : (int)(unit % tiles);
    const RowPieces<T> p(x + row * x_stride, cols);
    T* out = dx + row * dx_stride;
    int64_t tok = has_tokens ? tokens[row] : -1;
    const float peak = in.peak[row], logsum = in.logsum[row], dent = in.dentropy ? in.dentropy[row] : 0.0f, h = in.dentropy ? in.entropy[row] : 0.0f;
    const float dlogp = in.dlogp && tok >= 0 ? in.dlogp[row] : 0.0f, dlse = in.dlse ? in.dlse[row] : 0.0f;
    if (tok >= cols && tile == 0 && t == 0) *error = 1;
    // grad = p (a + b d), d = log2 p
    const bool broken = peak != peak || tok >= cols, none = peak == -INFINITY;
    const float top = none ? 0.0f : peak, less = logsum * kLog2e;
    const float a = broken ? __builtin_nanf("") : none ? 0.0f : scale * (dlse - dlogp - dent * h);
    const float b = none ? 0.0f : -scale * dent * kLn2;
    const int tok_piece = tok >= 0 && tok < cols && !none && !broken ? (int)((tok + p.shift) / V) : -1;
    auto value = [&](float v) {
      const float d = fmaxf(fmaf(v - top, c, -less), -200.0f);
      return pow2(d) * fmaf(b, d, a);
    };
    auto piece = [&](float(&v)[V], int j) {
      float own = 0.0f;
      if (j == tok_piece) {  // at the token itself 1 - p, exact where p is close to 1
        const float d = fmaf(static_cast<float>(p.row[tok]) - peak, scale, -logsum), q = expf(d);
        own = scale * (dlse * q - dlogp * expm1f(d) - (q > 0.0f ? dent * (q * (d + h)) : 0.0f));
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = value(v[i]);
        if (j == tok_piece && (int64_t)j * V - p.shift + i == tok) v[i] = own;
      }
    };
    auto store_part = [&](const float(&v)[V], int j) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int64_t e = (int64_t)j * V - p.shift + i;
        if (e >= 0 && e < cols) out[e] = static_cast<T>(v[i]);
      }
    };
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = (tile * 4 + u) * LANES + t;
      if (j >= p.count) continue;
      float v[V];
      if (p.is_whole(j)) {
        p.load_whole(v, j);
        piece(v, j);
        T* to = out + ((int64_t)j * V - p.shift);
        Some<T, V> o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.e[i] = static_cast<T>(v[i]);
        o.template store<SAME>(to);
      } else {
        p.load_part(v, j, 0.0f);
        piece(v, j);
        store_part(v, j);
      }
    }
  }
}

}  // namespace artopk
