// Log probabilities of given tokens, with entropy and top alternatives, and their gradient, for gfx950.
//
//   peak = max x,  logsum = log(sum e^(scale (x - peak))),  log p = scale (x - peak) - logsum,  logp = log p[token],
//   entropy = -sum p log p,  lse = scale peak + logsum
//   dx = scale (dlogp (delta - p) + dlse p - dentropy p (log p + entropy))
//
// Both are bound by memory: forward reads a row once, backward reads and writes it once.  Two numbers of a row are kept for the
// backward pass, not lse alone: beside a large peak (a row that is masked with the type's lowest value) lse would hold nothing of
// logsum.  Exponentials are powers of two of c (x - ..), c = scale log2(e).  A thread's largest element M stays out of its sum
// R = sum over the others of 2^(c (x - M)): then log(1 + R) loses nothing where one token is nearly sure, as it would beside the
// largest element's own 1.  Exponents are taken relative to a reference that lies at most 16 below M's (sums stay below 2^50) and
// so rarely moves.
#pragma once

#include "embedding_kernels.h"

namespace artopk {

constexpr int kMostTop = 64;
constexpr int kListRoom = 1024;  // candidates for a row's alternatives that are held on chip
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

// A thread's share of a row, element by element.
struct Gather {
  float m = -INFINITY, r = 0.0f, u = 0.0f, ref = 0.0f, most = -INFINITY;
  bool bad = false;
  // V elements; with one of them NaN nothing but `bad` counts
  template <int V>
  __device__ __forceinline__ void add(float (&x)[V], float c) {
    if constexpr (V == 1) {
      bad |= x[0] != x[0];
      const float lo = fminf(x[0], m);
      m = fmaxf(x[0], m);
      x[0] = lo;
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        bad |= __builtin_isunordered(x[i], x[i + 1]);
        const float hi = fmaxf(fmaxf(x[i], x[i + 1]), m);
        const float mid = __builtin_amdgcn_fmed3f(x[i], x[i + 1], m), lo = fminf(fminf(x[i], x[i + 1]), m);
        m = hi;
        x[i] = mid;
        x[i + 1] = lo;
      }
    }
    if (m > most) {  // the reference moves (the first time from nothing)
      if (most > -INFINITY) {
        const float d = fminf((m - ref) * c, 200.0f), f = pow2(-d);
        u = (u - r * d) * f;
        r *= f;
      }
      ref = m;
      most = m + 16.0f / c;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = fmaxf((x[i] - ref) * c, -200.0f), e = pow2(d);
      r += e;
      u = fmaf(e, d, u);
    }
  }
  __device__ __forceinline__ RowSum sum(float c) const {
    if (!(m > -INFINITY)) return {-INFINITY, 0.0f, 0.0f};
    const float d = (m - ref) * c, f = pow2(-d);
    return {m, r * f, (u - r * d) * f};
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

// Thread t of a block of 256 has pieces whole0 + t + 256 i; thread 255 the part in front, thread 254 the part behind.  `i` runs
// to steps() - 1.
template <class T>
struct Share {
  const RowPieces<T>& p;
  __device__ __forceinline__ int steps() const { return (p.whole1 - p.whole0 + 255) / 256 + 2; }
  __device__ __forceinline__ int piece(int t, int i) const {  // -1: none
    const int n = steps();
    if (i == n - 2) return t == 255 && p.whole0 > 0 ? 0 : -1;
    if (i == n - 1) return t == 254 && p.count > p.whole1 ? p.count - 1 : -1;
    const int j = p.whole0 + t + 256 * i;
    return j < p.whole1 ? j : -1;
  }
};

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint64_t o = __shfl_xor(v, off, 64);
    v = o > v ? o : v;
  }
  return v;
}

// One row a block.
template <class T, bool TOP>
__global__ __launch_bounds__(256) void k_logp(const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols, Tokens tokens,
                                              int has_tokens, float scale, float c, int top, LogpOut out, int* __restrict__ error) {
  constexpr int V = RowPieces<T>::V;
  __shared__ RowSum sums[4];
  __shared__ int bads[4];
  __shared__ uint64_t keys[TOP ? 256 : 1], list[TOP ? kListRoom : 1], bound, best[4];
  __shared__ int chosen[TOP ? kMostTop : 1], chosen_count, list_count;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const RowPieces<T> p(x + row * x_stride, cols);
    const Share<T> share{p};
    int64_t tok = -1;
    float xt = 0.0f;
    if (t == 0 && has_tokens) {
      tok = tokens[row];
      if (tok >= cols) *error = 1;
      if (tok >= 0 && tok < cols) xt = static_cast<float>(p.row[tok]);
    }
    Gather g;
    int where = -1;  // the first piece with the thread's largest element
    auto piece = [&](float(&v)[V], int j) {
      const float before = g.m;
      g.add(v, c);
      if (TOP && (g.m > before || where < 0)) where = j;
    };
    if (t == 255 && p.whole0 > 0) {
      float v[V];
      p.load_part(v, 0, -INFINITY);
      piece(v, 0);
    }
    for (int j = p.whole0 + t; j < p.whole1; j += 256) {
      float v[V];
      p.load_whole(v, j);
      piece(v, j);
    }
    if (t == 254 && p.count > p.whole1) {
      float v[V];
      p.load_part(v, p.count - 1, -INFINITY);
      piece(v, p.count - 1);
    }
    RowSum s = g.sum(c);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s = join(s, RowSum{__shfl_xor(s.m, off, 64), __shfl_xor(s.r, off, 64), __shfl_xor(s.u, off, 64)}, c);
    const int bad = __any(g.bad);
    if (lane == 0) {
      sums[wave] = s;
      bads[wave] = bad;
    }
    if (TOP) {
      // a thread's key: its largest element, the lower place first; 0 where it has none
      keys[t] = where < 0 ? 0 : (uint64_t)ordered(g.m) << 32 | (uint32_t)~where;
      if (t == 0) {
        bound = 0;
        chosen_count = list_count = 0;
      }
    }
    __syncthreads();
    s = join(join(sums[0], sums[1], c), join(sums[2], sums[3], c), c);
    const bool broken = bads[0] | bads[1] | bads[2] | bads[3] || s.m == INFINITY;  // NaN or infinity in the row
    const bool none = s.m == -INFINITY;
    const float log = log1pf(s.r), nan = __builtin_nanf("");
    if (t == 0) {
      if (out.peak) out.peak[row] = broken ? nan : s.m;
      if (out.logsum) out.logsum[row] = broken ? nan : log;
      if (out.entropy) out.entropy[row] = broken ? nan : none ? 0.0f : log - s.u * kLn2 / (1.0f + s.r);
      if (out.logp)
        out.logp[row] = broken || tok >= cols ? nan : tok < 0 ? 0.0f : none ? -INFINITY : (xt - s.m) * scale - log;
    }
    if (TOP && broken) {
      if (t < top) {
        out.top_ids[row * top + t] = -1;
        out.top_logp[row * top + t] = nan;
      }
    } else if constexpr (TOP) {
      auto put = [&](int at, uint64_t key) {
        const float v = from_ordered((uint32_t)(key >> 32));
        out.top_ids[row * top + at] = (int32_t)~(uint32_t)key;
        out.top_logp[row * top + at] = none ? -INFINITY : (v - s.m) * scale - log;
      };
      // The row's alternatives are elements of the threads with the `top` largest keys, and not below the last of these.
      const uint64_t mine = keys[t];
      int rank = 0;
      for (int i = 0; i < 256; ++i) rank += keys[i] > mine;
      if (mine && rank < top) {
        chosen[atomicAdd(&chosen_count, 1)] = t;
        if (rank == top - 1) bound = mine;
      }
      __syncthreads();
      const uint64_t least = bound;
      const int steps = share.steps(), work = chosen_count * steps;
      auto each = [&](auto&& f) {
        for (int w = t; w < work; w += 256) {
          const int j = share.piece(chosen[w / steps], w % steps);
          if (j < 0) continue;
          float v[V];
          if (p.is_whole(j)) p.load_whole(v, j); else p.load_part(v, j, 0.0f);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int64_t e = (int64_t)j * V - p.shift + i;
            if (e < 0 || e >= cols) continue;
            const uint64_t o = (uint64_t)ordered(v[i]) << 32;
            if ((o | (uint32_t)~j) >= least) f(o | (uint32_t)~(uint32_t)e);
          }
        }
      };
      each([&](uint64_t key) {
        const int at = atomicAdd(&list_count, 1);
        if (at < kListRoom) list[at] = key;
      });
      __syncthreads();
      const int n = list_count;
      if (n <= kListRoom) {
        for (int i = t; i < n; i += 256) {
          const uint64_t key = list[i];
          int above = 0;
          for (int j = 0; j < n; ++j) above += list[j] > key;
          if (above < top) put(above, key);
        }
      } else {
        // too many candidates (a row in ascending order, say): one alternative after the other
        uint64_t last = ~0ull;
        for (int k = 0; k < top; ++k) {
          uint64_t b = 0;
          each([&](uint64_t key) { b = key < last && key > b ? key : b; });
          b = wave_max(b);
          if (lane == 0) best[wave] = b;
          __syncthreads();
          last = best[0];
          for (int i = 1; i < 4; ++i) last = best[i] > last ? best[i] : last;
          if (t == 0) put(k, last);
          __syncthreads();
        }
      }
    }
    __syncthreads();  // read before the next row's
  }
}

struct LogpGrads {
  const float *peak, *logsum, *entropy, *dlogp, *dlse, *dentropy;  // rows each; dlogp, dlse, and entropy with dentropy may be NULL
};

// 1024 pieces of a row a block.  dx may be x itself: a thread reads its elements before it writes them.
template <class T, bool SAME>  // SAME: dx's rows lie within sixteen bytes as x's do
__global__ __launch_bounds__(256) void k_logp_backward(const T* x, int64_t x_stride, int64_t rows, int cols, Tokens tokens,
                                                       int has_tokens, float scale, float c, LogpGrads in, T* dx,
                                                       int64_t dx_stride, int64_t units, int tiles, int* error) {
  constexpr int V = RowPieces<T>::V;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t row = unit / tiles;
    const int tile = (int)(unit % tiles);
    const RowPieces<T> p(x + row * x_stride, cols);
    T* out = dx + row * dx_stride;
    int64_t tok = has_tokens ? tokens[row] : -1;
    const float peak = in.peak[row], logsum = in.logsum[row], dent = in.dentropy ? in.dentropy[row] : 0.0f, h = in.dentropy ? in.entropy[row] : 0.0f;
    const float dlogp = in.dlogp && tok >= 0 ? in.dlogp[row] : 0.0f, dlse = in.dlse ? in.dlse[row] : 0.0f;
    if (tok >= cols && tile == 0 && threadIdx.x == 0) *error = 1;
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
      const int j = tile * 1024 + u * 256 + threadIdx.x;
      if (j >= p.count) continue;
      float v[V];
      if (p.is_whole(j)) {
        p.load_whole(v, j);
        piece(v, j);
        T* to = out + ((int64_t)j * V - p.shift);
        if constexpr (SAME) {
          store_elems<V>(to, v);
        } else {
          Some<T, V> o;
#pragma unroll
          for (int i = 0; i < V; ++i) o.e[i] = static_cast<T>(v[i]);
          o.store(to);
        }
      } else {
        p.load_part(v, j, 0.0f);
        piece(v, j);
        store_part(v, j);
      }
    }
  }
}

}  // namespace artopk
