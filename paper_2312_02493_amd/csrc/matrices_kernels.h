// Orthogonalised updates of matrices in a flat vector, for gfx950.
//
// Newton-Schulz steps on X, m x n with m <= n (a matrix with more rows than columns is taken as its transpose):
//   X_0 = G / (||G|| + eps),   A = X X^T,   Q = a I + b A + c A^2,   X <- Q X.
// A and Q are symmetric, so only their tiles on and below the diagonal are computed, and each is stored twice.
//
// Operands.  The products run on the matrix cores in float16 with float32 sums.  Entries of X are at most 2 in size,
// those of A at most 4, those of Q at most 15 (the host refuses coefficients that would pass these bounds), so each is
// stored times 2^12: 2^16 is never reached, and a matrix of 16384 x 16384 still has its first X's typical entry, 2^-14,
// at 2^-2, far above the smallest normal 2^-14.  bfloat16 would need no scale, but rounds eight times as coarsely, and
// the steps multiply small singular values, and what roundings put there, by up to a^5 = 485.  With one part an operand
// keeps 11 bits; with two (hi + lo, and hi hi + hi lo + lo hi for a product) 22, which leaves the result as exact as
// float32 products do.
//
// Layout.  All products have the form P Q^T with both operands' rows along the summed index: X X^T from X, A A^T from
// the symmetric A, and Q X = Q (X^T)^T from a second copy of X, transposed, which is written beside the first (a
// product writes 4 bytes for every 2 m operations on them).  Everything is padded with zeros to whole tiles, so that
// the products have no edges; only the final product, which writes the caller's buffer, knows the true sizes.
#pragma once

#include "elements.h"

namespace artopk {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kOperandScale = 4096.0f;  // 2^12, of every stored operand

// One matrix.  Places are in halves from the start of the iterates' memory; with two parts the low one follows the
// high one's mp * np (or mp * mp) halves.
struct MatDesc {
  int64_t at;           // first element in the flat vector
  int32_t m, n;         // the smaller and the larger of rows and columns
  int32_t mp, np;       // padded
  int32_t tall;         // the flat vector holds n rows of m
  float scale;
  int64_t x, xt[2], a, q;
  int32_t part, parts;  // its sums of squares
};

// A piece of the flat vector inside one matrix, or of none (mat < 0).
struct MatChunk {
  int64_t begin, end;
  int32_t mat, slot;  // slot: where its sum of squares goes
};

struct MatTile {
  uint32_t mat;
  uint16_t i, j;  // in tiles
};

// What the elements of a step are made of.
struct MuonArgs {
  float mu, scale;  // momentum <- mu momentum + scale update
  int32_t nesterov;
  float eta, decay_by, eta_rest;  // decay_by = 1 - eta decay
};

enum { kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2 };

__device__ __forceinline__ float muon_direction(const MuonArgs& a, float momentum, float update) {
  return a.nesterov ? fmaf(a.mu, momentum, a.scale * update) : momentum;
}

__device__ __forceinline__ double block_sum(double v, double* room) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = room[0];
  for (int i = 1; i < (int)blockDim.x / 64; ++i) s += room[i];
  __syncthreads();
  return s;
}

// Sums of squares of the matrices' pieces.
template <class T>
__global__ __launch_bounds__(256) void k_mat_squares(const T* __restrict__ x, const MatChunk* __restrict__ chunks,
                                                     double* __restrict__ sums) {
  __shared__ double room[4];
  const MatChunk c = chunks[blockIdx.x];
  if (c.mat < 0) return;
  double s = 0.0;
  for (int64_t i = c.begin + threadIdx.x; i < c.end; i += 256) {
    const double v = static_cast<double>(static_cast<float>(x[i]));
    s = fma(v, v, s);
  }
  s = block_sum(s, room);
  if (threadIdx.x == 0) sums[c.slot] = s;
}

// Momentum, the sums of squares of the direction v, and the weights of no matrix.
template <class T>
__global__ __launch_bounds__(256) void k_mat_momentum(T* __restrict__ w, float* __restrict__ momentum,
                                                      const float* __restrict__ update, MuonArgs a,
                                                      const MatChunk* __restrict__ chunks, double* __restrict__ sums) {
  __shared__ double room[4];
  const MatChunk c = chunks[blockIdx.x];
  double s = 0.0;
  for (int64_t i = c.begin + threadIdx.x; i < c.end; i += 256) {
    const float u = update[i];
    const float m = fmaf(a.mu, momentum[i], a.scale * u);
    momentum[i] = m;
    const float v = muon_direction(a, m, u);
    if (c.mat < 0) {
      if (a.eta_rest != 0.0f) w[i] = static_cast<T>(fmaf(-a.eta_rest, v, static_cast<float>(w[i])));
    } else {
      s = fma((double)v, (double)v, s);
    }
  }
  if (c.mat < 0) return;
  s = block_sum(s, room);
  if (threadIdx.x == 0) sums[c.slot] = s;
}

// 1 / (norm + eps) of a matrix, in every thread of a block of 256.
__device__ __forceinline__ float inverse_norm(const MatDesc& d, const double* sums, float eps, double* room) {
  double s = 0.0;
  for (int i = threadIdx.x; i < d.parts; i += 256) s += sums[d.part + i];
  s = block_sum(s, room);
  return static_cast<float>(1.0 / (sqrt(s) + (double)eps));
}

template <int PARTS>
__device__ __forceinline__ void split_half(float v, _Float16 (&out)[PARTS]) {
  out[0] = static_cast<_Float16>(v);
  if constexpr (PARTS == 2) out[1] = static_cast<_Float16>(v - static_cast<float>(out[0]));
}

// Where the flat vector's direction comes from: the vector itself, or momentum and update.
template <class T>
struct FromVector {
  const T* x;
  __device__ __forceinline__ float operator()(int64_t i) const { return static_cast<float>(x[i]); }
};
struct FromMomentum {
  const float* momentum;
  const float* update;
  MuonArgs a;
  __device__ __forceinline__ float operator()(int64_t i) const {
    return muon_direction(a, momentum[i], a.nesterov ? update[i] : 0.0f);
  }
};

// X_0 and its transpose, 64 x 64 elements a block, zeros beyond the true sizes.
template <int PARTS, class From>
__global__ __launch_bounds__(256) void k_mat_begin(From from, const MatDesc* __restrict__ mats,
                                                   const MatTile* __restrict__ tiles, const double* __restrict__ sums,
                                                   float eps, _Float16* __restrict__ mem) {
  __shared__ float tile[64][65];
  __shared__ double room[4];
  const MatTile t = tiles[blockIdx.x];
  const MatDesc d = mats[t.mat];
  const float by = inverse_norm(d, sums, eps, room);
  const int rows = d.tall ? d.n : d.m, cols = d.tall ? d.m : d.n;  // as they lie
  const int r0 = (d.tall ? t.j : t.i) * 64, c0 = (d.tall ? t.i : t.j) * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 4
  for (int r = wave; r < 64; r += 4) {
    float v = 0.0f;
    if (r0 + r < rows && c0 + lane < cols) v = from(d.at + (int64_t)(r0 + r) * cols + c0 + lane) * by * kOperandScale;
    if (d.tall)
      tile[lane][r] = v;
    else
      tile[r][lane] = v;
  }
  __syncthreads();
  // tile[i][j] = X's element (i0 + i, j0 + j)
  const int i0 = t.i * 64, j0 = t.j * 64;
  const int at = threadIdx.x >> 3, k = (threadIdx.x & 7) * 8;
#pragma unroll
  for (int half = 0; half < 64; half += 32) {
    const int r = at + half;
    _Float16 p[8][PARTS], q[8][PARTS];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      split_half<PARTS>(tile[r][k + e], p[e]);
      split_half<PARTS>(tile[k + e][r], q[e]);
    }
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
      half8 u, v;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = p[e][s];
        v[e] = q[e][s];
      }
      const int64_t plane = (int64_t)s * d.mp * d.np;
      *reinterpret_cast<half8*>(mem + d.x + plane + (int64_t)(i0 + r) * d.np + j0 + k) = u;
      *reinterpret_cast<half8*>(mem + d.xt[0] + plane + (int64_t)(j0 + r) * d.mp + i0 + k) = v;
    }
  }
}

// What the last product does with X's elements: out = scale X, or the weights' update.
struct FinishArgs {
  void* out;
  int32_t type, muon;
  MuonArgs a;
};

template <class T>
__device__ __forceinline__ void finish_as(T* p, const FinishArgs& f, float scaled) {
  *p = static_cast<T>(f.muon ? fmaf(-f.a.eta, scaled, static_cast<float>(*p) * f.a.decay_by) : scaled);
}

__device__ __forceinline__ void finish(const FinishArgs& f, int64_t i, float scaled) {
  if (f.type == kTypeF32)
    finish_as(static_cast<float*>(f.out) + i, f, scaled);
  else if (f.type == kTypeBf16)
    finish_as(static_cast<__bf16*>(f.out) + i, f, scaled);
  else
    finish_as(static_cast<_Float16*>(f.out) + i, f, scaled);
}

// No step at all: the scaled matrix itself.
template <class From>
__global__ __launch_bounds__(256) void k_mat_scaled(From from, const MatDesc* __restrict__ mats,
                                                    const MatChunk* __restrict__ chunks,
                                                    const double* __restrict__ sums, float eps, FinishArgs f) {
  __shared__ double room[4];
  const MatChunk c = chunks[blockIdx.x];
  if (c.mat < 0) return;
  const MatDesc d = mats[c.mat];
  const float by = inverse_norm(d, sums, eps, room);
  for (int64_t i = c.begin + threadIdx.x; i < c.end; i += 256) finish(f, i, from(i) * by * d.scale);
}

enum { kGram = 0, kSquare = 1, kApply = 2, kFinal = 3 };

// One tile of a product.  TILE x TILE elements, WM x WN waves.
template <int TILE>
struct ProductShape;
template <>
struct ProductShape<64> {
  static constexpr int kWM = 2, kWN = 2;
};
template <>
struct ProductShape<128> {
  static constexpr int kWM = 2, kWN = 2;
};
template <>
struct ProductShape<256> {
  static constexpr int kWM = 2, kWN = 4;
};
template <int TILE>
constexpr int product_threads() {
  return ProductShape<TILE>::kWM * ProductShape<TILE>::kWN * 64;
}
constexpr int product_depth(int parts) { return parts == 2 ? 32 : 64; }  // of the summed index, a stage
template <int TILE, int PARTS>
constexpr int product_lds() {
  return 2 * PARTS * 2 * TILE * product_depth(PARTS) * 2;  // two stages of both operands, bytes
}

template <int TILE, int PARTS, int MODE>
__global__ __launch_bounds__(product_threads<TILE>()) void k_mat_product(
    const MatDesc* __restrict__ mats, const MatTile* __restrict__ tiles, _Float16* __restrict__ mem, int from, float ca,
    float cb, float cc, FinishArgs f) {
  using S = ProductShape<TILE>;
  constexpr int THREADS = product_threads<TILE>();
  constexpr int BK = product_depth(PARTS);
  constexpr int CH = BK / 8;                 // 16-byte chunks of a row
  constexpr int FM = TILE / S::kWM / 32, FN = TILE / S::kWN / 32;
  constexpr int LOADS = TILE * CH / THREADS;  // chunks of one operand's part a thread brings
  __shared__ __align__(16) _Float16 lds[product_lds<TILE, PARTS>() / 2];
  constexpr int PLANE = TILE * BK;            // halves of one operand's part in a stage
  constexpr int STAGE = 2 * PARTS * PLANE;

  const MatTile t = tiles[blockIdx.x];
  const MatDesc& d = mats[t.mat];
  const bool swap = MODE == kFinal && d.tall;  // X^T wanted: its rows are X^T's, Q is symmetric
  const int64_t mm = (int64_t)d.mp * d.mp, mn = (int64_t)d.mp * d.np;
  const _Float16 *p, *q;
  int64_t p_plane, q_plane;
  int K;
  if constexpr (MODE == kGram) {
    p = q = mem + d.x;
    p_plane = q_plane = mn;
    K = d.np;
  } else if constexpr (MODE == kSquare) {
    p = q = mem + d.a;
    p_plane = q_plane = mm;
    K = d.mp;
  } else {
    p = mem + (swap ? d.xt[from] : d.q);
    q = mem + (swap ? d.q : d.xt[from]);
    p_plane = swap ? mn : mm;
    q_plane = swap ? mm : mn;
    K = d.mp;
  }
  const int i0 = t.i * TILE, j0 = t.j * TILE;
  p += (int64_t)i0 * K;
  q += (int64_t)j0 * K;

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wi = wave / S::kWN * (FM * 32), wj = wave % S::kWN * (FN * 32);

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  // chunk c of row r lies at place c ^ (r & 7) of the row (with 32 halves a row: of two rows), so that the rows a wave
  // reads side by side lie in different banks
  auto place = [](int r, int c) {
    if constexpr (CH == 8)
      return r * BK + ((c ^ (r & 7)) << 3);
    else
      return r * BK + ((c ^ ((r >> 1) & 3)) << 3);
  };
  half8 held[2 * PARTS][LOADS];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int s = 0; s < PARTS; ++s)
#pragma unroll
      for (int l = 0; l < LOADS; ++l) {
        const int u = l * THREADS + threadIdx.x;
        const int64_t at = (int64_t)(u / CH) * K + k0 + u % CH * 8;
        held[s][l] = *reinterpret_cast<const half8*>(p + s * p_plane + at);
        held[PARTS + s][l] = *reinterpret_cast<const half8*>(q + s * q_plane + at);
      }
  };
  auto put = [&](int stage) {
#pragma unroll
    for (int s = 0; s < 2 * PARTS; ++s)
#pragma unroll
      for (int l = 0; l < LOADS; ++l) {
        const int u = l * THREADS + threadIdx.x;
        *reinterpret_cast<half8*>(lds + stage * STAGE + s * PLANE + place(u / CH, u % CH)) = held[s][l];
      }
  };
  fetch(0);
  put(0);
  __syncthreads();
  const int steps = K / BK;
  for (int k = 0; k < steps; ++k) {
    if (k + 1 < steps) fetch((k + 1) * BK);
    const _Float16* here = lds + (k & 1) * STAGE;
#pragma unroll
    for (int ks = 0; ks < BK / 16; ++ks) {
      half8 fp[PARTS][FM], fq[PARTS][FN];
      const int c = ks * 2 + (lane >> 5);
#pragma unroll
      for (int s = 0; s < PARTS; ++s) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
          fp[s][i] = *reinterpret_cast<const half8*>(here + s * PLANE + place(wi + i * 32 + (lane & 31), c));
#pragma unroll
        for (int j = 0; j < FN; ++j)
          fq[s][j] = *reinterpret_cast<const half8*>(here + (PARTS + s) * PLANE + place(wj + j * 32 + (lane & 31), c));
      }
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          if constexpr (PARTS == 2) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fp[1][i], fq[0][j], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fp[0][i], fq[1][j], acc[i][j], 0, 0, 0);
          }
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fp[0][i], fq[0][j], acc[i][j], 0, 0, 0);
        }
    }
    if (k + 1 < steps) put((k + 1) & 1);
    __syncthreads();
  }

  // a lane has column lane & 31 and, of each 8 rows, the four from 4 (lane >> 5) on
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int row = i0 + wi + i * 32 + g * 8 + (lane >> 5) * 4, col = j0 + wj + j * 32 + (lane & 31);
        if constexpr (MODE == kFinal) {
          const int rows = d.tall ? d.n : d.m, cols = d.tall ? d.m : d.n;
          if (col < cols) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (row + e < rows)
                finish(f, d.at + (int64_t)(row + e) * cols + col,
                       acc[i][j][g * 4 + e] * (d.scale / (kOperandScale * kOperandScale)));
          }
        } else {
          const int64_t ld = MODE == kApply ? d.np : d.mp, ldt = d.mp;
          const int64_t plane = MODE == kApply ? mn : mm;
          _Float16* out = mem + (MODE == kGram ? d.a : MODE == kSquare ? d.q : d.x);
          _Float16* out_t = MODE == kApply ? mem + d.xt[from ^ 1] : out;
          _Float16 h[4][PARTS];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = acc[i][j][g * 4 + e] * (1.0f / kOperandScale);
            if constexpr (MODE == kSquare) {
              const _Float16* pa = mem + d.a + (int64_t)(row + e) * ld + col;
              float av = static_cast<float>(pa[0]);
              if constexpr (PARTS == 2) av += static_cast<float>(pa[mm]);
              v = fmaf(cc, v, cb * av);
              if (row + e == col) v += ca * kOperandScale;
            }
            split_half<PARTS>(v, h[e]);
          }
#pragma unroll
          for (int s = 0; s < PARTS; ++s) {
#pragma unroll
            for (int e = 0; e < 4; ++e) out[s * plane + (int64_t)(row + e) * ld + col] = h[e][s];
            if (MODE == kApply || t.i != t.j) {  // (a tile on the diagonal holds its own transpose)
              typedef _Float16 half4 __attribute__((ext_vector_type(4)));
              half4 v4 = {h[0][s], h[1][s], h[2][s], h[3][s]};
              *reinterpret_cast<half4*>(out_t + s * plane + (int64_t)col * ldt + row) = v4;
            }
          }
        }
      }
}

}  // namespace artopk
