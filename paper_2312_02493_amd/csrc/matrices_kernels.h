// Orthogonalised updates of matrices in a flat vector, for gfx950.
//
// Newton-Schulz steps on X, m x n with m <= n (a matrix with more rows than columns is taken as its transpose):
//   X_0 = G / (||G|| + eps),   A = X X^T,   Q = a I + b A + c A^2,   X <- Q X.
// A and Q are symmetric, so only their tiles on and below the diagonal are computed, and each is stored twice.
//
// Two steps at once.  Every A and Q is a polynomial in the first A, so they commute and all their products are symmetric, too.
// After X_1 = Q_1 X_0 the next A is Q_1 A_0 Q_1 and X_2 = (Q_2 Q_1) X_0: five products of m x m by halves and one of each that
// is n long, instead of two and two.  With many more columns than rows that is up to twice as fast.  What it costs: A_1's
// small eigenvalues keep the error of A_0's roundings times up to a^2, which Q_2, whose first term is a I, damps again
// (errors of the result, simulated: 5e-7 to 7e-7 instead of 4e-7 to 6e-7 with two parts, 1.1e-3 to 1.9e-3 instead of 1.1e-3 to
// 1.7e-3 with one).  Three steps at once would not do: the error grows by another a^2, and Q_3 Q_2 Q_1 passes the range below.
//
// Operands.  The products run on the matrix cores in float16 with float32 sums.  Entries of X are at most 2 in size,
// those of A at most 4, those of Q at most 15 (the host refuses coefficients that would pass these bounds), so each is
// stored times 2^12: 2^16 is never reached, and a matrix of 16384 x 16384 still has its first X's typical entry, 2^-14,
// at 2^-2, far above the smallest normal 2^-14.  bfloat16 would need no scale, but rounds eight times as coarsely, and
// the steps multiply small singular values, and what roundings put there, by up to a^5 = 485.  With one part an operand
// keeps 11 bits; with two (hi + lo, and hi hi + hi lo + lo hi for a product) 22, which leaves the result as exact as
// float32 products do.
// A matrix whose X is small, since its norm is below eps or its coefficients shrink it, would sink into float16's smallest
// numbers so.  Its X_k is stored times another 2^e_k, A times 2^(2 e_k): with g the power of two above ||X_0|| times the largest
// factors of the steps before, which ||X_k|| does not pass, e_k is the whole part of -log2(g), or 0 (as it is for every matrix
// whose norm is above eps: growing iterates never need it).  Powers of two round nothing.
//
// Layout.  X X^T and A A^T (A is symmetric) have both operands' rows along the summed index, as the matrix cores take
// them; in Q X the second operand's lie across it, and are turned on their way from LDS to registers.  (A second copy of
// X, transposed, would spare that, and cost more: every step would write it, and with few rows a step is bound by what it
// writes.)  Everything is padded with zeros to multiples of 64, so that the products' summed index has no edge; the
// final product, which writes the caller's buffer, knows the true sizes.
#pragma once

#include "elements.h"

namespace artopk {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kOperandScale = 4096.0f;  // 2^12, of every stored operand

// One matrix.  Places are in halves from the start of the iterates' memory; with two parts the low one follows the
// high one's mp * np (or mp * mp) halves.
struct MatDesc {
  int64_t at;           // first element in the flat vector
  int32_t m, n;         // the smaller and the larger of rows and columns
  int32_t mp, np;       // padded
  int32_t tall;         // the flat vector holds n rows of m
  float scale;
  int64_t x[2];   // X before and after a step, in turn
  int64_t sq[3];  // A, Q and their products, m x m
  int32_t part, parts;  // its sums of squares
  int32_t id;           // its own place in the table
};

// A piece of the flat vector inside one matrix, or of none (mat < 0).
struct MatChunk {
  int64_t begin, end;
  int32_t mat, slot;  // slot: where its sum of squares goes
};

// One block's tile of a product, or its share of the summed index where a tile's sum is cut (shares > 1): the shares
// meet at `slot` of the memory for partial sums.  The matrix is described in every tile: a short product's time is that
// of what it waits for one after the other, and so this is one load.
struct MatTile {
  MatDesc d;
  uint16_t i, j;  // in tiles
  uint16_t share, shares;
  uint32_t slot;
};

// What the elements of a step are made of.
struct MuonArgs {
  float mu, scale;  // momentum <- mu momentum + scale update
  int32_t nesterov;
  float eta, decay_by, eta_rest;  // decay_by = 1 - eta decay
};

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

// Sums of squares of the matrices' pieces.  Sixteen bytes a load from the first aligned place on; a thread's sums are
// float64.
template <class T>
__global__ __launch_bounds__(256) void k_mat_squares(const T* __restrict__ x, const MatChunk* __restrict__ chunks,
                                                     double* __restrict__ sums) {
  constexpr int V = 16 / sizeof(T);
  __shared__ double room[4];
  const MatChunk c = chunks[blockIdx.x];
  if (c.mat < 0) return;
  double s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = 0.0;
  auto add = [&](int i, float v) { s[i] = fma((double)v, (double)v, s[i]); };
  const int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(x + c.begin) / sizeof(T) % V);
  const int64_t body = c.begin + (off ? V - off : 0);
  if (body >= c.end) {
    if (c.begin + (int64_t)threadIdx.x < c.end) add(0, static_cast<float>(x[c.begin + threadIdx.x]));
  } else {
    if (c.begin + (int64_t)threadIdx.x < body) add(0, static_cast<float>(x[c.begin + threadIdx.x]));
    const int64_t whole = body + (c.end - body) / V * V;
#pragma unroll 4
    for (int64_t i = body + threadIdx.x * V; i < whole; i += 256 * V) {
      float v[V];
      load_elems<V>(v, x + i);
#pragma unroll
      for (int e = 0; e < V; ++e) add(e, v[e]);
    }
    if (whole + (int64_t)threadIdx.x < c.end) add(1, static_cast<float>(x[whole + threadIdx.x]));
  }
#pragma unroll
  for (int i = 1; i < V; ++i) s[0] += s[i];
  const double total = block_sum(s[0], room);
  if (threadIdx.x == 0) sums[c.slot] = total;
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

// 1 / (norm + eps) from a matrix's sum of squares; NaN where that is.  It stays float64 until it has multiplied an element: its
// own rounding to float32 would be one error for the whole matrix, which the steps multiply by up to ten.
__device__ __forceinline__ double inverse_of_norm(double squares, float eps) { return 1.0 / (sqrt(squares) + (double)eps); }
__device__ __forceinline__ float normalised(float v, double by) { return static_cast<float>((double)v * by); }

// A matrix's sum of squares from those of its pieces, in every thread of a block of 256.
__device__ __forceinline__ double all_squares(const MatDesc& d, const double* sums, double* room) {
  double s = 0.0;
  for (int i = threadIdx.x; i < d.parts; i += 256) s += sums[d.part + i];
  return block_sum(s, room);
}

// The whole number s with 2^(s - 1) <= ||X_0|| < 2^s, from the sum of squares and the inverse above.
__device__ __forceinline__ float size_of(double squares, double inverse) {
  int s;
  (void)frexp(sqrt(squares) * inverse, &s);
  return (float)s;
}

// e_k of a matrix with ||X_0|| < 2^size; `grown` is log2 of the largest factors of the steps before.  (Not beyond 110: 2^e
// and its inverse times 2^12 stay ordinary float32 numbers.)
__device__ __forceinline__ int exponent_of(float size, float grown) {
  const float e = floorf(-(size + grown));
  return e > 0.0f ? (int)fminf(e, 110.0f) : 0;  // (0 for NaN, too)
}
__device__ __forceinline__ float power_of_two(int e) { return ldexpf(1.0f, e); }

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

// X_0, 64 x 64 elements a block, zeros beyond the true sizes, and how large its norm is.
template <int PARTS, class From>
__global__ __launch_bounds__(256) void k_mat_begin(From from, const MatTile* __restrict__ tiles, const double* __restrict__ sums,
                                                   float eps, _Float16* __restrict__ mem, float* __restrict__ sizes) {
  __shared__ float tile[64][65];
  __shared__ double room[4];
  const MatTile& t = tiles[blockIdx.x];
  const MatDesc& d = t.d;
  const double squares = all_squares(d, sums, room), inverse = inverse_of_norm(squares, eps);
  const float size = size_of(squares, inverse);
  const double by = ldexp(inverse * (double)kOperandScale, exponent_of(size, 0.0f));
  if (t.i == 0 && t.j == 0 && threadIdx.x == 0) sizes[d.id] = size;
  const int rows = d.tall ? d.n : d.m, cols = d.tall ? d.m : d.n;  // as they lie
  const int r0 = (d.tall ? t.j : t.i) * 64, c0 = (d.tall ? t.i : t.j) * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 8
  for (int r = wave; r < 64; r += 4) {
    float v = 0.0f;
    if (r0 + r < rows && c0 + lane < cols) v = normalised(from(d.at + (int64_t)(r0 + r) * cols + c0 + lane), by);
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
    half8 u[PARTS];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 p[PARTS];
      split_half<PARTS>(tile[r][k + e], p);
#pragma unroll
      for (int s = 0; s < PARTS; ++s) u[s][e] = p[s];
    }
#pragma unroll
    for (int s = 0; s < PARTS; ++s)
      *reinterpret_cast<half8*>(mem + d.x[0] + (int64_t)s * d.mp * d.np + (int64_t)(i0 + r) * d.np + j0 + k) = u[s];
  }
}

// What the last product does with X's elements: out = scale X, or the weights' update.
struct FinishArgs {
  void* out;
  int32_t type, muon;
  MuonArgs a;
};

__device__ __forceinline__ float updated(const FinishArgs& f, float weight, float scaled) {
  return fmaf(-f.a.eta, scaled, weight * f.a.decay_by);
}

template <class T>
__device__ __forceinline__ void finish_one(T* p, const FinishArgs& f, float scaled) {
  *p = static_cast<T>(f.muon ? updated(f, static_cast<float>(*p), scaled) : scaled);
}

__device__ __forceinline__ void finish(const FinishArgs& f, int64_t i, float scaled) {
  if (f.type == kTypeF32)
    finish_one(static_cast<float*>(f.out) + i, f, scaled);
  else if (f.type == kTypeBf16)
    finish_one(static_cast<__bf16*>(f.out) + i, f, scaled);
  else
    finish_one(static_cast<_Float16*>(f.out) + i, f, scaled);
}

// Four elements side by side, at a place aligned to all of them.
template <class T>
struct alignas(4 * sizeof(T)) Four {
  T e[4];
};
template <class T>
__device__ __forceinline__ float4 read_four_of(const T* p) {
  const Four<T> v = *reinterpret_cast<const Four<T>*>(p);
  return float4{static_cast<float>(v.e[0]), static_cast<float>(v.e[1]), static_cast<float>(v.e[2]), static_cast<float>(v.e[3])};
}
template <class T>
__device__ __forceinline__ void write_four_of(T* p, const float (&v)[4]) {
  const Four<T> o = {{static_cast<T>(v[0]), static_cast<T>(v[1]), static_cast<T>(v[2]), static_cast<T>(v[3])}};
  *reinterpret_cast<Four<T>*>(p) = o;
}
__device__ __forceinline__ float4 read_four(const FinishArgs& f, int64_t i) {
  if (f.type == kTypeF32) return read_four_of(static_cast<const float*>(f.out) + i);
  if (f.type == kTypeBf16) return read_four_of(static_cast<const __bf16*>(f.out) + i);
  return read_four_of(static_cast<const _Float16*>(f.out) + i);
}
__device__ __forceinline__ void write_four(const FinishArgs& f, int64_t i, const float (&v)[4]) {
  if (f.type == kTypeF32)
    write_four_of(static_cast<float*>(f.out) + i, v);
  else if (f.type == kTypeBf16)
    write_four_of(static_cast<__bf16*>(f.out) + i, v);
  else
    write_four_of(static_cast<_Float16*>(f.out) + i, v);
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
  const double by = inverse_of_norm(all_squares(d, sums, room), eps);
  for (int64_t i = c.begin + threadIdx.x; i < c.end; i += 256) {
    finish(f, i, normalised(from(i), by) * d.scale);
  }
}

// kGram: sq[out] = X X^T;  kSquare: sq[out] = ca I + cb A + cc A^2, A = sq[in];  kTimes: sq[out] = sq[in] sq[in2], which commute;
// kApply: the other X = sq[in] X;  kFinal: the same to the caller's buffer.
enum { kGram = 0, kSquare = 1, kApply = 2, kFinal = 3, kTimes = 4 };

struct ProductArgs {
  int32_t from;  // which X
  int32_t in, in2, out;
  float ca, cb, cc;
  float grown, then;  // log2 of the largest factors of the steps before what is read, and before what is written
};

// The shape of a product's tile: TILE x TILE elements by WM x WN waves, the summed index in stages of kDepth, kStages of
// them in LDS.  A stage is brought by loads that go to LDS without passing registers, two stages ahead of its use at most,
// and every wave reads the next 32 of the summed index into registers while it multiplies the present ones.
// What bounds it is the matrix cores' rate at the clock that the chip holds under them: 4096 x 4096, HALF, Q X in tiles of 256
// 108 us = 1.27 PFLOP/s (a loop of matrix instructions alone reaches 1.5 to 1.6, a large library product 1.4), X X^T's half in
// tiles of 192 70 us = 1.03 PFLOP/s (253 tiles on 256 units, each stored twice).  Larger tiles feed the cores from fewer reads
// of LDS, smaller ones fill the chip; the host takes the class that its table of costs says is soonest done.
constexpr int kDeep = 1;  // added to a TILE: more stages, and one block a compute unit
template <int TILE_, int PARTS_>
struct ProductShape {
  static constexpr int TILE = TILE_ & ~kDeep, PARTS = PARTS_;
  static constexpr int kWM = 2, kWN = TILE >= 192 ? 4 : 2;
  // Two groups of waves take turns along the summed index and add up at the end, where a tile has little work for a stage.
  static constexpr int kGroups = TILE == 64 && PARTS == 2 ? 2 : 1;
  static constexpr int kWaves = kWM * kWN * kGroups, kThreads = kWaves * 64;
  static constexpr int kDepth = PARTS == 2 ? 32 * kGroups : 64;
  static constexpr int kStages = TILE == 256 || TILE == 128 ? 2 : TILE == 192 ? 3 : kGroups == 1 ? 4 : TILE_ & kDeep ? 3 : 2;
  static constexpr int kChunks = kDepth / 8;        // of 16 bytes in a row of a stage
  static constexpr int kLoadRows = 64 / kChunks;    // rows that one load of a wave brings
  static constexpr int kRowsM = TILE / kWM, kRowsN = TILE / kWN;  // of a wave
  static constexpr int kFM = kRowsM / 16, kFN = kRowsN / 16;
  static constexpr int kOutM = kFM / kGroups;  // fragments of rows that a wave has in the end
  static constexpr int kLoads = 2 * PARTS * TILE / kLoadRows / kWaves;  // of a wave, a stage
  static constexpr int kPlane = TILE * kDepth, kStage = 2 * PARTS * kPlane;  // halves
  static constexpr int kHalves = kStages * kStage;
  // Two blocks of the smaller tiles share a compute unit.
  static constexpr int kBlocks = TILE >= 192 || kHalves > 40960 ? 1 : 2;
  // A second set of operands in registers has no room beside the sums of a 256 tile in two parts.
  static constexpr bool kAhead = !(TILE == 256 && PARTS == 2);
  // Where there is room the small products of two parts are summed by themselves: a third of the roundings against the large
  // sum (500 x 900, error of the result 1.5e-6 without, 0.9e-6 with).
  static constexpr bool kLow = TILE == 64 && PARTS == 2;
};

// Chunk c of row r of a stage lies at place c ^ (r & 7) of its row (with 32 halves a row: of the pair of rows), so that
// the sixteen rows that a wave reads together lie in different banks.
template <int CHUNKS>
__device__ __forceinline__ int stage_place(int r, int c) {
  if constexpr (CHUNKS == 8)
    return r * 64 + ((c ^ (r & 7)) << 3);
  else
    return r * 32 + ((c ^ ((r >> 1) & 3)) << 3);
}

// A stage of an operand whose rows lie across the summed index is kDepth rows of TILE; sixteen columns of row r, 32 bytes,
// lie at their place with this flipped, so that the rows that a wave reads together lie in different banks: r, r + 8, r + 16
// and r + 24 for four r side by side.
template <int TILE>
__device__ __forceinline__ int turned_flip(int r) {
  if constexpr (TILE == 64) return ((r >> 1) & 1) | (((r >> 3) & 1) << 1);
  if constexpr (TILE == 128) return (r & 3) | (((r >> 3) & 1) << 2);
  if constexpr (TILE == 192) return r & 3;  // (twelve sixteens a row)
  return (r & 3) | (((r >> 3) & 3) << 2);
}

template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N loads are outstanding, and LDS reads are through
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void block_barrier() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// out = P Q^T over `steps` stages (one at least), P's and Q's rows `ld` and `q_ld` apart.  With `TURNED`
// out = P Q instead: Q's rows lie across the summed index.  P's rows from p_rows on count as zeros (and Q's from q_rows on; of
// a turned Q, columns from `q_rows` on may count as anything that lies in memory behind them up to the matrix's end, or as
// zeros), and so do stages behind the last: the loads' descriptors end there.
template <class S, bool TURNED>
__device__ __forceinline__ void multiply(const _Float16* p, int64_t p_plane, int p_rows, int ld, const _Float16* q,
                                         int64_t q_plane, int q_rows, int q_ld, int steps, _Float16* lds,
                                         f32x4 (&out)[S::kOutM][S::kFN]) {
#if defined(__HIP_DEVICE_COMPILE__)  // (the loads to LDS are unknown to the host's compiler)
  constexpr int TILE = S::TILE, PARTS = S::PARTS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave / (S::kWM * S::kWN), wave2 = wave % (S::kWM * S::kWN);
  const int wi = wave2 / S::kWN * S::kRowsM, wj = wave2 % S::kWN * S::kRowsN;
  const int lr = lane / S::kChunks;
  const int lc = S::kChunks == 8 ? (lane % 8) ^ (lr & 7) : (lane % 4) ^ ((lr >> 1) & 3);
  constexpr int G = TILE / S::kLoadRows;    // loads of one operand's part
  constexpr int EACH = S::kLoads / 2;       // a wave's loads of one operand
  static_assert(S::kLoadRows % (S::kChunks == 8 ? 8 : 16) == 0, "every load's rows lie alike");
  const int p_off = (lr * ld + lc * 8) * 2, q_off = (lr * q_ld + lc * 8) * 2;  // bytes from a load's first row
  int turned_off[TURNED ? EACH : 1];                                          // of a turned operand from the stage's
  if constexpr (TURNED)
#pragma unroll
    for (int l = 0; l < EACH; ++l) {
      const int at = (l * S::kWaves + wave) % G * 64 + lane, r = at / (TILE / 8);
      turned_off[l] = (r * q_ld + ((at % (TILE / 8)) ^ (turned_flip<TILE>(r) << 1)) * 8) * 2;
    }
  // one of a wave's loads for stage k, to place `stage`: EACH of P, then EACH of Q
  auto fetch_one = [&](int k, int stage, int piece) {
    const int there = k < steps ? -1 : 0;
    const bool is_q = piece >= EACH;
    const int l = is_q ? piece - EACH : piece;
    const int u = l * S::kWaves + wave, s = PARTS == 1 ? 0 : u / G;
    const _Float16* base = is_q ? q + s * q_plane : p + s * p_plane;
    int bytes = is_q ? q_rows * q_ld * 2 : p_rows * ld * 2;
    int off = (is_q ? q_off : p_off) + (u % G * (S::kLoadRows * 2) * (is_q ? q_ld : ld) + k * (S::kDepth * 2));
    if (TURNED && is_q) {
      base += (int64_t)k * S::kDepth * q_ld;
      bytes = ((S::kDepth - 1) * q_ld + q_rows) * 2;  // from the stage's first row to the last one's end
      off = turned_off[TURNED ? l : 0];
    }
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        __builtin_amdgcn_make_buffer_rsrc(const_cast<_Float16*>(base), 0, bytes & there, 0x00027000),
        (__attribute__((address_space(3))) void*)(lds + stage * S::kStage + (is_q ? PARTS * S::kPlane : 0) + u * 512), 16,
        off, 0, 0, 0);
  };
  auto fetch = [&](int k, int stage) {
#pragma unroll
    for (int i = 0; i < 2 * EACH; ++i) fetch_one(k, stage, i);
  };
  constexpr int KS = S::kDepth / 32 / S::kGroups;  // of a group
  constexpr int N = TURNED ? 2 : S::kStages;
  constexpr int SETS = S::kAhead ? 2 : 1, Q_SETS = TURNED && KS == 2 ? 3 : SETS;
  half8 fp[PARTS][S::kFM], fq[Q_SETS][PARTS][S::kFN];
  // (of a turned operand a lane names four columns of one row and is given four rows of one column: in each sixteen lanes,
  // lane i names row i / 4 and columns 4 (i % 4) .. and is given rows 0 .. 3 of column i)
  const int tr = (lane >> 4) * 8 + ((lane & 15) >> 2);
  const int flip = turned_flip<TILE>(tr);  // the same for r + 4 and r + 32
  // (a stage's place is worked out anew for every read: all of them at hand would fill the registers)
  auto stage_at = [&](int stage) {
    int at = stage * S::kStage;
    asm volatile("" : "+s"(at));
    return lds + at;
  };
  auto read_p = [&](const _Float16* here, int ks, int i) {
    const int c = (ks + group * KS) * 4 + (lane >> 4);
#pragma unroll
    for (int s = 0; s < PARTS; ++s)
      fp[s][i] = *reinterpret_cast<const half8*>(here + s * S::kPlane + stage_place<S::kChunks>(wi + i * 16 + (lane & 15), c));
  };
  auto read_q = [&](const _Float16* here, int ks, int to, int j) {
    ks += group * KS;
    const int c = ks * 4 + (lane >> 4);
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
      const _Float16* at = here + (PARTS + s) * S::kPlane;
      if constexpr (TURNED) {
        typedef short short4v __attribute__((ext_vector_type(4)));
        at += (ks * 32 + tr) * TILE + ((((wj >> 4) + j) ^ flip) << 4) + (lane & 3) * 4;
        const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at);
        const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(at + 4 * TILE));
        fq[to][s][j] = __builtin_shufflevector(__builtin_bit_cast(half4, a), __builtin_bit_cast(half4, b), 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        fq[to][s][j] = *reinterpret_cast<const half8*>(at + stage_place<S::kChunks>(wj + j * 16 + (lane & 15), c));
      }
    }
  };
  auto read_all = [&](int stage, int ks, int q_to, bool of_p, bool of_q) {
    const _Float16* here = stage_at(stage);
    if (of_p)
#pragma unroll
      for (int i = 0; i < S::kFM; ++i) read_p(here, ks, i);
    if (of_q)
#pragma unroll
      for (int j = 0; j < S::kFN; ++j) read_q(here, ks, q_to, j);
  };
  f32x4 acc[S::kFM][S::kFN];
#pragma unroll
  for (int i = 0; i < S::kFM; ++i)
#pragma unroll
    for (int j = 0; j < S::kFN; ++j) acc[i][j] = 0.0f;
  f32x4 low[S::kLow ? S::kFM : 1][S::kLow ? S::kFN : 1];
#pragma unroll
  for (int i = 0; i < (S::kLow ? S::kFM : 1); ++i)
#pragma unroll
    for (int j = 0; j < (S::kLow ? S::kFN : 1); ++j) low[i][j] = 0.0f;
  // The second operand goes first: so a lane is given four columns of one row side by side.
  auto mul_row = [&](int i, int q_of) {
#pragma unroll
    for (int j = 0; j < S::kFN; ++j) {
      if constexpr (PARTS == 2) {
        f32x4& to = S::kLow ? low[i][j] : acc[i][j];
        to = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[q_of][0][j], fp[PARTS - 1][i], to, 0, 0, 0);
        to = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[q_of][PARTS - 1][j], fp[0][i], to, 0, 0, 0);
      }
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[q_of][0][j], fp[0][i], acc[i][j], 0, 0, 0);
    }
  };
  // What is read and asked for stands between the rows of products, P's next fragment where the last row's was: with all of it
  // in front, the waves' loads wait for each other while nothing multiplies (4096 x 4096, HALF, tiles of 256: X X^T 92 us, Q X
  // 114, so 89 and 110; sixteen 1280 x 1280 and eight 1280 x 5120, SPLIT, tiles of 128: Q X 671, so 610; but X X^T of four
  // 512 x 4608, HALF, tiles of 64, alone on their units, 16.2, so 17.6).
  auto rows = [&](int q_of, auto&& between) {
#pragma unroll
    for (int i = 0; i < S::kFM; ++i) {
      between(i);
      mul_row(i, q_of);
      __builtin_amdgcn_sched_barrier(0);  // (or the reads sink to their uses)
    }
    between(S::kFM);
  };
  constexpr int ROW_LOADS = (2 * EACH + S::kFM - 1) / S::kFM;  // of a row
  constexpr int ROW_Q = (S::kFN + S::kFM - 1) / S::kFM;
  int st = 0;
  auto after = [&](int of) { return of + 1 == N ? 0 : of + 1; };
  if constexpr (S::kAhead) {
#pragma unroll
    for (int s = 0; s < N; ++s) fetch(s, s);
    wait_loads<(N - 1) * S::kLoads>();
    block_barrier();
    read_all(0, 0, 0, true, true);
    if constexpr (TURNED && KS == 2) read_all(0, 1, 1, false, true);
    // the products with Q's set `q_of` beside which the next stage's first operands come, Q's to `q_to`, and the loads of stage
    // k + N go out
    auto last_of_stage = [&](int k, bool more, int q_of, int q_to) {
      if (!more) return rows(q_of, [](int) {});
      wait_loads<(N - 2) * S::kLoads>();  // the next stage is there, and this one read whole
      block_barrier();
      const int next = after(st), here = st;
      // A turned operand is read before the next loads go out, both halves of it where a stage has two: the compiler lets no such
      // read pass a load to LDS that is on its way, whatever stage it is for.  (So two stages do for it.)
      if constexpr (TURNED) {
        read_all(next, 0, q_to, false, true);
        if constexpr (KS == 2) read_all(next, 1, 2, false, true);
      }
      st = next;
      const _Float16* at = stage_at(next);
      rows(q_of, [&](int i) {
#pragma unroll
        for (int l = i * ROW_LOADS; l < (i + 1) * ROW_LOADS; ++l)
          if (l < 2 * EACH) fetch_one(k + N, here, l);
        if (i > 0) read_p(at, 0, i - 1);
        if constexpr (!TURNED)
#pragma unroll
          for (int j = i * ROW_Q; j < (i + 1) * ROW_Q; ++j)
            if (j < S::kFN) read_q(at, 0, q_to, j);
      });
    };
    auto stage = [&](int k, int odd, bool more) {
      if constexpr (KS == 2) {
        const _Float16* at = stage_at(st);
        rows(0, [&](int i) {
          if (i > 0) read_p(at, 1, i - 1);
          if constexpr (!TURNED)
#pragma unroll
            for (int j = i * ROW_Q; j < (i + 1) * ROW_Q; ++j)
              if (j < S::kFN) read_q(at, 1, 1, j);
        });
        last_of_stage(k, more, 1, 0);
        if constexpr (TURNED) {
          if (more)
#pragma unroll
            for (int s = 0; s < PARTS; ++s)
#pragma unroll
              for (int j = 0; j < S::kFN; ++j) fq[1][s][j] = fq[Q_SETS - 1][s][j];
        }
      } else {
        last_of_stage(k, more, odd, odd ^ 1);
      }
    };
    int k = 0;
    if constexpr (KS == 2) {
      for (; k + 1 < steps; ++k) stage(k, 0, true);
    } else {
      for (; k + 2 < steps; k += 2) {
        stage(k, 0, true);
        stage(k + 1, 1, true);
      }
    }
    if (KS == 1 && steps - k == 2) {
      stage(k, 0, true);
      stage(k + 1, 1, false);
    } else {
      stage(k, 0, false);
    }
  } else {
    static_assert(N == 2 && KS == 1, "");
    fetch(0, 0);
    for (int k = 0; k < steps; ++k) {
      wait_loads<0>();
      block_barrier();
      if constexpr (!TURNED) fetch(k + 1, st ^ 1);
      read_all(st, 0, 0, true, true);
      if constexpr (TURNED) fetch(k + 1, st ^ 1);
#pragma unroll
      for (int i = 0; i < S::kFM; ++i) mul_row(i, 0);
      st ^= 1;
    }
  }
  if constexpr (S::kLow)
#pragma unroll
    for (int i = 0; i < S::kFM; ++i)
#pragma unroll
      for (int j = 0; j < S::kFN; ++j) acc[i][j] += low[i][j];
  wait_loads<0>();  // the loads behind the last stage still write
  block_barrier();
  if constexpr (S::kGroups == 1) {
#pragma unroll
    for (int i = 0; i < S::kFM; ++i)
#pragma unroll
      for (int j = 0; j < S::kFN; ++j) out[i][j] = acc[i][j];
  } else {  // each group finishes half of the rows, with what the other has of them
    f32x4* room = reinterpret_cast<f32x4*>(lds);
    constexpr int H = S::kOutM, T = S::kWM * S::kWN * 64;
    const int t = wave2 * 64 + lane;
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < S::kFN; ++j) room[((group * H + i) * S::kFN + j) * T + t] = group ? acc[i][j] : acc[H + i][j];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < S::kFN; ++j)
        out[i][j] = (group ? acc[H + i][j] : acc[i][j]) + room[(((group ^ 1) * H + i) * S::kFN + j) * T + t];
    __syncthreads();
  }
#endif
}

// One wave's rows of a tile, by way of its own part of LDS: `value(i, j)` are four sums of row 16 i + lane % 16 and columns
// 16 j + 4 (lane / 16) ..; they go as halves to out[row ld + col] and, `both`, to out_t[col ld_t + row].  Rows and
// columns from `rows` and `cols` on are left out (whole chunks of eight: both are multiples of 64).
template <int FM, int FN, int PARTS, class Value>
__device__ __forceinline__ void store_halves(Value&& value, _Float16* room, int row0, int col0, int rows, int cols,
                                             _Float16* out, int64_t ld, _Float16* out_t, int64_t ld_t, int64_t plane,
                                             bool both) {
  constexpr int CF = FM > 4 ? FM / 2 : FM;  // fragments of rows at a time
  constexpr int CR = CF * 16, CC = FN * 16;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int h = 0; h < FM; h += CF) {
    half4 v[PARTS][CF][FN];
#pragma unroll
    for (int i = 0; i < CF; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const f32x4 x = value(h + i, j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          _Float16 p[PARTS];
          split_half<PARTS>(x[e], p);
#pragma unroll
          for (int s = 0; s < PARTS; ++s) v[s][i][j][e] = p[s];
        }
      }
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < CF; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          *reinterpret_cast<half4*>(room + (i * 16 + (lane & 15)) * (CC + 8) + j * 16 + (lane >> 4) * 4) = v[s][i][j];
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < CR * CC / 8; u += 64) {
        const int r = (u + lane) / (CC / 8), c = (u + lane) % (CC / 8) * 8;
        if ((CR * CC / 8) % 64 && u + lane >= CR * CC / 8) continue;
        const half8 x = *reinterpret_cast<const half8*>(room + r * (CC + 8) + c);
        const int row = row0 + h * 16 + r, col = col0 + c;
        if (row < rows && col < cols) *reinterpret_cast<half8*>(out + s * plane + row * ld + col) = x;
      }
      asm volatile("" ::: "memory");
      if (!both) continue;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < CF; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            room[(j * 16 + (lane >> 4) * 4 + e) * (CR + 8) + i * 16 + (lane & 15)] = v[s][i][j][e];
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < CR * CC / 8; u += 64) {
        const int c = (u + lane) / (CR / 8), r = (u + lane) % (CR / 8) * 8;
        if ((CR * CC / 8) % 64 && u + lane >= CR * CC / 8) continue;
        const half8 x = *reinterpret_cast<const half8*>(room + c * (CR + 8) + r);
        const int row = row0 + h * 16 + r, col = col0 + c;
        if (row < rows && col < cols) *reinterpret_cast<half8*>(out_t + s * plane + col * ld_t + row) = x;
      }
      asm volatile("" ::: "memory");
    }
  }
}

// Halves of LDS that a wave's stores need: 16 bytes between rows beyond their length.
template <int FM, int FN>
constexpr int store_room() {
  constexpr int CR = (FM > 4 ? FM / 2 : FM) * 16, CC = FN * 16;
  constexpr int a = CR * (CC + 8), b = CC * (CR + 8), c = 2 * 36 * (CC + 4);  // c: 32 rows of floats, or as many columns
  return a > b ? (a > c ? a : c) : (b > c ? b : c);
}

// The same for the caller's buffer, as floats: out = scale X, or the weights' update, whose old values are asked for before the
// sums pass through LDS (asked for one by one where they are needed, the product that ends 78.6 M bf16 weights took 324 us;
// so, and with faster sums, 311).
template <int FM, int FN, bool TALL>
__device__ __forceinline__ void finish_rows(const f32x4 (&acc)[FM][FN], float* fl, int row0, int col0, const MatDesc& d,
                                            const FinishArgs& f, float down) {
  const int lane = threadIdx.x & 63;
  constexpr int CC = FN * 16, HM = FM > 1 ? 2 : 1, HR = HM * 16;  // rows at a time
  constexpr int RUN = TALL ? HR : CC, PITCH = RUN + 4;            // as they lie
  constexpr int EACH = HR * CC / 4 / 64;                          // fours of a lane
  const int lines = TALL ? d.n : d.m, length = TALL ? d.m : d.n;
  const float by = d.scale * (1.0f / (kOperandScale * kOperandScale));
  const int size = f.type == kTypeF32 ? 4 : 2;
  const bool wide = length % 4 == 0 && (reinterpret_cast<uintptr_t>(f.out) + d.at * size) % (4 * size) == 0;
#pragma unroll
  for (int h = 0; h < FM; h += HM) {
    const int line0 = TALL ? col0 : row0 + h * 16, place0 = TALL ? row0 + h * 16 : col0;
    int64_t at[EACH];
    float4 old[EACH];
    if (wide) {
#pragma unroll
      for (int u = 0; u < EACH; ++u) {
        const int r = (u * 64 + lane) / (RUN / 4), c = (u * 64 + lane) % (RUN / 4) * 4;
        const bool there = line0 + r < lines && place0 + c < length;
        at[u] = there ? d.at + (int64_t)(line0 + r) * length + place0 + c : -1;
        if (f.muon && there) old[u] = read_four(f, at[u]);
      }
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < HM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const f32x4 v = acc[h + i][j] * by * down;
        if constexpr (TALL) {
#pragma unroll
          for (int e = 0; e < 4; ++e) fl[(j * 16 + (lane >> 4) * 4 + e) * PITCH + i * 16 + (lane & 15)] = v[e];
        } else {
          *reinterpret_cast<f32x4*>(fl + (i * 16 + (lane & 15)) * PITCH + j * 16 + (lane >> 4) * 4) = v;
        }
      }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    if (wide) {
#pragma unroll
      for (int u = 0; u < EACH; ++u) {
        const int r = (u * 64 + lane) / (RUN / 4), c = (u * 64 + lane) % (RUN / 4) * 4;
        const f32x4 x = *reinterpret_cast<const f32x4*>(fl + r * PITCH + c);
        float v[4] = {x[0], x[1], x[2], x[3]};
        if (f.muon) {
          const float w[4] = {old[u].x, old[u].y, old[u].z, old[u].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = updated(f, w[e], v[e]);
        }
        if (at[u] >= 0) write_four(f, at[u], v);
      }
    } else {
#pragma unroll 4
      for (int u = lane; u < HR * CC; u += 64) {
        const int r = u / RUN, c = u % RUN;
        if (line0 + r < lines && place0 + c < length) {
          finish(f, d.at + (int64_t)(line0 + r) * length + place0 + c, fl[r * PITCH + c]);
        }
      }
    }
    asm volatile("" ::: "memory");
  }
}

template <int SHAPE, int PARTS, int MODE>
__global__ __launch_bounds__((ProductShape<SHAPE, PARTS>::kThreads), (ProductShape<SHAPE, PARTS>::kBlocks)) void k_mat_product(
    const MatTile* __restrict__ tiles, _Float16* __restrict__ mem, ProductArgs a, FinishArgs f, float* __restrict__ partial,
    const float* __restrict__ sizes) {
  using S = ProductShape<SHAPE, PARTS>;
  constexpr int TILE = S::TILE, FM = S::kOutM, FN = S::kFN;
  constexpr int kRoom = store_room<FM, FN>();
  constexpr int kStaged = MODE == kApply || MODE == kFinal ? 2 * S::kStage : S::kHalves;
  constexpr int kNeed = kRoom * S::kWaves > kStaged ? kRoom * S::kWaves : kStaged;
  __shared__ __align__(16) _Float16 lds[kNeed];

  const MatTile& t = tiles[blockIdx.x];
  const MatDesc& d = t.d;
  const int64_t mm = (int64_t)d.mp * d.mp, mn = (int64_t)d.mp * d.np;
  const float size = MODE == kGram ? 0.0f : sizes[d.id];
  const int i0 = t.i * TILE, j0 = t.j * TILE;
  constexpr bool kTurned = MODE == kApply || MODE == kFinal;
  const int rows = d.mp, cols = kTurned ? d.np : d.mp;
  const int p_rows = rows - i0 < TILE ? rows - i0 : TILE, q_rows = cols - j0 < TILE ? cols - j0 : TILE;
  f32x4 acc[FM][FN];
  if constexpr (kTurned) {
    multiply<S, true>(mem + d.sq[a.in] + (int64_t)i0 * d.mp, mm, p_rows, d.mp, mem + d.x[a.from] + j0, mn, q_rows, d.np,
                      d.mp / S::kDepth, lds, acc);
  } else {
    const _Float16* p = mem + (MODE == kGram ? d.x[a.from] : d.sq[a.in]);
    const _Float16* q = MODE == kTimes ? mem + d.sq[a.in2] : p;
    const int ld = MODE == kGram ? d.np : d.mp;
    // a share is whole pieces of 64
    const int begin = MODE == kGram ? (int)((int64_t)(ld / 64) * t.share / t.shares) * 64 : 0;
    const int end = MODE == kGram ? (int)((int64_t)(ld / 64) * (t.share + 1) / t.shares) * 64 : ld;
    const int64_t plane = MODE == kGram ? mn : mm;
    multiply<S, false>(p + (int64_t)i0 * ld + begin, plane, p_rows, ld, q + (int64_t)j0 * ld + begin, plane, q_rows, ld,
                       (end - begin) / S::kDepth, lds, acc);
  }

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave2 = wave % (S::kWM * S::kWN), group = wave / (S::kWM * S::kWN);
  const int row0 = i0 + wave2 / S::kWN * S::kRowsM + group * (FM * 16), col0 = j0 + wave2 % S::kWN * S::kRowsN;
  _Float16* room = lds + wave * kRoom;
  const int up = MODE == kGram ? 0 : exponent_of(size, a.grown);
  if constexpr (MODE == kGram) {
    if (t.shares > 1) {  // the sums of this share, for k_mat_join
      f32x4* mine = reinterpret_cast<f32x4*>(partial + ((int64_t)t.slot + t.share) * (TILE * TILE)) + threadIdx.x;
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) mine[(i * FN + j) * S::kThreads] = acc[i][j];
      return;
    }
  }
  if constexpr (MODE == kFinal) {
    // Elements of a tall matrix lie column by column of X.  A few rows of the wave's part at a time go through LDS as floats, in
    // the order in which they lie.
    const float down = power_of_two(-up);
    if (d.tall)
      finish_rows<FM, FN, true>(acc, reinterpret_cast<float*>(room), row0, col0, d, f, down);
    else
      finish_rows<FM, FN, false>(acc, reinterpret_cast<float*>(room), row0, col0, d, f, down);
  } else if constexpr (MODE == kSquare) {
    const float cb = ldexpf(a.cb, -2 * up), cc = ldexpf(a.cc, -4 * up) / kOperandScale;
    auto value = [&](int i, int j) {
      const int row = row0 + i * 16 + (lane & 15), col = col0 + j * 16 + (lane >> 4) * 4;
      f32x4 v = acc[i][j] * cc;
      // (a place outside is read at the edge, and not stored: no load waits behind a branch; 78.6 M bf16 weights 2298 us, so 2283)
      const _Float16* pa = mem + d.sq[a.in] + (int64_t)(row < rows ? row : rows - 1) * d.mp + (col < cols ? col : cols - 4);
      const half4 hi = *reinterpret_cast<const half4*>(pa);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float av = static_cast<float>(hi[e]);
        if constexpr (PARTS == 2) av += static_cast<float>(reinterpret_cast<const half4*>(pa + mm)[0][e]);
        v[e] = fmaf(cb, av, v[e]);
        if (row == col + e) v[e] += a.ca * kOperandScale;
      }
      return v;
    };
    store_halves<FM, FN, PARTS>(value, room, row0, col0, rows, cols, mem + d.sq[a.out], d.mp, mem + d.sq[a.out], d.mp, mm, t.i != t.j);
  } else {
    const int to = MODE == kGram ? 0 : exponent_of(size, a.then);
    const float by = power_of_two(to - up), by2 = (MODE == kTimes ? by : 1.0f) * (1.0f / kOperandScale);
    auto value = [&](int i, int j) { return acc[i][j] * by2 * by; };
    if constexpr (MODE == kGram || MODE == kTimes)
      store_halves<FM, FN, PARTS>(value, room, row0, col0, rows, cols, mem + d.sq[a.out], d.mp, mem + d.sq[a.out], d.mp, mm,
                                  t.i != t.j);
    else
      store_halves<FM, FN, PARTS>(value, room, row0, col0, rows, cols, mem + d.x[a.from ^ 1], d.np, nullptr, 0, mn, false);
  }
}

// Whole steps of small matrices, one block each, with everything on chip: X, A and Q lie in LDS as halves (rows padded by
// eight), sums in registers.  A step's products of a matrix that one compute unit holds take some microseconds there, less
// than the launches and the trips through memory that they would otherwise be.
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;
constexpr int kSmallElems = kSmallWaves * 32 * 32;           // of X, padded, at most: a block of 32 x 32 for each wave
constexpr int kSmallHeld = kSmallElems / kSmallThreads;      // that a thread brings
struct PolarSteps {
  int32_t steps;
  float co[32][3];
  float grown[32];  // log2 of the largest factors of the steps before each
};
__host__ __device__ constexpr int small_pad(int v) { return (v + 31) / 32 * 32; }
__host__ __device__ constexpr int64_t small_halves(int m, int n, int parts) {
  return (int64_t)parts * small_pad(m) * ((small_pad(n) + 8) + 2 * (small_pad(m) + 8));
}

template <int PARTS, class From>
__global__ __launch_bounds__(kSmallThreads) void k_mat_small(From from, const MatDesc* __restrict__ mats, PolarSteps st,
                                                             float eps, FinishArgs f) {
  extern __shared__ __align__(16) _Float16 small_lds[];
  __shared__ double room[kSmallWaves];
  const MatDesc d = mats[blockIdx.x];
  const int mp = small_pad(d.m), np = small_pad(d.n), xp = np + 8;
  _Float16* X = small_lds;
  const int size = d.m * d.n, cols = d.tall ? d.m : d.n;
  float held[kSmallHeld];
#pragma unroll
  for (int u = 0; u < kSmallHeld; ++u) {
    const int i = threadIdx.x + u * kSmallThreads;
    held[u] = i < size ? from(d.at + i) : 0.0f;
  }
  const half8 zeros = {};
  for (int i = threadIdx.x * 8; i < PARTS * mp * xp; i += kSmallThreads * 8) *reinterpret_cast<half8*>(X + i) = zeros;
  double sum = 0.0;
#pragma unroll
  for (int u = 0; u < kSmallHeld; ++u) sum = fma((double)held[u], (double)held[u], sum);
  sum = block_sum(sum, room);
  const double inverse = inverse_of_norm(sum, eps);
  const float norm_size = size_of(sum, inverse);
  int up = exponent_of(norm_size, 0.0f);  // of the present X
  const double by = ldexp(inverse * (double)kOperandScale, up);
#pragma unroll
  for (int u = 0; u < kSmallHeld; ++u) {
    const int i = threadIdx.x + u * kSmallThreads;
    if (i < size) {
      const int r = i / cols, c = i - r * cols;
      _Float16 h[PARTS];
      split_half<PARTS>(normalised(held[u], by), h);
#pragma unroll
      for (int p = 0; p < PARTS; ++p) X[(p * mp + (d.tall ? c : r)) * xp + (d.tall ? r : c)] = h[p];
    }
  }
  __syncthreads();

#if defined(__HIP_DEVICE_COMPILE__)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ap = mp + 8;
  _Float16* A = X + PARTS * mp * xp;
  _Float16* Q = A + PARTS * mp * ap;
  int l15 = lane & 15, l4 = lane >> 4;
  const int am = mp / 32, an = np / 32;
  // A wave takes a block of 32 x 32, whose four tiles share what is read: the sums of block (i, j) of P B^T, times 2^-12;
  // with `turned` of P^T B^T.  P's rows are p_pitch apart.  A lane is given four rows of a column, that is, of the transposed
  // block four columns side by side: so A and Q, which are symmetric, are stored as their transposes, whole (a wave with the
  // mirrored block costs nothing where there are waves enough), and X' = Q X is worked out as X^T Q.
  auto block = [&](const _Float16* P, int p_pitch, int i, const _Float16* B, int b_pitch, int j, int depth, auto turned,
                   f32x4 (&out)[2][2]) {
    f32x4 acc[2][2], low[2][2], low2[2][2];
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[x >> 1][x & 1] = low[x >> 1][x & 1] = low2[x >> 1][x & 1] = 0.0f;
    const int p_plane = mp * p_pitch, b_plane = mp * b_pitch;
    // (turned as in multiply())
    const _Float16* a = turned() ? P + (l4 * 8 + (l15 >> 2)) * p_pitch + i * 32 + (l15 & 3) * 4 : P + (i * 32 + l15) * p_pitch + l4 * 8;
    const _Float16* b = B + (j * 32 + l15) * b_pitch + l4 * 8;
    typedef short short4v __attribute__((ext_vector_type(4)));
    auto four = [&](const _Float16* at) {
      return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at));
    };
#pragma clang loop unroll(disable)
    for (int k = 0; k < depth; k += 32) {
      half8 fa[PARTS][2], fb[PARTS][2];
#pragma unroll
      for (int s = 0; s < PARTS; ++s)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if constexpr (turned()) {
            const _Float16* at = a + s * p_plane + k * p_pitch + x * 16;
            fa[s][x] = __builtin_shufflevector(four(at), four(at + 4 * p_pitch), 0, 1, 2, 3, 4, 5, 6, 7);
          } else {
            fa[s][x] = *reinterpret_cast<const half8*>(a + s * p_plane + x * 16 * p_pitch + k);
          }
          fb[s][x] = *reinterpret_cast<const half8*>(b + s * b_plane + x * 16 * b_pitch + k);
        }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int u = x >> 1, v = x & 1;
        if constexpr (PARTS == 2) {
          low[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[PARTS - 1][u], fb[0][v], low[u][v], 0, 0, 0);
          low2[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[0][u], fb[PARTS - 1][v], low2[u][v], 0, 0, 0);
        }
        acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[0][u], fb[0][v], acc[u][v], 0, 0, 0);
      }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
      out[x >> 1][x & 1] = (acc[x >> 1][x & 1] + (low[x >> 1][x & 1] + low2[x >> 1][x & 1])) * (1.0f / kOperandScale);
  };
  // the transpose of block (i, j) at block (j, i)
  auto put = [&](_Float16* M, int pitch, int i, int j, const f32x4 (&v)[2][2]) {
    _Float16* at = M + (j * 32 + l15) * pitch + i * 32 + l4 * 4;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      half4 t[PARTS];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        _Float16 h[PARTS];
        split_half<PARTS>(v[x >> 1][x & 1][e], h);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) t[p][e] = h[p];
      }
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
        *reinterpret_cast<half4*>(at + (p * mp + (x & 1) * 16) * pitch + (x >> 1) * 16) = t[p];
    }
  };
  const bool has_a = wave < am * am, has_x = wave < am * an;
  const int ai = wave / am, aj = wave - ai * am;  // of A and Q
  const int xj = wave / am, xi = wave - xj * am;  // of X
  constexpr std::integral_constant<bool, true> kTurned;
  constexpr std::integral_constant<bool, false> kStraight;
  f32x4 v[2][2];
  for (int step = 0; step < st.steps; ++step) {
    asm volatile("" : "+v"(l15), "+v"(l4));  // (places worked out once for all steps would fill the registers)
    const float ca = st.co[step][0], cb = ldexpf(st.co[step][1], -2 * up), cc = ldexpf(st.co[step][2], -4 * up);
    if (has_a) {
      block(X, xp, ai, X, xp, aj, np, kStraight, v);
      put(A, ap, ai, aj, v);
    }
    __syncthreads();
    if (has_a) {
      block(A, ap, ai, A, ap, aj, mp, kStraight, v);
      const _Float16* at = A + (aj * 32 + l15) * ap + ai * 32 + l4 * 4;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const half4 hi = *reinterpret_cast<const half4*>(at + (x & 1) * 16 * ap + (x >> 1) * 16);
        half4 lo = {};
        if constexpr (PARTS == 2) lo = *reinterpret_cast<const half4*>(at + (mp + (x & 1) * 16) * ap + (x >> 1) * 16);
        const int row = ai * 32 + (x >> 1) * 16 + l4 * 4, col = aj * 32 + (x & 1) * 16 + l15;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float w = fmaf(cb, static_cast<float>(hi[e]) + static_cast<float>(lo[e]), v[x >> 1][x & 1][e] * cc);
          if (row + e == col) w += ca * kOperandScale;
          v[x >> 1][x & 1][e] = w;
        }
      }
      put(Q, ap, ai, aj, v);
    }
    __syncthreads();
    if (has_x) block(X, xp, xj, Q, ap, xi, mp, kTurned, v);
    if (step + 1 == st.steps) break;
    const int to = exponent_of(norm_size, st.grown[step + 1]);
    if (to != up) {
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x >> 1][x & 1] *= power_of_two(to - up);
      up = to;
    }
    __syncthreads();
    if (has_x) put(X, xp, xj, xi, v);
    __syncthreads();
  }
  if (!has_x) return;
  const int size4 = f.type == kTypeF32 ? 16 : 8;
  const bool wide = !d.tall && d.n % 4 == 0 && (reinterpret_cast<uintptr_t>(f.out) + d.at * (size4 / 4)) % size4 == 0;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int row = xi * 32 + (x & 1) * 16 + l15, col = xj * 32 + (x >> 1) * 16 + l4 * 4;
    const f32x4 scaled = v[x >> 1][x & 1] * (d.scale / kOperandScale) * power_of_two(-up);
    const float w[4] = {scaled[0], scaled[1], scaled[2], scaled[3]};
    if (row >= d.m || col >= d.n) continue;
    if (wide) {
      const int64_t at = d.at + (int64_t)row * d.n + col;
      float o[4] = {w[0], w[1], w[2], w[3]};
      if (f.muon) {
        const float4 old = read_four(f, at);
        o[0] = updated(f, old.x, w[0]), o[1] = updated(f, old.y, w[1]), o[2] = updated(f, old.z, w[2]), o[3] = updated(f, old.w, w[3]);
      }
      write_four(f, at, o);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (col + e < d.n) finish(f, d.at + (d.tall ? (int64_t)(col + e) * d.m + row : (int64_t)row * d.n + col + e), w[e]);
      }
    }
  }
#endif
}

// Adds the shares of a Gram matrix's tiles in their order and stores the tile, half of each wave's fragments a block.
// (The blocks of the product cannot do it themselves, the last one of a tile: that takes a write-back of a die's whole cache
// by every block before it says that it is through.  480 blocks of 128 x 128 sums took 150 us so, 20 in two launches.)
template <int TILE, int PARTS>
__global__ __launch_bounds__((ProductShape<TILE, PARTS>::kThreads)) void k_mat_join(
    const MatTile* __restrict__ tiles, _Float16* __restrict__ mem, const float* __restrict__ partial) {
  using S = ProductShape<TILE, PARTS>;
  constexpr int FM = S::kOutM, FN = S::kFN, QN = FN / 2;
  constexpr int kRoom = store_room<FM, QN>();
  __shared__ __align__(16) _Float16 lds[kRoom * S::kWaves];
  const MatTile& t = tiles[blockIdx.x];
  const MatDesc& d = t.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave2 = wave % (S::kWM * S::kWN), group = wave / (S::kWM * S::kWN), qj = blockIdx.y * QN;
  const int row0 = t.i * TILE + wave2 / S::kWN * S::kRowsM + group * (FM * 16);
  const int col0 = t.j * TILE + wave2 % S::kWN * S::kRowsN + qj * 16;
  const f32x4* all = reinterpret_cast<const f32x4*>(partial + (int64_t)t.slot * (TILE * TILE)) + threadIdx.x;
  f32x4 sum[FM][QN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < QN; ++j) sum[i][j] = all[(i * FN + qj + j) * S::kThreads];
  for (int s = 1; s < t.shares; ++s)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < QN; ++j) sum[i][j] += all[(int64_t)s * (TILE * TILE / 4) + (i * FN + qj + j) * S::kThreads];
  auto value = [&](int i, int j) { return sum[i][j] * (1.0f / kOperandScale); };
  store_halves<FM, QN, PARTS>(value, lds + wave * kRoom, row0, col0, d.mp, d.mp, mem + d.sq[0], d.mp, mem + d.sq[0], d.mp,
                              (int64_t)d.mp * d.mp, t.i != t.j);
}

}  // namespace artopk
