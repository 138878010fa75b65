// Layer norm over rows, forward and backward, for gfx950.
//
//   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps)
//   h = (x - mean) rstd,  y = h gamma + beta
//   d = dy gamma,  dx = rstd (d - mean(d) - h mean(d h))
//   dgamma = sum over the rows of dy h,  dbeta = sum over the rows of dy
//
// Both are bound by memory: forward moves every element twice, backward three times, with some ten operations on
// each.  So a row is read once and kept in registers as float32 until its sums are known (the variance is that of the
// differences from the mean, a second sum over registers, not a difference of large sums), and in the backward pass
// a thread keeps the same columns in every row, so that the weight gradients gather in registers, too.  All sums are
// float32, in an order that depends on the sizes, on what may be read sixteen bytes at a time, and on the number of blocks.
//
// Measured: forward 32768 x 4096 bfloat16 108 us = 5.0 TB/s (a copy of 2 GiB 4.95); backward 32768 x 2048 80 us and 6 for the
// shares of the weights' gradients = 4.7 TB/s; 8 x 4096 forward 3.6 us, a launch.
#pragma once

#include "elements.h"

namespace artopk {

// Rows of R columns kept by TPR threads of E elements each; a block holds kNormThreads / TPR rows at a time
// (one if TPR is larger).  V elements lie side by side in memory, thread by thread.
template <int TPR>
struct NormShape {
  static constexpr int kThreads = TPR < 256 ? 256 : TPR;
  static constexpr int kRows = kThreads / TPR;
  static constexpr int kWaves = TPR / 64;  // of one row
};

// The weights' gradients as the caller wants them: dgamma (0) and dbeta (1), either of which may be missing, of one of the
// three element types; `add` adds to what is there, in float32.
struct GradOut {
  void* out[2];
  int32_t type, add;
  __device__ __forceinline__ bool wanted(int which) const { return out[which] != nullptr; }
  template <class G>
  __device__ __forceinline__ void put_as(G* p, float s) const {
    *p = static_cast<G>(add ? s + static_cast<float>(*p) : s);
  }
  __device__ __forceinline__ void put(int which, int64_t c, float s) const {
    if (!out[which]) return;
    if (type == kTypeF32)
      put_as(static_cast<float*>(out[which]) + c, s);
    else if (type == kTypeBf16)
      put_as(static_cast<__bf16*>(out[which]) + c, s);
    else
      put_as(static_cast<_Float16*>(out[which]) + c, s);
  }
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Sums of N values over the TPR threads of a row, in every one of them.  `turn` alternates between calls, so that one
// barrier a call is enough: who is still reading one half of `room` holds up nobody before the call after the next.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* room, int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* at = room + turn * (N * W);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * W + wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = at[i * W];
#pragma unroll
      for (int j = 1; j < W; ++j) s += at[i * W + j];
      v[i] = s;
    }
  }
}

// V elements of a row as they lie, zeros behind its end.  A load stands in no branch, behind which it would be waited for:
// places behind the end read the row's last ones instead (32768 x 2048 bf16 backward 93 us with a branch around each load, 78
// so).  With ANY rows may begin at any element and end inside V: sixteen bytes are then read and written wherever they lie,
// over a row's end into what follows, but never beyond the last row's (`last`: its last V elements), and settle(), where
// the elements are first needed, brings in order what lies there.
template <class T, int V, bool ANY>
struct alignas(V * sizeof(T)) Piece {
  T e[V];
  __device__ __forceinline__ void load(const T* row, int c, int cols, const T* last) {
    const T* at = row + (c < cols ? c : cols - V);
    if constexpr (ANY)
      __builtin_memcpy(e, at < last ? at : last, sizeof(e));
    else
      *this = *reinterpret_cast<const Piece*>(at);
  }
  __device__ __forceinline__ void settle(const T* row, int c, int cols, const T* last) {
    if constexpr (ANY) {
      if (c + V > cols) {
        if (c < cols && row + c > last) {
#pragma unroll
          for (int i = 0; i < V; ++i) e[i] = c + i < cols ? row[c + i] : static_cast<T>(0.0f);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) e[i] = c + i < cols ? e[i] : static_cast<T>(0.0f);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = c < cols ? e[i] : static_cast<T>(0.0f);
    }
  }
  __device__ __forceinline__ void store(T* row, int c, int cols) const {
    if (c + V <= cols) {
      if constexpr (ANY)
        __builtin_memcpy(row + c, e, sizeof(e));
      else
        *reinterpret_cast<Piece*>(row + c) = *this;
    } else if constexpr (ANY) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < cols) row[c + i] = e[i];
    }
  }
};

// V float32 weights from column c on, `other` where there are none.  They may lie anywhere in a flat vector.
template <int V>
__device__ __forceinline__ void load_weights(float (&out)[V], const float* w, int c, int cols, float other) {
  if (w && V % 4 == 0 && (reinterpret_cast<uintptr_t>(w) & 15) == 0 && c + V <= cols) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(w + c + i);
      out[i] = v.x;
      out[i + 1 < V ? i + 1 : 0] = v.y;
      out[i + 2 < V ? i + 2 : 0] = v.z;
      out[i + 3 < V ? i + 3 : 0] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = w && c + i < cols ? w[c + i] : other;
  }
}

// Rows blockIdx.x, blockIdx.x + gridDim.x, .. (times the rows a block has); the next row is on its way while one is summed.
template <class T, int V, bool ANY, int TPR, int E>
__global__ __launch_bounds__(NormShape<TPR>::kThreads) void k_norm_forward(
    const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols, const float* __restrict__ gamma,
    const float* __restrict__ beta, float eps, T* __restrict__ y, int64_t y_stride, float* __restrict__ mean_out,
    float* __restrict__ rstd_out) {
  constexpr int R = E / V;
  __shared__ float room[2 * (TPR / 64) + 2];
  const int t = threadIdx.x % TPR;
  const float inv = 1.0f / static_cast<float>(cols);
  const int64_t step = (int64_t)gridDim.x * NormShape<TPR>::kRows;
  int64_t row = (int64_t)blockIdx.x * NormShape<TPR>::kRows + threadIdx.x / TPR;
  const T* last = x + (rows - 1) * x_stride + cols - V;
  Piece<T, V, ANY> next[R];
#pragma unroll
  for (int r = 0; r < R; ++r) next[r].load(x + (row < rows ? row : rows - 1) * x_stride, (r * TPR + t) * V, cols, last);
  float gm[R][V], bt[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    load_weights<V>(gm[r], gamma, (r * TPR + t) * V, cols, 1.0f);
    load_weights<V>(bt[r], beta, (r * TPR + t) * V, cols, 0.0f);
  }
  // (the rows of a block's waves end together or one turn apart: nobody waits for a wave that has left, since several
  // waves to a row share it)
  for (; row < rows; row += step) {
    float v[R][V];
    float s[1] = {0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      next[r].settle(x + row * x_stride, (r * TPR + t) * V, cols, last);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[r][i] = static_cast<float>(next[r].e[i]);
        s[0] += v[r][i];
      }
    }
    {
      const int64_t then = row + step < rows ? row + step : rows - 1;
#pragma unroll
      for (int r = 0; r < R; ++r) next[r].load(x + then * x_stride, (r * TPR + t) * V, cols, last);
    }
    row_sums<TPR>(s, room, 0);
    const float mean = s[0] * inv;
    float q[1] = {0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int c = (r * TPR + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) v[r][i] -= mean;
      if (c + V > cols) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (c + i >= cols) v[r][i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) q[0] = fmaf(v[r][i], v[r][i], q[0]);
    }
    row_sums<TPR>(q, room, 1);
    const float rstd = 1.0f / sqrtf(fmaf(q[0], inv, eps));
    if (t == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      Piece<T, V, ANY> o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.e[i] = static_cast<T>(fmaf(v[r][i] * rstd, gm[r][i], bt[r][i]));
      o.store(y + row * y_stride, (r * TPR + t) * V, cols);
    }
  }
}

// Rows longer than a block's registers: three passes over the row, the later two mostly from caches.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_forward_long(
    const T* __restrict__ x, int64_t x_stride, int64_t rows, int64_t cols, const float* __restrict__ gamma,
    const float* __restrict__ beta, float eps, T* __restrict__ y, int64_t y_stride, float* __restrict__ mean_out,
    float* __restrict__ rstd_out) {
  __shared__ float room[2 * 16];
  const float inv = 1.0f / static_cast<float>(cols);
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* xr = x + row * x_stride;
    T* yr = y + row * y_stride;
    float s[1] = {0.0f}, q[1] = {0.0f};
    for (int64_t c = threadIdx.x; c < cols; c += 1024) s[0] += static_cast<float>(xr[c]);
    row_sums<1024>(s, room, 0);
    const float mean = s[0] * inv;
    for (int64_t c = threadIdx.x; c < cols; c += 1024) {
      const float d = static_cast<float>(xr[c]) - mean;
      q[0] = fmaf(d, d, q[0]);
    }
    row_sums<1024>(q, room, 1);
    const float rstd = 1.0f / sqrtf(fmaf(q[0], inv, eps));
    if (threadIdx.x == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
    for (int64_t c = threadIdx.x; c < cols; c += 1024) {
      const float h = (static_cast<float>(xr[c]) - mean) * rstd;
      yr[c] = static_cast<T>(fmaf(h, gamma ? gamma[c] : 1.0f, beta ? beta[c] : 0.0f));
    }
  }
}

// The weights' gradients of 64 columns over all rows, by one block of NT threads: its waves take every NT / 64-th row.
template <class T, int NT>
__device__ void norm_columns(int64_t c0, const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t rows, int cols,
                             const float* mean, const float* rstd, const GradOut& g, float* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = c0 + lane;
  float a = 0.0f, b = 0.0f;
  if (c < cols)
#pragma unroll 8
    for (int64_t row = wave; row < rows; row += NT / 64) {
      const float d = static_cast<float>(dy[row * dy_stride + c]);
      a = fmaf(d, (static_cast<float>(x[row * x_stride + c]) - mean[row]) * rstd[row], a);
      b += d;
    }
  room[wave * 128 + lane] = a;
  room[wave * 128 + 64 + lane] = b;
  __syncthreads();
  if (wave < 2 && c < cols) {  // wave 0 dgamma, wave 1 dbeta
    float s = 0.0f;
    for (int i = 0; i < NT / 64; ++i) s += room[i * 128 + wave * 64 + lane];
    g.put(wave, c, s);
  }
}

// The backward pass over rows blockIdx.x, blockIdx.x + row_blocks, ..; the block's share of the weight gradients goes to
// part[0][blockIdx.x][..] (dgamma) and part[1][blockIdx.x][..] (dbeta), rows of `cols`.  Blocks from row_blocks on, if there
// are such, take 64 columns each instead and write their weights' gradients whole: few rows are read a second time sooner
// than a second launch adds up shares (then `part` is NULL).
template <class T, int V, bool ANY, int TPR, int E>
__global__ __launch_bounds__(NormShape<TPR>::kThreads) void k_norm_backward(
    const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols,
    const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd,
    T* __restrict__ dx, int64_t dx_stride, float* __restrict__ part, int row_blocks, GradOut grads) {
  constexpr int R = E / V;
  constexpr int kRows = NormShape<TPR>::kRows;
  constexpr int kRoomRows = kRows > 1 ? 2 * kRows * TPR * E : 4 * (TPR / 64);
  constexpr int kRoomCols = NormShape<TPR>::kThreads / 64 * 128;
  constexpr int kRoom = kRoomRows > kRoomCols ? kRoomRows : kRoomCols;
  __shared__ float room[kRoom];
  if ((int)blockIdx.x >= row_blocks) {
    norm_columns<T, NormShape<TPR>::kThreads>((int64_t)(blockIdx.x - row_blocks) * 64, dy, dy_stride, x, x_stride, rows, cols,
                                              mean, rstd, grads, room);
    return;
  }
  const int t = threadIdx.x % TPR;
  const float inv = 1.0f / static_cast<float>(cols);
  const int64_t step = (int64_t)row_blocks * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  const T *last_x = x + (rows - 1) * x_stride + cols - V, *last_d = dy + (rows - 1) * dy_stride + cols - V;
  Piece<T, V, ANY> next_x[R], next_d[R];
  float next_mu = 0.0f, next_rs = 0.0f;
  auto ask = [&](int64_t of) {
    if (of >= rows) of = rows - 1;  // (not used)
    next_mu = mean[of];
    next_rs = rstd[of];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      next_x[r].load(x + of * x_stride, (r * TPR + t) * V, cols, last_x);
      next_d[r].load(dy + of * dy_stride, (r * TPR + t) * V, cols, last_d);
    }
  };
  // (with wide loads the second row's registers cost more waves than it gains: 32768 x 2048 bf16 81 us, 78 without)
  constexpr bool kAhead = V == 1;
  if (kAhead) ask(row);
  float dg[R][V], db[R][V], gm[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    load_weights<V>(gm[r], gamma, (r * TPR + t) * V, cols, 1.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) dg[r][i] = db[r][i] = 0.0f;
  }
  int turn = 0;
  for (; row < rows; row += step) {
    if (!kAhead) ask(row);
    float h[R][V], d[R][V];
    const float mu = next_mu, rs = next_rs;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      // Behind the row's end d is zero, and nothing may come of h there: it is the row's last piece's, or zero where that is not
      // known ((0 - mu) rs may be beyond float32).
      if constexpr (ANY) next_x[r].settle(x + row * x_stride, (r * TPR + t) * V, cols, last_x);
      next_d[r].settle(dy + row * dy_stride, (r * TPR + t) * V, cols, last_d);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        d[r][i] = static_cast<float>(next_d[r].e[i]);
        h[r][i] = (static_cast<float>(next_x[r].e[i]) - mu) * rs;
      }
      if (ANY && (r * TPR + t) * V + V > cols) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if ((r * TPR + t) * V + i >= cols) h[r][i] = 0.0f;
      }
    }
    if (kAhead) ask(row + step);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dg[r][i] = fmaf(d[r][i], h[r][i], dg[r][i]);
        db[r][i] += d[r][i];
        d[r][i] *= gm[r][i];
        s[0] += d[r][i];
        s[1] = fmaf(d[r][i], h[r][i], s[1]);
      }
    if (!dx) continue;
    row_sums<TPR>(s, room, turn);
    turn ^= 1;
    const float m1 = s[0] * inv, m2 = s[1] * inv;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      Piece<T, V, ANY> o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.e[i] = static_cast<T>(rs * (d[r][i] - fmaf(h[r][i], m2, m1)));
      o.store(dx + row * dx_stride, (r * TPR + t) * V, cols);
    }
  }
  if (!part) return;
  float* pg = part + (int64_t)blockIdx.x * cols;
  float* pb = pg + (int64_t)row_blocks * cols;
  if constexpr (kRows > 1) {
    const int mine = threadIdx.x / TPR;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = (r * TPR + t) * V + i;
        room[mine * (TPR * E) + c] = dg[r][i];
        room[(kRows + mine) * (TPR * E) + c] = db[r][i];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += NormShape<TPR>::kThreads) {
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        a += room[j * (TPR * E) + c];
        b += room[(kRows + j) * (TPR * E) + c];
      }
      pg[c] = a;
      pb[c] = b;
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int c = (r * TPR + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < cols) {
          pg[c + i] = dg[r][i];
          pb[c + i] = db[r][i];
        }
    }
  }
}

// Rows longer than a block's registers: dx, two passes over the row ...
template <class T>
__global__ __launch_bounds__(1024) void k_norm_backward_long(
    const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride, int64_t rows, int64_t cols,
    const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd,
    T* __restrict__ dx, int64_t dx_stride) {
  __shared__ float room[4 * 16];
  const float inv = 1.0f / static_cast<float>(cols);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* xr = x + row * x_stride;
    const T* dr = dy + row * dy_stride;
    const float mu = mean[row], rs = rstd[row];
    float s[2] = {0.0f, 0.0f};
    for (int64_t c = threadIdx.x; c < cols; c += 1024) {
      const float h = (static_cast<float>(xr[c]) - mu) * rs;
      const float d = static_cast<float>(dr[c]) * (gamma ? gamma[c] : 1.0f);
      s[0] += d;
      s[1] = fmaf(d, h, s[1]);
    }
    row_sums<1024>(s, room, turn);
    turn ^= 1;
    const float m1 = s[0] * inv, m2 = s[1] * inv;
    for (int64_t c = threadIdx.x; c < cols; c += 1024) {
      const float h = (static_cast<float>(xr[c]) - mu) * rs;
      const float d = static_cast<float>(dr[c]) * (gamma ? gamma[c] : 1.0f);
      dx[row * dx_stride + c] = static_cast<T>(rs * (d - fmaf(h, m2, m1)));
    }
  }
}

// ... and the weight gradients: 256 columns a block, one share of the rows for each blockIdx.y.
template <class T>
__global__ __launch_bounds__(256) void k_norm_backward_cols(
    const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride, int64_t rows, int64_t cols,
    const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ part) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float a = 0.0f, b = 0.0f;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const float h = (static_cast<float>(x[row * x_stride + c]) - mean[row]) * rstd[row];
    const float d = static_cast<float>(dy[row * dy_stride + c]);
    a = fmaf(d, h, a);
    b += d;
  }
  part[(int64_t)blockIdx.y * cols + c] = a;
  part[((int64_t)gridDim.y + blockIdx.y) * cols + c] = b;
}

// Sums the blocks' shares column by column, blockIdx.y = 0 dgamma, 1 dbeta; 64 columns a block at a time, each of whose sixteen
// waves takes every sixteenth share.
__global__ __launch_bounds__(1024) void k_norm_join(const float* __restrict__ part, int shares, int64_t cols, GradOut grads) {
  __shared__ float room[16][64];
  if (!grads.wanted(blockIdx.y)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* p = part + (int64_t)blockIdx.y * shares * cols;
  for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < cols; c0 += (int64_t)gridDim.x * 64) {
    const int64_t c = c0 + lane;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 16
      for (int j = wave; j < shares; j += 16) s += p[(int64_t)j * cols + c];
    room[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
#pragma unroll
      for (int i = 1; i < 16; ++i) s += room[i][lane];
      grads.put(blockIdx.y, c, s);
    }
    __syncthreads();  // read before the next columns' sums
  }
}

}  // namespace artopk
