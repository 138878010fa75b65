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
// float32, in an order that depends on the sizes alone.
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

template <class T, int V, int TPR, int E>
__global__ __launch_bounds__(NormShape<TPR>::kThreads) void k_norm_forward(
    const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols, const float* __restrict__ gamma,
    const float* __restrict__ beta, float eps, T* __restrict__ y, int64_t y_stride, float* __restrict__ mean_out,
    float* __restrict__ rstd_out) {
  constexpr int R = E / V;
  __shared__ float room[2 * (TPR / 64) + 2];
  const int t = threadIdx.x % TPR;
  const float inv = 1.0f / static_cast<float>(cols);
  float gm[R][V], bt[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int c = (r * TPR + t) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      gm[r][i] = gamma && c < cols ? gamma[c + i] : 1.0f;
      bt[r][i] = beta && c < cols ? beta[c + i] : 0.0f;
    }
  }
  for (int64_t row0 = (int64_t)blockIdx.x * NormShape<TPR>::kRows; row0 < rows;
       row0 += (int64_t)gridDim.x * NormShape<TPR>::kRows) {
    const int64_t row = row0 + threadIdx.x / TPR;
    const bool there = row < rows;  // (whole waves; with several waves to a row always)
    const T* xr = x + row * x_stride;
    float v[R][V];
    float s[1] = {0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int c = (r * TPR + t) * V;
      if (there && c < cols) {
        load_elems<V>(v[r], xr + c);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[r][i] = 0.0f;
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += v[r][i];
    row_sums<TPR>(s, room, 0);
    const float mean = s[0] * inv;
    float q[1] = {0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if ((r * TPR + t) * V < cols) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          v[r][i] -= mean;
          q[0] = fmaf(v[r][i], v[r][i], q[0]);
        }
      }
    }
    row_sums<TPR>(q, room, 1);
    const float rstd = 1.0f / sqrtf(fmaf(q[0], inv, eps));
    if (!there) continue;
    if (t == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
    T* yr = y + row * y_stride;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int c = (r * TPR + t) * V;
      if (c < cols) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float h = v[r][i] * rstd;
          o[i] = fmaf(h, gm[r][i], bt[r][i]);
        }
        store_elems<V>(yr + c, o);
      }
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

// The backward pass over rows blockIdx.x, blockIdx.x + gridDim.x, ..; the block's share of the weight gradients goes
// to part[0][blockIdx.x][..] (dgamma) and part[1][blockIdx.x][..] (dbeta), rows of `cols`.
template <class T, int V, int TPR, int E>
__global__ __launch_bounds__(NormShape<TPR>::kThreads) void k_norm_backward(
    const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride, int64_t rows, int cols,
    const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd,
    T* __restrict__ dx, int64_t dx_stride, float* __restrict__ part) {
  constexpr int R = E / V;
  constexpr int kRows = NormShape<TPR>::kRows;
  constexpr int kRoom = kRows > 1 ? 2 * kRows * TPR * E : 4 * (TPR / 64);
  __shared__ float room[kRoom];
  const int t = threadIdx.x % TPR;
  const float inv = 1.0f / static_cast<float>(cols);
  float dg[R][V], db[R][V], gm[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int c = (r * TPR + t) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dg[r][i] = db[r][i] = 0.0f;
      gm[r][i] = c < cols ? (gamma ? gamma[c + i] : 1.0f) : 0.0f;
    }
  }
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < rows; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = row0 + threadIdx.x / TPR;
    const bool there = row < rows;
    float h[R][V], d[R][V];
    const float mu = there ? mean[row] : 0.0f, rs = there ? rstd[row] : 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int c = (r * TPR + t) * V;
      if (there && c < cols) {
        load_elems<V>(h[r], x + row * x_stride + c);
        load_elems<V>(d[r], dy + row * dy_stride + c);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) h[r][i] = d[r][i] = 0.0f;
      }
    }
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (there && (r * TPR + t) * V < cols) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          h[r][i] = (h[r][i] - mu) * rs;
          dg[r][i] = fmaf(d[r][i], h[r][i], dg[r][i]);
          db[r][i] += d[r][i];
          d[r][i] *= gm[r][i];
          s[0] += d[r][i];
          s[1] = fmaf(d[r][i], h[r][i], s[1]);
        }
      }
    }
    if (!dx) continue;
    row_sums<TPR>(s, room, turn);
    turn ^= 1;
    const float m1 = s[0] * inv, m2 = s[1] * inv;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int c = (r * TPR + t) * V;
      if (there && c < cols) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = rs * (d[r][i] - fmaf(h[r][i], m2, m1));
        store_elems<V>(dx + row * dx_stride + c, o);
      }
    }
  }
  if (!part) return;
  float* pg = part + (int64_t)blockIdx.x * cols;
  float* pb = pg + (int64_t)gridDim.x * cols;
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
      if (c < cols) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          pg[c + i] = dg[r][i];
          pb[c + i] = db[r][i];
        }
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

// Sums the blocks' shares column by column, blockIdx.y = 0 dgamma, 1 dbeta; 64 columns a block, whose four waves take
// a quarter of the shares each.  `add` adds to what out holds, in float32.
template <class G>
__global__ __launch_bounds__(256) void k_norm_join(const float* __restrict__ part, int shares, int64_t cols,
                                                   G* __restrict__ dgamma, G* __restrict__ dbeta, int add) {
  __shared__ float room[4][64];
  G* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  const float* p = part + (int64_t)blockIdx.y * shares * cols;
  float s = 0.0f;
  if (c < cols)
#pragma unroll 8
    for (int j = wave; j < shares; j += 4) s += p[(int64_t)j * cols + c];
  room[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    s = (room[0][lane] + room[1][lane]) + (room[2][lane] + room[3][lane]);
    if (add) s += static_cast<float>(out[c]);
    out[c] = static_cast<G>(s);
  }
}

}  // namespace artopk
