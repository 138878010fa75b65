// AdamW over many tensors of a flat vector, moments in 32 or 8 bits, for gfx950.
//
//   g = s update,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2
//   w <- w (1 - eta decay) - (eta / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: 28 bytes an element with float32 weights and moments of 32 bits, 16 with 8 bits (12 for 16-bit weights).
//
// Moments of 8 bits.  The 256 elements of a block (of one tensor; its last block may be shorter) share E, the largest exponent
// field among them, one byte for each moment.  A code is an exponent field f and three bits of mantissa b:
//   f > 0: 2^(f - top + E - 127) (1 + b / 8),   f = 0: 2^(1 - top + E - 127) b / 8,
// the first moment with a sign in front, four bits of f and top = 14, the second with five bits and top = 30.  Rounding is up with
// the probability of what is cut off, by 16 bits from a hash of the step, the caller's seed and the place: the second moment
// moves by 1 - b2 = 0.001 of itself a step and codes are a sixteenth to an eighth apart, so rounded to nearest it would never
// move, while so its mean is exact.  top + 1 is free for what is rounded up beyond the block's largest, whose mean is exact, too.
// A second moment that is not zero does not become zero (its element would move by m / eps): the least is f = 1, b = 0.
// E = 255 (infinity or NaN somewhere in the block) stands for NaN throughout the block.
#pragma once

#include "elements.h"

namespace artopk {

constexpr int kAdamBlock = 256;      // elements that share an exponent: four for each lane of a wave
constexpr int kAdamBlocks = 16;      // blocks a workgroup takes, four a wave
constexpr int kTop1 = 14, kTop2 = 30;

// What a workgroup works on: up to kAdamBlocks blocks of one tensor.
struct AdamChunk {
  int64_t at;       // first element in the flat vector
  uint32_t block;   // first block of the moments
  int32_t count;    // elements
  float factor, decay;
};

// What changes from step to step.
struct AdamTerms {
  float rate;       // eta / (1 - b1^t)
  float root;       // 1 / sqrt(1 - b2^t)
  uint32_t key;     // of the random bits
};

struct AdamFixed {
  float scale, eta, b1, c1, b2, c2, eps;  // c1 = 1 - b1, c2 = 1 - b2, each rounded once
};

// 32 random bits of a place: two rounds of multiplying and folding the upper bits onto the lower ones.  The factors are odd whole
// numbers next to 2^32 times the golden ratio's and the roots of 2 and 3's fractions.
__device__ __forceinline__ uint32_t adam_random(uint32_t place, uint32_t key) {
  uint32_t x = place * 0x9E3779B1u + key;
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ float decode1(uint32_t code, int e) {
  if (e == 255) return __builtin_nanf("");
  return ldexpf(__uint_as_float((code & 127) << 20 | (code & 128) << 24), e - kTop1);
}
__device__ __forceinline__ float decode2(uint32_t code, int e) {
  if (e == 255) return __builtin_nanf("");
  return ldexpf(__uint_as_float(code << 20), e - kTop2);
}

// `e` is the block's exponent field, at least top + 1 (so that field 1 is a normal number); `half` 16 random bits.
__device__ __forceinline__ uint32_t encode1(float m, int e, uint32_t half) {
  const uint32_t bits = __float_as_uint(m), mag = bits & 0x7fffffffu, rnd = half << 4 | 8;
  const int32_t t = (int32_t)mag - ((e - kTop1) << 23);
  const float step = ldexpf(__uint_as_float(mag), 127 + kTop1 + 2 - e);  // in steps of field 0
  uint32_t low = (uint32_t)fmaf((float)rnd, 0x1p-20f, step);
  low = low > 8 ? 8 : low;
  return (t >= 1 << 23 ? (uint32_t)(t + (int32_t)rnd) >> 20 : low) | (bits >> 31) << 7;
}
__device__ __forceinline__ uint32_t encode2(float v, int e, uint32_t half) {
  const uint32_t bits = __float_as_uint(v), rnd = half << 4 | 8;
  const int32_t t = (int32_t)bits - ((e - kTop2) << 23);
  return t >= 1 << 23 ? (uint32_t)(t + (int32_t)rnd) >> 20 : bits ? 8u : 0u;
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint32_t o = __shfl_xor(v, off, 64);
    v = o > v ? o : v;
  }
  return v;
}

template <class T>
struct alignas(4 * sizeof(T)) Four {
  T e[4];
};

// Steps a counter on the device and works out the step's terms, for steps that are replayed from a graph.
__global__ void k_adamw_terms(int64_t* counter, AdamTerms* out, double eta, double b1, double b2, uint64_t seed) {
  const int64_t t = *counter + 1;
  *counter = t;
  out->rate = (float)(eta / (1.0 - pow(b1, (double)t)));
  out->root = (float)(1.0 / sqrt(1.0 - pow(b2, (double)t)));
  const uint64_t wide = seed + (uint64_t)t * 0x9E3779B97F4A7C15ull;
  out->key = (uint32_t)(wide ^ (wide >> 32));
}

__global__ void k_adamw_counter(int64_t* counter, int64_t value) { *counter = value; }

template <class T, bool CODES>
__global__ __launch_bounds__(256) void k_adamw(const AdamChunk* __restrict__ chunks, T* __restrict__ weights,
                                               const float* __restrict__ update, void* __restrict__ first,
                                               void* __restrict__ second, uint8_t* __restrict__ scales, AdamFixed f, AdamTerms terms,
                                               const AdamTerms* __restrict__ later) {
  const AdamChunk chunk = chunks[blockIdx.x];
  if (later) terms = *later;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float rate = terms.rate * chunk.factor, keep = 1.0f - f.eta * chunk.factor * chunk.decay;
#pragma unroll
  for (int q = 0; q < kAdamBlocks / 4; ++q) {
    const int b = wave * (kAdamBlocks / 4) + q, c = b * kAdamBlock + lane * 4;
    if (b * kAdamBlock >= chunk.count) continue;
    const uint32_t block = chunk.block + b;
    const int64_t place = (int64_t)block * kAdamBlock + lane * 4;
    const int64_t at = chunk.at + c;
    const int n = chunk.count - c;  // elements from here on
    float w[4], g[4], m[4], v[4];
    if (n >= 4) {
      Four<T> x;
      Four<float> u;
      __builtin_memcpy(&x, weights + at, sizeof(x));
      __builtin_memcpy(&u, update + at, sizeof(u));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = static_cast<float>(x.e[i]);
        g[i] = u.e[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = i < n ? static_cast<float>(weights[at + i]) : 0.0f;
        g[i] = i < n ? update[at + i] : 0.0f;
      }
    }
    if constexpr (CODES) {
      const uint32_t c1 = static_cast<const uint32_t*>(first)[place >> 2], c2 = static_cast<const uint32_t*>(second)[place >> 2];
      const int e1 = scales[2 * (size_t)block], e2 = scales[2 * (size_t)block + 1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[i] = decode1(c1 >> (8 * i) & 255, e1);
        v[i] = decode2(c2 >> (8 * i) & 255, e2);
      }
    } else {
      const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(first) + place);
      const float4 d = *reinterpret_cast<const float4*>(static_cast<const float*>(second) + place);
      m[0] = a.x, m[1] = a.y, m[2] = a.z, m[3] = a.w;
      v[0] = d.x, v[1] = d.y, v[2] = d.z, v[3] = d.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = g[i] * f.scale;
      m[i] = m[i] * f.b1 + x * f.c1;
      v[i] = v[i] * f.b2 + (x * x) * f.c2;
      const float way = m[i] / fmaf(sqrtf(v[i]), terms.root, f.eps);
      w[i] = fmaf(-rate, way, w[i] * keep);
    }
    if (n >= 4) {
      Four<T> x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x.e[i] = static_cast<T>(w[i]);
      __builtin_memcpy(weights + at, &x, sizeof(x));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < n) weights[at + i] = static_cast<T>(w[i]);
        else m[i] = v[i] = 0.0f;  // (places behind the tensor's end hold zeros)
      }
    }
    if constexpr (CODES) {
      uint32_t big1 = 0, big2 = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(m[i]) & 0x7fffffffu, d = __float_as_uint(v[i]) & 0x7fffffffu;
        big1 = a > big1 ? a : big1;
        big2 = d > big2 ? d : big2;
      }
      int e1 = (int)(wave_max_u32(big1) >> 23), e2 = (int)(wave_max_u32(big2) >> 23);
      e1 = e1 > kTop1 + 1 ? e1 : kTop1 + 1;
      e2 = e2 > kTop2 + 1 ? e2 : kTop2 + 1;
      uint32_t c1 = 0, c2 = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t r = adam_random((uint32_t)place + i, terms.key);
        c1 |= encode1(m[i], e1, r & 0xffff) << (8 * i);
        c2 |= encode2(v[i], e2, r >> 16) << (8 * i);
      }
      static_cast<uint32_t*>(first)[place >> 2] = c1;
      static_cast<uint32_t*>(second)[place >> 2] = c2;
      if (lane == 0) {
        scales[2 * (size_t)block] = (uint8_t)e1;
        scales[2 * (size_t)block + 1] = (uint8_t)e2;
      }
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(first) + place) = make_float4(m[0], m[1], m[2], m[3]);
      *reinterpret_cast<float4*>(static_cast<float*>(second) + place) = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
}

// Moments of 8 bits as values.
template <class T>
__global__ __launch_bounds__(256) void k_adamw_values(const uint32_t* __restrict__ first, const uint32_t* __restrict__ second,
                                                      const uint8_t* __restrict__ scales, int64_t blocks, T* __restrict__ first_out,
                                                      T* __restrict__ second_out) {
  const int lane = threadIdx.x & 63;
  for (int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); b < blocks; b += (int64_t)gridDim.x * 4) {
    const int64_t place = b * kAdamBlock + lane * 4;
    Four<T> o;
    if (first_out) {
      const uint32_t c = first[place >> 2];
      const int e = scales[2 * b];
#pragma unroll
      for (int i = 0; i < 4; ++i) o.e[i] = static_cast<T>(decode1(c >> (8 * i) & 255, e));
      *reinterpret_cast<Four<T>*>(first_out + place) = o;
    }
    if (second_out) {
      const uint32_t c = second[place >> 2];
      const int e = scales[2 * b + 1];
#pragma unroll
      for (int i = 0; i < 4; ++i) o.e[i] = static_cast<T>(decode2(c >> (8 * i) & 255, e));
      *reinterpret_cast<Four<T>*>(second_out + place) = o;
    }
  }
}

}  // namespace artopk
