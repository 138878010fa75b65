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
#include "lanes.h"

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
  float quick;  // second moments from here on take the quick square root and reciprocal: 2^-96, or infinity for a large eps
};

// 32 random bits of a place: two rounds of multiplying and folding the upper bits onto the lower ones.  The factors are odd whole
// numbers next to 2^32 times the golden ratio's and the roots of 2 and 3's fractions.
__device__ __forceinline__ uint32_t adam_random(uint32_t place, uint32_t key) {
  uint32_t x = place * 0x9E3779B1u + key;
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// Four codes of a word as values; e, the block's exponent field, is the same in all lanes.
__device__ __forceinline__ void decode1(float (&m)[4], uint32_t codes, int e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = i < 3 ? codes << (20 - 8 * i) : codes >> 4;  // the code in bits 20 to 27
    m[i] = ldexpf(__uint_as_float((c & 0x07f00000u) | (c << 4 & 0x80000000u)), e - kTop1);
  }
  if (e == 255)
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __builtin_nanf("");
}
__device__ __forceinline__ void decode2(float (&v)[4], uint32_t codes, int e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = i < 3 ? codes << (20 - 8 * i) : codes >> 4;
    v[i] = ldexpf(__uint_as_float(c & 0x0ff00000u), e - kTop2);
  }
  if (e == 255)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_nanf("");
}

// The top bytes of four words as one.
__device__ __forceinline__ uint32_t top_bytes(const uint32_t (&x)[4]) {
  const uint32_t lo = __builtin_amdgcn_perm(x[1], x[0], 0x0c0c0703), hi = __builtin_amdgcn_perm(x[3], x[2], 0x07030c0c);
  return lo | hi;
}

// `e` is the block's exponent field, at least top + 1 (so that field 1 is a normal number); the random bits' lower half.
__device__ __forceinline__ uint32_t encode1(const float (&m)[4], int e, const uint32_t (&random)[4]) {
  uint32_t x[4];
  bool low = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t bits = __float_as_uint(m[i]), t = (bits & 0x7fffffffu) - ((uint32_t)(e - kTop1) << 23);
    low |= (int32_t)t < 1 << 23;
    x[i] = ((t + ((random[i] & 0xffffu) << 4 | 8u)) << 4 & 0x7fffffffu) | (bits & 0x80000000u);
  }
  if (__any(low)) {  // steps of field 0; rare: below 2^-13 of the block's largest
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bits = __float_as_uint(m[i]), mag = bits & 0x7fffffffu;
      if ((int32_t)mag - (int32_t)((uint32_t)(e - kTop1) << 23) < 1 << 23) {
        const uint32_t rnd = (random[i] & 0xffffu) << 4 | 8u;
        const uint32_t code = (uint32_t)fmaf((float)rnd, 0x1p-20f, ldexpf(__uint_as_float(mag), 127 + kTop1 + 2 - e));
        x[i] = (code > 8 ? 8 : code) << 24 | (bits & 0x80000000u);
      }
    }
  }
  return top_bytes(x);
}
// The same for the second moment, by the upper half.
__device__ __forceinline__ uint32_t encode2(const float (&v)[4], int e, const uint32_t (&random)[4]) {
  uint32_t x[4];
  bool low = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = __float_as_uint(v[i]) - ((uint32_t)(e - kTop2) << 23);
    low |= (int32_t)t < 1 << 23;
    x[i] = (t + ((random[i] >> 12 & 0xffff0u) | 8u)) << 4;
  }
  if (__any(low))
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((int32_t)(__float_as_uint(v[i]) - ((uint32_t)(e - kTop2) << 23)) < 1 << 23) x[i] = v[i] != 0.0f ? 8u << 24 : 0;
  return top_bytes(x);
}

// Four elements; at a place of their type only by get and put (words at once: of single elements the compiler may make
// single loads).
template <class T>
struct alignas(4 * sizeof(T)) Four {
  T e[4];
  typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t Words2 __attribute__((ext_vector_type(2), aligned(2)));
  using Words = std::conditional_t<sizeof(T) == 4, Words4, Words2>;
  __device__ __forceinline__ void get(const T* p) {
    const Words w = *reinterpret_cast<const Words*>(p);
    __builtin_memcpy(e, &w, sizeof(e));
  }
  __device__ __forceinline__ void put(T* p) const {
    Words w;
    __builtin_memcpy(&w, e, sizeof(e));
    *reinterpret_cast<Words*>(p) = w;
  }
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
  constexpr int kAhead = CODES ? 2 : 1;  // blocks a wave has under way
  const AdamChunk chunk = chunks[blockIdx.x];
  if (later) terms = *later;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float rate = terms.rate * chunk.factor, keep = 1.0f - f.eta * chunk.factor * chunk.decay;
  for (int b0 = wave * (kAdamBlocks / 4); b0 < (wave + 1) * (kAdamBlocks / 4) && b0 * kAdamBlock < chunk.count; b0 += kAhead) {
    Four<T> in_w[kAhead];
    Four<float> in_g[kAhead], in_m[kAhead], in_v[kAhead];
    uint32_t in_c1[kAhead], in_c2[kAhead];
    int in_e[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      // (blocks behind the tensor's end: its last one again, which is not written)
      const int b = (b0 + q) * kAdamBlock < chunk.count ? b0 + q : (chunk.count - 1) / kAdamBlock, n = chunk.count - b * kAdamBlock;
      const uint32_t block = chunk.block + b;
      const int64_t at = chunk.at + b * kAdamBlock + lane * 4;
      if (n >= kAdamBlock || lane * 4 + 4 <= n) {
        in_w[q].get(weights + at);
        in_g[q].get(update + at);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          in_w[q].e[i] = lane * 4 + i < n ? weights[at + i] : static_cast<T>(0.0f);
          in_g[q].e[i] = lane * 4 + i < n ? update[at + i] : 0.0f;
        }
      }
      const size_t word = (size_t)block * (kAdamBlock / 4) + lane;
      if constexpr (CODES) {
        in_c1[q] = static_cast<const uint32_t*>(first)[word];
        in_c2[q] = static_cast<const uint32_t*>(second)[word];
        in_e[q] = reinterpret_cast<const uint16_t*>(scales)[block];
      } else {
        in_m[q] = static_cast<const Four<float>*>(first)[word];
        in_v[q] = static_cast<const Four<float>*>(second)[word];
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // (all loads go out before one is waited for)
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int b = b0 + q, n = chunk.count - b * kAdamBlock - lane * 4;  // elements from the lane's first on
      if (b * kAdamBlock >= chunk.count) break;
      const uint32_t block = chunk.block + b;
      const int64_t at = chunk.at + b * kAdamBlock + lane * 4;
      const size_t word = (size_t)block * (kAdamBlock / 4) + lane;
      float w[4], m[4], v[4];
      if constexpr (CODES) {
        const int e = __builtin_amdgcn_readfirstlane(in_e[q]);
        decode1(m, in_c1[q], e & 255);
        decode2(v, in_c2[q], e >> 8);
      }
      bool tiny = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = in_g[q].e[i] * f.scale;
        m[i] = (CODES ? m[i] : in_m[q].e[i]) * f.b1 + x * f.c1;
        v[i] = (CODES ? v[i] : in_v[q].e[i]) * f.b2 + (x * x) * f.c2;
        w[i] = static_cast<float>(in_w[q].e[i]) * keep;
        tiny |= v[i] < f.quick;
      }
      if (__any(tiny)) {  // (the quick square root and reciprocal neither take nor give numbers below the normal ones)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = fmaf(-rate, m[i] / fmaf(sqrtf(v[i]), terms.root, f.eps), w[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = fmaf(-rate, m[i] * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[i]), terms.root, f.eps)), w[i]);
      }
      if (n >= 4) {
        Four<T> o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.e[i] = static_cast<T>(w[i]);
        o.put(weights + at);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i < n) weights[at + i] = static_cast<T>(w[i]);
          else m[i] = v[i] = 0.0f;  // (places behind the tensor's end hold zeros)
        }
      }
      if constexpr (CODES) {
        uint32_t big1 = 0, big2 = 0, random[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a = __float_as_uint(m[i]) & 0x7fffffffu, d = __float_as_uint(v[i]) & 0x7fffffffu;
          big1 = a > big1 ? a : big1;
          big2 = d > big2 ? d : big2;
          random[i] = adam_random((uint32_t)word * 4 + i, terms.key);
        }
        int e1 = (int)(wave_max(big1) >> 23), e2 = (int)(wave_max(big2) >> 23);
        e1 = e1 > kTop1 + 1 ? e1 : kTop1 + 1;
        e2 = e2 > kTop2 + 1 ? e2 : kTop2 + 1;
        static_cast<uint32_t*>(first)[word] = encode1(m, e1, random);
        static_cast<uint32_t*>(second)[word] = encode2(v, e2, random);
        if (lane == 0) reinterpret_cast<uint16_t*>(scales)[block] = (uint16_t)(e1 | e2 << 8);
      } else {
        Four<float> o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.e[i] = m[i];
        static_cast<Four<float>*>(first)[word] = o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.e[i] = v[i];
        static_cast<Four<float>*>(second)[word] = o;
      }
    }
  }
}

// Moments of 8 bits as values: blockIdx.y = 0 the first, 1 the second.  A wave takes four blocks at a time.
template <class T>
__global__ __launch_bounds__(256) void k_adamw_values(const uint32_t* __restrict__ first, const uint32_t* __restrict__ second,
                                                      const uint8_t* __restrict__ scales, int64_t blocks, T* __restrict__ first_out,
                                                      T* __restrict__ second_out) {
  const int lane = threadIdx.x & 63;
  const bool one = blockIdx.y == 0;
  const uint32_t* codes = one ? first : second;
  T* out = one ? first_out : second_out;
  if (!out) return;
  for (int64_t b = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 4; b < blocks; b += (int64_t)gridDim.x * 16) {
    uint32_t c[4];
    int e[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t from = b + q < blocks ? b + q : blocks - 1;
      c[q] = codes[from * (kAdamBlock / 4) + lane];
      e[q] = scales[2 * from + (one ? 0 : 1)];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (b + q >= blocks) break;
      float v[4];
      const int at = __builtin_amdgcn_readfirstlane(e[q]);
      if (one) decode1(v, c[q], at); else decode2(v, c[q], at);
      Four<T> o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o.e[i] = static_cast<T>(v[i]);
      reinterpret_cast<Four<T>*>(out)[(b + q) * (kAdamBlock / 4) + lane] = o;
    }
  }
}

}  // namespace artopk
