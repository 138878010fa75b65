// Host side of the AdamW entry points: argument checks, the table of what each workgroup works on, launches.

#include "artopk.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <new>
#include <vector>

#include "adamw_kernels.h"
#include "host_common.h"

using namespace artopk;

struct artopk_adamw {
  hipStream_t stream = nullptr;
  int device = 0;
  int64_t n = 0, elems = 0;
  int32_t type = 0, bits = 32;
  unsigned chunk_count = 0;
  uint8_t* slab = nullptr;
  AdamChunk* chunks = nullptr;  // within the slab, and what a counted step needs
  AdamTerms* terms = nullptr;
  int64_t* counter = nullptr;
  char err[kErrText] = {0};
};

namespace {

// A handle's memory and stream belong to the device that was current when it was made.
int check_device(char* err, int device) {
  int now = -1;
  if (hipGetDevice(&now) != hipSuccess || now != device)
    return fail_text(err, ARTOPK_EINVAL, "the current device is %d, the handle's %d", now, device);
  return ARTOPK_OK;
}

constexpr int64_t kMostTensors = 65535;
constexpr int64_t kChunk = kAdamBlock * kAdamBlocks;

#define ADAMW_TRY(h, expr)                                                                                     \
  do {                                                                                                         \
    hipError_t e_ = (expr);                                                                                    \
    if (e_ != hipSuccess)                                                                                      \
      return fail_text((h)->err, ARTOPK_EHIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, \
                       __LINE__);                                                                              \
  } while (0)

// Elements of the moments, or -1 with the reason in the error text of calls without a handle.
int64_t checked_elems(const artopk_tensor* tensors, int32_t count, int64_t n) {
  auto bad = [](const char* what, int i) {
    fail_text(g_noctx_err, ARTOPK_EINVAL, "tensor %d: %s", i, what);
    return (int64_t)-1;
  };
  if (!tensors || count < 1 || count > kMostTensors) {
    fail_text(g_noctx_err, ARTOPK_EINVAL, "tensors is NULL, or %d of them are outside [1, %lld]", count, (long long)kMostTensors);
    return -1;
  }
  if (n < 1 || n >= (1ll << 31)) {
    fail_text(g_noctx_err, ARTOPK_EINVAL, "n=%lld outside [1, 2^31)", (long long)n);
    return -1;
  }
  int64_t elems = 0;
  for (int i = 0; i < count; ++i) {
    const artopk_tensor& t = tensors[i];
    if (t.count < 1 || t.count > n || t.offset < 0 || t.offset > n - t.count) return bad("not within the vector", i);
    if (!std::isfinite(t.eta_scale) || !std::isfinite(t.decay)) return bad("eta_scale or decay is not finite", i);
    elems += (t.count + kAdamBlock - 1) / kAdamBlock * kAdamBlock;
  }
  return elems;
}

// Whether no two tensors overlap.
int check_apart(const artopk_tensor* tensors, int32_t count) {
  std::vector<std::pair<int64_t, int64_t>> places;
  places.reserve(count);
  for (int i = 0; i < count; ++i) places.emplace_back(tensors[i].offset, tensors[i].count);
  std::sort(places.begin(), places.end());
  for (int i = 1; i < count; ++i)
    if (places[i - 1].first + places[i - 1].second > places[i].first)
      return fail_text(g_noctx_err, ARTOPK_EINVAL, "two tensors overlap at element %lld", (long long)places[i].first);
  return ARTOPK_OK;
}

int64_t chunks_of(const artopk_tensor* tensors, int32_t count) {
  int64_t c = 0;
  for (int i = 0; i < count; ++i) c += (tensors[i].count + kChunk - 1) / kChunk;
  return c;
}

// No exception leaves an entry point.
template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  } catch (...) {
    return fail_text(g_noctx_err, ARTOPK_EHIP, "unexpected exception");
  }
}

int create(artopk_adamw** out, const artopk_tensor* tensors, int32_t count, int64_t n, int32_t type, int32_t bits, void* stream) {
  const int64_t elems = checked_elems(tensors, count, n);
  if (elems < 0) return ARTOPK_EINVAL;
  if (!known_type(type)) return fail_text(g_noctx_err, ARTOPK_EINVAL, "unknown element type %d", type);
  if (bits != 32 && bits != 8) return fail_text(g_noctx_err, ARTOPK_EINVAL, "moments of %d bits: 32 or 8 are taken", bits);
  int rc;
  if ((rc = check_apart(tensors, count))) return rc;
  std::vector<AdamChunk> chunks;
  chunks.reserve((size_t)chunks_of(tensors, count));
  uint32_t block = 0;
  for (int i = 0; i < count; ++i) {
    const artopk_tensor& t = tensors[i];
    for (int64_t at = 0; at < t.count; at += kChunk)
      chunks.push_back({t.offset + at, block + (uint32_t)(at / kAdamBlock), (int32_t)std::min<int64_t>(kChunk, t.count - at),
                        t.eta_scale, t.decay});
    block += (uint32_t)((t.count + kAdamBlock - 1) / kAdamBlock);
  }
  artopk_adamw* h = new (std::nothrow) artopk_adamw();
  if (!h) return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  h->stream = reinterpret_cast<hipStream_t>(stream);
  h->n = n;
  h->elems = elems;
  h->type = type;
  h->bits = bits;
  h->chunk_count = (unsigned)chunks.size();
  const size_t table = align_up(chunks.size() * sizeof(AdamChunk), 256);
  void* p = nullptr;
  hipError_t e = hipGetDevice(&h->device);
  if (e != hipSuccess) {
    delete h;
    return fail_text(g_noctx_err, ARTOPK_EHIP, "no device: %s", hipGetErrorString(e));
  }
  e = hipMalloc(&p, table + 512);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "hipMalloc failed: %s", hipGetErrorString(e));
  }
  h->slab = static_cast<uint8_t*>(p);
  h->chunks = reinterpret_cast<AdamChunk*>(h->slab);
  h->terms = reinterpret_cast<AdamTerms*>(h->slab + table);
  h->counter = reinterpret_cast<int64_t*>(h->slab + table + 256);
  const int64_t zero = 0;
  e = hipMemcpy(h->chunks, chunks.data(), chunks.size() * sizeof(AdamChunk), hipMemcpyHostToDevice);
  if (e == hipSuccess) e = hipMemcpy(h->counter, &zero, sizeof(zero), hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipFree(p);
    delete h;
    return fail_text(g_noctx_err, ARTOPK_EHIP, "hipMemcpy failed: %s", hipGetErrorString(e));
  }
  *out = h;
  return ARTOPK_OK;
}

int check_moments(artopk_adamw* h, const void* first, const void* second, const void* scales) {
  if (!first || !second) return fail_text(h->err, ARTOPK_EINVAL, "first or second is NULL");
  if (!aligned16(first) || !aligned16(second)) return fail_text(h->err, ARTOPK_EINVAL, "first or second is not 16-byte aligned");
  if (h->bits == 8 && !scales) return fail_text(h->err, ARTOPK_EINVAL, "scales is NULL");
  if (h->bits != 8 && scales) return fail_text(h->err, ARTOPK_EINVAL, "scales is given for moments of 32 bits");
  if (!aligned16(scales)) return fail_text(h->err, ARTOPK_EINVAL, "scales is not 16-byte aligned");
  return ARTOPK_OK;
}

}  // namespace

int64_t artopk_adamw_state_elems(const artopk_tensor* tensors, int32_t count, int64_t n) {
  const int64_t elems = checked_elems(tensors, count, n);
  return elems < 0 || guarded([&] { return check_apart(tensors, count); }) ? -1 : elems;
}

int64_t artopk_adamw_scratch_bytes(const artopk_tensor* tensors, int32_t count, int64_t n) {
  if (artopk_adamw_state_elems(tensors, count, n) < 0) return -1;
  return (int64_t)(align_up((size_t)chunks_of(tensors, count) * sizeof(AdamChunk), 256) + 512);
}

int artopk_adamw_create(artopk_adamw** out, const artopk_tensor* tensors, int32_t count, int64_t n, int32_t type, int32_t state_bits,
                        void* hip_stream) {
  if (!out) return fail_text(g_noctx_err, ARTOPK_EINVAL, "out is NULL");
  return guarded([&] { return create(out, tensors, count, n, type, state_bits, hip_stream); });
}

int artopk_adamw_destroy(artopk_adamw* h) {
  if (!h) return ARTOPK_EINVAL;
  if (h->slab) (void)hipFree(h->slab);
  delete h;
  return ARTOPK_OK;
}

const char* artopk_adamw_last_error(const artopk_adamw* h) { return h ? h->err : g_noctx_err; }

int artopk_adamw_set_step(artopk_adamw* h, int64_t step) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_adamw_set_step: handle is NULL");
  if (step < 0) return fail_text(h->err, ARTOPK_EINVAL, "step is negative");
  int rc;
  if ((rc = check_device(h->err, h->device))) return rc;
  k_adamw_counter<<<1, 1, 0, h->stream>>>(h->counter, step);
  ADAMW_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_adamw_step(artopk_adamw* h, void* weights, const float* update, void* first, void* second, uint8_t* scales, int64_t step,
                      float update_scale, float eta, double beta1, double beta2, float eps, uint64_t seed) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_adamw_step: handle is NULL");
  int rc;
  if ((rc = check_device(h->err, h->device))) return rc;
  if (!weights || !update) return fail_text(h->err, ARTOPK_EINVAL, "weights or update is NULL");
  const size_t size = elem_size(h->type);
  if (reinterpret_cast<uintptr_t>(weights) % size) return fail_text(h->err, ARTOPK_EINVAL, "weights is not aligned to its elements");
  if (reinterpret_cast<uintptr_t>(update) % 4) return fail_text(h->err, ARTOPK_EINVAL, "update is not aligned to its elements");
  if ((rc = check_moments(h, first, second, scales))) return rc;
  if (step < 0) return fail_text(h->err, ARTOPK_EINVAL, "step is negative");
  if (!std::isfinite(update_scale) || !std::isfinite(eta)) return fail_text(h->err, ARTOPK_EINVAL, "update_scale or eta is not finite");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail_text(h->err, ARTOPK_EINVAL, "beta1 or beta2 is outside [0, 1)");
  if (!(eps > 0.0f) || !std::isfinite(eps)) return fail_text(h->err, ARTOPK_EINVAL, "eps is not positive and finite");
  {
    const size_t moment = (size_t)h->elems * (h->bits / 8);
    RangeSet rs;
    rs.add(weights, (size_t)h->n * size, true, "weights");
    rs.add(update, (size_t)h->n * 4, false, "update");
    rs.add(first, moment, true, "first");
    rs.add(second, moment, true, "second");
    rs.add(scales, (size_t)h->elems / kAdamBlock * 2, true, "scales");
    if ((rc = rs.check(h->err))) return rc;
  }
  const AdamFixed f = {update_scale, eta, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), eps,
                       // (the root's part of the divisor stays below 2^92, so eps alone can make its reciprocal that small)
                       eps > 0x1p100f ? INFINITY : 0x1p-96f};
  AdamTerms terms = {0.0f, 0.0f, 0};
  const AdamTerms* later = nullptr;
  if (step > 0) {
    terms.rate = (float)((double)eta / (1.0 - std::pow(beta1, (double)step)));
    terms.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    const uint64_t wide = seed + (uint64_t)step * 0x9E3779B97F4A7C15ull;
    terms.key = (uint32_t)(wide ^ (wide >> 32));
  } else {
    k_adamw_terms<<<1, 1, 0, h->stream>>>(h->counter, h->terms, (double)eta, beta1, beta2, seed);
    later = h->terms;
  }
  auto go = [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    if (h->bits == 8)
      k_adamw<T, true><<<h->chunk_count, 256, 0, h->stream>>>(h->chunks, static_cast<T*>(weights), update, first, second, scales, f,
                                                              terms, later);
    else
      k_adamw<T, false><<<h->chunk_count, 256, 0, h->stream>>>(h->chunks, static_cast<T*>(weights), update, first, second, nullptr, f,
                                                               terms, later);
  };
  if (h->type == ARTOPK_G_F32) go((float*)nullptr);
  else if (h->type == ARTOPK_G_BF16) go((__bf16*)nullptr);
  else go((_Float16*)nullptr);
  ADAMW_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_adamw_values(artopk_adamw* h, const void* first, const void* second, const uint8_t* scales, int32_t type, void* first_out,
                        void* second_out) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_adamw_values: handle is NULL");
  int rc;
  if ((rc = check_device(h->err, h->device))) return rc;
  if (h->bits != 8) return fail_text(h->err, ARTOPK_EINVAL, "moments of 32 bits are values already");
  if ((rc = check_moments(h, first, second, scales))) return rc;
  if (type != ARTOPK_G_F32 && type != ARTOPK_G_BF16)
    return fail_text(h->err, ARTOPK_EINVAL, "values of type %d: float32 or bfloat16 hold them all", type);
  if (!first_out && !second_out) return fail_text(h->err, ARTOPK_EINVAL, "first_out and second_out are NULL");
  if (!aligned16(first_out) || !aligned16(second_out))
    return fail_text(h->err, ARTOPK_EINVAL, "first_out or second_out is not 16-byte aligned");
  {
    RangeSet rs;
    rs.add(first, (size_t)h->elems, false, "first");
    rs.add(second, (size_t)h->elems, false, "second");
    rs.add(scales, (size_t)h->elems / kAdamBlock * 2, false, "scales");
    rs.add(first_out, (size_t)h->elems * elem_size(type), true, "first_out");
    rs.add(second_out, (size_t)h->elems * elem_size(type), true, "second_out");
    if ((rc = rs.check(h->err))) return rc;
  }
  const int64_t blocks = h->elems / kAdamBlock;
  auto go = [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    k_adamw_values<T><<<dim3((unsigned)std::min<int64_t>((blocks + 15) / 16, 1 << 20), 2), 256, 0, h->stream>>>(
        static_cast<const uint32_t*>(first), static_cast<const uint32_t*>(second), scales, blocks, static_cast<T*>(first_out),
        static_cast<T*>(second_out));
  };
  if (type == ARTOPK_G_F32) go((float*)nullptr);
  else go((__bf16*)nullptr);
  ADAMW_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}
