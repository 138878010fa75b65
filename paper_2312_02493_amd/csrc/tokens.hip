// Host side of the token entry points (embedding and log probabilities): argument checks, the choice of a kernel's shape, launches.

#include "artopk.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "host_common.h"
#include "logprobs_kernels.h"

using namespace artopk;

struct artopk_tokens {
  hipStream_t stream = nullptr;
  int device = 0;
  int num_cu = 256;
  int64_t max_tokens = 0, max_vocab = 0, max_width = 0;
  uint8_t* slab = nullptr;
  // within the slab: sorted tokens and their places (two of each, one pass reads what the other wrote), how often tiles have
  // digits, shares of heavy tokens' sums, the error word
  uint32_t *key[2] = {nullptr, nullptr}, *pos[2] = {nullptr, nullptr}, *counts = nullptr;
  float* part = nullptr;
  uint8_t* marks = nullptr;  // rows of a table that are named; zeros between calls
  LogpPart* parts = nullptr;     // of rows that several blocks share, and their alternatives
  uint64_t* part_keys = nullptr;
  HeavyToken* heavy = nullptr;
  uint32_t* heavy_count = nullptr;
  int* error = nullptr;
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

static_assert(kMostTop == ARTOPK_MAX_TOP, "");

constexpr int64_t kMostWidth = 65536;
constexpr int64_t kMostBlocks = 1 << 20;

#define TOKENS_TRY(h, expr)                                                                                    \
  do {                                                                                                         \
    hipError_t e_ = (expr);                                                                                    \
    if (e_ != hipSuccess)                                                                                      \
      return fail_text((h)->err, ARTOPK_EHIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, \
                       __LINE__);                                                                              \
  } while (0)

constexpr int64_t kNarrowRow = 512, kSomeTop = 56, kShortRow = 2048, kLongerRow = 16384, kManyRows = 2048;
static_assert(kNarrowRow / 2 >= RowRun<__bf16>::V, "k_logp's rows have a whole piece");
constexpr int64_t kPartBlocks = 1024;  // that parts of rows make, at most
constexpr int64_t kFewTokens = 8192, kFewTokensAlone = 14336;  // (at most what LDS holds beside the counts, 14336 keys)

bool valid_limits(int64_t max_tokens, int64_t max_vocab, int64_t max_width) {
  return max_tokens >= 1 && max_tokens < (1ll << 31) && max_vocab >= 1 && max_vocab < (1ll << 31) && max_width >= 1 &&
         max_width <= kMostWidth;
}

int64_t runs_of(int64_t count) { return (count + kSumRun - 1) / kSumRun; }

struct Layout {
  size_t key[2], pos[2], counts, part, marks, heavy, parts, part_keys, error, bytes;
  Layout(int64_t tokens, int64_t vocab, int64_t width) {
    size_t at = 0;
    auto take = [&](size_t n) {
      const size_t here = at;
      at = align_up(at + n, 256);
      return here;
    };
    for (int i = 0; i < 2; ++i) {
      key[i] = take((size_t)tokens * 4);
      pos[i] = take((size_t)tokens * 4);
    }
    counts = take((size_t)kSortTiles * kSortDigits * 4);
    part = tokens > kSumMost ? take((size_t)runs_of(tokens) * 2 * (size_t)part_pitch(width) * 4) : 0;
    marks = tokens > kFewTokens ? take((size_t)vocab) : 0;
    heavy = take((size_t)(tokens / kSumMost + 1) * sizeof(HeavyToken));
    parts = take((size_t)kPartBlocks * sizeof(LogpPart));
    part_keys = take((size_t)kPartBlocks * kMostTop * 8);
    error = take(8);  // and the list's length
    bytes = at;
  }
};

int check_vector(char* err, const char* name, const void* p, size_t size) {
  if (reinterpret_cast<uintptr_t>(p) % size) return fail_text(err, ARTOPK_EINVAL, "%s is not aligned to its elements", name);
  return ARTOPK_OK;
}

int check_tokens(artopk_tokens* h, const void* tokens, int32_t bits, int64_t count, int64_t vocab) {
  int rc;
  if ((rc = check_device(h->err, h->device))) return rc;
  if (count < 0 || count > h->max_tokens)
    return fail_text(h->err, ARTOPK_EINVAL, "%lld tokens are outside [0, %lld]", (long long)count, (long long)h->max_tokens);
  if (vocab < 1 || vocab > h->max_vocab)
    return fail_text(h->err, ARTOPK_EINVAL, "vocab=%lld outside [1, %lld]", (long long)vocab, (long long)h->max_vocab);
  if (bits != 32 && bits != 64) return fail_text(h->err, ARTOPK_EINVAL, "tokens of %d bits: 32 or 64 are taken", bits);
  return check_vector(h->err, "tokens", tokens, bits / 8);
}

int check_scale(artopk_tokens* h, float scale) {
  if (!std::isfinite(scale)) return fail_text(h->err, ARTOPK_EINVAL, "scale is not finite");
  return ARTOPK_OK;
}

// Of log probabilities.  Below 2^-120 an element counts though its difference from the row's peak may be beyond float32 (2^128 scaled
// is at least 256 otherwise, and e^-256 is zero there); above 2^127, scale log2(e) may be.
int check_logp_scale(artopk_tokens* h, float scale) {
  if (!(scale >= 0x1p-120f && scale <= 0x1p127f)) return fail_text(h->err, ARTOPK_EINVAL, "scale=%g outside [2^-120, 2^127]", scale);
  return ARTOPK_OK;
}

template <class TT, class TY, int V>
void embed(artopk_tokens* h, const TT* table, int64_t table_stride, int64_t vocab, int64_t cols, const Tokens& tokens, int64_t count,
           float scale, TY* y, int64_t y_stride) {
  const int64_t pieces = (cols + V - 1) / V;
  int lg = 0;
  while (lg < 6 && (kEmbedPieces << lg) < pieces) ++lg;
  const int64_t tiles = (pieces + (kEmbedPieces << lg) - 1) / (kEmbedPieces << lg), per = 64 >> lg;
  const int64_t units = (count + per - 1) / per * tiles;
  const unsigned blocks = (unsigned)std::min<int64_t>((units + 3) / 4, kMostBlocks);
  k_embed<TT, TY, V><<<blocks, 256, 0, h->stream>>>(table, table_stride, vocab, tokens, count, cols, scale, y, y_stride, lg, units,
                                                    tiles, h->error);
}

// Bytes of zeros that a launch of the sort writes beside its own work: as much as took no longer than that did where it was measured,
// 32768 tokens of 2048 columns into 64000 rows of float32 (48 MB instead of 80 beside the placing: 152 us in all, so 146).  The
// sort takes longer with more tokens, and could write more there; more tokens are correct but not tuned for.
constexpr int64_t kBesideCount = 32 << 20, kBesidePlace = 80 << 20;
constexpr int64_t kFewZeros = 16 << 20;   // up to here the sums' launch writes them all
constexpr int64_t kZeroShare = 64 << 10;  // and a block of the sums' launch
constexpr int64_t kSumBlocks = 4096;      // of it, to be reached where columns can be shared
constexpr int kZeroBlocks = 448;  // with the sort's own two on a compute unit

// Sorts the places of `count` tokens by token; the result is in key[r], pos[r], r returned.  `zero` are the table's rows that
// have to be zeros, of which some are written on the way; those left are in it afterwards.
int sort_places(artopk_tokens* h, const Tokens& tokens, int64_t count, int64_t vocab, ZeroRows& zero) {
  // (with zeros to write beside them the passes cost nothing more)
  if (count <= (zero.at ? kFewTokens : kFewTokensAlone)) {
    const SortKeys in = {tokens, nullptr, nullptr, (uint32_t)vocab, 1, h->heavy_count, nullptr};
    auto go = [&](auto B) {
      constexpr int kParts = kSortThreads / B();
      const int each = (int)((count + 4 * kParts - 1) / (4 * kParts) * 4);
      k_sort_few<B()><<<(unsigned)((count + B() - 1) / B()), kSortThreads, (size_t)each * kParts * 4, h->stream>>>(
          in, (int)count, h->key[0], h->pos[0], h->error);
    };
    if (count <= kFewTokens) go(std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 64>());
    zero.key = h->key[0];
    zero.count = count;
    return 0;
  }
  int all = 1;
  while (vocab >> all) ++all;  // bits of 0 .. vocab, which stands for no token
  const int passes = (all + kSortBits - 1) / kSortBits;
  const int keys = count <= 131072 ? 1 : 4;  // a thread has in a round
  const int64_t round = kSortThreads * keys;
  const int64_t per = std::max<int64_t>(1, (count + round * kSortTiles - 1) / (round * kSortTiles)) * round;
  const int tiles = (int)((count + per - 1) / per);
  const bool beside_sort = zero.at && zero.end * zero.bytes >= kFewZeros;
  zero.marks = beside_sort ? h->marks : nullptr;
  int64_t next = 0;
  auto beside = [&](int64_t bytes) {
    ZeroRows z = zero;
    if (beside_sort) {
      z.begin = next;
      z.end = next = std::min(zero.end, next + std::max<int64_t>(1, bytes / z.bytes));
    }
    return z;
  };
  int from = 1, shift = 0;
  for (int pass = 0; pass < passes; ++pass) {
    const int bits = (all - shift + passes - pass - 1) / (passes - pass);
    const SortKeys in = {tokens, h->key[from], h->pos[from], (uint32_t)vocab, pass == 0, h->heavy_count, zero.marks ? h->marks : nullptr};
    // (the first launch finds out which rows are named)
    const bool fill = beside_sort && pass > 0;
    k_sort_count<<<tiles + (fill ? kZeroBlocks : 0), kSortThreads, 0, h->stream>>>(in, count, per, shift, bits, tiles, h->counts,
                                                                                  h->error, fill ? beside(kBesideCount) : zero);
    auto go = [&](auto R) {
      k_sort_place<R()><<<tiles + (beside_sort ? kZeroBlocks : 0), kSortThreads, 0, h->stream>>>(
          in, count, per, shift, bits, h->counts, tiles, h->key[1 - from], h->pos[1 - from], beside(kBesidePlace));
    };
    if (keys == 1) go(std::integral_constant<int, 1>());
    else go(std::integral_constant<int, 4>());
    shift += bits;
    from = 1 - from;
  }
  zero.begin = next;
  if (!beside_sort) {
    zero.key = h->key[from];
    zero.count = count;
  }
  return from;
}

template <class TD, class TG, int V, bool ONCE>
void embed_sums(artopk_tokens* h, const uint32_t* key, const uint32_t* pos, int64_t count, int64_t vocab, const TD* dy,
                int64_t dy_stride, int64_t cols, float scale, TG* dtable, int64_t grad_stride, int add, const ZeroRows& zero) {
  const int tiles = (int)((cols + 64 * V - 1) / (64 * V));
  const int64_t rows = zero.at ? std::max<int64_t>(0, zero.end - zero.begin) : 0;
  // (of narrow rows two rounds of the block's lanes: looking up whether a row is named takes longer than its zeros:
  // 500 tokens, 131072 rows of 4 bytes 62 us, so 14)
  const int64_t each = std::min<int64_t>(std::max<int64_t>(1, kZeroShare / std::max(1, zero.bytes)), 2 * kSumWaves * (64 >> zero.lg));
  const int zeros = (int)std::min<int64_t>((rows + each - 1) / each, 16384);
  const int64_t runs = runs_of(count);
  // as many blocks to a run as its tokens and column tiles can occupy, until there are enough of them
  const int most = (kSumRun / 4 * tiles + kSumWaves - 1) / kSumWaves;
  const int split = (int)std::max<int64_t>(1, std::min<int64_t>(most, kSumBlocks / std::max<int64_t>(1, runs)));
  const int64_t blocks = std::min<int64_t>(runs, kMostBlocks) * split;
  k_embed_sum<TD, TG, V, ONCE><<<(unsigned)(blocks + zeros), kSumWaves * 64, 0, h->stream>>>(
      key, pos, count, (uint32_t)vocab, dy, dy_stride, cols, scale, dtable, grad_stride, add, h->part, runs, split, tiles, h->heavy,
      h->heavy_count, zeros, zero);
}

}  // namespace

int64_t artopk_tokens_scratch_bytes(int64_t max_tokens, int64_t max_vocab, int64_t max_width) {
  if (!valid_limits(max_tokens, max_vocab, max_width)) return -1;
  return (int64_t)Layout(max_tokens, max_vocab, max_width).bytes;
}

int artopk_tokens_create(artopk_tokens** out, int64_t max_tokens, int64_t max_vocab, int64_t max_width, void* hip_stream) {
  if (!out) return fail_text(g_noctx_err, ARTOPK_EINVAL, "out is NULL");
  if (!valid_limits(max_tokens, max_vocab, max_width))
    return fail_text(g_noctx_err, ARTOPK_EINVAL,
                     "max_tokens=%lld and max_vocab=%lld have to be in [1, 2^31), max_width=%lld in [1, %lld]", (long long)max_tokens,
                     (long long)max_vocab, (long long)max_width, (long long)kMostWidth);
  artopk_tokens* h = new (std::nothrow) artopk_tokens();
  if (!h) return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  h->stream = reinterpret_cast<hipStream_t>(hip_stream);
  h->max_tokens = max_tokens;
  h->max_vocab = max_vocab;
  h->max_width = max_width;
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) {
    delete h;
    return fail_text(g_noctx_err, ARTOPK_EHIP, "no device: %s", hipGetErrorString(e));
  }
  if (cus > 0) h->num_cu = cus;
  h->device = dev;
  const Layout at(max_tokens, max_vocab, max_width);
  void* p = nullptr;
  e = hipMalloc(&p, at.bytes);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "hipMalloc failed: %s", hipGetErrorString(e));
  }
  h->slab = static_cast<uint8_t*>(p);
  for (int i = 0; i < 2; ++i) {
    h->key[i] = reinterpret_cast<uint32_t*>(h->slab + at.key[i]);
    h->pos[i] = reinterpret_cast<uint32_t*>(h->slab + at.pos[i]);
  }
  h->counts = reinterpret_cast<uint32_t*>(h->slab + at.counts);
  h->part = reinterpret_cast<float*>(h->slab + at.part);
  h->marks = h->slab + at.marks;
  h->parts = reinterpret_cast<LogpPart*>(h->slab + at.parts);
  h->part_keys = reinterpret_cast<uint64_t*>(h->slab + at.part_keys);
  h->heavy = reinterpret_cast<HeavyToken*>(h->slab + at.heavy);
  h->heavy_count = reinterpret_cast<uint32_t*>(h->slab + at.error) + 1;
  h->error = reinterpret_cast<int*>(h->slab + at.error);
  e = hipMemset(h->error, 0, sizeof(int));
  if (e == hipSuccess && max_tokens > kFewTokens) e = hipMemset(h->marks, 0, (size_t)max_vocab);
  if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
  if (e != hipSuccess) {
    (void)hipFree(h->slab);
    delete h;
    return fail_text(g_noctx_err, ARTOPK_EHIP, "hipMemset failed: %s", hipGetErrorString(e));
  }
  *out = h;
  return ARTOPK_OK;
}

int artopk_tokens_destroy(artopk_tokens* tokens) {
  if (!tokens) return ARTOPK_EINVAL;
  if (tokens->slab) (void)hipFree(tokens->slab);
  delete tokens;
  return ARTOPK_OK;
}

const char* artopk_tokens_last_error(const artopk_tokens* tokens) { return tokens ? tokens->err : g_noctx_err; }

int artopk_tokens_status(artopk_tokens* tokens) {
  if (!tokens) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_tokens_status: tokens is NULL");
  int rc;
  if ((rc = check_device(tokens->err, tokens->device))) return rc;  // (a NULL stream would be another device's)
  TOKENS_TRY(tokens, hipStreamSynchronize(tokens->stream));
  int word = 0;
  TOKENS_TRY(tokens, hipMemcpy(&word, tokens->error, sizeof(word), hipMemcpyDeviceToHost));
  if (!word) return ARTOPK_OK;
  const int zero = 0;
  TOKENS_TRY(tokens, hipMemcpy(tokens->error, &zero, sizeof(zero), hipMemcpyHostToDevice));
  return fail_text(tokens->err, ARTOPK_ESTATE, "a token was not below vocab");
}

int artopk_embedding_forward(artopk_tokens* h, const void* table, int64_t table_stride, int32_t table_type, int64_t vocab,
                             int64_t width, const void* tokens, int32_t token_bits, int64_t count, float scale, void* y,
                             int64_t y_stride, int32_t type) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_embedding_forward: handle is NULL");
  int rc;
  if (!known_type(type) || !known_type(table_type)) return fail_text(h->err, ARTOPK_EINVAL, "unknown element type");
  if ((rc = check_tokens(h, tokens, token_bits, count, vocab)) || (rc = check_scale(h, scale))) return rc;
  if (width < 1 || width > h->max_width)
    return fail_text(h->err, ARTOPK_EINVAL, "width=%lld outside [1, %lld]", (long long)width, (long long)h->max_width);
  if ((rc = check_rows(h->err, "table", table, table_stride, elem_size(table_type), vocab, width))) return rc;
  if ((rc = check_rows(h->err, "y", y, y_stride, elem_size(type), count, width))) return rc;
  if (!tokens && count > 0) return fail_text(h->err, ARTOPK_EINVAL, "tokens is NULL");
  {
    RowSet rs;
    rs.add(table, table_stride, vocab, width, elem_size(table_type), false, "table");
    rs.add(tokens, count, token_bits / 8, false, "tokens");
    rs.add(y, y_stride, count, width, elem_size(type), true, "y");
    if ((rc = rs.check(h->err))) return rc;
  }
  if (count == 0) return ARTOPK_OK;
  const Tokens tok = {tokens, token_bits == 64};
  with_type(table_type, [&](auto* tt) {
    using TT = std::remove_pointer_t<decltype(tt)>;
    with_type(type, [&](auto* ty) {
      using TY = std::remove_pointer_t<decltype(ty)>;
      constexpr int kWide = 16 / (sizeof(TT) < sizeof(TY) ? sizeof(TT) : sizeof(TY));
      auto go = [&](auto V) {
        embed<TT, TY, V()>(h, static_cast<const TT*>(table), table_stride, vocab, width, tok, count, scale, static_cast<TY*>(y),
                           y_stride);
      };
      if (width >= kWide) go(std::integral_constant<int, kWide>());
      else go(std::integral_constant<int, 1>());
    });
  });
  TOKENS_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_embedding_backward(artopk_tokens* h, const void* dy, int64_t dy_stride, int32_t type, const void* tokens,
                              int32_t token_bits, int64_t count, int64_t width, float scale, void* dtable, int64_t grad_stride,
                              int32_t grad_type, int64_t vocab, int32_t accumulate) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_embedding_backward: handle is NULL");
  int rc;
  if (!known_type(type) || !known_type(grad_type)) return fail_text(h->err, ARTOPK_EINVAL, "unknown element type");
  if ((rc = check_tokens(h, tokens, token_bits, count, vocab)) || (rc = check_scale(h, scale))) return rc;
  if (width < 1 || width > h->max_width)
    return fail_text(h->err, ARTOPK_EINVAL, "width=%lld outside [1, %lld]", (long long)width, (long long)h->max_width);
  if ((rc = check_rows(h->err, "dy", dy, dy_stride, elem_size(type), count, width))) return rc;
  if ((rc = check_rows(h->err, "dtable", dtable, grad_stride, elem_size(grad_type), vocab, width))) return rc;
  if (!tokens && count > 0) return fail_text(h->err, ARTOPK_EINVAL, "tokens is NULL");
  {
    RowSet rs;
    rs.add(dy, dy_stride, count, width, elem_size(type), false, "dy");
    rs.add(tokens, count, token_bits / 8, false, "tokens");
    rs.add(dtable, grad_stride, vocab, width, elem_size(grad_type), true, "dtable");
    if ((rc = rs.check(h->err))) return rc;
  }
  const Tokens tok = {tokens, token_bits == 64};
  ZeroRows zero = {};
  if (!accumulate) {
    zero.at = static_cast<uint8_t*>(dtable);
    zero.pitch = grad_stride * (int64_t)elem_size(grad_type);
    zero.bytes = (int32_t)(width * (int64_t)elem_size(grad_type));
    zero.end = vocab;
    while (zero.lg < 6 && (64 << zero.lg) < zero.bytes) ++zero.lg;
  }
  int sorted = 0;
  if (count > 0) sorted = sort_places(h, tok, count, vocab, zero);
  with_type(grad_type, [&](auto* tg) {
    using TG = std::remove_pointer_t<decltype(tg)>;
    TG* out = static_cast<TG*>(dtable);
    if (count == 0 && accumulate) return;
    with_type(type, [&](auto* td) {
      using TD = std::remove_pointer_t<decltype(td)>;
      constexpr int kWide = 16 / sizeof(TD);
      auto go = [&](auto V, auto ONCE) {
        embed_sums<TD, TG, V(), ONCE()>(h, h->key[sorted], h->pos[sorted], count, vocab, static_cast<const TD*>(dy), dy_stride, width,
                                        scale, out, grad_stride, accumulate != 0, zero);
      };
      using Wide = std::integral_constant<int, kWide>;
      if (width < kWide) go(std::integral_constant<int, 1>(), std::false_type());
      else if (width % kWide == 0 && aligned16(dy) && dy_stride % kWide == 0) go(Wide(), std::true_type());
      else go(Wide(), std::false_type());
    });
    if (count <= kSumMost) return;
    const unsigned tiles = (unsigned)((width + 255) / 256);
    const unsigned groups = (unsigned)std::max<int64_t>(1, std::min<int64_t>(count / kSumMost, 2 * h->num_cu / tiles));
    k_embed_join<TG><<<dim3(groups, tiles), 1024, 0, h->stream>>>(h->part, vocab, width, scale, out, grad_stride, accumulate != 0,
                                                                  h->heavy, h->heavy_count, zero.marks ? h->marks : nullptr);
  });
  TOKENS_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_token_logprobs(artopk_tokens* h, const void* logits, int64_t stride, int32_t type, int64_t rows, int64_t vocab,
                          const void* tokens, int32_t token_bits, float scale, float* logp_out, float* peak_out, float* logsum_out,
                          float* entropy_out, int32_t top, int32_t* top_ids_out, float* top_logp_out) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_token_logprobs: handle is NULL");
  int rc;
  if (!known_type(type)) return fail_text(h->err, ARTOPK_EINVAL, "unknown element type %d", type);
  if ((rc = check_tokens(h, tokens, token_bits, rows, vocab)) || (rc = check_logp_scale(h, scale))) return rc;
  if ((rc = check_rows(h->err, "logits", logits, stride, elem_size(type), rows, vocab))) return rc;
  if (logp_out && !tokens && rows > 0) return fail_text(h->err, ARTOPK_EINVAL, "tokens is NULL");
  if (top < 0 || top > ARTOPK_MAX_TOP || top > vocab)
    return fail_text(h->err, ARTOPK_EINVAL, "top=%d outside [0, %d] or more than vocab", top, ARTOPK_MAX_TOP);
  if (top && rows > 0 && (!top_ids_out || !top_logp_out))
    return fail_text(h->err, ARTOPK_EINVAL, "top_ids_out or top_logp_out is NULL");
  if (rows > 0 && !logp_out && !peak_out && !logsum_out && !entropy_out && !top)
    return fail_text(h->err, ARTOPK_EINVAL, "nothing is asked for");
  if ((rc = check_vector(h->err, "logp_out", logp_out, 4)) || (rc = check_vector(h->err, "peak_out", peak_out, 4)) ||
      (rc = check_vector(h->err, "logsum_out", logsum_out, 4)) || (rc = check_vector(h->err, "entropy_out", entropy_out, 4)) ||
      (rc = check_vector(h->err, "top_ids_out", top_ids_out, 4)) || (rc = check_vector(h->err, "top_logp_out", top_logp_out, 4)))
    return rc;
  {
    RowSet rs;
    rs.add(logits, stride, rows, vocab, elem_size(type), false, "logits");
    rs.add(tokens, rows, token_bits / 8, false, "tokens");
    rs.add(logp_out, rows, 4, true, "logp_out");
    rs.add(peak_out, rows, 4, true, "peak_out");
    rs.add(logsum_out, rows, 4, true, "logsum_out");
    rs.add(entropy_out, rows, 4, true, "entropy_out");
    rs.add(top ? top_ids_out : nullptr, rows * top, 4, true, "top_ids_out");
    rs.add(top ? top_logp_out : nullptr, rows * top, 4, true, "top_logp_out");
    if ((rc = rs.check(h->err))) return rc;
  }
  if (rows == 0) return ARTOPK_OK;
  const Tokens tok = {tokens, token_bits == 64};
  const LogpOut out = {logp_out, peak_out, logsum_out, entropy_out, top_ids_out, top_logp_out};
  with_type(type, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int V = RowRun<T>::V;
    const T* at = static_cast<const T*>(logits);
    const float c = scale * kLog2e;
    const int has_tokens = logp_out != nullptr;
    // Narrow rows four a wave, but some alternatives of 257 to 512 columns, which come faster all at once (8192 x 512 bfloat16: 8 14.3 us
    // and 17.3, 20 22.9 and 18.4, 57 48.8 and 34.7, 64 54 and 165) as long as the wave has keys
    // enough to bound them (8192 x 257, 48 with 33 keys: 42.6 and 161).
    if (vocab <= kNarrowRow / 2 || (vocab <= kNarrowRow && (top <= 8 || top > std::min(kSomeTop, vocab / V * 15 / 16)))) {
      const unsigned blocks = (unsigned)std::min<int64_t>((rows + 15) / 16, kMostBlocks);
      auto go = [&](auto PIECES, auto TOP) {
        k_logp_narrow<T, PIECES(), TOP()><<<blocks, 256, 0, h->stream>>>(at, stride, rows, (int)vocab, tok, has_tokens, scale, c, top, out,
                                                                         h->error);
      };
      auto with_top = [&](auto PIECES) {
        if (top) go(PIECES, std::true_type());
        else go(PIECES, std::false_type());
      };
      if (vocab <= 128) with_top(std::integral_constant<int, 8 / V>());
      else if (vocab <= 256) with_top(std::integral_constant<int, 16 / V>());
      else with_top(std::integral_constant<int, 32 / V>());
      return;
    }
    // Short rows a wave each, unless its 64 keys bound the alternatives badly (32768 x 1000 bfloat16: 50 93 us, 64 1020, by four
    // waves 216).  Few long ones in parts, as many as keep every compute unit busy, from sixteen pieces a thread on, where
    // that saves more than the second launch costs: 8 x 40000 bfloat16 14.3 us, so 11.1, 8 x 20000 8.1 and 11.3; 300 x 128000 36 and 25,
    // 400 x 100000 float32 33 and 35.
    const bool short_rows = top <= kSomeTop && (vocab <= kShortRow || (vocab <= kLongerRow && rows >= kManyRows));
    int split = 1;
    if (!short_rows && rows * 3 <= kPartBlocks && vocab / V / 256 >= 16)
      split = (int)std::max<int64_t>(1, std::min<int64_t>({64, kPartBlocks / rows, vocab / V / 256}));
    const int64_t units = short_rows ? (rows + 3) / 4 : rows * split;
    const unsigned blocks = (unsigned)std::min<int64_t>(units, kMostBlocks);
    auto go = [&](auto WAVES, auto TOP) {
      k_logp<T, WAVES(), TOP()><<<blocks, 256, 0, h->stream>>>(at, stride, rows, (int)vocab, tok, has_tokens, scale, c, top, out, split,
                                                               h->parts, h->part_keys, h->error);
    };
    auto with_top = [&](auto WAVES) {
      if (top) go(WAVES, std::true_type());
      else go(WAVES, std::false_type());
    };
    if (short_rows) with_top(std::integral_constant<int, 1>());
    else with_top(std::integral_constant<int, 4>());
    if (split > 1)
      k_logp_join<<<(unsigned)rows, 1024, 0, h->stream>>>(h->parts, h->part_keys, split, stride, logits, type, (int)vocab, tok, has_tokens,
                                                          scale, c, top, out, h->error);
  });
  TOKENS_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_token_logprobs_backward(artopk_tokens* h, const void* logits, int64_t stride, int32_t type, int64_t rows, int64_t vocab,
                                   const void* tokens, int32_t token_bits, float scale, const float* peak, const float* logsum,
                                   const float* entropy, const float* dlogp, const float* dlse, const float* dentropy,
                                   void* dlogits, int64_t dstride) {
  if (!h) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_token_logprobs_backward: handle is NULL");
  int rc;
  if (!known_type(type)) return fail_text(h->err, ARTOPK_EINVAL, "unknown element type %d", type);
  if ((rc = check_tokens(h, tokens, token_bits, rows, vocab)) || (rc = check_logp_scale(h, scale))) return rc;
  const size_t size = elem_size(type);
  if ((rc = check_rows(h->err, "logits", logits, stride, size, rows, vocab))) return rc;
  if ((rc = check_rows(h->err, "dlogits", dlogits, dstride, size, rows, vocab))) return rc;
  if (rows > 0 && (!peak || !logsum)) return fail_text(h->err, ARTOPK_EINVAL, "peak or logsum is NULL");
  if (rows > 0 && !dlogp && !dlse && !dentropy) return fail_text(h->err, ARTOPK_EINVAL, "dlogp, dlse and dentropy are all NULL");
  if (dlogp && !tokens && rows > 0) return fail_text(h->err, ARTOPK_EINVAL, "tokens is NULL");
  if (dentropy && !entropy && rows > 0) return fail_text(h->err, ARTOPK_EINVAL, "dentropy is given without entropy");
  const struct {
    const char* name;
    const float* p;
  } vectors[] = {{"peak", peak}, {"logsum", logsum}, {"entropy", entropy}, {"dlogp", dlogp}, {"dlse", dlse}, {"dentropy", dentropy}};
  RowSet rs;
  for (const auto& v : vectors) {
    if ((rc = check_vector(h->err, v.name, v.p, 4))) return rc;
    rs.add(v.p, rows, 4, false, v.name);
  }
  rs.add(tokens, rows, token_bits / 8, false, "tokens");
  // (in place: the same rows of the same matrix)
  const bool in_place = logits == dlogits && (rows <= 1 || stride == dstride);
  if (!in_place) rs.add(logits, stride, rows, vocab, size, false, "logits");
  rs.add(dlogits, dstride, rows, vocab, size, true, "dlogits");
  if ((rc = rs.check(h->err))) return rc;
  if (rows == 0) return ARTOPK_OK;
  const Tokens tok = {tokens, token_bits == 64};
  const LogpGrads in = {peak, logsum, entropy, dlogp, dlse, dentropy};
  // pieces of both at the same places within sixteen bytes
  const bool same = (reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(dlogits)) % 16 == 0 &&
                    (rows <= 1 || (stride - dstride) * (int64_t)size % 16 == 0);
  with_type(type, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int V = RowPieces<T>::V;
    // at most, wherever rows begin
    const bool whole = vocab % V == 0 && aligned16(logits) && (rows <= 1 || stride % V == 0);
    const int64_t pieces = whole ? vocab / V : (vocab + 2 * (V - 1)) / V;
    const int lanes = pieces <= 64 ? 16 : pieces <= 256 ? 64 : 256;
    const int tiles = lanes < 256 ? 1 : (int)((pieces + 1023) / 1024);
    const int64_t units = rows * tiles;
    const unsigned blocks = (unsigned)std::min<int64_t>((units * lanes + 255) / 256, kMostBlocks);
    auto go = [&](auto SAME, auto LANES) {
      k_logp_backward<T, SAME(), LANES()><<<blocks, 256, 0, h->stream>>>(static_cast<const T*>(logits), stride, rows, (int)vocab, tok,
                                                                         dlogp != nullptr, scale, scale * kLog2e, in,
                                                                         static_cast<T*>(dlogits), dstride, units, tiles, h->error);
    };
    auto with_lanes = [&](auto SAME) {
      if (lanes == 16) go(SAME, std::integral_constant<int, 16>());
      else if (lanes == 64) go(SAME, std::integral_constant<int, 64>());
      else go(SAME, std::integral_constant<int, 256>());
    };
    if (same) with_lanes(std::true_type());
    else with_lanes(std::false_type());
  });
  TOKENS_TRY(h, hipGetLastError());
  return ARTOPK_OK;
}
