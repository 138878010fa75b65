// Host side of the layer norm entry points: argument checks, the choice of a kernel's shape, launches.

#include "artopk.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "host_common.h"
#include "norm_kernels.h"

using namespace artopk;

struct artopk_norm {
  hipStream_t stream = nullptr;
  int num_cu = 256;
  int64_t max_rows = 0, max_cols = 0;
  float* part = nullptr;  // the blocks' shares of the weight gradients
  char err[kErrText] = {0};
};

namespace {

constexpr int64_t kRegisterCols = 16384;  // longest row that a block's registers hold
constexpr int kWaveCols = 512;        // what a wave's eight elements a lane hold
constexpr int kSingleCols = 8192;  // the same in the backward pass, taken one by one
constexpr int kMaxShares = 1024;          // blocks of a backward pass, at most
constexpr int kLongShares = 64;
constexpr int64_t kJoinBlocks = 1 << 20;  // a launch has fewer than 2^32 threads along an axis
constexpr int64_t kMostElems = 1ll << 46;  // between the first and the last row
// Up to this many rows, and elements, the weight gradients are summed column by column beside the rows' blocks.
constexpr int64_t kColumnRows = 512, kColumnElems = 1 << 20;

#define NORM_TRY(h, expr)                                                                                      \
  do {                                                                                                         \
    hipError_t e_ = (expr);                                                                                    \
    if (e_ != hipSuccess)                                                                                      \
      return fail_text((h)->err, ARTOPK_EHIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, \
                       __LINE__);                                                                              \
  } while (0)

bool valid_limits(int64_t max_rows, int64_t max_cols) {
  return max_rows >= 1 && max_rows < (1ll << 31) && max_cols >= 1 && max_cols < (1ll << 31);
}

int64_t shares_limit(int64_t max_rows, int64_t max_cols) {
  const int64_t most = max_cols > kRegisterCols ? kLongShares : kMaxShares;
  return max_rows < most ? max_rows : most;
}

// Floats of scratch; shorter rows than max_cols have more shares, but no more floats than the longest kept in registers.
int64_t part_floats(int64_t max_rows, int64_t max_cols) {
  const int64_t in_regs = max_cols < kRegisterCols ? max_cols : kRegisterCols;
  int64_t f = 2 * shares_limit(max_rows, in_regs) * in_regs;
  if (max_cols > kRegisterCols) {
    const int64_t g = 2 * shares_limit(max_rows, max_cols) * max_cols;
    if (g > f) f = g;
  }
  return f;
}

size_t elem_size(int32_t type) { return type == ARTOPK_G_F32 ? 4 : 2; }

bool known_type(int32_t type) { return type == ARTOPK_G_F32 || type == ARTOPK_G_BF16 || type == ARTOPK_G_F16; }

int check_rows(artopk_norm* h, const char* name, const void* p, int64_t stride, int32_t type, int64_t rows, int64_t cols) {
  if (!p && rows > 0) return fail_text(h->err, ARTOPK_EINVAL, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % elem_size(type))
    return fail_text(h->err, ARTOPK_EINVAL, "%s is not aligned to its elements", name);
  if (rows > 1 && stride < cols)
    return fail_text(h->err, ARTOPK_EINVAL, "%s's rows are %lld apart and %lld long", name, (long long)stride, (long long)cols);
  if (stride < 0 || stride >= (1ll << 40)) return fail_text(h->err, ARTOPK_EINVAL, "%s's stride is outside [0, 2^40)", name);
  // (so that places of elements, and of bytes, are far from 2^63)
  if (rows > 1 && stride > kMostElems / (rows - 1))
    return fail_text(h->err, ARTOPK_EINVAL, "%s's rows reach over more than 2^46 elements", name);
  return ARTOPK_OK;
}

int check_problem(artopk_norm* h, int32_t type, int64_t rows, int64_t cols) {
  if (!known_type(type)) return fail_text(h->err, ARTOPK_EINVAL, "unknown element type %d", type);
  if (rows < 0 || rows > h->max_rows)
    return fail_text(h->err, ARTOPK_EINVAL, "rows=%lld outside [0, %lld]", (long long)rows, (long long)h->max_rows);
  if (cols < 1 || cols > h->max_cols)
    return fail_text(h->err, ARTOPK_EINVAL, "cols=%lld outside [1, %lld]", (long long)cols, (long long)h->max_cols);
  return ARTOPK_OK;
}

int check_floats(artopk_norm* h, const char* name, const void* p, size_t size = 4) {
  if (reinterpret_cast<uintptr_t>(p) % size)
    return fail_text(h->err, ARTOPK_EINVAL, "%s is not aligned to its elements", name);
  return ARTOPK_OK;
}

// The buffers of one call, as rows of bytes; those of x, dy, y and dx may be columns of one matrix and so lie between each
// other's rows.  A buffer that is written must not share a byte with any other.
class RowSet {
 public:
  void add(const void* p, int64_t stride, int64_t rows, int64_t cols, size_t size, bool written, const char* name) {
    if (!p || rows == 0) return;
    r_[n_++] = Rows{reinterpret_cast<uintptr_t>(p), rows > 1 ? (size_t)stride * size : 0, (size_t)cols * size, rows, written, name};
  }
  void add(const void* p, int64_t count, size_t size, bool written, const char* name) { add(p, 0, 1, count, size, written, name); }
  // ARTOPK_OK, or ARTOPK_EINVAL with the first offending pair in `err`
  int check(char* err) const {
    for (int i = 0; i < n_; ++i)
      for (int j = 0; j < i; ++j)
        if ((r_[i].written || r_[j].written) && (r_[j].at < r_[i].at ? meet(r_[j], r_[i]) : meet(r_[i], r_[j])))
          return fail_text(err, ARTOPK_EINVAL, "buffers %s and %s overlap", r_[j].name, r_[i].name);
    return ARTOPK_OK;
  }

 private:
  struct Rows {
    uintptr_t at;
    size_t pitch, width;  // pitch: 0 for one row
    int64_t rows;
    bool written;
    const char* name;
    uintptr_t end() const { return at + (size_t)(rows - 1) * pitch + width; }
  };
  // a begins where b does, or before
  static bool meet(const Rows& a, const Rows& b) {
    if (b.at >= a.end()) return false;
    if (!a.pitch) return true;                    // b begins inside
    const size_t in = (b.at - a.at) % a.pitch;    // b's first byte, from the row of a before it
    if (in < a.width) return true;
    if (b.pitch && b.pitch != a.pitch) return true;  // (may be; taken for yes)
    // between two rows of a, or behind the last, which b.at < a.end() rules out
    return in + b.width > a.pitch;
  }
  Rows r_[8];  // as many as a call has
  int n_ = 0;
};

// Whether rows at p can be read sixteen bytes at a time.
bool wide_rows(const void* p, int64_t stride, int64_t rows, size_t size) {
  return aligned16(p) && (rows <= 1 || stride * (int64_t)size % 16 == 0);
}

// Calls f(V, whether rows may lie anywhere, threads of a row, elements of a thread) as compile-time constants: a wave where it
// holds the row, then the fewest threads that do; with fewer rows than compute units twice as many, of half the elements.
template <int V, bool ANY, int MOST, class F>  // at most MOST columns
void with_shape(int64_t cols, bool few, F&& f) {
  auto go = [&](auto tpr, auto e) { f(std::integral_constant<int, V>(), std::integral_constant<bool, ANY>(), tpr, e); };
  using std::integral_constant;
  if (MOST <= kWaveCols || cols <= kWaveCols) return go(integral_constant<int, 64>(), integral_constant<int, 8>());
  if constexpr (MOST > kWaveCols) {
    if (cols <= 1024 && !few) return go(integral_constant<int, 64>(), integral_constant<int, 16>());
    if (cols <= 2048) return go(integral_constant<int, 256>(), integral_constant<int, 8>());
    if (cols <= 4096 && !few) return go(integral_constant<int, 256>(), integral_constant<int, 16>());
    if (cols <= 4096) return go(integral_constant<int, 512>(), integral_constant<int, 8>());
    if (cols <= 8192 && !few) return go(integral_constant<int, 512>(), integral_constant<int, 16>());
    if (MOST <= 8192 || cols <= 8192) return go(integral_constant<int, 1024>(), integral_constant<int, 8>());
    if constexpr (MOST > 8192) go(integral_constant<int, 1024>(), integral_constant<int, 16>());
  }
}

template <class T>
void forward(artopk_norm* h, const T* x, int64_t x_stride, int64_t rows, int64_t cols, const float* gamma,
             const float* beta, float eps, T* y, int64_t y_stride, float* mean, float* rstd) {
  if (cols > kRegisterCols) {
    const int blocks = (int)std::min<int64_t>(rows, 2 * h->num_cu);
    k_norm_forward_long<T><<<blocks, 1024, 0, h->stream>>>(x, x_stride, rows, cols, gamma, beta, eps, y, y_stride, mean, rstd);
    return;
  }
  auto go = [&](auto V, auto ANY, auto TPR, auto E) {
    using S = NormShape<TPR()>;
    const int64_t units = (rows + S::kRows - 1) / S::kRows;
    const int blocks = (int)std::min<int64_t>(units, (int64_t)h->num_cu * (2048 / S::kThreads));
    k_norm_forward<T, V(), ANY(), TPR(), E()><<<blocks, S::kThreads, 0, h->stream>>>(x, x_stride, rows, (int)cols, gamma, beta, eps,
                                                                              y, y_stride, mean, rstd);
  };
  constexpr int kWide = 16 / sizeof(T);
  const bool few = rows <= h->num_cu;
  const bool wide = wide_rows(x, x_stride, rows, sizeof(T)) && wide_rows(y, y_stride, rows, sizeof(T));
  // Where sixteen bytes are not aligned they still move faster than one 16-bit element at a time (8191 x 2501 f16 25 us, so 22;
  // 4000 x 10001 bf16 44, so 41), but not than one float32 (4099 x 1111 10.3, so 11.8), nor in a wave's row (30000 x 333 bf16
  // 12.2, so 14.7).
  if (wide && cols % kWide == 0)
    with_shape<kWide, false, kRegisterCols>(cols, few, go);
  else if (cols >= kWide && (wide || (sizeof(T) == 2 && cols > kWaveCols)))
    with_shape<kWide, true, kRegisterCols>(cols, few, go);
  else
    with_shape<1, false, sizeof(T) == 2 ? kWaveCols : kRegisterCols>(cols, few, go);
}

// Returns the number of shares of the weight gradients to be added up, 0 if they are done.
template <class T>
int backward(artopk_norm* h, const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t rows, int64_t cols,
             const float* gamma, const float* mean, const float* rstd, T* dx, int64_t dx_stride, float* part,
             const GradOut& grads) {
  int shares = 0;
  if (cols > kRegisterCols) {
    if (dx) {
      const int blocks = (int)std::min<int64_t>(rows, 2 * h->num_cu);
      k_norm_backward_long<T><<<blocks, 1024, 0, h->stream>>>(dy, dy_stride, x, x_stride, rows, cols, gamma, mean, rstd, dx,
                                                              dx_stride);
    }
    shares = (int)std::min<int64_t>(rows, kLongShares);
    if (part)
      k_norm_backward_cols<T><<<dim3((unsigned)((cols + 255) / 256), shares), 256, 0, h->stream>>>(
          dy, dy_stride, x, x_stride, rows, cols, mean, rstd, part);
    return shares;
  }
  const bool columns = part && rows <= kColumnRows && rows * cols <= kColumnElems;
  auto go = [&](auto V, auto ANY, auto TPR, auto E) {
    using S = NormShape<TPR()>;
    const int64_t units = (rows + S::kRows - 1) / S::kRows;
    shares = (int)std::min<int64_t>(units, std::min<int64_t>(kMaxShares, (int64_t)h->num_cu * (1024 / S::kThreads)));
    const int row_blocks = columns && !dx ? 0 : shares;
    const int blocks = row_blocks + (columns ? (int)((cols + 63) / 64) : 0);
    k_norm_backward<T, V(), ANY(), TPR(), E()><<<blocks, S::kThreads, 0, h->stream>>>(
        dy, dy_stride, x, x_stride, rows, (int)cols, gamma, mean, rstd, dx, dx_stride, columns ? nullptr : part, row_blocks, grads);
  };
  constexpr int kWide = 16 / sizeof(T);
  const bool few = rows <= h->num_cu;
  const bool wide = wide_rows(x, x_stride, rows, sizeof(T)) && wide_rows(dy, dy_stride, rows, sizeof(T)) &&
                    (!dx || wide_rows(dx, dx_stride, rows, sizeof(T)));
  // Where sixteen bytes are not aligned one element at a time is faster (8191 x 2501 f16, of which only dx is off its boundary, 42
  // us, 54 by sixteen bytes) as long as its registers hold the row (4000 x 10001 bf16 290 and 86, f32 291 and 121).
  if (wide && cols % kWide == 0)
    with_shape<kWide, false, kRegisterCols>(cols, few, go);
  else if (cols >= kWide && (wide || cols > kSingleCols))
    with_shape<kWide, true, kRegisterCols>(cols, few, go);
  else
    with_shape<1, false, kSingleCols>(cols, few, go);
  if (columns) shares = 0;
  return shares;
}

}  // namespace

int64_t artopk_norm_scratch_bytes(int64_t max_rows, int64_t max_cols) {
  if (!valid_limits(max_rows, max_cols)) return -1;
  return 4 * part_floats(max_rows, max_cols);
}

int artopk_norm_create(artopk_norm** out, int64_t max_rows, int64_t max_cols, void* hip_stream) {
  if (!out) return fail_text(g_noctx_err, ARTOPK_EINVAL, "out is NULL");
  if (!valid_limits(max_rows, max_cols))
    return fail_text(g_noctx_err, ARTOPK_EINVAL, "max_rows=%lld and max_cols=%lld have to be in [1, 2^31)", (long long)max_rows,
                     (long long)max_cols);
  artopk_norm* h = new (std::nothrow) artopk_norm();
  if (!h) return fail_text(g_noctx_err, ARTOPK_ENOMEM, "out of host memory");
  h->stream = reinterpret_cast<hipStream_t>(hip_stream);
  h->max_rows = max_rows;
  h->max_cols = max_cols;
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) {
    delete h;
    return fail_text(g_noctx_err, ARTOPK_EHIP, "no device: %s", hipGetErrorString(e));
  }
  if (cus > 0) h->num_cu = cus;
  void* p = nullptr;
  e = hipMalloc(&p, (size_t)part_floats(max_rows, max_cols) * 4);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete h;
    return fail_text(g_noctx_err, ARTOPK_ENOMEM, "hipMalloc failed: %s", hipGetErrorString(e));
  }
  h->part = static_cast<float*>(p);
  *out = h;
  return ARTOPK_OK;
}

int artopk_norm_destroy(artopk_norm* norm) {
  if (!norm) return ARTOPK_EINVAL;
  if (norm->part) (void)hipFree(norm->part);
  delete norm;
  return ARTOPK_OK;
}

const char* artopk_norm_last_error(const artopk_norm* norm) { return norm ? norm->err : g_noctx_err; }

int artopk_layernorm_forward(artopk_norm* norm, const void* x, int64_t x_stride, int32_t type, int64_t rows,
                             int64_t cols, const float* gamma, const float* beta, float eps, void* y, int64_t y_stride,
                             float* mean_out, float* rstd_out) {
  if (!norm) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_layernorm_forward: norm is NULL");
  int rc;
  if ((rc = check_problem(norm, type, rows, cols))) return rc;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail_text(norm->err, ARTOPK_EINVAL, "eps is negative or not finite");
  if ((rc = check_rows(norm, "x", x, x_stride, type, rows, cols))) return rc;
  if ((rc = check_rows(norm, "y", y, y_stride, type, rows, cols))) return rc;
  if ((rc = check_floats(norm, "gamma", gamma)) || (rc = check_floats(norm, "beta", beta)) ||
      (rc = check_floats(norm, "mean_out", mean_out)) || (rc = check_floats(norm, "rstd_out", rstd_out)))
    return rc;
  {
    RowSet rs;
    rs.add(x, x_stride, rows, cols, elem_size(type), false, "x");
    rs.add(y, y_stride, rows, cols, elem_size(type), true, "y");
    rs.add(gamma, cols, 4, false, "gamma");
    rs.add(beta, cols, 4, false, "beta");
    rs.add(mean_out, rows, 4, true, "mean_out");
    rs.add(rstd_out, rows, 4, true, "rstd_out");
    if ((rc = rs.check(norm->err))) return rc;
  }
  if (rows == 0) return ARTOPK_OK;
  auto go = [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    forward<T>(norm, static_cast<const T*>(x), x_stride, rows, cols, gamma, beta, eps, static_cast<T*>(y), y_stride, mean_out,
               rstd_out);
  };
  if (type == ARTOPK_G_F32) go((float*)nullptr);
  else if (type == ARTOPK_G_BF16) go((__bf16*)nullptr);
  else go((_Float16*)nullptr);
  NORM_TRY(norm, hipGetLastError());
  return ARTOPK_OK;
}

int artopk_layernorm_backward(artopk_norm* norm, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                              int32_t type, int64_t rows, int64_t cols, const float* gamma, const float* mean,
                              const float* rstd, void* dx, int64_t dx_stride, void* dgamma, void* dbeta,
                              int32_t grad_type, int32_t accumulate) {
  if (!norm) return fail_text(g_noctx_err, ARTOPK_EINVAL, "artopk_layernorm_backward: norm is NULL");
  int rc;
  if ((rc = check_problem(norm, type, rows, cols))) return rc;
  if (!known_type(grad_type)) return fail_text(norm->err, ARTOPK_EINVAL, "unknown gradient element type %d", grad_type);
  if (!dx && !dgamma && !dbeta) return fail_text(norm->err, ARTOPK_EINVAL, "dx, dgamma and dbeta are all NULL");
  if ((rc = check_rows(norm, "dy", dy, dy_stride, type, rows, cols))) return rc;
  if ((rc = check_rows(norm, "x", x, x_stride, type, rows, cols))) return rc;
  if (dx && (rc = check_rows(norm, "dx", dx, dx_stride, type, rows, cols))) return rc;
  if (rows > 0 && (!mean || !rstd)) return fail_text(norm->err, ARTOPK_EINVAL, "mean or rstd is NULL");
  const size_t gsize = elem_size(grad_type);
  if ((rc = check_floats(norm, "gamma", gamma)) || (rc = check_floats(norm, "mean", mean)) ||
      (rc = check_floats(norm, "rstd", rstd)) || (rc = check_floats(norm, "dgamma", dgamma, gsize)) ||
      (rc = check_floats(norm, "dbeta", dbeta, gsize)))
    return rc;
  {
    RowSet rs;
    rs.add(dy, dy_stride, rows, cols, elem_size(type), false, "dy");
    rs.add(x, x_stride, rows, cols, elem_size(type), false, "x");
    rs.add(gamma, cols, 4, false, "gamma");
    rs.add(mean, rows, 4, false, "mean");
    rs.add(rstd, rows, 4, false, "rstd");
    rs.add(dx, dx_stride, rows, cols, elem_size(type), true, "dx");
    rs.add(dgamma, cols, gsize, true, "dgamma");
    rs.add(dbeta, cols, gsize, true, "dbeta");
    if ((rc = rs.check(norm->err))) return rc;
  }
  float* part = dgamma || dbeta ? norm->part : nullptr;
  const GradOut grads = {{dgamma, dbeta}, grad_type, accumulate != 0};
  int shares = 0;
  if (rows > 0) {
    auto go = [&](auto* tag) {
      using T = std::remove_pointer_t<decltype(tag)>;
      shares = backward<T>(norm, static_cast<const T*>(dy), dy_stride, static_cast<const T*>(x), x_stride, rows, cols, gamma, mean,
                           rstd, static_cast<T*>(dx), dx_stride, part, grads);
    };
    if (type == ARTOPK_G_F32) go((float*)nullptr);
    else if (type == ARTOPK_G_BF16) go((__bf16*)nullptr);
    else go((_Float16*)nullptr);
  }
  if (part && (shares || rows == 0))
    k_norm_join<<<dim3((unsigned)std::min<int64_t>((cols + 63) / 64, kJoinBlocks), 2), 1024, 0, norm->stream>>>(part, shares, cols, grads);
  NORM_TRY(norm, hipGetLastError());
  return ARTOPK_OK;
}
