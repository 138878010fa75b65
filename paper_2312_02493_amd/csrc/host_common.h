// What the host sides of the library's entry points share: error texts and the check that no
// buffer a call writes overlaps another.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cstdarg>
#include <cstddef>
#include <cstdio>

#include "artopk.h"

namespace artopk {

constexpr size_t kErrText = 512;  // bytes of an error text

// error text of calls that have no context or handle; artopk_last_error(NULL) returns it
extern __thread char g_noctx_err[kErrText] __attribute__((visibility("hidden")));

inline int fail_text(char* err, int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(err, kErrText, fmt, ap);
  va_end(ap);
  return code;
}

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The buffers of one call as byte ranges.  Ranges that are only read may overlap each other
// (two workers may share a gradient buffer); a range that is written must not overlap any other.
class RangeSet {
 public:
  void add(const void* p, size_t bytes, bool written, const char* name, int index = -1) {
    if (!p || bytes == 0 || n_ >= kCap) return;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    r_[n_++] = Range{lo, lo + bytes, written, name, index};
  }
  void add_table(const void* const* tab, int32_t w, size_t bytes, bool written, const char* name) {
    for (int i = 0; i < w; ++i) add(tab[i], bytes, written, name, i);
  }
  // ARTOPK_OK, or ARTOPK_EINVAL with the first offending pair in `err`
  int check(char* err) {
    std::sort(r_, r_ + n_, [](const Range& a, const Range& b) { return a.lo < b.lo; });
    int far_any = -1, far_written = -1;  // ranges seen so far that reach furthest: any, written ones
    for (int i = 0; i < n_; ++i) {
      const int other = r_[i].written ? far_any : far_written;
      if (other >= 0 && r_[i].lo < r_[other].hi) {
        char a[48], b[48];
        label(r_[other], a, sizeof(a));
        label(r_[i], b, sizeof(b));
        return fail_text(err, ARTOPK_EINVAL, "buffers %s and %s overlap", a, b);
      }
      if (far_any < 0 || r_[i].hi > r_[far_any].hi) far_any = i;
      if (r_[i].written && (far_written < 0 || r_[i].hi > r_[far_written].hi)) far_written = i;
    }
    return ARTOPK_OK;
  }

 private:
  struct Range {
    uintptr_t lo, hi;
    bool written;
    const char* name;
    int index;
  };
  static void label(const Range& r, char* out, size_t cap) {
    if (r.index >= 0)
      snprintf(out, cap, "%s[%d]", r.name, r.index);
    else
      snprintf(out, cap, "%s", r.name);
  }
  static constexpr int kCap = 2 * ARTOPK_MAX_WORKERS + 8;
  Range r_[kCap];
  int n_ = 0;
};

inline size_t elem_size(int32_t type) { return type == ARTOPK_G_F32 ? 4 : 2; }

inline bool known_type(int32_t type) { return type == ARTOPK_G_F32 || type == ARTOPK_G_BF16 || type == ARTOPK_G_F16; }

constexpr int64_t kMostElems = 1ll << 46;  // between the first and the last row

inline int check_rows(char* err, const char* name, const void* p, int64_t stride, size_t size, int64_t rows, int64_t cols) {
  if (!p && rows > 0) return fail_text(err, ARTOPK_EINVAL, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % size) return fail_text(err, ARTOPK_EINVAL, "%s is not aligned to its elements", name);
  if (rows > 1 && stride < cols)
    return fail_text(err, ARTOPK_EINVAL, "%s's rows are %lld apart and %lld long", name, (long long)stride, (long long)cols);
  if (stride < 0 || stride >= (1ll << 40)) return fail_text(err, ARTOPK_EINVAL, "%s's stride is outside [0, 2^40)", name);
  // (so that places of elements, and of bytes, are far from 2^63)
  if (rows > 1 && stride > kMostElems / (rows - 1))
    return fail_text(err, ARTOPK_EINVAL, "%s's rows reach over more than 2^46 elements", name);
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
  Rows r_[12];  // as many as a call has, and more
  int n_ = 0;
};

}  // namespace artopk
