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

}  // namespace artopk
