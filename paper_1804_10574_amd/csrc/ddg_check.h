// What the C entry points of the operators of token models refuse: checks that they share.
#pragma once
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "ddg_internal.h"
#include "ddg_kernels.h"

namespace ddg {
namespace {

__attribute__((format(printf, 2, 3))) inline ddg_status fail(ddg_status st, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  ddg_internal_set_error(msg);
  return st;
}

inline ddg_status done(hipError_t e, const char* what) {
  return e == hipSuccess ? DDG_OK : fail(DDG_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// A tensor argument: [rows][cols] elements of `size` bytes, `ld` elements from row to row
struct Arg {
  const char* name;
  const void* p;
  long rows, cols, ld;
  size_t size;
  bool out;
  uintptr_t lo() const { return (uintptr_t)p; }
  uintptr_t hi() const { return (uintptr_t)p + ((size_t)(rows - 1) * ld + cols) * size; }
  bool empty() const { return !p || rows < 1 || cols < 1; }
};

// Columns of one wider tensor, none of them in both
inline bool side_by_side(const Arg& a, const Arg& b) {
  const uintptr_t row = a.ld * a.size, wa = a.cols * a.size, wb = b.cols * b.size;
  if (row != b.ld * b.size) return false;
  const uintptr_t apart = a.lo() <= b.lo() ? (b.lo() - a.lo()) % row : (row - (a.lo() - b.lo()) % row) % row;
  return apart >= wa && apart + wb <= row;
}

// Pointers lie on their elements, and no output overlaps another argument; `same` names pairs that may be one tensor.
struct Pair { const char* a; const char* b; };
template <int N, int S> ddg_status check_args(const Arg (&args)[N], const Pair (&same)[S]) {
  for (const Arg& a : args)
    if (a.lo() % a.size) return fail(DDG_ERR_INVALID_ARG, "%s must be aligned to its elements of %zu bytes", a.name, a.size);
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N; ++j) {
      const Arg& a = args[i]; const Arg& b = args[j];
      if (i == j || !a.out || (b.out && j < i) || a.empty() || b.empty()) continue;
      if (a.hi() <= b.lo() || b.hi() <= a.lo() || side_by_side(a, b)) continue;
      bool allowed = false;
      for (const Pair& s : same)
        if (s.a && !strcmp(s.a, a.name) && !strcmp(s.b, b.name)) allowed = a.p == b.p && a.ld == b.ld;
      if (!allowed) return fail(DDG_ERR_INVALID_ARG, "%s overlaps %s", a.name, b.name);
    }
  return DDG_OK;
}
constexpr Pair NONE[] = {{nullptr, nullptr}};

// Row numbers plus the rows of a round of workgroups stay inside an int, and a tensor's extent in bytes inside 63 bits
constexpr int ROWS_MAX = 1 << 30;
constexpr long LD_MAX = 1l << 30;

inline ddg_status check_rows(const char* what, int rows, int cols, int dtype) {
  if (dtype != DDG_F32 && dtype != DDG_BF16) return fail(DDG_ERR_INVALID_ARG, "%s: dtype must be DDG_F32 or DDG_BF16", what);
  if (rows < 0 || cols < 1) return fail(DDG_ERR_SHAPE, "%s: need rows >= 0 and columns >= 1 (%d, %d)", what, rows, cols);
  if (rows > ROWS_MAX) return fail(DDG_ERR_SHAPE, "%s: at most %d rows (%d)", what, ROWS_MAX, rows);
  return DDG_OK;
}
inline ddg_status check_ld(const char* name, long* ld, int cols) {
  if (*ld == 0) *ld = cols;
  if (*ld < cols) return fail(DDG_ERR_SHAPE, "%s = %ld is less than a row of %d", name, *ld, cols);
  if (*ld > LD_MAX) return fail(DDG_ERR_SHAPE, "%s = %ld is more than %ld", name, *ld, LD_MAX);
  return DDG_OK;
}
#define CHECK(expr)                          \
  do {                                       \
    const ddg_status st_ = (expr);           \
    if (st_ != DDG_OK) return st_;           \
  } while (0)

}  // namespace
}  // namespace ddg
