// What the operators on heads share: checks of [batch, row, head, column] arguments.
#pragma once

#include <math.h>

#include <algorithm>

#include "ops.h"

namespace antdt {

// x / d of x < 2^31 without a division: x m >> 31 + s, where 2^s is d or the next larger power of two and m = 2^(31 + s) / d, rounded up.
struct Divisor {
  uint32_t d, m, s;
  static Divisor of(uint32_t d) {
    uint32_t s = 0;
    while ((1u << s) < d) ++s;
    return Divisor{d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)((uint64_t)x * m >> 31 >> s); }
};

// Elements from one batch, row and head to the next (0 where there is only one); a head's columns are neighbours.
struct HeadStrides {
  int64_t b, l, h;
};
// An argument of B x L x H heads of D columns: strides of things there is one of are set to 0.  A result's elements must not share memory; an operand's
// may (a stride of 0 repeats it).
inline int op_heads(const char* call, const char* name, const void* p, int64_t B, int64_t L, int64_t H, int64_t D, HeadStrides& s, int64_t size,
                    bool written) {
  if (B < 0 || L < 0 || H < 0 || D < 0 || B >= ROWS_MAX || L >= ROWS_MAX || H >= ROWS_MAX || D >= ROWS_MAX)
    return op_fail(ANTDT_INVALID_ARG, "%s: %s: size out of range", call, name);
  if (B == 0 || L == 0 || H == 0 || D == 0) return ANTDT_OK;
  if (!p) return op_fail(ANTDT_INVALID_ARG, "%s: %s is null", call, name);
  if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)size) return op_fail(ANTDT_INVALID_ARG, "%s: %s is misaligned", call, name);
  std::pair<int64_t, int64_t> dim[3] = {{s.b, B}, {s.l, L}, {s.h, H}};
  __int128 last = D;
  for (const auto& d : dim) {
    if (d.second == 1) continue;
    if (d.first < 0 || d.first >= ROWS_MAX) return op_fail(ANTDT_INVALID_ARG, "%s: %s: stride %lld", call, name, (long long)d.first);
    last += (__int128)(d.second - 1) * d.first;
  }
  if (last * size >= ((__int128)1 << 62)) return op_fail(ANTDT_INVALID_ARG, "%s: %s: size out of range", call, name);
  if (written) {
    std::sort(dim, dim + 3);
    int64_t need = D;
    for (const auto& d : dim) {
      if (d.second == 1) continue;
      if (d.first < need) return op_fail(ANTDT_INVALID_ARG, "%s: %s: stride %lld, where %lld elements belong to one another", call, name, (long long)d.first, (long long)need);
      need += (d.second - 1) * d.first;
    }
  }
  if (B == 1) s.b = 0;
  if (L == 1) s.l = 0;
  if (H == 1) s.h = 0;
  return ANTDT_OK;
}
// Columns that a vector access of these heads takes, as row_quantum's.
inline int head_quantum(int64_t cols, int64_t size, const void* p, const HeadStrides& s) { return row_quantum(cols, size, {{p, s.b}, {p, s.l}, {p, s.h}}); }
// The same addresses, element for element.
inline bool same_heads(const void* p, const HeadStrides& a, const void* q, const HeadStrides& b) { return p == q && a.b == b.b && a.l == b.l && a.h == b.h; }

}  // namespace antdt
