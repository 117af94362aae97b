// What the operators on sequences of tokens share: checks of their arguments, rows in 8 columns at a time, the dropout.
#pragma once

#include <stdarg.h>
#include <stdio.h>

#include <initializer_list>
#include <utility>

#include "common.h"

namespace antdt {

// Sets the message of the calling thread's last failed call and returns `code`.
inline int op_fail(int code, const char* format, ...) {
  char text[256];
  va_list ap;
  va_start(ap, format);
  vsnprintf(text, sizeof(text), format, ap);
  va_end(ap);
  set_last_error(text);
  return code;
}
inline int op_hip(const char* call, hipError_t e) {
  return e == hipSuccess ? ANTDT_OK : op_fail(ANTDT_HIP_ERROR, "%s: %s", call, hipGetErrorString(e));
}
inline bool op_dtype(int32_t t) { return t == ANTDT_F32 || t == ANTDT_BF16; }
inline int64_t op_size(int32_t t) { return t == ANTDT_F32 ? 4 : 2; }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t ROWS_MAX = 1ll << 40;   // of a matrix's rows, columns and leading dimension: products with element sizes stay in 64 bits
// A matrix of an argument: rows that do not overlap, addresses in range, the element's alignment.  `name` for the message.
inline int op_matrix(const char* call, const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t size) {
  if (rows < 0 || cols < 0 || rows >= ROWS_MAX || cols >= ROWS_MAX) return op_fail(ANTDT_INVALID_ARG, "%s: %s: size out of range", call, name);
  if (rows == 0 || cols == 0) return ANTDT_OK;
  if (!p) return op_fail(ANTDT_INVALID_ARG, "%s: %s is null", call, name);
  if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)size) return op_fail(ANTDT_INVALID_ARG, "%s: %s is misaligned", call, name);
  if (ld < cols || ld >= ROWS_MAX || (__int128)rows * ld * size >= ((__int128)1 << 62))
    return op_fail(ANTDT_INVALID_ARG, "%s: %s: leading dimension %lld with %lld columns", call, name, (long long)ld, (long long)cols);
  return ANTDT_OK;
}
inline int op_workspace(const char* call, const void* ws, size_t given, size_t need) {
  if (need == 0) return ANTDT_OK;
  if (given < need) return op_fail(ANTDT_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes, %zu needed", call, given, need);
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return op_fail(ANTDT_INVALID_ARG, "%s: workspace is null or not 256-byte aligned", call);
  return ANTDT_OK;
}
#define OP_TRY(expr)            \
  do {                          \
    const int rc__ = (expr);    \
    if (rc__) return rc__;      \
  } while (0)

// ------------------------------------------------------------- rows, 8 columns at a time
// Columns that a vector access takes: 8 (16 bytes of bf16, twice 16 of fp32), 4 (8, 16), or 1 where rows start anywhere.
inline int row_quantum(int64_t cols, int64_t size, std::initializer_list<std::pair<const void*, int64_t>> rows) {
  int q = cols % 8 == 0 ? 8 : cols % 4 == 0 ? 4 : 1;
  for (const auto& r : rows)
    while (q > 1 && ((r.second % q) || (reinterpret_cast<uintptr_t>(r.first) % (uintptr_t)((q < 4 ? 1 : q) * size > 16 ? 16 : q * size))))
      q = q == 8 ? 4 : 1;
  return q;
}

// 16 or 8 bytes from or to memory; STREAM: not kept in the caches beyond this use.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <bool STREAM>
__device__ __forceinline__ uint4 load16(const void* p) {
  const u32x4* q = reinterpret_cast<const u32x4*>(p);
  const u32x4 v = STREAM ? __builtin_nontemporal_load(q) : *q;
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool STREAM>
__device__ __forceinline__ uint2 load8b(const void* p) {
  const u32x2* q = reinterpret_cast<const u32x2*>(p);
  const u32x2 v = STREAM ? __builtin_nontemporal_load(q) : *q;
  return make_uint2(v.x, v.y);
}
template <bool STREAM>
__device__ __forceinline__ void store16(void* p, uint4 w) {
  const u32x4 v = {w.x, w.y, w.z, w.w};
  if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = v;
}
__device__ __forceinline__ uint4 bits4(float a, float b, float c, float d) {
  return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
}

// v[0 .. n) from p, n <= 8 columns of which Q at a time exist.
template <int Q, bool STREAM = false, typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
  if constexpr (Q == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32(p[e]) : 0.0f;
  } else if constexpr (sizeof(T) == 4) {
    const uint4 a = load16<STREAM>(p);
    uint4 b = make_uint4(0, 0, 0, 0);
    if (Q == 8 || n > 4) b = load16<STREAM>(p + 4);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(w[e]);
  } else {
    uint4 a = make_uint4(0, 0, 0, 0);
    if constexpr (Q == 8) {
      a = load16<STREAM>(p);
    } else {
      const uint2 x = load8b<STREAM>(p);
      a.x = x.x; a.y = x.y;
      if (n > 4) {
        const uint2 y = load8b<STREAM>(p + 4);
        a.z = y.x; a.w = y.y;
      }
    }
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
}
template <int Q, typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
  if constexpr (Q == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  } else if constexpr (sizeof(T) == 4) {
    store16<false>(p, bits4(v[0], v[1], v[2], v[3]));
    if (Q == 8 || n > 4) store16<false>(p + 4, bits4(v[4], v[5], v[6], v[7]));
  } else {
    const uint4 a = make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
    if constexpr (Q == 8) {
      store16<false>(p, a);
    } else {
      *reinterpret_cast<uint2*>(p) = make_uint2(a.x, a.y);
      if (n > 4) *reinterpret_cast<uint2*>(p + 4) = make_uint2(a.z, a.w);
    }
  }
}

// ------------------------------------------------------------- dropout
struct DropArgs {
  uint32_t below;        // lots below are dropped; 65536: everything
  float factor;          // of what is kept
  uint32_t call;
  uint64_t seed;
  const uint64_t* step;
};
// The spec checked and taken apart; *none: nothing is ever dropped.
inline int op_dropout(const char* call, const antdt_dropout_spec* d, DropArgs& a, bool& none) {
  a = DropArgs{0, 1.0f, 0, 0, nullptr};
  none = true;
  if (!d) return ANTDT_OK;
  if (!(d->p >= 0.0f && d->p <= 1.0f)) return op_fail(ANTDT_INVALID_ARG, "%s: dropout probability outside 0..1", call);
  if (reinterpret_cast<uintptr_t>(d->step) & 7) return op_fail(ANTDT_INVALID_ARG, "%s: the dropout's step is misaligned", call);
  a.below = (uint32_t)((double)d->p * 65536.0 + 0.5);
  a.factor = a.below < 65536 ? (float)(65536.0 / (65536 - (int)a.below)) : 0.0f;
  a.call = d->call; a.seed = d->seed; a.step = d->step;
  none = a.below == 0;
  return ANTDT_OK;
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC'11).
__device__ __forceinline__ void philox4x32(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[0] = n0; c[1] = (uint32_t)b; c[2] = n2; c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}
struct DropKey {
  uint32_t k0, k1;
  __device__ __forceinline__ explicit DropKey(const DropArgs& d) {
    const uint64_t k = d.seed + (d.step ? *d.step : 0);
    k0 = (uint32_t)k;
    k1 = (uint32_t)(k >> 32);
  }
};
// x of columns 8 group .. + 7 of `row`: dropped (exactly 0, whatever it was) or times `scale`, which holds the factor.
// One draw of 10 rounds serves 8 columns in lots of 16 bits: with a word for each column the multiplications (a quarter of the vector rate), not
// the memory, bound a bf16 dropout.
__device__ __forceinline__ void drop8(const DropArgs& d, const DropKey& k, int64_t row, uint32_t group, float scale, float (&x)[8]) {
  uint32_t c[4] = {group, (uint32_t)row, (uint32_t)((uint64_t)row >> 32), d.call};
  philox4x32(c, k.k0, k.k1);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t lot = e & 1 ? c[e >> 1] >> 16 : c[e >> 1] & 0xFFFFu;
    x[e] = lot >= d.below ? x[e] * scale : 0.0f;
  }
}

}  // namespace antdt
