// Tiles and fragments of attention on the gfx950 matrix cores, of bf16 (v_mfma_f32_32x32x16_bf16) or fp32 (v_mfma_f32_32x32x2_f32) heads.
//
// A tile is 32 or more rows (keys, values, queries or gradients) of a head, DP columns each, in LDS as they lie in memory, 16-byte slots permuted.
// It is read in two ways, with one permutation that serves both:
//   along a row      the contraction is over the columns:  scores = K Q^T, dP = V dO^T
//   down a column    the contraction is over the rows:     out = P V, dQ = dS K, dV = P^T dO, dK = dS^T Q
// The products are formed transposed: of D = A B^T with A from the tile, lane l holds column l % 32 (a row of B) and rows
// 8 (e / 4) + 4 (l / 32) + e % 4, e < 16, of D's 32.  Those rows, in that order, are contraction slots of the second product whose operand D then is,
// so that probabilities go from one product to the next in the lane's registers: the tile's rows are read down the column in the same order.
#pragma once

#include "heads.h"
#include "product.h"

namespace antdt {

template <typename T>
struct Core;

template <>
struct Core<bf16_t> {
  typedef bf16x8 Fragment;
  static constexpr int STEP = 16, PER = 8;   // contraction slots of a product of fragments; elements of 16 bytes
  // c += A B^T, 32 x 32
  static __device__ __forceinline__ void multiply(const Fragment& a, const Fragment& b, f32x16& c) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // Contraction slots STEP i .. of what a product left.
  template <typename X>
  static __device__ __forceinline__ Fragment pack(const X& x, int i) {
    Words u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u.w[e] = f2bf2(x[8 * i + 2 * e], x[8 * i + 2 * e + 1]);
    return u.f;
  }
  // The same of x >= 0 in two parts, off by 2^-15 of x together: x cut off, and what that took away, rounded.  The last bit of x counts as set, so that there
  // is a second part of every x: a zero, or a part of the other sign, times an infinite value would be NaN.
  static constexpr int PARTS = 2;
  template <typename X>
  static __device__ __forceinline__ void pack(const X& x, int i, Fragment (&f)[2]) {
    Words u[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t a = __float_as_uint(x[8 * i + 2 * e]) | 1, b = __float_as_uint(x[8 * i + 2 * e + 1]) | 1, a1 = a & 0xFFFF0000u, b1 = b & 0xFFFF0000u;
      u[0].w[e] = a1 >> 16 | b1;
      u[1].w[e] = f2bf2(__uint_as_float(a) - __uint_as_float(a1), __uint_as_float(b) - __uint_as_float(b1));
    }
    f[0] = u[0].f;
    f[1] = u[1].f;
  }
  template <typename X>
  static __device__ __forceinline__ void pack(const X& x, int i, Fragment (&f)[1]) { f[0] = pack(x, i); }

 private:
  union Words {
    uint32_t w[4];
    Fragment f;
  };
};
template <>
struct Core<float> {
  typedef f32x4v Fragment;
  static constexpr int STEP = 8, PER = 4;
  static __device__ __forceinline__ void multiply(const Fragment& a, const Fragment& b, f32x16& c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  }
  static constexpr int PARTS = 1;
  template <typename X>
  static __device__ __forceinline__ Fragment pack(const X& x, int i) { return Fragment{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]}; }
  template <typename X>
  static __device__ __forceinline__ void pack(const X& x, int i, Fragment (&f)[1]) { f[0] = pack(x, i); }
};

// Rows of DP columns in LDS.
template <typename T, int DP>
struct HeadTile {
  typedef typename Core<T>::Fragment Fragment;
  static constexpr int STEP = Core<T>::STEP, PITCH = DP * (int)sizeof(T) / 16, ROW = DP * (int)sizeof(T);   // slots and bytes of a row
  // Along a row 16 lanes read one slot of 16 rows, down a column (bf16) 32 lanes four neighbouring slots of four rows: slots that have to differ modulo
  // 16 (256 bytes, all banks).
  static __host__ __device__ __forceinline__ constexpr int swizzle(int r) {
    if (PITCH >= 16) return sizeof(T) == 2 ? ((r & 3) << 2) | ((r >> 2) & 3) : r & 15;
    if (PITCH == 8) return sizeof(T) == 2 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : (r >> 1) & 7;
    return (r >> 2) & 3;
  }
  static __device__ __forceinline__ int slot(int r, int c) { return r * PITCH + (c ^ swizzle(r)); }

  // A lane's reads differ from one another by constants, added to the row and exclusive-ored to the slot (the permutation of rows 16 apart is the same),
  // so that one address serves them all: along_at, down_at of a tile (opaque, lest a register is kept for each).
  static __device__ __forceinline__ uint32_t at(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
  }
  static __device__ __forceinline__ uint32_t along_at(uint32_t tile, int lane) { return at(tile + slot(lane & 31, lane >> 5) * 16); }
  static __device__ __forceinline__ uint32_t down_at(uint32_t tile, int lane) {
    if constexpr (sizeof(T) == 2) {
      const int j = lane & 15;
      return at(tile + slot(4 * (lane >> 5) + (j >> 2), ((lane >> 4) & 1) * 2 + ((j & 3) >> 1)) * 16 + (j & 1) * 8);
    } else {
      return at(tile + slot(4 * (lane >> 5), (lane & 31) >> 2) * 16 + (lane & 3) * 4);
    }
  }
  // Row r0 + lane % 32 (r0 a multiple of 32), contraction slots (columns) STEP i ..
  static __device__ __forceinline__ Fragment along(uint32_t at, int r0, int i) {
    typedef __attribute__((address_space(3))) Fragment lds_fragment;
    return *(const lds_fragment*)(uintptr_t)((at ^ (32 * i)) + r0 * ROW);
  }
  // Column 32 d + lane % 32, contraction slots (rows r0 ..) STEP i .. in the order of pack().
  static __device__ __forceinline__ Fragment down(uint32_t at, int r0, int i, int d) {
    if constexpr (sizeof(T) == 2) {
      // (16 lanes read a block of four rows x 16 columns: lane j supplies the address of row j / 4, columns 4 (j % 4) .. + 3 and receives column j)
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      union {
        s16x4 s[2];
        Fragment v;
      } u;
      u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)((at ^ (64 * d)) + (r0 + 16 * i) * ROW));
      u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)((at ^ (64 * d) ^ 32) + (r0 + 16 * i + 8) * ROW));
      return u.v;
    } else {
      typedef __attribute__((address_space(3))) float lds_float;
      Fragment f;
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = *(const lds_float*)(uintptr_t)((at ^ (128 * d) ^ (swizzle(8 * (i & 1) + e) * 16)) + (r0 + 8 * i + e) * ROW);
      return f;
    }
  }
};

// Rows of a head in memory: bytes from one to the next.
struct Rows {
  const char* p;
  int64_t ld;
};

// ROWS x DP of a tile, moved straight to LDS by THREADS threads, 16 bytes each at a time.
template <typename T, int DP, int ROWS, int THREADS>
struct TileLoad {
  typedef HeadTile<T, DP> Tile;
  static constexpr int BYTES = ROWS * Tile::ROW, PIECES = BYTES / 16 / THREADS;
  static_assert(PIECES * THREADS * 16 == BYTES, "tile / thread count");
  static constexpr int STRIDE = THREADS / Tile::PITCH;   // rows from one piece to the next
  int row, column, width;   // of the first piece, column in bytes; bytes of a row that exist
  __device__ __forceinline__ TileLoad(int tid, int D) : row(tid / Tile::PITCH), column((tid % Tile::PITCH ^ Tile::swizzle(row)) * 16), width(D * (int)sizeof(T)) {}
  // (the permutation of a row is the exclusive or of those of its bits, and the first piece's row is below STRIDE)
  static __host__ __device__ __forceinline__ constexpr int turn(int i) { return Tile::swizzle(i * STRIDE) * 16; }
  static constexpr bool alike() {
    for (int i = 1; i < PIECES; ++i)
      if (turn(i)) return false;
    return true;
  }
  // f(row of the tile, byte in it, byte of LDS) of each piece that exists.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if ((column ^ turn(i)) < width) f(row + i * STRIDE, column ^ turn(i), i * (THREADS * 16));
  }
  // Rows t0 .. of `x` to LDS address `lds` (of the thread's wavefront); zeros from row `end` on.  What lies behind a row's end stays as it is: every
  // row's columns take part in each load, so a wavefront always has as many under way as it has pieces.  Of a tile within the rows, a lane's place in it
  // is one number for all pieces, the rest is the wavefront's (forward, 128 bf16 columns, 8 x 2048 queries and keys, 16 heads: 298-318 us for 330-340).
  __device__ __forceinline__ void operator()(const Rows& x, int64_t t0, int64_t end, uint32_t lds) const {
    const char* base = x.p + t0 * x.ld;
    if (t0 + ROWS <= end && x.ld < 1 << 24) {
      const uint32_t to_row = (uint32_t)row * (uint32_t)x.ld;
      if constexpr (alike()) {
        if (column < width) {
#pragma unroll
          for (int i = 0; i < PIECES; ++i) load_lds16(base + i * STRIDE * x.ld, to_row + column, lds + i * (THREADS * 16));
        }
      } else {
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
          if ((column ^ turn(i)) < width) load_lds16(base + i * STRIDE * x.ld, to_row + (column ^ turn(i)), lds + i * (THREADS * 16));
      }
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int r = row + i * STRIDE, c = column ^ turn(i);
        const char* src = t0 + r < end ? base + r * x.ld + c : reinterpret_cast<const char*>(mfma_zero16);
        if (c < width) load_lds16(src, lds + i * (THREADS * 16));
      }
    }
  }
};

// LDS of `bytes` (a multiple of 16 per thread) cleared by the block: columns behind a row's end are zeros from then on.
__device__ __forceinline__ void clear_lds(char* lds, int bytes, int threads) {
  for (int i = threadIdx.x * 16; i < bytes; i += threads * 16) *reinterpret_cast<uint4*>(lds + i) = make_uint4(0, 0, 0, 0);
}

// Fragments of 32 rows of a head for a whole wavefront, from memory; rows from `end` on and columns from D on are zeros.
template <typename T, int DP>
__device__ __forceinline__ void load_rows(const Rows& x, int64_t r0, int64_t end, int D, int lane, typename Core<T>::Fragment (&f)[DP / Core<T>::STEP]) {
  const int64_t r = r0 + (lane & 31);
  const char* p = x.p + r * x.ld;
#pragma unroll
  for (int i = 0; i < DP / Core<T>::STEP; ++i) {
    const int c = (2 * i + (lane >> 5)) * Core<T>::PER;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (r < end && c < D) w = load16<false>(p + c * (int)sizeof(T));
    f[i] = __builtin_bit_cast(typename Core<T>::Fragment, w);
  }
}

// use(i, read(i)) for i < N in order, with AHEAD fragments under way from LDS: left to itself the compiler asks for each one right before its product,
// which then waits for LDS and not for the matrix core.  first: the first ones may be asked for earlier, by start().
template <typename Fragment, int N, int AHEAD>
struct Fragments {
  Fragment f[AHEAD];
  template <typename R>
  __device__ __forceinline__ void start(R read) {
#pragma unroll
    for (int i = 0; i < AHEAD && i < N; ++i) f[i] = read(i);
    __builtin_amdgcn_sched_barrier(ARITHMETIC);
  }
  template <typename R, typename U>
  __device__ __forceinline__ void run(R read, U use) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      use(i, f[i % AHEAD]);
      __builtin_amdgcn_sched_barrier(ARITHMETIC);
      if (i + AHEAD < N) f[i % AHEAD] = read(i + AHEAD);
      __builtin_amdgcn_sched_barrier(ARITHMETIC);
    }
  }
  static constexpr int ARITHMETIC = 6;   // what may move: vector and scalar instructions
};

__device__ __forceinline__ f32x16 zeros() {
  f32x16 x;
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] = 0.0f;
  return x;
}
// f of what both halves of the wavefront hold for the same column (v_permlane32_swap: no way through LDS).
template <typename F>
__device__ __forceinline__ float over_halves(float x, F f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_of_halves(float x) {
  return over_halves(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_of_halves(float x) {
  return over_halves(x, [](float a, float b) { return a + b; });
}

// 2^x and log2 by one instruction each (off by a unit in the last place).
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }
constexpr float LOG2E = 1.4426950408889634f;

// ------------------------------------------------------------- few queries over many keys (stream.hip)
struct HeadsArg {
  const void* p;
  HeadStrides s;   // bytes
  __device__ __forceinline__ Rows rows(int64_t b, int64_t h) const { return Rows{reinterpret_cast<const char*>(p) + b * s.b + h * s.h, s.l}; }
};
struct StreamArgs {
  HeadsArg q, k, v, out;       // of a cache k and v are [pages, page, heads, D]
  const int32_t* table;        // pages of a cache [B, ldt], or NULL
  const int32_t* q_lengths;    // either may be NULL: all
  const int32_t* k_lengths;
  float* stats;                // [B, q_heads, S] or NULL, see cross_forward_kernel
  int64_t ldt, pages, B, S, T;
  Divisor page;                // tokens of a page
  int32_t q_heads, heads, group, D;
  int32_t row_tile, row_tiles, rows;   // a key head's queries (row r: query r / group of head r mod group) in 16s or 32s; rows of a partial result
  int32_t waves;               // of the launch
  uint32_t first;              // query of a head that a launch of the join begins with
  float scale2;
  uint32_t* before;            // [B + 1] tiles of 32 keys of the sequences before, of a single head and tile of rows
  float* top_sum;              // [waves, 2, rows, 2] maximum and sum of the partial results, and
  float* partial;              // [waves, 2, rows, DP]
};
bool stream_fits(int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads);   // fewer than 2^31 tiles
size_t stream_bytes(int64_t B, int64_t S, int64_t q_heads, int64_t heads, int64_t D);
// The rest of a's fields from its sizes and a workspace of that many bytes; the launches.
hipError_t launch_stream(StreamArgs a, int32_t dtype, void* workspace, hipStream_t s);

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int64_t b, int64_t most) {
  return lengths ? min(max((int64_t)lengths[b], (int64_t)0), most) : most;
}
// go(T, DP) for the type and the columns rounded up.
template <typename F>
auto by_size(int32_t dtype, int D, F go) {
  auto width = [&](auto t) {
    if (D <= 32) return go(t, std::integral_constant<int, 32>());
    if (D <= 64) return go(t, std::integral_constant<int, 64>());
    return go(t, std::integral_constant<int, 128>());
  };
  return dtype == ANTDT_F32 ? width(0.0f) : width((bf16_t)0);
}
// An argument whose heads are read or written 16 bytes at a time.
inline int op_wide_heads(const char* call, const char* name, const void* p, int64_t B, int64_t L, int64_t H, int64_t D, int32_t dtype, HeadStrides s,
                         bool written, HeadsArg& to) {
  const int64_t size = op_size(dtype);
  OP_TRY(op_heads(call, name, p, B, L, H, D, s, size, written));
  if (B == 0 || L == 0 || H == 0) return ANTDT_OK;
  if ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(s.b * size) | (uintptr_t)(s.l * size) | (uintptr_t)(s.h * size)) & 15)
    return op_fail(ANTDT_UNSUPPORTED, "%s: %s: heads start at multiples of 16 bytes", call, name);
  to = HeadsArg{p, {s.b * size, s.l * size, s.h * size}};
  return ANTDT_OK;
}
inline int op_scale(const char* call, float scale) {
  return scale >= 1e-30f && isfinite(scale * LOG2E) ? ANTDT_OK : op_fail(ANTDT_INVALID_ARG, "%s: scale is below 1e-30 or not finite", call);
}
inline int op_head_sizes(const char* call, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype) {
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  if (heads < 1 || q_heads < 1 || q_heads > (1 << 16) || q_heads % heads)
    return op_fail(ANTDT_INVALID_ARG, "%s: %lld heads for %lld of the queries", call, (long long)heads, (long long)q_heads);
  if (D < 8 || D > ANTDT_MAX_ATTENTION_DIM || D % 8)
    return op_fail(ANTDT_UNSUPPORTED, "%s: D is a multiple of 8, at most %d", call, ANTDT_MAX_ATTENTION_DIM);
  return ANTDT_OK;
}

}  // namespace antdt
