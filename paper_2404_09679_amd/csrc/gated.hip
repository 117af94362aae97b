// Gated feed-forward block: h = act(x Wg) * (x Wu), and its backward pass.
//
// Forward: a block multiplies a tile of x with the same columns of Wg and Wu, so that a lane holds both projections of an element of
// h and forms it in its registers; neither projection goes to memory.  For the backward pass it also stores
//   P = act(g),  R = u act'(g)    (fp32: dg = dh R and du = dh P are then rounded once)
// Backward: dz = [dh R | dh P] [N, 2H] (operands of the products, in the type of x), then
//   dx = dz [Wg | Wu]^T,   dWg = x^T dz[:, :H],   dWu = x^T dz[:, H:],
// the weights, x and dz read as they lie in memory.
#include <algorithm>

#include "ops.h"
#include "product.h"

namespace antdt {
namespace {

struct GatedArgs {
  const void* x;
  const void* wg;
  const void* wu;
  void* h;
  float* saved;         // P [N, H], R [N, H], or NULL
  int64_t ldx, ldw, ldh, N, K, H;
  int32_t act, tiles_m, tiles_n;
};

__device__ __forceinline__ float logistic(float x) { return 1.0f / (1.0f + __expf(-x)); }

// p = act(g), r = act'(g).
__device__ __forceinline__ void activation(int act, float g, float& p, float& r) {
  if (act == ANTDT_ACT_SILU) {
    const float s = logistic(g);
    p = g * s;
    r = s * (1.0f + g * (1.0f - s));
  } else if (act == ANTDT_ACT_GELU) {
    const float cdf = 0.5f * (1.0f + erff(g * 0.70710678f));
    p = g * cdf;
    r = cdf + g * __expf(-0.5f * g * g) * 0.39894228f;
  } else if (act == ANTDT_ACT_RELU) {
    p = g <= 0.0f ? 0.0f : g;   // (a NaN stays one)
    r = g > 0.0f ? 1.0f : 0.0f;
  } else {
    const float s = logistic(g);
    p = s;
    r = s * (1.0f - s);
  }
}

__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Tile of block `pid` of a grid of tiles_m x tiles_n: an XCD (block i runs on XCD i mod 8) has a share of consecutive tiles, neighbours
// along the shorter side (of the longer operand its L2 then fetches its share only).
__device__ __forceinline__ void tile_of(int pid, int nblk, int tiles_m, int tiles_n, int& tm, int& tn) {
  pid = (pid & 7) * (nblk >> 3) + min(pid & 7, nblk & 7) + (pid >> 3);
  if (tiles_m < tiles_n) {
    tn = pid / tiles_m;
    tm = pid - tn * tiles_m;
  } else {
    tm = pid / tiles_n;
    tn = pid - tm * tiles_n;
  }
}

// 32 rows of a wavefront's tile to memory, staged in LDS as fp32 so that a row's columns leave 16 bytes at a time.  x[j][e]: as an
// accumulator's elements.  `rows`, `cols`: that exist from there on; VEC: whole 16-byte groups may be written.
template <typename T, int TN, bool VEC>
__device__ __forceinline__ void store_rows(float* st, const f32x16 (&x)[TN], T* out, int64_t ld, int rows, int cols, int lane) {
  constexpr int WN = 32 * TN, SP = WN + 4, PER = 16 / sizeof(T);   // columns of a lane's store
  const int fr = lane & 31, fg = lane >> 5;
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      *reinterpret_cast<float4*>(st + fr * SP + j * 32 + 8 * v + 4 * fg) = make_float4(x[j][4 * v], x[j][4 * v + 1], x[j][4 * v + 2], x[j][4 * v + 3]);
  wave_order();
  constexpr int CPR = WN / PER, RPI = 64 / CPR;
  const int rr = lane / CPR, cc = (lane % CPR) * PER;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += RPI) {
    const int r = r0 + rr;
    const float* s = st + r * SP + cc;
    T* o = out + (int64_t)r * ld + cc;
    if (r < rows && cc < cols) {
      if (VEC) {   // (a whole group exists)
        const float4 a = *reinterpret_cast<const float4*>(s);
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(o) = a;
        } else {
          const float4 b = *reinterpret_cast<const float4*>(s + 4);
          *reinterpret_cast<uint4*>(o) = make_uint4(f2bf2(a.x, a.y), f2bf2(a.z, a.w), f2bf2(b.x, b.y), f2bf2(b.z, b.w));
        }
      } else {
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (cc + e < cols) o[e] = from_f32<T>(s[e]);
      }
    }
  }
  wave_order();
}

template <typename A>
__device__ __forceinline__ void zero(A& acc) {
  f32x16* p = reinterpret_cast<f32x16*>(&acc);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(A) / sizeof(f32x16)); ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) p[i][e] = 0.0f;
}

template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE, int ACT, bool SAVE>
__global__ __launch_bounds__(64 * WR * WC) void gated_kernel(GatedArgs a) {
  typedef TileProduct<T, 2, TM, TN, WR, WC, STAGES, false, true, PIECE> P;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int tm, tn;
  tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
  const int m0 = tm * P::BM, n0 = tn * P::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
  typename P::Acc acc;
  zero(acc);
  const Operand x = {a.x, a.ldx, (int)a.N, m0}, w[2] = {{a.wg, a.ldw, (int)a.H, n0}, {a.wu, a.ldw, (int)a.H, n0}};
  P::run(x, w, (int)a.K, lds, acc);

  constexpr int WN = 32 * TN;
  static_assert(WR * WC * 32 * (WN + 4) * 4 <= P::LDS_BYTES, "epilogue staging");
  float* st = reinterpret_cast<float*>(lds) + wave * (32 * (WN + 4));
  constexpr bool VEC = PIECE == 16;
  const int mw = m0 + wr * (32 * TM), nw = n0 + wc * WN;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = mw + 32 * i;
    const int rows = (int)min(a.N - m, (int64_t)32), cols = (int)a.H - nw;
    f32x16 h[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float p, r;
        const float u = acc[1][i][j][e];
        activation(ACT, acc[0][i][j][e], p, r);
        h[j][e] = p * u;
        if (SAVE) {
          acc[0][i][j][e] = p;
          acc[1][i][j][e] = u * r;
        }
      }
    store_rows<T, TN, VEC>(st, h, reinterpret_cast<T*>(a.h) + m * a.ldh + nw, a.ldh, rows, cols, lane);
    if (SAVE) {
      float* s = a.saved + m * a.H + nw;
      store_rows<float, TN, VEC>(st, acc[0][i], s, a.H, rows, cols, lane);
      store_rows<float, TN, VEC>(st, acc[1][i], s + a.N * a.H, a.H, rows, cols, lane);
    }
  }
}

// dz = [dh R | dh P], [N, 2H].
struct DzArgs {
  const void* dh;
  const float* saved;
  void* dz;
  int64_t lddh, N, H;
};
template <typename T, int Q>
__global__ __launch_bounds__(256) void gated_dz_kernel(DzArgs a) {
  const int64_t per_row = (a.H + 7) / 8, n = a.N * per_row, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const int64_t r = i / per_row, c = (i - r * per_row) * 8;
    const int cols = (int)min((int64_t)8, a.H - c);
    float d[8], p[8], q[8];
    load8<Q>(reinterpret_cast<const T*>(a.dh) + r * a.lddh + c, cols, d);
    load8<Q>(a.saved + r * a.H + c, cols, p);
    load8<Q>(a.saved + (a.N + r) * a.H + c, cols, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] *= d[e];
      q[e] *= d[e];
    }
    T* z = reinterpret_cast<T*>(a.dz) + r * 2 * a.H + c;
    store8<Q>(z, cols, q);
    store8<Q>(z + a.H, cols, p);
  }
}

// dx = dz [Wg | Wu]^T.
struct DxArgs {
  const void* dz;
  const void* wg;
  const void* wu;
  void* dx;
  int64_t ldw, lddx, N, K, H;
  int32_t tiles_m, tiles_n;
};
template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE>
__global__ __launch_bounds__(64 * WR * WC) void gated_dx_kernel(DxArgs a) {
  typedef TileProduct<T, 1, TM, TN, WR, WC, STAGES, false, false, PIECE> P;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int tm, tn;
  tile_of(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_n, tm, tn);
  const int m0 = tm * P::BM, n0 = tn * P::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
  typename P::Acc acc;
  zero(acc);
  const T* dz = reinterpret_cast<const T*>(a.dz);
#pragma unroll 1
  for (int q = 0; q < 2; ++q) {
    const Operand z = {dz + q * a.H, 2 * a.H, (int)a.N, m0}, w[1] = {{q ? a.wu : a.wg, a.ldw, (int)a.K, n0}};
    P::run(z, w, (int)a.H, lds, acc);
  }
  constexpr int WN = 32 * TN;
  static_assert(WR * WC * 32 * (WN + 4) * 4 <= P::LDS_BYTES, "epilogue staging");
  float* st = reinterpret_cast<float*>(lds) + wave * (32 * (WN + 4));
  const int mw = m0 + wr * (32 * TM), nw = n0 + wc * WN;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = mw + 32 * i;
    store_rows<T, TN, PIECE == 16>(st, acc[0][i], reinterpret_cast<T*>(a.dx) + m * a.lddx + nw, a.lddx, (int)min(a.N - m, (int64_t)32), (int)a.K - nw, lane);
  }
}

// dWg = x^T dz[:, :H] and dWu = x^T dz[:, H:]: tiles of both in one launch.
struct DwArgs {
  const void* x;
  const void* dz;
  void* dwg;
  void* dwu;
  int64_t ldx, lddw, N, K, H;
  int32_t tiles_m, tiles_n;   // of one of them
};
template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE>
__global__ __launch_bounds__(64 * WR * WC) void gated_dw_kernel(DwArgs a) {
  typedef TileProduct<T, 1, TM, TN, WR, WC, STAGES, true, true, PIECE> P;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int tm, tn;
  tile_of(blockIdx.x, gridDim.x, a.tiles_m, 2 * a.tiles_n, tm, tn);
  const int second = tn >= a.tiles_n;
  tn -= second ? a.tiles_n : 0;
  const int m0 = tm * P::BM, n0 = tn * P::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
  typename P::Acc acc;
  zero(acc);
  const Operand x = {a.x, a.ldx, (int)a.K, m0};
  const Operand z[1] = {{reinterpret_cast<const T*>(a.dz) + (second ? a.H : 0), 2 * a.H, (int)a.H, n0}};
  P::run(x, z, (int)a.N, lds, acc);
  constexpr int WN = 32 * TN;
  static_assert(WR * WC * 32 * (WN + 4) * 4 <= P::LDS_BYTES, "epilogue staging");
  float* st = reinterpret_cast<float*>(lds) + wave * (32 * (WN + 4));
  T* out = reinterpret_cast<T*>(second ? a.dwu : a.dwg);
  const int mw = m0 + wr * (32 * TM), nw = n0 + wc * WN;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = mw + 32 * i;
    store_rows<T, TN, PIECE == 16>(st, acc[0][i], out + m * a.lddw + nw, a.lddw, (int)min(a.K - m, (int64_t)32), (int)a.H - nw, lane);
  }
}

// ------------------------------------------------------------- launches
template <typename F, typename Args>
hipError_t launch_tiles(F kernel, int blocks, int threads, int bytes, std::atomic<uint64_t>& allowed, const Args& a, hipStream_t s) {
  const hipError_t ok = allow_lds(kernel, bytes, 0, allowed);
  if (ok != hipSuccess) return ok;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), bytes, s, a);
  return hipGetLastError();
}
template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE, int ACT>
hipError_t launch_gated(GatedArgs a, hipStream_t s) {
  typedef TileProduct<T, 2, TM, TN, WR, WC, STAGES, false, true, PIECE> P;
  a.tiles_m = (int)div_up(a.N, P::BM);
  a.tiles_n = (int)div_up(a.H, P::BN);
  static std::atomic<uint64_t> allowed[2];
  if (a.saved)
    return launch_tiles(gated_kernel<T, TM, TN, WR, WC, STAGES, PIECE, ACT, true>, a.tiles_m * a.tiles_n, P::THREADS, P::LDS_BYTES, allowed[1], a, s);
  return launch_tiles(gated_kernel<T, TM, TN, WR, WC, STAGES, PIECE, ACT, false>, a.tiles_m * a.tiles_n, P::THREADS, P::LDS_BYTES, allowed[0], a, s);
}
template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE>
hipError_t launch_gated(const GatedArgs& a, hipStream_t s) {
  switch (a.act) {
    case ANTDT_ACT_SILU: return launch_gated<T, TM, TN, WR, WC, STAGES, PIECE, ANTDT_ACT_SILU>(a, s);
    case ANTDT_ACT_GELU: return launch_gated<T, TM, TN, WR, WC, STAGES, PIECE, ANTDT_ACT_GELU>(a, s);
    case ANTDT_ACT_RELU: return launch_gated<T, TM, TN, WR, WC, STAGES, PIECE, ANTDT_ACT_RELU>(a, s);
    default: return launch_gated<T, TM, TN, WR, WC, STAGES, PIECE, ANTDT_ACT_SIGMOID>(a, s);
  }
}
template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE>
hipError_t launch_dx(DxArgs a, hipStream_t s) {
  typedef TileProduct<T, 1, TM, TN, WR, WC, STAGES, false, false, PIECE> P;
  a.tiles_m = (int)div_up(a.N, P::BM);
  a.tiles_n = (int)div_up(a.K, P::BN);
  static std::atomic<uint64_t> allowed{0};
  return launch_tiles(gated_dx_kernel<T, TM, TN, WR, WC, STAGES, PIECE>, a.tiles_m * a.tiles_n, P::THREADS, P::LDS_BYTES, allowed, a, s);
}
template <typename T, int TM, int TN, int WR, int WC, int STAGES, int PIECE>
hipError_t launch_dw(DwArgs a, hipStream_t s) {
  typedef TileProduct<T, 1, TM, TN, WR, WC, STAGES, true, true, PIECE> P;
  a.tiles_m = (int)div_up(a.K, P::BM);
  a.tiles_n = (int)div_up(a.H, P::BN);
  static std::atomic<uint64_t> allowed{0};
  return launch_tiles(gated_dw_kernel<T, TM, TN, WR, WC, STAGES, PIECE>, a.tiles_m * 2 * a.tiles_n, P::THREADS, P::LDS_BYTES, allowed, a, s);
}

// Tiles of 256 rows and columns as long as they give most compute units a block, smaller ones below.
int64_t tiles(int64_t m, int64_t n, int bm, int bn) { return div_up(m, bm) * div_up(n, bn); }

hipError_t gated_forward(const GatedArgs& a, bool bf16, bool vec, hipStream_t s) {
  if (bf16) {
    if (tiles(a.N, a.H, 256, 128) >= 150) return launch_gated<bf16_t, 4, 1, 2, 4, 2, 16>(a, s);
    return launch_gated<bf16_t, 1, 1, 2, 2, 3, 16>(a, s);
  }
  if (!vec) return launch_gated<float, 1, 1, 2, 2, 3, 4>(a, s);
  if (tiles(a.N, a.H, 128, 64) >= 150) return launch_gated<float, 2, 1, 2, 2, 3, 16>(a, s);
  return launch_gated<float, 1, 1, 2, 2, 3, 16>(a, s);
}
hipError_t gated_dx(const DxArgs& a, bool bf16, bool vec, hipStream_t s) {
  if (bf16) {
    if (tiles(a.N, a.K, 256, 256) >= 150) return launch_dx<bf16_t, 4, 2, 2, 4, 2, 16>(a, s);
    return launch_dx<bf16_t, 1, 1, 2, 2, 3, 16>(a, s);
  }
  if (!vec) return launch_dx<float, 1, 1, 2, 2, 3, 4>(a, s);
  if (tiles(a.N, a.K, 128, 128) >= 150) return launch_dx<float, 2, 2, 2, 2, 3, 16>(a, s);
  return launch_dx<float, 1, 1, 2, 2, 3, 16>(a, s);
}
hipError_t gated_dw(const DwArgs& a, bool bf16, bool vec, hipStream_t s) {
  if (bf16) {
    if (2 * tiles(a.K, a.H, 256, 256) >= 150) return launch_dw<bf16_t, 4, 2, 2, 4, 2, 16>(a, s);
    return launch_dw<bf16_t, 1, 1, 2, 2, 3, 16>(a, s);
  }
  if (!vec) return launch_dw<float, 1, 1, 2, 2, 3, 4>(a, s);
  if (2 * tiles(a.K, a.H, 128, 128) >= 150) return launch_dw<float, 2, 2, 2, 2, 3, 16>(a, s);
  return launch_dw<float, 1, 1, 2, 2, 3, 16>(a, s);
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t dz_bytes(int64_t N, int64_t H, int32_t dtype) { return align256((size_t)(N * 2 * H * op_size(dtype))); }

// Sizes below which a tile's offsets stay in 32 bits.
int gated_sizes(const char* call, int64_t N, int64_t K, int64_t H, int32_t dtype) {
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  if (N < 0 || N >= INT32_MAX - 512 || K < 1 || K >= (1 << 20) || H < 1 || H >= (1 << 20))
    return op_fail(ANTDT_INVALID_ARG, "%s: N, K or H out of range", call);
  const int64_t k = div_up(K, 64), h = div_up(H, 64);   // blocks of a launch, of 256 threads at least
  if (std::max(div_up(N, 64) * std::max(k, h), 2 * k * h) >= (1 << 24)) return op_fail(ANTDT_INVALID_ARG, "%s: N, K or H out of range", call);
  if (dtype == ANTDT_BF16 && ((K | H) & 7)) return op_fail(ANTDT_UNSUPPORTED, "%s: bf16 widths must be multiples of 8", call);
  return ANTDT_OK;
}
int gated_matrix(const char* call, const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype) {
  OP_TRY(op_matrix(call, name, p, rows, cols, ld, op_size(dtype)));
  if (rows == 0 || cols == 0) return ANTDT_OK;
  if (ld >= (1 << 21)) return op_fail(ANTDT_UNSUPPORTED, "%s: %s: leading dimension above 2^21", call, name);
  if (dtype == ANTDT_BF16 && ((ld & 7) || (reinterpret_cast<uintptr_t>(p) & 15)))
    return op_fail(ANTDT_UNSUPPORTED, "%s: %s: bf16 rows must be 16-byte aligned", call, name);
  return ANTDT_OK;
}
bool whole16(const void* p, int64_t ld) { return (ld & 3) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace
}  // namespace antdt

using namespace antdt;

extern "C" {

int antdt_gated_saved_bytes(int64_t N, int64_t H, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_gated_saved_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(gated_sizes(call, N, 8, H, dtype));
  *bytes = (size_t)N * (size_t)H * 8;
  return ANTDT_OK;
}

int antdt_gated_forward_bytes(int64_t N, int64_t K, int64_t H, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_gated_forward_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(gated_sizes(call, N, K, H, dtype));
  *bytes = 0;
  return ANTDT_OK;
}

int antdt_gated_forward(const void* x, int64_t ldx, const void* wg, const void* wu, int64_t ldw, int64_t N, int64_t K, int64_t H, int32_t dtype,
                        int32_t act, void* h, int64_t ldh, void* saved, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "antdt_gated_forward";
  OP_TRY(gated_sizes(call, N, K, H, dtype));
  if (act < ANTDT_ACT_SILU || act > ANTDT_ACT_SIGMOID) return op_fail(ANTDT_INVALID_ARG, "%s: act", call);
  OP_TRY(gated_matrix(call, "x", x, N, K, ldx, dtype));
  OP_TRY(gated_matrix(call, "wg", wg, K, H, ldw, dtype));
  OP_TRY(gated_matrix(call, "wu", wu, K, H, ldw, dtype));
  OP_TRY(gated_matrix(call, "h", h, N, H, ldh, dtype));
  if (saved && (reinterpret_cast<uintptr_t>(saved) & 255)) return op_fail(ANTDT_INVALID_ARG, "%s: saved is not 256-byte aligned", call);
  if (N == 0) return ANTDT_OK;
  GatedArgs a = {x, wg, wu, h, reinterpret_cast<float*>(saved), ldx, ldw, ldh, N, K, H, act, 0, 0};
  const bool vec = whole16(x, ldx) && whole16(wg, ldw) && whole16(wu, ldw) && whole16(h, ldh) && ((K | H) & 3) == 0;
  return op_hip(call, gated_forward(a, dtype == ANTDT_BF16, vec, (hipStream_t)stream));
}

int antdt_gated_backward_bytes(int64_t N, int64_t K, int64_t H, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_gated_backward_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(gated_sizes(call, N, K, H, dtype));
  *bytes = dz_bytes(N, H, dtype);
  return ANTDT_OK;
}

int antdt_gated_backward(const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* wg, const void* wu, int64_t ldw, int64_t N, int64_t K,
                         int64_t H, int32_t dtype, const void* saved, void* dx, int64_t lddx, void* dwg, void* dwu, int64_t lddw, void* workspace,
                         size_t workspace_bytes, void* stream) {
  const char* call = "antdt_gated_backward";
  OP_TRY(gated_sizes(call, N, K, H, dtype));
  if (!dwg != !dwu) return op_fail(ANTDT_INVALID_ARG, "%s: dwg and dwu are wanted together", call);
  OP_TRY(gated_matrix(call, "dh", dh, N, H, lddh, dtype));
  if (dx) OP_TRY(gated_matrix(call, "wg", wg, K, H, ldw, dtype));
  if (dx) OP_TRY(gated_matrix(call, "wu", wu, K, H, ldw, dtype));
  if (dx) OP_TRY(gated_matrix(call, "dx", dx, N, K, lddx, dtype));
  if (dwg) OP_TRY(gated_matrix(call, "x", x, N, K, ldx, dtype));
  if (dwg) OP_TRY(gated_matrix(call, "dwg", dwg, K, H, lddw, dtype));
  if (dwg) OP_TRY(gated_matrix(call, "dwu", dwu, K, H, lddw, dtype));
  if (!dx && !dwg) return ANTDT_OK;
  if (N > 0 && (!saved || (reinterpret_cast<uintptr_t>(saved) & 255))) return op_fail(ANTDT_INVALID_ARG, "%s: saved is null or not 256-byte aligned", call);
  OP_TRY(op_workspace(call, workspace, workspace_bytes, dz_bytes(N, H, dtype)));
  const bool bf16 = dtype == ANTDT_BF16;
  const hipStream_t s = (hipStream_t)stream;
  if (N > 0) {
    const DzArgs d = {dh, reinterpret_cast<const float*>(saved), workspace, lddh, N, H};
    const int q = row_quantum(H, bf16 ? 2 : 4, {{dh, lddh}});
    const dim3 grid((unsigned)std::min<int64_t>(div_up(N * div_up(H, 8), 256), 16384));
    if (bf16) hipLaunchKernelGGL((gated_dz_kernel<bf16_t, 8>), grid, dim3(256), 0, s, d);
    else if (q >= 4) hipLaunchKernelGGL((gated_dz_kernel<float, 4>), grid, dim3(256), 0, s, d);
    else hipLaunchKernelGGL((gated_dz_kernel<float, 1>), grid, dim3(256), 0, s, d);
    OP_TRY(op_hip(call, hipGetLastError()));
  }
  if (dx && N > 0) {
    const DxArgs a = {workspace, wg, wu, dx, ldw, lddx, N, K, H, 0, 0};
    OP_TRY(op_hip(call, gated_dx(a, bf16, whole16(wg, ldw) && whole16(wu, ldw) && whole16(dx, lddx) && ((K | H) & 3) == 0, s)));
  }
  if (dwg) {
    const DwArgs a = {x, workspace, dwg, dwu, ldx, lddw, N, K, H, 0, 0};
    OP_TRY(op_hip(call, gated_dw(a, bf16, whole16(x, ldx) && whole16(dwg, lddw) && whole16(dwu, lddw) && ((K | H) & 3) == 0, s)));
  }
  return ANTDT_OK;
}

}  // extern "C"
