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
  int32_t act;
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

// How the tiles of a product are handed out.  A compute unit holds a few blocks; tiles beyond the last whole filling of the chip would leave
// most of it idle for the time of a tile, so their contraction is cut into `parts`, whose sums go to memory in the order of the accumulators
// and are added up, in order, by a second launch.
struct Split {
  int32_t tiles_m, tiles_n, whole, parts, len;   // len: contraction slots of a part
  float* partial;
  __host__ __device__ int rest() const { return tiles_m * tiles_n - whole; }
  int blocks() const { return whole + rest() * parts; }
};
constexpr int COMPUTE_UNITS = 256, LDS_OF_A_UNIT = 160 * 1024;

template <typename P>
Split plan_split(int64_t rows, int64_t cols, int64_t contraction) {
  Split s = {};
  s.tiles_m = (int)div_up(rows, P::BM);
  s.tiles_n = (int)div_up(cols, P::BN);
  const int64_t tiles = (int64_t)s.tiles_m * s.tiles_n;
  constexpr int per_unit = LDS_OF_A_UNIT / P::LDS_BYTES < 2048 / P::THREADS ? LDS_OF_A_UNIT / P::LDS_BYTES : 2048 / P::THREADS;
  const int64_t slots = COMPUTE_UNITS * per_unit, rest = tiles % slots;
  s.whole = (int)tiles;
  s.parts = 1;
  s.len = (int)contraction;
  const int64_t parts = rest ? std::min<int64_t>({slots / rest, div_up(contraction, 4 * P::SLOTS), 8}) : 1;
  if (parts > 1) {
    s.whole = (int)(tiles - rest);
    s.len = (int)(div_up(div_up(contraction, parts), P::SLOTS) * P::SLOTS);
    s.parts = (int)div_up(contraction, s.len);
  }
  return s;
}
template <typename P>
size_t split_bytes(const Split& s) {
  return s.parts > 1 ? (size_t)s.rest() * s.parts * P::NB_ * P::BM * P::BN * 4 : 0;
}

// Place of block i of n in the order of the work: an XCD (block i runs on XCD i mod 8) has a share of consecutive places.
__device__ __forceinline__ int xcd_order(int i, int n) { return (i & 7) * (n >> 3) + min(i & 7, n & 7) + (i >> 3); }
// Tile `t`: in stripes of 8 along the shorter side, so that the 32 tiles an XCD works on at a time are 8 x 4 and read 12 panels of the operands
// between them (one stripe of all 32 rows: 33 panels, which the other caches have to deliver; 8192 x 2 x 5632 x 2048).
__device__ __forceinline__ void tile_at(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  const bool m_minor = tiles_m < tiles_n;
  const int minor = m_minor ? tiles_m : tiles_n, major = m_minor ? tiles_n : tiles_m;
  const int g = t / (8 * major), in = t - g * 8 * major, w = min(8, minor - 8 * g);
  const int j = in / w, i = 8 * g + (in - j * w);
  tm = m_minor ? i : j;
  tn = m_minor ? j : i;
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

// A product is described by an Op: P, its tiles; Args; product(), the sums of contraction slots [k0, k1) of a tile; finish(), what becomes
// of a tile's sums.
template <typename Op>
__global__ __launch_bounds__(Op::P::THREADS) void tile_kernel(typename Op::Args a, Split sp) {
  typedef typename Op::P P;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int t, part = -1;
  if ((int)blockIdx.x < sp.whole) {
    t = xcd_order(blockIdx.x, sp.whole);
  } else {   // (neighbours: other tiles, the same contraction slots)
    const int rest = sp.rest(), q = xcd_order(blockIdx.x - sp.whole, rest * sp.parts);
    part = q / rest;
    t = sp.whole + (q - part * rest);
  }
  int tm, tn;
  tile_at(t, sp.tiles_m, sp.tiles_n, tm, tn);
  typename P::Acc acc;
  zero(acc);
  const int length = Op::contraction(a);
  if (part < 0) {
    Op::product(a, tm, tn, 0, length, lds, acc);
    Op::finish(a, tm, tn, lds, acc);
  } else {
    Op::product(a, tm, tn, part * sp.len, min((part + 1) * sp.len, length), lds, acc);
    constexpr int N16 = (int)(sizeof(acc) / sizeof(f32x16));
    const f32x16* x = reinterpret_cast<const f32x16*>(&acc);
    f32x4v* out = reinterpret_cast<f32x4v*>(sp.partial) + ((int64_t)(t - sp.whole) * sp.parts + part) * (N16 * 4 * P::THREADS) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < N16; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        out[(i * 4 + v) * P::THREADS] = f32x4v{x[i][4 * v], x[i][4 * v + 1], x[i][4 * v + 2], x[i][4 * v + 3]};
  }
}
template <typename Op>
__global__ __launch_bounds__(Op::P::THREADS) void join_kernel(typename Op::Args a, Split sp) {
  typedef typename Op::P P;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int tm, tn;
  tile_at(sp.whole + blockIdx.x, sp.tiles_m, sp.tiles_n, tm, tn);
  typename P::Acc acc;
  zero(acc);
  constexpr int N16 = (int)(sizeof(acc) / sizeof(f32x16));
  f32x16* x = reinterpret_cast<f32x16*>(&acc);
  const f32x4v* in = reinterpret_cast<const f32x4v*>(sp.partial) + (int64_t)blockIdx.x * sp.parts * (N16 * 4 * P::THREADS) + threadIdx.x;
#pragma unroll 1
  for (int p = 0; p < sp.parts; ++p, in += N16 * 4 * P::THREADS)
#pragma unroll
    for (int i = 0; i < N16; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4v y = in[(i * 4 + v) * P::THREADS];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][4 * v + e] += y[e];
      }
  Op::finish(a, tm, tn, lds, acc);
}
// The part of an operand from contraction slot k on.
template <typename T, bool STRIDED>
__device__ __forceinline__ Operand operand(const void* x, int64_t ld, int64_t rows, int r0, int64_t k) {
  return Operand{reinterpret_cast<const T*>(x) + (STRIDED ? k * ld : k), ld, (int)rows, r0};
}
// Sums of a wavefront's tile to memory.
template <typename P, typename T, bool VEC>
__device__ __forceinline__ void store_tile(const f32x16 (&x)[P::TM_][P::TN_], char* lds, T* out, int64_t ld, int64_t rows, int64_t cols, int tm, int tn) {
  constexpr int WN = 32 * P::TN_;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / P::WC_, wc = wave % P::WC_;
  float* st = reinterpret_cast<float*>(lds) + wave * (32 * (WN + 4));
  const int64_t mw = (int64_t)tm * P::BM + wr * (32 * P::TM_), nw = (int64_t)tn * P::BN + wc * WN;
#pragma unroll
  for (int i = 0; i < P::TM_; ++i) {
    const int64_t m = mw + 32 * i;
    store_rows<T, P::TN_, VEC>(st, x[i], out + m * ld + nw, ld, (int)max(min(rows - m, (int64_t)32), (int64_t)0), (int)(cols - nw), lane);
  }
}

template <typename T, typename P_, bool VEC, int ACT, bool SAVE>
struct ForwardOp {
  typedef P_ P;
  typedef GatedArgs Args;
  static __device__ __forceinline__ int contraction(const Args& a) { return (int)a.K; }
  static __device__ __forceinline__ void product(const Args& a, int tm, int tn, int k0, int k1, char* lds, typename P::Acc& acc) {
    const Operand w[2] = {operand<T, true>(a.wg, a.ldw, a.H, tn * P::BN, k0), operand<T, true>(a.wu, a.ldw, a.H, tn * P::BN, k0)};
    P::run(operand<T, false>(a.x, a.ldx, a.N, tm * P::BM, k0), w, k1 - k0, lds, acc);
  }
  static __device__ __forceinline__ void finish(const Args& a, int tm, int tn, char* lds, typename P::Acc& acc) {
    constexpr int TN = P::TN_, WN = 32 * TN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / P::WC_, wc = wave % P::WC_;
    float* st = reinterpret_cast<float*>(lds) + wave * (32 * (WN + 4));
    const int64_t mw = (int64_t)tm * P::BM + wr * (32 * P::TM_), nw = (int64_t)tn * P::BN + wc * WN;
#pragma unroll
    for (int i = 0; i < P::TM_; ++i) {
      const int64_t m = mw + 32 * i;
      const int rows = (int)max(min(a.N - m, (int64_t)32), (int64_t)0), cols = (int)(a.H - nw);
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
};

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

// dx = dz [Wg | Wu]^T, a contraction over the columns of one and then of the other.
struct DxArgs {
  const void* dz;
  const void* wg;
  const void* wu;
  void* dx;
  int64_t ldw, lddx, N, K, H;
};
template <typename T, typename P_, bool VEC>
struct DxOp {
  typedef P_ P;
  typedef DxArgs Args;
  static __device__ __forceinline__ int contraction(const Args& a) { return (int)(2 * a.H); }
  static __device__ __forceinline__ void product(const Args& a, int tm, int tn, int k0, int k1, char* lds, typename P::Acc& acc) {
    const int H = (int)a.H;
#pragma unroll 1
    for (int q = 0; q < 2; ++q) {
      const int from = max(k0, q * H), to = min(k1, (q + 1) * H);
      const Operand w[1] = {operand<T, false>(q ? a.wu : a.wg, a.ldw, a.K, tn * P::BN, from - q * H)};
      P::run(operand<T, false>(a.dz, 2 * a.H, a.N, tm * P::BM, from), w, to - from, lds, acc);
    }
  }
  static __device__ __forceinline__ void finish(const Args& a, int tm, int tn, char* lds, typename P::Acc& acc) {
    store_tile<P, T, VEC>(acc[0], lds, reinterpret_cast<T*>(a.dx), a.lddx, a.N, a.K, tm, tn);
  }
};

// dWg = x^T dz[:, :H] and dWu = x^T dz[:, H:]: columns of tiles of the one, then of the other.
struct DwArgs {
  const void* x;
  const void* dz;
  void* dwg;
  void* dwu;
  int64_t ldx, lddw, N, K, H;
  int32_t tiles_h;   // tiles along H of one of them
};
template <typename T, typename P_, bool VEC>
struct DwOp {
  typedef P_ P;
  typedef DwArgs Args;
  static __device__ __forceinline__ int contraction(const Args& a) { return (int)a.N; }
  static __device__ __forceinline__ void product(const Args& a, int tm, int tn, int k0, int k1, char* lds, typename P::Acc& acc) {
    const bool second = tn >= a.tiles_h;
    const Operand z[1] = {
        operand<T, true>(reinterpret_cast<const T*>(a.dz) + (second ? a.H : 0), 2 * a.H, a.H, (second ? tn - a.tiles_h : tn) * P::BN, k0)};
    P::run(operand<T, true>(a.x, a.ldx, a.K, tm * P::BM, k0), z, k1 - k0, lds, acc);
  }
  static __device__ __forceinline__ void finish(const Args& a, int tm, int tn, char* lds, typename P::Acc& acc) {
    const bool second = tn >= a.tiles_h;
    store_tile<P, T, VEC>(acc[0], lds, reinterpret_cast<T*>(second ? a.dwu : a.dwg), a.lddw, a.K, a.H, tm, second ? tn - a.tiles_h : tn);
  }
};

// ------------------------------------------------------------- launches
template <typename Op>
hipError_t launch_op(const typename Op::Args& a, const Split& sp, hipStream_t s) {
  typedef typename Op::P P;
  static_assert(P::WAVES * 32 * (32 * P::TN_ + 4) * 4 <= P::LDS_BYTES, "staging of the results");
  static std::atomic<uint64_t> allowed[2];
  hipError_t e = allow_lds(tile_kernel<Op>, P::LDS_BYTES, 0, allowed[0]);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(tile_kernel<Op>, dim3(sp.blocks()), dim3(P::THREADS), P::LDS_BYTES, s, a, sp);
  e = hipGetLastError();
  if (e != hipSuccess || sp.parts == 1) return e;
  constexpr int bytes = P::WAVES * 32 * (32 * P::TN_ + 4) * 4;
  e = allow_lds(join_kernel<Op>, bytes, 0, allowed[1]);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(join_kernel<Op>, dim3(sp.rest()), dim3(P::THREADS), bytes, s, a, sp);
  return hipGetLastError();
}

template <typename P, typename T, bool VEC>
struct Tiling {   // of a product: its tiles' class, operands' type, whether whole 16-byte groups may be written
  typedef P Product;
  typedef T Type;
  static constexpr bool vec = VEC;
};
template <typename T, int NB, int TM, int TN, int WR, int WC, int STAGES, bool AS, bool BS, int PIECE>
using TilingOf = Tiling<TileProduct<T, NB, TM, TN, WR, WC, sizeof(T) == 2 ? 64 : 32, STAGES, AS, BS, PIECE>, T, PIECE == 16>;

int64_t tiles(int64_t m, int64_t n, int bm, int bn) { return div_up(m, bm) * div_up(n, bn); }

// f(tiling) with the tiles of a rows x cols result (of NB products at a time): of 256 rows and columns as long as they give most compute
// units a block, smaller ones below.
template <int NB, bool AS, bool BS, typename F>
auto with_tiles(bool bf16, bool vec, int64_t rows, int64_t cols, F&& f) {
  if (bf16) {
    if (tiles(rows, cols, 256, 256 / NB) >= 150) return f(TilingOf<bf16_t, NB, 4, 2 / NB, 2, 4, 2, AS, BS, 16>());
    return f(TilingOf<bf16_t, NB, 1, 1, 2, 2, 3, AS, BS, 16>());
  }
  if (!vec) return f(TilingOf<float, NB, 1, 1, 2, 2, 3, AS, BS, 4>());
  if (tiles(rows, cols, 128, 128 / NB) >= 150) return f(TilingOf<float, NB, 2, 2 / NB, 2, 2, 3, AS, BS, 16>());
  return f(TilingOf<float, NB, 1, 1, 2, 2, 3, AS, BS, 16>());
}

template <typename G, bool SAVE>
hipError_t launch_forward(const GatedArgs& a, const Split& sp, hipStream_t s) {
  typedef typename G::Product P;
  typedef typename G::Type T;
  switch (a.act) {
    case ANTDT_ACT_SILU: return launch_op<ForwardOp<T, P, G::vec, ANTDT_ACT_SILU, SAVE>>(a, sp, s);
    case ANTDT_ACT_GELU: return launch_op<ForwardOp<T, P, G::vec, ANTDT_ACT_GELU, SAVE>>(a, sp, s);
    case ANTDT_ACT_RELU: return launch_op<ForwardOp<T, P, G::vec, ANTDT_ACT_RELU, SAVE>>(a, sp, s);
    default: return launch_op<ForwardOp<T, P, G::vec, ANTDT_ACT_SIGMOID, SAVE>>(a, sp, s);
  }
}
hipError_t gated_forward(const GatedArgs& a, bool bf16, bool vec, float* partial, hipStream_t s) {
  return with_tiles<2, false, true>(bf16, vec, a.N, a.H, [&](auto g) {
    Split sp = plan_split<typename decltype(g)::Product>(a.N, a.H, a.K);
    sp.partial = partial;
    return a.saved ? launch_forward<decltype(g), true>(a, sp, s) : launch_forward<decltype(g), false>(a, sp, s);
  });
}
hipError_t gated_dx(const DxArgs& a, bool bf16, bool vec, float* partial, hipStream_t s) {
  return with_tiles<1, false, false>(bf16, vec, a.N, a.K, [&](auto g) {
    typedef decltype(g) G;
    Split sp = plan_split<typename G::Product>(a.N, a.K, 2 * a.H);
    sp.partial = partial;
    return launch_op<DxOp<typename G::Type, typename G::Product, G::vec>>(a, sp, s);
  });
}
// (both weights' tiles side by side; a column of tiles belongs to one of them)
template <typename P>
Split plan_dw(int64_t N, int64_t K, int64_t H) { return plan_split<P>(K, 2 * div_up(H, P::BN) * P::BN, N); }
hipError_t gated_dw(const DwArgs& args, bool bf16, bool vec, float* partial, hipStream_t s) {
  return with_tiles<1, true, true>(bf16, vec, args.K, 2 * args.H, [&](auto g) {
    typedef decltype(g) G;
    DwArgs a = args;
    Split sp = plan_dw<typename G::Product>(a.N, a.K, a.H);
    sp.partial = partial;
    a.tiles_h = sp.tiles_n / 2;
    return launch_op<DwOp<typename G::Type, typename G::Product, G::vec>>(a, sp, s);
  });
}

// Bytes of the partial sums, whichever way the rows lie.
template <typename F>
size_t most_bytes(bool bf16, F&& f) { return bf16 ? f(true) : std::max(f(false), f(true)); }
size_t forward_bytes(int64_t N, int64_t K, int64_t H, bool bf16) {
  if (N == 0) return 0;
  return most_bytes(bf16, [&](bool vec) {
    return with_tiles<2, false, true>(bf16, vec, N, H, [&](auto g) {
      typedef typename decltype(g)::Product P;
      return split_bytes<P>(plan_split<P>(N, H, K));
    });
  });
}
size_t backward_partial_bytes(int64_t N, int64_t K, int64_t H, bool bf16) {
  if (N == 0) return 0;
  const size_t dx = most_bytes(bf16, [&](bool vec) {
    return with_tiles<1, false, false>(bf16, vec, N, K, [&](auto g) {
      typedef typename decltype(g)::Product P;
      return split_bytes<P>(plan_split<P>(N, K, 2 * H));
    });
  });
  const size_t dw = most_bytes(bf16, [&](bool vec) {
    return with_tiles<1, true, true>(bf16, vec, K, 2 * H, [&](auto g) {
      typedef typename decltype(g)::Product P;
      return split_bytes<P>(plan_dw<P>(N, K, H));
    });
  });
  return std::max(dx, dw);   // (one after the other)
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
  *bytes = forward_bytes(N, K, H, dtype == ANTDT_BF16);
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
  OP_TRY(op_workspace(call, workspace, workspace_bytes, forward_bytes(N, K, H, dtype == ANTDT_BF16)));
  const GatedArgs a = {x, wg, wu, h, reinterpret_cast<float*>(saved), ldx, ldw, ldh, N, K, H, act};
  const bool vec = whole16(x, ldx) && whole16(wg, ldw) && whole16(wu, ldw) && whole16(h, ldh) && ((K | H) & 3) == 0;
  return op_hip(call, gated_forward(a, dtype == ANTDT_BF16, vec, reinterpret_cast<float*>(workspace), (hipStream_t)stream));
}

int antdt_gated_backward_bytes(int64_t N, int64_t K, int64_t H, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_gated_backward_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(gated_sizes(call, N, K, H, dtype));
  *bytes = dz_bytes(N, H, dtype) + backward_partial_bytes(N, K, H, dtype == ANTDT_BF16);
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
  const bool bf16 = dtype == ANTDT_BF16;
  OP_TRY(op_workspace(call, workspace, workspace_bytes, dz_bytes(N, H, dtype) + backward_partial_bytes(N, K, H, bf16)));
  float* partial = N > 0 ? reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + dz_bytes(N, H, dtype)) : nullptr;
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
    const DxArgs a = {workspace, wg, wu, dx, ldw, lddx, N, K, H};
    OP_TRY(op_hip(call, gated_dx(a, bf16, whole16(wg, ldw) && whole16(wu, ldw) && whole16(dx, lddx) && ((K | H) & 3) == 0, partial, s)));
  }
  if (dwg) {
    const DwArgs a = {x, workspace, dwg, dwu, ldx, lddw, N, K, H, 0};
    OP_TRY(op_hip(call, gated_dw(a, bf16, whole16(x, ldx) && whole16(dwg, lddw) && whole16(dwu, lddw) && ((K | H) & 3) == 0, partial, s)));
  }
  return ANTDT_OK;
}

}  // extern "C"
