// Gated feed-forward block: h = act(x Wg) * (x Wu), and its backward pass.
//
// Forward: a block multiplies a tile of x with the same columns of Wg and Wu, so that a lane holds both projections of an element of
// h and forms it in its registers; neither projection goes to memory.  For the backward pass it also stores
//   P = act(g),  R = u act'(g)    (fp32: dg = dh R and du = dh P are then rounded once)
// Backward: dz = [dh R | dh P] [N, 2H], rounded to the type of x (the matrix cores multiply bf16 operands; from exact dz the gradients would be off
// by the results' own rounding, 0.0017 of their norm, so by 0.0023), then
//   dx = dz [Wg | Wu]^T,   dWg = x^T dz[:, :H],   dWu = x^T dz[:, H:],
// the weights, x and dz read as they lie in memory.
#include <algorithm>

#include "ops.h"
#include "product.h"
#include "sort.h"

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

// (the reciprocal by one instruction, off by a unit at most: a correctly rounded quotient takes ten)
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// p = act(g), r = act'(g).
__device__ __forceinline__ void activation(int act, float g, float& p, float& r) {
  if (act == ANTDT_ACT_SILU) {
    const float s = logistic(g);
    p = g * s;
    r = fmaf(p, 1.0f - s, s);
  } else if (act == ANTDT_ACT_GELU) {
    const float cdf = 0.5f * (1.0f + erff(g * 0.70710678f));
    p = g * cdf;
    r = cdf + g * __expf(-0.5f * g * g) * 0.39894228f;
  } else if (act == ANTDT_ACT_RELU) {
    p = g <= 0.0f ? 0.0f : g;   // (a NaN stays one)
    r = g > 0.0f ? 1.0f : 0.0f;
  } else {   // s (1 - s) from e^-|g|: 1 - s has no digits left where s is near 1
    const float e = __expf(-fabsf(g)), t = __builtin_amdgcn_rcpf(1.0f + e);
    p = g < 0.0f ? e * t : t;
    r = e * t * t;
  }
}

// How the tiles of a product are handed out: the first `whole` to a block each, the contraction of the others in `parts`, whose sums go to
// memory in the order of the accumulators and are added up, in order, by a second launch.
struct Split {
  int32_t tiles_m, tiles_n, whole, parts, len;   // len: contraction slots of a part
  int32_t halves;                                // the others by two blocks of half the rows each instead (see halves_kernel)
  float* partial;
  __host__ __device__ int rest() const { return tiles_m * tiles_n - whole; }
  __host__ __device__ int blocks() const { return whole + rest() * (halves ? 2 : parts); }
};

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
  wave_lds_order();
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
          store16<false>(o, bits4(a.x, a.y, a.z, a.w));
        } else {
          const float4 b = *reinterpret_cast<const float4*>(s + 4);
          store16<false>(o, make_uint4(f2bf2(a.x, a.y), f2bf2(a.z, a.w), f2bf2(b.x, b.y), f2bf2(b.z, b.w)));
        }
      } else {
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (cc + e < cols) o[e] = from_f32<T>(s[e]);
      }
    }
  }
  wave_lds_order();
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
__device__ __forceinline__ void finish_tile(const typename Op::Args& a, int tm, int tn, char* lds, const typename Op::P::Acc& acc) {
  typedef typename Op::P P;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* st = reinterpret_cast<float*>(lds) + wave * (32 * (32 * P::TN_ + 4));
#pragma unroll
  for (int i = 0; i < P::TM_; ++i) {
    f32x16 x[P::NB_][P::TN_];
#pragma unroll
    for (int q = 0; q < P::NB_; ++q)
#pragma unroll
      for (int j = 0; j < P::TN_; ++j) x[q][j] = acc[q][i][j];
    Op::finish(a, tm, tn, wave, i, st, x);
  }
}
template <typename Op>
__device__ __forceinline__ void tile_block(const typename Op::Args& a, const Split& sp, int block, char* lds) {
  typedef typename Op::P P;
  int t, part = -1;
  if (block < sp.whole) {
    t = xcd_order(block, sp.whole);
  } else {   // (neighbours: other tiles, the same contraction slots)
    const int rest = sp.rest(), q = xcd_order(block - sp.whole, rest * sp.parts);
    part = q / rest;
    t = sp.whole + (q - part * rest);
  }
  int tm, tn;
  tile_at(t, sp.tiles_m, sp.tiles_n, tm, tn);
  typename P::Acc acc;
  zero(acc);
  const int length = Op::contraction(a);
  Op::product(a, tm, tn, part < 0 ? 0 : part * sp.len, part < 0 ? length : min((part + 1) * sp.len, length), lds, acc);
  if (part < 0) {
    finish_tile<Op>(a, tm, tn, lds, acc);
  } else {
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
// 32 rows of a wavefront's tile by one wavefront (few tiles are in parts, but each is as much to read as many results).  Blocks of two: 777
// tokens of 520-1400, backward pass, blocks of four 27.5 us, so 24.8.
constexpr int JOIN_WAVES = 2;
template <typename P>
constexpr int join_units() { return P::WAVES * P::TM_; }   // of a tile
template <typename Op>
__device__ __forceinline__ void join_rows(const typename Op::Args& a, const Split& sp, int unit, char* lds) {
  typedef typename Op::P P;
  constexpr int UNITS = join_units<P>(), N16 = P::NB_ * P::TM_ * P::TN_;
  const int tile = unit / UNITS, in_tile = unit - tile * UNITS, wave = in_tile / P::TM_, i = in_tile - wave * P::TM_;
  if (tile >= sp.rest()) return;
  int tm, tn;
  tile_at(sp.whole + tile, sp.tiles_m, sp.tiles_n, tm, tn);
  f32x16 x[P::NB_][P::TN_] = {};
  const int lane = threadIdx.x & 63;
  const f32x4v* in = reinterpret_cast<const f32x4v*>(sp.partial) + (int64_t)tile * sp.parts * (N16 * 4 * P::THREADS) + wave * 64 + lane;
#pragma unroll 2
  for (int p = 0; p < sp.parts; ++p, in += N16 * 4 * P::THREADS)
#pragma unroll
    for (int q = 0; q < P::NB_; ++q)
#pragma unroll
      for (int j = 0; j < P::TN_; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const f32x4v y = in[(((q * P::TM_ + i) * P::TN_ + j) * 4 + v) * P::THREADS];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[q][j][4 * v + e] += y[e];
        }
  Op::finish(a, tm, tn, wave, i, reinterpret_cast<float*>(lds) + (threadIdx.x >> 6) * (32 * (32 * P::TN_ + 4)), x);
}
template <typename Op>
__global__ __launch_bounds__(Op::P::THREADS) void tile_kernel(typename Op::Args a, Split sp) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  tile_block<Op>(a, sp, blockIdx.x, lds);
}
// Tiles of Op, and of those behind the last whole filling of the chip the upper and lower halves, tiles of Half.  The upper halves come first and the lower
// ones last: that halves what the last filling costs, without partial sums, and from then on some compute units write the results of a tile (10 bytes an
// element where they are saved) while others multiply.  (The upper halves to four XCDs and the lower ones to the others, so that the blocks of an XCD stay at
// the same contraction slots: 8192 tokens of 2048-5632 saving 378 / 382 us.)
template <typename Op, typename Half>
__global__ __launch_bounds__(Op::P::THREADS) void halves_kernel(typename Op::Args a, Split sp) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int rest = sp.rest(), block = blockIdx.x;
  int tm, tn;
  if (block >= rest && block < rest + sp.whole) {
    typename Op::P::Acc acc;
    zero(acc);
    tile_at(xcd_order(block - rest, sp.whole), sp.tiles_m, sp.tiles_n, tm, tn);
    Op::product(a, tm, tn, 0, Op::contraction(a), lds, acc);
    finish_tile<Op>(a, tm, tn, lds, acc);
  } else {
    const int lower = block >= rest;
    typename Half::P::Acc acc;
    zero(acc);
    tile_at(sp.whole + (lower ? block - sp.whole - rest : block), sp.tiles_m, sp.tiles_n, tm, tn);
    tm = 2 * tm + lower;
    if (tm * Half::P::BM >= Op::rows(a)) return;
    Half::product(a, tm, tn, 0, Op::contraction(a), lds, acc);
    finish_tile<Half>(a, tm, tn, lds, acc);
  }
}
template <typename Op>
__global__ __launch_bounds__(64 * JOIN_WAVES) void join_kernel(typename Op::Args a, Split sp) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  join_rows<Op>(a, sp, blockIdx.x * JOIN_WAVES + (threadIdx.x >> 6), lds);
}
// Two products that do not wait for each other in one launch: the second's blocks fill what the first's leave (and a launch is saved: of 777
// tokens of 520-1400, 25 us in two, 16 in one).
template <typename Op1, typename Op2>
__global__ __launch_bounds__(Op1::P::THREADS) void tile_pair_kernel(typename Op1::Args a1, Split sp1, typename Op2::Args a2, Split sp2) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int n = sp1.blocks();
  if ((int)blockIdx.x < n) tile_block<Op1>(a1, sp1, blockIdx.x, lds);
  else tile_block<Op2>(a2, sp2, blockIdx.x - n, lds);
}
template <typename Op1, typename Op2>
__global__ __launch_bounds__(64 * JOIN_WAVES) void join_pair_kernel(typename Op1::Args a1, Split sp1, typename Op2::Args a2, Split sp2) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int n = sp1.parts > 1 ? sp1.rest() * join_units<typename Op1::P>() : 0, unit = blockIdx.x * JOIN_WAVES + (threadIdx.x >> 6);
  if (unit < n) join_rows<Op1>(a1, sp1, unit, lds);
  else join_rows<Op2>(a2, sp2, unit - n, lds);
}
// The part of an operand from contraction slot k on.
template <typename T, bool STRIDED>
__device__ __forceinline__ Operand operand(const void* x, int64_t ld, int64_t rows, int r0, int64_t k) {
  return Operand{reinterpret_cast<const T*>(x) + (STRIDED ? k * ld : k), ld, (int)rows, r0};
}
// Where the 32 rows `i` of wavefront `wave`'s part of tile (tm, tn) lie in a rows x cols result, and how much of them exists.
struct Place {
  int64_t m, n;
  int rows, cols;
};
template <typename P>
__device__ __forceinline__ Place place(int tm, int tn, int wave, int i, int64_t rows, int64_t cols) {
  Place p;
  p.m = (int64_t)tm * P::BM + wave / P::WC_ * (32 * P::TM_) + 32 * i;
  p.n = (int64_t)tn * P::BN + wave % P::WC_ * (32 * P::TN_);
  p.rows = (int)max(min(rows - p.m, (int64_t)32), (int64_t)0);
  p.cols = (int)max(min(cols - p.n, (int64_t)(32 * P::TN_)), (int64_t)0);
  return p;
}

template <typename T, typename P_, bool VEC, int ACT, bool SAVE>
struct ForwardOp {
  typedef P_ P;
  typedef GatedArgs Args;
  static __device__ __forceinline__ int contraction(const Args& a) { return (int)a.K; }
  static __device__ __forceinline__ int64_t rows(const Args& a) { return a.N; }
  static __device__ __forceinline__ void product(const Args& a, int tm, int tn, int k0, int k1, char* lds, typename P::Acc& acc) {
    const Operand w[2] = {operand<T, true>(a.wg, a.ldw, a.H, tn * P::BN, k0), operand<T, true>(a.wu, a.ldw, a.H, tn * P::BN, k0)};
    P::run(operand<T, false>(a.x, a.ldx, a.N, tm * P::BM, k0), w, k1 - k0, lds, acc);
  }
  static __device__ __forceinline__ void finish(const Args& a, int tm, int tn, int wave, int i, float* st, f32x16 (&x)[2][P::TN_]) {
    constexpr int TN = P::TN_;
    const int lane = threadIdx.x & 63;
    const Place at = place<P>(tm, tn, wave, i, a.N, a.H);
    f32x16 h[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float p, r;
        const float u = x[1][j][e];
        activation(ACT, x[0][j][e], p, r);
        h[j][e] = p * u;
        if (SAVE) {
          x[0][j][e] = p;
          x[1][j][e] = u * r;
        }
      }
    store_rows<T, TN, VEC>(st, h, reinterpret_cast<T*>(a.h) + at.m * a.ldh + at.n, a.ldh, at.rows, at.cols, lane);
    if (SAVE) {
      float* s = a.saved + at.m * a.H + at.n;
      store_rows<float, TN, VEC>(st, x[0], s, a.H, at.rows, at.cols, lane);
      store_rows<float, TN, VEC>(st, x[1], s + a.N * a.H, a.H, at.rows, at.cols, lane);
    }
  }
};

// The forward pass for a few tokens, bound by reading the weights once: a block has 2^c lanes along H, of 16 bytes each, and as many rows of the
// weights at a time as its other lanes make; products and sums in fp32 on the vector units, the lanes' sums added up at the end.
// By tiles / here, us: bf16 1 and 2 tokens of 1024-4096 7.7 / 5.5 and 6.0, 4 of 2048-5632 14.6 / 17.7; fp32 8 of 1024-4096 18.4 / 12.1, of 4096-14336
// 145 / 129.
// Blocks of 256 / 512 / 1024 threads, other weights every time (the more loads under way the better): 1 token bf16 1024-4096 6.7 / 6.5 / 6.7, 2048-5632
// 17.0 / 15.4 / 15.5, 4096-14336 53 / 47 / 51; fp32 8 of 2048-5632 53 / 35 / 28.
constexpr int FEW_THREADS = 512;
constexpr int few_tokens(size_t element) { return element == 4 ? 8 : 2; }

// The sums of v[0 .. COUNT) over the lanes that differ in bits O and above: at every step a lane keeps one half of the values and hands
// on the other, so that COUNT values cost about COUNT exchanges.  Afterwards v[0] .. are those from the returned one on.
template <int COUNT, int O>
__device__ __forceinline__ int sum_over_lanes(float* v, int lane, int first) {
  if constexpr (O >= 64) {
    return first;
  } else if constexpr (COUNT > 1) {
    constexpr int HALF = COUNT / 2;
    const bool up = (lane & O) != 0;
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
      const float keep = up ? v[HALF + i] : v[i], give = up ? v[i] : v[HALF + i];
      v[i] = keep + __shfl_xor(give, O, 64);
    }
    return sum_over_lanes<HALF, 2 * O>(v, lane, first + (up ? HALF : 0));
  } else {
    v[0] += __shfl_xor(v[0], O, 64);
    return sum_over_lanes<1, 2 * O>(v, lane, first);
  }
}

template <typename T, int NT, int LANES>   // NT >= N
__global__ __launch_bounds__(FEW_THREADS) void gated_few_kernel(GatedArgs a) {
  constexpr int VN = 16 / sizeof(T), U = NT > 4 ? 2 : 4, WAVES = FEW_THREADS / 64, STEP = FEW_THREADS / LANES, WIDTH = LANES * VN, COUNT = NT * 2 * VN;
  constexpr int LEFT = COUNT * LANES / 64 > 0 ? COUNT * LANES / 64 : 1;   // values of a lane after the sum
  __shared__ float red[WAVES][LANES][COUNT];
  const int l = threadIdx.x & (LANES - 1), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c0 = (int64_t)xcd_order(blockIdx.x, gridDim.x) * WIDTH, c = min(c0 + l * VN, a.H - VN);   // (H is a multiple of VN; what lies behind is not stored)
  const T* x = reinterpret_cast<const T*>(a.x);
  const T* wg = reinterpret_cast<const T*>(a.wg) + c;
  const T* wu = reinterpret_cast<const T*>(a.wu) + c;
  float acc[COUNT] = {};   // [token][matrix][column]
  const int K = (int)a.K, N = (int)a.N;
  for (int k0 = threadIdx.x / LANES; k0 < K; k0 += U * STEP) {
    uint4 g[U], u[U];
    float xv[U][NT];
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int64_t k = min(k0 + q * STEP, K - 1);
      g[q] = *reinterpret_cast<const uint4*>(wg + k * a.ldw);
      u[q] = *reinterpret_cast<const uint4*>(wu + k * a.ldw);
#pragma unroll
      for (int t = 0; t < NT; ++t) xv[q][t] = to_f32(x[(int64_t)min(t, N - 1) * a.ldx + k]);
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
      if (k0 + q * STEP >= K) continue;
      const uint32_t gw[4] = {g[q].x, g[q].y, g[q].z, g[q].w}, uw[4] = {u[q].x, u[q].y, u[q].z, u[q].w};
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        const float gv = VN == 4 ? __uint_as_float(gw[e % 4]) : __uint_as_float(e & 1 ? gw[e / 2 % 4] & 0xFFFF0000u : gw[e / 2 % 4] << 16);
        const float uv = VN == 4 ? __uint_as_float(uw[e % 4]) : __uint_as_float(e & 1 ? uw[e / 2 % 4] & 0xFFFF0000u : uw[e / 2 % 4] << 16);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[(t * 2) * VN + e] = fmaf(xv[q][t], gv, acc[(t * 2) * VN + e]);
          acc[(t * 2 + 1) * VN + e] = fmaf(xv[q][t], uv, acc[(t * 2 + 1) * VN + e]);
        }
      }
    }
  }
  const int first = sum_over_lanes<COUNT, LANES>(acc, lane, 0);
#pragma unroll
  for (int i = 0; i < LEFT; ++i) red[wave][l][first + i] = acc[i];   // (lanes that hold the same value write the same)
  __syncthreads();
  for (int i = threadIdx.x; i < N * WIDTH; i += FEW_THREADS) {
    const int t = i / WIDTH, e = i % WIDTH;
    const int64_t col = c0 + e;
    if (col >= a.H) continue;
    float g = 0.0f, u = 0.0f, p, r;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      g += red[w][e / VN][(t * 2) * VN + e % VN];
      u += red[w][e / VN][(t * 2 + 1) * VN + e % VN];
    }
    activation(a.act, g, p, r);
    reinterpret_cast<T*>(a.h)[t * a.ldh + col] = from_f32<T>(p * u);
    if (a.saved) {
      a.saved[t * a.H + col] = p;
      a.saved[(a.N + t) * a.H + col] = u * r;
    }
  }
}

// dz = [dh R | dh P], [N, 2H].  Bound by memory: 8192 x 5632 bf16 100 us (6.5 TB/s).  A launch of its own, because a product would form every element
// again for each of its 8 or 22 tiles along the other side.
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
    load8<Q, true>(reinterpret_cast<const T*>(a.dh) + r * a.lddh + c, cols, d);
    load8<Q, true>(a.saved + r * a.H + c, cols, p);
    load8<Q, true>(a.saved + (a.N + r) * a.H + c, cols, q);
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

// The backward products of 8192 tokens of 2048-5632: 572-600 us in one launch (1.26-1.32 PFLOP/s; matrix cores busy 77 % of the cycles).
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
  static __device__ __forceinline__ void finish(const Args& a, int tm, int tn, int wave, int i, float* st, f32x16 (&x)[1][P::TN_]) {
    const Place at = place<P>(tm, tn, wave, i, a.N, a.K);
    store_rows<T, P::TN_, VEC>(st, x[0], reinterpret_cast<T*>(a.dx) + at.m * a.lddx + at.n, a.lddx, at.rows, at.cols, threadIdx.x & 63);
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
  static __device__ __forceinline__ void finish(const Args& a, int tm, int tn, int wave, int i, float* st, f32x16 (&x)[1][P::TN_]) {
    const bool second = tn >= a.tiles_h;
    const Place at = place<P>(tm, second ? tn - a.tiles_h : tn, wave, i, a.K, a.H);
    store_rows<T, P::TN_, VEC>(st, x[0], reinterpret_cast<T*>(second ? a.dwu : a.dwg) + at.m * a.lddw + at.n, a.lddw, at.rows, at.cols, threadIdx.x & 63);
  }
};

// ------------------------------------------------------------- plans
// Which tiles a product goes by, and which of them in parts: the plan of the shortest estimated time.  The classes of tiles (`cols`: of all
// products that a tile holds side by side) and what a tile costs a compute unit: ns a contraction slot, and us for filling the pipeline
// and writing the results.
struct TileClass {
  int32_t rows, cols, slots, at_once;   // at_once: blocks that a compute unit's LDS holds
  float ns, us;
};
enum { BF16_256, BF16_128, BF16_64, F32_64, F32_64_ANY, TILE_CLASSES };
constexpr TileClass TILE_CLASS[2][TILE_CLASSES] = {
    {{256, 256, 32, 1, 27.0f, 7.0f}, {128, 128, 64, 1, 10.0f, 2.5f}, {64, 64, 64, 3, 4.6f, 1.0f}, {64, 64, 32, 3, 16.0f, 2.0f}, {64, 64, 32, 3, 25.0f, 2.0f}},
    {{256, 256, 32, 1, 27.0f, 7.0f}, {128, 128, 64, 1, 10.0f, 2.5f}, {64, 64, 64, 3, 4.6f, 1.0f}, {64, 128, 32, 2, 32.0f, 3.0f}, {64, 128, 32, 2, 50.0f, 3.0f}}};
template <typename T, int C, int NB, bool AS, bool BS>
struct TilingOf;   // Product: its TileProduct; vec: whole 16-byte groups may be written
#define TILING(C, T, TM, TN, WR, WC, BK, STAGES, PIECE)                                                                                \
  template <int NB, bool AS, bool BS>                                                                                                  \
  struct TilingOf<T, C, NB, AS, BS> {                                                                                                  \
    typedef TileProduct<T, NB, TM, TN, WR, WC, BK, STAGES, AS, BS, PIECE> Product;                                                     \
    typedef T Type;                                                                                                                    \
    static constexpr bool vec = PIECE == 16;                                                                                           \
    static constexpr TileClass k = TILE_CLASS[NB - 1][C];                                                                              \
    static_assert(Product::BM == k.rows && NB * Product::BN == k.cols && Product::SLOTS == k.slots &&                                  \
                      160 * 1024 / Product::LDS_BYTES == k.at_once, "class");                                                          \
  };
TILING(BF16_256, bf16_t, 4, 4 / NB, 2, 2, 32, 4, 16)
TILING(BF16_128, bf16_t, 2 / NB, 1, 2 * NB, 4 / NB, 64, 3, 16)
TILING(BF16_64, bf16_t, 1, 1, 2, 2 / NB, 64, 3, 16)
TILING(F32_64, float, 1, 1, 2, 2, 32, 3, 16)
TILING(F32_64_ANY, float, 1, 1, 2, 2, 32, 3, 4)
#undef TILING

constexpr int COMPUTE_UNITS = 256, MOST_PARTS = 16;
constexpr double HALF_TILE = 0.75;   // of a tile's time
constexpr double JOIN_US = 6.0, PARTIAL_BYTES_PER_US = 2e6;   // a further launch; the sums written and read again

struct Jobs {   // of one length, in the order they are handed out
  int64_t n;
  double us;
};
// When the last of the jobs ends on `places` that each take the next one when they are free.
double finish_time(int64_t places, std::initializer_list<Jobs> all) {
  // places by the time they are free: a list of (time, how many), kept in order
  constexpr int MOST = 32;
  double at[MOST];
  int64_t n[MOST];
  int k = 1;
  at[0] = 0.0;
  n[0] = places;
  double last = 0.0;
  for (Jobs j : all) {
    if (j.n > 64 * places) {   // (so many that the ends do not matter)
      const int64_t rounds = j.n / places - 1;
      for (int i = 0; i < k; ++i) at[i] += rounds * j.us;
      j.n -= rounds * places;
      last = std::max(last, at[k - 1]);
    }
    while (j.n > 0) {
      const int64_t take = std::min(j.n, n[0]);
      const double end = at[0] + j.us;
      j.n -= take;
      n[0] -= take;
      last = std::max(last, end);
      if (n[0] == 0) {
        for (int i = 1; i < k; ++i) {
          at[i - 1] = at[i];
          n[i - 1] = n[i];
        }
        --k;
      }
      int i = k;
      if (k == MOST) {   // (then the last two are taken for one)
        n[k - 1] += take;
        at[k - 1] = std::max(at[k - 1], end);
        continue;
      }
      while (i > 0 && at[i - 1] > end) {
        at[i] = at[i - 1];
        n[i] = n[i - 1];
        --i;
      }
      at[i] = end;
      n[i] = take;
      ++k;
    }
  }
  return last;
}

// The same for jobs that all find a place at once: they are dealt out in turn, and a compute unit works on its jobs together.  0 where more
// than that are waiting.
double dealt_out(int at_once, std::initializer_list<Jobs> all) {
  int64_t n = 0;
  for (const Jobs& j : all) n += j.n;
  if (at_once == 1 || n > COMPUTE_UNITS * at_once) return 0.0;
  double unit[COMPUTE_UNITS] = {}, last = 0.0;
  int64_t at = 0;
  for (const Jobs& j : all)
    for (int64_t i = 0; i < j.n; ++i) unit[at++ % COMPUTE_UNITS] += j.us;
  for (double u : unit) last = std::max(last, u);
  return last;
}

// A product that is part of a launch: rows x cols of results, `copies` of them side by side (two weights' gradients), `contraction` slots.
struct Job {
  int64_t rows, cols, copies, contraction;
};
struct Plan {
  int cls;
  Split split[2];
  size_t bytes;
  double us;
};
// NB: products that a tile holds side by side.
Plan plan_of(int cls, int NB, const Job (&job)[2]) {
  const TileClass& c = TILE_CLASS[NB - 1][cls];
  Plan best = {};
  best.cls = cls;
  int64_t tiles[2], len[2];
  for (int q = 0; q < 2; ++q) {
    Split& s = best.split[q];
    s.tiles_m = (int)div_up(job[q].rows, c.rows);
    s.tiles_n = (int)(job[q].copies * div_up(job[q].cols, c.cols / NB));
    s.whole = s.tiles_m * s.tiles_n;
    s.parts = 1;
    tiles[q] = s.whole;
    len[q] = s.len = (int)job[q].contraction;
  }
  const int64_t places = COMPUTE_UNITS, all = tiles[0] + tiles[1];
  auto end = [&](std::initializer_list<Jobs> jobs) { return std::max(finish_time(places, jobs), dealt_out(c.at_once, jobs)); };
  auto us = [&](int64_t slots) { return slots * c.ns * 1e-3 + c.us; };
  best.us = end({{tiles[0], us(len[0])}, {tiles[1], us(len[1])}});
  auto parts_of = [&](int64_t slots, int64_t want) { return std::max<int64_t>(std::min<int64_t>({want, slots / (4 * c.slots), MOST_PARTS}), 1); };
  auto offer = [&](int64_t rest0, int64_t parts0, int64_t rest1, int64_t parts1) {
    const int64_t rest[2] = {parts0 > 1 ? rest0 : 0, parts1 > 1 ? rest1 : 0}, parts[2] = {parts0, parts1};
    if (rest[0] + rest[1] == 0) return;
    Plan p = best;
    int64_t sums = 0, part_len[2];
    for (int q = 0; q < 2; ++q) {
      Split& s = p.split[q];
      s.whole = (int)(tiles[q] - rest[q]);
      s.parts = 1;
      s.halves = 0;
      part_len[q] = s.len = (int)len[q];
      if (rest[q] == 0) continue;
      part_len[q] = s.len = (int)(div_up(div_up(len[q], parts[q]), c.slots) * c.slots);
      s.parts = (int)div_up(len[q], s.len);
      sums += rest[q] * s.parts;
    }
    p.bytes = (size_t)sums * c.rows * c.cols * 4;
    p.us = end({{p.split[0].whole, us(len[0])}, {rest[0] * p.split[0].parts, us(part_len[0])}, {p.split[1].whole, us(len[1])},
                                {rest[1] * p.split[1].parts, us(part_len[1])}}) +
           JOIN_US + p.bytes / PARTIAL_BYTES_PER_US;
    if (p.us < best.us) best = p;
  };
  if (all == 0) return best;
  // the tiles behind the last whole filling of the chip
  const int64_t rest = all % places, last = tiles[1] ? 1 : 0;
  if (all > places && rest > 0 && rest <= tiles[last])
    for (int64_t p : {2, 3, 4, 6}) {
      const int64_t parts = parts_of(len[last], p);
      if (last) offer(0, 1, rest, parts);
      else offer(rest, parts, 0, 1);
    }
  // Those by halves.  Saving, in parts or whole / by halves, us: 8192 tokens of 2048-5632 (128 left over) 384 / 364, 6500 of 520-1704 (108) 55 / 45, 8192 of
  // 1024-1408 (96) 70 / 61; of few the contraction's parts cost less: 5000 of 640-2048 (64) 44 / 48, 3000 of 1024-3200 (44) 58 / 62.
  if (cls == BF16_256 && NB == 2 && rest > places / 4 && rest <= places / 2 && all > places) {
    Plan p = best;
    p.bytes = 0;
    Split& s = p.split[0];
    s.whole = (int)(all - rest);
    s.parts = 1;
    s.len = (int)len[0];
    s.halves = 1;
    const double half = HALF_TILE * us(len[0]);
    p.us = end({{rest, half}, {s.whole, us(len[0])}, {rest, half}});
    if (p.us < best.us) best = p;
  }
  // all of those that take longer than an equal share of the work
  const double each = std::max((double)(tiles[0] * len[0] + tiles[1] * len[1]) / places, 4.0 * c.slots);
  if (len[0] > each || len[1] > each)
    for (int more : {1, 2}) offer(tiles[0], parts_of(len[0], (int64_t)(more * len[0] / each)), tiles[1], parts_of(len[1], (int64_t)(more * len[1] / each)));
  return best;
}
Plan best_plan(bool bf16, bool vec, int NB, const Job (&job)[2]) {
  if (!bf16 && !vec) return plan_of(F32_64_ANY, NB, job);
  if (!bf16) return plan_of(F32_64, NB, job);
  Plan best = plan_of(BF16_256, NB, job);
  for (int c : {BF16_128, BF16_64}) {
    const Plan p = plan_of(c, NB, job);
    if (p.us < best.us) best = p;
  }
  return best;
}
// The last few plans of the calling thread, by all they depend on: making one takes microseconds.
struct PlanKey {
  int64_t N, K, H;
  int32_t what;   // operands, alignment and results
  bool operator==(const PlanKey& o) const { return N == o.N && K == o.K && H == o.H && what == o.what; }
};
template <typename F>
Plan kept_plan(const PlanKey& key, F&& make) {
  constexpr int KEPT = 32;
  static thread_local PlanKey keys[KEPT];
  static thread_local Plan plans[KEPT];
  static thread_local int next = 0;
  for (int i = 0; i < KEPT; ++i)
    if (keys[i] == key) return plans[i];
  const int at = next;
  next = (next + 1) % KEPT;
  keys[at] = key;
  plans[at] = make();
  return plans[at];
}
Plan forward_plan(int64_t N, int64_t K, int64_t H, bool bf16, bool vec) {
  return kept_plan({N, K, H, 1 | bf16 << 1 | vec << 2}, [&] { return best_plan(bf16, vec, 2, {{N, H, 1, K}, {0, 0, 1, 0}}); });
}
// dx first where its tiles take longer, else the weights' gradients
bool dx_first(int64_t N, int64_t H) { return 2 * H >= N; }
Plan backward_plan(int64_t N, int64_t K, int64_t H, bool bf16, bool vec, bool dx, bool dw) {
  return kept_plan({N, K, H, bf16 << 1 | vec << 2 | dx << 3 | dw << 4}, [&] {
    const Job x = {dx ? N : 0, K, 1, 2 * H}, w = {dw ? K : 0, H, 2, N};
    return dx_first(N, H) ? best_plan(bf16, vec, 1, {x, w}) : best_plan(bf16, vec, 1, {w, x});
  });
}
// The partial sums' bytes, whichever way the rows lie and whichever results are wanted.
size_t forward_bytes(int64_t N, int64_t K, int64_t H, bool bf16) {
  if (N == 0) return 0;
  return std::max(N <= few_tokens(bf16 ? 2 : 4) ? 0 : forward_plan(N, K, H, bf16, true).bytes, bf16 ? 0 : forward_plan(N, K, H, false, false).bytes);
}
size_t backward_partial_bytes(int64_t N, int64_t K, int64_t H, bool bf16) {
  if (N == 0) return 0;
  size_t most = 0;
  for (int vec = bf16 ? 1 : 0; vec < 2; ++vec)
    for (int want = 1; want < 4; ++want) most = std::max(most, backward_plan(N, K, H, bf16, vec, want & 1, want & 2).bytes);
  return most;
}

// ------------------------------------------------------------- launches
template <typename P>
constexpr int staging(int waves) { return waves * 32 * (32 * P::TN_ + 4) * 4; }   // of the results, in LDS

template <typename Op>
hipError_t launch_op(const typename Op::Args& a, const Split& sp, hipStream_t s) {
  typedef typename Op::P P;
  static_assert(staging<P>(P::WAVES) <= P::LDS_BYTES && staging<P>(JOIN_WAVES) <= 64 * 1024, "staging of the results");
  static std::atomic<uint64_t> allowed{0};
  hipError_t e = allow_lds(tile_kernel<Op>, P::LDS_BYTES, 0, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(tile_kernel<Op>, dim3(sp.blocks()), dim3(P::THREADS), P::LDS_BYTES, s, a, sp);
  e = hipGetLastError();
  if (e != hipSuccess || sp.parts == 1) return e;
  hipLaunchKernelGGL(join_kernel<Op>, dim3((unsigned)div_up(sp.rest() * join_units<P>(), JOIN_WAVES)), dim3(64 * JOIN_WAVES), staging<P>(JOIN_WAVES), s, a,
                     sp);
  return hipGetLastError();
}
template <typename Op, typename Half>
hipError_t launch_halves(const typename Op::Args& a, const Split& sp, hipStream_t s) {
  typedef typename Op::P P;
  static_assert(P::THREADS == Half::P::THREADS && P::BM == 2 * Half::P::BM && P::BN == Half::P::BN && P::LDS_BYTES >= Half::P::LDS_BYTES &&
                    staging<typename Half::P>(P::WAVES) <= P::LDS_BYTES, "halves of the same tiles");
  static std::atomic<uint64_t> allowed{0};
  const hipError_t e = allow_lds(halves_kernel<Op, Half>, P::LDS_BYTES, 0, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((halves_kernel<Op, Half>), dim3(sp.blocks()), dim3(P::THREADS), P::LDS_BYTES, s, a, sp);
  return hipGetLastError();
}
template <typename Op1, typename Op2>
hipError_t launch_pair(const typename Op1::Args& a1, const Split& s1, const typename Op2::Args& a2, const Split& s2, hipStream_t s) {
  typedef typename Op1::P P;
  typedef typename Op2::P P2;
  constexpr int bytes = std::max((int)P::LDS_BYTES, (int)P2::LDS_BYTES);
  static_assert(P::THREADS == P2::THREADS && staging<P>(1) == staging<P2>(1) && staging<P>(P::WAVES) <= bytes && join_units<P>() == join_units<P2>(), "one block");
  static std::atomic<uint64_t> allowed{0};
  hipError_t e = allow_lds(tile_pair_kernel<Op1, Op2>, bytes, 0, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tile_pair_kernel<Op1, Op2>), dim3(s1.blocks() + s2.blocks()), dim3(P::THREADS), bytes, s, a1, s1, a2, s2);
  e = hipGetLastError();
  const int joins = ((s1.parts > 1 ? s1.rest() : 0) + (s2.parts > 1 ? s2.rest() : 0)) * join_units<P>();
  if (e != hipSuccess || joins == 0) return e;
  hipLaunchKernelGGL((join_pair_kernel<Op1, Op2>), dim3((unsigned)div_up(joins, JOIN_WAVES)), dim3(64 * JOIN_WAVES), staging<P>(JOIN_WAVES), s, a1, s1, a2, s2);
  return hipGetLastError();
}

template <typename G, int ACT, bool SAVE>
hipError_t launch_forward(const GatedArgs& a, const Split& sp, hipStream_t s) {
  typedef typename G::Product P;
  typedef typename G::Type T;
  typedef ForwardOp<T, P, G::vec, ACT, SAVE> Op;
  if constexpr (G::k.rows == 256) {
    typedef TileProduct<T, 2, 2, 2, 2, 2, 32, 4, false, true, 16> HalfP;
    if (sp.halves) return launch_halves<Op, ForwardOp<T, HalfP, G::vec, ACT, SAVE>>(a, sp, s);
  }
  return launch_op<Op>(a, sp, s);
}
template <typename G, bool SAVE>
hipError_t launch_forward(const GatedArgs& a, const Split& sp, hipStream_t s) {
  switch (a.act) {
    case ANTDT_ACT_SILU: return launch_forward<G, ANTDT_ACT_SILU, SAVE>(a, sp, s);
    case ANTDT_ACT_GELU: return launch_forward<G, ANTDT_ACT_GELU, SAVE>(a, sp, s);
    case ANTDT_ACT_RELU: return launch_forward<G, ANTDT_ACT_RELU, SAVE>(a, sp, s);
    default: return launch_forward<G, ANTDT_ACT_SIGMOID, SAVE>(a, sp, s);
  }
}
template <typename T, int LANES>
hipError_t launch_few(const GatedArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)div_up(a.H, LANES * (16 / (int)sizeof(T))));
  if (a.N == 1) hipLaunchKernelGGL((gated_few_kernel<T, 1, LANES>), grid, dim3(FEW_THREADS), 0, s, a);
  else if (a.N == 2) hipLaunchKernelGGL((gated_few_kernel<T, 2, LANES>), grid, dim3(FEW_THREADS), 0, s, a);
  else if constexpr (few_tokens(sizeof(T)) > 2) {
    if (a.N <= 4) hipLaunchKernelGGL((gated_few_kernel<T, 4, LANES>), grid, dim3(FEW_THREADS), 0, s, a);
    else hipLaunchKernelGGL((gated_few_kernel<T, 8, LANES>), grid, dim3(FEW_THREADS), 0, s, a);
  }
  return hipGetLastError();
}
// Lanes along H: as many (128 bytes of a row; of fp32 and up to four tokens 256) as leave 150 blocks.  1 token, us: bf16, blocks of 256 threads,
// 2 / 4 / 8 lanes 1024-4096 5.5 / 5.4 / 7.3, 2048-5632 16.3 / 13.8 / 19.0; fp32 2048-5632 4 lanes 22.6, 8 18.2; of 512 threads, other weights every time,
// 8 / 16 lanes fp32 4096-14336 101 / 80 (8 tokens 103 / 118), bf16 2048-5632 4 / 8 lanes 15.5 / 17.8.
template <typename T>
hipError_t launch_few(const GatedArgs& a, hipStream_t s) {
  constexpr int VN = 16 / sizeof(T), ENOUGH = 150;
  if constexpr (sizeof(T) == 4) {
    if (a.N <= 4 && a.H / (16 * VN) >= ENOUGH) return launch_few<T, 16>(a, s);
  }
  if (a.H / (8 * VN) >= ENOUGH) return launch_few<T, 8>(a, s);
  if (a.H / (4 * VN) >= ENOUGH) return launch_few<T, 4>(a, s);
  return launch_few<T, 2>(a, s);
}
template <typename T, int C>
hipError_t launch_forward_class(const GatedArgs& a, const Split& sp, hipStream_t s) {
  typedef TilingOf<T, C, 2, false, true> G;
  return a.saved ? launch_forward<G, true>(a, sp, s) : launch_forward<G, false>(a, sp, s);
}
hipError_t gated_forward(const GatedArgs& a, bool bf16, bool vec, float* partial, hipStream_t s) {
  if (vec && a.N <= few_tokens(bf16 ? 2 : 4)) return bf16 ? launch_few<bf16_t>(a, s) : launch_few<float>(a, s);
  Plan p = forward_plan(a.N, a.K, a.H, bf16, vec);
  Split& sp = p.split[0];
  sp.partial = partial;
  switch (p.cls) {
    case BF16_256: return launch_forward_class<bf16_t, BF16_256>(a, sp, s);
    case BF16_128: return launch_forward_class<bf16_t, BF16_128>(a, sp, s);
    case BF16_64: return launch_forward_class<bf16_t, BF16_64>(a, sp, s);
    case F32_64: return launch_forward_class<float, F32_64>(a, sp, s);
    default: return launch_forward_class<float, F32_64_ANY>(a, sp, s);
  }
}
template <typename T, int C>
hipError_t launch_backward(const DxArgs& x, const DwArgs& w, const Split (&sp)[2], hipStream_t s) {
  typedef TilingOf<T, C, 1, false, false> GX;
  typedef TilingOf<T, C, 1, true, true> GW;
  typedef DxOp<T, typename GX::Product, GX::vec> OpX;
  typedef DwOp<T, typename GW::Product, GW::vec> OpW;
  if (dx_first(x.N, x.H)) return launch_pair<OpX, OpW>(x, sp[0], w, sp[1], s);
  return launch_pair<OpW, OpX>(w, sp[0], x, sp[1], s);
}
hipError_t gated_products(const DxArgs& x, DwArgs w, bool bf16, bool vec, float* partial, hipStream_t s) {
  Plan p = backward_plan(x.N, x.K, x.H, bf16, vec, x.dx != nullptr, w.dwg != nullptr);
  const TileClass& c = TILE_CLASS[0][p.cls];
  w.tiles_h = (int32_t)div_up(x.H, c.cols);
  p.split[0].partial = partial;
  p.split[1].partial = partial;
  if (p.split[0].parts > 1) p.split[1].partial += (size_t)p.split[0].rest() * p.split[0].parts * c.rows * c.cols;
  switch (p.cls) {
    case BF16_256: return launch_backward<bf16_t, BF16_256>(x, w, p.split, s);
    case BF16_128: return launch_backward<bf16_t, BF16_128>(x, w, p.split, s);
    case BF16_64: return launch_backward<bf16_t, BF16_64>(x, w, p.split, s);
    case F32_64: return launch_backward<float, F32_64>(x, w, p.split, s);
    default: return launch_backward<float, F32_64_ANY>(x, w, p.split, s);
  }
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t dz_bytes(int64_t N, int64_t H, int32_t dtype) { return align256((size_t)(N * 2 * H * op_size(dtype))); }

// Sizes below which a tile's offsets stay in 32 bits.
int gated_sizes(const char* call, int64_t N, int64_t K, int64_t H, int32_t dtype) {
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  if (N < 0 || N >= INT32_MAX - 512 || K < 1 || K >= (1 << 20) || H < 1 || H >= (1 << 20))
    return op_fail(ANTDT_INVALID_ARG, "%s: N, K or H out of range", call);
  const int64_t k = div_up(K, 64), h = div_up(H, 64);   // blocks of a launch, of 256 threads at least (2^32 threads are the most)
  const int64_t tiles = dtype == ANTDT_F32 ? std::max(k, div_up(H, 32)) : std::max(k, h);   // (of the forward pass in fp32: 64 x 32)
  if (std::max(div_up(N, 64) * tiles, 2 * k * h) >= (1 << 24)) return op_fail(ANTDT_INVALID_ARG, "%s: N, K or H out of range", call);
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
  const bool vec = dtype == ANTDT_BF16 || (whole16(x, ldx) && whole16(wg, ldw) && whole16(wu, ldw) && whole16(h, ldh) && ((K | H) & 3) == 0);
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
  if (N == 0) dx = nullptr;   // (nothing of it; the weights' gradients are zeros)
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
  const DxArgs x_args = {workspace, wg, wu, dx, ldw, lddx, N, K, H};
  const DwArgs w_args = {x, workspace, dwg, dwu, ldx, lddw, N, K, H, 0};
  const bool vec = ((K | H) & 3) == 0 && (!dx || (whole16(wg, ldw) && whole16(wu, ldw) && whole16(dx, lddx))) &&
                   (!dwg || (whole16(x, ldx) && whole16(dwg, lddw) && whole16(dwu, lddw)));
  OP_TRY(op_hip(call, gated_products(x_args, w_args, bf16, vec, partial, s)));
  return ANTDT_OK;
}

}  // extern "C"
