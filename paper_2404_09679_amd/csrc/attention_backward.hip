// Backward pass of the attention of queries over keys and values of another length (see cross.h).
#include "cross.h"

namespace antdt {
namespace {

// ------------------------------------------------------------- d
// From out as it was kept; of few keys, which fit in LDS, the sum of p dP instead (the same number): dP - d nearly vanishes there, and what out lost to
// its rounding would show (2 keys, bf16: dQ off by 0.005 of its norm, so by 0.0025, the operands' rounding).  Bound by memory: 134 MB 27 us.
template <typename T, int DP, int COLS>
struct FewKeys {
  static constexpr int KEYS = 64, STEPS = COLS / Core<T>::STEP;
  typedef HeadTile<T, DP> Tile;
  typedef TileLoad<T, DP, KEYS, 256> Load;
};
template <typename T, int DP, int COLS>
__global__ __launch_bounds__(256, 2) void cross_d_kernel(CrossArgs a) {
  typedef FewKeys<T, DP, COLS> F;
  typedef Core<T> C;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int tiles = (int)((a.S + 127) >> 7), tile = blockIdx.x % tiles;
  const int64_t bh = blockIdx.x / tiles, b = bh / a.q_heads;
  const int h = (int)(bh - b * a.q_heads);
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t r0 = (int64_t)tile * 128 + wave * 32, r = r0 + (lane & 31);
  if (k_len == 0 || (int64_t)tile * 128 >= q_len) return;
  typename C::Fragment x[F::STEPS], g[F::STEPS];
  load_rows<T, COLS>(a.dout.rows(b, h), r0, q_len, a.D, lane, g);
  float d = 0.0f;
  if (k_len > F::KEYS) {
    load_rows<T, COLS>(a.out.rows(b, h), r0, q_len, a.D, lane, x);
#pragma unroll
    for (int i = 0; i < F::STEPS; ++i)
#pragma unroll
      for (int e = 0; e < C::PER; ++e) d = fmaf((float)x[i][e], (float)g[i][e], d);
  } else {
    if (a.D < COLS) {
      clear_lds(lds, 2 * F::Load::BYTES, 256);
      __syncthreads();
    }
    const typename F::Load load(threadIdx.x, a.D);
    const uint32_t tile0 = lds_address(lds);
    load(a.k.rows(b, h / a.group), 0, k_len, tile0 + wave * 1024);
    load(a.v.rows(b, h / a.group), 0, k_len, tile0 + F::Load::BYTES + wave * 1024);
    load_rows<T, COLS>(a.q.rows(b, h), r0, q_len, a.D, lane, x);
    const float sum = r < q_len ? a.stats[bh * a.S + r] : INFINITY;
    arrive<0, true>();
    const uint32_t tk = F::Tile::along_at(tile0, lane), tv = F::Tile::along_at(tile0 + F::Load::BYTES, lane);
    for (int j = 0; j < F::KEYS / 32; ++j) {
      f32x16 s = zeros(), dp = zeros();
#pragma unroll
      for (int i = 0; i < F::STEPS; ++i) {
        C::multiply(F::Tile::along(tk, 32 * j, i), x[i], s);
        C::multiply(F::Tile::along(tv, 32 * j, i), g[i], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (32 * j + 8 * (e >> 2) + 4 * half + (e & 3) < k_len) d = fmaf(exp2_(fmaf(s[e], a.scale2, -sum)), dp[e], d);
    }
  }
  d = sum_of_halves(d);
  if (r < q_len && lane < 32) a.delta[bh * a.S + r] = d;
}

// ------------------------------------------------------------- gradient of the queries
// As the forward pass; a lane has the sums L and d of its row.
template <typename W>
__device__ __forceinline__ void dq_block(const CrossArgs& a, int index, char* lds) {
  typedef typename W::T T;
  typedef typename W::Tile Tile;
  typedef Core<T> C;
  typedef KeyTiles<W> F;
  constexpr int BT = W::TILE;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  if (wave >= W::WAVES) return;
  const Share& share = a.queries;
  int unit, block;
  place_of(a, index, a.group * share.tiles * share.parts, unit, block);
  const int part = block % share.parts, tile = block / share.parts % share.tiles, h = unit % a.heads * a.group + block / share.parts / share.tiles;
  const Entry of = entry_of(a, unit / a.heads, lane);
  const int64_t b = of.b, bh = b * a.q_heads + h, q_len = of.q_len, k_len = of.k_len;
  const int64_t first = (int64_t)tile * W::ROWS, last = min(first + W::ROWS, a.S), r0 = first + (W::SPLIT ? 0 : wave * 32);
  const int64_t end = k_len > 0 ? min(max(q_len, first), last) : first;
  const Rows dq = a.dq.rows(b, h);
  if (part == 0) clear_rows<T>(dq, end, last, a.D, W::THREADS);
  if (end == first) return;
  typename C::Fragment q[W::STEPS], g[W::STEPS];
  load_rows<T, W::COLS>(a.q.rows(b, h), r0, q_len, a.D, lane, q);
  load_rows<T, W::COLS>(a.dout.rows(b, h), r0, q_len, a.D, lane, g);
  const int64_t r = r0 + (lane & 31);
  const float sum = r < end ? a.stats[bh * a.S + r] : INFINITY, delta = r < end ? a.delta[bh * a.S + r] : 0.0f;
  if (a.D < W::COLS) {
    clear_lds(lds, F::ALL, W::THREADS);
    __syncthreads();
  }
  const typename W::Load load(W::SPLIT ? lane : threadIdx.x, a.D);
  const Rows k = a.k.rows(b, h / a.group), v = a.v.rows(b, h / a.group);
  const uint32_t ring0 = lds_address(lds) + (W::SPLIT ? wave * F::RING : 0), lds0 = ring0 + (W::SPLIT ? 0 : wave * 1024);
  // the part's tiles, and the wavefront's of them
  const int64_t tiles = (k_len + BT - 1) / BT, behind = share.parts == 1 ? tiles : tiles * (part + 1) / share.parts;
  constexpr int STEP = W::SPLIT ? W::WAVES : 1;
  const int64_t i0 = (share.parts == 1 ? 0 : tiles * part / share.parts) + (W::SPLIT ? wave : 0);
  int64_t asked = i0 * BT;
  auto issue = [&](uint32_t to) {
    load(k, asked, k_len, lds0 + to);
    load(v, asked, k_len, lds0 + to + W::Load::BYTES);
    asked += STEP * BT;
  };
  Sums<W> o;
  clear_sums<W>(o);
  typename F::Ring ring((behind - i0 + STEP - 1) / STEP);
  ring.start(issue);
  for (int64_t t = i0 * BT; t < behind * BT; t += STEP * BT, ring.done()) {
    ring.next(issue);
    const uint32_t tile0 = ring0 + ring.read;
    const uint32_t tk = Tile::along_at(tile0, lane), tv = Tile::along_at(tile0 + W::Load::BYTES, lane), kt = Tile::down_at(tile0, lane);
#pragma unroll
    for (int j = 0; j < BT / 32; ++j) {
      f32x16 s = zeros(), dp = zeros();   // scores, then p, then dZ of keys 32 j .. of the tile; dP
      auto row = [&](int i) { return Tile::along(i < W::STEPS ? tk : tv, 32 * j, i % W::STEPS); };
      Fragments<typename C::Fragment, 2 * W::STEPS, W::AHEAD> rows;
      rows.start(row);
      rows.run(row, [&](int i, const typename C::Fragment& x) {
        if (i < W::STEPS) C::multiply(x, q[i], s);
        else C::multiply(x, g[i % W::STEPS], dp);
      });
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = exp2_(fmaf(s[e], a.scale2, -sum));
      if (t + BT > k_len) {
        const int left = (int)(k_len - t) - 32 * j - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[e] = where_left(8 * (e >> 2) + (e & 3), left, s[e], 0.0f);
          dp[e] = where_left(8 * (e >> 2) + (e & 3), left, dp[e], 0.0f);
        }
      }
      auto column = [&](int i) { return Tile::down(kt, 32 * j, i / W::DT, i % W::DT); };
      Fragments<typename C::Fragment, W::PACKS * W::DT, W::AHEAD> columns;
      columns.start(column);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= dp[e] - delta;
      typename C::Fragment ds;
      columns.run(column, [&](int i, const typename C::Fragment& x) {
        if (i % W::DT == 0) ds = C::pack(s, i / W::DT);
        C::multiply(x, ds, o[i % W::DT]);
      });
    }
  }
  arrive<0, true>();
  float* sums = share.parts == 1 ? nullptr : share.partial + ((int64_t)part * a.units * a.group + bh) * a.S * a.D;
  write_result<W>(lds, o, a.scale, dq, sums, r0, end, a.D, wave, lane);
}


// ------------------------------------------------------------- gradients of keys and values
// A block has keys of a head, 32 to a wavefront, and goes through tiles of queries and their outputs' gradients, of every head that shares the keys.
// HELD: the values' fragments are held in registers, else (where registers would be spilled, and reloaded behind the tiles' loads) in LDS.
template <typename W, bool HELD>
struct QueryTiles {
  static constexpr int STATS = 2 * W::TILE * 4;   // L and d of the rows, for each wavefront: (L, d) of 32 rows behind each other
  typedef TileLoad<typename W::T, W::DP, W::ROWS, W::THREADS> Values;
  static constexpr int STAGE = 2 * W::Load::BYTES + (W::SPLIT ? (STATS + 1023) / 1024 * 1024 : W::WAVES * STATS);
  static constexpr int RING = W::STAGES * STAGE, ALL = W::SPLIT ? W::WAVES * RING : RING, CLEARED = ALL + (HELD ? 0 : W::ROWS * W::Tile::ROW), LDS = W::lds(CLEARED);
  static_assert(STAGE % 1024 == 0, "tiles start at multiples of a row");
  typedef antdt::Ring<W::STAGES, 2 * W::Load::PIECES + W::TILE / 32, STAGE, !W::SPLIT> Ring;
};
template <typename W, bool HELD>
__device__ __forceinline__ void dkv_block(const CrossArgs& a, int index, char* lds) {
  typedef typename W::T T;
  typedef typename W::Tile Tile;
  typedef Core<T> C;
  typedef QueryTiles<W, HELD> F;
  constexpr int BR = W::TILE;
  static_assert(HELD || !W::SPLIT, "values in LDS are the block's");
  constexpr int UNROLL = W::DP <= 64 ? 2 : 1;   // (of wider heads there are no registers for two)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  if (wave >= W::WAVES) return;
  const Share& share = a.keys;
  int unit, block;
  place_of(a, index, share.tiles * share.parts, unit, block);
  const int part = block % share.parts, tile = block / share.parts, h = unit % a.heads;
  const Entry of = entry_of(a, unit / a.heads, lane);
  const int64_t b = of.b, q_len = of.q_len, k_len = of.k_len;
  const int64_t first = (int64_t)tile * W::ROWS, last = min(first + W::ROWS, a.T), t0 = first + (W::SPLIT ? 0 : wave * 32);
  const int64_t end = q_len > 0 ? min(max(k_len, first), last) : first;
  const Rows dk = a.dk.rows(b, h), dv = a.dv.rows(b, h);
  if (part == 0) {
    clear_rows<T>(dk, end, last, a.D, W::THREADS);
    clear_rows<T>(dv, end, last, a.D, W::THREADS);
  }
  if (end == first) return;
  if (a.D < W::COLS) {
    clear_lds(lds, F::CLEARED, W::THREADS);
    __syncthreads();
  }
  const typename W::Load load(W::SPLIT ? lane : threadIdx.x, a.D);
  const uint32_t ring0 = lds_address(lds) + (W::SPLIT ? wave * F::RING : 0), lds0 = ring0 + (W::SPLIT ? 0 : wave * 1024);
  const uint32_t stats0 = 2 * W::Load::BYTES + (W::SPLIT ? 0 : wave * F::STATS);
  // Tiles of queries: those of a head, head by head; the part's, and the wavefront's of them.
  const int64_t per_head = (q_len + BR - 1) / BR, tiles = per_head * a.group, behind = share.parts == 1 ? tiles : tiles * (part + 1) / share.parts;
  constexpr int STEP = W::SPLIT ? W::WAVES : 1;
  const int64_t i0 = (share.parts == 1 ? 0 : tiles * part / share.parts) + (W::SPLIT ? wave : 0);
  struct At {
    int64_t g, r;
  };
  auto step = [&](At& x) {
    x.r += STEP * BR;
    while (x.r >= per_head * BR) {
      x.r -= per_head * BR;
      ++x.g;
    }
  };
  At now = {i0 / per_head, 0};
  now.r = (i0 - now.g * per_head) * BR;
  At asked = now;
  const float* const sums_of = half ? a.delta : a.stats;
  auto issue = [&](uint32_t to) {
    const int64_t hq = (int64_t)h * a.group + asked.g;
    load(a.q.rows(b, hq), asked.r, q_len, lds0 + to);
    load(a.dout.rows(b, hq), asked.r, q_len, lds0 + to + W::Load::BYTES);
#pragma unroll
    for (int j = 0; j < BR / 32; ++j)
      load_lds4(sums_of + (b * a.q_heads + hq) * a.S + min(asked.r + 32 * j + (lane & 31), q_len - 1), ring0 + to + stats0 + j * 256);
    step(asked);
  };
  typename C::Fragment k[W::STEPS], v[HELD ? W::STEPS : 1];
  load_rows<T, W::COLS>(a.k.rows(b, h), t0, k_len, a.D, lane, k);
  if constexpr (HELD) load_rows<T, W::COLS>(a.v.rows(b, h), t0, k_len, a.D, lane, v);
  Sums<W> ok, ov;
  clear_sums<W>(ok);
  clear_sums<W>(ov);
  if constexpr (!HELD) {
    const typename F::Values values(threadIdx.x, a.D);
    values(a.v.rows(b, h), first, k_len, lds_address(lds) + F::ALL + wave * 1024);
  }
  typename F::Ring ring((behind - i0 + STEP - 1) / STEP);
  ring.start(issue);
  for (int64_t i = i0; i < behind; i += STEP, ring.done(), step(now)) {
    ring.next(issue);
    const uint32_t tile0 = ring0 + ring.read;
    const float* sums = reinterpret_cast<const float*>(lds + (W::SPLIT ? wave * F::RING : 0) + ring.read + stats0);
    const uint32_t tq = Tile::along_at(tile0, lane), tg = Tile::along_at(tile0 + W::Load::BYTES, lane);
    const uint32_t vt = HELD ? 0 : Tile::along_at(lds_address(lds) + F::ALL + wave * (32 * Tile::ROW), lane);
    const uint32_t qt = Tile::down_at(tile0, lane), gt = Tile::down_at(tile0 + W::Load::BYTES, lane);
#pragma unroll UNROLL
    for (int j = 0; j < BR / 32; ++j) {
      f32x16 s = zeros(), dp = zeros();
      auto row = [&](int i) { return Tile::along(i < W::STEPS ? tq : tg, 32 * j, i % W::STEPS); };
      Fragments<typename C::Fragment, 2 * W::STEPS, W::AHEAD> rows;
      rows.start(row);
      rows.run(row, [&](int i, const typename C::Fragment& x) {
        if (i < W::STEPS) {
          C::multiply(x, k[i], s);
        } else {
          if constexpr (HELD) C::multiply(x, v[i % W::STEPS], dp);
          else C::multiply(x, Tile::along(vt, 0, i % W::STEPS), dp);
        }
      });
      auto column = [&](int i) { return Tile::down(i & 1 ? qt : gt, 32 * j, i / (2 * W::DT), i / 2 % W::DT); };
      Fragments<typename C::Fragment, 2 * W::PACKS * W::DT, W::AHEAD> columns;
      columns.start(column);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4v sum = *reinterpret_cast<const f32x4v*>(sums + 64 * j + 8 * v + 4 * half), d = *reinterpret_cast<const f32x4v*>(sums + 64 * j + 32 + 8 * v + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[4 * v + e] = exp2_(fmaf(s[4 * v + e], a.scale2, -sum[e]));
          dp[4 * v + e] = s[4 * v + e] * (dp[4 * v + e] - d[e]);
        }
      }
      if (now.r + BR > q_len) {
        const int left = (int)(q_len - now.r) - 32 * j - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[e] = where_left(8 * (e >> 2) + (e & 3), left, s[e], 0.0f);
          dp[e] = where_left(8 * (e >> 2) + (e & 3), left, dp[e], 0.0f);
        }
      }
      typename C::Fragment p, ds;
      columns.run(column, [&](int i, const typename C::Fragment& x) {
        if (i % (2 * W::DT) == 0) {
          p = C::pack(s, i / (2 * W::DT));
          ds = C::pack(dp, i / (2 * W::DT));
        }
        if (i & 1) C::multiply(x, ds, ok[i / 2 % W::DT]);
        else C::multiply(x, p, ov[i / 2 % W::DT]);
      });
    }
  }
  arrive<0, true>();
  const int64_t all = (int64_t)a.units * a.T * a.D;
  float* sums = share.parts == 1 ? nullptr : share.partial + 2 * part * all + (b * a.heads + h) * a.T * a.D;
  write_result<W>(lds, ok, a.scale, dk, sums, t0, end, a.D, wave, lane);
  write_result<W>(lds, ov, 1.0f, dv, sums ? sums + all : nullptr, t0, end, a.D, wave, lane);
}

// Both in one launch: blocks of keys first, which take longer, so that blocks of queries fill the chip while the last of them run (8 ragged histories of
// 2048 queries and 4096 keys, 16 and 4 heads of 128 bf16 columns: 640 + 980 us in two launches, 1460 so; 13 of 77 and 777, 6 and 2 heads of 64: 13 + 16,
// so 18; with what was saved since 1260-1320 and 16.5).  Wavefronts behind a kind's own leave at once.
// Bound by the matrix cores, whose operands LDS and the vector units have to keep up with: 14 products of 18 that the large case computes in all run at
// 1010-1060 TFLOP/s there (a library product of 8192 cubed: 1131).
template <typename WQ, typename WK, bool HELD>
__global__ __launch_bounds__(256, (WQ::PER_CU < WK::PER_CU ? WQ::PER_CU : WK::PER_CU)) void cross_backward_kernel(CrossArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int keys = (a.keys.blocks + 7) & ~7;   // (so that blocks of queries, too, start with the first XCD)
  if ((int)blockIdx.x < keys) {
    if ((int)blockIdx.x < a.keys.blocks) dkv_block<WK, HELD>(a, blockIdx.x, lds);
  } else {
    dq_block<WQ>(a, blockIdx.x - keys, lds);
  }
}

// The parts' sums, in their order: partial [parts, n, L, D] to the heads of `to` that the lengths leave, four columns to a thread.
struct JoinArgs {
  HeadsArg to[2];
  const float* partial;
  const int32_t* lengths;     // of `to`'s rows, and of the others
  const int32_t* others;
  int64_t L, other, quads;    // quads: of columns, over all heads
  int32_t heads, D, parts, results;
};
template <typename T>
__global__ __launch_bounds__(256) void cross_join_kernel(JoinArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.quads) return;
  const int per = a.D >> 2, c = (int)(i % per) * 4, which = blockIdx.y;
  const int64_t row = i / per, bh = row / a.L, r = row - bh * a.L, b = bh / a.heads;
  if (r >= length_of(a.lengths, b, a.L) || length_of(a.others, b, a.other) == 0) return;   // (zeros already)
  float x[4] = {};
  for (int p = 0; p < a.parts; ++p) {
    const float4 y = *reinterpret_cast<const float4*>(a.partial + (((int64_t)p * a.results + which) * a.quads + i) * 4);
    x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
  }
  const HeadsArg& to = which ? a.to[1] : a.to[0];
  T* p = reinterpret_cast<T*>(const_cast<char*>(to.rows(b, bh - b * a.heads).p + r * to.s.l)) + c;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  else *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]));
}

template <typename T, int DP, int COLS>
hipError_t launch_d(const CrossArgs& a, int64_t blocks, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int LDS = 2 * FewKeys<T, DP, COLS>::Load::BYTES;
  const hipError_t e = allow_lds(cross_d_kernel<T, DP, COLS>, LDS, 0, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((cross_d_kernel<T, DP, COLS>), dim3((unsigned)blocks), dim3(256), LDS, s, a);
  return hipGetLastError();
}
template <typename WQ, typename WK, bool HELD>
hipError_t launch_backward(CrossArgs a, const Shape& z, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int LDS = KeyTiles<WQ>::LDS > QueryTiles<WK, HELD>::LDS ? KeyTiles<WQ>::LDS : QueryTiles<WK, HELD>::LDS;
  const hipError_t e = allow_lds(cross_backward_kernel<WQ, WK, HELD>, LDS, 0, allowed);
  if (e != hipSuccess) return e;
  a.longest_first = longest_first(z, a.k_lengths || a.q_lengths, a.keys.blocks + a.queries.blocks, 256 * std::min(WQ::PER_CU, WK::PER_CU));
  const auto go = [&](const CrossArgs& x, int64_t blocks) { hipLaunchKernelGGL((cross_backward_kernel<WQ, WK, HELD>), dim3((unsigned)blocks), dim3(256), LDS, s, x); };
  const int64_t both = div_up(a.keys.blocks, 8) * 8 + a.queries.blocks;
  if (both < 1 << 24) {
    go(a, both);
  } else {   // (2^32 threads are the most; each kind's blocks are fewer than 2^24)
    CrossArgs keys = a, queries = a;
    keys.queries.blocks = queries.keys.blocks = 0;
    if (a.keys.blocks) go(keys, a.keys.blocks);
    if (a.queries.blocks) go(queries, a.queries.blocks);
  }
  return hipGetLastError();
}
// Floats of the parts' sums.
int64_t dq_partial(const Shape& z) { return dq_plan(z).parts > 1 ? dq_plan(z).parts * z.B * z.q_heads * z.S * z.D : 0; }
int64_t dkv_partial(const Shape& z) { return dkv_plan(z).parts > 1 ? 2 * dkv_plan(z).parts * z.B * z.heads * z.T * z.D : 0; }

}  // namespace
}  // namespace antdt

using namespace antdt;

extern "C" {

int antdt_cross_attention_backward_bytes(int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_cross_attention_backward_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  const Shape z = {B, S, T, q_heads, heads, D, dtype};
  OP_TRY(cross_sizes(call, z));
  *bytes = (size_t)(delta_bytes(z) + 4 * (dq_partial(z) + dkv_partial(z)));
  return ANTDT_OK;
}

int antdt_cross_attention_backward(const void* dout, int64_t lddo_batch, int64_t lddo, int64_t lddo_head, const void* q, int64_t ldq_batch, int64_t ldq,
                                   int64_t ldq_head, const void* k, int64_t ldk_batch, int64_t ldk, int64_t ldk_head, const void* v, int64_t ldv_batch,
                                   int64_t ldv, int64_t ldv_head, const void* out, int64_t ldo_batch, int64_t ldo, int64_t ldo_head, const float* stats,
                                   int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, const int32_t* q_lengths,
                                   const int32_t* k_lengths, float scale, void* dq, int64_t lddq_batch, int64_t lddq, int64_t lddq_head, void* dk,
                                   int64_t lddk_batch, int64_t lddk, int64_t lddk_head, void* dv, int64_t lddv_batch, int64_t lddv, int64_t lddv_head,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "antdt_cross_attention_backward";
  CrossArgs a = {};
  const Shape z = {B, S, T, q_heads, heads, D, dtype};
  OP_TRY(cross_sizes(call, z));
  OP_TRY(op_scale(call, scale));
  a.scale = scale; a.scale2 = scale * LOG2E;
  OP_TRY(op_wide_heads(call, "dout", dout, B, S, q_heads, D, dtype, {lddo_batch, lddo, lddo_head}, false, a.dout));
  OP_TRY(op_wide_heads(call, "q", q, B, S, q_heads, D, dtype, {ldq_batch, ldq, ldq_head}, false, a.q));
  OP_TRY(op_wide_heads(call, "k", k, B, T, heads, D, dtype, {ldk_batch, ldk, ldk_head}, false, a.k));
  OP_TRY(op_wide_heads(call, "v", v, B, T, heads, D, dtype, {ldv_batch, ldv, ldv_head}, false, a.v));
  OP_TRY(op_wide_heads(call, "out", out, B, S, q_heads, D, dtype, {ldo_batch, ldo, ldo_head}, false, a.out));
  if (dq) OP_TRY(op_wide_heads(call, "dq", dq, B, S, q_heads, D, dtype, {lddq_batch, lddq, lddq_head}, true, a.dq));
  if (dk || dv) {
    OP_TRY(op_wide_heads(call, "dk", dk, B, T, heads, D, dtype, {lddk_batch, lddk, lddk_head}, true, a.dk));
    OP_TRY(op_wide_heads(call, "dv", dv, B, T, heads, D, dtype, {lddv_batch, lddv, lddv_head}, true, a.dv));
  }
  OP_TRY(cross_lengths(call, q_lengths, k_lengths));
  OP_TRY(op_matrix(call, "stats", stats, B * q_heads, S, S, 4));
  size_t need;
  OP_TRY(antdt_cross_attention_backward_bytes(B, S, T, q_heads, heads, D, dtype, &need));
  const bool keys = dk && B > 0 && T > 0, queries = B > 0 && S > 0 && (dq || keys);
  if (!keys && !queries) return ANTDT_OK;
  OP_TRY(op_workspace(call, workspace, workspace_bytes, need));
  a.q_lengths = q_lengths; a.k_lengths = k_lengths; a.stats = const_cast<float*>(stats); a.delta = reinterpret_cast<float*>(workspace); a.S = S; a.T = T;
  a.q_heads = (int)q_heads; a.heads = (int)heads; a.group = (int)(q_heads / heads); a.D = (int)D; a.units = (int)(B * heads); a.B = (int)B;
  const hipStream_t s = (hipStream_t)stream;
  float* partial = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + delta_bytes(z));
  const Plan of_q = dq_plan(z), of_k = dkv_plan(z);
  const bool has_dq = dq && S > 0;
  if (has_dq) a.queries = of_q.share(partial);
  if (keys) a.keys = of_k.share(partial + dq_partial(z));
  OP_TRY(op_hip(call, by_columns(dtype, (int)D, [&](auto way, auto cols) {
    typedef decltype(way) Z;
    constexpr int COLS = decltype(cols)::value;
    typedef typename Z::template SplitKeys<COLS> SQ;
    typedef typename Z::template KeysDq<COLS> Q;
    typedef typename Z::template SplitQueries<COLS> SK;
    typedef typename Z::template Queries<COLS> K;
    if (S > 0 && T > 0) {
      const hipError_t e = launch_d<typename Q::T, Q::DP, COLS>(a, B * q_heads * div_up(S, 128), s);
      if (e != hipSuccess) return e;
    }
    if (of_q.split) return of_k.split ? launch_backward<SQ, SK, true>(a, z, s) : launch_backward<SQ, K, Z::HELD>(a, z, s);
    return of_k.split ? launch_backward<Q, SK, true>(a, z, s) : launch_backward<Q, K, Z::HELD>(a, z, s);
  })));
  // The parts' sums to the results.
  auto join = [&](const Share& sh, const HeadsArg& x, const HeadsArg& y, int results, int64_t H, int64_t L, int64_t other, const int32_t* lengths, const int32_t* others) {
    JoinArgs j = {{x, y}, sh.partial, lengths, others, L, other, B * H * L * D / 4, (int32_t)H, (int32_t)D, sh.parts, results};
    const dim3 grid((unsigned)div_up(j.quads, 256), results);
    if (dtype == ANTDT_F32) hipLaunchKernelGGL(cross_join_kernel<float>, grid, dim3(256), 0, s, j);
    else hipLaunchKernelGGL(cross_join_kernel<bf16_t>, grid, dim3(256), 0, s, j);
    return hipGetLastError();
  };
  if (a.queries.parts > 1) OP_TRY(op_hip(call, join(a.queries, a.dq, a.dq, 1, q_heads, S, T, q_lengths, k_lengths)));
  if (a.keys.parts > 1) OP_TRY(op_hip(call, join(a.keys, a.dk, a.dv, 2, heads, T, S, k_lengths, q_lengths)));
  return ANTDT_OK;
}

}  // extern "C"
