// Attention of queries over keys and values of another length, and its backward pass.
//
// With scores z = scale q k^T over the keys that there are, p = softmax(z), out = p v.  Forward: one pass over the keys with the running maximum m and
// sum l of a row's softmax; a sum of values under an older maximum is scaled by 2^(old - new).  Kept for the backward pass: L = log2 of the sum of
// 2^(z log2 e), so that p = 2^(z log2 e - L) again.  With g the gradient of out and d = sum of g out over a row's columns:
//   dP = g v^T,  dZ = p (dP - d),  dQ = scale dZ k,  dK = scale dZ^T q,  dV = p^T g,
// dQ in blocks of queries and dK, dV in blocks of keys: each forms p and dP anew (14 products for the 10 there are), and every sum has one order.
// Of bf16 heads p and dZ are rounded to bf16 as the matrix cores' operands.
#include "attend.h"

namespace antdt {
namespace {

struct CrossArgs {
  HeadsArg q, k, v, out, dout, dq, dk, dv;
  const int32_t* q_lengths;
  const int32_t* k_lengths;
  float* stats;        // L [B, q_heads, S], +infinity for a row without keys: its p come out 0
  float* delta;        // d, the same shape
  int64_t S, T;
  int32_t q_heads, heads, group, D;
  int32_t tiles, units;   // of a head; heads of all batch entries' keys
  int32_t parts;       // blocks that share a result's sums, through:
  float* partial;      // [parts, heads, rows, D], of keys and values [parts, 2, ...]
  float scale, scale2;   // scale2: scale log2 e
};

// Own loads but the last N have arrived and own reads of LDS are done; BLOCK: then everybody's.
template <int N, bool BLOCK>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
  if (BLOCK) block_barrier();
}
// Tiles through a ring of STAGES buffers in LDS, LOADS of a wavefront each: while one is worked on, the next STAGES - 1 are under way.  The ring is the
// block's, or (not BLOCK) a wavefront's own.
template <int STAGES, int LOADS, int BYTES, bool BLOCK>
struct Ring {
  uint32_t fill = 0, read = 0;   // bytes from the ring's start: the next buffer to fill, the one to read
  int64_t left;                  // tiles not asked for yet
  int32_t behind = 0;            // tiles asked for and not worked on
  __device__ __forceinline__ explicit Ring(int64_t tiles) : left(tiles) {}
  template <typename F>
  __device__ __forceinline__ void ask(F issue) {
    if (left <= 0) return;
    issue(fill);
    fill = fill == (STAGES - 1) * BYTES ? 0 : fill + BYTES;
    --left;
    ++behind;
  }
  template <typename F>
  __device__ __forceinline__ void start(F issue) {
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) ask(issue);
  }
  // The next tile is in LDS, and the buffer of the one before is asked for again.
  template <typename F>
  __device__ __forceinline__ void next(F issue) {
    if (behind == STAGES - 1) arrive<(STAGES - 2) * LOADS, BLOCK>();
    else arrive<0, BLOCK>();
    --behind;
    ask(issue);
  }
  __device__ __forceinline__ void done() { read = read == (STAGES - 1) * BYTES ? 0 : read + BYTES; }
};

// x where there are more than `row` rows left, else `other`.  Said to be unforeseeable, lest the choices are made for every tile and not for the last.
__device__ __forceinline__ float where_left(int row, int left, float x, float other) {
  x = row < left ? x : other;
  asm volatile("" : "+v"(x));
  return x;
}
// Block i of `units` x n: which unit, and which of its blocks.  Blocks of a unit (a head of one batch entry's keys, and who reads it) share an XCD (block
// i runs on XCD i mod 8), whose L2 then has the rows they all read; neighbouring units are on different ones, so that a batch entry of long
// sequences is everybody's work.  What is left of less than 8 units is spread over all.
__device__ __forceinline__ void place_of(int i, int units, int n, int& unit, int& block) {
  const int whole = (units & ~7) * n;
  const int x = i < whole ? i & 7 : 0, j = i < whole ? i >> 3 : i - whole;
  const int u = j / n;
  block = j - u * n;
  unit = i < whole ? 8 * u + x : (units & ~7) + u;
}

// How a kernel goes about its work.  DP columns of a row in LDS, the first COLS of which take part; TILE rows to a stage of the ring, STAGES of them.
// A block's wavefronts have 32 rows of results each and share the tiles; SPLIT: they share 32 rows, every one has a part of the tiles, in a ring of its
// own, and their sums are added up at the end (four times the blocks, each a quarter as long).
template <typename T_, int DP_, int COLS_, int TILE_, int STAGES_, int WAVES_, bool SPLIT_, int PER_CU_, int AHEAD_>
struct Way {
  typedef T_ T;
  static constexpr int DP = DP_, COLS = COLS_, TILE = TILE_, STAGES = STAGES_, WAVES = WAVES_, PER_CU = PER_CU_, THREADS = 64 * WAVES;
  static constexpr bool SPLIT = SPLIT_;
  static constexpr int ROWS = SPLIT ? 32 : 32 * WAVES;       // of a block
  static constexpr int STEPS = COLS / Core<T>::STEP, DT = COLS / 32, PACKS = 32 / Core<T>::STEP;
  static constexpr int AHEAD = AHEAD_;
  typedef HeadTile<T, DP> Tile;
  typedef TileLoad<T, DP, TILE, SPLIT ? 64 : THREADS> Load;
  // Sums on their way to memory: a wavefront's, some columns at a time, or all of the block's
  static constexpr int TN = COLS % 64 ? 1 : 2, STAGING = 32 * (32 * TN + 4) * 4;
  static constexpr int PITCH = COLS + 4, MERGE = SPLIT ? WAVES * 32 * (PITCH + 2) * 4 : WAVES * STAGING;
  static constexpr int lds(int ring) { return ring > MERGE ? ring : MERGE; }
};
// A lane's row and columns of 32 x COLS sums: row lane % 32, columns 32 d + 8 (e / 4) + 4 (lane / 32) + e % 4.
template <typename W>
using Sums = f32x16[W::DT];

template <typename W>
__device__ __forceinline__ void clear_sums(Sums<W>& x) {
#pragma unroll
  for (int d = 0; d < W::DT; ++d) x[d] = zeros();
}
// f x, rows r0 .. of `to` that lie before `end`.  (A wavefront's own rows.)
template <typename W, typename TO>
__device__ __forceinline__ void write_rows(char* staging, const Sums<W>& x, float f, const Rows& to, int64_t r0, int64_t end, int D, int lane) {
  const int left = (int)max(min(end - r0, (int64_t)32), (int64_t)0);
  TO* p = reinterpret_cast<TO*>(const_cast<char*>(to.p + r0 * to.ld));
#pragma unroll
  for (int i = 0; i < W::DT; i += W::TN) {
    f32x16 y[W::TN];
#pragma unroll
    for (int j = 0; j < W::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) y[j][e] = x[i + j][e] * f;
    store_rows<TO, W::TN, true>(reinterpret_cast<float*>(staging), y, p + 32 * i, to.ld / (int64_t)sizeof(TO), left, D - 32 * i, lane);
  }
}
// The wavefronts' sums of the same 32 rows to LDS, with a maximum and a sum of each row; then, wavefront by wavefront, added up with factors f(w).
template <typename W>
__device__ __forceinline__ void put_sums(float* lds, const Sums<W>& x, float m, float l, int wave, int lane) {
  float* to = lds + (wave * 32 + (lane & 31)) * W::PITCH + 4 * (lane >> 5);
#pragma unroll
  for (int d = 0; d < W::DT; ++d)
#pragma unroll
    for (int v = 0; v < 4; ++v) *reinterpret_cast<float4*>(to + 32 * d + 8 * v) = make_float4(x[d][4 * v], x[d][4 * v + 1], x[d][4 * v + 2], x[d][4 * v + 3]);
  if (lane < 32) *reinterpret_cast<float2*>(lds + W::WAVES * 32 * W::PITCH + (wave * 32 + lane) * 2) = make_float2(m, l);
}
template <typename W, typename TO>
__device__ __forceinline__ void write_merged(const float* lds, const float (&f)[W::WAVES], const Rows& to, int64_t r0, int64_t end, int D) {
  constexpr int LANES = W::THREADS / 32;   // of a row
  const int row = threadIdx.x / LANES;
  if (r0 + row >= end) return;
  TO* p = reinterpret_cast<TO*>(const_cast<char*>(to.p + (r0 + row) * to.ld));
  for (int c = threadIdx.x % LANES * 4; c < D; c += LANES * 4) {
    float x[4] = {};
#pragma unroll
    for (int w = 0; w < W::WAVES; ++w) {
      const float4 y = *reinterpret_cast<const float4*>(lds + (w * 32 + row) * W::PITCH + c);
      x[0] = fmaf(y.x, f[w], x[0]); x[1] = fmaf(y.y, f[w], x[1]); x[2] = fmaf(y.z, f[w], x[2]); x[3] = fmaf(y.w, f[w], x[3]);
    }
    if constexpr (sizeof(TO) == 4) *reinterpret_cast<float4*>(p + c) = make_float4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<uint2*>(p + c) = make_uint2(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]));
  }
}
// Zeros to rows [r0, r1) of a head, by the block.
template <typename T>
__device__ __forceinline__ void clear_rows(const Rows& to, int64_t r0, int64_t r1, int D) {
  const int per = D / Core<T>::PER;
  for (int64_t i = threadIdx.x; i < (r1 - r0) * per; i += blockDim.x)
    store16<false>(const_cast<char*>(to.p + (r0 + i / per) * to.ld + i % per * 16), make_uint4(0, 0, 0, 0));
}
// Sums to their results, or to a part's sums in the workspace.
template <typename W>
__device__ __forceinline__ void write_result(char* lds, const Sums<W>& x, float f, const Rows& to, float* part, int64_t r0, int64_t end, int D, int wave, int lane) {
  const Rows parts = {reinterpret_cast<const char*>(part), (int64_t)D * 4};
  if constexpr (W::SPLIT) {
    float* sums = reinterpret_cast<float*>(lds);
    put_sums<W>(sums, x, 0.0f, 0.0f, wave, lane);
    __syncthreads();
    float g[W::WAVES];
#pragma unroll
    for (int w = 0; w < W::WAVES; ++w) g[w] = f;
    if (part) write_merged<W, float>(sums, g, parts, r0, end, D);
    else write_merged<W, typename W::T>(sums, g, to, r0, end, D);
    __syncthreads();
  } else {
    if (part) write_rows<W, float>(lds + wave * W::STAGING, x, f, parts, r0, end, D, lane);
    else write_rows<W, typename W::T>(lds + wave * W::STAGING, x, f, to, r0, end, D, lane);
  }
}

// ------------------------------------------------------------- forward
// A block has queries of a head; tiles of keys and values go through LDS, the next one's loads under way.
template <typename W>
struct KeyTiles {
  static constexpr int STAGE = 2 * W::Load::BYTES, RING = W::STAGES * STAGE, ALL = W::SPLIT ? W::WAVES * RING : RING, LDS = W::lds(ALL);
  typedef antdt::Ring<W::STAGES, 2 * W::Load::PIECES, STAGE, !W::SPLIT> Ring;
};
template <typename W>
__global__ __launch_bounds__(W::THREADS, W::PER_CU) void cross_forward_kernel(CrossArgs a) {
  typedef typename W::T T;
  typedef typename W::Tile Tile;
  typedef Core<T> C;
  typedef KeyTiles<W> F;
  constexpr int BT = W::TILE;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, block;
  place_of(blockIdx.x, a.units, a.group * a.tiles, unit, block);
  const int tile = block % a.tiles, h = unit % a.heads * a.group + block / a.tiles;
  const int64_t b = unit / a.heads, bh = b * a.q_heads + h;
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t first = (int64_t)tile * W::ROWS, last = min(first + W::ROWS, a.S), r0 = first + (W::SPLIT ? 0 : wave * 32);
  const Rows out = a.out.rows(b, h);
  float* stats = a.stats ? a.stats + bh * a.S : nullptr;
  const int64_t end = k_len > 0 ? min(max(q_len, first), last) : first;   // rows with keys
  clear_rows<T>(out, end, last, a.D);
  if (stats)
    for (int64_t r = end + threadIdx.x; r < last; r += W::THREADS) stats[r] = INFINITY;
  if (end == first) return;
  if (a.D < W::COLS) {
    clear_lds(lds, F::ALL, W::THREADS);
    __syncthreads();
  }
  const typename W::Load load(W::SPLIT ? lane : threadIdx.x, a.D);
  const Rows k = a.k.rows(b, h / a.group), v = a.v.rows(b, h / a.group);
  const uint32_t ring0 = lds_address(lds) + (W::SPLIT ? wave * F::RING : 0), lds0 = ring0 + (W::SPLIT ? 0 : wave * 1024);
  constexpr int64_t STEP = (W::SPLIT ? W::WAVES : 1) * BT;
  const int64_t t0 = W::SPLIT ? wave * BT : 0;
  int64_t asked = t0;
  auto issue = [&](uint32_t to) {
    load(k, asked, k_len, lds0 + to);
    load(v, asked, k_len, lds0 + to + W::Load::BYTES);
    asked += STEP;
  };
  typename C::Fragment q[W::STEPS];
  load_rows<T, W::COLS>(a.q.rows(b, h), r0, q_len, a.D, lane, q);
  Sums<W> o;
  clear_sums<W>(o);
  float m = -INFINITY, l = 0.0f;   // of row lane % 32; l: of this lane's keys
  typename F::Ring ring((k_len - t0 + STEP - 1) / STEP);
  ring.start(issue);
  for (int64_t t = t0; t < k_len; t += STEP, ring.done()) {
    ring.next(issue);
    const uint32_t tile0 = ring0 + ring.read;
    const uint32_t tk = Tile::along_at(tile0, lane), tv = Tile::down_at(tile0 + W::Load::BYTES, lane);
    f32x16 s[BT / 32];
#pragma unroll
    for (int j = 0; j < BT / 32; ++j) s[j] = zeros();
    auto key = [&](int i) { return Tile::along(tk, i / W::STEPS * 32, i % W::STEPS); };
    Fragments<typename C::Fragment, BT / 32 * W::STEPS, W::AHEAD> keys;
    keys.start(key);
    keys.run(key, [&](int i, const typename C::Fragment& x) { C::multiply(x, q[i % W::STEPS], s[i / W::STEPS]); });
    auto value = [&](int i) { return Tile::down(tv, i / (W::DT * W::PACKS) * 32, i / W::DT % W::PACKS, i % W::DT); };
    Fragments<typename C::Fragment, BT / 32 * W::PACKS * W::DT, W::AHEAD> values;
    values.start(value);   // (there when the probabilities are)
    if (t + BT > k_len) {
      const int left = (int)(k_len - t) - 4 * half;
#pragma unroll
      for (int j = 0; j < BT / 32; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[j][e] = where_left(32 * j + 8 * (e >> 2) + (e & 3), left, s[j][e], -INFINITY);
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < BT / 32; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[j][e]);
    top = max_of_halves(top);
    // The sums are scaled anew only where a maximum grew by more than 2^8: until then p may exceed 1.
    if (__any(top > m && (top - m) * a.scale2 > 8.0f)) {
      const float now = fmaxf(m, top), f = m == -INFINITY ? 0.0f : exp2_((m - now) * a.scale2);
      m = now;
      l *= f;
#pragma unroll
      for (int d = 0; d < W::DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= f;
    }
    const float mc = m == -INFINITY ? 0.0f : m * a.scale2;
#pragma unroll
    for (int j = 0; j < BT / 32; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[j][e] = exp2_(fmaf(s[j][e], a.scale2, -mc));
        l += s[j][e];
      }
    typename C::Fragment p;
    values.run(value, [&](int i, const typename C::Fragment& x) {
      if (i % W::DT == 0) p = C::pack(s[i / (W::DT * W::PACKS)], i / W::DT % W::PACKS);
      C::multiply(x, p, o[i % W::DT]);
    });
  }
  arrive<0, true>();   // (the buffers are free)
  l = sum_of_halves(l);
  const float top2 = m == -INFINITY ? 0.0f : m * a.scale2;
  if constexpr (W::SPLIT) {
    float* sums = reinterpret_cast<float*>(lds);
    put_sums<W>(sums, o, l == 0.0f ? -INFINITY : top2, l, wave, lane);
    __syncthreads();
    const int row = threadIdx.x / (W::THREADS / 32);
    const float2* ml = reinterpret_cast<const float2*>(sums + W::WAVES * 32 * W::PITCH) + row;
    float f[W::WAVES], most = -INFINITY;
#pragma unroll
    for (int w = 0; w < W::WAVES; ++w) most = fmaxf(most, ml[32 * w].x);
    const float base = most == -INFINITY ? 0.0f : most;
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < W::WAVES; ++w) {
      f[w] = exp2_(ml[32 * w].x - base);
      l += ml[32 * w].y * f[w];
    }
#pragma unroll
    for (int w = 0; w < W::WAVES; ++w) f[w] *= l == 0.0f ? 0.0f : 1.0f / l;
    write_merged<W, T>(sums, f, out, first, end, a.D);
    if (stats && threadIdx.x % (W::THREADS / 32) == 0 && first + row < end) stats[first + row] = l == 0.0f ? INFINITY : base + log2_(l);
  } else {
    write_rows<W, T>(lds + wave * W::STAGING, o, l == 0.0f ? 0.0f : 1.0f / l, out, r0, end, a.D, lane);
    const int64_t r = r0 + (lane & 31);
    if (stats && lane < 32 && r < end) stats[r] = l == 0.0f ? INFINITY : top2 + log2_(l);
  }
}

// ------------------------------------------------------------- gradient of the queries
// As the forward pass; a lane has the sums L and d of its row.  Also leaves d for the gradients of keys and values.  d comes from out as it was
// kept; where one tile has all the keys it is the sum of p dP instead (the same number): of few keys dP - d nearly vanishes, and what out lost to its
// rounding would show (2 keys, bf16: dQ off by 0.005 of its norm, so by 0.0025, the operands' rounding).
template <typename W>
__global__ __launch_bounds__(W::THREADS, W::PER_CU) void cross_dq_kernel(CrossArgs a) {
  typedef typename W::T T;
  typedef typename W::Tile Tile;
  typedef Core<T> C;
  typedef KeyTiles<W> F;
  constexpr int BT = W::TILE;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, block;
  place_of(blockIdx.x, a.units, a.group * a.tiles * a.parts, unit, block);
  const int part = block % a.parts, tile = block / a.parts % a.tiles, h = unit % a.heads * a.group + block / a.parts / a.tiles;
  const int64_t b = unit / a.heads, bh = b * a.q_heads + h;
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t first = (int64_t)tile * W::ROWS, last = min(first + W::ROWS, a.S), r0 = first + (W::SPLIT ? 0 : wave * 32);
  const int64_t end = k_len > 0 ? min(max(q_len, first), last) : first;
  const bool wanted = a.dq.p != nullptr;
  const Rows dq = a.dq.rows(b, h);
  if (wanted && part == 0) clear_rows<T>(dq, end, last, a.D);
  if (end == first) return;
  typename C::Fragment q[W::STEPS], g[W::STEPS];
  load_rows<T, W::COLS>(a.dout.rows(b, h), r0, q_len, a.D, lane, g);
  load_rows<T, W::COLS>(a.out.rows(b, h), r0, q_len, a.D, lane, q);
  float delta = 0.0f;
#pragma unroll
  for (int i = 0; i < W::STEPS; ++i)
#pragma unroll
    for (int e = 0; e < C::PER; ++e) delta = fmaf((float)q[i][e], (float)g[i][e], delta);
  delta = sum_of_halves(delta);
  const int64_t r = r0 + (lane & 31);
  const float sum = r < end ? a.stats[bh * a.S + r] : INFINITY;
  const bool one_tile = k_len <= BT, writes_d = r < end && lane < 32 && part == 0 && (!W::SPLIT || wave == 0);
  if (!one_tile) {
    if (writes_d) a.delta[bh * a.S + r] = delta;
    if (!wanted) return;
  }
  load_rows<T, W::COLS>(a.q.rows(b, h), r0, q_len, a.D, lane, q);
  if (a.D < W::COLS) {
    clear_lds(lds, F::ALL, W::THREADS);
    __syncthreads();
  }
  const typename W::Load load(W::SPLIT ? lane : threadIdx.x, a.D);
  const Rows k = a.k.rows(b, h / a.group), v = a.v.rows(b, h / a.group);
  const uint32_t ring0 = lds_address(lds) + (W::SPLIT ? wave * F::RING : 0), lds0 = ring0 + (W::SPLIT ? 0 : wave * 1024);
  // the part's tiles, and the wavefront's of them
  const int64_t tiles = (k_len + BT - 1) / BT, behind = a.parts == 1 ? tiles : tiles * (part + 1) / a.parts;
  constexpr int STEP = W::SPLIT ? W::WAVES : 1;
  const int64_t i0 = (a.parts == 1 ? 0 : tiles * part / a.parts) + (W::SPLIT ? wave : 0);
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
    // p and dP of keys 32 j .. of the tile
    auto scores = [&](int j, f32x16& s, f32x16& dp) {
      s = dp = zeros();
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
    };
    if (one_tile) {   // (a block's, or, SPLIT, the first wavefront's, in the last part)
      delta = 0.0f;
      for (int j = 0; j < BT / 32; ++j) {
        f32x16 s, dp;
        scores(j, s, dp);
#pragma unroll
        for (int e = 0; e < 16; ++e) delta = fmaf(s[e], dp[e], delta);
      }
      delta = sum_of_halves(delta);
      if (r < end && lane < 32) a.delta[bh * a.S + r] = delta;
      if (!wanted) break;   // (nothing is under way)
    }
#pragma unroll
    for (int j = 0; j < BT / 32; ++j) {
      f32x16 s, dp;
      scores(j, s, dp);
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
  if (!wanted) return;
  float* sums = a.parts == 1 ? nullptr : a.partial + ((int64_t)part * a.units * a.group + bh) * a.S * a.D;
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
__global__ __launch_bounds__(W::THREADS, W::PER_CU) void cross_dkv_kernel(CrossArgs a) {
  typedef typename W::T T;
  typedef typename W::Tile Tile;
  typedef Core<T> C;
  typedef QueryTiles<W, HELD> F;
  constexpr int BR = W::TILE;
  static_assert(HELD || !W::SPLIT, "values in LDS are the block's");
  constexpr int UNROLL = W::DP <= 64 ? 2 : 1;   // (of wider heads there are no registers for two)
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, block;
  place_of(blockIdx.x, a.units, a.tiles * a.parts, unit, block);
  const int part = block % a.parts, tile = block / a.parts, h = unit % a.heads;
  const int64_t b = unit / a.heads;
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t first = (int64_t)tile * W::ROWS, last = min(first + W::ROWS, a.T), t0 = first + (W::SPLIT ? 0 : wave * 32);
  const int64_t end = q_len > 0 ? min(max(k_len, first), last) : first;
  const Rows dk = a.dk.rows(b, h), dv = a.dv.rows(b, h);
  if (part == 0) {
    clear_rows<T>(dk, end, last, a.D);
    clear_rows<T>(dv, end, last, a.D);
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
  const int64_t per_head = (q_len + BR - 1) / BR, tiles = per_head * a.group, behind = a.parts == 1 ? tiles : tiles * (part + 1) / a.parts;
  constexpr int STEP = W::SPLIT ? W::WAVES : 1;
  const int64_t i0 = (a.parts == 1 ? 0 : tiles * part / a.parts) + (W::SPLIT ? wave : 0);
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
      for (int e = 0; e < 16; ++e) {
        const int row = 64 * j + 8 * (e >> 2) + 4 * half + (e & 3);
        s[e] = exp2_(fmaf(s[e], a.scale2, -sums[row]));
        dp[e] = s[e] * (dp[e] - sums[32 + row]);
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
  float* sums = a.parts == 1 ? nullptr : a.partial + 2 * part * all + (int64_t)unit * a.T * a.D;
  write_result<W>(lds, ok, a.scale, dk, sums, t0, end, a.D, wave, lane);
  write_result<W>(lds, ov, 1.0f, dv, sums ? sums + all : nullptr, t0, end, a.D, wave, lane);
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

// ------------------------------------------------------------- launches
template <typename T, int DP>
struct Ways {
  static constexpr int ROW = DP * sizeof(T);   // bytes
  template <int COLS> using Keys = Way<T, DP, COLS, ROW == 512 ? 32 : 64, 2, 4, false, 2, 4>;
  template <int COLS> using KeysDq = Way<T, DP, COLS, ROW == 512 ? 32 : 64, 2, 4, false, ROW == 512 ? 1 : 2, 4>;
  template <int COLS> using Queries = Way<T, DP, COLS, ROW >= 256 ? 32 : 64, 2, 4, false, ROW == 512 ? 1 : 2, 4>;
  template <int COLS> using SplitKeys = Way<T, DP, COLS, 32, 2, ROW == 512 ? 2 : 4, true, ROW >= 256 ? 1 : 2, 4>;
  template <int COLS> using SplitQueries = Way<T, DP, COLS, 32, 2, 2, true, ROW >= 256 ? 1 : 2, 4>;
  static constexpr bool HELD = !(sizeof(T) == 2 && DP == 128);
};
struct Plan {
  bool split;
  int32_t tiles, parts;
  int64_t blocks;
};
template <typename K>
hipError_t launch(K kernel, int threads, int lds, std::atomic<uint64_t>& allowed, const Plan& pl, CrossArgs a, hipStream_t s) {
  const hipError_t e = allow_lds(kernel, lds, 0, allowed);
  if (e != hipSuccess) return e;
  a.tiles = pl.tiles; a.parts = pl.parts;
  hipLaunchKernelGGL(kernel, dim3((unsigned)pl.blocks), dim3(threads), lds, s, a);
  return hipGetLastError();
}
template <typename W>
hipError_t launch_forward(const CrossArgs& a, const Plan& pl, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  return launch(cross_forward_kernel<W>, W::THREADS, KeyTiles<W>::LDS, allowed, pl, a, s);
}
template <typename W>
hipError_t launch_dq(const CrossArgs& a, const Plan& pl, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  return launch(cross_dq_kernel<W>, W::THREADS, KeyTiles<W>::LDS, allowed, pl, a, s);
}
template <typename W, bool HELD>
hipError_t launch_dkv(const CrossArgs& a, const Plan& pl, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  return launch(cross_dkv_kernel<W, HELD>, W::THREADS, QueryTiles<W, HELD>::LDS, allowed, pl, a, s);
}
// go(Ways<T, DP>, COLS)
template <typename F>
hipError_t by_columns(int32_t dtype, int D, F go) {
  return by_size(dtype, D, [&](auto t, auto dp) {
    constexpr int DP = decltype(dp)::value;
    typedef Ways<decltype(t), DP> Z;
    if constexpr (DP == 128) {
      if (D <= 96) return go(Z(), std::integral_constant<int, 96>());
    }
    return go(Z(), dp);
  });
}

struct Shape {
  int64_t B, S, T, q_heads, heads, D;
  int32_t dtype;
};
// Microseconds that a wavefront takes for 32 queries and 32 keys in the forward pass, alone on its SIMD (measured; of a multiple of 32 columns).
double tile_us(const Shape& z) {
  const int columns = (int)div_up(z.D, 32) - 1;
  constexpr double BF16[] = {0.6, 0.9, 1.3, 1.6}, F32[] = {1.7, 3.1, 4.3, 5.5};
  return z.dtype == ANTDT_F32 ? F32[columns] : BF16[columns];
}
// Results' rows in blocks of 128, or of 32 whose `waves` wavefronts share the other side's rows (`tiles` of 32), or these again in parts.
//  - Blocks of 32 as long as all of them run at once: `most` of them.  bf16, 1024 queries and keys, 64 columns, us of blocks of 128 / 32: 16 heads 22 / 15,
//    32 heads 23.5 / 28; gradient of the queries 27 / 19, 28 / 32; 128 columns, gradient of the keys: 16 heads 57 / 44, 32 heads 62 / 90.
//  - Parts where their shorter way outweighs the launch that adds them up, about 6 us.
Plan cross_plan(int64_t heads, int64_t rows, int64_t tiles, int64_t most, int waves, double us, bool parted) {
  Plan p = {false, (int32_t)div_up(rows, 128), 1, 0};
  p.blocks = heads * p.tiles;
  const int64_t split = heads * div_up(rows, 32);
  if (split == 0 || split > most || tiles < 2) return p;
  p.split = true;
  p.tiles = (int32_t)div_up(rows, 32);
  p.blocks = split;
  const int64_t parts = std::min<int64_t>(256 / split, tiles / (2 * waves));
  if (parted && parts > 1 && us * tiles / waves * (1.0 - 1.0 / parts) > 6.0) {
    p.parts = (int32_t)parts;
    p.blocks *= parts;
  }
  return p;
}
int64_t delta_bytes(const Shape& z) { return div_up(z.B * z.S * z.q_heads * 4, 256) * 256; }
bool wide(const Shape& z) { return z.dtype == ANTDT_BF16 && z.D > 64; }          // (a block of 32 fills a compute unit's LDS)
int key_waves(const Shape& z) { return z.dtype == ANTDT_F32 && z.D > 64 ? 2 : 4; }
Plan forward_plan(const Shape& z) { return cross_plan(z.B * z.q_heads, z.S, div_up(z.T, 32), wide(z) ? 256 : 512, key_waves(z), tile_us(z), false); }
Plan dq_plan(const Shape& z) { return cross_plan(z.B * z.q_heads, z.S, div_up(z.T, 32), wide(z) ? 256 : 512, key_waves(z), 1.3 * tile_us(z), true); }
Plan dkv_plan(const Shape& z) { return cross_plan(z.B * z.heads, z.T, div_up(z.S, 32) * (z.q_heads / z.heads), 512, 2, 2.0 * tile_us(z), true); }
// Whether the forward pass goes by an equal share of all keys to each wavefront (stream.hip) instead, by the time that both would take: that costs a
// second launch, about 9 us, and the tiles of 32 keys and 16 or 32 queries of a key's heads take 1.4 times as long.  us by blocks / shares, 8 heads of
// 64 bf16 columns: 1 query, 500 keys 8 / 16, 2000 19 / 15, 8000 61 / 16; 4 x 128 queries, 2000 keys 20 / 31, 8000 75 / 64; fp32, 1 query, 500 keys 16 / 14.
bool cross_streams(const Shape& z) {
  if (z.B == 0 || z.S == 0 || !stream_fits(z.B, z.S, z.T, z.q_heads, z.heads)) return false;
  const int64_t tiles = div_up(z.T, 32), rows = z.S * (z.q_heads / z.heads), row_tiles = rows <= 16 ? 1 : div_up(rows, 32);
  const Plan p = forward_plan(z);
  const double blocks = p.split ? (double)div_up(tiles, key_waves(z)) : std::max(1.0, p.blocks / 512.0) * tiles * 1.1;
  return 9.0 + 1.4 * tile_us(z) * z.B * z.heads * row_tiles * tiles / 1024 < tile_us(z) * blocks;
}
int cross_sizes(const char* call, const Shape& z) {
  OP_TRY(op_head_sizes(call, z.q_heads, z.heads, z.D, z.dtype));
  constexpr int64_t MOST = (1ll << 31) - 1;
  if (z.B < 0 || z.B >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: B out of range", call);
  if (z.S < 0 || z.S >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: S out of range", call);
  if (z.T < 0 || z.T >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: T out of range", call);
  const int64_t longest = div_up(std::max(z.S, z.T), 128);
  if ((__int128)z.B * z.q_heads * longest >= 1 << 24) return op_fail(ANTDT_UNSUPPORTED, "%s: B q_heads and the longer of S and T in 128s: 2^24 or more blocks", call);
  return ANTDT_OK;
}
int cross_lengths(const char* call, const int32_t* q_lengths, const int32_t* k_lengths) {
  if ((reinterpret_cast<uintptr_t>(q_lengths) | reinterpret_cast<uintptr_t>(k_lengths)) & 3) return op_fail(ANTDT_INVALID_ARG, "%s: lengths are misaligned", call);
  return ANTDT_OK;
}
}  // namespace
}  // namespace antdt

using namespace antdt;

extern "C" {

int antdt_cross_attention_bytes(int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_cross_attention_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  const Shape z = {B, S, T, q_heads, heads, D, dtype};
  OP_TRY(cross_sizes(call, z));
  *bytes = cross_streams(z) && z.B > 0 ? stream_bytes(B, S, q_heads, heads, D) : 0;
  return ANTDT_OK;
}

int antdt_cross_attention(const void* q, int64_t ldq_batch, int64_t ldq, int64_t ldq_head, const void* k, int64_t ldk_batch, int64_t ldk, int64_t ldk_head,
                          const void* v, int64_t ldv_batch, int64_t ldv, int64_t ldv_head, int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads,
                          int64_t D, int32_t dtype, const int32_t* q_lengths, const int32_t* k_lengths, float scale, void* out, int64_t ldo_batch,
                          int64_t ldo, int64_t ldo_head, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "antdt_cross_attention";
  CrossArgs a = {};
  const Shape z = {B, S, T, q_heads, heads, D, dtype};
  OP_TRY(cross_sizes(call, z));
  OP_TRY(op_scale(call, scale));
  a.scale = scale; a.scale2 = scale * LOG2E;
  OP_TRY(op_wide_heads(call, "q", q, B, S, q_heads, D, dtype, {ldq_batch, ldq, ldq_head}, false, a.q));
  OP_TRY(op_wide_heads(call, "k", k, B, T, heads, D, dtype, {ldk_batch, ldk, ldk_head}, false, a.k));
  OP_TRY(op_wide_heads(call, "v", v, B, T, heads, D, dtype, {ldv_batch, ldv, ldv_head}, false, a.v));
  OP_TRY(op_wide_heads(call, "out", out, B, S, q_heads, D, dtype, {ldo_batch, ldo, ldo_head}, true, a.out));
  OP_TRY(cross_lengths(call, q_lengths, k_lengths));
  if (reinterpret_cast<uintptr_t>(stats) & 3) return op_fail(ANTDT_INVALID_ARG, "%s: stats is misaligned", call);
  if (B == 0 || S == 0) return ANTDT_OK;
  const hipStream_t s = (hipStream_t)stream;
  if (cross_streams(z)) {
    OP_TRY(op_workspace(call, workspace, workspace_bytes, stream_bytes(B, S, q_heads, heads, D)));
    StreamArgs f = {};
    f.q = a.q; f.k = a.k; f.v = a.v; f.out = a.out; f.q_lengths = q_lengths; f.k_lengths = k_lengths; f.stats = stats;
    f.B = B; f.S = S; f.T = T; f.q_heads = (int)q_heads; f.heads = (int)heads; f.group = (int)(q_heads / heads); f.D = (int)D; f.scale2 = a.scale2;
    return op_hip(call, launch_stream(f, dtype, workspace, s));
  }
  a.q_lengths = q_lengths; a.k_lengths = k_lengths; a.stats = stats; a.S = S; a.T = T;
  a.q_heads = (int)q_heads; a.heads = (int)heads; a.group = (int)(q_heads / heads); a.D = (int)D; a.units = (int)(B * heads);
  const Plan pl = forward_plan(z);
  return op_hip(call, by_columns(dtype, (int)D, [&](auto z, auto cols) {
    typedef decltype(z) Z;
    constexpr int COLS = decltype(cols)::value;
    return pl.split ? launch_forward<typename Z::template SplitKeys<COLS>>(a, pl, s) : launch_forward<typename Z::template Keys<COLS>>(a, pl, s);
  }));
}

int antdt_cross_attention_backward_bytes(int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_cross_attention_backward_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  const Shape z = {B, S, T, q_heads, heads, D, dtype};
  OP_TRY(cross_sizes(call, z));
  *bytes = (size_t)delta_bytes(z) + 4 * D * std::max(dq_plan(z).parts > 1 ? dq_plan(z).parts * B * q_heads * S : 0, dkv_plan(z).parts > 1 ? 2 * dkv_plan(z).parts * B * heads * T : 0);
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
  a.q_heads = (int)q_heads; a.heads = (int)heads; a.group = (int)(q_heads / heads); a.D = (int)D; a.units = (int)(B * heads);
  const hipStream_t s = (hipStream_t)stream;
  a.partial = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + delta_bytes(z));
  // The parts' sums to the results.
  auto join = [&](const Plan& pl, const HeadsArg& x, const HeadsArg& y, int results, int64_t H, int64_t L, int64_t other, const int32_t* lengths, const int32_t* others) {
    JoinArgs j = {{x, y}, a.partial, lengths, others, L, other, B * H * L * D / 4, (int32_t)H, (int32_t)D, pl.parts, results};
    const dim3 grid((unsigned)div_up(j.quads, 256), results);
    if (dtype == ANTDT_F32) hipLaunchKernelGGL(cross_join_kernel<float>, grid, dim3(256), 0, s, j);
    else hipLaunchKernelGGL(cross_join_kernel<bf16_t>, grid, dim3(256), 0, s, j);
    return hipGetLastError();
  };
  if (queries) {
    const Plan pl = dq_plan(z);
    OP_TRY(op_hip(call, by_columns(dtype, (int)D, [&](auto z, auto cols) {
      typedef decltype(z) Z;
      constexpr int COLS = decltype(cols)::value;
      return pl.split ? launch_dq<typename Z::template SplitKeys<COLS>>(a, pl, s) : launch_dq<typename Z::template KeysDq<COLS>>(a, pl, s);
    })));
    if (dq && pl.parts > 1) OP_TRY(op_hip(call, join(pl, a.dq, a.dq, 1, q_heads, S, T, q_lengths, k_lengths)));
  }
  if (keys) {
    const Plan pl = dkv_plan(z);
    OP_TRY(op_hip(call, by_columns(dtype, (int)D, [&](auto z, auto cols) {
      typedef decltype(z) Z;
      constexpr int COLS = decltype(cols)::value;
      return pl.split ? launch_dkv<typename Z::template SplitQueries<COLS>, true>(a, pl, s) : launch_dkv<typename Z::template Queries<COLS>, Z::HELD>(a, pl, s);
    })));
    if (pl.parts > 1) OP_TRY(op_hip(call, join(pl, a.dk, a.dv, 2, heads, T, S, k_lengths, q_lengths)));
  }
  return ANTDT_OK;
}

}  // extern "C"
