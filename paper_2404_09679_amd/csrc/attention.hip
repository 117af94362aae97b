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
  float scale, scale2;   // scale2: scale log2 e
};

// Own loads but the last N have arrived, own reads of LDS are done; then everybody's.
template <int N>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
  block_barrier();
}
// Tiles through a ring of STAGES buffers in LDS, LOADS of a wavefront each: while one is worked on, the next STAGES - 1 are under way.
template <int STAGES, int LOADS, int BYTES>
struct Ring {
  uint32_t fill = 0, read = 0;   // bytes from the ring's start: the next buffer to fill, the one to read
  int64_t left;                  // tiles not asked for yet
  int64_t behind = 0;            // tiles asked for and not worked on
  __device__ __forceinline__ explicit Ring(int64_t tiles) : left(tiles) {}
  template <typename F>
  __device__ __forceinline__ void ask(F issue) {
    if (left == 0) return;
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
    if (behind == STAGES - 1) arrive<(STAGES - 2) * LOADS>();
    else arrive<0>();
    --behind;
    ask(issue);
  }
  __device__ __forceinline__ void done() { read = read == (STAGES - 1) * BYTES ? 0 : read + BYTES; }
};

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

constexpr int BLOCK_ROWS = 128;   // queries or keys of a block, 32 to a wavefront

template <int DP>
struct Staging {   // a wavefront's rows on their way to memory, some columns at a time
  static constexpr int TN = DP >= 64 ? 2 : 1, BYTES = 32 * (32 * TN + 4) * 4;
};
// 32 rows x DP of sums, columns in elements: f x, to `rows` rows of `to`.
template <typename T, int DP>
__device__ __forceinline__ void write_rows(char* staging, const f32x16 (&x)[DP / 32], float f, const Rows& to, int64_t r0, int64_t rows, int D, int lane) {
  constexpr int TN = Staging<DP>::TN;
  const int left = (int)max(min(rows - r0, (int64_t)32), (int64_t)0);
  T* p = reinterpret_cast<T*>(const_cast<char*>(to.p + r0 * to.ld));
#pragma unroll
  for (int i = 0; i < DP / 32; i += TN) {
    f32x16 y[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) y[j][e] = x[i + j][e] * f;
    store_rows<T, TN, true>(reinterpret_cast<float*>(staging), y, p + 32 * i, to.ld / (int64_t)sizeof(T), left, D - 32 * i, lane);
  }
}
// Zeros to rows [r0, r1) of a head, by the block.
template <typename T>
__device__ __forceinline__ void clear_rows(const Rows& to, int64_t r0, int64_t r1, int D) {
  const int per = D / Core<T>::PER;
  for (int64_t i = threadIdx.x; i < (r1 - r0) * per; i += blockDim.x)
    store16<false>(const_cast<char*>(to.p + (r0 + i / per) * to.ld + i % per * 16), make_uint4(0, 0, 0, 0));
}

// ------------------------------------------------------------- forward
// A block has 128 queries of a head, 32 to a wavefront; tiles of BT keys and values go through LDS, the next one's loads under way.
template <typename T, int DP, int BT, int STAGES_>
struct KeyTiles {
  typedef HeadTile<T, DP> Tile;
  typedef TileLoad<T, DP, BT, 256> Load;
  static constexpr int STAGES = STAGES_, STAGE = 2 * Load::BYTES, RING = STAGES * STAGE;
  static constexpr int LDS = RING > 4 * Staging<DP>::BYTES ? RING : 4 * Staging<DP>::BYTES;
  typedef ::antdt::Ring<STAGES, 2 * Load::PIECES, STAGE> Ring;
};
template <typename T, int DP, int BT, int STAGES>
__global__ __launch_bounds__(256, 2) void cross_forward_kernel(CrossArgs a) {
  typedef KeyTiles<T, DP, BT, STAGES> F;
  typedef typename F::Tile Tile;
  typedef Core<T> C;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, block;
  place_of(blockIdx.x, a.units, a.group * a.tiles, unit, block);
  const int tile = block % a.tiles, h = unit % a.heads * a.group + block / a.tiles;
  const int64_t b = unit / a.heads, bh = b * a.q_heads + h;
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t first = (int64_t)tile * BLOCK_ROWS, last = min(first + BLOCK_ROWS, a.S), r0 = first + wave * 32;
  const Rows out = a.out.rows(b, h);
  float* stats = a.stats ? a.stats + (bh * a.S) : nullptr;
  const int64_t end = k_len > 0 ? min(max(q_len, first), last) : first;   // rows with keys
  clear_rows<T>(out, end, last, a.D);
  if (stats)
    for (int64_t r = end + threadIdx.x; r < last; r += 256) stats[r] = INFINITY;
  if (end == first) return;
  if (a.D < DP) {
    clear_lds(lds, F::RING, 256);
    __syncthreads();
  }
  const typename F::Load load(threadIdx.x, a.D);
  const Rows k = a.k.rows(b, h / a.group), v = a.v.rows(b, h / a.group);
  const uint32_t lds0 = lds_address(lds) + wave * 1024;
  int64_t asked = 0;
  auto issue = [&](uint32_t to) {
    load(k, asked, k_len, lds0 + to);
    load(v, asked, k_len, lds0 + to + F::Load::BYTES);
    asked += BT;
  };
  typename C::Fragment q[DP / C::STEP];
  load_rows<T, DP>(a.q.rows(b, h), r0, q_len, a.D, lane, q);
  f32x16 o[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) o[d] = zeros();
  float m = -INFINITY, l = 0.0f;   // of row lane % 32; l: of this lane's keys
  typename F::Ring ring((k_len + BT - 1) / BT);
  ring.start(issue);
  for (int64_t t = 0; t < k_len; t += BT, ring.done()) {
    ring.next(issue);
    const uint32_t tile0 = lds_address(lds) + ring.read;
    const uint32_t tk = Tile::along_at(tile0, lane), tv = Tile::down_at(tile0 + F::Load::BYTES, lane);
    f32x16 s[BT / 32];
#pragma unroll
    for (int j = 0; j < BT / 32; ++j) {
      s[j] = zeros();
#pragma unroll
      for (int i = 0; i < DP / C::STEP; ++i) C::multiply(Tile::along(tk, 32 * j, i), q[i], s[j]);
    }
    if (t + BT > k_len) {
#pragma unroll
      for (int j = 0; j < BT / 32; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (t + 32 * j + 8 * (e >> 2) + 4 * half + (e & 3) >= k_len) s[j][e] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < BT / 32; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[j][e]);
    top = fmaxf(top, other_half(top));
    // The sums are scaled anew only where a maximum grew by more than 2^8: until then p may exceed 1.
    if (__any(top > m && (top - m) * a.scale2 > 8.0f)) {
      const float now = fmaxf(m, top), f = m == -INFINITY ? 0.0f : exp2_((m - now) * a.scale2);
      m = now;
      l *= f;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
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
#pragma unroll
    for (int j = 0; j < BT / 32; ++j)
#pragma unroll
      for (int i = 0; i < 32 / C::STEP; ++i) {
        const typename C::Fragment p = C::pack(s[j], i);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) C::multiply(Tile::down(tv, 32 * j, i, d), p, o[d]);
      }
  }
  arrive<0>();   // (the buffers are free)
  l += other_half(l);
  write_rows<T, DP>(lds + wave * Staging<DP>::BYTES, o, l == 0.0f ? 0.0f : 1.0f / l, out, r0, end, a.D, lane);
  const int64_t r = r0 + (lane & 31);
  if (stats && lane < 32 && r < end) stats[r] = l == 0.0f ? INFINITY : m * a.scale2 + log2_(l);
}

// ------------------------------------------------------------- gradient of the queries
// As the forward pass; a lane has the sums L and d of its row.  Also leaves d for the gradients of keys and values.  d comes from out as it was
// kept; where one tile has all the keys it is the sum of p dP instead (the same number): of few keys dP - d nearly vanishes, and what out lost to its
// rounding would show (2 keys, bf16: dQ off by 0.005 of its norm, so by 0.0025, the operands' rounding).
template <typename T, int DP, int BT, int STAGES>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP == 128 ? 1 : 2) void cross_dq_kernel(CrossArgs a) {
  typedef KeyTiles<T, DP, BT, STAGES> F;
  typedef typename F::Tile Tile;
  typedef Core<T> C;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, block;
  place_of(blockIdx.x, a.units, a.group * a.tiles, unit, block);
  const int tile = block % a.tiles, h = unit % a.heads * a.group + block / a.tiles;
  const int64_t b = unit / a.heads, bh = b * a.q_heads + h;
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t first = (int64_t)tile * BLOCK_ROWS, last = min(first + BLOCK_ROWS, a.S), r0 = first + wave * 32;
  const int64_t end = k_len > 0 ? min(max(q_len, first), last) : first;
  const bool wanted = a.dq.p != nullptr;
  const Rows dq = a.dq.rows(b, h);
  if (wanted) clear_rows<T>(dq, end, last, a.D);
  if (end == first) return;
  typename C::Fragment q[DP / C::STEP], g[DP / C::STEP];
  load_rows<T, DP>(a.dout.rows(b, h), r0, q_len, a.D, lane, g);
  load_rows<T, DP>(a.out.rows(b, h), r0, q_len, a.D, lane, q);
  float delta = 0.0f;
#pragma unroll
  for (int i = 0; i < DP / C::STEP; ++i)
#pragma unroll
    for (int e = 0; e < C::PER; ++e) delta = fmaf((float)q[i][e], (float)g[i][e], delta);
  delta += other_half(delta);
  const int64_t r = r0 + (lane & 31);
  const float sum = r < end ? a.stats[bh * a.S + r] : INFINITY;
  const bool one_tile = k_len <= BT;
  if (!one_tile) {
    if (r < end && lane < 32) a.delta[bh * a.S + r] = delta;
    if (!wanted) return;
  }
  load_rows<T, DP>(a.q.rows(b, h), r0, q_len, a.D, lane, q);
  if (a.D < DP) {
    clear_lds(lds, F::RING, 256);
    __syncthreads();
  }
  const typename F::Load load(threadIdx.x, a.D);
  const Rows k = a.k.rows(b, h / a.group), v = a.v.rows(b, h / a.group);
  const uint32_t lds0 = lds_address(lds) + wave * 1024;
  int64_t asked = 0;
  auto issue = [&](uint32_t to) {
    load(k, asked, k_len, lds0 + to);
    load(v, asked, k_len, lds0 + to + F::Load::BYTES);
    asked += BT;
  };
  f32x16 o[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) o[d] = zeros();
  typename F::Ring ring((k_len + BT - 1) / BT);
  ring.start(issue);
  for (int64_t t = 0; t < k_len; t += BT, ring.done()) {
    ring.next(issue);
    const uint32_t tile0 = lds_address(lds) + ring.read;
    const uint32_t tk = Tile::along_at(tile0, lane), tv = Tile::along_at(tile0 + F::Load::BYTES, lane), kt = Tile::down_at(tile0, lane);
    // p and dP of keys 32 j .. of the tile
    auto scores = [&](int j, f32x16& s, f32x16& dp) {
      s = dp = zeros();
#pragma unroll
      for (int i = 0; i < DP / C::STEP; ++i) C::multiply(Tile::along(tk, 32 * j, i), q[i], s);
#pragma unroll
      for (int i = 0; i < DP / C::STEP; ++i) C::multiply(Tile::along(tv, 32 * j, i), g[i], dp);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = exp2_(fmaf(s[e], a.scale2, -sum));
      if (t + BT > k_len) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (t + 32 * j + 8 * (e >> 2) + 4 * half + (e & 3) >= k_len) s[e] = dp[e] = 0.0f;
      }
    };
    if (one_tile) {
      delta = 0.0f;
      for (int j = 0; j < BT / 32; ++j) {
        f32x16 s, dp;
        scores(j, s, dp);
#pragma unroll
        for (int e = 0; e < 16; ++e) delta = fmaf(s[e], dp[e], delta);
      }
      delta += other_half(delta);
      if (r < end && lane < 32) a.delta[bh * a.S + r] = delta;
      if (!wanted) return;   // (nothing is under way)
    }
#pragma unroll
    for (int j = 0; j < BT / 32; ++j) {
      f32x16 s, dp;
      scores(j, s, dp);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= dp[e] - delta;
#pragma unroll
      for (int i = 0; i < 32 / C::STEP; ++i) {
        const typename C::Fragment ds = C::pack(s, i);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) C::multiply(Tile::down(kt, 32 * j, i, d), ds, o[d]);
      }
    }
  }
  arrive<0>();
  write_rows<T, DP>(lds + wave * Staging<DP>::BYTES, o, a.scale, dq, r0, end, a.D, lane);
}

// ------------------------------------------------------------- gradients of keys and values
// A block has 128 keys of a head, 32 to a wavefront, and goes through tiles of BR queries and their outputs' gradients, of every head that shares
// the keys.
template <typename T, int DP, int BR, int STAGES_, int KEYS, bool HELD>
struct QueryTiles {
  typedef HeadTile<T, DP> Tile;
  typedef TileLoad<T, DP, BR, 256> Load;
  static constexpr int STATS = 2 * BR * 4;   // L and d of the rows, for each wavefront: (L, d) of 32 rows behind each other
  typedef TileLoad<T, DP, KEYS, 256> Values;
  static constexpr int STAGES = STAGES_, STAGE = 2 * Load::BYTES + 4 * STATS, RING = STAGES * STAGE + (HELD ? 0 : Values::BYTES);
  static constexpr int LDS = RING > 4 * Staging<DP>::BYTES ? RING : 4 * Staging<DP>::BYTES;
  typedef ::antdt::Ring<STAGES, 2 * Load::PIECES + BR / 32, STAGE> Ring;
};
template <typename T, int DP, int BR, int STAGES, int NT, bool HELD, int PER_CU>
__global__ __launch_bounds__(256, PER_CU) void cross_dkv_kernel(CrossArgs a) {
  typedef QueryTiles<T, DP, BR, STAGES, 128 * NT, HELD> F;
  typedef typename F::Tile Tile;
  typedef Core<T> C;
  constexpr int KEYS = 128 * NT;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, tile;
  place_of(blockIdx.x, a.units, a.tiles, unit, tile);
  const int h = unit % a.heads;
  const int64_t b = unit / a.heads;
  const int64_t q_len = length_of(a.q_lengths, b, a.S), k_len = length_of(a.k_lengths, b, a.T);
  const int64_t first = (int64_t)tile * KEYS, last = min(first + KEYS, a.T), t0 = first + wave * (32 * NT);
  const int64_t end = q_len > 0 ? min(max(k_len, first), last) : first;
  const Rows dk = a.dk.rows(b, h), dv = a.dv.rows(b, h);
  clear_rows<T>(dk, end, last, a.D);
  clear_rows<T>(dv, end, last, a.D);
  if (end == first) return;
  if (a.D < DP) {
    clear_lds(lds, F::RING, 256);
    __syncthreads();
  }
  const typename F::Load load(threadIdx.x, a.D);
  const uint32_t lds0 = lds_address(lds) + wave * 1024;
  int64_t asked_g = 0, asked = 0;
  const float* const sums_of = half ? a.delta : a.stats;
  auto issue = [&](uint32_t to) {
    const int64_t hq = (int64_t)h * a.group + asked_g;
    load(a.q.rows(b, hq), asked, q_len, lds0 + to);
    load(a.dout.rows(b, hq), asked, q_len, lds0 + to + F::Load::BYTES);
#pragma unroll
    for (int j = 0; j < BR / 32; ++j)
      load_lds4(sums_of + (b * a.q_heads + hq) * a.S + min(asked + 32 * j + (lane & 31), q_len - 1),
                lds_address(lds) + to + 2 * F::Load::BYTES + wave * F::STATS + j * 256);
    asked += BR;
    if (asked >= q_len) {
      asked = 0;
      ++asked_g;
    }
  };
  typename C::Fragment k[NT][DP / C::STEP], v[HELD ? NT : 1][HELD ? DP / C::STEP : 1];
  f32x16 ok[NT][DP / 32], ov[NT][DP / 32];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    load_rows<T, DP>(a.k.rows(b, h), t0 + 32 * n, k_len, a.D, lane, k[n]);
    if constexpr (HELD) load_rows<T, DP>(a.v.rows(b, h), t0 + 32 * n, k_len, a.D, lane, v[n]);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) ok[n][d] = ov[n][d] = zeros();
  }
  if constexpr (!HELD) {
    const typename F::Values values(threadIdx.x, a.D);
    values(a.v.rows(b, h), first, k_len, lds0 + STAGES * F::STAGE);
  }
  typename F::Ring ring((q_len + BR - 1) / BR * a.group);
  ring.start(issue);
  for (int64_t g = 0, r = 0; g < a.group; ring.done()) {
    ring.next(issue);
    const uint32_t tile0 = lds_address(lds) + ring.read;
    const float* sums = reinterpret_cast<const float*>(lds + ring.read + 2 * F::Load::BYTES + wave * F::STATS);
    const uint32_t tq = Tile::along_at(tile0, lane), tg = Tile::along_at(tile0 + F::Load::BYTES, lane);
    const uint32_t vt = HELD ? 0 : Tile::along_at(lds_address(lds) + STAGES * F::STAGE + wave * (32 * NT * Tile::ROW), lane);
    const uint32_t qt = Tile::down_at(tile0, lane), gt = Tile::down_at(tile0 + F::Load::BYTES, lane);
#pragma unroll 1
    for (int j = 0; j < BR / 32; ++j) {
      f32x16 s[NT], dp[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n] = dp[n] = zeros();
#pragma unroll
      for (int i = 0; i < DP / C::STEP; ++i) {
        const typename C::Fragment x = Tile::along(tq, 32 * j, i);
#pragma unroll
        for (int n = 0; n < NT; ++n) C::multiply(x, k[n][i], s[n]);
      }
#pragma unroll
      for (int i = 0; i < DP / C::STEP; ++i) {
        const typename C::Fragment x = Tile::along(tg, 32 * j, i);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if constexpr (HELD) C::multiply(x, v[n][i], dp[n]);
          else C::multiply(x, Tile::along(vt, 32 * n, i), dp[n]);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int row = 64 * j + 8 * (e >> 2) + 4 * half + (e & 3);
          s[n][e] = exp2_(fmaf(s[n][e], a.scale2, -sums[row]));
          dp[n][e] = s[n][e] * (dp[n][e] - sums[32 + row]);
        }
      if (r + BR > q_len) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (r + 32 * j + 8 * (e >> 2) + 4 * half + (e & 3) >= q_len) s[n][e] = dp[n][e] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 32 / C::STEP; ++i) {
        typename C::Fragment p[NT], ds[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          p[n] = C::pack(s[n], i);
          ds[n] = C::pack(dp[n], i);
        }
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
          const typename C::Fragment x = Tile::down(gt, 32 * j, i, d), y = Tile::down(qt, 32 * j, i, d);
#pragma unroll
          for (int n = 0; n < NT; ++n) C::multiply(x, p[n], ov[n][d]);
#pragma unroll
          for (int n = 0; n < NT; ++n) C::multiply(y, ds[n], ok[n][d]);
        }
      }
    }
    r += BR;
    if (r >= q_len) {
      r = 0;
      ++g;
    }
  }
  arrive<0>();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    write_rows<T, DP>(lds + wave * Staging<DP>::BYTES, ok[n], a.scale, dk, t0 + 32 * n, end, a.D, lane);
    write_rows<T, DP>(lds + wave * Staging<DP>::BYTES, ov[n], 1.0f, dv, t0 + 32 * n, end, a.D, lane);
  }
}

// ------------------------------------------------------------- launches
template <typename K>
hipError_t launch(K kernel, int lds, std::atomic<uint64_t>& allowed, int64_t blocks, const CrossArgs& a, hipStream_t s) {
  const hipError_t e = allow_lds(kernel, lds, 0, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), lds, s, a);
  return hipGetLastError();
}
// Tiles: rows, and buffers of the ring.
template <typename T, int DP>
struct Tiles {
  static constexpr bool LARGE = DP * sizeof(T) >= 256;
  static constexpr int KEYS = DP * sizeof(T) == 512 ? 32 : 64, KEY_STAGES = 2;
  static constexpr int QUERIES = LARGE ? 32 : 64, QUERY_STAGES = 2;
  static constexpr bool HELD = !(sizeof(T) == 2 && DP == 128);
  static constexpr int KEY_TILES = 1, PER_CU = DP * sizeof(T) == 512 ? 1 : 2;
};
template <typename T, int DP>
hipError_t launch_forward(const CrossArgs& a, int64_t blocks, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  typedef Tiles<T, DP> Z;
  return launch(cross_forward_kernel<T, DP, Z::KEYS, Z::KEY_STAGES>, KeyTiles<T, DP, Z::KEYS, Z::KEY_STAGES>::LDS, allowed, blocks, a, s);
}
template <typename T, int DP>
hipError_t launch_dq(const CrossArgs& a, int64_t blocks, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  typedef Tiles<T, DP> Z;
  return launch(cross_dq_kernel<T, DP, Z::KEYS, Z::KEY_STAGES>, KeyTiles<T, DP, Z::KEYS, Z::KEY_STAGES>::LDS, allowed, blocks, a, s);
}
template <typename T, int DP>
hipError_t launch_dkv(CrossArgs a, int64_t heads, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  typedef Tiles<T, DP> Z;
  a.tiles = (int)div_up(a.T, 128 * Z::KEY_TILES);
  return launch(cross_dkv_kernel<T, DP, Z::QUERIES, Z::QUERY_STAGES, Z::KEY_TILES, Z::HELD, Z::PER_CU>,
                QueryTiles<T, DP, Z::QUERIES, Z::QUERY_STAGES, 128 * Z::KEY_TILES, Z::HELD>::LDS, allowed, heads * a.tiles, a, s);
}

struct Shape {
  int64_t B, S, T, q_heads, heads, D;
  int32_t dtype;
};
int cross_sizes(const char* call, const Shape& z) {
  OP_TRY(op_head_sizes(call, z.q_heads, z.heads, z.D, z.dtype));
  constexpr int64_t MOST = (1ll << 31) - 1;
  if (z.B < 0 || z.B >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: B out of range", call);
  if (z.S < 0 || z.S >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: S out of range", call);
  if (z.T < 0 || z.T >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: T out of range", call);
  const int64_t longest = div_up(std::max(z.S, z.T), BLOCK_ROWS);
  if ((__int128)z.B * z.q_heads * longest >= 1 << 24) return op_fail(ANTDT_UNSUPPORTED, "%s: B q_heads and the longer of S and T in 128s: 2^24 or more blocks", call);
  return ANTDT_OK;
}
// Few queries for each head of the keys: by an equal share of the keys to each wavefront.
bool cross_streams(const Shape& z) { return z.S * (z.q_heads / z.heads) <= 32 && stream_fits(z.B, z.S, z.T, z.q_heads, z.heads); }
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
  a.tiles = (int)div_up(S, BLOCK_ROWS);
  return op_hip(call, by_size(dtype, (int)D, [&](auto t, auto dp) { return launch_forward<decltype(t), decltype(dp)::value>(a, B * q_heads * a.tiles, s); }));
}

int antdt_cross_attention_backward_bytes(int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_cross_attention_backward_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(cross_sizes(call, Shape{B, S, T, q_heads, heads, D, dtype}));
  *bytes = (size_t)div_up(B * S * q_heads * 4, 256) * 256;
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
  OP_TRY(cross_sizes(call, Shape{B, S, T, q_heads, heads, D, dtype}));
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
  if (queries) {
    a.tiles = (int)div_up(S, BLOCK_ROWS);
    OP_TRY(op_hip(call, by_size(dtype, (int)D, [&](auto t, auto dp) { return launch_dq<decltype(t), decltype(dp)::value>(a, B * q_heads * a.tiles, s); })));
  }
  if (keys) OP_TRY(op_hip(call, by_size(dtype, (int)D, [&](auto t, auto dp) { return launch_dkv<decltype(t), decltype(dp)::value>(a, B * heads, s); })));
  return ANTDT_OK;
}

}  // extern "C"
