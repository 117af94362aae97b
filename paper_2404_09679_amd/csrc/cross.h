// Attention of queries over keys and values of another length, and its backward pass.
//
// With scores z = scale q k^T over the keys that there are, p = softmax(z), out = p v.  Forward: one pass over the keys with the running maximum m and
// sum l of a row's softmax; a sum of values under an older maximum is scaled by 2^(old - new).  Kept for the backward pass: L = log2 of the sum of
// 2^(z log2 e), so that p = 2^(z log2 e - L) again.  With g the gradient of out and d = sum of g out over a row's columns:
//   dP = g v^T,  dZ = p (dP - d),  dQ = scale dZ k,  dK = scale dZ^T q,  dV = p^T g,
// dQ in blocks of queries and dK, dV in blocks of keys: each forms p and dP anew (14 products for the 10 there are), and every sum has one order.
// Of bf16 heads p and dZ are rounded to bf16 as the matrix cores' operands (results off by 0.0025 of their norm, of which their own rounding is 0.0017):
// in two parts, as over a cache, they would take more products, which bound these kernels (8 ragged histories of 2048 queries and 4096 keys, 16 and 4 heads of
// 128 columns: forward 427 -> 547 us, gradients 1310 -> 1690; 13 of 77 and 777, 6 and 2 heads of 64: 11 -> 12 and 17 -> 20; blocks of 32 alone 1 to 14 %).
#pragma once

#include "attend.h"

namespace antdt {

// How rows of results are shared out: `tiles` blocks of rows to a head, each by `parts` blocks, whose sums go through
// partial [parts, heads, rows, D] (of keys and values [parts, 2, ...]).
struct Share {
  int32_t tiles, parts, blocks;
  float* partial;
};
struct CrossArgs {
  HeadsArg q, k, v, out, dout, dq, dk, dv;
  const int32_t* q_lengths;
  const int32_t* k_lengths;
  float* stats;        // L [B, q_heads, S], +infinity for a row without keys: its p come out 0
  float* delta;        // d, the same shape
  int64_t S, T;
  int32_t q_heads, heads, group, D;
  int32_t units;       // heads of all batch entries' keys
  int32_t B;
  int32_t longest_first;   // whether batch entries are gone through by length, see entry_of
  float scale, scale2;   // scale2: scale log2 e
  Share queries, keys;   // blocks of queries, and (backward) of keys
  // Of a cache, whose keys and values are [pages, page, heads, D]:
  const int32_t* table;
  int64_t ldt, pages;
  Divisor page;
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
// sequences is everybody's work.  What is left of less than 8 units is spread over all.  Longest first, the longer ones of 8 go to one half of the XCDs
// and to the other in turn.
__device__ __forceinline__ void place_of(const CrossArgs& a, int i, int n, int& unit, int& block) {
  const int units = a.units, whole = (units & ~7) * n;
  const int x = i < whole ? i & 7 : 0, j = i < whole ? i >> 3 : i - whole;
  const int u = j / n;
  block = j - u * n;
  unit = i < whole ? 8 * u + (a.longest_first ? x ^ (4 * (u & 1)) : x) : (units & ~7) + u;
}

// A batch entry and the rows it has.
struct Entry {
  int64_t b, q_len, k_len;
};
// Entry in place i when those of most keys come first (of as many those of most queries), so that the last blocks are short ones: of each 16 entries, one in
// each lane, by counting.
// Forward / backward in us, of 128 bf16 columns, in the order given and so: 32 entries of 1 to 1024 queries and keys, 8 heads 72 / 191, 63 / 182; 8 of 1366
// to 2048 queries and 2560 to 4096 keys, 16 and 4 heads, in four orders 430-480 / 1311-1463, 435-439 / 1333-1341.
__device__ __forceinline__ Entry entry_of(const CrossArgs& a, int64_t i, int lane) {
  if (!a.longest_first) return Entry{i, length_of(a.q_lengths, i, a.S), length_of(a.k_lengths, i, a.T)};
  const int64_t first = i & ~15ll, mine = min(first + (lane & 15), (int64_t)a.B - 1);
  const int q = (int)length_of(a.q_lengths, mine, a.S), k = (int)length_of(a.k_lengths, mine, a.T);
  const bool there = first + lane < a.B;
  const uint32_t high = there ? k : 0, low = (there ? min(q, (1 << 27) - 1) : 0) << 4 | (15 - (lane & 15));   // (no two alike, and behind the last entry less)
  const uint64_t key = (uint64_t)high << 32 | low;
  int before = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j)
    before += ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, j)) > key ? 1 : 0;
  const int at = __ffsll((unsigned long long)__ballot(before == (int)(i - first))) - 1;
  return Entry{first + at, __builtin_amdgcn_readlane(q, at), __builtin_amdgcn_readlane(k, at)};
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
// Zeros to rows [r0, r1) of a head, by a block of that many threads.
template <typename T>
__device__ __forceinline__ void clear_rows(const Rows& to, int64_t r0, int64_t r1, int D, int threads) {
  const int per = D / Core<T>::PER;
  for (int64_t i = threadIdx.x; i < (r1 - r0) * per; i += threads)
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

// Tiles of keys and values go through LDS.
template <typename W>
struct KeyTiles {
  static constexpr int STAGE = 2 * W::Load::BYTES, RING = W::STAGES * STAGE, ALL = W::SPLIT ? W::WAVES * RING : RING, LDS = W::lds(ALL);
  typedef antdt::Ring<W::STAGES, 2 * W::Load::PIECES, STAGE, !W::SPLIT> Ring;
};
// ------------------------------------------------------------- which way
template <typename T, int DP>
struct Ways {
  static constexpr int ROW = DP * sizeof(T);   // bytes
  static constexpr bool HELD = !(sizeof(T) == 2 && DP == 128);   // (see QueryTiles; nor are there registers for fragments ahead)
  template <int COLS> using Keys = Way<T, DP, COLS, ROW == 512 ? 32 : 64, 2, 4, false, 2, 4>;
  template <int COLS> using KeysDq = Way<T, DP, COLS, ROW == 512 ? 32 : 64, 2, 4, false, ROW == 512 ? 1 : 2, 4>;
  template <int COLS> using Queries = Way<T, DP, COLS, ROW >= 256 ? 32 : 64, 2, 4, false, ROW == 512 ? 1 : 2, HELD ? 4 : 1>;
  template <int COLS> using SplitKeys = Way<T, DP, COLS, 32, 2, ROW == 512 ? 2 : 4, true, ROW >= 256 ? 1 : 2, 4>;
  template <int COLS> using SplitQueries = Way<T, DP, COLS, 32, 2, ROW == 512 ? 2 : 4, true, ROW >= 256 ? 1 : 2, 4>;
};
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

struct Plan {
  bool split;
  int32_t tiles, parts;
  int64_t blocks;
  Share share(float* partial) const { return Share{tiles, parts, (int32_t)blocks, partial}; }
};
struct Shape {
  int64_t B, S, T, q_heads, heads, D;
  int32_t dtype;
};
// Microseconds that a wavefront takes for 32 queries and 32 keys in the forward pass, alone on its SIMD (measured; of a multiple of 32 columns).
inline double tile_us(const Shape& z) {
  const int columns = (int)div_up(z.D, 32) - 1;
  constexpr double BF16[] = {0.53, 0.71, 1.10, 1.22}, F32[] = {1.53, 2.88, 4.12, 4.90};
  return z.dtype == ANTDT_F32 ? F32[columns] : BF16[columns];
}
// Results' rows in blocks of 128, or of 32 whose `waves` wavefronts share the other side's rows (`tiles` of 32), or these again in parts.
//  - Blocks of 32 as long as there are no more than `most`: all of them run at once, of fp32 heads above 32 columns in two rounds.  bf16, 1024 queries and
//    keys, 64 columns, us of blocks of 128 / 32: 16 heads 20 / 15, 32 heads 22 / 26; gradient of the queries 24 / 16, 26 / 30; 128 columns, gradient of the
//    keys: 16 heads 60 / 46, 32 heads 63 / 89.  Two rounds of fp32, 512 blocks, 1000 rows of the other side, gradients of queries and of keys: 64 columns, 16
//    heads of 1024 rows 108 / 74 and 153 / 94; 128 columns 224 / 247 and 287 / 306, but 500 heads of 20 rows 466 / 271 and 746 / 495.
//  - Parts where their shorter way outweighs the launch that adds them up, about 6 us.
inline Plan cross_plan(int64_t heads, int64_t rows, int64_t tiles, int64_t most, int waves, double us, bool parted, int64_t least = 2) {
  Plan p = {false, (int32_t)div_up(rows, 128), 1, 0};
  p.blocks = heads * p.tiles;
  const int64_t split = heads * div_up(rows, 32);
  if (split == 0 || split > most || tiles < least) return p;
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
inline int64_t delta_bytes(const Shape& z) { return div_up(z.B * z.S * z.q_heads * 4, 256) * 256; }
inline bool wide(const Shape& z) { return z.dtype == ANTDT_BF16 && z.D > 64; }          // (a block of 32 fills a compute unit's LDS)
inline int at_once(const Shape& z) { return z.D > (z.dtype == ANTDT_BF16 ? 64 : 32) ? 256 : 512; }   // blocks of 32
inline int key_waves(const Shape& z) { return z.dtype == ANTDT_F32 && z.D > 64 ? 2 : 4; }
inline Plan forward_plan(const Shape& z) { return cross_plan(z.B * z.q_heads, z.S, div_up(z.T, 32), wide(z) ? 256 : 512, key_waves(z), tile_us(z), false); }
inline Plan dq_plan(const Shape& z) { return cross_plan(z.B * z.q_heads, z.S, div_up(z.T, 32), wide(z) ? 256 : 512, key_waves(z), 1.6 * tile_us(z), true); }
inline Plan dkv_plan(const Shape& z) { return cross_plan(z.B * z.heads, z.T, div_up(z.S, 32) * (z.q_heads / z.heads), wide(z) ? 256 : 512, key_waves(z), 2.6 * tile_us(z), true); }
// Whether entries are gone through by length: costs a block about a microsecond and shortens the end by some of the longest block's time
// (200 entries of 1 to 300, 8 and 2 heads of 64: 41 / 105 us, by length 43 / 116).
inline bool longest_first(const Shape& z, bool ragged, int64_t blocks, int at_once) {
  const double rounds = (double)blocks / at_once;
  return ragged && z.B > 1 && rounds > 1.0 && tile_us(z) * div_up(std::max(z.S, z.T), 32) > 3.0 * rounds;
}
// Whether an equal share of all keys to each wavefront (stream.hip) takes less time than the forward pass's blocks: it has a second launch, `fixed` us in all
// (and in fp32 0.9 for 1000 rows), and tiles that nobody else reads, each `share` times tile_us on one of 1024 SIMDs; a block's take `own` times that, in as
// many rounds as there are.  Two rounds of fp32, us by blocks / shares: 70 users' caches, 4 heads of 64 columns, 200 and 500 tokens 21 / 14, 40 / 24; 128 users of
// 128 columns, 100 tokens 35 / 23; 300 keys of 64 columns, 260 heads of 2 queries 28 / 18; of 128 columns, 16 heads of 1024 queries, 100 and 1000 keys 31 / 43,
// 167 / 134.
inline bool by_shares(const Shape& z, const Plan& p, double fixed, double share, double own) {
  if (z.B == 0 || z.S == 0 || !stream_fits(z.B, z.S, z.T, z.q_heads, z.heads)) return false;
  const int64_t tiles = div_up(z.T, 32), rows = z.S * (z.q_heads / z.heads), row_tiles = rows <= 16 ? 1 : div_up(rows, 32);
  const double blocks = p.split ? div_up(tiles, key_waves(z)) * (p.blocks < 128 ? 1.0 : 1.25) * div_up(p.blocks, at_once(z)) : std::max(1.0, p.blocks / 512.0) * tiles;
  const double shares = (double)z.B * z.heads * row_tiles * tiles / 1024;
  const double joined = z.dtype == ANTDT_F32 ? 0.0009 * z.B * z.S * z.q_heads : 0.0;
  return fixed + joined + tile_us(z) * share * shares < 4.5 + tile_us(z) * own * blocks;
}
// us by blocks / shares of 500, 2000 and 8000 keys, 8 heads: 64 bf16 columns, 1 query 7 / 18, 16 / 17, 49 / 21; 4 x 128 queries 8 / 21, 17 / 27, 61 / 55; 128
// columns 10 / 17, 25 / 17, 84 / 22 and 12 / 25, 29 / 41, 96 / 97; 64 fp32 columns 16 / 18, 49 / 16, 184 / 17 and 17 / 26, 55 / 46, 195 / 114.
inline bool cross_streams(const Shape& z) { return by_shares(z, forward_plan(z), 16.0, z.dtype == ANTDT_F32 ? 1.3 : 2.0, 1.0); }
// The same for one token of each user over a cache of room for T: the tokens of a key's heads are one block's rows, which looks up the user's pages once.
// us of 100, 500, 1000 and 2000 tokens in pages of 16: 16 users, 16 and 4 heads of 64 bf16 columns 5.5 / 16, 9 / 16, 13 / 17, 23 / 17; 64 users of 128
// columns 8 / 15, 17 / 20, 28 / 29, 49 / 50; fp32, 64 users of 64 columns 8 / 17, 23 / 21, 40 / 30, 72 / 52.
constexpr int TABLE = 2048;   // pages of a user, at most
inline Shape cache_shape(int64_t B, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype) {
  return Shape{B, q_heads / heads, T, heads, heads, D, dtype};
}
// Blocks of 32 for a single tile, too, where all of them run at once (us by shares / blocks of 20 tokens: 16 users, 16 and 4 heads of 64 bf16 columns 7.7 / 5.0, fp32
// 8.8 / 7.3; 200 users, 8 and 2 heads of 64 fp32 columns, two rounds, 10.0 / 13.2).  Many rounds read less evenly: 4096 users of 100 tokens, 8 heads of 64 bf16
// columns 215 / 309, of 128 344 / 731, fp32 391 / 836; but one head of 64 bf16 columns 79 / 41, where most of the shares' time goes into the users' lengths.
inline Plan cache_plan(const Shape& z) {
  const int most = z.T <= 32 ? at_once(z) : wide(z) ? 256 : 512;
  return cross_plan(z.B * z.q_heads, z.S, div_up(z.T, 32), most, key_waves(z), tile_us(z), false, 1);
}
inline bool cache_streams(const Shape& z, int64_t page) {
  const Plan p = cache_plan(z);
  return !p.split || div_up(z.T, page) > TABLE || by_shares(z, p, 15.0, z.dtype == ANTDT_F32 ? 1.0 : 1.5, 1.5);
}
hipError_t launch_cache_blocks(const CrossArgs& a, const Shape& z, hipStream_t s);

inline int cross_sizes(const char* call, const Shape& z) {
  OP_TRY(op_head_sizes(call, z.q_heads, z.heads, z.D, z.dtype));
  constexpr int64_t MOST = (1ll << 31) - 1;
  if (z.B < 0 || z.B >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: B out of range", call);
  if (z.S < 0 || z.S >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: S out of range", call);
  if (z.T < 0 || z.T >= MOST) return op_fail(ANTDT_INVALID_ARG, "%s: T out of range", call);
  const int64_t longest = div_up(std::max(z.S, z.T), 128);
  if ((__int128)z.B * z.q_heads * longest >= 1 << 24) return op_fail(ANTDT_UNSUPPORTED, "%s: B q_heads and the longer of S and T in 128s: 2^24 or more blocks", call);
  return ANTDT_OK;
}
inline int cross_lengths(const char* call, const int32_t* q_lengths, const int32_t* k_lengths) {
  if ((reinterpret_cast<uintptr_t>(q_lengths) | reinterpret_cast<uintptr_t>(k_lengths)) & 3) return op_fail(ANTDT_INVALID_ARG, "%s: lengths are misaligned", call);
  return ANTDT_OK;
}
}  // namespace antdt
