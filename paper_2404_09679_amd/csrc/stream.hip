// Attention of few queries over many keys: one new token of each user over a paged cache, or a few queries over an encoded history (where there are few
// keys, by the blocks of attention.hip: cross_streams, cache_streams).
//
// Every wavefront reads an equal share of all the keys and values there are, whoever they belong to: the work is the list of 32-key tiles of all
// sequences, heads and 32s of queries, cut into equal pieces (lengths are known to the device only, and differ).  A wavefront works alone: it moves
// its tiles to LDS, several ahead, and keeps the running maximum, sum and output of a softmax over its part of a sequence.  Where a sequence lies
// in one piece, that is the result; else the pieces' are joined by a second launch:
//   m = max m_i,  l = sum l_i 2^(m_i - m),  out = sum o_i 2^(m_i - m) / l.
// Bound by memory, a key head's queries share what is read of it: one user's 131072 tokens (8 heads of 128 bf16 columns, 537 MB) 92 us (5.8 TB/s) and 5.3 to
// join; 64 users of 16 to 8192 tokens (178 MB) 39 and 5.1.  Where there is little to read, by the chain of a wavefront's loads (lengths, page, rows) and
// by its code's: one tile takes 10 us.
// Probabilities of bf16 heads are multiplied in two parts: rounded to bf16 they would take results off by 0.0025 of their norm instead of the 0.0017 of the
// results' own rounding, and the matrix cores are busy 6 % of the time (131072 tokens 92.5 -> 92.9 us, 64 users 39.1 -> 39.5).
#include "cross.h"
#include "sort.h"

namespace antdt {
namespace {

constexpr int WAVES = 4;                // of a block
constexpr int BLOCKS = 512;             // of the largest launch

// Work in tiles, [0, total), to the wavefronts: the first `more` have one more than the others.
struct Shares {
  uint32_t total, waves, each, more;
  __device__ __forceinline__ Shares(uint32_t n, uint32_t most) : total(n), waves(max(1u, min(most, n))), each(n / waves), more(n - each * waves) {}
  __device__ __forceinline__ uint32_t first(uint32_t w) const { return min(w * each + min(w, more), total); }
  __device__ __forceinline__ uint32_t owner(uint32_t tile) const {
    const uint32_t large = more * (each + 1);
    return tile < large ? tile / (each + 1) : more + (tile - large) / each;
  }
};

__device__ __forceinline__ uint32_t tiles_of(const StreamArgs& a, int64_t b) { return (uint32_t)((length_of(a.k_lengths, b, a.T) + 31) >> 5); }

// As load_lds16, not kept in the caches beyond this use.
__device__ __forceinline__ void load_lds16_once(const void* src, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"{m0}"(lds), "v"(src) : "memory");
}

// What a row that there is not is read from.
static __device__ __attribute__((aligned(16))) uint32_t zero_row[128];

// Products of R queries at a time, 32 or 16 (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32): as Core and HeadTile, with 64 / R lanes to a query
// instead of two.  Lane l has query l % R and, of 32 keys or columns, 4 GROUPS (e / 4) + 4 (l / R) + e % 4, e < R / 2.
template <typename T, int R>
struct Few;
template <typename T>
struct Few<T, 32> {
  static constexpr int STEP = Core<T>::STEP;
  typedef f32x16 Acc;
  static __device__ __forceinline__ void multiply(const typename Core<T>::Fragment& a, const typename Core<T>::Fragment& b, Acc& c) { Core<T>::multiply(a, b, c); }
};
template <>
struct Few<bf16_t, 16> {
  static constexpr int STEP = 32;
  typedef f32x4v Acc;
  static __device__ __forceinline__ void multiply(const bf16x8& a, const bf16x8& b, Acc& c) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Few<float, 16> {
  static constexpr int STEP = 16;
  typedef f32x4v Acc;
  static __device__ __forceinline__ void multiply(const f32x4v& a, const f32x4v& b, Acc& c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  }
};

template <typename T, int DP, int R>
struct Stream {
  typedef HeadTile<T, DP> Tile;
  typedef typename Core<T>::Fragment Fragment;
  static constexpr int BYTES = 32 * Tile::ROW, PIECES = BYTES / 1024, PIECE_ROWS = 64 / Tile::PITCH;
  static constexpr int STAGES = BYTES >= 8192 ? 1 : BYTES >= 4096 ? 2 : 4;
  static constexpr int PER_CU = BYTES >= 16384 ? 1 : 2;   // blocks of a compute unit
  // A wavefront's LDS: the rings of keys and of values, where a tile's rows are, the pages of the next tiles' rows.
  static constexpr int VALUES = STAGES * BYTES, WHERE = 2 * VALUES, PAGES = WHERE + 512, AHEAD = 2 * STAGES + 1;
  static constexpr int WAVE = (PAGES + AHEAD * 256 + 1023) / 1024 * 1024, LDS = WAVES * WAVE;

  // A lane's addresses for both ways of reading a tile, see HeadTile.
  static __device__ __forceinline__ uint32_t along_at(uint32_t tile, int lane) { return Tile::at(tile + Tile::slot(lane % R, lane / R) * 16); }
  static __device__ __forceinline__ uint32_t down_at(uint32_t tile, int lane) {
    if constexpr (R == 32) return Tile::down_at(tile, lane);
    if constexpr (sizeof(T) == 2) {
      const int j = lane & 15;
      return Tile::at(tile + Tile::slot(4 * (lane >> 4) + (j >> 2), (j & 3) >> 1) * 16 + (j & 1) * 8);
    } else {
      return Tile::at(tile + Tile::slot(4 * (lane >> 4), (lane & 15) >> 2) * 16 + (lane & 3) * 4);
    }
  }
  // Key r0 + lane % R (r0: 0, or 16 of R = 16), columns STEP i ..
  static __device__ __forceinline__ Fragment along(uint32_t at, int r0, int i) {
    typedef __attribute__((address_space(3))) Fragment lds_fragment;
    return *(const lds_fragment*)(uintptr_t)((at ^ (1024 / R * i)) + r0 * Tile::ROW);
  }
  // Column R d + lane % R, contraction slots (keys) i of pack().
  static __device__ __forceinline__ Fragment down(uint32_t at, int i, int d) {
    if constexpr (R == 32) return Tile::down(at, 0, i, d);
    if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      union {
        s16x4 s[2];
        Fragment v;
      } u;
#pragma unroll
      for (int s = 0; s < 2; ++s) u.s[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)((at ^ (32 * d)) + 16 * s * Tile::ROW));
      return u.v;
    } else {
      typedef __attribute__((address_space(3))) float lds_float;
      Fragment f;
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = *(const lds_float*)(uintptr_t)((at ^ (64 * d) ^ (Tile::swizzle(e) * 16)) + (16 * i + e) * Tile::ROW);
      return f;
    }
  }
};

// Over the lanes of a query.
template <int R, typename F>
__device__ __forceinline__ float over_lanes(float x, F f) {
  x = over_halves(x, f);
  if (R == 16) x = f(x, __shfl_xor(x, 16, 64));
  return x;
}

// DP columns of a row in LDS, of which the first COLS take part.  The loops that only move data stay rolled up: a launch this short waits for its code
// as well as for its data (of 34 KB, 20 us before the first tile was done).
template <typename T, int DP, int COLS, int R, bool PAGED>
__global__ __launch_bounds__(64 * WAVES, (Stream<T, DP, R>::PER_CU)) void stream_kernel(StreamArgs a) {
  typedef Stream<T, DP, R> F;
  typedef typename F::Tile Tile;
  typedef Few<T, R> C;
  typedef typename F::Fragment Fragment;
  constexpr int N = F::PIECES, S = F::STAGES, STEPS = COLS / C::STEP, DT = COLS / R, GROUPS = 64 / R, EL = R / 2, PER = R * R / 64;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = lane / R;
  const uint32_t w = blockIdx.x * WAVES + wave;
  const int64_t per = (a.B + 63) >> 6;   // sequences of a lane
  uint32_t before, total;                // tiles of the sequences before a lane's (of one head and one R of queries); of all
  {
    uint32_t n = 0;
    const int64_t b0 = min(lane * per, a.B), b1 = min(b0 + per, a.B);
    for (int64_t b = b0; b < b1; ++b) n += tiles_of(a, b);
    const uint32_t upto = wave_prefix(n);
    before = upto - n;
    total = __builtin_amdgcn_readlane(upto, 63);
    if (w == 0) {   // for the second launch
      uint32_t x = before;
      for (int64_t b = b0; b < b1; ++b) {
        a.before[b] = x;
        x += tiles_of(a, b);
      }
      if (lane == 63) a.before[a.B] = total;
    }
  }
  const uint32_t times = a.heads * a.row_tiles;
  const Shares shares(total * times, a.waves);
  // Keys and values that take more than a quarter of the last-level cache (256 MB) and are read once are not kept there: a step of answering reads those of
  // other layers before it comes back.  us, kept / not: eight caches in turn of 16 MB 8.9 / 9.0, 33 MB 12.6 / 14.0, 262 MB 54 / 47; three of 178 MB 43 / 39
  // (one alone 35 / 36); 537 MB 102 / 92.
  const bool once = a.row_tiles == 1 && (int64_t)shares.total * 2 * F::BYTES > 64 << 20;
  uint32_t at = shares.first(w);
  const uint32_t stop = shares.first(w + 1);
  if (at >= stop) return;
  const int in = __popcll(__ballot(before * times <= at)) - 1;   // the lane whose sequences `at` lies in
  int64_t b = in * per;
  uint32_t start = __builtin_amdgcn_readlane(before, in) * times, n = tiles_of(a, b);   // start: b's first tile
  char* mine = lds + wave * F::WAVE;
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_address(mine));
  const int width = a.D * (int)sizeof(T);
  if (a.D < DP) {
    for (int i = lane * 16; i < F::WHERE; i += 1024) *reinterpret_cast<uint4*>(mine + i) = make_uint4(0, 0, 0, 0);
  }

  while (at < stop) {
    while (start + n * times <= at) {   // (sequences of no keys too)
      start += n * times;
      n = tiles_of(a, ++b);
    }
    const int64_t k_len = length_of(a.k_lengths, b, a.T), q_len = length_of(a.q_lengths, b, a.S);
    const uint32_t segment = (at - start) / n, begin = start + segment * n;   // a head and its R queries
    const uint32_t h = segment / (uint32_t)a.row_tiles, rt = segment - h * a.row_tiles;
    const uint32_t i0 = at - begin, i1 = min(stop - begin, n);
    const bool came = i0 > 0, goes = i1 < n;

    const int32_t* table = PAGED ? a.table + b * a.ldt : nullptr;
    auto first_of = [&](uint32_t t) { return a.page(t); };
    // The pages of tile i's rows, to LDS.
    auto pages = [&](uint32_t i) {
      load_lds4(table + first_of((uint32_t)min((int64_t)32 * i + (lane & 31), k_len - 1)), ring + F::PAGES + (i - i0) % F::AHEAD * 256);
    };
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // (the rings are free)
    if (PAGED) {
#pragma unroll 1
      for (int j = 0; j < S; ++j) pages(i0 + j);
    }
    const uint32_t row = rt * R + lane % R, query = row / (uint32_t)a.group;
    const int64_t hq = (int64_t)h * a.group + (row - query * a.group);
    const bool there = query < q_len;   // (rows behind the last head's: query >= S)
    Fragment q[STEPS];
    {
      const char* p = reinterpret_cast<const char*>(a.q.p) + b * a.q.s.b + query * a.q.s.l + hq * a.q.s.h;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int c = (GROUPS * i + group) * 16;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (there && c < width) x = load16<false>(p + c);
        q[i] = __builtin_bit_cast(Fragment, x);
      }
    }
    // Lanes below 32 look after the rows of the keys, the others after those of the values.
    const HeadsArg& kv = lane >= 32 ? a.v : a.k;
    const char* rows = reinterpret_cast<const char*>(kv.p) + (PAGED ? 0 : b * kv.s.b) + h * kv.s.h;
    // Where tile i's rows are, to LDS; which of them there are.
    auto places = [&](uint32_t i) {
      const int64_t t = (int64_t)32 * i + (lane & 31);
      bool x = t < k_len;
      int64_t off;
      if (PAGED) {
        const int e = *reinterpret_cast<const int*>(mine + F::PAGES + (i - i0) % F::AHEAD * 256 + lane * 4);
        x = x && e >= 0 && e < a.pages;
        off = e * a.k.s.b + ((uint32_t)t - first_of((uint32_t)t) * a.page.d) * a.k.s.l;
      } else {
        off = t * kv.s.l;
      }
      *reinterpret_cast<const char**>(mine + F::WHERE + lane * 8) = x ? rows + off : reinterpret_cast<const char*>(zero_row);
      wave_lds_order();
      return (uint32_t)__ballot(x);
    };
    auto move = [&](int which, uint32_t to) {
      constexpr int U = N < 4 ? N : 4;
#pragma unroll 1
      for (int p = 0; p < N; p += U) {
        const char* src[U];
        int c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = (p + u) * F::PIECE_ROWS + lane / Tile::PITCH;
          c[u] = ((lane % Tile::PITCH) ^ Tile::swizzle(r)) * 16;
          src[u] = *reinterpret_cast<const char* const*>(mine + F::WHERE + which * 256 + r * 8);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c[u] < width) {
            if (once) load_lds16_once(src[u] + c[u], to + (p + u) * 1024);
            else load_lds16(src[u] + c[u], to + (p + u) * 1024);
          }
      }
    };
    typename C::Acc o[DT];
    float s[EL];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < PER; ++e) o[d][e] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    uint32_t some[S] = {};   // keys of the next tiles that there are
    if (PAGED) wait_loads<0>();
    // Behind a tile of keys S of values and S - 1 of keys with their pages are under way, behind one of values the other way round (fewer towards
    // the end, where everything is waited for).
    constexpr int E = PAGED ? 1 : 0;
    uint32_t slot = 0;
#pragma unroll 1
    for (int64_t i = (int64_t)i0 - S; i < i1; ++i) {
      const bool work = i >= i0, more = i + S < i1;
      if (work) {
        if (more) wait_loads<S * N + (S - 1) * (N + E)>();
        else wait_loads<0>();
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t tk = F::along_at(ring + slot, lane);
#pragma unroll
        for (int t = 0; t < 32 / R; ++t) {
          typename C::Acc x;
#pragma unroll
          for (int e = 0; e < PER; ++e) x[e] = 0.0f;
#pragma unroll
          for (int j = 0; j < STEPS; ++j) C::multiply(F::along(tk, R * t, j), q[j], x);
#pragma unroll
          for (int e = 0; e < PER; ++e) s[PER * t + e] = x[e];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
      const uint32_t now_some = some[0];
#pragma unroll
      for (int j = 0; j + 1 < S; ++j) some[j] = some[j + 1];
      if (more) {
        if (PAGED) pages((uint32_t)(i + 2 * S));
        some[S - 1] = places((uint32_t)(i + S));
        move(0, ring + slot);
      }
      if (work) {
        if (now_some != ~0u) {
#pragma unroll
          for (int e = 0; e < EL; ++e)
            if (!(now_some >> (4 * GROUPS * (e >> 2) + 4 * group + (e & 3)) & 1)) s[e] = -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int e = 1; e < EL; ++e) top = fmaxf(top, s[e]);
        top = over_lanes<R>(top, [](float x, float y) { return fmaxf(x, y); });
        if (__any(top > m && (top - m) * a.scale2 > 8.0f)) {   // (else sums stay under the older maximum)
          const float now = fmaxf(m, top), f = m == -INFINITY ? 0.0f : exp2_((m - now) * a.scale2);
          m = now;
          l *= f;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < PER; ++e) o[d][e] *= f;
        }
        const float mc = m == -INFINITY ? 0.0f : m * a.scale2;
#pragma unroll
        for (int e = 0; e < EL; ++e) {
          s[e] = exp2_(fmaf(s[e], a.scale2, -mc));
          l += s[e];
        }
        if (more) wait_loads<S * (N + E) + (S - 1) * N>();
        else wait_loads<0>();
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t tv = F::down_at(ring + F::VALUES + slot, lane);
#pragma unroll
        for (int j = 0; j < EL / Core<T>::PER; ++j) {
          Fragment p[Core<T>::PARTS];
          Core<T>::pack(s, j, p);
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const Fragment x = F::down(tv, j, d);
#pragma unroll
            for (const Fragment& part : p) C::multiply(x, part, o[d]);
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
      if (more) move(1, ring + F::VALUES + slot);
      slot = slot == (S - 1) * F::BYTES ? 0 : slot + F::BYTES;
    }
    l = over_lanes<R>(l, [](float x, float y) { return x + y; });
    const float top2 = m == -INFINITY ? 0.0f : m * a.scale2;
    const bool part = came || goes;
    const int64_t at_part = ((int64_t)w * 2 + (came ? 0 : 1)) * a.rows + lane % R;
    const bool stored = part ? lane % R < a.rows : query < a.S;
    if (part && stored && group == 0) *reinterpret_cast<float2*>(a.top_sum + 2 * at_part) = make_float2(m == -INFINITY ? -INFINITY : top2, l);
    if (!part && stored && group == 0 && a.stats) a.stats[(b * a.q_heads + hq) * a.S + query] = m == -INFINITY || !there ? INFINITY : top2 + log2_(l);
    const float f = part ? 1.0f : m == -INFINITY ? 0.0f : 1.0f / l;   // (a largest score beyond fp32: l is 0 or infinite, and NaN comes out)
    float* to_part = a.partial + at_part * DP;
    T* to = reinterpret_cast<T*>(reinterpret_cast<char*>(const_cast<void*>(a.out.p)) + b * a.out.s.b + query * a.out.s.l + hq * a.out.s.h);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int v = 0; v < PER / 4; ++v) {
        const int c = R * d + 4 * GROUPS * v + 4 * group;
        float4 x = make_float4(o[d][4 * v] * f, o[d][4 * v + 1] * f, o[d][4 * v + 2] * f, o[d][4 * v + 3] * f);
        if (!there) x = make_float4(0, 0, 0, 0);
        if (!stored || c >= a.D) continue;
        if (part) *reinterpret_cast<float4*>(to_part + c) = x;
        else if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to + c) = x;
        else *reinterpret_cast<uint2*>(to + c) = make_uint2(f2bf2(x.x, x.y), f2bf2(x.z, x.w));
      }
    at = begin + i1;
  }
}

// One query of one head to a block: its parts, THREADS / (DP / 4) of them at a time, each thread's in the order of the wavefronts.
constexpr int64_t ROWS_OF_A_JOIN = 1 << 22;   // (2^32 threads are the most)
template <typename T, int DP, int THREADS>
__global__ __launch_bounds__(THREADS) void stream_join_kernel(StreamArgs a) {
  constexpr int LANES = DP / 4, GROUPS = THREADS / LANES;
  __shared__ float4 sums[GROUPS][LANES];
  __shared__ float2 parts[GROUPS];   // maximum and sum
  const uint32_t id = a.first + blockIdx.x, bh = id / (uint32_t)a.S, query = id - bh * (uint32_t)a.S;   // (below 2^31)
  const uint32_t b = bh / (uint32_t)a.q_heads, hq = bh - b * (uint32_t)a.q_heads, h = hq / (uint32_t)a.group, row = query * a.group + hq - h * a.group;
  const uint32_t n = a.before[b + 1] - a.before[b], times = a.heads * a.row_tiles;
  const bool there = n > 0 && query < length_of(a.q_lengths, b, a.S);
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  float4 sum = make_float4(0, 0, 0, 0);
  float l = 0.0f, top = -INFINITY;
  if (there) {
    const Shares shares(a.before[a.B] * times, a.waves);
    const uint32_t begin = a.before[b] * times + (h * a.row_tiles + row / a.row_tile) * n;
    const int w0 = (int)shares.owner(begin), w1 = (int)shares.owner(begin + n - 1);
    if (w0 == w1) return;   // (written by that wavefront)
    auto slot = [&](int w) { return (int64_t)(w * 2 + (w == w0 ? 1 : 0)) * a.rows + row % a.row_tile; };
#pragma unroll 4
    for (int w = w0 + group; w <= w1; w += GROUPS) {   // (one pass: nothing waits for the maximum of all)
      const float2 ml = *reinterpret_cast<const float2*>(a.top_sum + 2 * slot(w));
      const float4 x = *reinterpret_cast<const float4*>(a.partial + slot(w) * DP + 4 * lane);
      const float now = fmaxf(top, ml.x), base = now == -INFINITY ? 0.0f : now, f = exp2_(top - base), g = exp2_(ml.x - base);
      top = now;
      l = l * f + ml.y * g;
      sum.x = sum.x * f + x.x * g; sum.y = sum.y * f + x.y * g; sum.z = sum.z * f + x.z * g; sum.w = sum.w * f + x.w * g;
    }
  }
  sums[group][lane] = sum;
  if (lane == 0) parts[group] = make_float2(top, l);
  __syncthreads();
  if (group > 0) return;
  l = 0.0f;
  sum = make_float4(0, 0, 0, 0);
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) top = fmaxf(top, parts[g].x);
  const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    const float f = exp2_(parts[g].x - base);
    const float4 x = sums[g][lane];
    l += parts[g].y * f;
    sum.x += x.x * f; sum.y += x.y * f; sum.z += x.z * f; sum.w += x.w * f;
  }
  const float f = top == -INFINITY ? 0.0f : 1.0f / l;
  if (4 * lane < a.D) {
    char* to = reinterpret_cast<char*>(const_cast<void*>(a.out.p)) + b * a.out.s.b + query * a.out.s.l + hq * a.out.s.h;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to + 16 * lane) = make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f);
    else *reinterpret_cast<uint2*>(to + 8 * lane) = make_uint2(f2bf2(sum.x * f, sum.y * f), f2bf2(sum.z * f, sum.w * f));
  }
  if (a.stats && lane == 0) a.stats[(int64_t)bh * a.S + query] = top == -INFINITY ? INFINITY : top + log2_(l);
}

struct StreamPlan {
  int64_t before, top_sum, partial, bytes;
  int32_t row_tile, rows, row_tiles;
};
StreamPlan stream_plan(int64_t B, int64_t S, int64_t q_heads, int64_t heads, int64_t D) {
  StreamPlan p;
  const int64_t all = S * (q_heads / heads), dp = D <= 32 ? 32 : D <= 64 ? 64 : 128;
  p.row_tile = all <= 16 ? 16 : 32;
  p.row_tiles = (int)div_up(all, p.row_tile);
  p.rows = (int)std::min<int64_t>(all, p.row_tile);
  auto room = [](int64_t n) { return div_up(n, 256) * 256; };
  p.before = 0;
  p.top_sum = room((B + 1) * 4);
  p.partial = p.top_sum + room((int64_t)BLOCKS * WAVES * 2 * p.rows * 8);
  p.bytes = p.partial + (int64_t)BLOCKS * WAVES * 2 * p.rows * dp * 4;
  return p;
}

template <typename T, int DP, int COLS, int R, bool PAGED>
hipError_t launch(StreamArgs a, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  typedef Stream<T, DP, R> F;
  a.waves = 256 * F::PER_CU * WAVES;
  const hipError_t e = allow_lds(stream_kernel<T, DP, COLS, R, PAGED>, F::LDS, 0, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((stream_kernel<T, DP, COLS, R, PAGED>), dim3(a.waves / WAVES), dim3(64 * WAVES), F::LDS, s, a);
  // (few sequences and heads: many parts each.  One user's 131072 tokens, 8 heads, us of 128 / 512 threads: 11.1 / 6.4; 64 users, 4 heads 5.1 / 6.1)
  const int64_t n = a.B * a.S * a.q_heads;   // (below 2^31: 128 queries to a block of the other way, whose blocks are below 2^24)
  const bool few = a.B * a.heads * a.row_tiles <= 64;
  for (int64_t first = 0; first < n; first += ROWS_OF_A_JOIN) {
    a.first = (uint32_t)first;
    const dim3 rows((unsigned)std::min(n - first, ROWS_OF_A_JOIN));
    if (few) hipLaunchKernelGGL((stream_join_kernel<T, DP, 512>), rows, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((stream_join_kernel<T, DP, 128>), rows, dim3(128), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

bool stream_fits(int64_t B, int64_t S, int64_t T, int64_t q_heads, int64_t heads) {
  return (__int128)B * heads * div_up(S * (q_heads / heads), 16) * div_up(T, 32) < 1ll << 31;
}
size_t stream_bytes(int64_t B, int64_t S, int64_t q_heads, int64_t heads, int64_t D) { return (size_t)stream_plan(B, S, q_heads, heads, D).bytes; }

hipError_t launch_stream(StreamArgs a, int32_t dtype, void* workspace, hipStream_t s) {
  const StreamPlan p = stream_plan(a.B, a.S, a.q_heads, a.heads, a.D);
  char* ws = reinterpret_cast<char*>(workspace);
  a.row_tile = p.row_tile; a.row_tiles = p.row_tiles; a.rows = p.rows;
  a.before = reinterpret_cast<uint32_t*>(ws + p.before);
  a.top_sum = reinterpret_cast<float*>(ws + p.top_sum);
  a.partial = reinterpret_cast<float*>(ws + p.partial);
  return by_size(dtype, a.D, [&](auto t, auto dp) {
    typedef decltype(t) T;
    constexpr int DP = decltype(dp)::value;
    auto go = [&](auto cols, auto r) {
      constexpr int COLS = decltype(cols)::value, R = decltype(r)::value;
      return a.table ? launch<T, DP, COLS, R, true>(a, s) : launch<T, DP, COLS, R, false>(a, s);
    };
    auto rows = [&](auto cols) { return a.row_tile == 16 ? go(cols, std::integral_constant<int, 16>()) : go(cols, std::integral_constant<int, 32>()); };
    if constexpr (DP == 128) {
      if (a.D <= 96) return rows(std::integral_constant<int, 96>());
    }
    return rows(std::integral_constant<int, DP>());
  });
}

}  // namespace antdt

using namespace antdt;

extern "C" {

static int cache_attention_sizes(const char* call, int64_t B, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype) {
  OP_TRY(op_head_sizes(call, q_heads, heads, D, dtype));
  if (B < 0 || B >= 1 << 24 || B * q_heads >= 1 << 24) return op_fail(ANTDT_UNSUPPORTED, "%s: B q_heads: 2^24 or more", call);
  return ANTDT_OK;
}

int antdt_cache_attention_bytes(int64_t B, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, size_t* bytes) {
  const char* call = "antdt_cache_attention_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(cache_attention_sizes(call, B, q_heads, heads, D, dtype));
  *bytes = B == 0 ? 0 : stream_bytes(B, 1, q_heads, heads, D);
  return ANTDT_OK;
}

int antdt_cache_attention(const void* q, int64_t ldq, int64_t ldq_head, const void* k_cache, const void* v_cache, int64_t ld_page, int64_t ld_row,
                          int64_t ld_head, int64_t pages, int64_t page_size, const int32_t* table, int64_t ld_table, int64_t B, int64_t table_cols,
                          const int32_t* lengths, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype, float scale, void* out, int64_t ldo,
                          int64_t ldo_head, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "antdt_cache_attention";
  OP_TRY(cache_attention_sizes(call, B, q_heads, heads, D, dtype));
  OP_TRY(op_scale(call, scale));
  if (page_size < 1 || page_size >= (1ll << 31)) return op_fail(ANTDT_INVALID_ARG, "%s: page_size out of range", call);
  if (pages < 0 || pages >= (1ll << 31)) return op_fail(ANTDT_INVALID_ARG, "%s: pages out of range", call);
  if (table_cols < 0 || table_cols >= (1ll << 31)) return op_fail(ANTDT_INVALID_ARG, "%s: table_cols out of range", call);
  StreamArgs a = {};
  OP_TRY(op_wide_heads(call, "q", q, B, 1, q_heads, D, dtype, {ldq, 0, ldq_head}, false, a.q));
  OP_TRY(op_wide_heads(call, "k_cache", k_cache, pages, page_size, heads, D, dtype, {ld_page, ld_row, ld_head}, false, a.k));
  OP_TRY(op_wide_heads(call, "v_cache", v_cache, pages, page_size, heads, D, dtype, {ld_page, ld_row, ld_head}, false, a.v));
  OP_TRY(op_wide_heads(call, "out", out, B, 1, q_heads, D, dtype, {ldo, 0, ldo_head}, true, a.out));
  OP_TRY(op_matrix(call, "table", table, B, table_cols, ld_table, 4));
  OP_TRY(op_matrix(call, "lengths", lengths, B, 1, 1, 4));
  if (B == 0) return ANTDT_OK;
  OP_TRY(op_workspace(call, workspace, workspace_bytes, stream_bytes(B, 1, q_heads, heads, D)));
  const Shape z = cache_shape(B, std::min<int64_t>(table_cols * page_size, (1ll << 31) - 1), q_heads, heads, D, dtype);
  if (!stream_fits(B, 1, z.T, q_heads, heads)) return op_fail(ANTDT_UNSUPPORTED, "%s: B heads table_cols page_size / 32: 2^31 or more", call);
  if (!cache_streams(z, page_size)) {
    CrossArgs f = {};
    f.q = {a.q.p, {a.q.s.b, a.q.s.h, a.q.s.h * (q_heads / heads)}};
    f.out = {a.out.p, {a.out.s.b, a.out.s.h, a.out.s.h * (q_heads / heads)}};
    f.k = a.k; f.v = a.v; f.k_lengths = lengths; f.S = z.S; f.T = z.T; f.B = (int)B;
    f.q_heads = f.heads = (int)heads; f.group = 1; f.D = (int)D; f.units = (int)(B * heads); f.scale = scale; f.scale2 = scale * LOG2E;
    f.table = table; f.ldt = ld_table; f.pages = pages; f.page = Divisor::of((uint32_t)page_size);
    return op_hip(call, launch_cache_blocks(f, z, (hipStream_t)stream));
  }
  static const int32_t none = 0;
  a.table = table_cols > 0 ? table : &none;   // (without columns no length is above 0, and nothing reads it)
  a.ldt = ld_table; a.pages = pages; a.k_lengths = lengths; a.B = B; a.S = 1;
  a.T = z.T;
  a.page = Divisor::of((uint32_t)page_size);
  a.q_heads = (int)q_heads; a.heads = (int)heads; a.group = (int)(q_heads / heads); a.D = (int)D; a.scale2 = scale * LOG2E;
  return op_hip(call, launch_stream(a, dtype, workspace, (hipStream_t)stream));
}

}  // extern "C"
