// Attention of few queries over many keys: one new token of each user over a paged cache, or a few queries over an encoded history.
//
// Every wavefront reads an equal share of all the keys and values there are, whoever they belong to: the work is the list of 32-key tiles of all
// sequences, heads and 32s of queries, cut into equal pieces (lengths are known to the device only, and differ).  A wavefront works alone: it moves
// its tiles to LDS, several ahead, and keeps the running maximum, sum and output of a softmax over its part of a sequence.  Where a sequence lies
// in one piece, that is the result; else the pieces' are joined by a second launch:
//   m = max m_i,  l = sum l_i 2^(m_i - m),  out = sum o_i 2^(m_i - m) / l.
// Bound by memory: a key head's queries share what is read of it.
#include "attend.h"

namespace antdt {
namespace {

constexpr int WAVES = 4;                // of a block
constexpr int BLOCKS = 256;             // one to a compute unit
constexpr int LEAST = 4;                // tiles of a wavefront, before the next one gets some

// Work in tiles: [0, total) in `waves` pieces.
struct Pieces {
  int64_t total, waves;
  __device__ __forceinline__ Pieces(int64_t n, int most) : total(n), waves(max((int64_t)1, min((int64_t)most, (n + LEAST - 1) / LEAST))) {}
  __device__ __forceinline__ int64_t first(int64_t w) const { return w >= waves ? total : w * total / waves; }
  __device__ __forceinline__ int64_t owner(int64_t tile) const { return ((tile + 1) * waves - 1) / total; }
};

__device__ __forceinline__ int64_t tiles_of(const StreamArgs& a, int64_t b) { return (length_of(a.k_lengths, b, a.T) + 31) >> 5; }

template <typename T, int DP>
struct Stream {
  typedef HeadTile<T, DP> Tile;
  static constexpr int BYTES = 32 * Tile::ROW, PIECES = BYTES / 1024;
  static constexpr int STAGES = BYTES >= 16384 ? 1 : BYTES >= 8192 ? 2 : 4;
  static constexpr int ENTRIES = 2 * STAGES + 1, WAVE = (2 * STAGES * BYTES + ENTRIES * 256 + 1023) / 1024 * 1024, LDS = WAVES * WAVE;
};

template <typename T, int DP, bool PAGED>
__global__ __launch_bounds__(64 * WAVES, 1) void stream_kernel(StreamArgs a) {
  typedef Stream<T, DP> F;
  typedef typename F::Tile Tile;
  typedef Core<T> C;
  constexpr int N = F::PIECES, S = F::STAGES;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  __shared__ int64_t upto[64 * WAVES + 1];   // tiles of the sequences before a thread's
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int64_t per = (a.B + 64 * WAVES - 1) / (64 * WAVES);   // sequences of a thread
  {
    int64_t n = 0;
    const int64_t b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
    for (int64_t b = b0; b < b1; ++b) n += tiles_of(a, b);
    upto[tid + 1] = n;
    if (tid == 0) upto[0] = 0;
    __syncthreads();
    for (int step = 1; step < 64 * WAVES; step <<= 1) {
      const int64_t x = tid + 1 > step ? upto[tid + 1 - step] : 0;
      __syncthreads();
      upto[tid + 1] += x;
      __syncthreads();
    }
    if (blockIdx.x == 0) {
      int64_t at = upto[tid];
      for (int64_t b = b0; b < b1; ++b) {
        a.before[b] = at;
        at += tiles_of(a, b);
      }
      if (tid == 0) a.before[a.B] = upto[64 * WAVES];
    }
  }
  const int64_t w = (int64_t)blockIdx.x * WAVES + wave;
  const int64_t times = (int64_t)a.heads * a.row_tiles;
  const Pieces pieces(upto[64 * WAVES] * times, a.waves);
  int64_t at = pieces.first(w);
  const int64_t stop = pieces.first(w + 1);
  if (at >= stop) return;
  // the sequence that `at` lies in
  int64_t b = 0, start = 0;   // start: its first tile
  {
    int lo = 0, hi = 64 * WAVES;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (upto[mid] * times <= at) lo = mid;
      else hi = mid;
    }
    b = lo * per;
    start = upto[lo] * times;
  }
  int64_t n = tiles_of(a, b);
  while (start + n * times <= at) {
    start += n * times;
    n = tiles_of(a, ++b);
  }
  char* mine = lds + wave * F::WAVE;
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_address(mine)), entries = ring + 2 * S * F::BYTES;
  const int width = a.D * (int)sizeof(T);
  if (a.D < DP)
    for (int i = lane * 16; i < 2 * S * F::BYTES; i += 1024) *reinterpret_cast<uint4*>(mine + i) = make_uint4(0, 0, 0, 0);

  while (at < stop) {
    while (start + n * times <= at) {   // (sequences of no keys too)
      start += n * times;
      n = tiles_of(a, ++b);
    }
    const int64_t k_len = length_of(a.k_lengths, b, a.T), q_len = length_of(a.q_lengths, b, a.S);
    const int64_t segment = (at - start) / n, begin = start + segment * n;   // a head and its 32 queries
    const int h = (int)(segment / a.row_tiles), rt = (int)(segment % a.row_tiles);
    const int64_t i0 = at - begin, i1 = min(stop - begin, n);
    const bool came = i0 > 0, goes = i1 < n;

    const int64_t row = (int64_t)rt * 32 + (lane & 31), query = row / a.group;
    const int64_t hq = (int64_t)h * a.group + (row - query * a.group);
    const bool there = query < q_len;   // (rows behind the last head's: query >= S)
    typename C::Fragment q[DP / C::STEP];
    {
      const char* p = reinterpret_cast<const char*>(a.q.p) + b * a.q.s.b + query * a.q.s.l + hq * a.q.s.h;
#pragma unroll
      for (int i = 0; i < DP / C::STEP; ++i) {
        const int c = (2 * i + half) * 16;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (there && c < width) x = load16<false>(p + c);
        q[i] = __builtin_bit_cast(typename C::Fragment, x);
      }
    }
    const char* kp = reinterpret_cast<const char*>(a.k.p) + (PAGED ? 0 : b * a.k.s.b) + h * a.k.s.h;
    const char* vp = reinterpret_cast<const char*>(a.v.p) + (PAGED ? 0 : b * a.v.s.b) + h * a.v.s.h;
    const int32_t* table = PAGED ? a.table + b * a.ldt : nullptr;
    // Tile i's pages, one for each of its rows, to LDS.
    auto pages = [&](int64_t i) {
      const uint32_t t = (uint32_t)min(32 * i + (lane & 31), k_len - 1);
      load_lds4(table + (uint32_t)((uint64_t)t * a.page_magic >> a.page_shift), entries + (uint32_t)(i - i0) % F::ENTRIES * 256);
    };
    auto entry = [&](int64_t i, int r) {
      return *reinterpret_cast<const int*>(mine + 2 * S * F::BYTES + (uint32_t)(i - i0) % F::ENTRIES * 256 + r * 4);
    };
    // Tile i of keys or values; a row that there is not, or whose page is none of the cache's, is zeros.
    auto tile = [&](const char* x, int64_t ld, int64_t i, uint32_t to) {
#pragma unroll
      for (int p = 0; p < N; ++p) {
        const int slot = p * 64 + lane, r = slot / Tile::PITCH, c = ((slot % Tile::PITCH) ^ Tile::swizzle(r)) * 16;
        const int64_t t = 32 * i + r;
        const char* src = reinterpret_cast<const char*>(mfma_zero16);
        if (i < i1 && t < k_len) {
          if (PAGED) {
            const int e = entry(i, r);
            const uint32_t first = (uint32_t)((uint64_t)(uint32_t)t * a.page_magic >> a.page_shift);
            if (e >= 0 && e < a.pages) src = x + e * a.k.s.b + ((uint32_t)t - first * (uint32_t)a.page) * ld + c;
          } else {
            src = x + t * ld + c;
          }
        }
        if (c < width) load_lds16(src, to + p * 1024);
      }
    };
    auto slot_of = [&](int64_t i) { return (uint32_t)(i - i0) % S * F::BYTES; };
    auto keys = [&](int64_t i) {
      if (PAGED) pages(i + S);
      tile(kp, a.k.s.l, i, ring + slot_of(i));
    };
    auto values = [&](int64_t i) { tile(vp, a.v.s.l, i, ring + S * F::BYTES + slot_of(i)); };

    f32x16 o[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = zeros();
    float m = -INFINITY, l = 0.0f;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // (the ring is free)
    if (PAGED) {
      for (int j = 0; j < S; ++j) pages(i0 + j);
      wait_loads<0>();
    }
    for (int j = 0; j < S; ++j) {
      keys(i0 + j);
      values(i0 + j);
    }
    // Behind a tile of keys: S of values and S - 1 of keys with their pages; behind one of values the other way round.
    constexpr int E = PAGED ? 1 : 0;
    for (int64_t i = i0; i < i1; ++i) {
      wait_loads<S * N + (S - 1) * (N + E)>();
      __builtin_amdgcn_sched_barrier(0);
      uint32_t some = ~0u;   // keys of the tile that are there
      {
        bool x = 32 * i + (lane & 31) < k_len;
        if (PAGED) {
          const int e = entry(i, lane & 31);
          x = x && e >= 0 && e < a.pages;
        }
        some = (uint32_t)__ballot(x);
      }
      const uint32_t tk = Tile::along_at(ring + slot_of(i), lane);
      f32x16 s = zeros();
#pragma unroll
      for (int j = 0; j < DP / C::STEP; ++j) C::multiply(Tile::along(tk, 0, j), q[j], s);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      keys(i + S);
      if (some != ~0u) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(some >> (8 * (e >> 2) + 4 * half + (e & 3)) & 1)) s[e] = -INFINITY;
      }
      float top = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
      top = fmaxf(top, other_half(top));
      if (__any(top > m && (top - m) * a.scale2 > 8.0f)) {   // (else sums stay under the older maximum)
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
      for (int e = 0; e < 16; ++e) {
        s[e] = exp2_(fmaf(s[e], a.scale2, -mc));
        l += s[e];
      }
      wait_loads<S * (N + E) + (S - 1) * N>();
      __builtin_amdgcn_sched_barrier(0);
      const uint32_t tv = Tile::down_at(ring + S * F::BYTES + slot_of(i), lane);
#pragma unroll
      for (int j = 0; j < 32 / C::STEP; ++j) {
        const typename C::Fragment p = C::pack(s, j);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) C::multiply(Tile::down(tv, 0, j, d), p, o[d]);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      values(i + S);
    }
    l += other_half(l);
    const float top2 = m == -INFINITY ? 0.0f : m * a.scale2;
    if (came || goes) {
      const int64_t slot = (w * 2 + (came ? 0 : 1)) * a.rows + (lane & 31);
      if ((lane & 31) < a.rows) {
        if (half == 0) *reinterpret_cast<float2*>(a.top_sum + 2 * slot) = make_float2(l == 0.0f ? -INFINITY : top2, l);
        float* to = a.partial + slot * DP + 4 * half;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            *reinterpret_cast<float4*>(to + 32 * d + 8 * v) = make_float4(o[d][4 * v], o[d][4 * v + 1], o[d][4 * v + 2], o[d][4 * v + 3]);
      }
    } else if (query < a.S) {
      const float f = l == 0.0f || !there ? 0.0f : 1.0f / l;
      char* to = reinterpret_cast<char*>(const_cast<void*>(a.out.p)) + b * a.out.s.b + query * a.out.s.l + hq * a.out.s.h;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int c = 32 * d + 8 * v + 4 * half;
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = there ? o[d][4 * v + e] * f : 0.0f;
          if (c >= a.D) continue;
          if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to + c * 4) = make_float4(x[0], x[1], x[2], x[3]);
          else *reinterpret_cast<uint2*>(to + c * 2) = make_uint2(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]));
        }
      if (a.stats && half == 0) a.stats[(b * a.q_heads + hq) * a.S + query] = l == 0.0f || !there ? INFINITY : top2 + log2_(l);
    }
    at = begin + i1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing is under way to LDS when the block ends)
}

// One query of one head to a block: its parts, 256 / (DP / 4) of them at a time, added up in the order of the wavefronts.
template <typename T, int DP>
__global__ __launch_bounds__(256) void stream_join_kernel(StreamArgs a) {
  constexpr int LANES = DP / 4, GROUPS = 256 / LANES;
  __shared__ float4 sums[GROUPS][LANES];
  __shared__ float parts[GROUPS];
  const int64_t id = blockIdx.x, query = id % a.S, bh = id / a.S, hq = bh % a.q_heads, b = bh / a.q_heads;
  const int64_t h = hq / a.group, row = query * a.group + hq - h * a.group;
  const int64_t n = a.before[b + 1] - a.before[b], times = (int64_t)a.heads * a.row_tiles;
  const bool there = n > 0 && query < length_of(a.q_lengths, b, a.S);
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  float4 sum = make_float4(0, 0, 0, 0);
  float l = 0.0f, top = -INFINITY;
  if (there) {
    const Pieces pieces(a.before[a.B] * times, a.waves);
    const int64_t begin = a.before[b] * times + (h * a.row_tiles + row / 32) * n;
    const int64_t w0 = pieces.owner(begin), w1 = pieces.owner(begin + n - 1);
    if (w0 == w1) return;   // (written by that wavefront)
    auto slot = [&](int64_t w) { return (w * 2 + (w == w0 ? 1 : 0)) * a.rows + row % 32; };
    for (int64_t w = w0 + threadIdx.x % 64; w <= w1; w += 64) top = fmaxf(top, a.top_sum[2 * slot(w)]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
    for (int64_t w = w0 + group; w <= w1; w += GROUPS) {
      const float2 ml = *reinterpret_cast<const float2*>(a.top_sum + 2 * slot(w));
      const float4 x = *reinterpret_cast<const float4*>(a.partial + slot(w) * DP + 4 * lane);
      const float f = exp2_(ml.x - base);
      // (a part without keys that are there: nothing, whatever its sums hold)
      l += ml.y * f;
      sum.x += x.x * f; sum.y += x.y * f; sum.z += x.z * f; sum.w += x.w * f;
    }
  }
  sums[group][lane] = sum;
  if (lane == 0) parts[group] = l;
  __syncthreads();
  if (group > 0) return;
  l = 0.0f;
  sum = make_float4(0, 0, 0, 0);
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    l += parts[g];
    sum.x += sums[g][lane].x; sum.y += sums[g][lane].y; sum.z += sums[g][lane].z; sum.w += sums[g][lane].w;
  }
  const float f = l == 0.0f ? 0.0f : 1.0f / l;
  if (4 * lane < a.D) {
    char* to = reinterpret_cast<char*>(const_cast<void*>(a.out.p)) + b * a.out.s.b + query * a.out.s.l + hq * a.out.s.h;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to + 16 * lane) = make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f);
    else *reinterpret_cast<uint2*>(to + 8 * lane) = make_uint2(f2bf2(sum.x * f, sum.y * f), f2bf2(sum.z * f, sum.w * f));
  }
  if (a.stats && lane == 0) a.stats[bh * a.S + query] = l == 0.0f ? INFINITY : top + log2_(l);
}

struct StreamPlan {
  int64_t before, top_sum, partial, bytes;
  int32_t rows, row_tiles;
};
StreamPlan stream_plan(int64_t B, int64_t S, int64_t q_heads, int64_t heads, int64_t D) {
  StreamPlan p;
  const int64_t all = S * (q_heads / heads), dp = D <= 32 ? 32 : D <= 64 ? 64 : 128;
  p.row_tiles = (int)div_up(all, 32);
  p.rows = (int)std::min<int64_t>(all, 32);
  auto room = [](int64_t n) { return div_up(n, 256) * 256; };
  p.before = 0;
  p.top_sum = room((B + 1) * 8);
  p.partial = p.top_sum + room((int64_t)BLOCKS * WAVES * 2 * p.rows * 8);
  p.bytes = p.partial + (int64_t)BLOCKS * WAVES * 2 * p.rows * dp * 4;
  return p;
}

template <typename T, int DP, bool PAGED>
hipError_t launch(const StreamArgs& a, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  typedef Stream<T, DP> F;
  const hipError_t e = allow_lds(stream_kernel<T, DP, PAGED>, F::LDS, (64 * WAVES + 1) * 8, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((stream_kernel<T, DP, PAGED>), dim3(BLOCKS), dim3(64 * WAVES), F::LDS, s, a);
  hipLaunchKernelGGL((stream_join_kernel<T, DP>), dim3((unsigned)(a.B * a.S * a.q_heads)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

size_t stream_bytes(int64_t B, int64_t S, int64_t q_heads, int64_t heads, int64_t D) { return (size_t)stream_plan(B, S, q_heads, heads, D).bytes; }

hipError_t launch_stream(StreamArgs a, int32_t dtype, void* workspace, hipStream_t s) {
  const StreamPlan p = stream_plan(a.B, a.S, a.q_heads, a.heads, a.D);
  char* ws = reinterpret_cast<char*>(workspace);
  a.row_tiles = p.row_tiles; a.rows = p.rows; a.waves = BLOCKS * WAVES;
  a.before = reinterpret_cast<int64_t*>(ws + p.before);
  a.top_sum = reinterpret_cast<float*>(ws + p.top_sum);
  a.partial = reinterpret_cast<float*>(ws + p.partial);
  return by_size(dtype, a.D, [&](auto t, auto dp) {
    typedef decltype(t) T;
    return a.table ? launch<T, decltype(dp)::value, true>(a, s) : launch<T, decltype(dp)::value, false>(a, s);
  });
}

}  // namespace antdt

using namespace antdt;

extern "C" {

static int cache_attention_sizes(const char* call, int64_t B, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype) {
  OP_TRY(op_head_sizes(call, q_heads, heads, D, dtype));
  if (B < 0 || B * q_heads >= 1 << 24) return op_fail(ANTDT_UNSUPPORTED, "%s: B q_heads: 2^24 or more", call);
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
  static const int32_t none = 0;
  a.table = table_cols > 0 ? table : &none;   // (without columns no length is above 0, and nothing reads it)
  a.ldt = ld_table; a.pages = pages; a.k_lengths = lengths; a.B = B; a.S = 1;
  a.T = std::min<int64_t>(table_cols * page_size, (1ll << 31) - 1);
  a.page = (int)page_size;
  int shift = 0;
  while ((1ll << shift) < page_size) ++shift;
  a.page_shift = 31 + shift;
  a.page_magic = (uint32_t)((((__int128)1 << (31 + shift)) + page_size - 1) / page_size);
  a.q_heads = (int)q_heads; a.heads = (int)heads; a.group = (int)(q_heads / heads); a.D = (int)D; a.scale2 = scale * LOG2E;
  return op_hip(call, launch_stream(a, dtype, workspace, (hipStream_t)stream));
}

}  // extern "C"
