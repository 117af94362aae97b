// Attention of queries over keys and values of another length, forward (see cross.h).
#include "cross.h"

namespace antdt {
namespace {

// A block has queries of a head; tiles of keys and values go through LDS, the next one's loads under way.  A wavefront's 32 queries take a pass over the
// vector units (maximum, exponential, sum) for each over the matrix core, about as long; two wavefronts on a SIMD have them at the same time.  8 ragged
// histories of 2048 queries and 4096 keys, 16 and 4 heads of 128 bf16 columns: 381 GFLOP in 426-441 us (by the clock that
// power leaves), an eighth of it the last blocks, when not all compute units have one.
// PAGED: keys and values are a cache's, the user's pages looked up before the first tile; probabilities in two parts, see stream.hip (16 users of 100 and
// 1000 tokens, 16 and 4 heads of 64 bf16 columns, all of it in the caches: 5.0 -> 5.1 us, 12.4 -> 13.5).
template <typename W, bool PAGED>
__global__ __launch_bounds__(W::THREADS, W::PER_CU) void cross_forward_kernel(CrossArgs a) {
  typedef typename W::T T;
  typedef typename W::Tile Tile;
  typedef Core<T> C;
  typedef KeyTiles<W> F;
  constexpr int BT = W::TILE, PARTS = PAGED ? C::PARTS : 1;   // (of the probabilities)
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int unit, block;
  place_of(a, blockIdx.x, a.group * a.queries.tiles, unit, block);
  const int tile = block % a.queries.tiles, h = unit % a.heads * a.group + block / a.queries.tiles;
  const Entry of = entry_of(a, unit / a.heads, lane);
  const int64_t b = of.b, bh = b * a.q_heads + h, q_len = of.q_len, k_len = of.k_len;
  const int64_t first = (int64_t)tile * W::ROWS, last = min(first + W::ROWS, a.S), r0 = first + (W::SPLIT ? 0 : wave * 32);
  const Rows out = a.out.rows(b, h);
  float* stats = a.stats ? a.stats + bh * a.S : nullptr;
  const int64_t end = k_len > 0 ? min(max(q_len, first), last) : first;   // rows with keys
  clear_rows<T>(out, end, last, a.D, W::THREADS);
  if (stats)
    for (int64_t r = end + threadIdx.x; r < last; r += W::THREADS) stats[r] = INFINITY;
  if (end == first) return;
  if (a.D < W::COLS) {
    clear_lds(lds, F::ALL, W::THREADS);
    __syncthreads();
  }
  const typename W::Load load(W::SPLIT ? lane : threadIdx.x, a.D);
  const Rows k = a.k.rows(PAGED ? 0 : b, h / a.group), v = a.v.rows(PAGED ? 0 : b, h / a.group);
  int* const pages = reinterpret_cast<int*>(lds + F::LDS);
  // Page of key t, below 0 where there is none.
  auto page_of = [&](int64_t t, uint32_t& row) {
    const uint32_t i = a.page((uint32_t)t);
    row = (uint32_t)t - i * a.page.d;
    return t < k_len ? pages[i] : -1;
  };
  if constexpr (PAGED) {
    const int n = (int)a.page((uint32_t)k_len - 1) + 1;
    for (int i = threadIdx.x; i < n; i += W::THREADS) {
      const int e = a.table[b * a.ldt + i];
      pages[i] = e < a.pages ? e : -1;
    }
    __syncthreads();
  }
  const uint32_t ring0 = lds_address(lds) + (W::SPLIT ? wave * F::RING : 0), lds0 = ring0 + (W::SPLIT ? 0 : wave * 1024);
  constexpr int64_t STEP = (W::SPLIT ? W::WAVES : 1) * BT;
  const int64_t t0 = W::SPLIT ? wave * BT : 0;
  int64_t asked = t0;
  auto issue = [&](uint32_t to) {
    if constexpr (PAGED) {
      load.each([&](int row, int column, uint32_t at) {
        uint32_t in;
        const int e = page_of(asked + row, in);
        const int64_t off = e * a.k.s.b + in * k.ld + column;
        load_lds16(e < 0 ? reinterpret_cast<const char*>(mfma_zero16) : k.p + off, lds0 + to + at);
        load_lds16(e < 0 ? reinterpret_cast<const char*>(mfma_zero16) : v.p + off, lds0 + to + W::Load::BYTES + at);
      });
    } else {
      load(k, asked, k_len, lds0 + to);
      load(v, asked, k_len, lds0 + to + W::Load::BYTES);
    }
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
    if constexpr (PAGED) {
      uint32_t in;
      const uint32_t some = (uint32_t)__ballot(page_of(t + (lane & 31), in) >= 0);   // keys of the tile that there are
      if (some != ~0u) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(some >> (8 * (e >> 2) + 4 * half + (e & 3)) & 1)) s[0][e] = -INFINITY;
      }
    } else if (t + BT > k_len) {
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
    typename C::Fragment p[PARTS];
    values.run(value, [&](int i, const typename C::Fragment& x) {
      if (i % W::DT == 0) C::pack(s[i / (W::DT * W::PACKS)], i / W::DT % W::PACKS, p);
#pragma unroll
      for (const typename C::Fragment& part : p) C::multiply(x, part, o[i % W::DT]);
    });
  }
  arrive<0, true>();   // (the buffers are free)
  l = sum_of_halves(l);
  const float top2 = m == -INFINITY ? 0.0f : m * a.scale2;
  if constexpr (W::SPLIT) {
    float* sums = reinterpret_cast<float*>(lds);
    put_sums<W>(sums, o, m == -INFINITY ? -INFINITY : top2, l, wave, lane);
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
    for (int w = 0; w < W::WAVES; ++w) f[w] *= most == -INFINITY ? 0.0f : 1.0f / l;
    write_merged<W, T>(sums, f, out, first, end, a.D);
    if (stats && threadIdx.x % (W::THREADS / 32) == 0 && first + row < end) stats[first + row] = most == -INFINITY ? INFINITY : base + log2_(l);
  } else {
    write_rows<W, T>(lds + wave * W::STAGING, o, m == -INFINITY ? 0.0f : 1.0f / l, out, r0, end, a.D, lane);
    const int64_t r = r0 + (lane & 31);
    if (stats && lane < 32 && r < end) stats[r] = m == -INFINITY ? INFINITY : top2 + log2_(l);
  }
}

template <typename W, bool PAGED = false>
hipError_t launch_forward(CrossArgs a, const Shape& z, const Plan& pl, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int LDS = KeyTiles<W>::LDS + (PAGED ? TABLE * 4 : 0);
  const hipError_t e = allow_lds(cross_forward_kernel<W, PAGED>, LDS, 0, allowed);
  if (e != hipSuccess) return e;
  a.queries = pl.share(nullptr);
  a.longest_first = longest_first(z, a.k_lengths || a.q_lengths, pl.blocks, 256 * W::PER_CU);
  hipLaunchKernelGGL((cross_forward_kernel<W, PAGED>), dim3((unsigned)pl.blocks), dim3(W::THREADS), LDS, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_blocks(const CrossArgs& a, const Shape& z, hipStream_t s) {
  return by_columns(z.dtype, (int)z.D, [&](auto way, auto cols) {
    return launch_forward<typename decltype(way)::template SplitKeys<decltype(cols)::value>, true>(a, z, cache_plan(z), s);
  });
}
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
  a.q_heads = (int)q_heads; a.heads = (int)heads; a.group = (int)(q_heads / heads); a.D = (int)D; a.units = (int)(B * heads); a.B = (int)B;
  const Plan pl = forward_plan(z);
  return op_hip(call, by_columns(dtype, (int)D, [&](auto way, auto cols) {
    typedef decltype(way) Z;
    constexpr int COLS = decltype(cols)::value;
    return pl.split ? launch_forward<typename Z::template SplitKeys<COLS>>(a, z, pl, s) : launch_forward<typename Z::template Keys<COLS>>(a, z, pl, s);
  }));
}

}  // extern "C"
