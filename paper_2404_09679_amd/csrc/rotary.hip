// Rotation of heads by their tokens' positions, and the same on the way into a paged cache.
//
// Pair i of a head's R rotated columns, at position p, is turned by the angle a = p w_i:
//   (u, v) -> m (u cos a - v sin a, v cos a + u sin a);   its gradient: the same with -a.
// Angles are kept in turns as 64-bit fixed-point fractions: p times the pair's fraction of a turn, modulo 2^64, drops whole turns without a
// rounding, so that a position of 2^31 is as exact as 1 (in fp32 a product of 10^6 radians is off by 0.03).
#include "heads.h"
#include "sort.h"

namespace antdt {
namespace {

constexpr int WAVES = 4, MOST_TOKENS = 16, MOST_PAIRS = 512;   // of a wavefront, at a time

// Some heads of every token: queries, keys or values.  A chunk is 16 columns of a head: 8 pairs, or columns that are copied.
struct HeadsPart {
  const void* x;
  void* y;
  int64_t xl, xh;        // strides of the token and the head
  int64_t yp, yl, yh;    // of the page, the row in it (without pages: of the token) and the head
  int32_t first;         // chunk of a token that is the part's first
  Divisor chunks;        // of a head
  int32_t turned;        // how many of them are turned
  int32_t paged;
};
struct RotaryArgs {
  HeadsPart part[3];
  const uint64_t* turns;
  const int32_t* positions;   // or, for a cache:
  const int32_t* lengths;
  const int32_t* offsets;
  const int32_t* table;
  int64_t N, B, ldt, room, pages;   // room: tokens that a row of the table has pages for
  int32_t parts, half, interleaved, D;
  int32_t pitch;                    // of a token's cosines in LDS: pairs, rounded up to a multiple of 8
  int32_t tokens, slices, span;     // tokens of a wavefront; wavefronts of a token, chunks of one
  Divisor per_token, pairs, pages_of;   // chunks and pairs of a token, tokens of a page
  float magnitude, sign;
};

// cos and sin of t 2^-64 turns.  The nearest quarter turn is taken off in whole numbers; what is left, x in -1/2 .. 1/2 quarter turns, goes into
// Taylor's series of sin(x pi / 2) (to x^9, remainder below 2e-9) and cos(x pi / 2) (to x^10, below 1e-9).  With u = 2^-24 a value is off by 3 u at most:
// x and the last product round once each, the rest of the series, below a third of the value, twice.
__device__ __forceinline__ void turn(uint64_t t, float& c, float& s) {
  const uint64_t w = t + (1ull << 61);
  const float x = (float)((int32_t)((uint32_t)(w >> 30) ^ 0x80000000u)) * 2.3283064365386963e-10f, y = x * x;
  const float a = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.6044118e-4f, -4.6817541e-3f), 7.9692626e-2f), -0.64596410f), 1.5707963f);
  const float b = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.5202043e-5f, 9.1926027e-4f), -2.0863481e-2f), 0.25366951f), -1.2337006f), 1.0f);
  const uint32_t quarter = (uint32_t)(w >> 62);
  c = quarter & 1 ? a : b;
  s = quarter & 1 ? b : a;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter >= 2) s = -s;
}

// Position of each lane's token n in its sequence (-1: in none), and where in the cache it belongs (row -1: nowhere).  Called by the whole wavefront:
// the sequence is found among 64 of the offsets, one in each lane, and then (of 64 sequences and more) between two of them in memory.  Of fewer
// sequences the lanes hold the lengths too, so that nothing but the page waits for another load.
__device__ __forceinline__ int place(const RotaryArgs& a, int64_t n, int lane, int& page, int& row) {
  int64_t b = n, first = n, behind = n + 1, length;
  page = 0; row = -1;
  if (a.B == 0) return -1;
  if (a.offsets) {
    const int64_t step = (a.B + 63) >> 6;
    const bool all = a.B < 64;
    const int mine = a.offsets[min(lane * step, a.B)], of_mine = all ? a.lengths[min((int64_t)lane, a.B - 1)] : 0;
    int at = 0;   // the last lane whose sequence starts at n or before
#pragma unroll
    for (int s = 32; s > 0; s >>= 1)
      if (__shfl(mine, at + s, 64) <= n) at += s;
    b = min(at * step, a.B - 1);
    if (all) {
      first = __shfl(mine, (int)b, 64);
      behind = __shfl(mine, (int)b + 1, 64);
      length = __shfl(of_mine, (int)b, 64);
    } else {
      int64_t end = min(b + step, a.B);
      while (end - b > 1) {
        const int64_t mid = (b + end) >> 1;
        if (a.offsets[mid] <= n) b = mid;
        else end = mid;
      }
      first = a.offsets[b];
      behind = a.offsets[b + 1];
      length = a.lengths[b];
    }
  } else {
    length = a.lengths[b];
  }
  const int64_t at = length - (behind - n);
  if (n < first || n >= behind || at < 0) return -1;
  if (at < a.room) {
    const uint32_t i = a.pages_of((uint32_t)at);
    page = a.table[b * a.ldt + i];
    if (page >= 0 && page < a.pages) row = (int)(at - (int64_t)i * a.pages_of.d);
  }
  return (int)at;
}

// Every wavefront has some tokens, or a part of one.  Its first columns are asked for before the positions are; cosines and sines go to LDS once, for
// all heads.  Bound by memory: 65536 tokens of 16 heads of 128 bf16 columns (537 MB) 99 us; a token alone by its chain of loads (place in the sequence,
// page): 64 of them, 16 + 2 x 4 heads of 128, 5 us.
template <typename T, int Q, bool INTERLEAVED, bool CACHE>
__global__ __launch_bounds__(64 * WAVES) void rotary_kernel(RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) float cosines[WAVES][MOST_PAIRS], sines[WAVES][MOST_PAIRS];
  __shared__ int where[WAVES][3][MOST_TOKENS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t groups = (a.N + a.tokens - 1) / a.tokens;
  float* cs = cosines[wave];
  float* sn = sines[wave];
  int(&at)[3][MOST_TOKENS] = where[wave];
  // f of a part, by selects: a lane's own part would be read from the arguments' memory.
  auto of_part = [&](int which, auto f) {
    if constexpr (!CACHE) return f(a.part[0]);
    else return which == 0 ? f(a.part[0]) : which == 1 ? f(a.part[1]) : f(a.part[2]);
  };
  for (int64_t w = (int64_t)blockIdx.x * WAVES + wave; w < groups * a.slices; w += (int64_t)gridDim.x * WAVES) {
    const int64_t group = a.slices == 1 ? w : w / a.slices, t0 = group * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.N - t0);
    const int begin = (int)(w - group * a.slices) * a.span, end = min(begin + a.span, tokens * (int)a.per_token.d);
    // A lane's chunk: 16 columns of a head, two halves of n0 and n1.
    float v[2][8];
    int part, token, head, pair, at0, at1, n0, n1;
    auto load = [&](int i) {
      const bool some = i < end;
      i = some ? i : 0;
      token = a.per_token(i);
      const int c = i - token * (int)a.per_token.d;
      part = !CACHE ? 0 : a.parts > 2 && c >= a.part[2].first ? 2 : a.parts > 1 && c >= a.part[1].first ? 1 : 0;
      const int in = c - of_part(part, [](const HeadsPart& p) { return p.first; });
      const Divisor chunks = {of_part(part, [](const HeadsPart& p) { return p.chunks.d; }), of_part(part, [](const HeadsPart& p) { return p.chunks.m; }),
                              of_part(part, [](const HeadsPart& p) { return p.chunks.s; })};
      const int turned = of_part(part, [](const HeadsPart& p) { return p.turned; });
      head = chunks(in);
      const int e = in - head * (int)chunks.d;
      int left0, left1;
      if (e < turned) {
        pair = 8 * e;
        at0 = INTERLEAVED ? 16 * e : 8 * e;
        at1 = INTERLEAVED ? 16 * e + 8 : a.half + 8 * e;
        left0 = INTERLEAVED ? 2 * a.half - 16 * e : a.half - 8 * e;
        left1 = INTERLEAVED ? left0 - 8 : left0;
      } else {
        pair = -1;
        at0 = (turned ? 2 * a.half : 0) + 16 * (e - turned);
        at1 = at0 + 8;
        left0 = a.D - at0;
        left1 = left0 - 8;
      }
      n0 = some ? min(8, left0) : 0;
      n1 = some ? max(0, min(8, left1)) : 0;
      const T* x = reinterpret_cast<const T*>(of_part(part, [](const HeadsPart& p) { return p.x; })) + (t0 + token) * of_part(part, [](const HeadsPart& p) { return p.xl; }) +
                   head * of_part(part, [](const HeadsPart& p) { return p.xh; });
      if (n0 > 0) load8<Q>(x + at0, n0, v[0]);
      if (n1 > 0) load8<Q>(x + at1, n1, v[1]);
    };
    load(begin + lane);   // (two under way a lane: 115 us for 95)
    const int pairs = tokens * a.half;
    uint64_t f = lane < pairs ? a.turns[lane - a.pairs(lane) * a.half] : 0;
    {
      int page = 0, row = 0, p = 0;
      if (CACHE) p = place(a, t0 + min(lane, tokens - 1), lane, page, row);
      else if (lane < tokens) p = a.positions[t0 + lane];
      if (lane < tokens) {
        at[0][lane] = p;
        at[1][lane] = page;
        at[2][lane] = row;
      }
    }
    wave_lds_order();
    for (int i = lane; i < pairs; i += 64) {
      const int j = a.pairs(i), k = i - j * a.half;
      if (i != lane) f = a.turns[k];
      float c, s;
      turn((uint64_t)(int64_t)at[0][j] * f, c, s);
      cs[j * a.pitch + k] = c * a.magnitude;
      sn[j * a.pitch + k] = s * a.magnitude * a.sign;
    }
    wave_lds_order();
    for (int i = begin;;) {
      const bool paged = CACHE && of_part(part, [](const HeadsPart& p) { return p.paged; }) != 0;
      if (n0 > 0 && !(paged && at[2][token] < 0)) {
        if (pair >= 0) {
          float c[8], s[8];
          load8<4>(cs + token * a.pitch + pair, 8, c);   // (behind the last pair whatever lies there, for columns that are not stored)
          load8<4>(sn + token * a.pitch + pair, 8, s);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float& x = INTERLEAVED ? v[e >> 2][2 * (e & 3)] : v[0][e];
            float& y = INTERLEAVED ? v[e >> 2][2 * (e & 3) + 1] : v[1][e];
            const float x0 = x;
            x = fmaf(-y, s[e], x0 * c[e]);   // (said so: every layout's kernel rounds alike)
            y = fmaf(x0, s[e], y * c[e]);
          }
        }
        if (CACHE && !paged && at[0][token] < 0) {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e >> 3][e & 7] = 0.0f;
        }
        const int64_t yl = of_part(part, [](const HeadsPart& p) { return p.yl; }), yh = of_part(part, [](const HeadsPart& p) { return p.yh; });
        T* y = reinterpret_cast<T*>(of_part(part, [](const HeadsPart& p) { return p.y; })) + head * yh;
        if (paged) y += at[1][token] * of_part(part, [](const HeadsPart& p) { return p.yp; }) + at[2][token] * yl;
        else y += (t0 + token) * yl;
        store8<Q>(y + at0, n0, v[0]);
        if (n1 > 0) store8<Q>(y + at1, n1, v[1]);
      }
      i += 64;
      if (i >= end) break;
      load(i + lane);
    }
    wave_lds_order();   // (the next tokens' go to the same places)
  }
}

// Wavefronts: several small tokens to one, or several to a large token.
void share(RotaryArgs& a, int per_token) {
  a.per_token = Divisor::of(per_token);
  a.pairs = Divisor::of(std::max(a.half, 1));
  a.pitch = (a.half + 7) & ~7;
  a.tokens = std::max(1, std::min(64 / per_token, MOST_TOKENS));
  if (a.half) a.tokens = std::max(1, std::min(a.tokens, MOST_PAIRS / a.pitch));
  a.slices = 1;
  a.span = a.tokens * per_token;
  if (per_token > 64) {
    int turns = 4;
    while (turns > 1 && a.N * div_up(per_token, 64 * turns) < 8192) turns >>= 1;
    a.span = 64 * turns;
    a.slices = (int)div_up(per_token, a.span);
  }
}

template <typename T, bool CACHE>
hipError_t launch_rotary(const RotaryArgs& a, int quantum, hipStream_t s) {
  const int64_t waves = div_up(a.N, a.tokens) * a.slices;
  const dim3 grid((unsigned)std::min<int64_t>(div_up(waves, WAVES), 1 << 20)), block(64 * WAVES);
  auto go = [&](auto q) {
    constexpr int Q = decltype(q)::value;
    if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, Q, true, CACHE>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<T, Q, false, CACHE>), grid, block, 0, s, a);
  };
  if (quantum == 8) go(std::integral_constant<int, 8>());
  else if (quantum == 4) go(std::integral_constant<int, 4>());
  else go(std::integral_constant<int, 1>());
  return hipGetLastError();
}

constexpr int64_t HEADS_MAX = 1 << 16;

int rotary_sizes(const char* call, int64_t N, int64_t H, int64_t D) {
  if (N < 0 || N >= (1ll << 31) - 1) return op_fail(ANTDT_INVALID_ARG, "%s: N out of range", call);
  if (H < 0 || H > HEADS_MAX) return op_fail(ANTDT_INVALID_ARG, "%s: heads out of range", call);
  if (D < 0 || D > ANTDT_MAX_HEAD_DIM) return op_fail(ANTDT_INVALID_ARG, "%s: D out of range", call);
  return ANTDT_OK;
}
// The spec checked and taken over; the columns that a vector access takes of its pairs.
int rotary_spec(const char* call, const antdt_rotary_spec* r, int64_t D, RotaryArgs& a, int& quantum) {
  if (r->dim < 2 || r->dim % 2 || r->dim > D) return op_fail(ANTDT_INVALID_ARG, "%s: rotary: %d of %lld columns", call, r->dim, (long long)D);
  if (r->interleaved != 0 && r->interleaved != 1) return op_fail(ANTDT_INVALID_ARG, "%s: rotary: interleaved is 0 or 1", call);
  if (!isfinite(r->magnitude)) return op_fail(ANTDT_INVALID_ARG, "%s: rotary: magnitude is not finite", call);
  if (!r->turns || (reinterpret_cast<uintptr_t>(r->turns) & 7)) return op_fail(ANTDT_INVALID_ARG, "%s: rotary: turns is null or misaligned", call);
  a.turns = r->turns; a.half = r->dim / 2; a.interleaved = r->interleaved; a.magnitude = r->magnitude;
  const int wide = a.interleaved ? r->dim : a.half;   // (a chunk's halves start at multiples of it, or of 8)
  quantum = wide % 8 == 0 ? 8 : wide % 4 == 0 ? 4 : 1;
  return ANTDT_OK;
}
// Chunks of the parts, in the order of a token; `per_token` those of the parts so far.
void chunks(RotaryArgs& a, int part, int64_t heads, bool turned, bool copied, int& per_token) {
  HeadsPart& p = a.part[part];
  p.first = per_token;
  p.turned = turned ? (int)div_up(a.half, 8) : 0;
  p.chunks = Divisor::of(p.turned + (copied ? (int)div_up(a.D - (turned ? 2 * a.half : 0), 16) : 0));
  per_token += p.chunks.d * (int)heads;
  a.parts = part + 1;
}

}  // namespace
}  // namespace antdt

using namespace antdt;

extern "C" {

int antdt_rotary_turns(int32_t dim, double base, double factor, double original, double low, double high, uint64_t* turns) {
  const char* call = "antdt_rotary_turns";
  if (dim < 2 || dim % 2 || dim > ANTDT_MAX_HEAD_DIM) return op_fail(ANTDT_INVALID_ARG, "%s: dim", call);
  if (!(base >= 1.0) || !isfinite(base)) return op_fail(ANTDT_INVALID_ARG, "%s: base below 1 or not finite", call);
  if (!(factor >= 1.0) || !isfinite(factor)) return op_fail(ANTDT_INVALID_ARG, "%s: factor below 1 or not finite", call);
  const bool by_parts = high != 0.0;
  if (by_parts && (!(low >= 0.0) || !(high > low) || !isfinite(high) || !(original > 0.0) || !isfinite(original)))
    return op_fail(ANTDT_INVALID_ARG, "%s: low, high and original: 0 <= low < high, original > 0", call);
  if (!turns) return op_fail(ANTDT_INVALID_ARG, "%s: turns is null", call);
  constexpr double TWO_PI = 6.283185307179586476925286766559;
  for (int i = 0; i < dim / 2; ++i) {
    const double f = pow(base, -2.0 * i / dim) / TWO_PI;
    const double keep = by_parts ? std::min(1.0, std::max(0.0, (f * original - low) / (high - low))) : 0.0;
    turns[i] = (uint64_t)(f * (keep + (1.0 - keep) / factor) * 18446744073709551616.0 + 0.5);   // (below 2^62)
  }
  return ANTDT_OK;
}

int antdt_rotary(const void* x, int64_t ldx, int64_t ldx_head, int64_t N, int64_t H, int64_t D, int32_t dtype, const int32_t* positions,
                 const antdt_rotary_spec* rotary, int32_t inverse, void* y, int64_t ldy, int64_t ldy_head, void* stream) {
  const char* call = "antdt_rotary";
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  OP_TRY(rotary_sizes(call, N, H, D));
  if (!rotary) return op_fail(ANTDT_INVALID_ARG, "%s: rotary is null", call);
  RotaryArgs a = {};
  int q;
  if (N == 0 || H == 0 || D == 0) return ANTDT_OK;
  OP_TRY(rotary_spec(call, rotary, D, a, q));
  HeadStrides sx = {0, ldx, ldx_head}, sy = {0, ldy, ldy_head};
  const int64_t size = op_size(dtype);
  OP_TRY(op_heads(call, "x", x, 1, N, H, D, sx, size, false));
  OP_TRY(op_heads(call, "y", y, 1, N, H, D, sy, size, true));
  OP_TRY(op_matrix(call, "positions", positions, N, 1, 1, 4));
  a.N = N; a.D = (int)D; a.positions = positions; a.sign = inverse ? -1.0f : 1.0f;
  a.part[0] = HeadsPart{x, y, sx.l, sx.h, 0, sy.l, sy.h, 0, Divisor(), 0, 0};
  const bool copied = rotary->dim < D && !same_heads(x, sx, y, sy);
  int per_token = 0;
  chunks(a, 0, H, true, copied, per_token);
  share(a, per_token);
  q = std::min(q, std::min(head_quantum(copied ? D : 2 * a.half, size, x, sx), head_quantum(copied ? D : 2 * a.half, size, y, sy)));
  const hipStream_t s = (hipStream_t)stream;
  return op_hip(call, dtype == ANTDT_F32 ? launch_rotary<float, false>(a, q, s) : launch_rotary<bf16_t, false>(a, q, s));
}

int antdt_cache_append(const void* q, int64_t ldq, int64_t ldq_head, void* q_out, int64_t ldqo, int64_t ldqo_head, const void* k, int64_t ldk,
                       int64_t ldk_head, const void* v, int64_t ldv, int64_t ldv_head, int64_t N, int64_t q_heads, int64_t heads, int64_t D, int32_t dtype,
                       const antdt_rotary_spec* rotary, void* k_cache, void* v_cache, int64_t ld_page, int64_t ld_row, int64_t ld_head, int64_t pages,
                       int64_t page_size, const int32_t* table, int64_t ld_table, int64_t B, int64_t table_cols, const int32_t* lengths, const int32_t* offsets,
                       void* stream) {
  const char* call = "antdt_cache_append";
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  OP_TRY(rotary_sizes(call, N, q_heads, D));
  OP_TRY(rotary_sizes(call, B, heads, D));
  if (!offsets && N != B) return op_fail(ANTDT_INVALID_ARG, "%s: without offsets a token for each sequence", call);
  if (page_size < 1 || page_size >= (1ll << 31)) return op_fail(ANTDT_INVALID_ARG, "%s: page_size out of range", call);
  if (table_cols < 0 || table_cols >= (1ll << 31)) return op_fail(ANTDT_INVALID_ARG, "%s: table_cols out of range", call);
  if (pages < 0 || pages >= (1ll << 31)) return op_fail(ANTDT_INVALID_ARG, "%s: pages out of range", call);
  RotaryArgs a = {};
  int quantum = 8;
  if (N == 0 || D == 0 || (heads == 0 && q_heads == 0)) return ANTDT_OK;
  if (rotary) OP_TRY(rotary_spec(call, rotary, D, a, quantum));
  const int64_t size = op_size(dtype);
  HeadStrides sq = {0, ldq, ldq_head}, so = {0, ldqo, ldqo_head}, sk = {0, ldk, ldk_head}, sv = {0, ldv, ldv_head};
  HeadStrides sc = {ld_page, ld_row, ld_head}, sc2 = sc;
  OP_TRY(op_heads(call, "q", q, 1, N, q_heads, D, sq, size, false));
  OP_TRY(op_heads(call, "q_out", q_out, 1, N, q_heads, D, so, size, true));
  OP_TRY(op_heads(call, "k", k, 1, N, heads, D, sk, size, false));
  OP_TRY(op_heads(call, "v", v, 1, N, heads, D, sv, size, false));
  OP_TRY(op_heads(call, "k_cache", k_cache, pages, page_size, heads, D, sc, size, true));
  OP_TRY(op_heads(call, "v_cache", v_cache, pages, page_size, heads, D, sc2, size, true));
  OP_TRY(op_matrix(call, "table", table, B, table_cols, ld_table, 4));
  OP_TRY(op_matrix(call, "lengths", lengths, B, 1, 1, 4));
  if (offsets) OP_TRY(op_matrix(call, "offsets", offsets, B + 1, 1, 1, 4));
  a.N = N; a.B = B; a.D = (int)D; a.sign = 1.0f;
  a.lengths = lengths; a.offsets = offsets; a.table = table; a.ldt = ld_table;
  a.pages_of = Divisor::of((uint32_t)page_size); a.pages = pages; a.room = table_cols * page_size;
  int part = 0, per_token = 0;
  if (q_heads > 0) {
    a.part[part] = HeadsPart{q, q_out, sq.l, sq.h, 0, so.l, so.h, 0, Divisor(), 0, 0};
    chunks(a, part++, q_heads, rotary != nullptr, !rotary || rotary->dim < D, per_token);
    quantum = std::min(quantum, std::min(head_quantum(D, size, q, sq), head_quantum(D, size, q_out, so)));
  }
  if (heads > 0) {
    a.part[part] = HeadsPart{k, k_cache, sk.l, sk.h, sc.b, sc.l, sc.h, 0, Divisor(), 0, 1};
    chunks(a, part++, heads, rotary != nullptr, !rotary || rotary->dim < D, per_token);
    a.part[part] = HeadsPart{v, v_cache, sv.l, sv.h, sc.b, sc.l, sc.h, 0, Divisor(), 0, 1};
    chunks(a, part++, heads, false, true, per_token);
    quantum = std::min(std::min(quantum, head_quantum(D, size, k_cache, sc)), std::min(head_quantum(D, size, k, sk), head_quantum(D, size, v, sv)));
    quantum = std::min(quantum, head_quantum(D, size, v_cache, sc));
  }
  share(a, per_token);
  const hipStream_t s = (hipStream_t)stream;
  return op_hip(call, dtype == ANTDT_F32 ? launch_rotary<float, true>(a, quantum, s) : launch_rotary<bf16_t, true>(a, quantum, s));
}

}  // extern "C"
