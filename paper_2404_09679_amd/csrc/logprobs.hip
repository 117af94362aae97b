// Log probabilities of given tokens under rows of logits, with entropy and top alternatives, and the gradient of the logits.
// With m the largest logit of a row, s = sum e^(x - m) and q = sum e^(x - m) (x - m):
//   log p_j = (x_j - m) - log s,   H = log s - q / s,
// all three kept up in one pass (a new maximum scales s and q), so that a row is read once; bound by memory.
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "sort.h"

namespace antdt {
namespace {

constexpr int LP_THREADS = 512, LP_WAVES = LP_THREADS / 64;
constexpr int LP_LIST = 1024;           // candidates kept for the top
constexpr int64_t ROWS_OF_A_LAUNCH = 1 << 22;   // (2^32 threads are the most)
constexpr float NEG_INF = -__builtin_inff();

// Logits of more bytes than this are read, and their gradient written, without being kept in the last-level cache (256 MB), which they would
// leave before they are used again.  Kept / not, us, another buffer every time: forward and gradient of 128 / 192 / 256 / 400 MB 80 / 74, 118 / 106,
// 154 / 137, 235 / 212; with the gradient read by what follows 100 / 114, 160 / 161, 212 / 205, 320 / 311.
constexpr int64_t STREAM_BYTES = 192 << 20;

struct LpArgs {
  const void* x;
  int64_t ld, N, V;
  const int32_t* tokens;
  float* logp;
  float* entropy;
  float4* stats;
  float* top_logp;
  int32_t* top_index;
  int32_t top, pieces;
  int64_t piece;      // columns of one (the last may have fewer)
  float4* part;       // [N, pieces] m, s, q
  uint64_t* part_top; // [N, top, pieces]
};

// A logit as a whole number: larger values first, NaN above all, equal values equal; never 0 or all ones.  And with its column, equal values by
// the lower one.
__device__ __forceinline__ uint32_t value_order(float x) {
  const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
  return x != x ? 0xFFFFFFF0u : (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t col) { return (uint64_t)value_order(x) << 32 | (uint32_t)~col; }
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o >> 31) ? o & 0x7FFFFFFFu : ~o);   // (NaN stays one)
}
__device__ __forceinline__ int32_t key_column(uint64_t k) { return (int32_t) ~(uint32_t)k; }

// A NaN, or two infinities, make s a NaN, and it stays one.
struct Softmax {
  float m = NEG_INF, s = 0.0f, q = 0.0f;
  // what logits are taken relative to
  static __device__ __forceinline__ float base(float m) { return m == NEG_INF ? 0.0f : m; }
  // The sums relative to `to` >= m.
  __device__ __forceinline__ void rescale(float to) {
    const float d = base(m) - base(to), r = m == NEG_INF ? 0.0f : __expf(d);
    q = r == 0.0f ? 0.0f : r * (q + d * s);
    s *= r;
    m = to;
  }
  // x <= m.  FINITE: x - m is not -infinity (which the lowest finite logits are below a large one, too: terms of e = 0, not of NaN).
  template <bool FINITE>
  __device__ __forceinline__ void add(float x) {
    const float d = x - base(m), e = __expf(d);
    s += e;
    q += FINITE || e != 0.0f ? e * d : 0.0f;
  }
  // n logits.
  template <int n>
  __device__ __forceinline__ void add_all(const float (&v)[n]) {
    float lo = v[0];
#pragma unroll
    for (int e = 1; e < n; ++e) lo = fminf(lo, v[e]);
    if (lo - base(m) > NEG_INF) {
#pragma unroll
      for (int e = 0; e < n; ++e) add<true>(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) add<false>(v[e]);
    }
  }
};
template <int n>
__device__ __forceinline__ float largest(const float (&v)[n]) {
  float m = v[0];
#pragma unroll
  for (int e = 1; e < n; ++e) m = fmaxf(m, v[e]);
  return m;
}

// Columns [c0, c1) of a row, shared out among THREADS threads: up to the first 16-byte boundary and from the last on one by one, 16 bytes
// (a vector) at a time in between.
template <typename T, int THREADS, bool STREAM>
struct RowWalk {
  static constexpr int VN = 16 / sizeof(T), U = 2;
  const T* row;
  int64_t c0, c1, body, vecs;   // first whole vector's column, whole vectors
  __device__ __forceinline__ RowWalk(const T* row_, int64_t c0_, int64_t c1_) : row(row_), c0(c0_), c1(c1_) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row + c0) & 15) / sizeof(T));
    body = min(c1, c0 + (off ? VN - off : 0));
    vecs = (c1 - body) / VN;
  }
  static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (VN == 4) {
        v[e] = __uint_as_float(u[e]);
      } else {
        v[2 * e] = __uint_as_float(u[e] << 16);
        v[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    }
  }
  // The thread's share, columns ascending: U vectors at a time, THREADS of them apart, to batch(words, first column) as long as there are as
  // many, else vector(words, first column), single columns to one(value, column).
  struct Words {
    uint4 v[U];
  };
  template <typename B, typename V, typename O>
  __device__ __forceinline__ void each(int tid, B&& batch, V&& vector, O&& one) const {
    if (c0 + tid < body) one(to_f32(row[c0 + tid]), c0 + tid);
    const uint4* p = reinterpret_cast<const uint4*>(row + body);
    int64_t i = tid;
    constexpr int64_t LAST = (U - 1) * THREADS;
    if (i + LAST < vecs) {   // the next vectors are requested before these are worked on
      Words w, next = {};
#pragma unroll
      for (int q = 0; q < U; ++q) w.v[q] = load16<STREAM>(p + i + q * THREADS);
      while (true) {
        const bool more = i + U * THREADS + LAST < vecs;
        if (more) {
#pragma unroll
          for (int q = 0; q < U; ++q) next.v[q] = load16<STREAM>(p + i + (U + q) * THREADS);
        }
        batch(w, body + i * VN);
        i += U * THREADS;
        if (!more) break;
        w = next;
      }
    }
#pragma unroll 1
    for (; i < vecs; i += THREADS) vector(p[i], body + i * VN);
    const int64_t c = body + vecs * VN + tid;
    if (c < c1) one(to_f32(row[c]), c);
  }
  // f(value, column) for the same share, in little code.
  template <typename F>
  __device__ __forceinline__ void again(int tid, F&& f) const {
    if (c0 + tid < body) f(to_f32(row[c0 + tid]), c0 + tid);
#pragma unroll 1
    for (int64_t i = tid; i < vecs; i += THREADS) {
      float v[VN];
      unpack(reinterpret_cast<const uint4*>(row + body)[i], v);
#pragma unroll
      for (int e = 0; e < VN; ++e) f(v[e], body + i * VN + e);
    }
    const int64_t c = body + vecs * VN + tid;
    if (c < c1) f(to_f32(row[c]), c);
  }
  // The same for another share, every THREADS-th column.
  template <typename F>
  __device__ __forceinline__ void each_column(int tid, F&& f) const {
#pragma unroll 1
    for (int64_t c = c0 + tid; c < c1; c += THREADS) f(to_f32(row[c]), c);
  }
};

// Over the 64 lanes, by DPP (exchanges through LDS took twice the block's whole sum): what all lanes then hold.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, ROWS, 0xF, false);
}
template <typename Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, uint32_t none, Op&& op) {
  x = op(x, dpp<0x111, 0xF>(none, x));   // rows of 16 lanes: one lane down, ...
  x = op(x, dpp<0x112, 0xF>(none, x));
  x = op(x, dpp<0x114, 0xF>(none, x));
  x = op(x, dpp<0x118, 0xF>(none, x));   // ... eight
  x = op(x, dpp<0x142, 0xA>(none, x));   // last lane of a row to the next row (rows 1 and 3)
  x = op(x, dpp<0x143, 0xC>(none, x));   // lane 31 to rows 2 and 3
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ float wave_max(float x) {
  return __uint_as_float(wave_reduce(__float_as_uint(x), __float_as_uint(NEG_INF), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ float wave_sum(float x) {
  return __uint_as_float(wave_reduce(__float_as_uint(x), 0u, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return wave_reduce(x, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}

struct LpLds {
  uint64_t list[LP_LIST];
  uint32_t best[LP_THREADS], column[LP_THREADS];
  uint64_t threshold;
  int count, digit, above;
  float m[LP_WAVES], s[LP_WAVES], q[LP_WAVES];
};

// The block's sums from its threads': the largest logit first, then every thread's sums relative to it, added up.
__device__ __forceinline__ Softmax block_softmax(LpLds& lds, Softmax x) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, waves = blockDim.x >> 6;
  float m = wave_max(x.m);
  if (lane == 0) lds.m[w] = m;
  __syncthreads();
  for (int i = 0; i < waves; ++i) m = fmaxf(m, lds.m[i]);
  x.rescale(m);
  x.s = wave_sum(x.s);
  x.q = wave_sum(x.q);
  if (lane == 0) {
    lds.s[w] = x.s; lds.q[w] = x.q;
  }
  __syncthreads();
  x.s = x.q = 0.0f;
  for (int i = 0; i < waves; ++i) {
    x.s += lds.s[i]; x.q += lds.q[i];
  }
  return x;
}

// The 256 counters of digits, turned into the digit (counted from `last` on downwards) at which `want` keys are reached: lds.digit, how many
// are in the digits before it (lds.above) and in it (lds.count; 0 if there are not as many keys).  By the first wavefront.
__device__ __forceinline__ void digit_at_rank(LpLds& lds, const uint32_t* hist, uint32_t want, bool ascending) {
  const int lane = threadIdx.x & 63;
  uint32_t c[4], mine = 0;   // digits 4 lane .. + 3, in the order asked for
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int at = 4 * lane + q;
    c[q] = hist[ascending ? at : 255 - at];
    mine += c[q];
  }
  const uint32_t up = wave_prefix(mine);   // of this lane's digits and those before
  uint32_t run = up - mine;
  if (run < want && up >= want) {   // (one lane; none if there are fewer keys)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (run + c[q] >= want && run < want) {
        lds.digit = ascending ? 4 * lane + q : 255 - (4 * lane + q);
        lds.above = (int)run;
        lds.count = (int)c[q];
      }
      run += c[q];
    }
  }
  if (lane == 63 && up < want) {
    lds.digit = ascending ? 255 : 0; lds.above = (int)up; lds.count = 0;
  }
}

// A key with at least k of the block's keys at or above it, and at most `most` (>= k) if they differ: the digits of the k-th largest
// from the highest on, until few enough remain.  each(f): f(key) for the thread's keys.
template <typename Each>
__device__ __forceinline__ uint64_t key_at_rank(LpLds& lds, int k, int most, Each&& each) {
  const int tid = threadIdx.x;
  uint32_t* hist = lds.best;   // [256]
  uint64_t prefix = 0;
  int kept = 0;   // keys above the prefix's
  for (int shift = 56; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    each([&](uint64_t key) {
      if (key != 0 && (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8)))) atomicAdd(&hist[(key >> shift) & 255], 1u);
    });
    __syncthreads();
    if (tid < 64) digit_at_rank(lds, hist, (uint32_t)(k - kept), false);
    __syncthreads();
    prefix |= (uint64_t)lds.digit << shift;
    kept += lds.above;
    if (kept + lds.count <= most) break;
  }
  return prefix;
}

// The k largest keys, in order, to out(rank, key).  `mine`: the largest key of this thread's share, 0 without one; `highest`: the order of the
// largest value of all; rescan(f, t) calls f(key) for every key of the share that is at least t (and may for others).  The k-th largest of the
// threads' largest keys is a threshold that k keys reach, and few more.  It is found by counting the values by their distance from the largest, in
// 64ths of a factor of two: where the k-th lies is near enough unless many are about as large, or it lies 16 times lower.  Then, and for one or
// two, up to FEW_TOP by taking the largest values away until k are gone, else digit by digit.  (Us, 2000 x 10000 fp32, by distance / taken away /
// by digits: top 5 24 / 27 / -, 8 25 / 29 / -, 17 27 / - / 32, 64 35 / - / 41.)  What reaches the threshold is listed and ranked; if
// that is more than the list holds, or `exact`, the threshold comes from all keys.  At least k keys exist.
// (The threshold has to be close: a thread with a second key above it goes through its whole share again.  With the least of the largest
// keys of 8 groups of threads, about 22 keys at k = 5, 4096 x 50000 bf16 took 182 us.)
constexpr int FEW_TOP = 6, NEAR_BITS = 17;
template <typename Rescan, typename Out>
__device__ __forceinline__ void block_top(LpLds& lds, int k, uint64_t mine, uint32_t highest, bool exact, Rescan&& rescan, Out&& out) {
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t order = (uint32_t)(mine >> 32);
  uint64_t threshold = 0;
  bool found = exact;
  if (!found && k > 2) {
    uint32_t* hist = lds.best;
    __syncthreads();         // (lds.best may still be read)
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    if (mine != 0) atomicAdd(&hist[min((highest - order) >> NEAR_BITS, 255u)], 1u);
    __syncthreads();
    if (tid < 64) digit_at_rank(lds, hist, (uint32_t)k, true);
    __syncthreads();
    found = lds.digit < 255 && lds.above + lds.count <= k + 8 + k / 4;
    const uint32_t below = (uint32_t)(lds.digit + 1) << NEAR_BITS;   // (not below the order of -infinity)
    if (found) threshold = (uint64_t)max(highest - min(below, highest) + 1, 0x007FFFFFu) << 32;
  }
  if (!found && k <= FEW_TOP) {
    __syncthreads();
    lds.best[tid] = order;
    lds.column[tid] = (uint32_t)mine;
    __syncthreads();
    if (tid < 64) {
      uint32_t x[LP_WAVES], t = 0, c = 0;
#pragma unroll
      for (int w = 0; w < LP_WAVES; ++w) x[w] = lds.best[w * 64 + lane];
      // the largest of x, taken away, until `left` are gone; what is left of that is returned
      auto take = [&](int left, uint32_t& last, int& before) {
        while (left > 0) {
          last = 0;
#pragma unroll
          for (int w = 0; w < LP_WAVES; ++w) last = max(last, x[w]);
          last = wave_max(last);
          if (last == 0) break;
          before = left;
#pragma unroll
          for (int w = 0; w < LP_WAVES; ++w) {
            left -= __popcll(__ballot(x[w] == last));
            x[w] = x[w] == last ? 0 : x[w];
          }
        }
        return left;
      };
      int among = 0, ignored;
      if (take(k, t, among) < 0) {   // more equal ones than are wanted: the first of their columns
#pragma unroll
        for (int w = 0; w < LP_WAVES; ++w) x[w] = lds.best[w * 64 + lane] == t ? lds.column[w * 64 + lane] : 0;
        take(among, c, ignored);
      }
      if (tid == 0) lds.threshold = (uint64_t)t << 32 | c;
    }
    __syncthreads();
    threshold = lds.threshold;
  } else if (!found) {
    threshold = key_at_rank(lds, k, k + k / 4, [&](auto&& f) { f(mine); });
  }
  for (bool all = exact;; all = true) {
    if (all) threshold = key_at_rank(lds, k, LP_LIST, [&](auto&& f) { rescan(f, (uint64_t)0); });
    __syncthreads();
    if (tid == 0) lds.count = 0;
    __syncthreads();
    if (mine >= threshold || all)
      rescan(
          [&](uint64_t key) {
            if (key != 0 && key >= threshold) {
              const int at = atomicAdd(&lds.count, 1);   // (in any order: ranked below)
              if (at < LP_LIST) lds.list[at] = key;
            }
          },
          all ? (uint64_t)0 : threshold);
    __syncthreads();
    if (all || lds.count <= LP_LIST) break;
  }
  const int n = min(lds.count, LP_LIST);
  for (int i = tid; i < n; i += blockDim.x) {
    const uint64_t key = lds.list[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += lds.list[j] > key;
    if (above < k) out(above, key);
  }
}

// A row's results from its sums (by one thread).
__device__ __forceinline__ void write_row_stats(const LpArgs& a, int64_t row, const Softmax& t, float log_s) {
  const bool none = t.m == NEG_INF && t.s == 0.0f;
  const float h = none ? 0.0f : log_s - t.q / t.s;
  if (a.entropy) a.entropy[row] = h;
  if (a.stats) a.stats[row] = make_float4(t.m, log_s, h, 0.0f);
}
__device__ __forceinline__ float log_prob(const Softmax& t, float log_s, float x) {
  return t.m == NEG_INF && t.s == 0.0f ? NEG_INF : (x - Softmax::base(t.m)) - log_s;
}
// The logit of the row's given token (asked for at the start: two loads behind each other).
struct Given {
  bool there = false;
  float x = 0.0f;
  template <typename T>
  __device__ __forceinline__ void load(const LpArgs& a, const T* x_row, int64_t row) {
    if (!a.logp) return;
    const int64_t tok = a.tokens[row];
    there = tok >= 0 && tok < a.V;
    if (there) x = to_f32(x_row[tok]);
  }
  __device__ __forceinline__ void write(const LpArgs& a, int64_t row, const Softmax& t, float log_s) const {
    if (a.logp) a.logp[row] = there ? log_prob(t, log_s, x) : 0.0f;
  }
};

// A block per row, or per piece of one: its sums and top then go to memory for lp_join_kernel.  Rows: bound by memory and the vector units alike, 4096 x
// 50000 bf16 68 us (6.0 TB/s; vector instructions in 95 % of the cycles), with the top 5 99 (what a block does behind its row is not hidden).  Pieces: by the
// chain of loads and barriers, 1 x 1000000 fp32 with the top 10 7.0 us, the join 4.4.
template <typename T, bool TOP, bool STREAM>
__global__ __launch_bounds__(LP_THREADS, 6) void lp_kernel(LpArgs a) {
  __shared__ LpLds lds;
  const int64_t row = a.pieces == 1 ? blockIdx.x : blockIdx.x / (unsigned)a.pieces;
  const int piece = (int)(blockIdx.x - row * a.pieces), tid = threadIdx.x;
  typedef RowWalk<T, LP_THREADS, STREAM> W;
  const W walk(reinterpret_cast<const T*>(a.x) + row * a.ld, piece * a.piece, min((piece + 1) * a.piece, a.V));
  Given given;
  if (tid == 0 && a.pieces == 1) given.load(a, walk.row, row);
  constexpr int VN = W::VN, U = W::U;
  Softmax t;
  // of the thread: the group of logits that holds its first largest one, kept in LDS (a single one at the front), and the largest of the
  // other groups' largest
  __shared__ uint4 held[TOP ? U : 1][TOP ? LP_THREADS : 1];
  int64_t group = 0;
  int held_n = 0;   // logits in it
  float second = NEG_INF;
  auto note = [&](float vm, int64_t c, int n, auto&& words) {
    if (vm > t.m || (TOP && held_n == 0)) {
      if (TOP) {
        second = t.m;
        words();
        group = c;
        held_n = n;
      }
      t.rescale(fmaxf(vm, t.m));
    } else if (TOP) {
      second = fmaxf(second, vm);
    }
  };
  walk.each(
      tid,
      [&](const typename W::Words& w, int64_t c) {
        float v[U * VN];
#pragma unroll
        for (int q = 0; q < U; ++q) W::unpack(w.v[q], v + q * VN);
        note(largest(v), c, U * VN, [&] {
#pragma unroll
          for (int q = 0; q < U; ++q) held[q][tid] = w.v[q];
        });
        t.add_all(v);
      },
      [&](const uint4& w, int64_t c) {
        float v[VN];
        W::unpack(w, v);
        note(largest(v), c, VN, [&] { held[0][tid] = w; });
        t.add_all(v);
      },
      [&](float x, int64_t c) {
        note(x, c, 1, [&] { *reinterpret_cast<T*>(&held[0][tid]) = from_f32<T>(x); });
        t.template add<false>(x);
      });
  const float top_value = t.m;
  t = block_softmax(lds, t);
  const float log_s = logf(t.s);
  if constexpr (TOP) {
    // the group held: f(value, column)
    auto each_held = [&](auto&& f) {
#pragma unroll
      for (int q = 0; q < U; ++q) {
        float v[VN];
        W::unpack(held[q][tid], v);
#pragma unroll
        for (int e = 0; e < VN; ++e)
          if (q * VN + e < held_n) f(v[e], (uint32_t)(group + (int64_t)q * (LP_THREADS * VN) + e));
      }
    };
    uint32_t first = 0xFFFFFFFEu;
    each_held([&](float x, uint32_t c) { first = x == top_value ? min(first, c) : first; });
    const uint64_t mine = held_n ? rank_key(top_value, first) : 0;   // (of a row with a NaN any number: not asked for)
    block_top(
        lds, a.top, mine, value_order(t.m), t.s != t.s,
        [&](auto&& f, uint64_t least) {
          if (least == 0) {
            walk.each_column(tid, [&](float x, int64_t c) { f(rank_key(x, (uint32_t)c)); });
            return;
          }
          const float at_least = key_value(least);
          if (value_order(second) < (uint32_t)(least >> 32)) {   // none reaches it in the other groups
            each_held([&](float x, uint32_t c) {
              if (x >= at_least) f(rank_key(x, c));
            });
          } else {
            walk.again(tid, [&](float x, int64_t c) {
              if (x >= at_least) f(rank_key(x, (uint32_t)c));
            });
          }
        },
        [&](int r, uint64_t key) {
          if (a.pieces > 1) {   // (rank by rank: neighbours are of other pieces, so that every group of lp_join_kernel has a large one)
            a.part_top[(row * a.top + r) * a.pieces + piece] = key;
          } else {
            a.top_logp[row * a.top + r] = log_prob(t, log_s, key_value(key));
            a.top_index[row * a.top + r] = key_column(key);
          }
        });
  }
  if (tid == 0) {
    if (a.pieces > 1) {
      a.part[blockIdx.x] = make_float4(t.m, t.s, t.q, 0.0f);
    } else {
      write_row_stats(a, row, t, log_s);
      given.write(a, row, t, log_s);
    }
  }
}

// The pieces of a row put together: a block per row.
constexpr int JOIN_KEYS = 4096, JOIN_PIECES = LP_THREADS;   // pieces * top, pieces at most
template <typename T>
__global__ __launch_bounds__(LP_THREADS) void lp_join_kernel(LpArgs a) {
  __shared__ LpLds lds;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  // (everything is asked for first: the block's time is that of its loads behind each other)
  Given given;
  if (tid == 0) given.load(a, reinterpret_cast<const T*>(a.x) + row * a.ld, row);
  const int n = a.pieces * a.top;
  uint64_t key[JOIN_KEYS / LP_THREADS];
#pragma unroll
  for (int i = 0; i < JOIN_KEYS / LP_THREADS; ++i) {
    const int at = tid + i * LP_THREADS;
    key[i] = at < n ? a.part_top[row * n + at] : 0;
  }
  Softmax t;
  if (tid < a.pieces) {
    const float4 v = a.part[row * a.pieces + tid];
    t.m = v.x; t.s = v.y; t.q = v.z;
  }
  t = block_softmax(lds, t);
  const float log_s = logf(t.s);
  if (a.top > 0) {
    uint64_t mine = 0;
#pragma unroll
    for (uint64_t k : key) mine = max(mine, k);
    block_top(
        lds, a.top, mine, t.s != t.s ? 0xFFFFFFF0u : value_order(t.m), false,
        [&](auto&& f, uint64_t) {
#pragma unroll
          for (uint64_t k : key) f(k);
        },
        [&](int r, uint64_t k) {
          a.top_logp[row * a.top + r] = log_prob(t, log_s, key_value(k));
          a.top_index[row * a.top + r] = key_column(k);
        });
  }
  if (tid == 0) {
    write_row_stats(a, row, t, log_s);
    given.write(a, row, t, log_s);
  }
}

// Pieces of a row: with fewer rows than the chip holds blocks, until they fill it, but no shorter than a block's threads have
// two vectors each to read.
int lp_pieces(int64_t N, int64_t V, int32_t top) {
  int64_t p = std::min(JOIN_PIECES / std::max<int64_t>(N, 1), V / 4096);
  if (top > 0) p = std::min<int64_t>(p, JOIN_KEYS / top);
  return (int)std::max<int64_t>(p, 1);
}

// ------------------------------------------------------------- gradient
struct LpGradArgs {
  const void* x;
  void* dx;
  int64_t ld, ldd, N, V;
  const int32_t* tokens;
  const float4* stats;
  const float* d_logp;
  const float* d_entropy;
  int64_t pieces, piece;   // columns of a piece
};
constexpr int LG_THREADS = 256;

// One read and one write of the row, bound by memory: 4096 x 50000 bf16 136 us (6.0 TB/s); where both rows reach 16 bytes at different columns 314.
template <typename T, bool SAME, bool STREAM>   // SAME: both rows reach a 16-byte boundary at the same column
__global__ __launch_bounds__(LG_THREADS) void lp_grad_kernel(LpGradArgs a) {
  constexpr int VN = 16 / sizeof(T);
  for (int64_t id = blockIdx.x; id < a.N * a.pieces; id += gridDim.x) {
    const int64_t row = id / a.pieces, c0 = (id - row * a.pieces) * a.piece, c1 = min(c0 + a.piece, a.V);
    const float4 st = a.stats[row];
    int64_t tok = -1;
    float ga = 0.0f;
    if (a.d_logp) {
      tok = a.tokens[row];
      ga = tok >= 0 && tok < a.V ? a.d_logp[row] : 0.0f;
    }
    const float gb = a.d_entropy ? a.d_entropy[row] : 0.0f;
    const bool none = (st.x == NEG_INF && st.y == NEG_INF) || (ga == 0.0f && gb == 0.0f);
    T* out = reinterpret_cast<T*>(a.dx) + row * a.ldd;
    auto grad = [&](float x, int64_t c) {
      const float lp = (x - st.x) - st.y, p = __expf(lp);
      float g = ga * ((c == tok ? 1.0f : 0.0f) - p);
      if (gb != 0.0f) g -= p == 0.0f ? 0.0f : gb * p * (lp + st.z);
      return none ? 0.0f : g;
    };
    typedef RowWalk<T, LG_THREADS, false> W;
    const W walk(reinterpret_cast<const T*>(a.x) + row * a.ld, c0, c1);
    if constexpr (SAME) {
      auto vector = [&](const uint4& w, int64_t c) {
        float g[VN];
        W::unpack(w, g);
#pragma unroll
        for (int e = 0; e < VN; ++e) g[e] = grad(g[e], c + e);
        if constexpr (VN == 4) store16<STREAM>(out + c, bits4(g[0], g[1], g[2], g[3]));
        else store16<STREAM>(out + c, make_uint4(f2bf2(g[0], g[1]), f2bf2(g[2], g[3]), f2bf2(g[4], g[5]), f2bf2(g[6], g[7])));
      };
      walk.each(
          threadIdx.x,
          [&](const typename W::Words& w, int64_t c) {
#pragma unroll
            for (int q = 0; q < W::U; ++q) vector(w.v[q], c + (int64_t)q * (LG_THREADS * VN));
          },
          vector, [&](float x, int64_t c) { out[c] = from_f32<T>(grad(x, c)); });
    } else {
      for (int64_t c = c0 + threadIdx.x; c < c1; c += LG_THREADS) out[c] = from_f32<T>(grad(to_f32(walk.row[c]), c));
    }
  }
}

}  // namespace
}  // namespace antdt

using namespace antdt;

static int lp_sizes(const char* call, int64_t N, int64_t V, int32_t top) {
  if (N < 0 || N >= INT32_MAX / 4 || V < 1 || V >= INT32_MAX) return op_fail(ANTDT_INVALID_ARG, "%s: N or V out of range", call);
  if (top < 0 || top > ANTDT_MAX_TOP || top > V) return op_fail(ANTDT_INVALID_ARG, "%s: top must be 0 .. min(V, %d)", call, ANTDT_MAX_TOP);
  return ANTDT_OK;
}
static size_t lp_bytes(int64_t N, int64_t V, int32_t top) {
  const int64_t p = lp_pieces(N, V, top);
  return N == 0 || p == 1 ? 0 : (size_t)(N * p) * (sizeof(float4) + 8 * (size_t)top);
}

extern "C" {

int antdt_token_logprobs_bytes(int64_t N, int64_t V, int32_t top, size_t* bytes) {
  const char* call = "antdt_token_logprobs_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(lp_sizes(call, N, V, top));
  *bytes = lp_bytes(N, V, top);
  return ANTDT_OK;
}

int antdt_token_logprobs(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int32_t* tokens, float* logp, float* entropy,
                         float* stats, int32_t top, float* top_logp, int32_t* top_index, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "antdt_token_logprobs";
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  OP_TRY(lp_sizes(call, N, V, top));
  OP_TRY(op_matrix(call, "logits", logits, N, V, ld, op_size(dtype)));
  if (N == 0) return ANTDT_OK;
  if (logp) OP_TRY(op_matrix(call, "tokens", tokens, N, 1, 1, 4));
  if (logp) OP_TRY(op_matrix(call, "logp", logp, N, 1, 1, 4));
  if (entropy) OP_TRY(op_matrix(call, "entropy", entropy, N, 1, 1, 4));
  if (stats) OP_TRY(op_matrix(call, "stats", stats, N, 4, 4, 16));
  if (top) OP_TRY(op_matrix(call, "top_logp", top_logp, N, top, top, 4));
  if (top) OP_TRY(op_matrix(call, "top_index", top_index, N, top, top, 4));
  OP_TRY(op_workspace(call, workspace, workspace_bytes, lp_bytes(N, V, top)));
  LpArgs a = {};
  a.x = logits; a.ld = ld; a.N = N; a.V = V; a.tokens = tokens; a.logp = logp; a.entropy = entropy;
  a.stats = reinterpret_cast<float4*>(stats); a.top_logp = top_logp; a.top_index = top_index; a.top = top;
  a.pieces = lp_pieces(N, V, top);
  a.piece = div_up(V, a.pieces);   // (at least 4096 columns and at most 512 pieces: the last is not shorter than `top`)
  if (a.pieces > 1) {
    a.part = reinterpret_cast<float4*>(workspace);
    a.part_top = reinterpret_cast<uint64_t*>(a.part + N * a.pieces);
  }
  const hipStream_t s = (hipStream_t)stream;
  const bool far = N * V * op_size(dtype) > STREAM_BYTES;
  auto go = [&](auto t, auto with_top, const LpArgs& rows) {
    typedef decltype(t) T;
    constexpr bool TOP = decltype(with_top)::value;
    const dim3 grid((unsigned)(rows.N * rows.pieces));
    if (far) hipLaunchKernelGGL((lp_kernel<T, TOP, true>), grid, dim3(LP_THREADS), 0, s, rows);
    else hipLaunchKernelGGL((lp_kernel<T, TOP, false>), grid, dim3(LP_THREADS), 0, s, rows);
  };
  auto typed = [&](auto t, const LpArgs& rows) {
    if (top) go(t, std::true_type(), rows);
    else go(t, std::false_type(), rows);
  };
  for (int64_t r = 0; r < N; r += ROWS_OF_A_LAUNCH) {
    LpArgs rows = a;
    rows.N = std::min(ROWS_OF_A_LAUNCH, N - r);
    rows.x = reinterpret_cast<const char*>(a.x) + r * ld * op_size(dtype);
    if (logp) { rows.tokens += r; rows.logp += r; }
    if (entropy) rows.entropy += r;
    if (stats) rows.stats += r;
    if (top) { rows.top_logp += r * top; rows.top_index += r * top; }
    if (dtype == ANTDT_F32) typed(0.0f, rows);
    else typed((bf16_t)0, rows);
  }
  OP_TRY(op_hip(call, hipGetLastError()));
  if (a.pieces > 1) {
    if (dtype == ANTDT_F32) hipLaunchKernelGGL(lp_join_kernel<float>, dim3((unsigned)N), dim3(LP_THREADS), 0, s, a);
    else hipLaunchKernelGGL(lp_join_kernel<bf16_t>, dim3((unsigned)N), dim3(LP_THREADS), 0, s, a);
  }
  return op_hip(call, hipGetLastError());
}

int antdt_token_logprobs_gradient(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int32_t* tokens, const float* stats,
                                  const float* d_logp, const float* d_entropy, void* d_logits, int64_t ldd, void* stream) {
  const char* call = "antdt_token_logprobs_gradient";
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  OP_TRY(lp_sizes(call, N, V, 0));
  OP_TRY(op_matrix(call, "logits", logits, N, V, ld, op_size(dtype)));
  OP_TRY(op_matrix(call, "d_logits", d_logits, N, V, ldd, op_size(dtype)));
  OP_TRY(op_matrix(call, "stats", stats, N, 4, 4, 16));
  if (d_logp) OP_TRY(op_matrix(call, "d_logp", d_logp, N, 1, 1, 4));
  if (d_logp) OP_TRY(op_matrix(call, "tokens", tokens, N, 1, 1, 4));
  if (d_entropy) OP_TRY(op_matrix(call, "d_entropy", d_entropy, N, 1, 1, 4));
  if (N == 0) return ANTDT_OK;
  LpGradArgs a = {};
  a.x = logits; a.dx = d_logits; a.ld = ld; a.ldd = ldd; a.N = N; a.V = V; a.tokens = tokens;
  a.stats = reinterpret_cast<const float4*>(stats); a.d_logp = d_logp; a.d_entropy = d_entropy;
  // (fewer columns a block where that leaves compute units idle)
  a.piece = 8192;
  while (a.piece > 2048 && N * div_up(V, a.piece) < 2048) a.piece /= 2;
  a.pieces = div_up(V, a.piece);
  const int64_t size = op_size(dtype);
  const bool same = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(d_logits)) & 15) == 0 && ((ld - ldd) * size) % 16 == 0;
  const dim3 grid((unsigned)std::min<int64_t>(N * a.pieces, 1 << 20));
  const hipStream_t s = (hipStream_t)stream;
  const bool far = N * V * size > STREAM_BYTES;
  auto go = [&](auto t) {
    typedef decltype(t) T;
    if (same && far) hipLaunchKernelGGL((lp_grad_kernel<T, true, true>), grid, dim3(LG_THREADS), 0, s, a);
    else if (same) hipLaunchKernelGGL((lp_grad_kernel<T, true, false>), grid, dim3(LG_THREADS), 0, s, a);
    else hipLaunchKernelGGL((lp_grad_kernel<T, false, false>), grid, dim3(LG_THREADS), 0, s, a);
  };
  if (dtype == ANTDT_F32) go(0.0f);
  else go((bf16_t)0);
  return op_hip(call, hipGetLastError());
}

}  // extern "C"
