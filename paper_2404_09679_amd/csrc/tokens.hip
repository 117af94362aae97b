// Rows of a table for a sequence of tokens, their gradient, and the dropout: one pass over the data each.
#include <algorithm>
#include <initializer_list>
#include <utility>

#include "ops.h"
#include "sort.h"

namespace antdt {
namespace {

// ------------------------------------------------------------- lookup and dropout
// y[r, :] = residual[r, :] + dropout(scale * x[row(r), :]), row(r) = r or tokens[r].  8 columns a lane: the generator's draw, and 16 bytes of bf16.
// Dropout is bound by memory: 65536 x 1024 bf16 with residual 71.6 us (5.6 TB/s, a large copy's rate).  A lookup waits for a token and then for its row:
// 131072 tokens of 200000 x 256 bf16 28 us for 91 MB, without dropout 26.5, with table and result in the last-level cache 19 and 17.6.
struct RowsArgs {
  const void* x;
  const void* residual;
  void* y;
  const int32_t* tokens;
  int64_t ldx, ldr, ldy, rows, cols, V;
  int32_t lanes_log2;   // lanes of a row, of 8 columns each (in turns where that is fewer than the row has)
  float scale;
  DropArgs drop;
};

template <typename TI, typename TO, int Q, bool LOOKUP, bool RESIDUAL, bool DROP>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a) {
  const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1);
  const int64_t step = (int64_t)gridDim.x << (8 - a.lanes_log2);
  const DropKey key(a.drop);
  const float scale = a.scale * a.drop.factor;
  for (int64_t r = ((int64_t)blockIdx.x << (8 - a.lanes_log2)) + (threadIdx.x >> a.lanes_log2); r < a.rows; r += step) {
    int64_t from = r;
    if (LOOKUP) from = a.tokens[r];
    const bool there = !LOOKUP || (from >= 0 && from < a.V);
    const TI* x = reinterpret_cast<const TI*>(a.x) + (there ? from : 0) * a.ldx;
    TO* y = reinterpret_cast<TO*>(a.y) + r * a.ldy;
    for (int64_t c = 8 * (int64_t)lane; c < a.cols; c += (int64_t)8 << a.lanes_log2) {
      const int n = (int)min((int64_t)8, a.cols - c);
      float v[8] = {};
      if (there) {
        load8<Q>(x + c, n, v);
        if (DROP) {
          drop8(a.drop, key, r, (uint32_t)(c >> 3), scale, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= scale;
        }
      }
      if (RESIDUAL) {
        float b[8];
        load8<Q>(reinterpret_cast<const TO*>(a.residual) + r * a.ldr + c, n, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += b[e];
      }
      store8<Q>(y + c, n, v);
    }
  }
}

// Lanes of a row of `cols` columns, as a power of two.
int row_lanes_log2(int64_t cols, int most_log2) {
  int l = 0;
  while (l < most_log2 && ((int64_t)8 << l) < cols) ++l;
  return l;
}

template <typename TI, typename TO, bool LOOKUP, bool RESIDUAL, bool DROP>
hipError_t launch_rows(RowsArgs a, int quantum, hipStream_t s) {
  a.lanes_log2 = row_lanes_log2(a.cols, 8);
  const dim3 grid((unsigned)std::min<int64_t>(div_up(a.rows, 256 >> a.lanes_log2), 16384));
  if (quantum == 8) hipLaunchKernelGGL((rows_kernel<TI, TO, 8, LOOKUP, RESIDUAL, DROP>), grid, dim3(256), 0, s, a);
  else if (quantum == 4) hipLaunchKernelGGL((rows_kernel<TI, TO, 4, LOOKUP, RESIDUAL, DROP>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rows_kernel<TI, TO, 1, LOOKUP, RESIDUAL, DROP>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------- gradient of the table
// grad[v, :] = scale * sum over the n with tokens[n] == v of dropout(dy[n, :]).  The positions are sorted by token (stable, so a
// row's sum is in the order of the sequence).  L lanes walk C positions of the sorted list, 8 columns each, adding up dy rows and
// writing a row whenever the token changes; a block has 256 / L such walks behind each other and puts the ends of its walks together in LDS.
// Bound by the chain of loads (a token, its position, the row; 8 rows under way): 131072 tokens of 256 bf16 columns 26.5 us for 93 MB, without
// dropout 22.4.
// A run of one token over several blocks leaves a partial sum per block: slot 0 for a run that came in from the block before, slot 1
// for one that starts in it and goes on; a second launch adds them up.
struct GradArgs {
  const int32_t* key;     // tokens ascending, padding (V) last
  const int32_t* pay;     // their positions
  const void* dy;
  float* grad;
  float* partial;         // [chunks, 2, ldp]
  int64_t lddy, ldg, ldp, N, V, D;
  int32_t walk, chunk, chunks, lanes_log2;   // positions of a walk and of a block, blocks
  float scale;
  DropArgs drop;
};

// Keys and positions of the sort; further blocks clear their part of the gradient.
__global__ __launch_bounds__(256) void token_keys_kernel(const int32_t* tokens, int32_t* key, int32_t* pay, int N, int V, ClearPart clear) {
  if ((int)blockIdx.x >= clear.first) {
    clear_part<256>(clear);
    return;
  }
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < N) {
    const int t = tokens[i];
    key[i] = t >= 0 && t < V ? t : V;
    pay[i] = i;
  }
}
// The same and the whole sort, of as many tokens as one block sorts (the first; 3001 tokens: launches of 5.5 and 8.2 us in one of 9).
template <int IT>
__global__ __launch_bounds__(SMALL_THREADS) void token_sort_kernel(const int32_t* tokens, int32_t* key_in, int32_t* pay_in, int32_t* key, int32_t* pay, int N,
                                                                   int V, int passes, int rb, ClearPart clear) {
  __shared__ SmallSortLds lds;
  extern __shared__ int32_t stage[];
  if (blockIdx.x > 0) {
    clear_part<SMALL_THREADS>(clear);
    return;
  }
  for (int i = threadIdx.x; i < N; i += SMALL_THREADS) {
    const int t = tokens[i];
    key_in[i] = t >= 0 && t < V ? t : V;
    pay_in[i] = i;
  }
  __syncthreads();   // (read by other threads of the block)
  sort_small_field<IT>(lds, stage, key_in, pay_in, key, pay, N, passes, rb);
}
template <int IT>
hipError_t launch_token_sort(const int32_t* tokens, const SortBuffers& sb, int N, int V, const SortPlan& sp, const ClearRows& clear, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int bytes = SMALL_THREADS * IT * 4;
  const hipError_t e = allow_lds(token_sort_kernel<IT>, bytes, (int)sizeof(SmallSortLds), allowed);
  if (e != hipSuccess) return e;
  const ClearPart part = {clear, 1, 0, 1};
  hipLaunchKernelGGL(token_sort_kernel<IT>, dim3(1 + clear_blocks(part, SMALL_THREADS)), dim3(SMALL_THREADS), bytes, s, tokens, sb.key[1], sb.pay[1],
                     sb.key[0], sb.pay[0], N, V, sp.passes, sp.radix_bits, part);
  return hipGetLastError();
}

template <bool ACCUMULATE>
__device__ __forceinline__ void write_row(const GradArgs& a, int v, int64_t c, int n, bool vec, float (&x)[8]) {
  float* g = a.grad + (int64_t)v * a.ldg + c;
  if (vec) {
    if (ACCUMULATE) {
      float b[8];
      load8<4>(g, n, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += b[e];
    }
    store8<4>(g, n, x);
  } else {
    if (ACCUMULATE) {
      float b[8];
      load8<1>(g, n, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += b[e];
    }
    store8<1>(g, n, x);
  }
}

template <typename T, int Q, bool DROP, bool ACCUMULATE>
__global__ __launch_bounds__(256) void token_sum_kernel(GradArgs a, bool vec_grad) {
  // of the walks of the block: the sum of the run that came in and of the one that goes on, whether there is the one, and whether it is
  // the whole walk and goes on
  __shared__ float sums[2][256][8];
  __shared__ uint8_t came[256], through[256];
  const int lanes = 1 << a.lanes_log2, walks = 256 >> a.lanes_log2;
  const int lane = threadIdx.x & (lanes - 1), g = threadIdx.x >> a.lanes_log2;
  const int64_t c = 8 * (((int64_t)blockIdx.y << a.lanes_log2) + lane);
  const int64_t p0 = (int64_t)blockIdx.x * a.chunk + (int64_t)g * a.walk, p1 = min(p0 + a.walk, a.N);
  const int n = (int)max(min((int64_t)8, a.D - c), (int64_t)0);
  const DropKey dk(a.drop);
  const float scale = a.scale * a.drop.factor;
  const T* dy = reinterpret_cast<const T*>(a.dy) + c;

  bool has_in = false, is_through = false, has_out = false;
  int run = (int)a.V;
  if (p0 < a.N) {
    run = a.key[p0];
    const int before = a.key[max(p0 - 1, (int64_t)0)], behind = a.key[min(p1, a.N - 1)];   // (asked for here: one wait for all three)
    has_in = run < a.V && p0 > 0 && before == run;
    bool in = has_in;
    float sum[8] = {};
    if (n > 0) {
      constexpr int U = 8;
      for (int64_t p = p0; p < p1 && run < a.V; p += U) {
        int k[U], at[U];
        float x[U][8];
#pragma unroll
        for (int q = 0; q < U; ++q) {
          const int64_t i = min(p + q, p1 - 1);
          k[q] = a.key[i];
          at[q] = a.pay[i];
        }
#pragma unroll
        for (int q = 0; q < U; ++q) load8<Q, true>(dy + (int64_t)at[q] * a.lddy, n, x[q]);
#pragma unroll
        for (int q = 0; q < U; ++q) {
          if (p + q >= p1 || run >= a.V) continue;
          if (k[q] != run) {
            if (in) store8<4>(sums[0][threadIdx.x], 8, sum);
            else write_row<ACCUMULATE>(a, run, c, n, vec_grad, sum);
            in = false;
            run = k[q];
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
            if (run >= a.V) continue;
          }
          if (DROP) {
            drop8(a.drop, dk, at[q], (uint32_t)(c >> 3), scale, x[q]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[q][e];
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = fmaf(x[q][e], scale, sum[e]);
          }
        }
      }
    } else {   // (a lane without columns: the flags alone)
      run = a.key[p1 - 1];
      in = has_in && run == a.key[p0];
    }
    if (run < a.V) {
      const bool goes_on = p1 < a.N && behind == run;
      is_through = in && goes_on;
      has_out = !in && goes_on;
      if (in) store8<4>(sums[0][threadIdx.x], 8, sum);
      else if (goes_on) store8<4>(sums[1][threadIdx.x], 8, sum);
      else if (n > 0) write_row<ACCUMULATE>(a, run, c, n, vec_grad, sum);
    }
  }
  if (lane == 0) {
    came[g] = has_in; through[g] = is_through;
  }
  __syncthreads();
  float* slots = a.partial + (int64_t)blockIdx.x * 2 * a.ldp + c;
  // the sums of the walks from q on that belong to the run, added to sum; whether it goes on behind the block
  auto follow = [&](int q, float (&sum)[8]) {
    for (; q < walks; ++q) {
      if (!came[q]) return false;
      float x[8];
      load8<4>(sums[0][q * lanes + lane], 8, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += x[e];
      if (!through[q]) return false;
    }
    return true;
  };
  float sum[8];
  if (has_out && n > 0) {
    load8<4>(sums[1][threadIdx.x], 8, sum);
    if (follow(g + 1, sum)) store8<4>(slots + a.ldp, 8, sum);
    else write_row<ACCUMULATE>(a, run, c, n, vec_grad, sum);
  }
  if (g == 0 && has_in && n > 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    follow(0, sum);
    store8<4>(slots, 8, sum);
  }
}

// Runs over several blocks of the first launch (`chunks` here): those over up to JOIN_FEW more are added up by the lanes of the chunk where
// they start, the others by a whole block.  (Bound by the chains of loads: how far a run goes is asked by all lanes at once.)
// Lookup and gradient with blocks of 1024 / 512 / 256 / 128 threads, us: 131072 tokens of 200000 x 256 bf16 126.1 / 125.5 / 125.2 / 126.4, 100000 of 1000000 x
// 32 fp32 98.5 / 94 / 90 / 89; JOIN_FEW 8 / 16 / 32 / 64 (1024 threads) 131.6 / 129.3 / 128.4 / 126.4 and 122.9 / 99.5 / 99.8 / 89.4 (of 256 no different).
constexpr int JOIN_THREADS = 256, JOIN_FEW = 32;
template <bool ACCUMULATE>
__global__ __launch_bounds__(JOIN_THREADS) void token_join_kernel(GradArgs a, bool vec_grad) {
  extern __shared__ float part[];   // [groups][8 lanes]
  __shared__ int many[JOIN_THREADS], n_many;
  const int groups = JOIN_THREADS >> a.lanes_log2, lanes = 1 << a.lanes_log2;
  const int lane = threadIdx.x & (lanes - 1), g = threadIdx.x >> a.lanes_log2;
  const int64_t c = 8 * (((int64_t)blockIdx.y << a.lanes_log2) + lane);
  const int n = (int)max(min((int64_t)8, a.D - c), (int64_t)0);
  if (threadIdx.x == 0) n_many = 0;
  __syncthreads();
  // the chunk behind j begins inside the run
  auto begins_in = [&](int64_t i, int run) { return i < a.chunks && a.key[i * a.chunk] == run; };
  // slot 0 of U chunks, `step` apart, up to `end`, added to sum
  constexpr int U = 8;
  auto add = [&](int64_t i, int64_t step, int64_t end, float (&sum)[8]) {
    float x[U][8];
#pragma unroll
    for (int q = 0; q < U; ++q) load8<4>(a.partial + min(i + q * step, end - 1) * 2 * a.ldp + c, 8, x[q]);
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (i + q * step < end) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += x[q][e];
      }
  };
  const int64_t j = (int64_t)blockIdx.x * groups + g;
  const int64_t behind = (j + 1) * a.chunk;
  if (j < a.chunks && behind < a.N) {
    const int run = a.key[behind - 1];
    const int64_t p0 = j * a.chunk;
    if (run < a.V && a.key[behind] == run && !(a.key[p0] == run && p0 > 0 && a.key[p0 - 1] == run)) {
      int more = 0, got = lanes;   // chunks that begin inside the run
      while (got == lanes && more <= JOIN_FEW) {
        const uint64_t yes = __ballot(begins_in(j + 1 + more + lane, run)) >> (threadIdx.x & 63 & ~(lanes - 1));
        got = __popcll(lanes == 64 ? yes : yes & ((1ull << lanes) - 1));
        more += got;
      }
      if (more > JOIN_FEW) {
        if (lane == 0) many[atomicAdd(&n_many, 1)] = (int)j;   // (in any order: each is summed by itself)
      } else if (n > 0) {
        float sum[8];
        load8<4>(a.partial + (j * 2 + 1) * a.ldp + c, 8, sum);
        for (int64_t i = j + 1; i <= j + more; i += U) add(i, 1, j + more + 1, sum);
        write_row<ACCUMULATE>(a, run, c, n, vec_grad, sum);
      }
    }
  }
  __syncthreads();
  for (int m = 0; m < n_many; ++m) {
    const int64_t from = many[m];
    const int run = a.key[(from + 1) * a.chunk - 1];
    int64_t lo = from + 1, hi = a.chunks;   // the first chunk that does not begin inside the run is in [lo, hi]
    while (lo < hi) {
      const int64_t step = (hi - lo + 63) / 64, at = lo + ((threadIdx.x & 63) + 1) * step - 1;
      const int in = __popcll(__ballot(at < hi && begins_in(at, run)));
      hi = min(hi, lo + (in + 1) * step - 1);
      lo += in * step;
    }
    float sum[8] = {};
    if (n > 0)
      for (int64_t i = from + 1 + g; i < hi; i += U * groups) add(i, groups, hi, sum);
    store8<4>(part + threadIdx.x * 8, 8, sum);
    __syncthreads();
    if (g == 0 && n > 0) {
      load8<4>(a.partial + (from * 2 + 1) * a.ldp + c, 8, sum);
      for (int q = 0; q < groups; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += part[(q * lanes + lane) * 8 + e];
      write_row<ACCUMULATE>(a, run, c, n, vec_grad, sum);
    }
    __syncthreads();
  }
}

// How the gradient's workspace is laid out.
struct GradPlan {
  int32_t passes, radix_bits, tiles, walk, chunk, chunks, lanes_log2;
  int64_t ldp;
  size_t key[2], pay[2], hist, digit_total, partial, bytes;
};
GradPlan grad_plan(int64_t N, int64_t V, int64_t D) {
  GradPlan p = {};
  int bits = 1;
  while ((1ll << bits) < V + 1) ++bits;   // keys 0 .. V
  p.passes = (bits + 9) / 10;
  p.radix_bits = (bits + p.passes - 1) / p.passes;
  p.tiles = (int32_t)div_up(N, ANTDT_SORT_TILE);
  p.lanes_log2 = row_lanes_log2(D, 6);
  p.ldp = div_up(D, 8) * 8;
  // Walks short enough that 2^18 threads find work, long enough that not most of them end inside a run.
  p.walk = (int32_t)std::max<int64_t>(8, div_up(N << p.lanes_log2, 1 << 18));
  p.chunk = p.walk * (256 >> p.lanes_log2);
  p.chunks = (int32_t)div_up(N, p.chunk);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  for (int q = 0; q < 2; ++q) {
    p.key[q] = take((size_t)N * 4);
    p.pay[q] = take((size_t)N * 4);
  }
  p.hist = take(((size_t)p.tiles << p.radix_bits) * 4);
  p.digit_total = take(((size_t)1 << p.radix_bits) * 4);
  p.partial = take((size_t)p.chunks * 2 * (size_t)p.ldp * 4);
  p.bytes = at;
  return p;
}

template <typename T, int Q, bool DROP>
hipError_t launch_token_sums(const GradArgs& a, bool accumulate, bool vec_grad, hipStream_t s) {
  const unsigned slices = (unsigned)div_up(a.D, (int64_t)8 << a.lanes_log2);
  const dim3 grid((unsigned)a.chunks, slices), join((unsigned)div_up(a.chunks, JOIN_THREADS >> a.lanes_log2), slices);
  constexpr int bytes = JOIN_THREADS * 8 * 4;
  if (accumulate) hipLaunchKernelGGL((token_sum_kernel<T, Q, DROP, true>), grid, dim3(256), 0, s, a, vec_grad);
  else hipLaunchKernelGGL((token_sum_kernel<T, Q, DROP, false>), grid, dim3(256), 0, s, a, vec_grad);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.chunks < 2) return e;
  if (accumulate) hipLaunchKernelGGL(token_join_kernel<true>, join, dim3(JOIN_THREADS), bytes, s, a, vec_grad);
  else hipLaunchKernelGGL(token_join_kernel<false>, join, dim3(JOIN_THREADS), bytes, s, a, vec_grad);
  return hipGetLastError();
}
template <typename T, bool DROP>
hipError_t launch_token_sums(const GradArgs& a, int quantum, bool accumulate, bool vec_grad, hipStream_t s) {
  if (quantum == 8) return launch_token_sums<T, 8, DROP>(a, accumulate, vec_grad, s);
  if (quantum == 4) return launch_token_sums<T, 4, DROP>(a, accumulate, vec_grad, s);
  return launch_token_sums<T, 1, DROP>(a, accumulate, vec_grad, s);
}

int token_sizes(const char* call, int64_t N, int64_t V, int64_t D) {
  if (N < 0 || N >= INT32_MAX || V < 0 || V >= INT32_MAX || D < 0 || D >= (1 << 24))
    return op_fail(ANTDT_INVALID_ARG, "%s: N, V or D out of range", call);
  return ANTDT_OK;
}

}  // namespace
}  // namespace antdt

using namespace antdt;

extern "C" {

int antdt_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int64_t cols, int32_t dtype,
                  const antdt_dropout_spec* drop, void* y, int64_t ldy, void* stream) {
  const char* call = "antdt_dropout";
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  if (!drop) return op_fail(ANTDT_INVALID_ARG, "%s: drop is null", call);
  if (cols >= INT32_MAX) return op_fail(ANTDT_INVALID_ARG, "%s: cols out of range", call);
  const int64_t size = op_size(dtype);
  RowsArgs a = {};
  bool none;
  OP_TRY(op_dropout(call, drop, a.drop, none));
  OP_TRY(op_matrix(call, "x", x, rows, cols, ldx, size));
  OP_TRY(op_matrix(call, "y", y, rows, cols, ldy, size));
  if (residual) OP_TRY(op_matrix(call, "residual", residual, rows, cols, ldr, size));
  if (rows == 0 || cols == 0) return ANTDT_OK;
  a.x = x; a.residual = residual; a.y = y; a.ldx = ldx; a.ldr = residual ? ldr : ldx; a.ldy = ldy; a.rows = rows; a.cols = cols; a.scale = 1.0f;
  const int q = row_quantum(cols, size, {{x, ldx}, {residual ? residual : x, a.ldr}, {y, ldy}});
  const hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (dtype == ANTDT_F32) e = residual ? launch_rows<float, float, false, true, true>(a, q, s) : launch_rows<float, float, false, false, true>(a, q, s);
  else e = residual ? launch_rows<bf16_t, bf16_t, false, true, true>(a, q, s) : launch_rows<bf16_t, bf16_t, false, false, true>(a, q, s);
  return op_hip(call, e);
}

int antdt_token_lookup(const void* table, int64_t ldt, int64_t V, int64_t D, int32_t dtype, const int32_t* tokens, int64_t N, float scale,
                       const antdt_dropout_spec* drop, void* out, int64_t ldo, int32_t out_dtype, void* stream) {
  const char* call = "antdt_token_lookup";
  if (!op_dtype(dtype) || !op_dtype(out_dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  OP_TRY(token_sizes(call, N, V, D));
  RowsArgs a = {};
  bool none;
  OP_TRY(op_dropout(call, drop, a.drop, none));
  OP_TRY(op_matrix(call, "table", table, V, D, ldt, op_size(dtype)));
  OP_TRY(op_matrix(call, "tokens", tokens, N, 1, 1, 4));
  OP_TRY(op_matrix(call, "out", out, N, D, ldo, op_size(out_dtype)));
  if (N == 0 || D == 0) return ANTDT_OK;
  a.x = table; a.y = out; a.tokens = tokens; a.ldx = ldt; a.ldy = ldo; a.rows = N; a.cols = D; a.V = V; a.scale = scale;
  const int q = std::min(row_quantum(D, op_size(dtype), {{table, ldt}}), row_quantum(D, op_size(out_dtype), {{out, ldo}}));
  const hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto ti, auto to) {
    return none ? launch_rows<decltype(ti), decltype(to), true, false, false>(a, q, s) : launch_rows<decltype(ti), decltype(to), true, false, true>(a, q, s);
  };
  const float f = 0.0f;
  const bf16_t b = 0;
  const hipError_t e = dtype == ANTDT_F32 ? (out_dtype == ANTDT_F32 ? go(f, f) : go(f, b)) : (out_dtype == ANTDT_F32 ? go(b, f) : go(b, b));
  return op_hip(call, e);
}

int antdt_token_gradient_bytes(int64_t N, int64_t V, int64_t D, size_t* bytes) {
  const char* call = "antdt_token_gradient_bytes";
  if (!bytes) return op_fail(ANTDT_INVALID_ARG, "%s: bytes is null", call);
  OP_TRY(token_sizes(call, N, V, D));
  *bytes = N == 0 || V == 0 || D == 0 ? 0 : grad_plan(N, V, D).bytes;
  return ANTDT_OK;
}

int antdt_token_gradient(const void* dy, int64_t lddy, int32_t dtype, const int32_t* tokens, int64_t N, float scale,
                         const antdt_dropout_spec* drop, float* grad, int64_t ldg, int64_t V, int64_t D, int32_t accumulate, void* workspace,
                         size_t workspace_bytes, void* stream) {
  const char* call = "antdt_token_gradient";
  if (!op_dtype(dtype)) return op_fail(ANTDT_INVALID_ARG, "%s: dtype", call);
  OP_TRY(token_sizes(call, N, V, D));
  GradArgs a = {};
  bool none;
  OP_TRY(op_dropout(call, drop, a.drop, none));
  OP_TRY(op_matrix(call, "dy", dy, N, D, lddy, op_size(dtype)));
  OP_TRY(op_matrix(call, "tokens", tokens, N, 1, 1, 4));
  OP_TRY(op_matrix(call, "grad", grad, V, D, ldg, 4));
  if (V == 0 || D == 0) return ANTDT_OK;
  const GradPlan pl = grad_plan(N, V, D);
  if (N > 0) OP_TRY(op_workspace(call, workspace, workspace_bytes, pl.bytes));
  if (N == 0 && accumulate) return ANTDT_OK;
  const hipStream_t s = (hipStream_t)stream;
  char* ws = reinterpret_cast<char*>(workspace);
  auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
  const bool whole = ldg == D && D % 4 == 0 && (reinterpret_cast<uintptr_t>(grad) & 15) == 0;
  const ClearRows clear = {accumulate ? nullptr : grad, ldg, V, D, whole};

  SortPlan sp = {};
  sp.F = 1; sp.passes = pl.passes; sp.radix_bits = pl.radix_bits; sp.total_tiles = pl.tiles; sp.rows = V + 1; sp.samples = N; sp.width = D;
  SortBuffers sb = {};
  sb.key[1] = N ? ints(pl.key[1]) : nullptr; sb.pay[1] = N ? ints(pl.pay[1]) : nullptr;
  sb.ids = sb.key[1]; sb.pay0 = sb.pay[1];   // (read by the first pass, written by the second)
  FieldPtr fp = {};
  TileBase tb = {};
  for (int f = 1; f <= ANTDT_MAX_FIELDS; ++f) {
    fp.p[f] = N;
    tb.t[f] = pl.tiles;
  }
  int sorted = 0;
  const int items = N ? small_sort_items(1, fp) : 0;
  if (items) {
    sb.key[0] = ints(pl.key[0]); sb.pay[0] = ints(pl.pay[0]);
    switch (items) {
      case 2: OP_TRY(op_hip(call, launch_token_sort<2>(tokens, sb, (int)N, (int)V, sp, clear, s))); break;
      case 4: OP_TRY(op_hip(call, launch_token_sort<4>(tokens, sb, (int)N, (int)V, sp, clear, s))); break;
      case 8: OP_TRY(op_hip(call, launch_token_sort<8>(tokens, sb, (int)N, (int)V, sp, clear, s))); break;
      default: OP_TRY(op_hip(call, launch_token_sort<16>(tokens, sb, (int)N, (int)V, sp, clear, s))); break;
    }
  } else {
    // A large gradient is cleared in parts beside all of the sort's launches, which leave the memory idle, a smaller one in this launch alone.  All
    // at once / in parts, us: 131072 tokens of 200000 x 256 98 / 93, 100000 of 1000000 x 48 79 / 73, of 2000 x 256 56.5 / 57.8.
    constexpr int64_t AT_ONCE = 32 << 20;
    const bool in_parts = N > 0 && !accumulate && V * D * 4 > AT_ONCE;
    const int parts = in_parts ? 1 + 3 * pl.passes : 1;
    const ClearPart part = {clear, (int32_t)div_up(N, 256), 0, parts};
    hipLaunchKernelGGL(token_keys_kernel, dim3((unsigned)(part.first + clear_blocks(part, 256))), dim3(256), 0, s, tokens, sb.key[1], sb.pay[1], (int)N,
                       (int)V, part);
    OP_TRY(op_hip(call, hipGetLastError()));
    if (N == 0) return ANTDT_OK;
    sb.key[0] = ints(pl.key[0]); sb.pay[0] = ints(pl.pay[0]);
    sb.hist = reinterpret_cast<uint32_t*>(ws + pl.hist); sb.digit_total = reinterpret_cast<uint32_t*>(ws + pl.digit_total);
    OP_TRY(op_hip(call, launch_sort(sp, sb, fp, tb, nullptr, s, &sorted, in_parts ? &clear : nullptr)));
  }

  a.key = sb.key[sorted]; a.pay = sb.pay[sorted];
  a.dy = dy; a.grad = grad; a.partial = reinterpret_cast<float*>(ws + pl.partial);
  a.lddy = lddy; a.ldg = ldg; a.ldp = pl.ldp; a.N = N; a.V = V; a.D = D;
  a.walk = pl.walk; a.chunk = pl.chunk; a.chunks = pl.chunks; a.lanes_log2 = pl.lanes_log2; a.scale = scale;
  const int q = row_quantum(D, op_size(dtype), {{dy, lddy}});
  const bool vec_grad = row_quantum(D, 4, {{grad, ldg}}) >= 4;
  hipError_t e;
  if (dtype == ANTDT_F32) e = none ? launch_token_sums<float, false>(a, q, accumulate != 0, vec_grad, s) : launch_token_sums<float, true>(a, q, accumulate != 0, vec_grad, s);
  else e = none ? launch_token_sums<bf16_t, false>(a, q, accumulate != 0, vec_grad, s) : launch_token_sums<bf16_t, true>(a, q, accumulate != 0, vec_grad, s);
  return op_hip(call, e);
}

}  // extern "C"
