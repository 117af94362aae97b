// Block-level matrix products of the gated feed-forward block, of bf16 or fp32 operands, on the gfx950 matrix cores:
//
//   acc[b][i][j] += sum_{k < len} A(m, k) * B_b(n, k),   b < NB
//
// with the operands of mfma.h (contiguous or strided along the contraction), moved to LDS the same way, STAGES deep.  With NB = 2 one tile of
// A is multiplied with a tile of each of two matrices, whose columns a wavefront holds side by side.
//   bf16: v_mfma_f32_32x32x16_bf16.
//   fp32: v_mfma_f32_32x32x2_f32 (fp32 products and sums); a lane's four slots of a step are four MFMAs.
// What bounds it is LDS: a wavefront's tile of 128 x 64 reads 96 bytes a cycle of a compute unit at the matrix cores' full rate, and the loads write
// another 32 of the 128 there are.  So
//  - the first fragments of a stage are read before the last multiplications of the one before (read behind its barrier they cost a fifth of the
//    time: 8192 x 2048 x 2 x 5632 336 us, so 327);
//  - large bf16 tiles are four wavefronts of 128 x 128 (64 and 32 bytes a cycle), one a SIMD.  Nothing else then fills the matrix core while a
//    wavefront issues reads and loads, so these go between its multiplications one at a time, stages of 32 slots, four deep: 322 us, and the
//    backward pass's products with what goes before them 727 / 699.  (Not interleaved: 362 and 770.)
#pragma once

#include "mfma.h"

namespace antdt {

typedef float f32x4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void load_lds4(const void* src, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(lds), "v"(src) : "memory");
}
__device__ __forceinline__ void load_lds4(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, %2" ::"{m0}"(lds), "v"(off), "s"(base) : "memory");
}

// BR rows x BK contraction slots of one operand.  PIECE: bytes that a lane moves at a time, 16 or (fp32 rows of any alignment and
// length) 4.
template <typename T, int BR, int BK, bool STRIDED, int PIECE>
struct ProductTile;

template <int BR, int BK, bool STRIDED>
struct ProductTile<bf16_t, BR, BK, STRIDED, 16> {
  typedef OperandTile<BR, BK, STRIDED> Base;
  typedef bf16x8 Fragment;
  static constexpr int STEP = 16, BYTES = Base::BYTES, PIECES = Base::SLOTS, PITCH = Base::PITCH;
  // (four 16-byte slots a row: rows 4 apart would meet in the same banks)
  static __device__ __forceinline__ int swizzle(int r) { return !STRIDED && PITCH == 4 ? (r >> 2) & 3 : Base::swizzle(r); }
  static __device__ __forceinline__ void piece(int slot, int64_t ld, int rows, int r0, uint32_t& off, int& k) {
    const int r = slot / PITCH, c = (slot % PITCH) ^ swizzle(r);
    if (!STRIDED) {
      k = c * 8;
      off = (uint32_t)(min(r, rows - 1 - r0) * ld + k) * 2;
    } else {
      k = r;
      off = (uint32_t)(r * ld + min(c * 8, ((rows - 1) & ~7) - r0)) * 2;
    }
  }
  static __device__ __forceinline__ Fragment fragment(const char* tile, int r0, int kk, int lane) {
    if constexpr (!STRIDED && PITCH == 4) {
      const int r = r0 + (lane & 31), c = (kk >> 3) + (lane >> 5);
      return *reinterpret_cast<const bf16x8*>(tile + (r * PITCH + (c ^ swizzle(r))) * 16);
    } else {
      return Base::fragment(tile, r0, kk, lane);
    }
  }
  static __device__ __forceinline__ void multiply(const Fragment& a, const Fragment& b, f32x16& acc) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, acc, 0, 0, 0);
  }
};

template <int BR, int BK, bool STRIDED, int PIECE>
struct ProductTile<float, BR, BK, STRIDED, PIECE> {
  typedef f32x4v Fragment;
  static constexpr int STEP = 8, BYTES = BR * BK * 4, PIECES = BYTES / PIECE;
  static constexpr int PITCH = STRIDED ? BR / 4 : BK / 4;   // 16-byte slots per LDS row
  // Contiguous operands are read 16 bytes down a column of slots; strided ones a word from 32 neighbours of a row.
  static_assert(BK == 32, "eight slots a row");
  static __device__ __forceinline__ int swizzle(int r) { return STRIDED ? 0 : (r >> 1) & 7; }
  static __device__ __forceinline__ void piece(int at, int64_t ld, int rows, int r0, uint32_t& off, int& k) {
    const int slot = PIECE == 16 ? at : at >> 2, e = PIECE == 16 ? 0 : at & 3;
    const int r = slot / PITCH, c = ((slot % PITCH) ^ swizzle(r)) * 4 + e;
    if (!STRIDED) {
      k = c;
      off = (uint32_t)(min(r, rows - 1 - r0) * ld + k) * 4;
    } else {
      k = r;
      off = (uint32_t)(r * ld + min(c, (PIECE == 16 ? (rows - 1) & ~3 : rows - 1) - r0)) * 4;
    }
  }
  // Contraction slots kk + 4 (lane / 32) + e, e < 4, of row r0 + lane % 32.
  static __device__ __forceinline__ Fragment fragment(const char* tile, int r0, int kk, int lane) {
    const int r = r0 + (lane & 31), k = kk + 4 * (lane >> 5);
    if (!STRIDED) return *reinterpret_cast<const Fragment*>(tile + (r * PITCH + ((k >> 2) ^ swizzle(r))) * 16);
    const float* p = reinterpret_cast<const float*>(tile) + k * BR + r;
    return Fragment{p[0], p[BR], p[2 * BR], p[3 * BR]};
  }
  static __device__ __forceinline__ void multiply(const Fragment& a, const Fragment& b, f32x16& acc) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(b[e], a[e], acc, 0, 0, 0);
  }
};

// One operand: its matrix, rows that exist, first row of the tile.
struct Operand {
  const void* x;
  int64_t ld;
  int rows, r0;
};

// WR x WC wavefronts of TM x (NB TN) MFMA tiles each.  Element e of acc[b][i][j] in a lane: row m = 32 i + lane % 32 of the wavefront's tile,
// column 32 j + 8 (e / 4) + 4 (lane / 32) + e % 4 of B_b's.
template <typename T, int NB, int TM, int TN, int WR, int WC, int BK, int STAGES, bool A_STRIDED, bool B_STRIDED, int PIECE>
struct TileProduct {
  static constexpr bool INTERLEAVED = TM * NB * TN >= 16;   // (else there are other wavefronts on the SIMD, or the loads' latency bounds the block)
  static constexpr int SLOTS = BK, NB_ = NB, TM_ = TM, TN_ = TN, WC_ = WC, WAVES = WR * WC;
  static constexpr int THREADS = 64 * WAVES, BM = 32 * TM * WR, BN = 32 * TN * WC;
  typedef ProductTile<T, BM, BK, A_STRIDED, PIECE> TA;
  typedef ProductTile<T, BN, BK, B_STRIDED, PIECE> TB;
  static constexpr int STEP = TA::STEP;
  static constexpr int STAGE_BYTES = TA::BYTES + NB * TB::BYTES, LDS_BYTES = STAGES * STAGE_BYTES;
  static constexpr int VA = TA::PIECES / THREADS, VB = TB::PIECES / THREADS;
  static_assert(VA * THREADS == TA::PIECES && VB * THREADS == TB::PIECES, "tile / thread count");
  typedef f32x16 Acc[NB][TM][TN];

  static __device__ __forceinline__ void load(const char* base, uint32_t off, uint32_t lds) {
    if constexpr (PIECE == 16) load_lds16(base, off, lds);
    else load_lds4(base, off, lds);
  }
  static __device__ __forceinline__ void load(const char* src, uint32_t lds) {
    if constexpr (PIECE == 16) load_lds16(src, lds);
    else load_lds4(src, lds);
  }
  static __device__ __forceinline__ const char* origin(const Operand& o, bool strided) {
    return reinterpret_cast<const char*>(o.x) + (strided ? (int64_t)o.r0 : (int64_t)o.r0 * o.ld) * (int64_t)sizeof(T);
  }

  // Every wavefront of the block calls it alike; `len` contraction slots (of bf16, a multiple of 8 unless both operands are strided).  The
  // LDS is free when it returns.
  static __device__ __forceinline__ void run(const Operand& a, const Operand (&b)[NB], int len, char* lds, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC;
    const uint32_t lds0 = lds_address(lds) + wave * (64 * PIECE);
    uint32_t oa[VA], ob[VB];
    int ka[VA], kb[VB];
#pragma unroll
    for (int i = 0; i < VA; ++i) TA::piece(tid + i * THREADS, a.ld, a.rows, a.r0, oa[i], ka[i]);
#pragma unroll
    for (int i = 0; i < VB; ++i) TB::piece(tid + i * THREADS, b[0].ld, b[0].rows, b[0].r0, ob[i], kb[i]);
    const char* pa = origin(a, A_STRIDED);
    const char* pb[NB];
#pragma unroll
    for (int q = 0; q < NB; ++q) pb[q] = origin(b[q], B_STRIDED);
    const int64_t step_a = (A_STRIDED ? a.ld * BK : BK) * (int64_t)sizeof(T), step_b = (B_STRIDED ? b[0].ld * BK : BK) * (int64_t)sizeof(T);
    const int nk = len > 0 ? (len + BK - 1) / BK : 0;

    constexpr int PER_STAGE = VA + NB * VB, Q = BK / STEP;
    static_assert(Q % 2 == 0, "the fragments' two buffers in turn, over the stages too");
    int left = len;
    uint32_t fill = lds0;
    auto issue = [&]() {
      if (left >= BK) {
#pragma unroll
        for (int i = 0; i < VA; ++i) load(pa, oa[i], fill + i * (THREADS * PIECE));
#pragma unroll
        for (int q = 0; q < NB; ++q)
#pragma unroll
          for (int i = 0; i < VB; ++i) load(pb[q], ob[i], fill + TA::BYTES + q * TB::BYTES + i * (THREADS * PIECE));
      } else {
        const char* zero = reinterpret_cast<const char*>(mfma_zero16);
#pragma unroll
        for (int i = 0; i < VA; ++i) load(ka[i] < left ? pa + oa[i] : zero, fill + i * (THREADS * PIECE));
#pragma unroll
        for (int q = 0; q < NB; ++q)
#pragma unroll
          for (int i = 0; i < VB; ++i) load(kb[i] < left ? pb[q] + ob[i] : zero, fill + TA::BYTES + q * TB::BYTES + i * (THREADS * PIECE));
      }
      pa += step_a;
#pragma unroll
      for (int q = 0; q < NB; ++q) pb[q] += step_b;
      left -= BK;
      fill = fill == lds0 + (STAGES - 1) * STAGE_BYTES ? lds0 : fill + STAGE_BYTES;
    };
    constexpr int LDS_READS_DONE = 0xC07F;   // lgkmcnt(0) alone
    typename TA::Fragment af[2][TM];
    typename TB::Fragment bf[2][NB][TN];
    auto fetch = [&](const char* la, int q, int to) {
      const char* lb = la + TA::BYTES;
#pragma unroll
      for (int i = 0; i < TM; ++i) af[to][i] = TA::fragment(la, (wr * TM + i) * 32, q * STEP, lane);
#pragma unroll
      for (int s = 0; s < NB; ++s)
#pragma unroll
        for (int j = 0; j < TN; ++j) bf[to][s][j] = TB::fragment(lb + s * TB::BYTES, (wc * TN + j) * 32, q * STEP, lane);
    };
    if constexpr (INTERLEAVED) {
      // The next step's fragments, then the loads, between the multiplications.
      constexpr int MF = TM * NB * TN, FR = TM + NB * TN, LOADS = PER_STAGE / Q;
      static_assert(LOADS * Q == PER_STAGE && FR + 2 * LOADS <= MF && STAGES >= 3, "room between the multiplications");
      auto fetch_one = [&](const char* la, int q, int to, int f) {
        if (f < TM) af[to][f] = TA::fragment(la, (wr * TM + f) * 32, q * STEP, lane);
        else bf[to][(f - TM) / TN][(f - TM) % TN] =
            TB::fragment(la + TA::BYTES + (f - TM) / TN * TB::BYTES, (wc * TN + (f - TM) % TN) * 32, q * STEP, lane);
      };
      auto load_one = [&](auto kind, int i) {
        const int q = i < VA ? 0 : (i - VA) / VB, j = i < VA ? i : (i - VA) % VB;
        const char* base = i < VA ? pa : pb[q];
        const uint32_t off = i < VA ? oa[j] : ob[j], to = fill + (i < VA ? 0 : TA::BYTES + q * TB::BYTES) + j * (THREADS * PIECE);
        if constexpr (decltype(kind)::value == 1) load(base, off, to);
        else load((i < VA ? ka[j] : kb[j]) < left ? base + off : reinterpret_cast<const char*>(mfma_zero16), to);
      };
#pragma unroll
      for (int t = 0; t < STAGES - 1; ++t)
        if (t < nk) issue();
      if (nk == 0) return;
      if (STAGES - 2 < nk) wait_loads<(STAGES - 2) * PER_STAGE>();
      else wait_loads<0>();
      block_barrier();
      fetch(lds, 0, 0);
      uint32_t read = 0;
      int t = 0;
      // Stage t, with the loads of stage t + STAGES - 1 (KIND 0: there is none; 1: a whole one; 2: the last one, partly filled).
      auto stage = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        const uint32_t next = read == (STAGES - 1) * STAGE_BYTES ? 0 : read + STAGE_BYTES;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          if (q + 1 == Q) {
            // this wavefront has read stage t, and its loads of stage t + 1 are there: behind them only stage t + 2 and what went of t + 3
            __builtin_amdgcn_s_waitcnt(LDS_READS_DONE);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (KIND != 0) {
              static_assert(STAGES == 4, "the stages behind it");
              wait_loads<(STAGES - 3) * PER_STAGE + (Q - 1) * LOADS>();
              block_barrier();
            } else if (t + 1 < nk) {
              wait_loads<0>();
              block_barrier();
            }
          }
          const char* from = lds + (q + 1 < Q ? read : next);   // (behind the last stage whatever lies there)
#pragma unroll
          for (int m = 0; m < MF; ++m) {
            const int i = m / (NB * TN), sj = m % (NB * TN);
            TA::multiply(af[q & 1][i], bf[q & 1][sj / TN][sj % TN], acc[sj / TN][i][sj % TN]);
            __builtin_amdgcn_sched_barrier(0);
            if (m < FR) fetch_one(from, q + 1 < Q ? q + 1 : 0, (q + 1) & 1, m);
            else if (KIND != 0 && (m - FR) % 2 == 0 && (m - FR) / 2 < LOADS) load_one(kind, q * LOADS + (m - FR) / 2);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if constexpr (KIND != 0) {
          pa += step_a;
#pragma unroll
          for (int q = 0; q < NB; ++q) pb[q] += step_b;
          left -= BK;
          fill = fill == lds0 + (STAGES - 1) * STAGE_BYTES ? lds0 : fill + STAGE_BYTES;
        }
        read = next;
        ++t;
      };
      while (left >= BK) stage(std::integral_constant<int, 1>());
      if (left > 0) stage(std::integral_constant<int, 2>());
      while (t < nk) stage(std::integral_constant<int, 0>());
      block_barrier();
      return;
    }
    // Stage t is in LDS, and everybody's fragments of the stage before have been read.
    auto arrived = [&](int t) {
      if (t + STAGES - 2 < nk) wait_loads<(STAGES - 2) * PER_STAGE>();
      else wait_loads<0>();
      block_barrier();
    };
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t)
      if (t < nk) issue();
    if (nk == 0) return;
    arrived(0);
    fetch(lds, 0, 0);
    // (the last buffer is free from the start)
    if (left > 0) issue();
    uint32_t read = 0;
    for (int t = 0; t < nk; ++t) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (q + 1 < Q) {
          fetch(lds + read, q + 1, (q + 1) & 1);
        } else {
          // (said so that the compiler knows: else it waits for the fragments requested below before the multiplications)
          __builtin_amdgcn_s_waitcnt(LDS_READS_DONE);
          __builtin_amdgcn_sched_barrier(0);
          if (t + 1 < nk) {
            read = read == (STAGES - 1) * STAGE_BYTES ? 0 : read + STAGE_BYTES;
            arrived(t + 1);
            fetch(lds + read, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int s = 0; s < NB; ++s)
#pragma unroll
            for (int j = 0; j < TN; ++j) TA::multiply(af[q & 1][i], bf[q & 1][s][j], acc[s][i][j]);
        __builtin_amdgcn_sched_barrier(0);
        if (q + 1 == Q && left > 0) issue();
      }
    }
    block_barrier();
  }
};

}  // namespace antdt
