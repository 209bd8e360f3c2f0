// The product of 8-bit operands with a factor for each block of 128 along k:
//
//   C[i][j] = sum_b s_P(i, b) s_Q(j, b) sum_{k in block b} P[i][k] Q[j][k]
//
// A step of the product's kernel is 128 bytes of k, one block: its products are added by the
// matrix cores from zero, and the step's sum enters C's in fp32, multiplied by its two factors.
//
// Into 16 bits the 8-bit matrix instruction of 128 k is used.  It lines up the products of eight
// consecutive k and cuts them, towards zero, to 2^-13 of the power of two that their largest pair of
// exponents gives (as measured, with one large and one small product at each place; the sums of
// eight are added with fp32's digits).  A product of two codes has eight digits, so one of up to a 64th of
// the largest loses none: 1.4e-5 of the results (2-norm) on normal data, 8.6e-5 where one column in eight
// is 1,000 times the others, started from zero for each block, against 2.1e-4 (fp16) and 1.7e-3 (bf16)
// of the output's rounding, which that makes larger by 8% at the most.  Into fp32 the codes are widened (exactly) to
// fp16 and products and sums are fp32's, at half the rate.
//
// The factors come into LDS with the operands: of the tile's rows, then of its columns, a dword a
// lane.  A lane multiplies its sums of a row by one factor (Q's blocks of 128 units:
// the wave's columns share theirs), or by the row's and by its columns' (blocks of one unit).
//
// Bound, large: a step's matrix instructions and the sums' entering, which take turns more than they
// overlap, and a tile's start and epilogue, which stand alone, since one workgroup fills a CU.  8,192 x
// 4,096 x 16,384 into bf16 (268 MB) takes 504 us, with GELU 556; of k = 512 128 and 192: so some 9 us a tile
// beside its steps (72 of the 504 us), GELU 6 to 8 more, and the rest steps of 1.7 us; the matrix cores are
// busy in 47% of the cycles with GELU.  8,192^3 into bf16 450 to 507 us over the cards measured on, 2,170 to
// 2,440 TFLOP/s; a variant without the factors took 442 us where with them it was 500, on zeros 359 and
// 391.  Factors of columns: 526 to 588, since a sum is multiplied twice (a tile's matrix
// instruction, four multiplications and four FMAs; else one and four).  Into fp32 903 to 942, 1,170 to
// 1,220.  Small, few rows: as the product's (one row of 4,096 x 4,096 6 us of device time).
#pragma once

#include "product.h"

namespace som {

struct BlockArgs : ProductArgs {
  const float *xs, *ws;                      // at (row >> shift) * row stride + (k / 128) * k stride
  int64_t xs_row, xs_k, ws_row, ws_k;
  int xs_shift, ws_shift;                    // 0 or 7
  bool exact;
};

ProductPlan plan_blocks(int64_t I, int64_t J, int64_t K, bool dma, bool exact);
hipError_t launch_blocks(BlockArgs a, float* partial, hipStream_t stream);

typedef int i8 __attribute__((ext_vector_type(8)));

// 128 k of 16 rows: chunks g and 4 + g of the lane's row (the same k in both operands, which is
// all that the order of k has to be).
struct Block8 {
  i4 half[2];
};
template <int BR>
__device__ __forceinline__ Block8 block_fragment(lds_char* step, uint32_t lane_base, int t) {
  Block8 b;
  b.half[0] = fragment<true, BR>(step, lane_base, t, 0);
  b.half[1] = fragment<true, BR>(step, lane_base, t, 1);
  return b;
}

// The block's sum, from zero.
template <bool EXACT>
__device__ __forceinline__ f4 block_sum(const Block8& q, const Block8& p) {
  f4 c = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (EXACT) {
#pragma unroll
    for (int h = 0; h < 2; ++h) c = mfma<kE4M3>(Frag<kE4M3>(q.half[h]), Frag<kE4M3>(p.half[h]), c);
  } else {
    union {
      i4 half[2];
      i8 all;
    } a, b;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      a.half[h] = q.half[h];
      b.half[h] = p.half[h];
    }
    // both E4M3 (format 0); scales of zero select the instruction without them
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.all, b.all, c, 0, 0, 0, 0, 0, 0);
  }
  return c;
}

// 4 bytes per lane from its own address to LDS at `lds` (uniform) + 4 * lane.
__device__ __forceinline__ void dma4(const float* p, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p), "{m0}"(lds) : "memory");
}

template <bool EXACT, bool UNITS, int WI, int WJ, int TI, int TJ, int NS>
__global__ void __launch_bounds__(WI* WJ * 64) k_product_blocks(const BlockArgs a) {
  constexpr int BI = WI * TI * 16, BJ = WJ * TJ * 16, THREADS = WI * WJ * 64;
  using OpP = Operand<1, true, BI, THREADS>;
  using OpQ = Operand<1, true, BJ, THREADS>;
  constexpr int kCodes = OpP::kBytes + OpQ::kBytes, kStage = kCodes + THREADS * 4;
  constexpr int kStep = 128, kTiles = TI * TJ, kRing = kTiles < 4 ? kTiles : 4, kLate = kRing - 1;
  static_assert(BI + BJ <= THREADS, "a dword of factors a thread");
  static_assert(kTiles % kRing == 0, "a tile's place in the ring is the same in every step");
  extern __shared__ __align__(1024) char lds[];

  const TilePlace place = tile_place(a);
  if (!place.live) return;
  const int64_t i0 = static_cast<int64_t>(place.ti) * BI, j0 = static_cast<int64_t>(place.tj) * BJ;
  const int32_t k0 = place.k0, k1 = place.k1;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ, lane = threadIdx.x & 63;
  OpP p;
  OpQ q;
  p.init(a.P, a.ldp, i0, a.I);
  q.init(a.Q, a.ldq, j0, a.J);
  const uint32_t pb = OpP::lane_base(wi * TI * 16), qb = OpQ::lane_base(wj * TJ * 16);
  lds_char* const l3 = (lds_char*)lds;
  const uint32_t l0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(l3));

  // this thread's factor: of a row, of a column, or (threads beyond) the first row's again
  const int r = threadIdx.x;
  const bool column = r >= BI && r < BI + BJ;
  const int64_t at = column ? (min(j0 + r - BI, a.J - 1) >> a.ws_shift) * a.ws_row
                            : (min(i0 + (r < BI ? r : 0), a.I - 1) >> a.xs_shift) * a.xs_row;
  const int64_t factor_step = column ? a.ws_k : a.xs_k;
  const float* const factors = (column ? a.ws : a.xs) + at;
  auto factor = [&](int32_t s) __attribute__((always_inline)) { return factors + (k0 / kStep + s) * factor_step; };

  f4 acc[TI][TJ];
#pragma unroll
  for (int x = 0; x < TI; ++x)
#pragma unroll
    for (int y = 0; y < TJ; ++y) acc[x][y] = f4{0.0f, 0.0f, 0.0f, 0.0f};

  Block8 fq[TJ], fp[2];
  f4 ring[kRing];                       // sums of blocks that are not in `acc` yet
  float by_row[2], by_unit = 0.0f;      // factors of rows of tiles x % 2; of the wave's columns
  f4 by_column[UNITS ? TJ : 1];
  float late_scale[kRing];
  // the ring's last sums enter in the next step (with columns' factors they do so before those
  // change)
  constexpr bool kCarry = !UNITS;
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < kRing; ++n) {
      ring[n] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      late_scale[n] = 0.0f;
    }
  };
  clear();
  typedef __attribute__((address_space(3))) float lds_float;
  typedef __attribute__((address_space(3))) f4 lds_f4;
  auto read_q = [&](int slot, int y) __attribute__((always_inline)) {
    fq[y] = block_fragment<BJ>(l3 + slot * kStage + OpP::kBytes, qb, y);
  };
  auto read_columns = [&](int slot) __attribute__((always_inline)) {
    lds_char* const s = l3 + slot * kStage + kCodes + (BI + wj * TJ * 16) * 4;
    if constexpr (UNITS) {
#pragma unroll
      for (int y = 0; y < TJ; ++y) by_column[y] = *reinterpret_cast<lds_f4*>(s + (y * 16 + (lane >> 4) * 4) * 4);
    } else {
      by_unit = *reinterpret_cast<lds_float*>(s);
    }
  };
  auto read_p = [&](int slot, int x) __attribute__((always_inline)) {
    fp[x & 1] = block_fragment<BI>(l3 + slot * kStage, pb, x);
    by_row[x & 1] = *reinterpret_cast<lds_float*>(l3 + slot * kStage + kCodes + ((wi * TI + x) * 16 + (lane & 15)) * 4);
  };
  // the sum that tile n left in the ring enters its place
  auto enter = [&](int n) __attribute__((always_inline)) {
    f4& c = acc[n / TJ][n % TJ];
    const int at = n % kRing;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (UNITS)
        c[e] = fmaf(ring[at][e] * late_scale[at], by_column[n % TJ][e], c[e]);
      else
        c[e] = fmaf(ring[at][e], late_scale[at], c[e]);
    }
  };
  auto multiply = [&](int x, int y) __attribute__((always_inline)) {
    const int n = x * TJ + y, at = n % kRing;
    // One matrix instruction, then, while it runs, the sums of the tile kLate before (the first
    // ones' are the last of the step before).  In this order: left to the compiler, three matrix
    // instructions follow each other and the sums wait for the last (1.81 us a step of 256 x 256).
    ring[at] = block_sum<EXACT>(fq[y], fp[x & 1]);
    late_scale[at] = UNITS ? by_row[x & 1] : by_row[x & 1] * by_unit;
    __builtin_amdgcn_sched_barrier(0);
    if (kCarry || n >= kLate) enter((n + kTiles - kLate) % kTiles);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto drain = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = kTiles - kLate; n < kTiles; ++n) enter(n);
  };

  const int32_t steps = (k1 - k0 + kStep - 1) / kStep;
  int32_t t = 0;
  if (a.dma) {
    // Whole steps.  A step's rows of tiles are multiplied one by one while the next row's
    // fragments are read; at the last but one every wave has asked for all of the step: one
    // barrier, by which step t + 1 has arrived, then the last two rows, while step t + NS is
    // sent for into t's place, a load or so a product (all of them before the first: 468 us for
    // 8,192^3 instead of 450), and t + 1's first fragments are read, each in the place of one that
    // has just been used.
    const int32_t full = (k1 - k0) / kStep;
    constexpr int kMost = OpP::kEach + OpQ::kEach + 1;
    static_assert(OpQ::whole, "every wave moves the same share of Q");
    const bool most = OpP::whole || (OpP::kEach - 1) * THREADS + wave * 64 < OpP::kChunks;
    auto fetch_one = [&](int n, int32_t s, int slot) __attribute__((always_inline)) {
      const uint32_t to = l0 + static_cast<uint32_t>(slot) * kStage;
      if (n < OpP::kEach)
        p.fetch(n, k0 + s * kStep, to);
      else if (n < OpP::kEach + OpQ::kEach)
        q.fetch(n - OpP::kEach, k0 + s * kStep, to + OpP::kBytes);
      else
        dma4(factor(s), to + kCodes + wave * 256);
    };
    auto arrived = [&](int32_t s, int after) __attribute__((always_inline)) {
      if (after == 0 || s + after >= full)
        arrive<0>();
      else if (after == 1)
        most ? arrive<kMost>() : arrive<kMost - 1>();
      else if (after == 2)
        most ? arrive<2 * kMost>() : arrive<2 * (kMost - 1)>();
      else
        most ? arrive<3 * kMost>() : arrive<3 * (kMost - 1)>();
    };
    static_assert(NS >= 2 && NS <= 4, "the waits are written for two to four steps");
    if (full > 0) {
#pragma unroll
      for (int s = 0; s < NS; ++s)
        if (s < full)
#pragma unroll
          for (int n = 0; n < kMost; ++n) fetch_one(n, s, s);
      arrived(0, NS - 1);
      int slot = 0;
      read_columns(0);
      read_p(0, 0);
#pragma unroll
      for (int y = 0; y < TJ; ++y) read_q(0, y);
      constexpr int kTurn = TI > 1 ? TI - 2 : 0;       // the row of tiles before which all has been read
      auto step = [&](auto fetches) __attribute__((always_inline)) {
        const int freed = slot, next = slot + 1 == NS ? 0 : slot + 1;
#pragma unroll
        for (int x = 0; x < TI; ++x) {
          __builtin_amdgcn_sched_barrier(0);
          if (x + 1 < TI) read_p(freed, x + 1);
          if (x == kTurn) arrived(t + 1, NS - 2);
#pragma unroll
          for (int y = 0; y < TJ; ++y) {
            if constexpr (decltype(fetches)::value) {
              constexpr int kOver = (TI - kTurn) * TJ;
              const int m = (x - kTurn) * TJ + y;
              if (x >= kTurn)
#pragma unroll
                for (int n = m * kMost / kOver; n < (m + 1) * kMost / kOver; ++n) fetch_one(n, t + NS, freed);
            }
            multiply(x, y);
            // (after the last step: bytes that no product uses)
            if (x == TI - 1) read_q(next, y);
          }
          if (x == TI - 1) {
            if constexpr (!kCarry) drain();
            read_columns(next);
            read_p(next, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        slot = next;
      };
      for (; t < full - NS; ++t) step(Yes{});
      for (; t < full; ++t) step(No{});
      if constexpr (kCarry) drain();
    }
  }
  if (t < steps) {
    // Through registers, the next step on its way.
    u4 vp[OpP::kEach], vq[OpQ::kEach];
    float vs;
    const int32_t full = (k1 - k0) / kStep;
    auto load = [&](int32_t s) __attribute__((always_inline)) {
      const int32_t k = k0 + s * kStep;
      if (s < full) {
        p.template load<false>(k, k1, a.K, vp);
        q.template load<false>(k, k1, a.K, vq);
      } else {
        p.template load<true>(k, k1, a.K, vp);
        q.template load<true>(k, k1, a.K, vq);
      }
      vs = *factor(s);
    };
    load(t);
    int slot = 0;
    __syncthreads();                   // the steps before are read
    for (; t < steps; ++t) {
      lds_char* const here = l3 + slot * kStage;
      p.store(lds + slot * kStage, a.K, vp);
      q.store(lds + slot * kStage + OpP::kBytes, a.K, vq);
      *reinterpret_cast<lds_float*>(here + kCodes + threadIdx.x * 4) = vs;
      arrive_lds();
      if (t + 1 < steps) load(t + 1);
      clear();                         // what the ring holds is in `acc` already
      read_columns(slot);
#pragma unroll
      for (int y = 0; y < TJ; ++y) read_q(slot, y);
#pragma unroll
      for (int x = 0; x < TI; ++x) {
        read_p(slot, x);
#pragma unroll
        for (int y = 0; y < TJ; ++y) multiply(x, y);
      }
      drain();
      slot ^= 1;
    }
  }
  __syncthreads();                     // every wave is done with the steps
  const Tile<WI, WJ, TI, TJ, NS * kStage> tile(a, l3, wave, i0, j0);
  tile.finish(a, acc, place.split);
}

}  // namespace som
