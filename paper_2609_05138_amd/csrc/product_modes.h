// The matrix product's kernel with epilogues of its own: sums and factors that stay on the
// device (kExtra), of symmetric products (kMirror), and the two passes of cross entropy (kLoss, kGrad;
// kGradFew, by itself so that its registers are not kGrad's, keeps what is rounded away from labels).
#pragma once

#include "product.h"

namespace som {

// out = alpha factor (sum + row_i column_j) + beta residual (of a type of its own), and the same
// times half_scale in the operands' type.
struct ExtraArgs : ProductArgs {
  const float* factor;       // or nullptr
  const float *row, *column; // or nullptr
  float beta;
  int res_type;
  void* half;                // [I][ldh] or nullptr
  int64_t ldh;
  float half_scale;
  // C is symmetric (I = J; `residual` too; no row, column, half and swap): kMirror, which
  // calculates the tiles on and above the diagonal and writes their transposes too, will do where
  // it is faster
  bool symmetric;
  // where *swap is not 0, P (or Q) is read from `swapped` instead
  const int32_t* swap;       // or nullptr
  const void* swapped;
  int64_t ld_swapped;
  bool swap_p;
  // Row i gets rest[i] times class labels[i]'s weights too (other_units: [class][ld_other], else [..][ld_other]
  // by class): what P has less than it should in that entry.  In the join: every tile leaves parts then.
  const float* rest;         // or nullptr
  const int32_t* labels;
  const void* other;
  int64_t ld_other;
  bool other_units;
};

// Scores v = alpha sum + bias of rows against J classes; of each row in each tile the largest and
// the sum of exponentials below it, and the score of the row's label.
struct LossArgs : ProductArgs {
  const int32_t* labels;
  float* part;               // [tiles_j][I] pairs
  float* label_score;        // [I]; not written where the label is none of the classes
};

// g = dloss (exp(v - lse) - [label]) times *factor in the operands' type to out (whose rows are
// padded to eight columns), its unscaled sums over the tile's rows, and of each row what the rounding
// of g times *factor took away in 16 TJ columns (those of a wave).
struct GradArgs : ProductArgs {
  const int32_t* labels;
  const float *lse, *dloss, *factor;
  int64_t first, classes;    // the first of these columns' classes, and all there are
  float* column_part;        // [tiles_i][ld_column] or nullptr
  int64_t ld_column;
  float* lost_part;          // [strips][I] or nullptr
  // [I]: what g's rounding takes from each row's label (kGradFew; not in lost_part then), or nullptr;
  // not written where the label is none of these columns' classes
  float* rest;
};
constexpr int kLostStrip = 512;        // columns of a strip where k_grad_scores makes g

template <>
struct ModeArgs<kExtra> {
  typedef ExtraArgs type;
};
template <>
struct ModeArgs<kMirror> {
  typedef ExtraArgs type;
};
template <>
struct ModeArgs<kLoss> {
  typedef LossArgs type;
};
template <>
struct ModeArgs<kGrad> {
  typedef GradArgs type;
};
template <>
struct ModeArgs<kGradFew> {
  typedef GradArgs type;
};

// The plan of a kExtra product (no kernels of few rows), and the product with the join of a split
// k axis.
inline RuledPlan plan_extra(int64_t I, int64_t J, int64_t K, int elem, bool p_kc, bool q_kc, bool dma,
                            bool symmetric = false) {
  return plan_product_by(I, J, K, elem, p_kc, q_kc, dma, {false, kShape256, symmetric});
}
hipError_t launch_extra(ExtraArgs a, float* partial, hipStream_t stream);
// The product alone, of `a` with `rest`, into parts that join_extra, of its join_threads, puts together;
// fills the launch's fields.
hipError_t launch_parts(ExtraArgs& a, float* partial, hipStream_t stream);
// The kernel alone; `a`, the mode's arguments, has its launch's fields.
hipError_t launch_mode(int mode, int shape, const ProductArgs& a, hipStream_t stream);
hipError_t launch_modes_f16(int mode, int shape, const ProductArgs& a, hipStream_t stream);
hipError_t launch_modes_bf16(int mode, int shape, const ProductArgs& a, hipStream_t stream);
hipError_t launch_mirror_f16(int shape, const ExtraArgs& a, hipStream_t stream);

// ---------------------------------------------------------------------------
// kExtra
// ---------------------------------------------------------------------------

__device__ __forceinline__ RowTerms extra_terms(const ExtraArgs& a, float scale, int64_t i, int64_t j, int n) {
  RowTerms r;
  r.scale = scale;
  r.residual[0] = r.residual[1] = u4{0, 0, 0, 0};
  if (n <= 0 || !a.residual) return r;
  float v[8];
  if (a.res_type == kF32) {
    load8(static_cast<const float*>(a.residual) + i * a.ldr + j, n, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) r.residual[e / 4][e % 4] = __float_as_uint(v[e]);
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(a.residual) + i * a.ldr + j;
    if (n == 8) {
      r.residual[0] = *reinterpret_cast<const u4_at2*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < n) r.residual[0][e / 2] |= static_cast<uint32_t>(p[e]) << (16 * (e % 2));
    }
  }
  return r;
}

// The rank-one term enters the sums.
__device__ __forceinline__ void add_outer(const ExtraArgs& a, int64_t i, const float (&column)[8], float (&v)[8]) {
  if (!a.row) return;
  const float r = a.row[i];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fmaf(r, column[e], v[e]);
}

__device__ __forceinline__ void add_rest(const ExtraArgs& a, int64_t i, int64_t j, int n, float (&v)[8]) {
  const float r = a.rest[i];
  if (r == 0.0f) return;               // (also where there is no label)
  const int64_t label = a.labels[i];
  auto add = [&](auto type) __attribute__((always_inline)) {
    const auto* const W = static_cast<const decltype(type)*>(a.other);
    float w[8];
    if (a.other_units) {
      load8(W + label * a.ld_other + j, n, w);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = e < n ? static_cast<float>(W[(j + e) * a.ld_other + label]) : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(r, w[e], v[e]);
  };
  if (a.elem == kF16)
    add(f16{});
  else
    add(bf16{});
}

template <bool kWhole>
__device__ __forceinline__ void finish_extra(const ExtraArgs& a, int64_t i, int64_t j, int n, float (&v)[8],
                                             const RowTerms& r) {
  if (a.residual) {
    float res[8] = {};
    residual8(a.res_type, r, res);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(a.beta, res[e], v[e] * r.scale);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= r.scale;
  }
  if (a.out) store8_as<kWhole>(a.out_type, a.out, i * a.ldo + j, n, v);
  if (a.half) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= a.half_scale;
    store8_as<false>(a.elem, a.half, i * a.ldh + j, n, v);
  }
}

__device__ __forceinline__ void finish8_extra(const ExtraArgs& a, int64_t i, int64_t j, int n, float (&v)[8],
                                              const RowTerms& r) {
  if (n == 8)
    finish_extra<true>(a, i, j, n, v, r);
  else
    finish_extra<false>(a, i, j, n, v, r);
}

__device__ __forceinline__ float extra_scale(const ExtraArgs& a);

// Eight columns of C from their parts: of the at'th thread.
inline int64_t join_threads(const ExtraArgs& a) { return (a.J + 7) / 8 * a.I; }
__device__ __forceinline__ void join_extra(const ExtraArgs& a, int64_t at) {
  const int64_t groups = (a.J + 7) / 8;
  if (at >= groups * a.I) return;
  const int64_t i = at / groups, j = at % groups * 8;
  const int n = static_cast<int>(min<int64_t>(8, a.J - j));
  const RowTerms r = extra_terms(a, extra_scale(a), i, j, n);
  float v[8];
  join8(a, i, j, v);
  if (a.row) {
    float column[8];
    load8(a.column + j, n, column);
    add_outer(a, i, column, v);
  }
  if (a.rest) add_rest(a, i, j, n, v);
  finish8_extra(a, i, j, n, v, r);
}

__device__ __forceinline__ float extra_scale(const ExtraArgs& a) { return a.factor ? a.alpha * *a.factor : a.alpha; }

template <class TileOf, int TI, int TJ>
__device__ __forceinline__ void extra_tile(const TileOf& tile, const ExtraArgs& a, const f4 (&acc)[TI][TJ],
                                           const TilePlace& place) {
  if (a.splits > 1 || a.rest) return tile.part(a, acc, place.split);
  constexpr int kAhead = TileOf::kAhead;
  const float scale = extra_scale(a);
  auto terms = [&](int g) __attribute__((always_inline)) {
    const int64_t i = tile.first + g * TileOf::kRows;
    return extra_terms(a, scale, i, tile.j, g < TileOf::kGroups && i < a.I ? tile.n : 0);
  };
  float column[8] = {};
  if (a.row) load8(a.column + tile.j, tile.n, column);
  RowTerms ahead[kAhead];
#pragma unroll
  for (int g = 0; g < kAhead; ++g) ahead[g] = terms(g);
  tile.rows(acc, [&](int g, int64_t i, float (&v)[8]) __attribute__((always_inline)) {
    const RowTerms now = ahead[0];
#pragma unroll
    for (int k = 0; k + 1 < kAhead; ++k) ahead[k] = ahead[k + 1];
    ahead[kAhead - 1] = terms(g + kAhead);
    if (i >= a.I || tile.n <= 0) return;
    add_outer(a, i, column, v);
    finish8_extra(a, i, tile.j, tile.n, v, now);
  });
}

// The same of a symmetric C, by itself so that its registers are not kExtra's.
template <class TileOf, int TI, int TJ>
__device__ __forceinline__ void mirror_tile(const TileOf& tile, const ExtraArgs& a, const f4 (&acc)[TI][TJ],
                                            const TilePlace& place) {
  tile.rows(acc, [&](int, int64_t i, float (&v)[8]) __attribute__((always_inline)) {
    if (i < a.I && tile.n > 0) finish8_extra(a, i, tile.j, tile.n, v, extra_terms(a, a.alpha, i, tile.j, tile.n));
  });
  if (place.ti == place.tj) return;
  tile.columns(acc, [&](int64_t i, int64_t j, float (&v)[8]) __attribute__((always_inline)) {
    const int n = static_cast<int>(min<int64_t>(8, a.J - j));
    if (i < a.I && n > 0) finish8_extra(a, i, j, n, v, extra_terms(a, a.alpha, i, j, n));
  });
}

// ---------------------------------------------------------------------------
// kLoss
// ---------------------------------------------------------------------------

// The largest m of some scores and s = sum exp(v - m), both pairs' (m = -infinity: none).
__device__ __forceinline__ void join_max_sum(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
  s = s * __builtin_amdgcn_exp2f(kLog2e * (m - base)) + s2 * __builtin_amdgcn_exp2f(kLog2e * (m2 - base));
  m = top;
}

// Straight from the matrix instructions' registers: a lane has 4 TJ scores of a row, the four lanes
// 16 apart the wave's 16 TJ.  exp(v - m) as a power of two: its argument's rounding, |v - m| 2^-24,
// is that of a difference of scores.
template <class TileOf, int TI, int TJ>
__device__ __forceinline__ void loss_tile(const TileOf& tile, const LossArgs& a, const f4 (&acc)[TI][TJ],
                                          const TilePlace& place) {
  if (a.splits > 1) return tile.part(a, acc, place.split);
  constexpr int WI = TileOf::kWI, WJ = TileOf::kWJ, BI = WI * TI * 16;
  const int wi = tile.wave / WJ, wj = tile.wave % WJ, g = tile.lane >> 4;
  const int64_t j = tile.j0 + wj * TJ * 16 + g * 4;
  float bias[TJ][4];
#pragma unroll
  for (int y = 0; y < TJ; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t at = j + y * 16 + e;
      bias[y][e] = at >= a.J ? -INFINITY : a.bias ? a.bias[at] : 0.0f;
    }
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) f2 lds_f2;
  lds_f2* const sums = reinterpret_cast<lds_f2*>(tile.lds);      // [WJ][BI]
#pragma unroll
  for (int x = 0; x < TI; ++x) {
    const int row = (wi * TI + x) * 16 + (tile.lane & 15);
    const int64_t i = tile.i0 + row;
    const int64_t label = (i < a.I ? a.labels[i] : -1) - j;     // in this lane's columns: y * 16 + e
    float v[TJ][4], m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int y = 0; y < TJ; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // past the classes: -infinity, whatever the sums there (which are of other columns)
        v[y][e] = bias[y][e] == -INFINITY ? -INFINITY : fmaf(acc[x][y][e], a.alpha, bias[y][e]);
        m = fmaxf(m, v[y][e]);
        if (label == y * 16 + e && tile.j0 < a.J) a.label_score[i] = v[y][e];
      }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int y = 0; y < TJ; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(kLog2e * (v[y][e] - base));
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (g == 0) sums[wj * BI + row] = f2{m, s};
  }
  __syncthreads();
  if (threadIdx.x < BI && tile.i0 + threadIdx.x < a.I) {
    f2 all = sums[threadIdx.x];
    float m = all[0], s = all[1];
#pragma unroll
    for (int w = 1; w < WJ; ++w) {
      const f2 one = sums[w * BI + threadIdx.x];
      join_max_sum(m, s, one[0], one[1]);
    }
    f2* const part = reinterpret_cast<f2*>(a.part);
    part[place.tj * a.I + tile.i0 + threadIdx.x] = f2{m, s};
  }
}

// ---------------------------------------------------------------------------
// kGrad
// ---------------------------------------------------------------------------

struct GradRow {
  int label;                 // counted from the caller's first column
  float lse, dloss;          // dloss: 0 where the row has no label, or no score to choose from
};

__device__ __forceinline__ GradRow grad_row(const GradArgs& a, int64_t i, int64_t j, bool in) {
  GradRow r = {-1, 0.0f, 0.0f};
  if (!in) return r;
  const int label = a.labels[i];
  const float lse = a.lse[i];
  if (label < 0 || label >= a.classes || lse == -INFINITY) return r;
  r.label = label - static_cast<int>(a.first + j);           // (classes are at most 2^30)
  r.lse = lse;
  r.dloss = a.dloss[i];
  return r;
}

// g times `factor` of eight columns from their sums, in place; a row without a label, and but for its
// label's d a class that is left out, give zeros whatever their sums.
__device__ __forceinline__ void grad8(const GradArgs& a, const GradRow& r, float factor, const float (&bias)[8],
                                      float (&v)[8]) {
  const float d = r.dloss * factor;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = bias[e] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(kLog2e * fmaf(v[e], a.alpha, bias[e] - r.lse));
    v[e] = r.dloss == 0.0f ? 0.0f : r.label == e ? fmaf(d, p, -d) : d * p;
  }
}

// What rounding to the operands' type takes from a value.
__device__ __forceinline__ float rest_of(int elem, float v) {
  return v - (elem == kF16 ? static_cast<float>(static_cast<f16>(v)) : static_cast<float>(static_cast<bf16>(v)));
}

// Four values rounded to the operands' type, as they are stored, and sum plus the rounded ones
// (by the dot product with ones: two values an instruction).
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u2 round4(int elem, const float (&v)[4], float* sum) {
  typedef bf16 b2 __attribute__((ext_vector_type(2)));
  u2 word;
  if (elem == kF16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const h2 r = {static_cast<f16>(v[2 * h]), static_cast<f16>(v[2 * h + 1])};
      *sum = __builtin_amdgcn_fdot2(r, h2{static_cast<f16>(1.0f), static_cast<f16>(1.0f)}, *sum, false);
      word[h] = __builtin_bit_cast(uint32_t, r);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const b2 r = {static_cast<bf16>(v[2 * h]), static_cast<bf16>(v[2 * h + 1])};
      *sum = __builtin_amdgcn_fdot2_f32_bf16(r, b2{static_cast<bf16>(1.0f), static_cast<bf16>(1.0f)}, *sum, false);
      word[h] = __builtin_bit_cast(uint32_t, r);
    }
  }
  return word;
}

// Straight from the matrix instructions' registers, as loss_tile: a lane has four consecutive classes
// of a row in each of TJ places.  v - lse is alpha sum + (bias - lse), rounded at its own size, since
// it is an exponent; the label's class is looked for once a row and wave.
template <bool FEW, class TileOf, int TI, int TJ>
__device__ __forceinline__ void grad_tile(const TileOf& tile, const GradArgs& a, const f4 (&acc)[TI][TJ],
                                          const TilePlace& place) {
  if (a.splits > 1) return tile.part(a, acc, place.split);
  constexpr int WI = TileOf::kWI, WJ = TileOf::kWJ, BJ = WJ * TJ * 16;
  const int wi = tile.wave / WJ, wj = tile.wave % WJ, g = tile.lane >> 4;
  const int64_t wave_j = tile.j0 + wj * TJ * 16, j = wave_j + g * 4;        // + y * 16 + e
  const float factor = *a.factor;
  float bias[TJ][4], sums[TJ][4];
  bool gaps = false;         // there are classes that are left out (or none, past the last)
  const int left = static_cast<int>(min<int64_t>(a.J - wave_j, TJ * 16));
#pragma unroll
  for (int y = 0; y < TJ; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bias[y][e] = y * 16 + g * 4 + e >= left ? -INFINITY : a.bias ? a.bias[j + y * 16 + e] : 0.0f;
      gaps |= bias[y][e] == -INFINITY;
      sums[y][e] = 0.0f;
    }
  gaps = __any(gaps);
  // The rows' terms by way of LDS: one wait for all of them, and no registers.
  typedef float f3 __attribute__((ext_vector_type(3)));
  typedef __attribute__((address_space(3))) f3 lds_f3;
  typedef __attribute__((address_space(3))) float lds_float;
  lds_float* const all = reinterpret_cast<lds_float*>(tile.lds);      // [WI][BJ], column sums
  lds_f3* const terms = reinterpret_cast<lds_f3*>(tile.lds + WI * BJ * 4);       // [BI], 16 bytes each
  if (threadIdx.x < WI * TI * 16) {
    const int64_t i = tile.i0 + threadIdx.x;
    const GradRow r = grad_row(a, i, tile.j0, i < a.I);
    terms[threadIdx.x] = f3{__int_as_float(r.label), r.lse, r.dloss * factor};
  }
  __syncthreads();
  const int rows = static_cast<int>(min<int64_t>(a.I - tile.i0, WI * TI * 16));
  int row = wi * TI * 16 + (tile.lane & 15);
  uint16_t* out = static_cast<uint16_t*>(a.out) + (tile.i0 + row) * a.ldo + wave_j;
  float* lost_part = a.lost_part + (place.tj * WJ + wj) * a.I + tile.i0;
#pragma unroll
  for (int x = 0; x < TI; ++x, row += 16, out += 16 * a.ldo) {
    // (row by row: all rows' terms at once take the registers that the sums are in)
    __builtin_amdgcn_sched_barrier(0);
    const f3 r = terms[row];
    const float lse = r[1], d = r[2];
    const int label = __float_as_int(r[0]) - wj * TJ * 16;
    const bool none = d == 0.0f, here = !none && label >= 0 && label < TJ * 16 && (label >> 2 & 3) == g;
    float v[TJ][4], lost = 0.0f, rest = 0.0f;
#pragma unroll
    for (int y = 0; y < TJ; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[y][e] = d * __builtin_amdgcn_exp2f(kLog2e * fmaf(acc[x][y][e], a.alpha, bias[y][e] - lse));
    if (gaps) {                          // zeros whatever the sums hold, infinities too
#pragma unroll
      for (int y = 0; y < TJ; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[y][e] = bias[y][e] == -INFINITY ? 0.0f : v[y][e];
    }
    if (__any(here)) {
#pragma unroll
      for (int y = 0; y < TJ; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (here && label == y * 16 + g * 4 + e) rest = v[y][e] -= d;
      rest = FEW ? rest_of(a.elem, rest) : 0.0f;
      if (FEW && here) a.rest[tile.i0 + row] = rest;
    }
    if (__any(none)) {                   // zeros whatever the sums hold
#pragma unroll
      for (int y = 0; y < TJ; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[y][e] = none ? 0.0f : v[y][e];
    }
    float rounded = 0.0f;
    u2 word[TJ];
#pragma unroll
    for (int y = 0; y < TJ; ++y) {
      word[y] = round4(a.elem, v[y], &rounded);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lost += v[y][e];
        sums[y][e] += v[y][e];
        // (here: left to the compiler, the sums are made where they are used, and v is kept for that)
        asm volatile("" : "+v"(sums[y][e]));
      }
    }
    lost -= rounded + rest;
    // Of two places 16 columns apart the lanes of odd g give up the first and those of even g the
    // second, so that a lane has eight consecutive columns and a row's lanes 64 bytes.
#pragma unroll
    for (int y = 0; y < TJ; y += 2) {
      u4 both;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u2 swapped = __builtin_amdgcn_permlane16_swap(word[y][h], word[y + 1][h], false, false);
        both[h] = swapped[0];
        both[2 + h] = swapped[1];
      }
      const int at = (y + (g & 1)) * 16 + (g >> 1) * 8;
      if (row < rows && at < left) *reinterpret_cast<u4*>(out + at) = both;
    }
    if (a.lost_part) {
      lost += __shfl_xor(lost, 16, 64);
      lost += __shfl_xor(lost, 32, 64);
      if (g == 0 && row < rows) lost_part[row] = lost;
    }
  }
  if (!a.column_part) return;
  // over the lanes that share the columns, then over the waves below each other, in order
#pragma unroll
  for (int y = 0; y < TJ; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) sums[y][e] += __shfl_xor(sums[y][e], off, 64);
      if ((tile.lane & 15) == 0) all[wi * BJ + wj * TJ * 16 + y * 16 + g * 4 + e] = sums[y][e];
    }
  __syncthreads();
  const int64_t col = tile.j0 + threadIdx.x;
  if (threadIdx.x < BJ && col < a.J) {
    float s = all[threadIdx.x];
#pragma unroll
    for (int w = 1; w < WI; ++w) s += all[w * BJ + threadIdx.x];
    a.column_part[place.ti * a.ld_column + col] = s / factor;          // (a power of two)
  }
}

template <int MODE, class TileOf, int TI, int TJ>
__device__ __forceinline__ void finish_mode(const TileOf& tile, const typename ModeArgs<MODE>::type& a,
                                            const f4 (&acc)[TI][TJ], const TilePlace& place) {
  if constexpr (MODE == kExtra)
    extra_tile(tile, a, acc, place);
  else if constexpr (MODE == kMirror)
    mirror_tile(tile, a, acc, place);
  else if constexpr (MODE == kLoss)
    loss_tile(tile, a, acc, place);
  else
    grad_tile<MODE == kGradFew>(tile, a, acc, place);
}

}  // namespace som
