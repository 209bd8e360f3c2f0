// Softmax cross entropy of rows against classes whose scores are a matrix product, and its
// gradients; the scores are never kept.
//
//   forward   v = alpha x W + b;  lse_m = log sum_n exp v_mn;  loss_m = lse_m - v_m,label
//   backward  g = dloss_m (exp(v - lse_m) - [n = label]);  dx = alpha g W^T, dW = alpha x^T g, db_n = sum_m g
//
// Forward: a tile of the product leaves for each of its rows the largest score m and s = sum
// exp(v - m) (8 bytes for 256 or 128 scores), and the label's score; k_loss_join puts a row's
// pairs together.  Where the k axis is split, or the kernels of few rows are faster, the scores go
// through the workspace, as fp32, to k_loss_scores, which makes the pairs of 8,192 columns, or of up to
// 16,384 the loss itself.
//
// Backward: the product again, a piece of the classes at a time: its epilogue makes g of the
// piece, in x's type because the matrix cores take 16 bits (as som_product_backward's dP), and
// its column sums unrounded; two products add the piece to dx (in fp32 until the last piece)
// and give its part of dW.  A row of g sums to zero, so what all classes' weights have in common (a
// codebook's are positive, with a mean far from zero) cancels in dx, but not what g's rounding does
// to it: that is the row's sum of roundings times the common part, which is added back (with the
// mean of up to 64 classes in its place; without it dx of a codebook of [0, 1) is 2.1 times as far
// from 64 bits as its own rounding, with it 1.4 times, as where nothing is in common).  g is scaled
// by a power of two that dloss's largest value sets, so that fp16 holds what a mean over many rows
// gives (1 / M times a probability).  Classes that are left out, and documents that count for nothing, give
// zeros to g whatever their scores.
//
// Most of a row of g is its label's entry, one rounding of which reaches all of the document's dx and of
// the label's dW.  Over many documents that averages out to the above; of one dx and dW are 2 to 3 times as far
// from 64 bits as their own rounding.  So of up to 256 what rounding takes from the labels' entries is kept: dx gets
// it where its parts are joined, and dW's rows of these classes are made again, on the vector units: 1.1
// times at the most (1 x 2,048 x 65,536 202 to 207 us, 128 documents 236 to 250, 64 x 512 x 637 32 to 39).
//
// Bound: the matrix cores at the clock that power leaves them (8,192 x 4,096 x 65,536 in bf16 3,172
// to 3,270 us, 1,340 to 1,390 TFLOP/s; gradients of 8,192 x 2,048 x 65,536 5,120 to 5,280 us, 1,250 to 1,290, of
// which the scores' third, whose epilogue makes and writes g, 40%); one row: the weights' bytes
// (65,536 x 2,048 40 us, 6.7 TB/s, feature-major 42, and 10 us for the two launches after it); small gradients: five
// launches, of few documents six.
#include "cross_entropy.h"

#include "product_modes.h"

namespace som {
namespace {

constexpr int kScoreThreads = 1024, kScoreColumns = kScoreThreads * 8;   // of a pass of k_loss_scores
// A row of so many goes without k_loss_join (one document, us, without and with it: 16,384 classes 15.8 and
// 17.0, 24,576 21.0 and 20.7, 32,768 26.1 and 24.4, 65,536 46.9 and 40.5).
constexpr int64_t kOneWorkgroup = 2 * kScoreColumns;
constexpr int64_t kRowsAtOnce = 65536;         // forward: rows of one launch, for the pairs' room
// Backward: a piece's g has 2^27 bytes, half of what the memory-side cache holds, but no fewer than
// 8,192 classes, since dx's sums are read and written for each (8,192 x 2,048 x 65,536: pieces of
// 2^27 bytes 5,261 us, 2^28 5,400, 2^30 5,347; 16,384 x 1,024 x 65,536: 6,705, 6,134 and 6,051).
constexpr int64_t kPieceBytes = int64_t(1) << 27;
constexpr int64_t kLeastPiece = 8192;

typedef float f2 __attribute__((ext_vector_type(2)));

// A row's loss and lse from its largest score and the sum of exponentials below it.
struct LossOut {
  const int32_t* labels;
  const float* label_score;
  float *loss, *lse;
  int64_t classes;
};
__device__ __forceinline__ void finish_loss(const LossOut& o, int64_t i, float m, float s, float own) {
  const float all = m + logf(s);       // no score but -infinity: -infinity
  o.lse[i] = all;
  const int32_t label = o.labels[i];
  // (a label that cannot be had costs infinitely much, also where nothing can)
  o.loss[i] = label < 0 || label >= o.classes ? 0.0f : all == -INFINITY ? INFINITY : all - own;
}

// One row and `passes` x 8,192 columns a workgroup, from fp32 sums; with one such chunk to a row
// its loss too.
__global__ void __launch_bounds__(kScoreThreads) k_loss_scores(const LossArgs a, const LossOut o, uint32_t chunks,
                                                               int passes) {
  __shared__ f2 sums[kScoreThreads / 64];
  __shared__ float own;
  const int64_t g = group_index(), i = g / chunks, chunk = g - i * chunks;
  if (i >= a.I) return;
  const int64_t first = chunk * passes * kScoreColumns + threadIdx.x * 8;
  const int64_t label = a.labels[i];
  float m = -INFINITY, s = 0.0f;
  for (int p = 0; p < passes; ++p) {
    const int64_t j = first + p * kScoreColumns;
    const int n = a.J - j >= 8 ? 8 : a.J > j ? static_cast<int>(a.J - j) : 0;
    if (n <= 0) break;
    float v[8], bias[8] = {}, top = -INFINITY, sum = 0.0f;
    join8(a, i, j, v);
    if (a.bias) load8(a.bias + j, n, bias);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = e >= n || bias[e] == -INFINITY ? -INFINITY : fmaf(v[e], a.alpha, bias[e]);
      top = fmaxf(top, v[e]);
      if (e < n && label - j == e) {
        if (chunks > 1)
          a.label_score[i] = v[e];
        else
          own = v[e];
      }
    }
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += __builtin_amdgcn_exp2f(kLog2e * (v[e] - base));
    join_max_sum(m, s, top, sum);
  }
#pragma unroll
  for (int off = 32; off; off >>= 1) join_max_sum(m, s, __shfl_xor(m, off, 64), __shfl_xor(s, off, 64));
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = f2{m, s};
  __syncthreads();
  if (threadIdx.x) return;
#pragma unroll
  for (int w = 1; w < kScoreThreads / 64; ++w) join_max_sum(m, s, sums[w][0], sums[w][1]);
  if (chunks > 1)
    reinterpret_cast<f2*>(a.part)[chunk * a.I + i] = f2{m, s};
  else
    finish_loss(o, i, m, s, own);
}

// 16 rows a workgroup, 16 threads a row, each every 16th pair.
__global__ void __launch_bounds__(256) k_loss_join(const f2* __restrict__ part, int64_t parts, int64_t rows,
                                                   const LossOut o) {
  __shared__ f2 sums[16][17];
  const int r = threadIdx.x & 15, slice = threadIdx.x >> 4;
  const int64_t i = group_index() * 16 + r;
  float m = -INFINITY, s = 0.0f;
  if (i < rows) {
    constexpr int kDeep = 4;           // pairs on their way
    for (int64_t p0 = slice; p0 < parts; p0 += 16 * kDeep) {
      f2 one[kDeep];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) one[d] = p0 + 16 * d < parts ? part[(p0 + 16 * d) * rows + i] : f2{-INFINITY, 0.0f};
#pragma unroll
      for (int d = 0; d < kDeep; ++d) join_max_sum(m, s, one[d][0], one[d][1]);
    }
  }
  sums[slice][r] = f2{m, s};
  __syncthreads();
  if (slice || i >= rows) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) join_max_sum(m, s, sums[w][r][0], sums[w][r][1]);
  finish_loss(o, i, m, s, o.label_score[i]);
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

// What the workspace's head holds.
struct GradHead {
  float factor, inverse;     // of g as it is stored: a power of two
  int32_t swap;              // 1: a row that counts for nothing holds a NaN or an infinity
};
constexpr int kScanGroups = 512;       // and as many flags
// Documents whose labels' roundings are kept and multiplied.  More are within 1.51 of their own rounding
// without (129 drawn sizes up to 256: 1.11 at the most; 70 larger ones: 1.51, two of them over 1.5), and
// the classes that are made again take the square of the documents.
constexpr int64_t kFewRows = 256;

// A row counts for nothing.
__device__ __forceinline__ bool no_row(const GradCall& c, int64_t i) {
  const int32_t label = c.labels[i];
  const float lse = c.lse[i], dloss = c.dloss[i];        // (three loads on their way at once)
  return label < 0 || label >= c.N || lse == -INFINITY || dloss == 0.0f;
}

// Workgroup 0: the head.  dloss's largest finite value is had by one workgroup, so it needs no second
// launch (8,192 rows: 6 us).
__device__ void grad_head(const GradCall& c, int bits, GradHead* head, uint32_t* tops) {
  uint32_t top = 0;
  for (int64_t i0 = threadIdx.x; i0 < c.M; i0 += 4 * 1024) {
    uint32_t one[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int64_t i = min(i0 + d * 1024, c.M - 1);
      const uint32_t size = __float_as_uint(c.dloss[i]) & 0x7fffffffu;
      one[d] = no_row(c, i) || size >= 0x7f800000u ? 0 : size;     // (finite ones: the others keep their digits)
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) top = max(top, one[d]);
  }
  top = group_max<1024>(top, tops);
  if (threadIdx.x) return;
  const float most = __uint_as_float(top);
  int e = 0;
  if (top) e = bits - min(max(ilogbf(most), -100), 100);
  head->factor = ldexpf(1.0f, e);
  head->inverse = ldexpf(1.0f, -e);
}

// No label's rounding is known yet.
__device__ __forceinline__ void clear_rest(const GradCall& c, float* rest) {
  if (threadIdx.x < c.M) rest[threadIdx.x] = 0.0f;
}

// common[k] = the mean weight of up to 64 classes, spread over all that are not left out; a feature a wave,
// a class a lane.  It is 0 where it is no more than the weights' mean distance from it and three
// errors of a mean of n (what they have by chance, or a few large ones make; not taking it back adds
// 0.6 to the error's square of 2 at the most), and where it is further than 0 from the classes that as
// many documents are labelled with (those whose bias leaves them no document may have any weights).
template <typename T>
__device__ void grad_common(const GradCall& c, int64_t group, float* common) {
  const T* const W = static_cast<const T*>(c.W);
  const int64_t k = group * 16 + (threadIdx.x >> 6);
  if (k >= c.K) return;
  const int lane = threadIdx.x & 63;
  auto weight = [&](int64_t n) { return static_cast<float>(c.units ? W[n * c.ldw + k] : W[k * c.ldw + n]); };
  auto spread = [&](int64_t all) { return all > 64 ? lane * all / 64 : lane < all ? lane : 0; };
  const int64_t one = spread(c.N), i = spread(c.M);
  const bool own = lane < c.M && !no_row(c, i), in = lane < c.N && !(c.bias && c.bias[one] == -INFINITY);
  const float w = weight(one), v = weight(own ? c.labels[i] : 0);
  float n = in ? 1.0f : 0.0f, s = in ? w : 0.0f;
#pragma unroll
  for (int off = 32; off; off >>= 1) {
    n += __shfl_xor(n, off, 64);
    s += __shfl_xor(s, off, 64);
  }
  s /= n;
  const float times = 1.0f + 3.0f * rsqrtf(n);
  float more = in ? fabsf(s) - times * fabsf(w - s) : 0.0f, nearer = own ? fabsf(v) - fabsf(v - s) : 0.0f;
#pragma unroll
  for (int off = 32; off; off >>= 1) {
    more += __shfl_xor(more, off, 64);
    nearer += __shfl_xor(nearer, off, 64);
  }
  // (of weights that are not finite both are NaN: they make NaNs of what they reach, and no more than that)
  if (lane == 0) common[k] = more > 0.0f && nearer > 0.0f ? s : 0.0f;
}

// Looks through the rows of x that count for nothing, a wave a row; a flag a workgroup.
template <typename T>
__device__ void grad_scan(const GradCall& c, int64_t group, int64_t groups, int32_t* flags) {
  bool bad = false;
  for (int64_t i = group * 16 + (threadIdx.x >> 6); i < c.M; i += groups * 16) {
    if (!no_row(c, i)) continue;
    for (int64_t k = (threadIdx.x & 63) * 8; k < c.K; k += 512) {
      const int n = c.K - k >= 8 ? 8 : static_cast<int>(c.K - k);
      float v[8];
      load8(static_cast<const T*>(c.x) + i * c.ldx + k, n, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) bad |= !(fabsf(v[e]) < INFINITY);
    }
  }
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0) flags[group] = any;
}

// Everything that goes before the scores, by workgroups: the head, `commons` for the common
// weights, `scans` for the rows (the grid may hold more).
template <typename T>
__global__ void __launch_bounds__(1024) k_grad_prepare(const GradCall c, int bits, GradHead* head, int64_t commons,
                                                       float* common, int64_t scans, int32_t* flags, float* rest) {
  __shared__ uint32_t tops[16];
  const int64_t g = group_index();
  if (g == 0 && rest) clear_rest(c, rest);
  if (g == 0)
    grad_head(c, bits, head, tops);
  else if (g <= commons)
    grad_common<T>(c, g - 1, common);
  else if (g - 1 - commons < scans)
    grad_scan<T>(c, g - 1 - commons, scans, flags);
}

// x with zeros in the rows that count for nothing, if one of them is not finite.
template <typename T>
__device__ void grad_clean(const GradCall& c, int64_t group, int64_t groups, const int32_t* flags, int nflags,
                           GradHead* head, T* out, int64_t ldo) {
  const int any = __syncthreads_or(threadIdx.x < nflags && flags[threadIdx.x]);
  if (group == 0 && threadIdx.x == 0) head->swap = any;
  if (!any) return;
  for (int64_t i = group * 16 + (threadIdx.x >> 6); i < c.M; i += groups * 16) {
    const bool none = no_row(c, i);
    for (int64_t k = (threadIdx.x & 63) * 8; k < c.K; k += 512) {
      const int n = c.K - k >= 8 ? 8 : static_cast<int>(c.K - k);
      float v[8] = {};
      if (!none) load8(static_cast<const T*>(c.x) + i * c.ldx + k, n, v);
      store8(out + i * ldo + k, 8, v);
    }
  }
}

// Columns' sums (out[j] = sum over g of part[g * ld + j], 64 columns a workgroup, in order within
// fixed groups) or rows' (of part[g * rows + i]), which are the same.
__device__ void sum_parts(const float* __restrict__ part, int64_t parts, int64_t ld, int64_t n, int64_t group,
                          float* __restrict__ out, float (&sums)[16][64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = group * 64 + lane;
  float s = 0.0f;
  if (c < n)
    for (int64_t g0 = wave; g0 < parts; g0 += 16 * 8) {
      float v[8];                       // eight on their way
#pragma unroll
      for (int d = 0; d < 8; ++d) v[d] = g0 + 16 * d < parts ? part[(g0 + 16 * d) * ld + c] : 0.0f;
#pragma unroll
      for (int d = 0; d < 8; ++d) s += v[d];
    }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < n) {
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    out[c] = s;
  }
}

// Everything between a piece's scores and its products, by workgroups: `columns` of them for
// dbias, `losts` for the rows' roundings, `cleans` for x (as many as there are flags).
struct GradBetween {
  const float *column_part, *lost_part;
  float *dbias, *lost;
  int64_t columns, column_parts, ld_column, n, losts, lost_parts;
  const int32_t* flags;
  GradHead* head;
  void* clean;
  int64_t ld_clean;
  int cleans;
};
template <typename T>
__global__ void __launch_bounds__(1024) k_grad_between(const GradCall c, const GradBetween b) {
  __shared__ float sums[16][64];
  const int64_t g = group_index(), rest = g - b.columns - b.losts;
  if (g < b.columns)
    sum_parts(b.column_part, b.column_parts, b.ld_column, b.n, g, b.dbias, sums);
  else if (rest < 0)
    sum_parts(b.lost_part, b.lost_parts, c.M, c.M, g - b.columns, b.lost, sums);
  else if (rest < b.cleans)
    grad_clean<T>(c, rest, b.cleans, b.flags, b.cleans, b.head, static_cast<T*>(b.clean), b.ld_clean);
}

// g, its column sums and what its rounding takes from each row, from a split product's parts: 512
// columns a workgroup, every (4 gridDim.y)th row, as k_act_grad.
__global__ void __launch_bounds__(256) k_grad_scores(const GradArgs a) {
  __shared__ float sums[4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = (static_cast<int64_t>(blockIdx.x) * 64 + lane) * 8;
  const int n = a.J - col >= 8 ? 8 : a.J > col ? static_cast<int>(a.J - col) : 0;
  const float factor = *a.factor;
  float bias[8] = {}, db[8] = {};
  if (a.bias) load8(a.bias + col, n, bias);
  for (int64_t row = static_cast<int64_t>(blockIdx.y) * 4 + wave; row < a.I; row += int64_t(gridDim.y) * 4) {
    float lost = 0.0f;
    if (n > 0) {
      float v[8];
      join8(a, row, col, v);
      const GradRow r = grad_row(a, row, col, true);
      grad8(a, r, factor, bias, v);
      if (a.rest && r.label >= 0 && r.label < n) {
        float own = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) own = r.label == e ? v[e] : own;
        own = rest_of(a.elem, own);
        a.rest[row] = own;
        lost -= own;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float four[4], rounded = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          four[e] = 4 * h + e < n ? v[4 * h + e] : 0.0f;
          db[4 * h + e] += four[e];
          lost += four[e];
        }
        const u2 word = round4(a.elem, four, &rounded);
        lost -= rounded;
        *reinterpret_cast<u2*>(static_cast<uint16_t*>(a.out) + row * a.ldo + col + 4 * h) = word;
      }
    }
    if (a.lost_part) {
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) lost += __shfl_xor(lost, off, 64);
      if (lane == 0) a.lost_part[blockIdx.x * a.I + row] = lost;
    }
  }
  if (!a.column_part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[wave][lane * 8 + e] = db[e];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += 256) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 512 + c;
    if (at < a.J)
      a.column_part[static_cast<int64_t>(blockIdx.y) * a.ld_column + at] =
          (sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c]) / factor;
  }
}

// dW of the classes that few documents are labelled with, once more, from g as it was before its rounding in
// the labels' entries: a workgroup a document (the first of its label works) and 512 features, a wave a
// quarter of the documents.
struct GradLabels {
  const void* g;
  const float* rest;
  const GradHead* head;
  int64_t ldg, first, classes, chunks;
};
template <typename T>
__device__ void grad_labels(const GradCall& c, const GradLabels& l, int64_t at) {
  constexpr int kBlocks = kFewRows / 64, kDeep = 8;      // of 64 documents; documents on their way
  __shared__ __align__(16) float sums[4][512];
  const T* const g = static_cast<const T*>(l.g);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = static_cast<int>(at / l.chunks), M = static_cast<int>(c.M);
  if (m >= M) return;
  const int32_t label = c.labels[m];
  const int64_t n = label - l.first, k = (at % l.chunks) * 512 + lane * 8;
  if (label < 0 || n < 0 || n >= l.classes) return;
  // every document's g for this class; the ones that are labelled with it
  float own[kBlocks];
  uint64_t mine[kBlocks];
  int one = M;                         // the first of them
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const int i = b * 64 + lane;
    const bool in = i < M;
    const bool same = in && c.labels[in ? i : 0] == label && c.lse[in ? i : 0] != -INFINITY && c.dloss[in ? i : 0] != 0.0f;
    own[b] = in ? static_cast<float>(g[i * l.ldg + n]) + (same ? l.rest[i] : 0.0f) : 0.0f;
    mine[b] = __ballot(same);
  }
#pragma unroll
  for (int b = kBlocks - 1; b >= 0; --b)
    if (mine[b]) one = b * 64 + __builtin_ctzll(mine[b]);
  if (one != m) return;
  const int some = c.K - k >= 8 ? 8 : c.K > k ? static_cast<int>(c.K - k) : 0;
  float s[8] = {};
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    // (a document whose g is 0 counts for nothing, or as good as that, and may hold anything)
    uint64_t left = __ballot(own[b] != 0.0f) & 0xffffull << 16 * wave;
    while (left) {
      float by[kDeep], v[kDeep][8];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        const int bit = left ? __builtin_ctzll(left) : 0;
        by[d] = left ? __shfl(own[b], bit, 64) : 0.0f;
        load8(static_cast<const T*>(c.x) + (b * 64 + bit) * c.ldx + k, left ? some : 0, v[d]);
        left &= left - 1;
      }
#pragma unroll
      for (int d = 0; d < kDeep; ++d)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = fmaf(by[d], v[d][e], s[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[wave][lane * 8 + e] = s[e];
  __syncthreads();
  if (wave) return;
  const float scale = c.alpha * l.head->inverse;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    for (int w = 1; w < 4; ++w) s[e] += sums[w][lane * 8 + e];
    s[e] *= scale;
  }
  T* const dW = static_cast<T*>(c.dW);
  if (c.units) {
    store8(dW + label * c.lddw + k, some, s);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < some) dW[(k + e) * c.lddw + label] = static_cast<T>(s[e]);
  }
}

// What follows the products of few documents, by workgroups: `joins` for dx, the rest for dW's labels.
template <typename T>
__global__ void __launch_bounds__(256) k_grad_few(const GradCall c, const ExtraArgs dx, int64_t joins, const GradLabels l) {
  const int64_t g = group_index();
  if (g < joins)
    join_extra(dx, g * 256 + threadIdx.x);
  else if (l.g)
    grad_labels<T>(c, l, g - joins);
}

int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }
size_t most(size_t a, size_t b) { return a > b ? a : b; }

int64_t scan_groups(int64_t rows) {
  const int64_t g = (rows + 15) / 16;
  return g < kScanGroups ? g : kScanGroups;
}
int64_t scores_groups(int64_t rows) {
  const int64_t g = (rows + 3) / 4;
  return g < 64 ? g : 64;
}

}  // namespace

// ---------------------------------------------------------------------------
// Workspaces
// ---------------------------------------------------------------------------

LossWs loss_ws(int64_t M, int64_t N, int64_t K, int elem) {
  LossWs w{};
  const int64_t rows = M < kRowsAtOnce ? M : kRowsAtOnce;
  w.label_score = 0;
  size_t o = align_up(sizeof(float) * rows, 256);
  w.part = o;
  o += align_up(2 * sizeof(float) * rows * ((N + 127) / 128), 256);
  w.scores = o;
  size_t need = 0;
  for (const bool dma : {true, false})
    for (const bool units : {true, false})
      for (const int64_t m : {rows, M % rows}) {          // the last rows may be fewer
        if (m == 0) continue;
        const ProductPlan p = plan_product(m, N, K, elem, true, units, dma);
        need = most(need, p.shape == kFew ? static_cast<size_t>(m) * round8(N) : p.partial_floats);
      }
  w.total = o + align_up(sizeof(float) * need, 256);
  return w;
}

int64_t grad_piece(int64_t M, int64_t N) {
  int64_t piece = kPieceBytes / 2 / M / 256 * 256;
  if (piece < kLeastPiece) piece = kLeastPiece;
  return piece < N ? piece : N;
}

GradWs grad_ws(int64_t M, int64_t N, int64_t K, int elem) {
  GradWs w{};
  w.piece = grad_piece(M, N);
  w.ldg = round8(w.piece);
  w.ldx = round8(K);
  w.ld_column = round8(w.piece);
  w.head = 0;
  size_t o = 256;
  w.g = o;
  o += align_up(static_cast<size_t>(M) * w.ldg * 2, 256);
  w.clean = o;
  o += align_up(static_cast<size_t>(M) * w.ldx * 2, 256);
  w.dx = o;
  if (w.piece < N) o += align_up(sizeof(float) * M * w.ldx, 256);
  size_t need = 0;
  int64_t groups = 1;                  // of rows, each with its column sums
  for (const bool dma : {true, false})
    for (const int64_t n : {w.piece, N % w.piece}) {
      if (n == 0) continue;
      for (const bool units : {true, false}) {
        const ProductPlan p = plan_extra(M, n, K, elem, true, units, dma);
        const int64_t g = p.splits > 1 ? scores_groups(M) : (M + kInfo[p.shape].bi - 1) / kInfo[p.shape].bi;
        if (g > groups) groups = g;
        need = most(need, p.partial_floats);
      }
      for (const ProductPlan& p :
           {plan_extra(M, K, n, elem, true, false, dma), plan_extra(M, K, n, elem, true, true, dma),
            plan_extra(K, n, M, elem, false, false, dma), plan_extra(n, K, M, elem, false, false, dma)})
        need = most(need, p.partial_floats);
    }
  w.column = o;
  o += align_up(sizeof(float) * groups * w.ld_column, 256);
  w.common = o;
  o += align_up(sizeof(float) * w.ldx, 256);
  w.lost = o;
  o += align_up(sizeof(float) * M, 256);
  w.flags = o;
  o += sizeof(int32_t) * kScanGroups;
  w.lost_part = o;                     // a wave's columns: 32 at the least
  o += align_up(sizeof(float) * M * ((w.piece + 255) / 256 * 8), 256);
  w.few = M <= kFewRows;
  w.rest = o;
  if (w.few) {
    o += align_up(sizeof(float) * M, 256);
    need = most(need, static_cast<size_t>(M) * w.ldx);           // dx's sums go by way of the join
  }
  w.partial = o;
  w.total = o + align_up(sizeof(float) * need, 256);
  return w;
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------

namespace {

template <typename P>
P* at(void* base, size_t off) {
  return reinterpret_cast<P*>(static_cast<char*>(base) + off);
}

}  // namespace

hipError_t launch_loss(const LossCall& c, void* ws, hipStream_t stream) {
  const LossWs w = loss_ws(c.M, c.N, c.K, c.dtype);
  for (int64_t m0 = 0; m0 < c.M; m0 += kRowsAtOnce) {
    const int64_t rows = c.M - m0 < kRowsAtOnce ? c.M - m0 : kRowsAtOnce;
    LossArgs a{};
    a.P = static_cast<const char*>(c.x) + m0 * c.ldx * 2;
    a.ldp = c.ldx;
    a.p_kc = true;
    a.Q = c.W;
    a.ldq = c.ldw;
    a.q_kc = c.units;
    a.I = rows;
    a.J = c.N;
    a.K = c.K;
    a.elem = c.dtype;
    a.alpha = c.alpha;
    a.bias = c.bias;
    a.labels = c.labels + m0;
    a.part = at<float>(ws, w.part);
    a.label_score = at<float>(ws, w.label_score);
    a.dma = rows_on_16(a);
    const ProductPlan p = plan_product(a.I, a.J, a.K, a.elem, true, a.q_kc, a.dma);
    float* const scores = at<float>(ws, w.scores);
    const LossOut o = {a.labels, a.label_score, c.loss + m0, c.lse + m0, c.N};
    hipError_t e;
    if (p.shape == kFew) {             // plain sums, which k_loss_scores takes like one split
      ProductArgs f = a;
      f.alpha = 1.0f;
      f.bias = nullptr;
      f.out = scores;
      f.ldo = round8(c.N);
      f.out_type = kF32;
      f.splits = 1;
      e = launch_product_few(f, stream);
      a.partial = scores;
      a.splits = 1;
    } else {
      set_launch(a, p, scores);
      e = launch_mode(kLoss, p.shape, a, stream);
    }
    if (e != hipSuccess) return e;
    int64_t parts = a.tiles_j;
    if (p.shape == kFew || p.splits > 1) {
      const bool one = c.N <= kOneWorkgroup;
      const int passes = one ? static_cast<int>((c.N + kScoreColumns - 1) / kScoreColumns) : 1;
      parts = one ? 1 : (c.N + kScoreColumns - 1) / kScoreColumns;
      hipLaunchKernelGGL(k_loss_scores, groups_grid(parts * rows), dim3(kScoreThreads), 0, stream, a, o,
                         static_cast<uint32_t>(parts), passes);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      if (one) continue;
    }
    hipLaunchKernelGGL(k_loss_join, groups_grid((rows + 15) / 16), dim3(256), 0, stream,
                       reinterpret_cast<const f2*>(a.part), parts, rows, o);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
static hipError_t prepare(const GradCall& c, const GradWs& w, void* ws, hipStream_t stream) {
  const int64_t commons = c.dx ? (c.K + 15) / 16 : 0, scans = c.dW ? scan_groups(c.M) : 0;
  hipLaunchKernelGGL(k_grad_prepare<T>, groups_grid(1 + commons + scans), dim3(1024), 0, stream, c,
                     c.dtype == kF16 ? 14 : 0, at<GradHead>(ws, w.head), commons, at<float>(ws, w.common),
                     scans, at<int32_t>(ws, w.flags), w.few ? at<float>(ws, w.rest) : nullptr);
  return hipGetLastError();
}

template <typename T>
static hipError_t between(const GradCall& c, const GradWs& w, const GradArgs& a, int64_t column_parts, int64_t strips,
                          bool first, void* ws, hipStream_t stream) {
  GradBetween b{};
  if (c.dbias) {
    b.columns = (a.J + 63) / 64;
    b.column_part = a.column_part;
    b.column_parts = column_parts;
    b.ld_column = a.ld_column;
    b.n = a.J;
    b.dbias = c.dbias + a.first;
  }
  if (c.dx) {
    b.losts = (c.M + 63) / 64;
    b.lost_part = a.lost_part;
    b.lost_parts = strips;
    b.lost = at<float>(ws, w.lost);
  }
  const int64_t scans = c.dW && first ? scan_groups(c.M) : 0;
  b.flags = at<int32_t>(ws, w.flags);
  b.cleans = static_cast<int>(scans);
  b.head = at<GradHead>(ws, w.head);
  b.clean = at<void>(ws, w.clean);
  b.ld_clean = w.ldx;
  const int64_t groups = b.columns + b.losts + scans;
  if (groups == 0) return hipSuccess;
  hipLaunchKernelGGL(k_grad_between<T>, groups_grid(groups), dim3(1024), 0, stream, c, b);
  return hipGetLastError();
}

// `dx` (its product launched into parts) is nullptr where it is not needed, or summed up as it is.
template <typename T>
static hipError_t finish_few(const GradCall& c, const GradWs& w, const ExtraArgs* dx, int64_t first, int64_t classes, void* ws,
                             hipStream_t stream) {
  GradLabels l{};
  if (c.dW) l = {at<const void>(ws, w.g), at<float>(ws, w.rest), at<GradHead>(ws, w.head), w.ldg, first, classes, (c.K + 511) / 512};
  const int64_t joins = dx ? (join_threads(*dx) + 255) / 256 : 0, labels = c.dW ? c.M * l.chunks : 0;
  if (joins + labels == 0) return hipSuccess;
  hipLaunchKernelGGL(k_grad_few<T>, groups_grid(joins + labels), dim3(256), 0, stream, c, dx ? *dx : ExtraArgs{}, joins, l);
  return hipGetLastError();
}

hipError_t launch_loss_back(const GradCall& c, void* ws, hipStream_t stream) {
  const GradWs w = grad_ws(c.M, c.N, c.K, c.dtype);
  hipError_t e = c.dtype == kF16 ? prepare<f16>(c, w, ws, stream) : prepare<bf16>(c, w, ws, stream);
  if (e != hipSuccess) return e;
  GradHead* const head = at<GradHead>(ws, w.head);
  float* const partial = at<float>(ws, w.partial);
  void* const g = at<void>(ws, w.g);
  for (int64_t n0 = 0; n0 < c.N; n0 += w.piece) {
    const int64_t n = c.N - n0 < w.piece ? c.N - n0 : w.piece;
    const int64_t skip = n0 * (c.units ? c.ldw : 1) * 2, dskip = n0 * (c.units ? c.lddw : 1) * 2;
    const void* const W = static_cast<const char*>(c.W) + skip;
    GradArgs a{};
    a.P = c.x;
    a.ldp = c.ldx;
    a.p_kc = true;
    a.Q = W;
    a.ldq = c.ldw;
    a.q_kc = c.units;
    a.I = c.M;
    a.J = n;
    a.K = c.K;
    a.elem = c.dtype;
    a.alpha = c.alpha;
    a.bias = c.bias ? c.bias + n0 : nullptr;
    a.out = g;
    a.ldo = w.ldg;
    a.labels = c.labels;
    a.lse = c.lse;
    a.dloss = c.dloss;
    a.factor = &head->factor;
    a.first = n0;
    a.classes = c.N;
    a.column_part = c.dbias ? at<float>(ws, w.column) : nullptr;
    a.ld_column = w.ld_column;
    a.lost_part = c.dx ? at<float>(ws, w.lost_part) : nullptr;
    a.rest = w.few ? at<float>(ws, w.rest) : nullptr;
    a.dma = rows_on_16(a);
    const ProductPlan p = plan_extra(a.I, a.J, a.K, a.elem, true, a.q_kc, a.dma);
    set_launch(a, p, partial);
    e = launch_mode(w.few ? kGradFew : kGrad, p.shape, a, stream);
    if (e != hipSuccess) return e;
    const int64_t strips = p.splits > 1 ? (n + kLostStrip - 1) / kLostStrip : int64_t(a.tiles_j) * kInfo[p.shape].waves_j;
    int64_t groups = a.tiles_i;
    if (p.splits > 1) {
      groups = scores_groups(c.M);
      const dim3 grid(static_cast<uint32_t>((n + 511) / 512), static_cast<uint32_t>(groups));
      hipLaunchKernelGGL(k_grad_scores, grid, dim3(256), 0, stream, a);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    e = c.dtype == kF16 ? between<f16>(c, w, a, groups, strips, n0 == 0, ws, stream)
                        : between<bf16>(c, w, a, groups, strips, n0 == 0, ws, stream);
    if (e != hipSuccess) return e;
    ExtraArgs d{};
    d.elem = c.dtype;
    d.alpha = c.alpha;
    d.factor = &head->inverse;
    d.beta = 1.0f;
    d.res_type = kF32;
    if (c.dW) {
      ExtraArgs dw = d;
      dw.P = c.units ? g : c.x;
      dw.ldp = c.units ? w.ldg : c.ldx;
      dw.p_kc = false;
      dw.Q = c.units ? c.x : g;
      dw.ldq = c.units ? c.ldx : w.ldg;
      dw.q_kc = false;
      dw.I = c.units ? n : c.K;
      dw.J = c.units ? c.K : n;
      dw.K = c.M;
      dw.out = static_cast<char*>(c.dW) + dskip;
      dw.ldo = c.lddw;
      dw.out_type = c.dtype;
      dw.swap = &head->swap;
      dw.swapped = at<void>(ws, w.clean);
      dw.ld_swapped = w.ldx;
      dw.swap_p = !c.units;
      e = launch_extra(dw, partial, stream);
      if (e != hipSuccess) return e;
    }
    const bool last = n0 + n == c.N, parts = w.few && last;
    if (c.dx) {
      float* const sum = at<float>(ws, w.dx);
      d.P = g;
      d.ldp = w.ldg;
      d.p_kc = true;
      d.Q = W;
      d.ldq = c.ldw;
      d.q_kc = !c.units;
      d.I = c.M;
      d.J = c.K;
      d.K = n;
      d.residual = n0 ? sum : nullptr;
      d.ldr = w.ldx;
      d.out = last ? c.dx : sum;
      d.ldo = last ? c.lddx : w.ldx;
      d.out_type = last ? c.dtype : kF32;
      d.row = at<float>(ws, w.lost);
      d.column = at<float>(ws, w.common);
      if (parts) {                     // every label's rounding is known by now
        d.rest = a.rest;
        d.labels = c.labels;
        d.other = c.W;
        d.ld_other = c.ldw;
        d.other_units = c.units;
      }
      e = parts ? launch_parts(d, partial, stream) : launch_extra(d, partial, stream);
      if (e != hipSuccess) return e;
    }
    if (w.few) {
      const ExtraArgs* const dx = c.dx && parts ? &d : nullptr;
      e = c.dtype == kF16 ? finish_few<f16>(c, w, dx, n0, n, ws, stream) : finish_few<bf16>(c, w, dx, n0, n, ws, stream);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace som
