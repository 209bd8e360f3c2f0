// The matrix product's kernel: C[i][j] = sum_k P(i, k) Q(j, k) on the matrix cores, with
// the epilogue of som_product or, where the k axis is split, fp32 partial sums.
//
// An operand lies in memory with k contiguous (KC: rows of its own index, P[i * ld
// + k]) or strided (rows of k, P[k * ld + i]); a feature-major weight matrix in the
// forward product is the strided kind, and the products of the backward pass have
// all three pairs.  A workgroup takes a BI x BJ tile of C and steps along k 128 bytes
// at a time (64 elements of 16 bits, 128 of 8): a step of an operand is BR * 128
// bytes of LDS in chunks of 16, moved straight from global memory (the lanes of a
// load write consecutive chunks; which global chunk each lane fetches is permuted, so
// that the fragment reads meet no bank twice):
//
//   KC   row r holds chunks c = 0..7 of its 128 bytes at slot c ^ (r / 2 % 8);
//        a lane reads the chunk (k group) of its row with one 128-bit read
//   KS   row k (64 of them) holds BR * 2 bytes in pairs of chunks (16 columns) at
//        pair ^ swizzle(k); a lane gets 4 k of its column from each transposing
//        64-bit read
//
// Where rows do not start on 16 bytes, at columns that end inside a chunk and in the
// last, partial step the chunks go through registers: a chunk that a row's end cuts is
// read as the 16 bytes up to that end and shifted, a row shorter than a chunk element
// by element, so no element outside the matrices is read, and what lies beyond k
// counts as zero in both operands (a NaN there cannot reach a sum).
//
// The matrix instructions take Q as their first operand: a lane then holds four
// consecutive j of one i, and puts them with one access into the LDS that the operands
// have left, from which the epilogue reads and writes whole rows of the tile.
//
// Bound, large: the matrix cores, at the clock that the card's power leaves them (8,192^3
// bf16 750 to 801 us, 1,370 to 1,470 TFLOP/s, and 8,192 x 4,096 x 16,384 775 to 832, 1,320 to
// 1,420, over the cards measured on; the instructions alone 1,950 to 2,000 on such data), less
// the tiles' start and epilogue; small: the launch and the latency of a step; few rows: the
// weights' bytes.
#pragma once

#include "dense.h"

namespace som {

struct ProductArgs {
  const void *P, *Q;
  int64_t ldp, ldq;          // elements
  int64_t I, J, K;
  int elem;                  // kF16, kBF16, kE4M3
  bool p_kc, q_kc;
  // epilogue
  float alpha;
  int act;
  const float *p_scale, *q_scale, *bias;
  const void* residual;
  int64_t ldr;
  void* pre;
  int64_t ldpre;
  void* out;
  int64_t ldo;
  int out_type;
  // launch
  float* partial;            // [splits][I][round_up(J, 8)] or nullptr
  int64_t k_split;           // elements of k per split (a multiple of the step)
  int splits;
  uint32_t tiles_i, tiles_j, per_xcd;
  bool dma;                  // rows of both operands start on 16 bytes
};

// Tile shapes, and the kernels of few rows (product_few.hip).
enum Shape { kShape256 = 0, kShape256x128, kShape128, kShape64, kShape32, kShape16, kShapes, kFew = kShapes };
struct ShapeInfo {
  int bi, bj;                // rows and columns of C
  int wgs;                   // workgroups that a CU holds
};
constexpr ShapeInfo kInfo[kShapes] = {{256, 256, 1}, {256, 128, 1}, {128, 128, 1}, {64, 128, 2}, {32, 128, 2}, {16, 128, 2}};
struct ProductPlan {
  int shape;
  int splits;
  int64_t k_split;
  size_t partial_floats;
};
// `dma`: the rows of both operands start on 16 bytes
ProductPlan plan_product(int64_t I, int64_t J, int64_t K, int elem, bool p_kc, bool q_kc, bool dma);
// Fills the launch's fields of `a` and enqueues it (and the join of a split k axis);
// `partial`: plan_product's floats.
hipError_t launch_product(ProductArgs a, float* partial, hipStream_t stream);
hipError_t launch_product_f16(int shape, const ProductArgs& a, hipStream_t stream);
hipError_t launch_product_bf16(int shape, const ProductArgs& a, hipStream_t stream);
hipError_t launch_product_e4m3(int shape, const ProductArgs& a, hipStream_t stream);
hipError_t launch_product_few(const ProductArgs& a, hipStream_t stream);

// dP = dy act'(pre), rounded to the type, and dP's column sums.
struct ActGradArgs {
  const void *dy, *pre;
  void* dp;                  // [M][ldp] or nullptr
  float *dbias, *part;       // or nullptr; part: act_grad_ws_floats
  int64_t lddy, ldpre, lddp, M, N;
  int elem, act;
};
size_t act_grad_ws_floats(int64_t M, int64_t N);
hipError_t launch_act_grad(const ActGradArgs& a, hipStream_t stream);

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef u4 u4_at1 __attribute__((aligned(1)));
typedef u4 u4_at2 __attribute__((aligned(2)));

constexpr int kStepBytes = 128;
constexpr int kXcds = 8;
constexpr int64_t kDmaMaxLd = int64_t(1) << 22;   // elements: a tile's offsets fit 32 bits

// ---------------------------------------------------------------------------
// Epilogue
// ---------------------------------------------------------------------------

constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4;   // som_act

constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + e^-z), within (8 + 2 |z|) 2^-24 of itself for z < 0 (the exponent's roundings), a few
// units of fp32 for z >= 0; 0 where it is below fp32's normal numbers (z < -87).
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z));
}

constexpr float kGeluK = 1.5957691216057308f;     // 2 sqrt(2 / pi): 1 + tanh(z) = 2 sigmoid(2 z)
constexpr float kGeluC = 0.044715f;

// The normal distribution's share below -|v|, and e = e^(-v^2 / 2): e t q(t) with t =
// 1 / (1 + 0.3 |v|).  q is the polynomial of degree 7 with the least largest relative error over
// |v| <= 14 (1.5e-7; fitted to the scaled complementary error function, 4.5e-7 as calculated in
// fp32), so no digits are lost far out.  e is within 1.5 v^2 2^-24 of itself (its exponent's
// roundings), the share within 2^-20 + 1.5 v^2 2^-24 of itself until it leaves fp32's normal
// numbers at -13.  `size`: |v|, or anything from 16 on where that is more.
__device__ __forceinline__ float normal_tail(float v, float size, float* e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, size, 1.0f));
  float q = fmaf(t, 0.0356747732f, -0.157203078f);
  q = fmaf(t, q, 0.2063535f);
  q = fmaf(t, q, -0.0536836423f);
  q = fmaf(t, q, 0.128561631f);
  q = fmaf(t, q, 0.0999134928f);
  q = fmaf(t, q, 0.120753959f);
  q = fmaf(t, q, 0.119629301f);
  *e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * v * v);
  return t * q * *e;
}

__device__ __forceinline__ void act8(int act, float (&v)[8]) {
  if (act == kActNone) return;
  if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] > 0.0f ? v[e] : (v[e] != v[e] ? v[e] : 0.0f);
  } else if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // v minus |v| times the share above v, or v times the share below; from 16 on the tail
      // is zero, which infinity must not meet (a NaN is one in the exponential)
      float exponential;
      const float size = fminf(fabsf(v[e]), 16.0f), tail = normal_tail(v[e], size, &exponential);
      v[e] = fmaf(-size, tail, fmaxf(v[e], 0.0f));
    }
  } else {
    // gelu_tanh: v sigmoid(k (v + c v^3)); silu: v sigmoid(v)
    const float k = act == kActSilu ? 1.0f : kGeluK, c = act == kActSilu ? 0.0f : kGeluK * kGeluC;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= sigmoid(v[e] * (act == kActSilu ? 1.0f : fmaf(c, v[e] * v[e], k)));
  }
}

// The activation's derivative.
__device__ __forceinline__ float act_grad(int act, float v) {
  switch (act) {
    case kActRelu:
      return v > 0.0f ? 1.0f : 0.0f;
    case kActGelu: {
      float e;
      const float tail = normal_tail(v, fabsf(v), &e), below = v >= 0.0f ? 1.0f - tail : tail;
      return fmaf(v * e, 0.39894228040143268f, below);
    }
    case kActGeluTanh: {
      // far out s (1 - s) is exactly 0 in fp32, and v^2 must not overflow to 0 times
      // infinity (bf16 goes up to 3.4e38); NaN stays NaN
      v = v > 1e4f ? 1e4f : v < -1e4f ? -1e4f : v;
      const float s = sigmoid(kGeluK * (v + kGeluC * v * v * v));
      return s + v * s * (1.0f - s) * kGeluK * (1.0f + 3.0f * kGeluC * v * v);
    }
    case kActSilu: {
      const float s = sigmoid(v);
      return s * (1.0f + v * (1.0f - s));
    }
    default:
      return 1.0f;
  }
}

// Rows of 16 bits go past the L2, whose lines the operands need (8,192 x 4,096 x 16,384
// 905 to 886 us); a lane's eight fp32 are two accesses of every other 16 bytes, which
// the L2 puts together (past it 4,096 x 2,048 x 16,384 took 305 us instead of 279).
template <typename T>
__device__ __forceinline__ void store8_stream(T* p, const float (&v)[8]) {
  typename Eight<T>::vec r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = static_cast<T>(v[e]);
  __builtin_nontemporal_store(r, reinterpret_cast<typename Eight<T>::at*>(p));
}

template <bool kWhole>
__device__ __forceinline__ void store8_as(int type, void* base, int64_t at, int n, const float (&v)[8]) {
  if (kWhole) n = 8;
  if (type == kF32)
    store8(static_cast<float*>(base) + at, n, v);
  else if (type == kF16)
    kWhole ? store8_stream(static_cast<f16*>(base) + at, v) : store8(static_cast<f16*>(base) + at, n, v);
  else
    kWhole ? store8_stream(static_cast<bf16*>(base) + at, v) : store8(static_cast<bf16*>(base) + at, n, v);
}

// What the epilogue takes from memory for eight columns: of all rows, and of one row
// (the residual as it lies there, so that it can be asked for ahead of its use).
struct ColumnTerms {
  float scale[8], bias[8];
};
struct RowTerms {
  float scale;
  u4 residual[2];
};

// n <= 0: nothing is read
__device__ __forceinline__ ColumnTerms column_terms(const ProductArgs& a, int64_t j, int n) {
  ColumnTerms c;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    c.scale[e] = 1.0f;
    c.bias[e] = 0.0f;
  }
  if (a.q_scale) load8(a.q_scale + j, n, c.scale);
  if (a.bias) load8(a.bias + j, n, c.bias);
  return c;
}

__device__ __forceinline__ RowTerms row_terms(const ProductArgs& a, int64_t i, int64_t j, int n) {
  RowTerms r;
  r.scale = a.alpha;
  r.residual[0] = r.residual[1] = u4{0, 0, 0, 0};
  if (n <= 0) return r;
  if (a.p_scale) r.scale *= a.p_scale[i];
  if (!a.residual) return r;
  if (a.out_type == kF32) {
    const float* p = static_cast<const float*>(a.residual) + i * a.ldr + j;
    if (n == 8) {
      r.residual[0] = *reinterpret_cast<const u4_at2*>(p);
      r.residual[1] = *reinterpret_cast<const u4_at2*>(p + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < n) r.residual[e / 4][e % 4] = __float_as_uint(p[e]);
    }
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

// The residual's eight values.
__device__ __forceinline__ void residual8(int type, const RowTerms& r, float (&v)[8]) {
  typedef f16 h8 __attribute__((ext_vector_type(8)));
  if (type == kF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(r.residual[e / 4][e % 4]);
  } else if (type == kF16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += static_cast<float>(__builtin_bit_cast(h8, r.residual[0])[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] += __uint_as_float(e % 2 ? r.residual[0][e / 2] & 0xffff0000u : r.residual[0][e / 2] << 16);
  }
}

template <bool kWhole>
__device__ __forceinline__ void finish_some(const ProductArgs& a, int64_t i, int64_t j, int n, float (&v)[8],
                                            const ColumnTerms& c, const RowTerms& r) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e] * r.scale, c.scale[e], c.bias[e]);
  if (a.pre) store8_as<kWhole>(a.out_type, a.pre, i * a.ldpre + j, n, v);
  act8(a.act, v);
  if (a.residual) residual8(a.out_type, r, v);
  store8_as<kWhole>(a.out_type, a.out, i * a.ldo + j, n, v);
}

// Columns [j, j + n), n in 1..8, of row i from their sums.
__device__ __forceinline__ void finish8(const ProductArgs& a, int64_t i, int64_t j, int n, float (&v)[8],
                                        const ColumnTerms& c, const RowTerms& r) {
  if (n == 8)
    finish_some<true>(a, i, j, n, v, c, r);
  else
    finish_some<false>(a, i, j, n, v, c, r);
}

// ---------------------------------------------------------------------------
// Operand steps in LDS
// ---------------------------------------------------------------------------

// Wait for all but the N newest vector-memory operations, and for this wave's LDS
// reads, then meet the workgroup.
template <int N>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The same for LDS alone: loads into registers stay on their way.
__device__ __forceinline__ void arrive_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 16 bytes per lane from base + off to LDS at `lds` (uniform) + 16 * lane.  A vector
// instruction may have written the base's scalar registers just before (a lane read
// into them): a memory instruction may read those five wait states later at the
// earliest, and the compiler, which keeps that distance elsewhere, does not look into
// this statement.  (m0 needs one.)
__device__ __forceinline__ void dma16(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}

// Pair swizzle of a k-strided row (see above): the rows that one transposing read
// takes (k % 4, k / 8 % 2 of them) go to different pairs of chunks.
template <int BR>
__device__ __forceinline__ int ks_swizzle(int k) {
  return BR >= 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
}

// A pointer that is the same in every lane, in scalar registers.
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
  return reinterpret_cast<const char*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// One operand's side of a workgroup: BR rows of C's axis, moved by THREADS threads.
template <int ES, bool KC, int BR, int THREADS>
struct Operand {
  static constexpr int kBytes = BR * kStepBytes;
  static constexpr int kChunks = kBytes / 16;
  static constexpr int kEach = (kChunks + THREADS - 1) / THREADS;    // per thread
  static constexpr int kPer = 16 / ES;                               // elements per chunk
  static constexpr int kStep = kStepBytes / ES;                      // k elements per step
  static_assert(KC || (ES == 2 && BR >= 64), "k-strided operands have 16 bits");
  static_assert(kChunks % 64 == 0, "whole waves move whole loads");

  const char* base;      // the tile's first row (KC) or column, at k = 0
  int64_t ld;            // bytes per row
  int64_t rows;          // rows (KC) or columns of the matrix from the tile's first on
  uint32_t off;          // this thread's first chunk from the tile's start
  uint32_t over;         // the same chunk of the tile's first row (KC)

  // this thread's nth chunk: position in LDS, and its row and first element
  static __device__ __forceinline__ int pos(int n) { return n * THREADS + static_cast<int>(threadIdx.x); }
  static __device__ __forceinline__ void place(int p, int* row, int* chunk) {
    if constexpr (KC) {
      *row = p >> 3;
      *chunk = (p & 7) ^ ((*row >> 1) & 7);
    } else {
      constexpr int kRow = BR / 8;
      *row = p / kRow;
      *chunk = (p % kRow) ^ (ks_swizzle<BR>(*row) << 1);
    }
  }
  static constexpr bool whole = kChunks % THREADS == 0;
  static __device__ __forceinline__ bool mine(int n) { return whole || pos(n) < kChunks; }

  __device__ __forceinline__ void init(const void* p, int64_t ld_elems, int64_t first, int64_t extent) {
    ld = ld_elems * ES;
    base = uniform(static_cast<const char*>(p) + (KC ? first * ld : first * ES));
    rows = extent - first;
    int r, c;
    place(pos(0), &r, &c);
    // chunks past the matrix's columns: the tile's first one, whose sums are not kept
    if (!KC && c * 8 >= rows) c = 0;
    off = static_cast<uint32_t>(r * ld + c * 16);
    over = static_cast<uint32_t>(c * 16);
  }
  // columns that end inside a chunk of this tile
  __device__ __forceinline__ bool ragged() const { return !KC && rows < BR && rows % 8 != 0; }
  __device__ __forceinline__ const char* at(int32_t k) const { return base + (KC ? int64_t(k) * ES : k * ld); }

  // Whole step from k on, asynchronously (rows on 16 bytes).  A thread's chunks lie kRowsEach rows apart at
  // one place of their rows (the swizzles repeat after 16 rows).  Rows past the matrix:
  // the tile's first one again.
  static constexpr int kRowsEach = KC ? THREADS / 8 : THREADS / (BR / 8);
  static_assert(kEach == 1 || kRowsEach % 16 == 0, "a thread's chunks are swizzled alike");
  // nth of the kEach loads of this wave
  __device__ __forceinline__ void fetch(int n, int32_t k, uint32_t lds) const {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds += wave * 1024 + n * THREADS * 16;
    if (!whole && n * THREADS + wave * 64 >= kChunks) return;
    if constexpr (!KC) {
      dma16(at(k) + n * (kRowsEach * ld), off, lds);
    } else {
      const int r = (threadIdx.x >> 3) + n * kRowsEach;
      dma16(at(k), r < rows ? off + static_cast<uint32_t>(n * kRowsEach * ld) : over, lds);
    }
  }

  // Steps through registers: 16 bytes at an address of any alignment.  Of a chunk that
  // the row's end cuts (KS: the matrix's last columns; KC, with kLast: `end`), the 16
  // bytes up to that end, which `store` or `load` shifts into place; the places after it
  // are zero.  A row shorter than a chunk goes element by element.
  // (Pointers into global memory by type: made from `uniform`'s integers they are not known
  // to be, and a flat load, which may be of LDS, holds up every wait for LDS.)
  template <typename V>
  using Global = const __attribute__((address_space(1))) V;
  static __device__ __forceinline__ u4 some(const char* p, int64_t n) {
    u4 v = {0, 0, 0, 0};
    if constexpr (ES == 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) v[e / 2] |= static_cast<uint32_t>(((Global<uint16_t>*)p)[e]) << (16 * (e % 2));
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < n) v[e / 4] |= static_cast<uint32_t>(((Global<uint8_t>*)p)[e]) << (8 * (e % 4));
    }
    return v;
  }
  static __device__ __forceinline__ u4 all(const char* p) {
    return ES == 2 ? u4(*(Global<u4_at2>*)p) : u4(*(Global<u4_at1>*)p);
  }
  // the last n (of kPer, 0 < n < kPer) elements moved to the front
  static __device__ __forceinline__ u4 front(u4 v, int n) {
    uint64_t lo = static_cast<uint64_t>(v[1]) << 32 | v[0], hi = static_cast<uint64_t>(v[3]) << 32 | v[2];
    const int bits = (kPer - n) * ES * 8;
    lo = bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits);
    hi = bits >= 64 ? 0 : hi >> bits;
    return u4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi),
              static_cast<uint32_t>(hi >> 32)};
  }
  // KS: columns in this thread's chunks, where the matrix's end cuts them, else 0
  __device__ __forceinline__ int cut() const {
    int r, c;
    place(pos(0), &r, &c);
    return !KC && c * 8 < rows && rows - c * 8 < 8 ? static_cast<int>(rows - c * 8) : 0;
  }
  // `extent`: columns (KS) or k (KC) of the matrix
  template <bool kLast>
  __device__ __forceinline__ void load(int32_t k, int32_t end, int64_t extent, u4 (&v)[kEach]) const {
    const char* const b = at(k);
    int r, c;
    place(pos(0), &r, &c);
    const int cols = cut();
    // KS: past the columns the tile's first chunk (its sums are not kept), where that is whole
    const bool none = !KC && cols == 0 && rows < 8;
    const int64_t at_col = KC ? c * 16 : c * 8 >= rows ? 0 : cols && extent >= 8 ? c * 16 - (8 - cols) * 2 : c * 16;
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      if (!mine(n)) continue;
      const int row = r + n * kRowsEach;
      const char* p = b + (KC && row >= rows ? 0 : row) * ld + at_col;     // 64 bits: any stride
      if constexpr (KC && kLast) {
        const int left = end - (k + c * kPer);
        if (left >= kPer)
          v[n] = all(p);
        else if (left <= 0)
          v[n] = u4{0, 0, 0, 0};
        else
          v[n] = extent >= kPer ? front(all(p - (kPer - left) * ES), left) : some(p, left);
      } else if constexpr (KC) {
        v[n] = all(p);
      } else {
        const bool in = !kLast || k + row < end;
        if (!in || none)
          v[n] = u4{0, 0, 0, 0};
        else if (extent >= 8)
          v[n] = all(p);
        else
          v[n] = some(p, cols);
      }
    }
  }
  // The same of a whole step, without a branch (KS: 8 columns and more): the number of
  // loads on their way is then known where one is waited for.  What is not kept is read
  // too: KS, past the columns, the tile's first 16 bytes or those up to the row's end.
  __device__ __forceinline__ void load_plain(int32_t k, u4 (&v)[kEach]) const {
    const char* const b = at(k);
    int r, c;
    place(pos(0), &r, &c);
    const int cols = cut();
    const int64_t first = rows < 8 ? (rows - 8) * 2 : 0;
    const int64_t at_col = KC ? c * 16 : c * 8 >= rows ? first : cols ? c * 16 - (8 - cols) * 2 : c * 16;
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
      const int row = r + n * kRowsEach;
      v[n] = all(b + (KC && row >= rows ? 0 : row) * ld + at_col);
    }
  }
  __device__ __forceinline__ void store(char* lds, int64_t extent, const u4 (&v)[kEach]) const {
    const int cols = cut();
    if (!KC && cols && extent >= 8) {
#pragma unroll
      for (int n = 0; n < kEach; ++n)
        if (mine(n)) *reinterpret_cast<u4*>(lds + pos(n) * 16) = front(v[n], cols);
    } else {
#pragma unroll
      for (int n = 0; n < kEach; ++n)
        if (mine(n)) *reinterpret_cast<u4*>(lds + pos(n) * 16) = v[n];
    }
  }

  // A lane's share of rows [16 t, 16 t + 16) of this wave's: `lane_base` is for
  // t = 0, k = 0 of a wave whose rows start at `first`.
  static __device__ __forceinline__ uint32_t lane_base(int first) {
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    if constexpr (KC) {
      return static_cast<uint32_t>((first + i) * kStepBytes + ((g ^ ((i >> 1) & 7)) << 4));
    } else {
      const int k = g * 8 + (i >> 2);
      return static_cast<uint32_t>(k * BR * 2 + ((((first >> 4) ^ ks_swizzle<BR>(k)) << 5) | (i & 3) << 3));
    }
  }
};

typedef short s8 __attribute__((ext_vector_type(8)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef f16 h2 __attribute__((ext_vector_type(2)));
typedef f16 h8 __attribute__((ext_vector_type(8)));
typedef bf16 b8 __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s4 lds_s4;
typedef __attribute__((address_space(3))) u4 lds_u4;

// 16 bytes (KC: chunk g + 4 h of the row; KS: k = 32 h + 8 g + 0..7 of the column).
template <bool KC, int BR>
__device__ __forceinline__ i4 fragment(lds_char* step, uint32_t lane_base, int t, int h) {
  if constexpr (KC) {
    const u4 v = *reinterpret_cast<lds_u4*>(step + ((lane_base ^ (h << 6)) + t * 16 * kStepBytes));
    return __builtin_bit_cast(i4, v);
  } else {
    const uint32_t at = (lane_base ^ (t << 5)) + h * 32 * BR * 2;
    union {
      s4 half[2];
      i4 all;
    } v;
    v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s4*>(step + at));
    v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s4*>(step + at + 4 * BR * 2));
    return v.all;
  }
}

// A fragment as the matrix instructions take it: 8 k of 16 bits, or two times 8 of 8
// bits, widened (exactly) to fp16.  The 8-bit matrix instructions are not used, a choice of
// digits over speed: they line products up before they add them and drop bits that a sum in
// fp32 keeps (errors of 2^-17 of the sum of magnitudes against the 64-bit oracle, the
// instructions of 32 k and of 128 k alike), but run at twice the 16-bit rate, which bounds this
// (16,384 x 4,096 x 4,096 378 us, 1,456 TFLOP/s).
template <int E>
struct Frag {
  static constexpr int kParts = E == kE4M3 ? 2 : 1;
  i4 part[kParts];
  __device__ __forceinline__ explicit Frag(i4 v) {
    if constexpr (E == kE4M3) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        h8 w;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const h2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * p + d], 1.0f, false);
          const h2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[2 * p + d], 1.0f, true);
          w[4 * d] = lo[0];
          w[4 * d + 1] = lo[1];
          w[4 * d + 2] = hi[0];
          w[4 * d + 3] = hi[1];
        }
        part[p] = __builtin_bit_cast(i4, w);
      }
    } else {
      part[0] = v;
    }
  }
};

// c + the products over the fragments' k.
template <int E>
__device__ __forceinline__ f4 mfma(const Frag<E>& q, const Frag<E>& p, f4 c) {
#pragma unroll
  for (int i = 0; i < Frag<E>::kParts; ++i) {
    if constexpr (E == kBF16)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, q.part[i]), __builtin_bit_cast(b8, p.part[i]),
                                                  c, 0, 0, 0);
    else
      c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, q.part[i]), __builtin_bit_cast(h8, p.part[i]),
                                                 c, 0, 0, 0);
  }
  return c;
}

// ---------------------------------------------------------------------------
// The kernel
// ---------------------------------------------------------------------------

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

// WI x WJ waves, each with TI x TJ tiles of 16 x 16; NS steps in LDS.
template <int E, bool PKC, bool QKC, int WI, int WJ, int TI, int TJ, int NS>
__global__ void __launch_bounds__(WI* WJ * 64) k_product(const ProductArgs a) {
  constexpr int ES = E == kE4M3 ? 1 : 2;
  constexpr int BI = WI * TI * 16, BJ = WJ * TJ * 16, THREADS = WI * WJ * 64;
  using OpP = Operand<ES, PKC, BI, THREADS>;
  using OpQ = Operand<ES, QKC, BJ, THREADS>;
  constexpr int kStage = OpP::kBytes + OpQ::kBytes;
  constexpr int kStep = kStepBytes / ES;
  extern __shared__ __align__(1024) char lds[];

  // XCD x (workgroups are dealt to the XCDs in turn) takes the tiles [x * per_xcd, ...):
  // tiles in bands of kBand rows of tiles, so that the ones it runs at once share
  // both operands' rows in its L2
  constexpr uint32_t kBand = 4;
  const uint32_t lin = blockIdx.x % kXcds * a.per_xcd + blockIdx.x / kXcds;
  const uint32_t tiles = a.tiles_i * a.tiles_j;
  if (lin >= tiles * a.splits) return;
  // (divisions go through the vector unit: back to scalar registers)
  const uint32_t split = __builtin_amdgcn_readfirstlane(lin / tiles), rest = lin - split * tiles;
  const uint32_t band = __builtin_amdgcn_readfirstlane(rest / (kBand * a.tiles_j)), in = rest - band * kBand * a.tiles_j;
  const uint32_t height = min(kBand, a.tiles_i - band * kBand);
  const uint32_t across = __builtin_amdgcn_readfirstlane(in / height);
  const int64_t i0 = static_cast<int64_t>(band * kBand + (in - across * height)) * BI;
  const int64_t j0 = static_cast<int64_t>(across) * BJ;
  const int32_t k0 = static_cast<int32_t>(split * a.k_split);
  const int32_t k1 = static_cast<int32_t>(min(a.K, k0 + a.k_split));

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  OpP p;
  OpQ q;
  p.init(a.P, a.ldp, i0, a.I);
  q.init(a.Q, a.ldq, j0, a.J);
  const uint32_t pb = OpP::lane_base(wi * TI * 16), qb = OpQ::lane_base(wj * TJ * 16);
  lds_char* const l3 = (lds_char*)lds;
  const uint32_t l0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(l3));

  f4 acc[TI][TJ];
#pragma unroll
  for (int x = 0; x < TI; ++x)
#pragma unroll
    for (int y = 0; y < TJ; ++y) acc[x][y] = f4{0.0f, 0.0f, 0.0f, 0.0f};

  // the fragments of half a step
  struct Half {
    i4 q[TJ], p[TI];
  };
  auto read_one = [&](Half& f, int slot, int h, int r) __attribute__((always_inline)) {
    lds_char* sp = l3 + slot * kStage;
    if (r < TJ)
      f.q[r] = fragment<QKC, BJ>(sp + OpP::kBytes, qb, r, h);
    else
      f.p[r - TJ] = fragment<PKC, BI>(sp, pb, r - TJ, h);
  };
  auto read = [&](Half& f, int slot, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < TJ + TI; ++r) read_one(f, slot, h, r);
  };
  auto multiply_row = [&](const Half& f, int x) __attribute__((always_inline)) {
    const Frag<E> fp(f.p[x]);
#pragma unroll
    for (int y = 0; y < TJ; ++y) acc[x][y] = mfma<E>(Frag<E>(f.q[y]), fp, acc[x][y]);
  };

  Half f[2];
  // products of `now`, row of tiles by row; between them half h of the step in `from` is
  // read into `next`, and `more` of each row is done
  auto phase = [&](const Half& now, Half& next, int from, int h, auto more) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < TI; ++x) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = x * (TI + TJ) / TI; r < (x + 1) * (TI + TJ) / TI; ++r) read_one(next, from, h, r);
      more(x);
      multiply_row(now, x);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  const int32_t steps = (k1 - k0 + kStep - 1) / kStep;
  int32_t t = 0;
  if (a.dma && !p.ragged() && !q.ragged()) {
    // Whole steps.  Step t's second half is read while its first is multiplied; then, all
    // of step t being read and step t + 1 there, one barrier; t + 1's first half is read
    // while t's second is multiplied, and step t + NS is sent for into t's place.  Reads
    // and loads are spread over the products, row of tiles by row: a wave issues in order,
    // and one that waits for the memory unit's queue starts no product (all loads of a
    // step at once: 1,313 TFLOP/s at 8,192^3 in bf16).
    const int32_t full = (k1 - k0) / kStep;
    // loads of this wave per step: the last one of P may be the other waves'
    constexpr int kMost = OpP::kEach + OpQ::kEach;
    static_assert(OpQ::whole, "every wave moves the same share of Q");
    const bool most = OpP::whole || (OpP::kEach - 1) * THREADS + wave * 64 < OpP::kChunks;
    auto fetch_one = [&](int n, int32_t s, int slot) __attribute__((always_inline)) {
      const uint32_t at = l0 + static_cast<uint32_t>(slot) * kStage;
      if (n < OpP::kEach)
        p.fetch(n, k0 + s * kStep, at);
      else
        q.fetch(n - OpP::kEach, k0 + s * kStep, at + OpP::kBytes);
    };
    // step s has arrived, with the steps after it up to the newest on their way
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
    int slot = 0;
    auto step = [&](auto fetches) __attribute__((always_inline)) {
      phase(f[0], f[1], slot, 1, [](int) {});
      arrived(t + 1, NS - 2);
      const int place = slot;
      slot = slot + 1 == NS ? 0 : slot + 1;
      // (after the last step: bytes that no product uses)
      phase(f[1], f[0], slot, 0, [&](int x) __attribute__((always_inline)) {
        if constexpr (decltype(fetches)::value)
#pragma unroll
          for (int n = x * kMost / TI; n < (x + 1) * kMost / TI; ++n) fetch_one(n, t + NS, place);
      });
    };
    if (full > 0) {
#pragma unroll
      for (int s = 0; s < NS; ++s)
        if (s < full)
#pragma unroll
          for (int n = 0; n < kMost; ++n) fetch_one(n, s, s);
      arrived(0, NS - 1);
      read(f[0], 0, 0);
      for (; t < full - NS; ++t) step(Yes{});
      for (; t < full; ++t) step(No{});
    }
  }
  if (t < steps) {
    // Through registers: kDeep steps on their way, two in LDS.  (One on its way costs a
    // memory latency per step, 0.8 us measured.)  A tile of 256 x 256 has the registers for
    // one.
    constexpr int kDeep = TI * TJ >= 32 ? 1 : TI * TJ >= 16 ? 2 : 3;
    u4 vp[kDeep][OpP::kEach], vq[kDeep][OpQ::kEach];
    const int64_t p_extent = PKC ? a.K : a.I, q_extent = QKC ? a.K : a.J;
    const int32_t full = (k1 - k0) / kStep;
    auto load = [&](int32_t s, int d) __attribute__((always_inline)) {
      const int32_t k = k0 + s * kStep;
      if (s < full) {
        p.template load<false>(k, k1, p_extent, vp[d]);
        q.template load<false>(k, k1, q_extent, vq[d]);
      } else {
        p.template load<true>(k, k1, p_extent, vp[d]);
        q.template load<true>(k, k1, q_extent, vq[d]);
      }
    };
    auto load_plain = [&](int32_t s, int d) __attribute__((always_inline)) {
      p.load_plain(k0 + s * kStep, vp[d]);
      q.load_plain(k0 + s * kStep, vq[d]);
    };
    int slot = 0;
    auto put = [&](int d) __attribute__((always_inline)) {
      p.store(lds + slot * kStage, p_extent, vp[d]);
      q.store(lds + slot * kStage + OpP::kBytes, q_extent, vq[d]);
      arrive_lds();
    };
    auto multiply = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        read(f[0], slot, h);
#pragma unroll
        for (int x = 0; x < TI; ++x) multiply_row(f[0], x);
      }
      slot ^= 1;
      ++t;
    };
    if (kDeep > 1 && full - t >= 2 * kDeep && (PKC || p_extent >= 8) && (QKC || q_extent >= 8)) {
#pragma unroll
      for (int d = 0; d < kDeep; ++d) load_plain(t + d, d);
      do {
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
          put(d);
          load_plain(t + kDeep, d);
          multiply();
        }
      } while (t + 2 * kDeep <= full);
    } else {
#pragma unroll
      for (int d = 0; d < kDeep; ++d)
        if (t + d < steps) load(t + d, d);
    }
    while (t < steps) {
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        if (t >= steps) break;
        put(d);
        if (t + kDeep < steps) load(t + kDeep, d);
        multiply();
      }
    }
  }

  // The epilogue by rows: up to 64 rows of the wave's columns at a time go through its own
  // part of LDS, so that a lane has eight consecutive columns and the wave's reads and
  // writes of C are whole lines.  Quads of columns are swizzled by row: the 16 lanes that
  // write a quad of their rows, and the ones that read two rows, meet no bank twice.
  // What a row needs from memory is asked for kAhead loads of the wave before.
  constexpr int kCols = TJ * 16, kLanes = kCols / 8, kRows = 64 / kLanes;    // rows per access of the wave
  constexpr int kBatch = TI < 4 ? TI : 4, kAhead = 3;
  static_assert(WI * WJ * kBatch * 16 * kCols * 4 <= NS * kStage, "the rows fit the steps' place");
  static_assert(TI % kBatch == 0 && TI / kBatch <= 2 && (TJ == 2 || TJ == 4), "see below");
  __syncthreads();                     // every wave is done with the steps
  typedef __attribute__((address_space(3))) f4 lds_f4;
  lds_char* const mine = l3 + wave * (kBatch * 16 * kCols * 4);
  const int lane = threadIdx.x & 63;
  auto quad = [&](int row, int k) {
    const int sw = TJ == 4 ? row : row >> 1;
    return reinterpret_cast<lds_f4*>(mine + (row * kCols + ((k ^ sw) & (TJ * 4 - 1)) * 4) * 4);
  };
  const int col = lane % kLanes;
  const int64_t j = j0 + wj * kCols + col * 8;
  const int n = static_cast<int>(min<int64_t>(8, a.J - j));
  const int64_t first = i0 + wi * TI * 16 + lane / kLanes;
  constexpr int kGroups = TI * 16 / kRows;                      // accesses of kRows rows
  const int32_t ld_part = static_cast<int32_t>((a.J + 7) / 8 * 8);
  // rows [b * kBatch * 16, ...) of the wave's into LDS
  auto stage = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
#pragma unroll
      for (int y = 0; y < TJ; ++y) {
        f4 v = acc[x][y];
        if constexpr (TI > kBatch) v = b ? acc[kBatch + x][y] : v;
        *quad(x * 16 + (lane & 15), y * 4 + (lane >> 4)) = v;
      }
    __builtin_amdgcn_wave_barrier();
  };
  // `take`(access, row of C, its eight sums) for every access
  auto rows = [&](auto take) __attribute__((always_inline)) {
#pragma unroll 1
    for (int b = 0; b < TI / kBatch; ++b) {
      stage(b);
#pragma unroll 1
      for (int r = 0; r < kBatch * 16; r += kRows) {
        const int row = r + lane / kLanes, g = (b * kBatch * 16 + r) / kRows;
        const f4 lo = *quad(row, 2 * col), hi = *quad(row, 2 * col + 1);
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        take(g, first + g * kRows, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  };
  auto terms = [&](int g) __attribute__((always_inline)) {
    const int64_t i = first + g * kRows;
    return row_terms(a, i, j, g < kGroups && i < a.I ? n : 0);
  };
  if (a.splits > 1) {
    rows([&](int, int64_t i, float (&v)[8]) __attribute__((always_inline)) {
      if (i < a.I && n > 0) store8(a.partial + (split * a.I + i) * ld_part + j, 8, v);
    });
    return;
  }
  ColumnTerms ct = column_terms(a, j, n);
  // (here, and not at their first use: in the loop below that would be a wait for the
  // stores of the rows before, since loads and stores are counted together)
#pragma unroll
  for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(ct.scale[e]), "+v"(ct.bias[e]));
  if (a.residual || a.p_scale) {
    RowTerms ahead[kAhead];
#pragma unroll
    for (int g = 0; g < kAhead; ++g) ahead[g] = terms(g);
    rows([&](int g, int64_t i, float (&v)[8]) __attribute__((always_inline)) {
      const RowTerms now = ahead[0];
#pragma unroll
      for (int k = 0; k + 1 < kAhead; ++k) ahead[k] = ahead[k + 1];
      ahead[kAhead - 1] = terms(g + kAhead);
      if (i < a.I && n > 0) finish8(a, i, j, n, v, ct, now);
    });
  } else {
    RowTerms none;
    none.scale = a.alpha;
    rows([&](int, int64_t i, float (&v)[8]) __attribute__((always_inline)) {
      if (i < a.I && n > 0) finish8(a, i, j, n, v, ct, none);
    });
  }
}

}  // namespace som
