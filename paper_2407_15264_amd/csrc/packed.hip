// Activations kept in 8 bits for the backward pass, and the gradients that read
// them.
//
// A block of 32 consecutive values of a row shares a power of two 2^s and keeps
// q = rint(x 2^-s) in [-127, 127].  With a power of two the quotient is exact, so
// only rint rounds, the kept value q 2^s has at most 7 significant bits, and it is
// exact in bfloat16: the weight gradient's products need no rounding.
//
// s from the largest magnitude's bits: floor(log2 amax) - 6, or one more where
// amax 2^-s would round to 128, that is where its mantissa is at least 127.5 / 64:
// adding 2^16 to the bits carries into the exponent exactly then.
//
// The passes over rows are bound by memory.  A lane takes 8 consecutive values, a
// block of 32 is four neighbouring lanes', and the largest magnitude crosses them
// in two exchanges.  Measured: 203003 x 1024 bf16 kept in 112 us, 5.6 TB/s read and
// written, and read back in 88; gated silu of 65537 x 1024 bf16 in 93 us with its kept
// input, its gradient in 90 (5.8 and 6.0), gelu in 98 and 103, which its arithmetic
// bounds.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lsmgnn.h"
#include "rows.h"

namespace lsm_packed {

using namespace lsm_rows;

constexpr int kLane = 8;                            // values per lane
constexpr int kPack = (int)LSMGNN_PACK_BLOCK;       // values per block
constexpr int kQuads = kPack / kLane;               // lanes per block

// A lane's place: row, block of the row, first element.
struct Place {
  uint64_t row;
  uint32_t block, col;
  int count;  // its values: kLane, or fewer at the end of a row, or none
};

struct Cut {
  uint64_t rows;
  uint32_t dim, nb;       // values and blocks of a row
  uint64_t div64, div32;  // by the lanes of a row (see rows.h)
};

__device__ __forceinline__ Place place_of(const Cut &c, uint64_t base, uint32_t x) {
  const uint32_t lanes = c.nb * kQuads;
  const uint64_t r0 = __umul64hi(base, c.div64);
  x += (uint32_t)(base - r0 * lanes);
  const uint32_t r = (uint32_t)((x * c.div32) >> 32), l = x - r * lanes;
  Place p;
  p.row = r0 + r;
  p.block = l / kQuads;
  p.col = l * kLane;
  p.count = p.row >= c.rows || p.col >= c.dim ? 0 : c.dim - p.col < kLane ? (int)(c.dim - p.col) : kLane;
  return p;
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, int count, float (&v)[kLane]) {
  if (count == kLane) {
    T t[kLane];
    load_row_once(p, t);
#pragma unroll
    for (int e = 0; e < kLane; ++e) v[e] = (float)t[e];
  } else {
#pragma unroll
    for (int e = 0; e < kLane; ++e) v[e] = e < count ? (float)p[e] : 0.0f;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int count, const float (&v)[kLane]) {
  T t[kLane];
#pragma unroll
  for (int e = 0; e < kLane; ++e) t[e] = (T)v[e];
  if (count == kLane) {
    store_row_once(p, t);
  } else {
#pragma unroll
    for (int e = 0; e < kLane; ++e)
      if (e < count) p[e] = t[e];
  }
}

constexpr uint32_t kInf = 0x7f800000u;  // a float's bits

// The largest magnitude's bits.
__device__ __forceinline__ uint32_t largest(const float (&v)[kLane]) {
  uint32_t big = 0;
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    const uint32_t m = __float_as_uint(v[e]) & 0x7fffffffu;
    big = m > big ? m : big;
  }
  return big;
}

// Keep a block's values: its lanes' quotients at q, the scale byte by its first
// lane.  Every lane of the wave calls it.
__device__ __forceinline__ void keep8(const float (&v)[kLane], const Place &p, int8_t *q, uint8_t *scale) {
  uint32_t big = largest(v);
  const uint32_t a = __shfl_xor(big, 1);
  big = a > big ? a : big;
  const uint32_t b = __shfl_xor(big, 2);
  big = b > big ? b : big;
  const bool fine = big < kInf;
  const int32_t field = (int32_t)((big + 0x10000u) >> 23) - 6;  // s + 127
  const uint32_t byte = !fine ? 255u : field < 1 ? 1u : (uint32_t)field;
  const float per_unit = __uint_as_float((254u - byte) << 23);  // 2^-s
  if (p.count == 0) return;
  int8_t o[kLane];
  // x 2^-s + 1.5 2^23 rounds to a whole number, to even, and its low byte is q
#pragma unroll
  for (int e = 0; e < kLane; ++e)
    o[e] = fine ? (int8_t)__float_as_uint(__builtin_fmaf(v[e], per_unit, 12582912.0f)) : (int8_t)0;
  if (p.count == kLane) {
    store_row(q, o);
  } else {
#pragma unroll
    for (int e = 0; e < kLane; ++e)
      if (e < p.count) q[e] = o[e];
  }
  if (p.col % kPack == 0) *scale = (uint8_t)byte;
}

// The kept values.  Scale 255 is 2^128, infinity, and its q are 0: NaN.
__device__ __forceinline__ void kept8(const int8_t *q, const uint8_t *scale, int count, float (&v)[kLane]) {
  const float unit = __uint_as_float(count ? (uint32_t)*scale << 23 : 0);
  int8_t t[kLane];
  if (count == kLane) {
    load_row(q, t);
  } else {
#pragma unroll
    for (int e = 0; e < kLane; ++e) t[e] = e < count ? q[e] : (int8_t)0;
  }
#pragma unroll
  for (int e = 0; e < kLane; ++e) v[e] = (float)t[e] * unit;
}

// exp(-a) = e 2^n for 0 <= a <= 800, e to about the last bit in [0.7, 1.5]: a log2(e) in
// two parts.  kRest: of a + rest, |rest| <= 2^-24 a.
template <bool kRest = false>
__device__ __forceinline__ float exp_neg(float a, int *n, float rest = 0.0f) {
#pragma clang fp contract(off)
  const float whole = rintf(a * -1.44269504088896340736f);
  float part = __builtin_fmaf(a, -1.9259629911266175e-8f, __builtin_fmaf(a, -1.44269504088896340736f, -whole));
  if (kRest) part = __builtin_fmaf(rest, -1.44269504088896340736f, part);
  *n = (int)whole;
  return __builtin_amdgcn_exp2f(part);
}

// Products of activations with other factors.  A float16 row's values, and their
// products, are far from a float's limits; those of the other types are not.
template <typename T>
constexpr bool kWide = !std::is_same<T, _Float16>::value;

// A factor as m 2^up, 0.5 <= |m| < 1 (0, infinities and NaNs as they are, up = 0): a
// product of such mantissas neither overflows nor underflows before its exponents
// are added to it.
template <typename T>
__device__ __forceinline__ float mantissa(float v, int *up) {
  if (!kWide<T>) return v;
  *up += __builtin_amdgcn_frexp_expf(v);
  return __builtin_amdgcn_frexp_mantf(v);
}

template <typename T>
__device__ __forceinline__ float scaled(float v, int up) {
  return kWide<T> ? __builtin_amdgcn_ldexpf(v, up) : v;
}

// exp(y^2 / 2) Phi(-y) = exp(y^2 / 2) erfc(y / sqrt 2) / 2 for 0 <= y <= 32, r times a
// polynomial in 1 - 8 r, r = 1 / (y + 4): fitted to the function for the least relative
// error, 1.6e-8.  In 32 bits, everywhere: 10 units of 2^-24 with the reciprocal's own
// error, 7 where kFull takes that away.
template <bool kFull>
__device__ __forceinline__ float scaled_tail(float y) {
  const float d = y + 4.0f;
  float r = __builtin_amdgcn_rcpf(d);
  if (kFull) r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
  const float t = __builtin_fmaf(-8.0f, r, 1.0f);
  float q = -1.569715823e-04f;
  q = __builtin_fmaf(q, t, 1.337611611e-04f);
  q = __builtin_fmaf(q, t, 1.567938598e-03f);
  q = __builtin_fmaf(q, t, -3.480502637e-03f);
  q = __builtin_fmaf(q, t, -7.516742218e-03f);
  q = __builtin_fmaf(q, t, 6.039651111e-02f);
  q = __builtin_fmaf(q, t, -1.865253896e-01f);
  q = __builtin_fmaf(q, t, 3.871374726e-01f);
  q = __builtin_fmaf(q, t, -6.078965068e-01f);
  q = __builtin_fmaf(q, t, 7.552851439e-01f);
  return r * q;
}

// f(x) and f'(x) of a finite x or a NaN, both to be multiplied by 2^up at last (0 if not
// kWide), so that a product with another factor is rounded once where it is subnormal.
// To 16 units of 2^-24 where x is negative and they are small, too (Phi from 1 + erf
// would lose all of them at -5.5); with 32-bit rows the reciprocals' own error is taken
// away and that of gelu's square, x^2 / 2 units in its tail, which 16 bits do not show.
template <uint32_t kAct, typename T>
__device__ __forceinline__ void act(float x, float *f, float *df, int *up) {
  constexpr bool kFull = sizeof(T) == 4;
  // past these |x|, where a is 400 or 512, exp(-a) is 0 to any factor a float can have
  const float y = fminf(fabsf(x), kAct == LSMGNN_SILU ? 400.0f : 32.0f);
  int n;
  if (kAct == LSMGNN_SILU) {
    // p = 1 / (1 + exp(-x)) and 1 - p from t = exp(-|x|), which cannot overflow
    const float e = exp_neg(y, &n), t = __builtin_amdgcn_ldexpf(e, n), d = 1.0f + t;
    float r = __builtin_amdgcn_rcpf(d);
    if (kFull) r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
    const float p = x < 0.0f ? (kWide<T> ? e : t) * r : r, rest = x < 0.0f ? r : t * r;
    *f = x * p;
    *df = p * __builtin_fmaf(x, rest, 1.0f);
  } else {
    // Phi(-y) = exp(-a) tail and the density exp(-a) 0.3989.. with a = y^2 / 2: x Phi(-y) and
    // Phi(-y) - y density are f and f' where x < 0, else what x and 1 have more than f and f'
    const float half = 0.5f * y, a = half * y;
    const float e = exp_neg<kFull>(a, &n, kFull ? __builtin_fmaf(half, y, -a) : 0.0f);
    const float tail = scaled_tail<kFull>(y);
    const float s = kWide<T> ? e : __builtin_amdgcn_ldexpf(e, n);
    const float less = y * (s * tail), dless = s * __builtin_fmaf(fabsf(x), -0.39894228040143268f, tail);
    *f = x < 0.0f ? -less : x - scaled<T>(less, n);
    *df = x < 0.0f ? dless : 1.0f - scaled<T>(dless, n);
  }
  *up = kWide<T> && x < 0.0f ? n : 0;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_pack(Cut c, const T *x, uint64_t ld, int8_t *q, uint8_t *scale) {
  const Place p = place_of(c, (uint64_t)blockIdx.x * kBlock, threadIdx.x);
  float v[kLane];
  load8(x + p.row * ld + p.col, p.count, v);
  keep8(v, p, q + p.row * c.dim + p.col, scale + p.row * c.nb + p.block);
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_unpack(Cut c, const int8_t *q, const uint8_t *scale, T *out, uint64_t ld) {
  const Place p = place_of(c, (uint64_t)blockIdx.x * kBlock, threadIdx.x);
  if (p.count == 0) return;
  float v[kLane];
  kept8(q + p.row * c.dim + p.col, scale + p.row * c.nb + p.block, p.count, v);
  store8(out + p.row * ld + p.col, p.count, v);
}

// A wave whose factors are all below this multiplies them as they are: f and f' are at
// most |x| and 1.1, 2^-up included 1.5 |x|.  Any other takes the mantissas' way (kFar),
// at three instructions more a factor: gated silu of 65537 x 1024 bf16, backward, 91 us;
// 96 where every wave does.
constexpr float kNear = 0x1p40f;

// At the head of the rare side of a branch: the compiler would compute both sides in
// every lane and select (ungated, backward: 60 us became 102).
__device__ __forceinline__ void rarely() { asm volatile(""); }

template <uint32_t kAct, typename T, bool kGated, bool kFar>
__device__ __forceinline__ void forward8(const float (&a)[kLane], const float (&b)[kLane], float (&o)[kLane]) {
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    const float x = a[e], gate = kGated ? b[e] : 1.0f;
    float f, df;
    int up;
    act<kAct, T>(x, &f, &df, &up);
    if (kGated) f *= kFar ? mantissa<T>(gate, &up) : gate;
    o[e] = scaled<T>(f, up);
    if (kFar) {
      // f(inf) = inf, f(-inf) is the formulas' NaN; an infinite gate of an f that is 0
      // in 32 bits alone
      if (fabsf(x) == __builtin_inff())
        o[e] = (x > 0.0f ? x : __builtin_nanf("")) * gate;
      else if (kGated && fabsf(gate) == __builtin_inff())
        o[e] = x * gate;
    }
  }
}

// The gradients of a lane's values, that of the gate into b.
template <uint32_t kAct, typename T, bool kGated, bool kFar>
__device__ __forceinline__ void backward8(const float (&g)[kLane], const float (&a)[kLane], float (&b)[kLane],
                                          float (&o)[kLane]) {
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    // a value of 2^128 is an infinity in a float: where its slope is asked for the
    // largest float stands for it
    auto finite = [](float v) { return fabsf(v) == __builtin_inff() ? copysignf(0x1.fffffep127f, v) : v; };
    float f, df;
    int up;
    act<kAct, T>(kFar ? finite(a[e]) : a[e], &f, &df, &up);
    const float m = kFar ? mantissa<T>(g[e], &up) : g[e];
    int up_b = up;
    if (kGated)
      o[e] = scaled<T>(m * (kFar ? mantissa<T>(finite(b[e]), &up_b) : b[e]) * df, up_b);
    else
      o[e] = scaled<T>(m * df, up);
    if (kGated) b[e] = scaled<T>(m * f, up);
  }
}

// One place a thread, as in the other passes: with two, whose loads are in flight
// together, gated silu of 65537 x 1024 bf16 takes 96 us instead of 92, its gradient 93
// instead of 92.
template <typename T, uint32_t kAct, bool kGated>
__global__ __launch_bounds__(kBlock) void k_act(Cut c, const T *x, uint64_t xld, T *y, uint64_t yld, int8_t *q,
                                                uint8_t *scale) {
  constexpr int kRows = kGated ? 2 : 1;  // kept rows of a row
  const Place p = place_of(c, (uint64_t)blockIdx.x * kBlock, threadIdx.x);
  float a[kLane], b[kLane], o[kLane];
  const T *row = x + p.row * xld + p.col;
  load8(row, p.count, a);
  if (kGated) load8(row + c.dim, p.count, b);
  const uint32_t big_a = largest(a), big_b = kGated ? largest(b) : 0;
  if (__any((big_a > big_b ? big_a : big_b) >= __float_as_uint(kNear))) {
    rarely();
    forward8<kAct, T, kGated, true>(a, b, o);
  } else {
    forward8<kAct, T, kGated, false>(a, b, o);
  }
  if (p.count) store8(y + p.row * yld + p.col, p.count, o);
  int8_t *qp = q + p.row * kRows * c.dim + p.col;
  uint8_t *sp = scale + p.row * kRows * c.nb + p.block;
  keep8(a, p, qp, sp);
  if (kGated) keep8(b, p, qp + c.dim, sp + c.nb);
}

template <typename T, uint32_t kAct, bool kGated>
__global__ __launch_bounds__(kBlock) void k_act_grad(Cut c, const T *dy, uint64_t dyld, const int8_t *q,
                                                     const uint8_t *scale, T *dx, uint64_t dxld) {
  constexpr int kRows = kGated ? 2 : 1;
  const Place p = place_of(c, (uint64_t)blockIdx.x * kBlock, threadIdx.x);
  float g[kLane], a[kLane], b[kLane], o[kLane];
  const int8_t *qp = q + p.row * kRows * c.dim + p.col;
  const uint8_t *sp = scale + p.row * kRows * c.nb + p.block;
  load8(dy + p.row * dyld + p.col, p.count, g);
  kept8(qp, sp, p.count, a);
  if (kGated) kept8(qp + c.dim, sp + c.nb, p.count, b);
  float big = 0.0f;  // a NaN is no larger: it comes through either way
  if (kWide<T>)
#pragma unroll
    for (int e = 0; e < kLane; ++e) {
      big = fmaxf(fmaxf(big, fabsf(g[e])), fabsf(a[e]));
      if (kGated) big = fmaxf(big, fabsf(b[e]));
    }
  if (__any(big >= kNear)) {
    rarely();
    backward8<kAct, T, kGated, true>(g, a, b, o);
  } else {
    backward8<kAct, T, kGated, false>(g, a, b, o);
  }
  if (p.count == 0) return;
  T *to = dx + p.row * dxld + p.col;
  store8(to, p.count, o);
  if (kGated) store8(to + c.dim, p.count, b);
}

Cut cut_of(uint64_t rows, uint64_t dim) {
  Cut c{};
  c.rows = rows;
  c.dim = (uint32_t)dim;
  c.nb = (uint32_t)((dim + kPack - 1) / kPack);
  c.div64 = ~0ull / (c.nb * kQuads) + 1;
  c.div32 = divider(c.nb * kQuads);
  return c;
}

uint64_t blocks_of(const Cut &c) { return blocks_for(c.rows * c.nb * kQuads, kBlock); }

// f(cut, first row) for launches of all rows.
template <typename F>
void cuts_of(uint64_t rows, uint64_t dim, F f) {
  in_launches(rows, blocks_for(dim, kPack) * kQuads, [&](uint64_t r, uint64_t n) { f(cut_of(n, dim), r); });
}

// ------------------------------------------------------------ weight gradient
// dw[e] = sum over the expert's rows of x^T dy, on the bfloat16 matrix units with
// 32-bit sums.  The kept values are exact in bfloat16; dy is one bfloat16, or the
// sum of two (float16) or three (float32), each multiplied by itself, so that every
// product is exact; the three end at 2^-133, a bfloat16's least.
//
// A block computes a tile of dw[e] over kc consecutive rows of the expert; an
// expert with more rows has its partial sums added, in order, by a second kernel.
// kc is a function of the sizes.  Both operands lie with the summed index (the row)
// outermost, and the matrix units take 8 values of it from a lane: a thread loads a
// few neighbouring columns of 8 rows, and turns them over in registers while it
// widens them, so that LDS holds each column's 8 rows as one 16-byte piece.
// 16 pieces make a 256-byte line of LDS; a piece's place in its line is exchanged
// by the line's number, which keeps both the threads' writes (a column every few)
// and the matrix units' reads (32 columns) free of bank conflicts.
//
// Measured: 1024 x 256 of 203003 rows bf16 in 136 to 152 us, 700 to 780 TFLOP/s, the
// second kernel 13 us; a product of large bf16 matrices reaches 1140.  Staging (the
// widening and the turning over) bounds it, unevenly: in steps of 32 rows a tile of 256
// has units of x for half of the threads, whose waves the others wait for, and so have
// a tile of 128 with dy in several parts and one of 64.  The threads without a unit
// load past the buffer's end, that is nothing.

constexpr uint32_t kXcds = 8;

struct Products {
  const int8_t *q;
  const uint8_t *scale;
  uint32_t rows, din, dout, nb;
  uint64_t dy_ld;
  const int32_t *offsets;
  uint32_t experts, kc;
  void *dw;
  uint32_t dw_type;
  float *part;  // a partial din x dout per item of an expert with more than one
};

constexpr uint32_t kMaxExperts = 1024;
constexpr uint32_t kFewParts = 4;  // partials of an expert that a join calls few

__device__ __forceinline__ uint32_t offset_at(const Products &p, uint32_t i) {
  const int32_t o = p.offsets[i];
  return o < 0 ? 0u : (uint32_t)o < p.rows ? (uint32_t)o : p.rows;
}

// With more experts than a wave's lanes the block reads all offsets at once, into
// LDS: a wave that walks them would wait for memory every 64.
__device__ __forceinline__ bool stage_offsets(const Products &p, uint32_t *staged) {
  if (p.experts <= 64) return false;
  for (uint32_t i = threadIdx.x; i <= p.experts; i += blockDim.x) staged[i] = offset_at(p, i);
  __syncthreads();
  return true;
}

// The rows of experts e0 .. e0 + 63, one a lane: [*from, *to), ascending and
// within the rows whatever the offsets say.  *end: where the experts before end
// (0 before the first call); staged: the offsets in LDS, or NULL; every lane of a wave
// calls it.
__device__ __forceinline__ void rows_of(const Products &p, const uint32_t *staged, uint32_t e0, uint32_t lane,
                                        uint32_t *end, uint32_t *from, uint32_t *to) {
  if (!p.offsets) {
    *from = 0;
    *to = lane == 0 ? p.rows : 0;
    return;
  }
  auto at = [&](uint32_t i) { return staged ? staged[i] : offset_at(p, i); };
  if (e0 == 0) *end = at(0);
  const uint32_t e = e0 + lane;
  uint32_t s = e < p.experts ? at(e + 1) : 0;
  s = s > *end ? s : *end;
  uint32_t before = __shfl_up(s, 1);
  if (__any(lane && before > s)) {  // not ascending, or past the last expert: the largest so far
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(s, d);
      if ((int)lane >= d) s = o > s ? o : s;
    }
    before = __shfl_up(s, 1);
  }
  *from = lane ? before : *end;
  *to = s;
  *end = __shfl(s, 63);
}

// An item: a stretch of at most kc rows of an expert.  part is its partial's
// index, or -1 where the expert has no other.
struct Item {
  int32_t expert, part;
  uint32_t from, to;
};

// Item i of the grid's.  Items go by expert; every thread of the block calls it.
// staged: LDS for kMaxExperts + 1 offsets, free again afterwards.
__device__ __forceinline__ Item item_of(const Products &p, uint32_t i, Item *shared, uint32_t *staged) {
  if (!stage_offsets(p, staged)) staged = nullptr;
  if (threadIdx.x < 64) {
    if (threadIdx.x == 0) shared->expert = -1;
    uint32_t items = 0, parts = 0, end = 0;  // of the experts before
    for (uint32_t e0 = 0; e0 < p.experts && items <= i; e0 += 64) {
      const uint32_t e = e0 + threadIdx.x;
      uint32_t from, to;
      rows_of(p, staged, e0, threadIdx.x, &end, &from, &to);
      const uint32_t mine = (to - from + p.kc - 1) / p.kc, part = mine > 1 ? mine : 0;
      uint32_t si = mine, sp = part;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t a = __shfl_up(si, d), b = __shfl_up(sp, d);
        if ((int)threadIdx.x >= d) si += a, sp += b;
      }
      const uint32_t before = items + si - mine;
      if (i >= before && i < before + mine) {
        const uint32_t c = i - before;
        shared->expert = (int32_t)e;
        shared->part = mine > 1 ? (int32_t)(parts + sp - part + c) : -1;
        shared->from = from + c * p.kc;
        shared->to = from + (c + 1) * p.kc < to ? from + (c + 1) * p.kc : to;
      }
      items += __shfl(si, 63);
      parts += __shfl(sp, 63);
    }
  }
  __syncthreads();
  // the same for every lane: held in scalar registers
  Item it;
  it.expert = __builtin_amdgcn_readfirstlane(shared->expert);
  it.part = __builtin_amdgcn_readfirstlane(shared->part);
  it.from = __builtin_amdgcn_readfirstlane(shared->from);
  it.to = __builtin_amdgcn_readfirstlane(shared->to);
  return it;
}

__device__ __forceinline__ void store_dw(void *dw, uint32_t type, uint64_t at, float v) {
  if (type == LSMGNN_F32)
    static_cast<float *>(dw)[at] = v;
  else if (type == LSMGNN_F16)
    static_cast<_Float16 *>(dw)[at] = (_Float16)v;
  else
    static_cast<__bf16 *>(dw)[at] = (__bf16)v;
}

typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef float F16v __attribute__((ext_vector_type(16)));

// The bfloat16 values whose sum is a value of T: leading bits cut off, not rounded
// (nothing overflows), and an infinity is the first part alone.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 2;
template <>
constexpr int kParts<__bf16> = 1;

template <typename T, int kM, int kN, int kWavesM, int kWavesN>
struct Tile {
  static constexpr int kThreads = 64 * kWavesM * kWavesN;
  static constexpr int kP = kParts<T>;
  // rows per step: two steps' pieces of both operands in 64 KiB of LDS.  There is more
  // of it, but 64 rows of the 256 tile take more registers than there are: 1024 x 256
  // of 203003 rows bf16 150 us, 298 so
  static constexpr int kK = (kM + kP * kN) * 64 * 2 * 2 <= 65536 ? 64 : 32;
  static constexpr int kPieces = kK / 8;       // pieces of a column in a step
  static constexpr int kCols = 16 / kPieces;   // columns per line of LDS
  static constexpr int kFragM = kM / kWavesM / 32, kFragN = kN / kWavesN / 32;
  // what the threads stage: 4 columns x 8 rows of x, 2 columns x 8 rows of dy
  static constexpr int kAllX = kM / 4 * kPieces, kAllY = kN / 2 * kPieces;
  static constexpr int kUnitsX = (kAllX + kThreads - 1) / kThreads, kUnitsY = (kAllY + kThreads - 1) / kThreads;
  static constexpr int kBytesX = kM * kK * 2, kBytesY = kN * kK * 2, kStep = kBytesX + kP * kBytesY;
  static __device__ __forceinline__ uint32_t at(uint32_t col, uint32_t piece) {
    const uint32_t line = col / kCols;
    return line * 256 + ((((col % kCols) * kPieces + piece) ^ line) & 15) * 16;
  }
};

// Two neighbouring values of dy, kept as they are loaded: taking them apart waits
// for the load.
template <int kBytes>
struct Raw;
template <>
struct Raw<2> {
  uint32_t both;
  __device__ __forceinline__ uint32_t bits(int c) const { return c ? both >> 16 : both & 0xffffu; }
  __device__ __forceinline__ void set(uint32_t a, uint32_t b) { both = a | b << 16; }
};
template <>
struct Raw<4> {
  uint32_t first, second;
  __device__ __forceinline__ uint32_t bits(int c) const { return c ? second : first; }
  __device__ __forceinline__ void set(uint32_t a, uint32_t b) { first = a, second = b; }
};

// The bits of a value, and the value of bits.
template <typename T>
__device__ __forceinline__ uint32_t bits_of(T v) {
  typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type b;
  __builtin_memcpy(&b, &v, sizeof(T));
  return b;
}
template <typename T>
__device__ __forceinline__ T value_of(uint32_t bits) {
  T v;
  __builtin_memcpy(&v, &bits, sizeof(T));
  return v;
}

// Memory that a wave reads with 32-bit offsets, and as zeros past `bytes`.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00027000);
}

__device__ __forceinline__ void load_pair(__amdgpu_buffer_rsrc_t b, uint32_t at, Raw<2> *v) {
  v->both = __builtin_amdgcn_raw_buffer_load_b32(b, at, 0, 0);
}
__device__ __forceinline__ void load_pair(__amdgpu_buffer_rsrc_t b, uint32_t at, Raw<4> *v) {
  const auto r = __builtin_amdgcn_raw_buffer_load_b64(b, at, 0, 0);
  v->first = r[0];
  v->second = r[1];
}

// kAny: shapes that the others refuse (see lsmgnn_weight_grad8): loaded value by value,
// with offsets of 64 bits.
template <typename T, int kM, int kN, int kWavesM, int kWavesN, bool kAny>
__global__ __launch_bounds__(64 * kWavesM *kWavesN) void k_weight_grad(Products p, const T *dy, uint32_t tiles,
                                                                         uint32_t tiles_n) {
  typedef Tile<T, kM, kN, kWavesM, kWavesN> G;
  __shared__ Item shared;
  __shared__ __align__(256) uint8_t lds[2][G::kStep];
  static_assert(sizeof(lds) >= (kMaxExperts + 1) * 4, "the offsets fit");
  // Blocks go round the 8 XCDs in turn: all tiles of an item to one of them, one
  // after the other, so that its rows are read into one L2.
  const uint32_t turn = blockIdx.x / kXcds, tile = turn % tiles;
  const Item it = item_of(p, turn / tiles * kXcds + blockIdx.x % kXcds, &shared,
                          reinterpret_cast<uint32_t *>(&lds[0][0]));
  if (it.expert < 0) return;
  const uint32_t m0 = tile / tiles_n * kM, n0 = tile % tiles_n * kN;
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t wm = wave / kWavesN * (kM / kWavesM), wn = wave % kWavesN * (kN / kWavesN);

  // Loads of a step are all in flight together and none is looked at before the next
  // step: a row past the item's end reads as zeros by the buffer's bounds, and a
  // unit that crosses the operand's last column loads the last ones there are, to
  // be shifted into place when it is staged.
  uint32_t xr[G::kUnitsX][8], sr[G::kUnitsX][8];
  Raw<sizeof(T)> yr[G::kUnitsY][8];
  uint32_t xo[G::kUnitsX], so[G::kUnitsX], yo[G::kUnitsY];  // columns, and offsets in bytes at a step's first row
#pragma unroll
  for (int u = 0; u < G::kUnitsX; ++u) {
    const uint32_t unit = u * G::kThreads + threadIdx.x, m = m0 + unit % (kM / 4) * 4, k = unit / (kM / 4) * 8;
    xo[u] = k * p.din + (m + 4 <= p.din ? m : p.din > 4 ? p.din - 4 : 0);
    so[u] = k * p.nb + (m < p.din ? m / kPack : p.nb - 1);
  }
#pragma unroll
  for (int u = 0; u < G::kUnitsY; ++u) {
    const uint32_t unit = u * G::kThreads + threadIdx.x, n = n0 + unit % (kN / 2) * 2, k = unit / (kN / 2) * 8;
    yo[u] = (k * (uint32_t)p.dy_ld + (n + 2 <= p.dout ? n : p.dout > 2 ? p.dout - 2 : 0)) * (uint32_t)sizeof(T);
  }
  auto load = [&](uint32_t k0) __attribute__((always_inline)) {
    const uint32_t rest = it.to > k0 ? it.to - k0 : 0, left = rest < (uint32_t)G::kK ? rest : (uint32_t)G::kK;
    const auto xb = buffer_of(p.q + (uint64_t)k0 * p.din, left * p.din);
    const auto sb = buffer_of(p.scale + (uint64_t)k0 * p.nb, left * p.nb);
    const uint32_t y_elems = left ? (left - 1) * (uint32_t)p.dy_ld + p.dout : 0;
    const auto yb = buffer_of(dy + (uint64_t)k0 * p.dy_ld, y_elems * (uint32_t)sizeof(T));
#pragma unroll
    for (int u = 0; u < G::kUnitsX; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xr[u][i] = __builtin_amdgcn_raw_buffer_load_b32(xb, xo[u] + i * p.din, 0, 0);
        sr[u][i] = __builtin_amdgcn_raw_buffer_load_b8(sb, so[u] + i * p.nb, 0, 0);
      }
#pragma unroll
    for (int u = 0; u < G::kUnitsY; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) load_pair(yb, yo[u] + i * (uint32_t)(p.dy_ld * sizeof(T)), &yr[u][i]);
  };
  // The same for any shape, value by value.
  auto load_any = [&](uint32_t k0) __attribute__((always_inline)) {
    for (int u = 0; u < G::kUnitsX; ++u) {
      const uint32_t unit = u * G::kThreads + threadIdx.x, m = m0 + unit % (kM / 4) * 4, k = k0 + unit / (kM / 4) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xr[u][i] = sr[u][i] = 0;
        if (k + i < it.to && m < p.din) {
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e)
            if (m + e < p.din) xr[u][i] |= (uint32_t)(uint8_t)p.q[(uint64_t)(k + i) * p.din + m + e] << (8 * e);
          sr[u][i] = p.scale[(uint64_t)(k + i) * p.nb + m / kPack];
        }
      }
    }
    for (int u = 0; u < G::kUnitsY; ++u) {
      const uint32_t unit = u * G::kThreads + threadIdx.x, n = n0 + unit % (kN / 2) * 2, k = k0 + unit / (kN / 2) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t v[2];
#pragma unroll
        for (uint32_t c = 0; c < 2; ++c)
          v[c] = k + i < it.to && n + c < p.dout ? bits_of(dy[(uint64_t)(k + i) * p.dy_ld + n + c]) : 0;
        yr[u][i].set(v[0], v[1]);
      }
    }
  };
  auto load_step = [&](uint32_t k0) __attribute__((always_inline)) {
    if (kAny)
      load_any(k0);
    else
      load(k0);
  };
  auto stage = [&](uint8_t *to) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < G::kUnitsX; ++u) {
      const uint32_t unit = u * G::kThreads + threadIdx.x;
      const uint32_t col = unit % (kM / 4) * 4, piece = unit / (kM / 4);
      if (G::kAllX % G::kThreads && unit >= G::kAllX) break;
      if (!kAny && m0 + kM > p.din) {  // the tile with the last columns
        const uint32_t m = m0 + col, shift = m + 4 <= p.din ? 0 : (m - (p.din - 4)) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) xr[u][i] = shift < 32 ? xr[u][i] >> shift : 0;
      }
      float s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = __uint_as_float(sr[u][i] << 23);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        __bf16 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)((float)(int8_t)(xr[u][i] >> (8 * c)) * s[i]);
        __builtin_memcpy(to + G::at(col + c, piece), o, 16);
      }
    }
#pragma unroll
    for (int u = 0; u < G::kUnitsY; ++u) {
      const uint32_t unit = u * G::kThreads + threadIdx.x;
      const uint32_t col = unit % (kN / 2) * 2, piece = unit / (kN / 2);
      if (G::kAllY % G::kThreads && unit >= G::kAllY) break;
      if (!kAny && n0 + kN > p.dout)
#pragma unroll
        for (int i = 0; i < 8; ++i) yr[u][i].set(yr[u][i].bits(n0 + col + 2 > p.dout), yr[u][i].bits(1));
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint8_t *at = to + G::kBytesX + G::at(col + c, piece);
        if (G::kP == 1) {
          uint16_t o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = (uint16_t)yr[u][i].bits(c);
          __builtin_memcpy(at, o, 16);
        } else {
          float rest[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) rest[i] = (float)value_of<T>(yr[u][i].bits(c));
#pragma unroll
          for (int part = 0; part < G::kP; ++part) {
            uint16_t o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t lead = __float_as_uint(rest[i]) & 0xffff0000u;
              o[i] = (uint16_t)(lead >> 16);
              // an infinity is all in the first part; later rests are finite or NaN
              const bool all = part == 0 && fabsf(rest[i]) == __builtin_inff();
              rest[i] = all ? 0.0f : rest[i] - __uint_as_float(lead);
            }
            __builtin_memcpy(at + part * G::kBytesY, o, 16);
          }
        }
      }
    }
  };

  F16v acc[G::kFragM][G::kFragN];
#pragma unroll
  for (int a = 0; a < G::kFragM; ++a)
#pragma unroll
    for (int b = 0; b < G::kFragN; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;

  // A step's operands are staged while the matrix units work on the step before,
  // from loads issued a step earlier still; past the last step both are of zeros.
  const uint32_t steps = (it.to - it.from + G::kK - 1) / G::kK;
  constexpr int kSteps = G::kK / 16;
  load_step(it.from);
  stage(lds[0]);
  load_step(it.from + G::kK);
  __syncthreads();
  for (uint32_t s = 0; s < steps; ++s) {
    const uint8_t *now = lds[s & 1];
    Bf8 x[kSteps][G::kFragM], y[kSteps][G::kP][G::kFragN];
    auto read = [&](int k) __attribute__((always_inline)) {
      const uint32_t piece = k * 2 + (lane >> 5);
#pragma unroll
      for (int a = 0; a < G::kFragM; ++a)
        __builtin_memcpy(&x[k][a], now + G::at(wm + a * 32 + (lane & 31), piece), 16);
#pragma unroll
      for (int part = 0; part < G::kP; ++part)
#pragma unroll
        for (int b = 0; b < G::kFragN; ++b)
          __builtin_memcpy(&y[k][part][b],
                           now + G::kBytesX + part * G::kBytesY + G::at(wn + b * 32 + (lane & 31), piece), 16);
    };
    // several parts: their fragments take the registers that staging needs
    if (G::kP == 1) read(0);
    stage(lds[(s + 1) & 1]);
    load_step(it.from + (s + 2) * G::kK);
    if (G::kP > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      if (k || G::kP > 1) read(k);
#pragma unroll
      for (int part = 0; part < G::kP; ++part)
#pragma unroll
        for (int a = 0; a < G::kFragM; ++a)
#pragma unroll
          for (int b = 0; b < G::kFragN; ++b)
            acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[k][a], y[k][part][b], acc[a][b], 0, 0, 0);
    }
    // one matrix instruction, then what of the staging and the loads fits beside it
    if constexpr (G::kP == 1) {
#pragma unroll
      for (int i = 0; i < kSteps * G::kFragM * G::kFragN; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);    // matrix
        __builtin_amdgcn_sched_group_barrier(0x2, 10, 0);   // vector
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);  // LDS writes
        __builtin_amdgcn_sched_group_barrier(0x20, 2, 0);   // loads
      }
    }
    __syncthreads();
  }

  const uint64_t size = (uint64_t)p.din * p.dout;
#pragma unroll
  for (int a = 0; a < G::kFragM; ++a)
#pragma unroll
    for (int b = 0; b < G::kFragN; ++b) {
      const uint32_t n = n0 + wn + b * 32 + (lane & 31);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t m = m0 + wm + a * 32 + (i & 3) + 8 * (i >> 2) + 4 * (lane >> 5);
        if (m >= p.din || n >= p.dout) continue;
        const uint64_t at = (uint64_t)m * p.dout + n;
        if (it.part >= 0)
          p.part[(uint64_t)it.part * size + at] = acc[a][b][i];
        else
          store_dw(p.dw, p.dw_type, (uint64_t)it.expert * size + at, acc[a][b][i]);
      }
    }
}

// Units first, first + stride, ... of those that a join's list has: kElems elements a
// thread, kAhead partials of each in flight.
template <uint32_t kElems, uint32_t kAhead>
__device__ __forceinline__ void join_units(const Products &p, uint32_t listed, const uint32_t *expert,
                                           const uint32_t *items, const uint32_t *first) {
  const uint64_t size = (uint64_t)p.din * p.dout;
  const uint32_t units = (uint32_t)((size + kBlock * kElems - 1) / (kBlock * kElems)), all = listed * units;
  for (uint32_t unit = blockIdx.x; unit < all; unit += gridDim.x) {
    const uint32_t slot = unit / units, n = items[slot];
    const uint64_t i = (uint64_t)(unit - slot * units) * kBlock * kElems + threadIdx.x;
    const float *part = p.part + first[slot] * size;
    float sum[kElems] = {};
    for (uint32_t j = 0; j < n; j += kAhead) {
      float v[kAhead][kElems];
#pragma unroll
      for (uint32_t a = 0; a < kAhead; ++a)
#pragma unroll
        for (uint32_t e = 0; e < kElems; ++e)
          v[a][e] = j + a < n && i + e * kBlock < size ? part[(j + a) * size + i + e * kBlock] : 0.0f;
#pragma unroll
      for (uint32_t a = 0; a < kAhead; ++a)
#pragma unroll
        for (uint32_t e = 0; e < kElems; ++e) sum[e] += v[a][e];
    }
#pragma unroll
    for (uint32_t e = 0; e < kElems; ++e)
      if (i + e * kBlock < size) store_dw(p.dw, p.dw_type, expert[slot] * size + i + e * kBlock, sum[e]);
  }
}

// Add experts' partials; zeros for experts without rows.  Each block lists the
// experts that are either, and the blocks share out their elements, kBlock a unit:
// with 1024 experts of one item each, blocks of their own per expert take 2266 us to
// find that there is nothing to do, these 5.  64 partials of 1024 x 256: 13 us, 5 TB/s.
__global__ __launch_bounds__(kBlock) void k_weight_grad_join(Products p) {
  __shared__ uint32_t staged_offsets[kMaxExperts + 1];
  __shared__ uint32_t expert[kMaxExperts], items[kMaxExperts], first[kMaxExperts], listed, many;
  const uint32_t *staged = stage_offsets(p, staged_offsets) ? staged_offsets : nullptr;
  if (threadIdx.x < 64) {
    uint32_t parts = 0, n = 0, end = 0;
    bool long_one = false;
    for (uint32_t e0 = 0; e0 < p.experts; e0 += 64) {
      const uint32_t e = e0 + threadIdx.x;
      uint32_t from, to;
      rows_of(p, staged, e0, threadIdx.x, &end, &from, &to);
      const uint32_t mine = (to - from + p.kc - 1) / p.kc;
      const bool list = e < p.experts && mine != 1;
      const uint64_t set = __ballot(list);
      uint32_t part = mine > 1 ? mine : 0;
      if (__any(part)) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const uint32_t o = __shfl_up(part, d);
          if (threadIdx.x >= (uint32_t)d) part += o;
        }
      }
      if (list) {
        const uint32_t at = n + (uint32_t)__popcll(set & ((1ull << threadIdx.x) - 1));
        expert[at] = e;
        items[at] = mine;
        first[at] = parts + part - mine;
      }
      long_one |= mine > kFewParts;
      n += (uint32_t)__popcll(set);
      parts += __shfl(part, 63);
    }
    const bool any_long = __any(long_one);
    if (threadIdx.x == 0) listed = n, many = any_long;
  }
  __syncthreads();
  // eight loads in flight a thread; where no expert has many partials, of four
  // elements (100000 rows of 1024 x 256 bf16 by 32 experts: 110 -> 90 us in all)
  if (many)
    join_units<1, 8>(p, listed, expert, items, first);
  else
    join_units<4, 2>(p, listed, expert, items, first);
}

// How a weight gradient is cut.
struct Shape {
  uint32_t m, n;          // the tile
  uint32_t tiles_m, tiles_n;
  uint32_t kc;            // rows per item
};

Shape shape_of(uint64_t rows, uint64_t din, uint64_t dout) {
  Shape s{};
  auto tiles_of = [&](uint32_t size) { return blocks_for(din, size) * blocks_for(dout, size); };
  const uint64_t t64 = tiles_of(64), t128 = tiles_of(128), t256 = tiles_of(256);
  // Few small tiles: the small one (192 x 192, 100003 rows: 30 us bf16, 62 f32;
  // 128: 37 and 68; 256: 42 and 64).  Else the large one, which reads LDS least a
  // product, unless its padding costs more (384 x 384: 71 against 54 us with 128;
  // 320 x 256: 47 against 60) or an item would be a few steps only (257 x 129,
  // 40009 rows f32: 61 against 50).
  s.m = t64 <= 9 ? 64 : t256 * 4 * 100 <= t128 * 145 && rows * t256 >= 512 * 256 ? 256 : 128;
  s.n = s.m;
  s.tiles_m = (uint32_t)blocks_for(din, s.m);
  s.tiles_n = (uint32_t)blocks_for(dout, s.n);
  // as many items as fill the chip: one block of the large tile a CU, two of the
  // others; more items would only add partial sums
  const uint64_t tiles = (uint64_t)s.tiles_m * s.tiles_n, slots = s.m == 256 ? 256 : 512;
  const uint64_t items = slots / tiles ? slots / tiles : 1;
  uint64_t kc = (rows + items - 1) / items;
  kc = (kc + 63) / 64 * 64;
  s.kc = (uint32_t)(kc < 256 ? 256 : kc);
  return s;
}

template <typename T, int kM, int kN, int kWavesM, int kWavesN, bool kAny = false>
void queue_products(const Products &p, const Shape &s, const void *dy, uint32_t items, hipStream_t st) {
  const uint32_t tiles = s.tiles_m * s.tiles_n, rounds = (items + kXcds - 1) / kXcds;
  hipLaunchKernelGGL((k_weight_grad<T, kM, kN, kWavesM, kWavesN, kAny>), dim3(tiles * rounds * kXcds),
                     dim3(64 * kWavesM * kWavesN), 0, st, p, static_cast<const T *>(dy), tiles, s.tiles_n);
}

// Partials: only experts with at least two items have any, and those have fewer
// than two for each kc rows.
uint64_t parts_of(uint64_t rows, uint32_t kc) { return rows > kc ? 2 * (rows / kc) + 1 : 0; }

bool kept_ok(const int8_t *q, const uint8_t *scale, uint64_t rows, uint64_t dim) {
  return dim >= 1 && dim <= kMaxDim && rows <= kMaxRows && rows * dim <= kMaxElems && (rows == 0 || (q && scale));
}

lsmgnn_status done() { return hipGetLastError() == hipSuccess ? LSMGNN_OK : LSMGNN_E_DEVICE; }

template <typename F>
void with_act(uint32_t name, uint32_t gated, F f) {
  typedef std::integral_constant<uint32_t, LSMGNN_SILU> Silu;
  typedef std::integral_constant<uint32_t, LSMGNN_GELU> Gelu;
  if (name == LSMGNN_SILU)
    gated ? f(Silu{}, std::true_type{}) : f(Silu{}, std::false_type{});
  else
    gated ? f(Gelu{}, std::true_type{}) : f(Gelu{}, std::false_type{});
}

}  // namespace lsm_packed

extern "C" {

uint64_t lsmgnn_pack_blocks(uint64_t dim) { return (dim + LSMGNN_PACK_BLOCK - 1) / LSMGNN_PACK_BLOCK; }

lsmgnn_status lsmgnn_pack8(const void *x, uint64_t rows, uint64_t dim, uint64_t x_ld, uint32_t type, int8_t *q,
                           uint8_t *scale, void *stream) {
  using namespace lsm_packed;
  if (!matrix_ok(x, rows, dim, x_ld, type) || !kept_ok(q, scale, rows, dim)) return LSMGNN_E_INVAL;
  if (rows == 0) return LSMGNN_OK;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    cuts_of(rows, dim, [&](const Cut &c, uint64_t r) {
      hipLaunchKernelGGL((k_pack<T>), dim3(blocks_of(c)), dim3(kBlock), 0, static_cast<hipStream_t>(stream), c,
                         static_cast<const T *>(x) + r * x_ld, x_ld, q + r * dim, scale + r * c.nb);
    });
  });
  return done();
}

lsmgnn_status lsmgnn_unpack8(const int8_t *q, const uint8_t *scale, uint64_t rows, uint64_t dim, void *out,
                             uint64_t out_ld, uint32_t type, void *stream) {
  using namespace lsm_packed;
  if (!matrix_ok(out, rows, dim, out_ld, type) || !kept_ok(q, scale, rows, dim)) return LSMGNN_E_INVAL;
  if (rows == 0) return LSMGNN_OK;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    cuts_of(rows, dim, [&](const Cut &c, uint64_t r) {
      hipLaunchKernelGGL((k_unpack<T>), dim3(blocks_of(c)), dim3(kBlock), 0, static_cast<hipStream_t>(stream), c,
                         q + r * dim, scale + r * c.nb, static_cast<T *>(out) + r * out_ld, out_ld);
    });
  });
  return done();
}

lsmgnn_status lsmgnn_act8(const void *x, uint64_t rows, uint64_t dim, uint64_t x_ld, uint32_t type, uint32_t act,
                          uint32_t gated, void *y, uint64_t y_ld, int8_t *q, uint8_t *scale, void *stream) {
  using namespace lsm_packed;
  if (act > LSMGNN_GELU || gated > 1 || dim > kMaxDim || !matrix_ok(x, rows, dim * (1 + gated), x_ld, type) ||
      !matrix_ok(y, rows, dim, y_ld, type) || !kept_ok(q, scale, rows * (1 + gated), dim))
    return LSMGNN_E_INVAL;
  if (rows == 0) return LSMGNN_OK;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  const uint64_t kept = 1 + gated;  // kept rows of a row
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    with_act(act, gated, [&](auto f, auto g) {
      cuts_of(rows, dim, [&](const Cut &c, uint64_t r) {
        hipLaunchKernelGGL((k_act<T, decltype(f)::value, decltype(g)::value>), dim3(blocks_of(c)), dim3(kBlock),
                           0, static_cast<hipStream_t>(stream), c, static_cast<const T *>(x) + r * x_ld,
                           x_ld, static_cast<T *>(y) + r * y_ld, y_ld, q + r * kept * dim, scale + r * kept * c.nb);
      });
    });
  });
  return done();
}

lsmgnn_status lsmgnn_act8_grad(const void *dy, uint64_t rows, uint64_t dim, uint64_t dy_ld, uint32_t type,
                               const int8_t *q, const uint8_t *scale, uint32_t act, uint32_t gated, void *dx,
                               uint64_t dx_ld, void *stream) {
  using namespace lsm_packed;
  if (act > LSMGNN_GELU || gated > 1 || dim > kMaxDim || !matrix_ok(dy, rows, dim, dy_ld, type) ||
      !matrix_ok(dx, rows, dim * (1 + gated), dx_ld, type) || !kept_ok(q, scale, rows * (1 + gated), dim))
    return LSMGNN_E_INVAL;
  if (rows == 0) return LSMGNN_OK;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  const uint64_t kept = 1 + gated;  // kept rows of a row
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    with_act(act, gated, [&](auto f, auto g) {
      cuts_of(rows, dim, [&](const Cut &c, uint64_t r) {
        hipLaunchKernelGGL((k_act_grad<T, decltype(f)::value, decltype(g)::value>), dim3(blocks_of(c)), dim3(kBlock),
                           0, static_cast<hipStream_t>(stream), c, static_cast<const T *>(dy) + r * dy_ld,
                           dy_ld, q + r * kept * dim, scale + r * kept * c.nb, static_cast<T *>(dx) + r * dx_ld, dx_ld);
      });
    });
  });
  return done();
}

uint64_t lsmgnn_weight_grad8_work_bytes(uint64_t rows, uint64_t din, uint64_t dout, uint32_t num_experts) {
  using namespace lsm_packed;
  (void)num_experts;  // however many there are, each item is of one of them
  if (din == 0 || dout == 0 || din > kMaxDim || dout > kMaxDim || rows > kMaxRows) return 0;
  return parts_of(rows, shape_of(rows, din, dout).kc) * din * dout * 4;
}

lsmgnn_status lsmgnn_weight_grad8(const int8_t *q, const uint8_t *scale, uint64_t rows, uint64_t din, const void *dy,
                                  uint64_t dout, uint64_t dy_ld, uint32_t dy_type, const int32_t *offsets,
                                  uint32_t num_experts, void *dw, uint32_t dw_type, void *work, uint64_t work_bytes,
                                  void *stream) {
  using namespace lsm_packed;
  const uint64_t need = lsmgnn_weight_grad8_work_bytes(rows, din, dout, num_experts);
  if (!kept_ok(q, scale, rows, din) || !matrix_ok(dy, rows, dout, dy_ld, dy_type) || num_experts < 1 ||
      num_experts > kMaxExperts || (!offsets && num_experts != 1) ||
      !matrix_ok(dw, num_experts * din, dout, dout, dw_type) ||
      (need && (!work || reinterpret_cast<uintptr_t>(work) % 256 || work_bytes < need)))
    return LSMGNN_E_INVAL;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  Products p{};
  p.q = q;
  p.scale = scale;
  p.rows = (uint32_t)rows;
  p.din = (uint32_t)din;
  p.dout = (uint32_t)dout;
  p.nb = (uint32_t)lsmgnn_pack_blocks(din);
  p.dy_ld = rows > 1 ? dy_ld : dout;  // the rows past the last are told by it
  p.offsets = offsets;
  p.experts = num_experts;
  Shape s = shape_of(rows, din, dout);
  // fewer than 4 columns of x or 2 of dy, or 64 rows of dy beyond 32-bit offsets
  const bool any = din < 4 || dout < 2 || p.dy_ld > (1u << 23);
  if (any) {
    s.m = s.n = 64;
    s.tiles_m = (uint32_t)blocks_for(din, 64);
    s.tiles_n = (uint32_t)blocks_for(dout, 64);
  }
  p.kc = s.kc;
  p.dw = dw;
  p.dw_type = dw_type;
  p.part = static_cast<float *>(work);
  const uint32_t items = (uint32_t)(rows / p.kc + num_experts);
  if (rows)
    with_type(dy_type, [&](auto tag) {
      typedef typename decltype(tag)::T T;
      if (any)
        queue_products<T, 64, 64, 2, 2, true>(p, s, dy, items, st);
      else if (s.m == 256)
        queue_products<T, 256, 256, 2, 4>(p, s, dy, items, st);
      else if (s.m == 128)
        queue_products<T, 128, 128, 2, 2>(p, s, dy, items, st);
      else
        queue_products<T, 64, 64, 2, 2>(p, s, dy, items, st);
    });
  // at most 2^25 units by matrix_ok's limit of elements and that of experts; the
  // blocks that are resident at once
  const uint32_t units = (uint32_t)blocks_for(din * dout, kBlock), most = units * num_experts;
  hipLaunchKernelGGL(k_weight_grad_join, dim3(most < 2048 ? most : 2048), dim3(kBlock), 0, st, p);
  return done();
}

}  // extern "C"
