// Rows sorted by expert (a node type, or a router's choice), for products with one
// matrix per expert, and the way back with weights; forward and backward.
//
// The plan is one stable counting pass over the n k choices (sort.h).  All row
// movement is by token: a token's row is read once and written to its k places,
// or its k rows are read and added in registers, in the order of the choices, so
// nothing is added by an atomic.  Lanes take consecutive 16-byte pieces of the
// tokens' rows, whatever the width.  Unused sorted rows (an expert's rounding, the
// end of the buffer) are written with zeros by blocks that look for -1 in
// `source`, 256 rows a block.  Bound by memory, 50021 tokens of 1024 bf16 with two
// choices of 64: the plan 17 us (three launches that wait on each other), the sorted
// rows 68 us (4.5 TB/s, whole rows written in scattered order), the way back 54 us
// (5.7), its gradients 100 us (5.1).  One token: 2 us a launch.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "lsmgnn.h"
#include "rows.h"
#include "sort.h"

namespace lsm_route {

using namespace lsm_rows;

constexpr uint32_t kBad = 0x80000000u;  // a choice that names no expert

struct FromExperts {
  typedef uint32_t Item;
  const int64_t *experts;
  uint32_t num;
  __device__ __forceinline__ Item load(uint32_t i) const {
    const int64_t e = experts[i];
    return e < 0 ? num : e >= (int64_t)num ? num | kBad : (uint32_t)e;
  }
  __device__ __forceinline__ uint32_t digit(Item e) const { return e & ~kBad; }
};

struct ToPlan {
  int32_t *offsets, *slot, *source;
  uint32_t num;
  uint32_t rows;
  uint64_t *status;
  __device__ __forceinline__ void put(uint32_t at, uint32_t e, uint32_t i) const {
    const bool kept = e < num;
    slot[i] = kept ? (int32_t)at : -1;
    if (kept) source[at] = (int32_t)i;
    if ((e & kBad) && status) *status = LSMGNN_E_RANGE;
  }
  __device__ __forceinline__ void start(uint32_t d, uint32_t at) const { offsets[d] = (int32_t)at; }
  __device__ __forceinline__ void unused(uint32_t d, uint32_t from, uint32_t to) const {
    if (d < num)
      for (uint32_t r = from; r < to; ++r) source[r] = -1;
  }
  __device__ __forceinline__ void after(uint32_t from) const {
    for (uint64_t r = from + (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; r < rows;
         r += (uint64_t)gridDim.x * blockDim.x)
      source[r] = -1;
  }
};

// No choices: every expert is empty, every row unused.
__global__ __launch_bounds__(kBlock) void k_no_choices(ToPlan p) {
  for (uint32_t e = threadIdx.x; e <= p.num; e += kBlock) p.offsets[e] = 0;
  for (uint32_t r = threadIdx.x; r < p.rows; r += kBlock) p.source[r] = -1;
}

// A token's place in the pieces of all tokens' rows (see rows.h).
struct Pieces {
  uint64_t n;        // tokens
  uint32_t dim, np;  // elements and pieces of a row
  uint64_t div64, div32;
};

template <int kN>
__device__ __forceinline__ bool piece_of(const Pieces &p, uint64_t base, uint32_t x, uint64_t *token, uint32_t *at) {
  const uint64_t t0 = p.div64 ? __umul64hi(base, p.div64) : base;
  x += (uint32_t)(base - t0 * p.np);
  const uint32_t r = (uint32_t)((x * p.div32) >> 32);
  *token = t0 + r;
  *at = (x - r * p.np) * kN;
  if (p.dim >= (uint32_t)kN && *at + kN > p.dim) *at = p.dim - kN;
  return *token < p.n;
}

// Elements of the piece at hand: kN, or the row's width where that is less.
template <int kN, typename T>
__device__ __forceinline__ void load_piece(const T *p, uint32_t dim, T (&v)[kN]) {
  if (dim >= (uint32_t)kN) {
    load_row_once(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] = e < (int)dim ? p[e] : (T)0.0f;
  }
}

template <bool kOnce, int kN, typename T>
__device__ __forceinline__ void store_piece(T *p, uint32_t dim, const T (&v)[kN]) {
  if (dim >= (uint32_t)kN) {
    store_row_as<kOnce>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < kN; ++e)
      if (e < (int)dim) p[e] = v[e];
  }
}

// Zeros in the unused ones of the block's kBlock sorted rows: a wave looks at 64
// and writes those that it finds, its lanes side by side.
template <bool kOnce, typename T>
__device__ __forceinline__ void zero_unused(uint64_t block, const int32_t *source, uint64_t rows, uint32_t dim, T *out,
                                            uint64_t ld) {
  constexpr int kN = kPiece<T>;
  const uint64_t r0 = block * kBlock + (threadIdx.x & ~63u), mine = r0 + (threadIdx.x & 63);
  uint64_t left = __ballot(mine < rows && source[mine < rows ? mine : 0] < 0);
  T zero[kN];
#pragma unroll
  for (int e = 0; e < kN; ++e) zero[e] = (T)0.0f;
  while (left) {
    const uint64_t r = r0 + __builtin_ctzll(left);
    left &= left - 1;
    for (uint32_t c = (threadIdx.x & 63) * kN; c < dim; c += 64 * kN)
      store_piece<kOnce, kN>(out + r * ld + (dim >= (uint32_t)kN && c + kN > dim ? dim - kN : c), dim, zero);
  }
}

constexpr int kUnroll = 2;  // pieces per thread

// kOnce: the sorted rows are written past the caches (see on_lines).
template <typename T, bool kOnce>
__global__ __launch_bounds__(kBlock) void k_route_rows(Pieces p, const T *x, uint64_t xld, const int32_t *slot,
                                                       uint32_t k, uint64_t move_blocks, const int32_t *source,
                                                       uint64_t rows, T *out, uint64_t old_) {
  constexpr int kN = kPiece<T>;
  if (blockIdx.x >= move_blocks) {
    zero_unused<kOnce>(blockIdx.x - move_blocks, source, rows, p.dim, out, old_);
    return;
  }
  const uint64_t base = (uint64_t)blockIdx.x * (kBlock * kUnroll);
  uint64_t t[kUnroll];
  uint32_t at[kUnroll];
  bool ok[kUnroll];
  T v[kUnroll][kN];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    ok[u] = piece_of<kN>(p, base, u * kBlock + threadIdx.x, &t[u], &at[u]);
    if (ok[u]) load_piece<kN>(x + t[u] * xld + at[u], p.dim, v[u]);
  }
  for (uint32_t j = 0; j < k; ++j)
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (!ok[u]) continue;
      const int32_t r = slot[t[u] * k + j];
      if (r >= 0 && (uint64_t)r < rows) store_piece<kOnce, kN>(out + (uint64_t)r * old_ + at[u], p.dim, v[u]);
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_route_combine(Pieces p, const T *z, uint64_t zld, uint64_t rows,
                                                          const int32_t *slot, const float *weights, uint32_t k, T *y,
                                                          uint64_t yld) {
  constexpr int kN = kPiece<T>;
  constexpr int kTogether = 4;  // choices whose rows are in flight
  uint64_t t;
  uint32_t at;
  if (!piece_of<kN>(p, (uint64_t)blockIdx.x * kBlock, threadIdx.x, &t, &at)) return;
  float acc[kN];
#pragma unroll
  for (int e = 0; e < kN; ++e) acc[e] = 0.0f;
  for (uint32_t j0 = 0; j0 < k; j0 += kTogether) {
    T v[kTogether][kN];
    float w[kTogether];
    bool ok[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int32_t r = j0 + j < k ? slot[t * k + j0 + j] : -1;
      ok[j] = r >= 0 && (uint64_t)r < rows;
      w[j] = ok[j] && weights ? weights[t * k + j0 + j] : 1.0f;
      if (ok[j]) load_piece<kN>(z + (uint64_t)r * zld + at, p.dim, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j)
      if (ok[j])
#pragma unroll
        for (int e = 0; e < kN; ++e) acc[e] = __builtin_fmaf(w[j], (float)v[j][e], acc[e]);
  }
  T o[kN];
#pragma unroll
  for (int e = 0; e < kN; ++e) o[e] = (T)acc[e];
  store_piece<true, kN>(y + t * yld + at, p.dim, o);
}

// dz and dweights: 2^shift lanes per token, each with every 2^shift-th piece.  The
// inner products are added over a lane's pieces, then over the lanes; the piece
// that ends a row and overlaps the one before counts its new elements only.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_route_combine_grad(uint64_t n, uint32_t dim, const T *dy, uint64_t dyld,
                                                               const T *z, uint64_t zld, const int32_t *slot,
                                                               const float *weights, uint32_t k, uint32_t shift,
                                                               uint64_t move_blocks, const int32_t *source,
                                                               uint64_t rows, T *dz, uint64_t dzld, float *dw) {
  constexpr int kN = kPiece<T>;
  if (blockIdx.x >= move_blocks) {
    zero_unused<true>(blockIdx.x - move_blocks, source, rows, dim, dz, dzld);
    return;
  }
  const uint32_t lanes = 1u << shift, lane = threadIdx.x & (lanes - 1);
  const uint64_t t = (uint64_t)blockIdx.x * (kBlock >> shift) + (threadIdx.x >> shift);
  const bool whole = dim >= (uint32_t)kN;
  constexpr int kTogether = 4;  // choices for one look at dy
  for (uint32_t j0 = 0; j0 < k; j0 += kTogether) {
    uint64_t at_row[kTogether];
    float w[kTogether], dot[kTogether];
    bool ok[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int32_t r = t < n && j0 + j < k ? slot[t * k + j0 + j] : -1;
      ok[j] = r >= 0 && (uint64_t)r < rows;
      at_row[j] = ok[j] ? (uint64_t)r : 0;
      w[j] = ok[j] && weights ? weights[t * k + j0 + j] : 1.0f;
      dot[j] = 0.0f;
    }
    for (uint32_t c = lane * kN; t < n && c < dim; c += lanes * kN) {
      const uint32_t at = whole && c + kN > dim ? dim - kN : c, seen = c - at;
      T g[kN], v[kTogether][kN];
      load_piece<kN>(dy + t * dyld + at, dim, g);
#pragma unroll
      for (int j = 0; j < kTogether; ++j)
        if (ok[j] && dw) load_piece<kN>(z + at_row[j] * zld + at, dim, v[j]);
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        if (!ok[j]) continue;
        T o[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) {
          o[e] = (T)(w[j] * (float)g[e]);
          if (dw && e >= (int)seen) dot[j] = __builtin_fmaf((float)v[j][e], (float)g[e], dot[j]);
        }
        store_piece<true, kN>(dz + at_row[j] * dzld + at, dim, o);
      }
    }
    if (dw) {
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        for (uint32_t d = lanes >> 1; d; d >>= 1) dot[j] += __shfl_xor(dot[j], d);
        if (lane == 0 && t < n && j0 + j < k) dw[t * k + j0 + j] = dot[j];
      }
    }
  }
}

Pieces pieces_of(uint64_t n, uint64_t dim, uint32_t piece) {
  Pieces p{};
  p.n = n;
  p.dim = (uint32_t)dim;
  p.np = pieces(dim, piece);
  p.div64 = p.np > 1 ? ~0ull / p.np + 1 : 0;
  p.div32 = divider(p.np);
  return p;
}

constexpr uint32_t kMaxExperts = 1024, kMaxChoices = 64, kMaxAlign = 4096;

bool choices_ok(uint64_t n, uint32_t k) {
  return k >= 1 && k <= kMaxChoices && n <= kMaxRows && n * k <= kMaxRows;
}

}  // namespace lsm_route

extern "C" {

uint64_t lsmgnn_route_max_rows(uint64_t n, uint32_t k, uint32_t num_experts, uint32_t align) {
  return n * k + (uint64_t)num_experts * (align ? align - 1 : 0);
}

uint64_t lsmgnn_route_work_bytes(uint64_t n, uint32_t k, uint32_t num_experts) {
  using namespace lsm_route;
  if (!choices_ok(n, k) || num_experts > kMaxExperts) return 0;
  if (n == 0 || lsm_sort::mode_of((uint32_t)(n * k)) == lsm_sort::kOneTile) return 0;  // one launch, no counts
  return lsm_sort::count_words(n * k, num_experts + 1) * 4;
}

lsmgnn_status lsmgnn_route_plan(const int64_t *experts, uint64_t n, uint32_t k, uint32_t num_experts, uint32_t align,
                                int32_t *offsets, int32_t *slot, int32_t *source, void *work, uint64_t work_bytes,
                                uint64_t *status, void *stream) {
  using namespace lsm_route;
  uint64_t *st_word;
  if (!choices_ok(n, k) || num_experts < 1 || num_experts > kMaxExperts || align < 1 || align > kMaxAlign)
    return LSMGNN_E_INVAL;
  const uint64_t rows = lsmgnn_route_max_rows(n, k, num_experts, align);
  const uint64_t need = lsmgnn_route_work_bytes(n, k, num_experts);
  if (rows > kMaxRows || !offsets || (rows && !source) || (n && (!experts || !slot)) ||
      (need && (!work || reinterpret_cast<uintptr_t>(work) % 256 || work_bytes < need)) ||
      !status_view(status, &st_word))
    return LSMGNN_E_INVAL;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const ToPlan to{offsets, slot, source, num_experts, (uint32_t)rows, st_word};
  if (n) {
    uint32_t bits = 0;
    while (num_experts >> bits) ++bits;
    uint32_t done = 0;
    lsm_sort::queue_pass(FromExperts{experts, num_experts}, to, (uint32_t)(n * k), num_experts + 1, bits, align,
                         static_cast<uint32_t *>(work), lsm_sort::Fill{}, &done, 1, st);
  } else {
    hipLaunchKernelGGL(k_no_choices, dim3(1), dim3(kBlock), 0, st, to);
  }
  return hipGetLastError() == hipSuccess ? LSMGNN_OK : LSMGNN_E_DEVICE;
}

lsmgnn_status lsmgnn_route_rows(const void *x, uint64_t n, uint64_t dim, uint64_t x_ld, uint32_t type,
                                const int32_t *slot, const int32_t *source, uint32_t k, uint64_t rows, void *out,
                                uint64_t out_ld, void *stream) {
  using namespace lsm_route;
  if (!choices_ok(n, k) || !matrix_ok(x, n, dim, x_ld, type) || !matrix_ok(out, rows, dim, out_ld, type) ||
      (n && !slot) || (rows && !source))
    return LSMGNN_E_INVAL;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    const Pieces p = pieces_of(n, dim, kPiece<T>);
    const uint64_t move = blocks_for(n * p.np, kBlock * kUnroll), grid = move + blocks_for(rows, kBlock);
    if (!grid) return;
    if (on_lines(out, out_ld, type))
      hipLaunchKernelGGL((k_route_rows<T, true>), dim3(grid), dim3(kBlock), 0, st, p, static_cast<const T *>(x), x_ld,
                         slot, k, move, source, rows, static_cast<T *>(out), out_ld);
    else
      hipLaunchKernelGGL((k_route_rows<T, false>), dim3(grid), dim3(kBlock), 0, st, p, static_cast<const T *>(x), x_ld,
                         slot, k, move, source, rows, static_cast<T *>(out), out_ld);
  });
  return hipGetLastError() == hipSuccess ? LSMGNN_OK : LSMGNN_E_DEVICE;
}

lsmgnn_status lsmgnn_route_combine(const void *z, uint64_t rows, uint64_t dim, uint64_t z_ld, uint32_t type,
                                   const int32_t *slot, const float *weights, uint64_t n, uint32_t k, void *y,
                                   uint64_t y_ld, void *stream) {
  using namespace lsm_route;
  if (!choices_ok(n, k) || !matrix_ok(z, rows, dim, z_ld, type) || !matrix_ok(y, n, dim, y_ld, type) ||
      (n && !slot))
    return LSMGNN_E_INVAL;
  if (n == 0) return LSMGNN_OK;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    const Pieces p = pieces_of(n, dim, kPiece<T>);
    hipLaunchKernelGGL((k_route_combine<T>), dim3(blocks_for(n * p.np, kBlock)), dim3(kBlock), 0, st, p,
                       static_cast<const T *>(z), z_ld, rows, slot, weights, k, static_cast<T *>(y), y_ld);
  });
  return hipGetLastError() == hipSuccess ? LSMGNN_OK : LSMGNN_E_DEVICE;
}

lsmgnn_status lsmgnn_route_combine_grad(const void *dy, uint64_t n, uint64_t dim, uint64_t dy_ld, uint32_t type,
                                        const void *z, uint64_t z_ld, const int32_t *slot, const int32_t *source,
                                        const float *weights, uint32_t k, uint64_t rows, void *dz, uint64_t dz_ld,
                                        float *dweights, void *stream) {
  using namespace lsm_route;
  if (!choices_ok(n, k) || !matrix_ok(dy, n, dim, dy_ld, type) || !matrix_ok(dz, rows, dim, dz_ld, type) ||
      (n && !slot) || (rows && !source) || (dweights && (!weights || !matrix_ok(z, rows, dim, z_ld, type))))
    return LSMGNN_E_INVAL;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    const uint32_t np = pieces(dim, kPiece<T>);
    uint32_t shift = 0;
    while (shift < 6 && (1u << shift) < np) ++shift;
    auto launch = [&](uint64_t t, uint64_t tokens, bool unused) {
      const uint64_t move = blocks_for(tokens, kBlock >> shift), grid = move + (unused ? blocks_for(rows, kBlock) : 0);
      hipLaunchKernelGGL((k_route_combine_grad<T>), dim3(grid), dim3(kBlock), 0, st, tokens, (uint32_t)dim,
                         static_cast<const T *>(dy) + t * dy_ld, dy_ld, static_cast<const T *>(z), z_ld, slot + t * k,
                         weights ? weights + t * k : nullptr, k, shift, move, source, rows, static_cast<T *>(dz), dz_ld,
                         dweights ? dweights + t * k : nullptr);
    };
    // the unused rows beside the first tokens
    in_launches(n, 1u << shift, [&](uint64_t t, uint64_t tokens) { launch(t, tokens, t == 0); });
    if (n == 0 && rows) launch(0, 0, true);
  });
  return hipGetLastError() == hipSuccess ? LSMGNN_OK : LSMGNN_E_DEVICE;
}

}  // extern "C"
