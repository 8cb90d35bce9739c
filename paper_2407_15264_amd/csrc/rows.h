// What the kernels on typed rows share (trained tables, rows by expert, 8-bit
// activations): element types, pieces of a row, arguments' checks.  Not part of
// the public C ABI (include/lsmgnn.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lsmgnn.h"

namespace lsm_rows {

constexpr int kBlock = 256;
constexpr uint64_t kMaxDim = 65536;             // elements of a row
constexpr uint64_t kMaxRows = (1ull << 31) - 1;  // rows or places that a 32-bit index names
// elements of a matrix: where a row's lanes take a 16-byte piece each and no row has
// spare ones, a launch has fewer than 2^32 lanes, as it must
constexpr uint64_t kMaxElems = 1ull << 33;

template <uint32_t kType>
struct Elem;
template <>
struct Elem<LSMGNN_F32> {
  typedef float T;
};
template <>
struct Elem<LSMGNN_F16> {
  typedef _Float16 T;
};
template <>
struct Elem<LSMGNN_BF16> {
  typedef __bf16 T;
};

inline uint32_t elem_bytes(uint32_t type) { return type == LSMGNN_F32 ? 4 : 2; }

// The type's tag: a kernel's element type chosen by a value (see with_type).
template <uint32_t kType>
struct Tag {
  typedef typename Elem<kType>::T T;
};

// f(Tag) for the element type named `type`, which the caller has checked.
template <typename F>
inline void with_type(uint32_t type, F f) {
  if (type == LSMGNN_F32)
    f(Tag<LSMGNN_F32>{});
  else if (type == LSMGNN_F16)
    f(Tag<LSMGNN_F16>{});
  else
    f(Tag<LSMGNN_BF16>{});
}

inline bool type_ok(uint32_t type) { return type <= LSMGNN_BF16; }

// A matrix argument: rows of `dim` elements whose starts are `ld` apart.
inline bool ld_ok(const void *p, uint64_t rows, uint64_t dim, uint64_t ld, uint32_t type) {
  return type_ok(type) && dim >= 1 && dim <= kMaxDim && (rows <= 1 || ld >= dim) && ld <= (1ull << 32) &&
         (rows == 0 || p) && reinterpret_cast<uintptr_t>(p) % elem_bytes(type) == 0;
}

// The same for a matrix of bounded size.
inline bool matrix_ok(const void *p, uint64_t rows, uint64_t dim, uint64_t ld, uint32_t type) {
  return rows <= kMaxRows && ld_ok(p, rows, dim, ld, type) && rows * dim <= kMaxElems;
}

// The address at which a kernel can write the caller's status words: device
// memory or pinned host memory.  False for anything else (NULL stays NULL).
inline bool status_view(uint64_t *p, uint64_t **out) {
  *out = nullptr;
  if (!p) return true;
  hipPointerAttribute_t a{};
  if (reinterpret_cast<uintptr_t>(p) % 8 || hipPointerGetAttributes(&a, p) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  if (a.type != hipMemoryTypeDevice && a.type != hipMemoryTypeHost && a.type != hipMemoryTypeManaged) return false;
  *out = static_cast<uint64_t *>(a.devicePointer ? a.devicePointer : p);
  return true;
}

// Makes the device of a caller's stream the current one; the NULL stream is the
// current device's already.
struct StreamDevice {
  int prev = -1;
  bool ok = true;
  explicit StreamDevice(void *stream) {
    int dev = -1, now = -1;
    if (!stream) return;
    ok = hipStreamGetDevice(static_cast<hipStream_t>(stream), &dev) == hipSuccess && hipGetDevice(&now) == hipSuccess;
    if (ok && dev != now) {
      ok = hipSetDevice(dev) == hipSuccess;
      if (ok) prev = now;
    }
    if (!ok) (void)hipGetLastError();
  }
  ~StreamDevice() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

// kN elements at p, which may be any address: rows of an odd width start anywhere,
// and the hardware takes vector accesses so.  Whole vectors (a copy of the elements
// would be taken apart by the compiler where another path reads some of them).
typedef uint32_t Piece4 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t Piece2 __attribute__((ext_vector_type(2), aligned(1)));

template <int kBytes>
struct PieceOf {
  typedef Piece4 V;
};
template <>
struct PieceOf<8> {
  typedef Piece2 V;
};

template <int kN, typename T>
__device__ __forceinline__ void load_row(const T *p, T (&v)[kN]) {
  typedef typename PieceOf<sizeof(v)>::V V;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T[kN]) / (sizeof(V))); ++i) {
    const V t = reinterpret_cast<const V *>(p)[i];
    __builtin_memcpy(reinterpret_cast<char *>(v) + sizeof(V) * i, &t, sizeof(V));
  }
}

template <int kN, typename T>
__device__ __forceinline__ void store_row(T *p, const T (&v)[kN]) {
  typedef typename PieceOf<sizeof(v)>::V V;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T[kN]) / (sizeof(V))); ++i) {
    V t;
    __builtin_memcpy(&t, reinterpret_cast<const char *>(v) + sizeof(V) * i, sizeof(V));
    reinterpret_cast<V *>(p)[i] = t;
  }
}

// The same with the non-temporal hint.  Which accesses take it is by measurement, in
// us, for none / loads / stores / both: looked-up rows 73 / 74 / 70 / 70 (389123 x
// 256 bf16) and 66 / 66 / 53 / 53 (300000 x 257): stores.  Rows by expert and
// back 145 / 139 / 137 / 135 and backward 163 / 162 / 159 / 153 (50021 x 2 of 1024
// bf16), but 82 / 76 / 87 / 87 (90000 x 2 of 257): both, the sorted rows' stores only
// where they do not share lines.  Row
// sums 780 / 788 / 788 / 754 (900000 x 1024 f16), 119 / 123 / 117 / 123 (123457 x
// 256 bf16), 142 / 144 / 144 / 152 (300000 x 257): both where the rows are more
// than the last-level cache, else none.  Activations 203 / 208 /
// 192 / 190 (200000 x 257 gated bf16, forward and backward): both.
template <int kN, typename T>
__device__ __forceinline__ void load_row_once(const T *p, T (&v)[kN]) {
  typedef typename PieceOf<sizeof(v)>::V V;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T[kN]) / (sizeof(V))); ++i) {
    const V t = __builtin_nontemporal_load(reinterpret_cast<const V *>(p) + i);
    __builtin_memcpy(reinterpret_cast<char *>(v) + sizeof(V) * i, &t, sizeof(V));
  }
}

template <int kN, typename T>
__device__ __forceinline__ void store_row_once(T *p, const T (&v)[kN]) {
  typedef typename PieceOf<sizeof(v)>::V V;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T[kN]) / (sizeof(V))); ++i) {
    V t;
    __builtin_memcpy(&t, reinterpret_cast<const char *>(v) + sizeof(V) * i, sizeof(V));
    __builtin_nontemporal_store(t, reinterpret_cast<V *>(p) + i);
  }
}

template <bool kOnce, int kN, typename T>
__device__ __forceinline__ void load_row_as(const T *p, T (&v)[kN]) {
  if constexpr (kOnce)
    load_row_once(p, v);
  else
    load_row(p, v);
}

template <bool kOnce, int kN, typename T>
__device__ __forceinline__ void store_row_as(T *p, const T (&v)[kN]) {
  if constexpr (kOnce)
    store_row_once(p, v);
  else
    store_row(p, v);
}

constexpr uint64_t kLastLevelCache = 256ull << 20;

// Whether the rows at p, ld elements apart, start at lines of the caches.
inline bool on_lines(const void *p, uint64_t ld, uint32_t type) {
  return reinterpret_cast<uintptr_t>(p) % 128 == 0 && ld * elem_bytes(type) % 128 == 0;
}

// Elements of a 16-byte piece.
template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);

// A row is handled in pieces of kPiece<T> elements.  The last piece of a row
// whose width is no multiple ends with the row and overlaps the one before it:
// its elements are computed twice and written twice with the same values.  A
// row narrower than a piece is one piece of fewer elements.
inline uint32_t pieces(uint64_t dim, uint32_t piece) { return (uint32_t)((dim + piece - 1) / piece); }

// x / d and x % d for x < 2^16 + 2^14 and d <= 2^14, with m = divider(d):
// x * (m d - 2^32) <= x d < 2^32 keeps the quotient exact.
inline uint64_t divider(uint32_t d) { return (1ull << 32) / d + 1; }

// Blocks for `work` units, `per` of them a block.
inline uint64_t blocks_for(uint64_t work, uint64_t per) { return (work + per - 1) / per; }

// f(first row, rows) for launches of `lanes` lanes a row that have spare ones in narrow
// rows: at most 2^30 lanes at once.
template <typename F>
inline void in_launches(uint64_t rows, uint64_t lanes, F f) {
  const uint64_t most = (1ull << 30) / lanes;
  for (uint64_t r = 0; r < rows; r += most) f(r, rows - r < most ? rows - r : most);
}

}  // namespace lsm_rows
