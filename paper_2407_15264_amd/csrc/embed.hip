// Rows of a trained table, looked up by ID, and the table's gradient.
//
// Lookup: out[i] = scale * table[ids[i]].  Each 16-byte piece of an output row is
// one lane's: consecutive lanes take consecutive pieces, so rows of any width
// fill the lanes, and each lane has kUnroll independent loads in flight.  Bound by
// memory: 389123 rows of 256 bf16 of a table of 5 GB in 70 us, 5.7 TB/s read and
// written; one row 2 us, the launch.
//
// Gradient: row v = scale * sum of dy[i] over ids[i] == v.  The places are sorted
// by ID (stable), then the rows of dy are summed along the sorted order: a group
// of lanes takes a chunk of consecutive sorted places and keeps one run's sum in
// registers, writing it out where the ID changes.  A run that crosses chunks
// leaves a 32-bit partial sum in each, and the join adds those.  Every order
// follows from the sizes and the IDs, no value is added by an atomic, and a node
// that occurs very often costs its chunks the same as any other rows.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "lsmgnn.h"
#include "rows.h"
#include "sort.h"

namespace lsm_embed {

using namespace lsm_rows;

// ------------------------------------------------------------------- lookup
constexpr int kUnroll = 4;  // pieces per thread (389123 rows of 256 bf16: 69 us; 1: 75; 8: 86)

template <typename Ti, typename To>
__global__ __launch_bounds__(kBlock) void k_embed_rows(const Ti *table, uint64_t num_rows, uint32_t dim, uint64_t tld,
                                                       const int64_t *ids, uint64_t n, int64_t pad, float scale,
                                                       To *out, uint64_t old_, uint32_t np, uint64_t div64,
                                                       uint64_t div32, uint64_t *status) {
  constexpr int kN = kPiece<Ti>;
  const uint64_t base = (uint64_t)blockIdx.x * (kBlock * kUnroll);
  const uint64_t row0 = div64 ? __umul64hi(base, div64) : base;
  const uint32_t col0 = (uint32_t)(base - row0 * np);
  int64_t id[kUnroll];
  uint64_t row[kUnroll];
  uint32_t at[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t x = col0 + u * kBlock + threadIdx.x;
    const uint32_t r = (uint32_t)((x * div32) >> 32);
    row[u] = row0 + r;
    at[u] = (x - r * np) * kN;
    id[u] = row[u] < n ? ids[row[u]] : -1;
  }
  if (dim >= (uint32_t)kN) {
    Ti v[kUnroll][kN];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      at[u] = at[u] + kN > dim ? dim - kN : at[u];
      const bool some = row[u] < n && id[u] != pad && (uint64_t)id[u] < num_rows;
      if (some) {
        load_row(table + (uint64_t)id[u] * tld + at[u], v[u]);
      } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) v[u][e] = (Ti)0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (row[u] >= n) continue;
      To o[kN];
      // a place without a row is zeros whatever the scale
      const bool some = id[u] != pad && (uint64_t)id[u] < num_rows;
#pragma unroll
      for (int e = 0; e < kN; ++e) o[e] = some ? (To)((float)v[u][e] * scale) : (To)0.0f;
      store_row_once(out + row[u] * old_ + at[u], o);
      if (status && id[u] != pad && (uint64_t)id[u] >= num_rows) *status = LSMGNN_E_RANGE;
    }
  } else {
    for (int u = 0; u < kUnroll; ++u) {
      if (row[u] >= n) continue;
      const bool some = id[u] != pad && (uint64_t)id[u] < num_rows;
      for (uint32_t e = 0; e < dim; ++e)
        out[row[u] * old_ + e] = some ? (To)((float)table[(uint64_t)id[u] * tld + e] * scale) : (To)0.0f;
      if (status && id[u] != pad && (uint64_t)id[u] >= num_rows) *status = LSMGNN_E_RANGE;
    }
  }
}

// --------------------------------------------------------- places sorted by ID
// A place is (key, place): the key is its ID, num_rows for a padding place and
// num_rows + 1 for an ID out of range, so that those come last and the last
// place says whether there is one out of range.
typedef uint64_t Place;
__device__ __forceinline__ uint32_t key_of(Place p) { return (uint32_t)(p >> 32); }

struct FromIds {
  typedef Place Item;
  const int64_t *ids;
  int64_t pad;
  uint32_t num_rows, shift, mask;
  __device__ __forceinline__ Item load(uint32_t i) const {
    const int64_t id = ids[i];
    const uint32_t key = id == pad ? num_rows : (uint64_t)id >= num_rows ? num_rows + 1 : (uint32_t)id;
    return (Place)key << 32 | i;
  }
  __device__ __forceinline__ uint32_t digit(Item p) const { return (key_of(p) >> shift) & mask; }
};

struct FromPlaces {
  typedef Place Item;
  const Place *in;
  uint32_t shift, mask;
  __device__ __forceinline__ Item load(uint32_t i) const { return in[i]; }
  __device__ __forceinline__ uint32_t digit(Item p) const { return (key_of(p) >> shift) & mask; }
};

struct ToPlaces {
  Place *out;
  __device__ __forceinline__ void put(uint32_t at, Place p, uint32_t) const { out[at] = p; }
  __device__ __forceinline__ void start(uint32_t, uint32_t) const {}
  __device__ __forceinline__ void unused(uint32_t, uint32_t, uint32_t) const {}
  __device__ __forceinline__ void after(uint32_t) const {}
};

// A block's places, item i of lane l of wave w being the place 64 (kN w + i) + l,
// sorted by key: digits of up to 8 bits, the places exchanged through LDS after
// each.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortBits = 8, kSortBins = 1 << kSortBits;
constexpr uint64_t kBlockSortMax = 1024 * 4;

template <int kN>
__device__ __forceinline__ void sort_items(Place (&item)[kN], const bool (&ok)[kN], uint32_t key_bits, Place *exch,
                                           uint32_t (*hist)[kSortBins], uint32_t *tmp) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t first = wave * 64 * kN + lane;
  const uint32_t passes = (key_bits + kSortBits - 1) / kSortBits, bits = (key_bits + passes - 1) / passes;
  const uint32_t bins = 1u << bits;
  for (uint32_t shift = 0; shift < key_bits; shift += bits) {
    for (uint32_t d = threadIdx.x; d < kSortWaves * bins; d += kSortThreads) hist[d >> bits][d & (bins - 1)] = 0;
    __syncthreads();
    uint32_t digit[kN], rank[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) digit[i] = (key_of(item[i]) >> shift) & (bins - 1);
    lsm_sort::wave_ranks<kN>(digit, ok, bits, hist[wave], rank);
    __syncthreads();
    uint32_t sum = 0, unused;
    if (threadIdx.x < bins)
      for (int w = 0; w < kSortWaves; ++w) sum += hist[w][threadIdx.x];
    uint32_t run = lsm_sort::block_scan<kSortThreads>(sum, tmp, &unused);
    if (threadIdx.x < bins)
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = hist[w][threadIdx.x];
        hist[w][threadIdx.x] = run;
        run += c;
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (ok[i]) exch[hist[wave][digit[i]] + rank[i]] = item[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) item[i] = ok[i] ? exch[first + i * 64] : 0;
    __syncthreads();
  }
}

// At most 1024 * kN places, sorted by block 0; the others fill (see Fill).  The gradient
// by rows of 64 bf16 out of 100000 so, and by the tiles of sort.h: 1000 places 20 and
// 24 us, 3000 26 and 35, 4096 28 and 35.
template <int kN>
__global__ __launch_bounds__(kSortThreads) void k_sort_block(FromIds src, uint32_t n, uint32_t key_bits, Place *out,
                                                             lsm_sort::Fill fill) {
  __shared__ Place exch[kSortThreads * kN];
  __shared__ uint32_t hist[kSortWaves][kSortBins];
  __shared__ uint32_t tmp[kSortWaves];
  if (blockIdx.x) {
    fill.zero(blockIdx.x - 1);
    return;
  }
  const uint32_t first = (threadIdx.x >> 6) * 64 * kN + (threadIdx.x & 63);
  Place item[kN];
  bool ok[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    ok[i] = first + i * 64 < n;
    item[i] = ok[i] ? src.load(first + i * 64) : 0;
  }
  sort_items<kN>(item, ok, key_bits, exch, hist, tmp);
#pragma unroll
  for (int i = 0; i < kN; ++i)
    if (ok[i]) out[first + i * 64] = item[i];
}

// --------------------------------------------------------------- sums of runs
constexpr uint32_t kNone = 0xffffffffu, kInside = 0xfffffffeu;
constexpr int kStage = 2048;     // sorted places that a block holds at most
constexpr int kHeadTile = 1024;  // places per count of the runs' heads

// How many runs begin in each tile of kHeadTile sorted places.
__global__ __launch_bounds__(kBlock) void k_count_heads(const Place *places, uint32_t n, uint32_t num_rows,
                                                        uint32_t *heads) {
  __shared__ uint32_t tmp[kBlock / 64];
  uint32_t mine = 0, all;
  for (uint32_t i = threadIdx.x; i < kHeadTile; i += kBlock) {
    const uint32_t at = blockIdx.x * kHeadTile + i;
    if (at < n) {
      const uint32_t key = key_of(places[at]);
      mine += key < num_rows && (at == 0 || key_of(places[at - 1]) != key);
    }
  }
  lsm_sort::block_scan<kBlock>(mine, tmp, &all);
  if (threadIdx.x == 0) heads[blockIdx.x] = all;
}

// With many tiles, how many begin before each: one block, so that the blocks of the
// sums, which otherwise add up the tiles before them, need not read them all, a
// square of the places in all.  Rows of 8 bf16, scanned and not: 4 million places 543
// and 537 us, 5 million 684 and 677, 10 million 1309 and 1315, 20 million 2688 and
// 2707.
constexpr uint32_t kScannedHeads = 4096;

__global__ __launch_bounds__(kSortThreads) void k_scan_heads(uint32_t *heads, uint32_t tiles) {
  __shared__ uint32_t tmp[kSortWaves];
  uint32_t before = 0, all;
  for (uint32_t t0 = 0; t0 < tiles; t0 += kSortThreads) {
    const uint32_t t = t0 + threadIdx.x, mine = t < tiles ? heads[t] : 0;
    const uint32_t run = before + lsm_sort::block_scan<kSortThreads>(mine, tmp, &all);
    if (t < tiles) heads[t] = run;
    before += all;
  }
}

// The first `count` of kN values, rounded to the type, at element `at` of out.
template <int kN>
__device__ __forceinline__ void store_as(void *out, uint32_t type, uint64_t at, const float (&v)[kN], int count) {
#pragma unroll
  for (int e = 0; e < kN; ++e) {
    if (e >= count) break;
    if (type == LSMGNN_F32)
      static_cast<float *>(out)[at + e] = v[e];
    else if (type == LSMGNN_F16)
      static_cast<_Float16 *>(out)[at + e] = (_Float16)v[e];
    else
      static_cast<__bf16 *>(out)[at + e] = (__bf16)v[e];
  }
}

// All of them.
template <int kN, bool kOnce = false>
__device__ __forceinline__ void store_as(void *out, uint32_t type, uint64_t at, const float (&v)[kN]) {
  if (type == LSMGNN_F32) {
    store_row_as<kOnce>(static_cast<float *>(out) + at, v);
  } else if (type == LSMGNN_F16) {
    _Float16 o[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) o[e] = (_Float16)v[e];
    store_row_as<kOnce>(static_cast<_Float16 *>(out) + at, o);
  } else {
    __bf16 o[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) o[e] = (__bf16)v[e];
    store_row_as<kOnce>(static_cast<__bf16 *>(out) + at, o);
  }
}

struct Sums {
  const Place *places;    // sorted
  const uint32_t *heads;  // runs that begin in each tile, or before each (rows form), else NULL
  bool scanned;           // the latter
  uint32_t n, num_rows, dim;
  uint32_t chunk;         // places per group of lanes, a power of two
  uint32_t lanes_shift;   // lanes per group, a power of two
  float scale;
  uint64_t dy_ld;
  void *out;              // the whole gradient, or the rows that occur
  uint64_t out_ld;
  uint32_t out_type;
  int64_t *unique;        // rows form, else NULL
  uint64_t *result;       // rows form: count and status; else the status word or NULL
  float *head, *tail;     // a chunk's partial sums of runs that cross it, part_ld apart
  uint64_t part_ld;
  uint32_t *tail_row;     // the output row of the run whose tail a chunk holds; kInside for a
                          // chunk in the middle of a run; else kNone
};

// Sum the rows of dy along the sorted places.  A block has 256 / lanes groups, a
// group a chunk of places; a row wider than a wave's lanes is cut in slices, whose
// blocks are neighbours, so that all of a row is read at about the same time.
// Bound by memory: 900000 x 1024 f16 onto 630000 rows in 608 us, 5.2 TB/s with the
// partial sums; 123457 x 256 bf16 in 20 us, latency for the most part.
template <typename T, bool kOnce>
__global__ __launch_bounds__(kBlock) void k_sum_runs(Sums s, const T *dy, uint32_t slices) {
  constexpr int kN = kPiece<T>;
  constexpr int kAhead = 8;  // rows in flight per lane
  __shared__ Place stage[kStage + 2];  // the block's places, the one before and the one after
  __shared__ uint32_t row_of[kStage];  // rows form: each place's output row
  __shared__ uint32_t tmp[kBlock / 64];
  const uint32_t groups = kBlock >> s.lanes_shift, span = groups * s.chunk;
  const uint32_t slice = blockIdx.x % slices, block = blockIdx.x / slices;
  const uint64_t p0 = (uint64_t)block * span;
  for (uint32_t i = threadIdx.x; i < span + 2; i += kBlock) {
    const uint64_t at = p0 + i;  // place at - 1
    stage[i] = at >= 1 && at <= s.n ? s.places[at - 1] : (Place)kNone << 32;
  }
  __syncthreads();
  if (s.unique) {
    // runs that begin before the block: whole tiles, then the tile's places
    uint32_t mine = 0, before, all;
    const uint32_t tile = (uint32_t)(p0 / kHeadTile);
    if (s.scanned)
      mine = threadIdx.x == 0 ? s.heads[tile] : 0;
    else
      for (uint32_t t = threadIdx.x; t < tile; t += kBlock) mine += s.heads[t];
    for (uint64_t at = (uint64_t)tile * kHeadTile + threadIdx.x; at < p0; at += kBlock) {
      const uint32_t key = key_of(s.places[at]);
      mine += key < s.num_rows && (at == 0 || key_of(s.places[at - 1]) != key);
    }
    lsm_sort::block_scan<kBlock>(mine, tmp, &before);
    const uint32_t per = (span + kBlock - 1) / kBlock, i0 = threadIdx.x * per;
    mine = 0;
    for (uint32_t i = i0; i < i0 + per && i < span; ++i) {
      const uint32_t key = key_of(stage[i + 1]);
      mine += key < s.num_rows && key_of(stage[i]) != key;
    }
    uint32_t run = before + lsm_sort::block_scan<kBlock>(mine, tmp, &all);
    for (uint32_t i = i0; i < i0 + per && i < span; ++i) {
      const uint32_t key = key_of(stage[i + 1]);
      const bool begins = key < s.num_rows && key_of(stage[i]) != key;
      run += begins;
      row_of[i] = run - 1;
      if (begins && slice == 0) s.unique[run - 1] = key;
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) {
      s.result[0] = before + all;
      s.result[1] = key_of(s.places[s.n - 1]) == s.num_rows + 1 ? LSMGNN_E_RANGE : LSMGNN_OK;
    }
    __syncthreads();
  } else if (s.result && blockIdx.x == 0 && threadIdx.x == 0) {
    if (key_of(s.places[s.n - 1]) == s.num_rows + 1) *s.result = LSMGNN_E_RANGE;
  }

  const uint32_t group = threadIdx.x >> s.lanes_shift, lane = threadIdx.x & ((1u << s.lanes_shift) - 1);
  const uint64_t chunk = (uint64_t)block * groups + group;
  if (chunk * s.chunk >= s.n) return;
  const uint32_t i0 = group * s.chunk;
  uint32_t col = (slice << s.lanes_shift) + lane;
  col *= kN;
  const bool whole = s.dim >= (uint32_t)kN;
  const bool works = col < s.dim;
  if (whole && works && col + kN > s.dim) col = s.dim - kN;
  const int count = whole ? kN : (int)s.dim;

  float acc[kN];
#pragma unroll
  for (int e = 0; e < kN; ++e) acc[e] = 0.0f;
  uint32_t key = key_of(stage[i0 + 1]);
  bool from_before = key_of(stage[i0]) == key;
  uint32_t first = i0;  // where the run begins, in the block
  auto partial = [&](float *to) {
    if (!works) return;
    float *p = to + chunk * s.part_ld + col;
    if (whole) {
      store_row(p, acc);
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e)
        if (e < count) p[e] = acc[e];
    }
  };
  auto finish = [&]() {
    if (!works) return;
    const uint64_t at = (uint64_t)(s.unique ? row_of[first] : key) * s.out_ld + col;
    float v[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] = acc[e] * s.scale;
    if (whole)
      store_as<kN, kOnce>(s.out, s.out_type, at, v);
    else
      store_as(s.out, s.out_type, at, v, count);
  };
  for (uint32_t i = i0; i < i0 + s.chunk; i += kAhead) {
    T v[kAhead][kN];
    uint32_t k[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const Place p = stage[i + u + 1];
      k[u] = key_of(p);
      if (k[u] < s.num_rows && works) {
        const T *row = dy + (uint64_t)(uint32_t)p * s.dy_ld + col;
        if (whole) {
          load_row_as<kOnce>(row, v[u]);
        } else {
#pragma unroll
          for (int e = 0; e < kN; ++e) v[u][e] = e < count ? row[e] : (T)0.0f;
        }
      } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) v[u][e] = (T)0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (k[u] != key) {
        if (key < s.num_rows) {
          if (from_before)
            partial(s.head);
          else
            finish();
        }
#pragma unroll
        for (int e = 0; e < kN; ++e) acc[e] = 0.0f;
        key = k[u];
        from_before = false;
        first = i + u;
      }
#pragma unroll
      for (int e = 0; e < kN; ++e) acc[e] += (float)v[u][e];
    }
  }
  const bool goes_on = key < s.num_rows && key_of(stage[i0 + s.chunk + 1]) == key;
  if (key < s.num_rows) {
    if (from_before)
      partial(s.head);
    else if (goes_on)
      partial(s.tail);
    else
      finish();
  }
  if (lane == 0 && slice == 0)
    s.tail_row[chunk] = !goes_on ? kNone : from_before ? kInside : s.unique ? row_of[first] : key;
}

// ------------------------------------------------------- runs that cross chunks
// A block has 1024 / lanes groups and as many chunks.  A group whose chunk holds
// the tail of a run finds the run's last chunk, the first that is not inside it,
// and adds the partial sums; runs over more than kAlone chunks are added by all
// groups of the block, each a consecutive share, joined through LDS.  14063 chunks of
// 1024 columns: 42 us, the reading of their partial sums; 3859 of 256: 5 us.
constexpr int kJoinThreads = 1024;
constexpr uint32_t kAlone = 16;

__device__ __forceinline__ void add_heads(const Sums &s, uint64_t from, uint64_t to, uint32_t col, float4 *acc) {
  constexpr int kAhead = 8;
  for (uint64_t c = from; c < to; c += kAhead) {
    float4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      v[u] = c + u < to ? *reinterpret_cast<const float4 *>(s.head + (c + u) * s.part_ld + col)
                        : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) acc->x += v[u].x, acc->y += v[u].y, acc->z += v[u].z, acc->w += v[u].w;
  }
}

__global__ __launch_bounds__(kJoinThreads) void k_join_runs(Sums s, uint32_t chunks, uint32_t join_shift,
                                                            uint32_t slices) {
  __shared__ float4 share[kJoinThreads];
  __shared__ uint32_t long_group[kJoinThreads], long_last[kJoinThreads], long_row[kJoinThreads], longs;
  const uint32_t groups = kJoinThreads >> join_shift, lanes = 1u << join_shift;
  const uint32_t group = threadIdx.x >> join_shift, lane = threadIdx.x & (lanes - 1);
  const uint64_t first = (uint64_t)(blockIdx.x / slices) * groups, chunk = first + group;
  const uint32_t row = chunk < chunks ? s.tail_row[chunk] : kNone;
  if (threadIdx.x == 0) longs = 0;
  __syncthreads();
  const uint32_t col = ((blockIdx.x % slices << join_shift) + lane) * 4;
  const int count = col >= s.dim ? 0 : s.dim - col < 4 ? (int)(s.dim - col) : 4;
  auto finish = [&](uint32_t out_row, const float4 &acc) {
    const float v[4] = {acc.x * s.scale, acc.y * s.scale, acc.z * s.scale, acc.w * s.scale};
    if (count == 4)
      store_as<4>(s.out, s.out_type, (uint64_t)out_row * s.out_ld + col, v);
    else
      store_as<4>(s.out, s.out_type, (uint64_t)out_row * s.out_ld + col, v, count);
  };
  auto tail = [&](uint64_t c) {
    const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    return count ? *reinterpret_cast<const float4 *>(s.tail + c * s.part_ld + col) : none;
  };
  if (row < kInside) {
    // the run's last chunk: kLook marks a lane at a time
    constexpr int kLook = 4;
    uint64_t at = chunk + 1, last = 0;
    while (!last) {
      uint32_t end = kLook * lanes;  // the first mark of these that is not kInside
#pragma unroll
      for (int u = kLook - 1; u >= 0; --u) {
        const uint64_t c = at + lane * kLook + u;
        if (c >= chunks || s.tail_row[c] != kInside) end = lane * kLook + u;
      }
      for (uint32_t d = lanes >> 1; d; d >>= 1) {
        const uint32_t o = __shfl_xor(end, d);
        end = o < end ? o : end;
      }
      if (end < kLook * lanes)
        last = at + end;
      else
        at += kLook * lanes;
    }
    if (last - chunk <= kAlone) {
      float4 acc = tail(chunk);
      if (count) add_heads(s, chunk + 1, last + 1, col, &acc);
      finish(row, acc);
    } else if (lane == 0) {
      const uint32_t i = atomicAdd(&longs, 1u);  // each is added up by itself: their order is free
      long_group[i] = group;
      long_last[i] = (uint32_t)last;
      long_row[i] = row;
    }
  }
  __syncthreads();
  for (uint32_t i = 0; i < longs; ++i) {
    const uint64_t owner = first + long_group[i], end = (uint64_t)long_last[i] + 1;
    const uint64_t per = (end - owner - 1 + groups - 1) / groups, from = owner + 1 + group * per;
    float4 acc = group == 0 ? tail(owner) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (count) add_heads(s, from < end ? from : end, from + per < end ? from + per : end, col, &acc);
    share[threadIdx.x] = acc;
    __syncthreads();
    // halves of the groups, in a fixed order
    for (uint32_t g = groups >> 1; g; g >>= 1) {
      if (group < g) {
        const float4 a = share[threadIdx.x], b = share[threadIdx.x + g * lanes];
        share[threadIdx.x] = make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
      }
      __syncthreads();
    }
    if (group == 0) finish(long_row[i], share[threadIdx.x]);
    __syncthreads();
  }
}

// ----------------------------------------------------------------- few places
// The whole gradient from at most 1024 * kN places, in one launch.  Each block
// reads all IDs and keeps the places of the table rows that are its own: a hash
// shares them out, so that neighbouring IDs, which often come together, do not.
// Up to 2^split_shift blocks have the same table rows and share out the columns,
// `units` pieces each: an ID that many places hold, which one block would add up
// alone, then has that many blocks.
// The block sorts its places in LDS, its groups of lanes take equal shares of them
// as k_sum_runs does, and a run that crosses shares is joined through LDS.  The
// rows that no ID names are written by blocks of consecutive rows, from a bit a
// row that the same look at the IDs sets.  Bound by this chain, not by bytes: 9001
// places of 128 f32 in 13.5 us, where reading the IDs ends at 6 and the rows take 4;
// 12288 take 15.5 us, and 12289 by the sort, the sums and the join 33.
constexpr uint64_t kFewPlaces = 1024 * 12;
constexpr uint32_t kFewBlocks = 256, kFewZeroRows = 1u << 16;
constexpr uint32_t kFewUnits = 32, kFewShare = 192;

template <typename T, int kN>
__global__ __launch_bounds__(kSortThreads) void k_few_places(Sums s, const T *dy, FromIds src, uint32_t key_bits,
                                                             uint32_t zero_rows, uint32_t split_shift,
                                                             uint32_t units) {
  constexpr int kP = kPiece<T>;
  constexpr int kAhead = 8;
  __shared__ __align__(16) Place exch[kSortThreads * kN];
  __shared__ union {
    uint32_t hist[kSortWaves][kSortBins];
    float head[kSortThreads * kP];
  } both;
  __shared__ uint32_t named[kFewZeroRows / 32];
  __shared__ uint32_t tmp[kSortWaves], inside[kSortThreads];
  const uint32_t wave = threadIdx.x >> 6, lane64 = threadIdx.x & 63;
  const uint32_t z0 = blockIdx.x * zero_rows;  // below 2^32: the rows are
  const uint32_t shares = gridDim.x >> split_shift, share = blockIdx.x >> split_shift;
  const uint32_t unit0 = (blockIdx.x & ((1u << split_shift) - 1)) * units;
  for (uint32_t i = threadIdx.x; i < (zero_rows + 31) / 32; i += kSortThreads) named[i] = 0;
  const uint32_t first = wave * 64 * kN + lane64;
  Place item[kN];
  bool mine[kN];
  uint32_t kept = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const bool ok = first + i * 64 < s.n;
    item[i] = ok ? src.load(first + i * 64) : (Place)kNone << 32;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const uint32_t key = key_of(item[i]);
    mine[i] = key < s.num_rows && (uint32_t)(((uint64_t)(key * 0x9e3779b1u) * shares) >> 32) == share;
    kept += (uint32_t)__popcll(__ballot(mine[i]));
    if (key < s.num_rows && key - z0 < zero_rows) atomicOr(&named[(key - z0) >> 5], 1u << ((key - z0) & 31));
    if (key == s.num_rows + 1 && s.result && blockIdx.x == 0) *s.result = LSMGNN_E_RANGE;
  }
  if (lane64 == 0) tmp[wave] = kept;
  __syncthreads();
  uint32_t m = 0, at = 0;
  for (uint32_t w = 0; w < kSortWaves; ++w) {
    if (w == wave) at = m;
    m += tmp[w];
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const uint64_t set = __ballot(mine[i]);
    if (mine[i]) exch[at + __popcll(set & ((1ull << lane64) - 1))] = item[i];
    at += (uint32_t)__popcll(set);
  }
  __syncthreads();
  if (m <= kSortThreads) {
    // each place's rank: how many are before it; waves without places look at none
    const Place p = threadIdx.x < m ? exch[threadIdx.x] : 0;
    uint32_t rank = 0;
    if (wave * 64 < m) {
      const ulonglong2 *two = reinterpret_cast<const ulonglong2 *>(exch);
#pragma unroll 16
      for (uint32_t i = 0; i < m / 2; ++i) {
        const ulonglong2 o = two[i];
        rank += (o.x < p) + (o.y < p);
      }
      if (m & 1) rank += exch[m - 1] < p;
    }
    __syncthreads();
    if (threadIdx.x < m) exch[rank] = p;
  } else {
    bool ok[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      ok[i] = first + i * 64 < m;
      item[i] = ok[i] ? exch[first + i * 64] : 0;
    }
    __syncthreads();
    sort_items<kN>(item, ok, key_bits, exch, both.hist, tmp);
  }
  __syncthreads();

  const uint32_t lanes = 1u << s.lanes_shift, groups = kSortThreads >> s.lanes_shift;
  const uint32_t group = threadIdx.x >> s.lanes_shift, lane = threadIdx.x & (lanes - 1);
  const bool whole = s.dim >= (uint32_t)kP;
  const int count = whole ? kP : (int)s.dim;
  const uint32_t slices = (units + lanes - 1) >> s.lanes_shift;
  const float zero[kP] = {};
  for (uint32_t r = group; r < zero_rows && r < s.num_rows - z0; r += groups) {
    if (z0 >= s.num_rows) break;
    if (named[r >> 5] >> (r & 31) & 1) continue;
    for (uint32_t c = lane * kP; c < s.dim; c += lanes * kP) {
      const uint64_t to = (uint64_t)(z0 + r) * s.out_ld + (whole && c + kP > s.dim ? s.dim - kP : c);
      if (whole)
        store_as<kP>(s.out, s.out_type, to, zero);
      else
        store_as(s.out, s.out_type, to, zero, count);
    }
  }
  const uint32_t per = (m + groups - 1) / groups, i0 = group * per, i1 = i0 + per < m ? i0 + per : m;
  for (uint32_t slice = 0; slice < slices; ++slice) {
    const uint32_t unit = (slice << s.lanes_shift) + lane;
    uint32_t col = (unit0 + unit) * kP;
    const bool works = unit < units && col < s.dim;
    if (whole && works && col + kP > s.dim) col = s.dim - kP;
    float acc[kP];
#pragma unroll
    for (int e = 0; e < kP; ++e) acc[e] = 0.0f;
    uint32_t key = i0 < i1 ? key_of(exch[i0]) : kNone;
    bool from_before = i0 < i1 && i0 > 0 && key_of(exch[i0 - 1]) == key;
    auto finish = [&]() {
      if (!works) return;
      float v[kP];
#pragma unroll
      for (int e = 0; e < kP; ++e) v[e] = acc[e] * s.scale;
      if (whole)
        store_as<kP>(s.out, s.out_type, (uint64_t)key * s.out_ld + col, v);
      else
        store_as(s.out, s.out_type, (uint64_t)key * s.out_ld + col, v, count);
    };
    auto keep = [&]() {
#pragma unroll
      for (int e = 0; e < kP; ++e) both.head[threadIdx.x * kP + e] = acc[e];
    };
    for (uint32_t i = i0; i < i1; i += kAhead) {
      T v[kAhead][kP];
      uint32_t k[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const Place p = i + u < i1 ? exch[i + u] : (Place)kNone << 32;
        k[u] = key_of(p);
#pragma unroll
        for (int e = 0; e < kP; ++e) v[u][e] = (T)0.0f;
        if (i + u < i1 && works) {
          const T *row = dy + (uint64_t)(uint32_t)p * s.dy_ld + col;
          if (whole) {
            load_row(row, v[u]);
          } else {
#pragma unroll
            for (int e = 0; e < kP; ++e) v[u][e] = e < count ? row[e] : (T)0.0f;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i + u >= i1) break;
        if (k[u] != key) {
          if (from_before)
            keep();
          else
            finish();
#pragma unroll
          for (int e = 0; e < kP; ++e) acc[e] = 0.0f;
          key = k[u];
          from_before = false;
        }
#pragma unroll
        for (int e = 0; e < kP; ++e) acc[e] += (float)v[u][e];
      }
    }
    const bool goes_on = i0 < i1 && i1 < m && key_of(exch[i1]) == key;
    if (i0 < i1) {
      if (from_before)
        keep();
      else if (!goes_on)
        finish();
    }
    if (lane == 0) inside[group] = from_before && goes_on;
    __syncthreads();
    if (goes_on && !from_before) {
      for (uint32_t g = group + 1;; ++g) {
#pragma unroll
        for (int e = 0; e < kP; ++e) acc[e] += both.head[(g * lanes + lane) * kP + e];
        if (!inside[g]) break;
      }
      finish();
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------ rows without IDs
// Zeros in `rows` rows of `per` elements that start `stride` elements
// apart.
template <typename U>
__global__ __launch_bounds__(kBlock) void k_zero_rows(U *out, uint64_t rows, uint64_t per, uint64_t stride) {
  for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (uint64_t e = threadIdx.x; e < per; e += kBlock) out[r * stride + e] = 0;
}

__global__ __launch_bounds__(kBlock) void k_fill(lsm_sort::Fill fill) { fill.zero(blockIdx.x); }

__global__ void k_no_rows(uint64_t *result) {
  result[0] = 0;
  result[1] = LSMGNN_OK;
}

// ------------------------------------------------------------------- the host
uint32_t bit_length(uint64_t x) {
  uint32_t b = 0;
  while (x) {
    ++b;
    x >>= 1;
  }
  return b;
}

// Lanes (as a shift) that cover `units` pieces of a row, at most a wave.
uint32_t lanes_shift(uint64_t units) {
  uint32_t s = 0;
  while (s < 6 && (1u << s) < units) ++s;
  return s;
}

// The sizes of a gradient's work: how the places are cut, and the memory.
struct Plan {
  uint32_t key_bits, passes, bits;
  uint32_t chunk, shift;
  uint64_t chunks, part_ld;
  uint64_t at_a, at_b, at_counts, at_heads, at_rows, at_head, at_tail, bytes;
};

Plan plan_of(uint64_t n, uint64_t num_rows, uint64_t dim, uint32_t piece) {
  Plan p{};
  p.key_bits = bit_length(num_rows + 1);
  p.passes = (p.key_bits + lsm_sort::kMaxDigitBits - 1) / lsm_sort::kMaxDigitBits;
  p.bits = (p.key_bits + p.passes - 1) / p.passes;
  p.shift = lanes_shift(pieces(dim, piece));
  // a chunk's two partial rows stay small beside its rows, and there are enough
  // chunks to keep the memory busy
  uint32_t c = 8;
  while (c < 64 && n / c >= 2 * 2048) c *= 2;
  const uint32_t most = (uint32_t)kStage >> (8 - p.shift);  // a block's places fit the stage
  p.chunk = c < most ? c : most;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  p.part_ld = (dim + 3) / 4 * 4;
  auto take = [&](uint64_t bytes) {
    const uint64_t at = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  p.at_a = take(n * 8);
  p.at_b = n > kBlockSortMax ? take(n * 8) : 0;
  p.at_counts = n > kBlockSortMax ? take(lsm_sort::count_words(n, 1ull << p.bits) * 4) : 0;
  p.at_heads = take((n + kHeadTile - 1) / kHeadTile * 4);
  p.at_rows = take(p.chunks * 4);
  p.at_head = take(p.chunks * p.part_ld * 4);
  p.at_tail = take(p.chunks * p.part_ld * 4);
  return p;
}

// The places of `ids` sorted by key into *sorted (one of the work's two arrays);
// zeros: memory to be cleared beside the sort, in equal parts by its launches,
// which leave most of the chip idle.
void queue_sort(const Plan &p, const int64_t *ids, uint32_t n, uint32_t num_rows, int64_t pad, uint8_t *work,
                const Place **sorted, lsm_sort::Fill zeros, hipStream_t st) {
  Place *a = reinterpret_cast<Place *>(work + p.at_a), *b = reinterpret_cast<Place *>(work + p.at_b);
  uint32_t *counts = reinterpret_cast<uint32_t *>(work + p.at_counts);
  FromIds from{ids, pad, num_rows, 0, (1u << p.bits) - 1};
  *sorted = a;
  if (n <= kBlockSortMax) {
    const dim3 grid(1 + zeros.blocks(kSortThreads));
    if (n <= 1024)
      hipLaunchKernelGGL(k_sort_block<1>, grid, dim3(kSortThreads), 0, st, from, n, p.key_bits, a, zeros);
    else
      hipLaunchKernelGGL(k_sort_block<4>, grid, dim3(kSortThreads), 0, st, from, n, p.key_bits, a, zeros);
    return;
  }
  const uint32_t launches = p.passes * lsm_sort::launches_of(n);
  uint32_t done = 0;
  lsm_sort::queue_pass(from, ToPlaces{a}, n, 1u << p.bits, p.bits, 1, counts, zeros, &done, launches, st);
  for (uint32_t pass = 1; pass < p.passes; ++pass) {
    lsm_sort::queue_pass(FromPlaces{a, pass * p.bits, (1u << p.bits) - 1}, ToPlaces{b}, n, 1u << p.bits, p.bits, 1,
                         counts, zeros, &done, launches, st);
    Place *t = a;
    a = b;
    b = t;
  }
  *sorted = a;
}

void queue_sums(const Plan &p, Sums s, const void *dy, uint32_t dy_type, uint8_t *work, hipStream_t st) {
  uint32_t *heads = reinterpret_cast<uint32_t *>(work + p.at_heads);
  s.heads = heads;
  s.chunk = p.chunk;
  s.lanes_shift = p.shift;
  s.head = reinterpret_cast<float *>(work + p.at_head);
  s.tail = reinterpret_cast<float *>(work + p.at_tail);
  s.part_ld = p.part_ld;
  s.tail_row = reinterpret_cast<uint32_t *>(work + p.at_rows);
  if (s.unique) {
    const uint32_t tiles = (s.n + kHeadTile - 1) / kHeadTile;
    hipLaunchKernelGGL(k_count_heads, dim3(tiles), dim3(kBlock), 0, st, s.places, s.n, s.num_rows, heads);
    s.scanned = tiles > kScannedHeads;
    if (s.scanned) hipLaunchKernelGGL(k_scan_heads, dim3(1), dim3(kSortThreads), 0, st, heads, tiles);
  }
  const uint32_t span = (kBlock >> p.shift) * p.chunk;
  with_type(dy_type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    const uint32_t slices = (pieces(s.dim, kPiece<T>) + (1u << p.shift) - 1) >> p.shift;
    const dim3 grid((s.n + span - 1) / span * slices);
    if ((uint64_t)s.n * s.dim * sizeof(T) > kLastLevelCache)
      hipLaunchKernelGGL((k_sum_runs<T, true>), grid, dim3(kBlock), 0, st, s, static_cast<const T *>(dy), slices);
    else
      hipLaunchKernelGGL((k_sum_runs<T, false>), grid, dim3(kBlock), 0, st, s, static_cast<const T *>(dy), slices);
  });
  if (p.chunks > 1) {
    const uint32_t js = lanes_shift(p.part_ld / 4), groups = kJoinThreads >> js;
    const uint32_t slices = (uint32_t)((p.part_ld / 4 + (1u << js) - 1) >> js);
    hipLaunchKernelGGL(k_join_runs, dim3((p.chunks + groups - 1) / groups * slices), dim3(kJoinThreads), 0, st, s,
                       (uint32_t)p.chunks, js, slices);
  }
}

// Whether k_few_places takes the whole gradient.  With fewer rows than blocks its
// places could not be shared out, and above its limit of rows a block has no room
// for their bits.
bool few_places(uint64_t n, uint64_t num_rows) {
  return n <= kFewPlaces && num_rows >= kFewBlocks && num_rows <= (uint64_t)kFewBlocks * kFewZeroRows;
}

void queue_few_places(Sums s, const void *dy, uint32_t dy_type, const int64_t *ids, int64_t pad, hipStream_t st) {
  const uint32_t zero_rows = (s.num_rows + kFewBlocks - 1) / kFewBlocks;
  const FromIds from{ids, pad, s.num_rows, 0, 0};
  const uint32_t key_bits = bit_length(s.num_rows - 1);
  with_type(dy_type, [&](auto tag) {
    typedef typename decltype(tag)::T T;
    const uint32_t all = pieces(s.dim, kPiece<T>);
    // the columns are cut while a block's part of a row is kFewUnits loads and its
    // places, were the rows shared evenly, are kFewShare: more places take longer to
    // sort than the cut saves.  20000 rows of 1024 f32, 12288 skewed IDs: uncut 39.5
    // us, 32.7 so, 35.1 with up to 384 places; all the same ID: 637, 185 and 112.
    // Parts of 16 loads cost narrow rows more than they save (16384 x 128 f32, 9001
    // IDs: 13.6 us uncut, 15.0 so)
    uint32_t split = 0;
    while ((2u << split) <= kFewBlocks && all >> (split + 1) >= kFewUnits &&
           ((uint64_t)s.n << (split + 1)) <= (uint64_t)kFewShare * kFewBlocks)
      ++split;
    const uint32_t units = (all + (1u << split) - 1) >> split;
    s.lanes_shift = lanes_shift(units);
    const T *g = static_cast<const T *>(dy);
    if (s.n <= 1024)
      hipLaunchKernelGGL((k_few_places<T, 1>), dim3(kFewBlocks), dim3(kSortThreads), 0, st, s, g, from, key_bits,
                         zero_rows, split, units);
    else if (s.n <= 4096)
      hipLaunchKernelGGL((k_few_places<T, 4>), dim3(kFewBlocks), dim3(kSortThreads), 0, st, s, g, from, key_bits,
                         zero_rows, split, units);
    else
      hipLaunchKernelGGL((k_few_places<T, 12>), dim3(kFewBlocks), dim3(kSortThreads), 0, st, s, g, from, key_bits,
                         zero_rows, split, units);
  });
}

bool grad_args_ok(const void *dy, uint64_t dim, uint64_t dy_ld, uint32_t dy_type, const int64_t *ids, uint64_t n,
                  uint64_t num_rows, const void *out, uint64_t out_rows, uint64_t out_ld, uint32_t out_type,
                  const void *work, uint64_t work_bytes, uint64_t need) {
  return num_rows >= 1 && num_rows <= 0xfffffffcull && matrix_ok(dy, n, dim, dy_ld, dy_type) &&
         type_ok(out_type) && ld_ok(out, out_rows, dim, out_ld, out_type) && (n == 0 || ids) &&
         (need == 0 || (work && reinterpret_cast<uintptr_t>(work) % 256 == 0 && work_bytes >= need));
}

}  // namespace lsm_embed

extern "C" {

lsmgnn_status lsmgnn_embed_rows(const void *table, uint64_t num_rows, uint64_t dim, uint64_t table_ld,
                                uint32_t table_type, const int64_t *ids, uint64_t n, int64_t pad, float scale,
                                void *out, uint64_t out_ld, uint32_t out_type, uint64_t *status, void *stream) {
  using namespace lsm_embed;
  uint64_t *st_word;
  if (num_rows > 0xfffffffcull || !type_ok(table_type) || !ld_ok(table, num_rows, dim, table_ld, table_type) ||
      !matrix_ok(out, n, dim, out_ld, out_type) || (n && !ids) || !status_view(status, &st_word))
    return LSMGNN_E_INVAL;
  if (n == 0) return LSMGNN_OK;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(table_type, [&](auto ti) {
    with_type(out_type, [&](auto to) {
      typedef typename decltype(ti)::T Ti;
      typedef typename decltype(to)::T To;
      const uint32_t np = pieces(dim, kPiece<Ti>);
      const uint64_t div64 = np > 1 ? ~0ull / np + 1 : 0;
      hipLaunchKernelGGL((k_embed_rows<Ti, To>), dim3(blocks_for(n * np, kBlock * kUnroll)), dim3(kBlock), 0, st,
                         static_cast<const Ti *>(table), num_rows, (uint32_t)dim, table_ld, ids, n, pad, scale,
                         static_cast<To *>(out), out_ld, np, div64, divider(np), st_word);
    });
  });
  if (hipGetLastError() != hipSuccess) return LSMGNN_E_DEVICE;
  return LSMGNN_OK;
}

uint64_t lsmgnn_embed_grad_work_bytes(uint64_t n, uint64_t num_rows, uint64_t dim) {
  using namespace lsm_embed;
  if (n == 0 || n > kMaxRows || dim == 0 || dim > kMaxDim) return 0;
  // the element type decides how a row is cut, not how much the cuts take: the
  // larger of the two
  const uint64_t a = plan_of(n, num_rows, dim, 4).bytes, b = plan_of(n, num_rows, dim, 8).bytes;
  return a > b ? a : b;
}

uint64_t lsmgnn_table_grad_work_bytes(uint64_t n, uint64_t num_rows, uint64_t dim) {
  return lsm_embed::few_places(n, num_rows) ? 0 : lsmgnn_embed_grad_work_bytes(n, num_rows, dim);
}

lsmgnn_status lsmgnn_embed_grad(const void *dy, uint64_t dim, uint64_t dy_ld, uint32_t dy_type, const int64_t *ids,
                                uint64_t n, uint64_t num_rows, int64_t pad, float scale, void *grad,
                                uint64_t grad_ld, uint32_t grad_type, void *work, uint64_t work_bytes,
                                uint64_t *status, void *stream) {
  using namespace lsm_embed;
  uint64_t *st_word;
  if (!grad || !grad_args_ok(dy, dim, dy_ld, dy_type, ids, n, num_rows, grad, num_rows, grad_ld, grad_type, work,
                             work_bytes, lsmgnn_table_grad_work_bytes(n, num_rows, dim)) ||
      !status_view(status, &st_word))
    return LSMGNN_E_INVAL;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t es = elem_bytes(grad_type);
  Sums s{};
  s.n = (uint32_t)n;
  s.num_rows = (uint32_t)num_rows;
  s.dim = (uint32_t)dim;
  s.scale = scale;
  s.dy_ld = dy_ld;
  s.out = grad;
  s.out_ld = grad_ld;
  s.out_type = grad_type;
  s.result = st_word;
  if (n && few_places(n, num_rows)) {
    queue_few_places(s, dy, dy_type, ids, pad, st);
  } else {
    lsm_sort::Fill zeros{};
    if (grad_ld == dim || num_rows <= 1)
      zeros = lsm_sort::Fill::of(grad, num_rows * dim * es);
    else if (es == 4)
      hipLaunchKernelGGL(k_zero_rows<uint32_t>, dim3(num_rows < 8192 ? num_rows : 8192), dim3(kBlock), 0, st,
                         static_cast<uint32_t *>(grad), num_rows, dim, grad_ld);
    else
      hipLaunchKernelGGL(k_zero_rows<uint16_t>, dim3(num_rows < 8192 ? num_rows : 8192), dim3(kBlock), 0, st,
                         static_cast<uint16_t *>(grad), num_rows, dim, grad_ld);
    constexpr uint64_t kMostFill = 1ull << 36;  // 2^30 lanes
    for (; zeros.bytes > kMostFill; zeros = lsm_sort::Fill::of(zeros.at + kMostFill, zeros.bytes - kMostFill)) {
      const lsm_sort::Fill some = lsm_sort::Fill::of(zeros.at, kMostFill);
      hipLaunchKernelGGL(k_fill, dim3(some.blocks(kBlock)), dim3(kBlock), 0, st, some);
    }
    if (n) {
      const Plan p = plan_of(n, num_rows, dim, 16 / elem_bytes(dy_type));
      uint8_t *w = static_cast<uint8_t *>(work);
      queue_sort(p, ids, s.n, s.num_rows, pad, w, &s.places, zeros, st);
      queue_sums(p, s, dy, dy_type, w, st);
    } else if (zeros.bytes) {
      hipLaunchKernelGGL(k_fill, dim3(zeros.blocks(kBlock)), dim3(kBlock), 0, st, zeros);
    }
  }
  if (hipGetLastError() != hipSuccess) return LSMGNN_E_DEVICE;
  return LSMGNN_OK;
}

lsmgnn_status lsmgnn_embed_grad_rows(const void *dy, uint64_t dim, uint64_t dy_ld, uint32_t dy_type,
                                     const int64_t *ids, uint64_t n, uint64_t num_rows, int64_t pad, float scale,
                                     int64_t *unique, void *rows, uint64_t rows_ld, uint32_t rows_type, void *work,
                                     uint64_t work_bytes, uint64_t *result_host, void *stream) {
  using namespace lsm_embed;
  uint64_t *res;
  if (!result_host || !grad_args_ok(dy, dim, dy_ld, dy_type, ids, n, num_rows, rows, n, rows_ld, rows_type, work,
                                    work_bytes, lsmgnn_embed_grad_work_bytes(n, num_rows, dim)) ||
      (n && !unique) || !status_view(result_host, &res))
    return LSMGNN_E_INVAL;
  const StreamDevice on(stream);
  if (!on.ok) return LSMGNN_E_DEVICE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n) {
    const Plan p = plan_of(n, num_rows, dim, 16 / elem_bytes(dy_type));
    uint8_t *w = static_cast<uint8_t *>(work);
    Sums s{};
    s.n = (uint32_t)n;
    s.num_rows = (uint32_t)num_rows;
    s.dim = (uint32_t)dim;
    s.scale = scale;
    s.dy_ld = dy_ld;
    s.out = rows;
    s.out_ld = rows_ld;
    s.out_type = rows_type;
    s.unique = unique;
    s.result = res;
    queue_sort(p, ids, s.n, s.num_rows, pad, w, &s.places, lsm_sort::Fill{}, st);
    queue_sums(p, s, dy, dy_type, w, st);
  } else {
    hipLaunchKernelGGL(k_no_rows, dim3(1), dim3(1), 0, st, res);
  }
  if (hipGetLastError() != hipSuccess) return LSMGNN_E_DEVICE;
  return LSMGNN_OK;
}

}  // extern "C"
