// Interface between the long-memory entry points (evo_memory.hip) and their
// kernels: rows of queries, keys and values (evo_memory_rows.hip) and
// attention over the paged cache (evo_memory_attention.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "evo.h"

namespace evo {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// formats whose values are codes of 8 or 4 bits with a scale
constexpr bool is_coded(int f) { return f == EVO_CACHE_INT8 || f == EVO_CACHE_FP8 || f == EVO_CACHE_FP4; }
// formats whose values can be a NaN or an infinity by themselves
constexpr bool holds_nan(int f) { return f != EVO_CACHE_INT8 && f != EVO_CACHE_FP4; }
// values in a byte of a code, of a page's row
constexpr int per_byte(int f) { return f == EVO_CACHE_FP4 ? 2 : 1; }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// LDS that one wave writes and reads: its accesses are in order, the compiler
// has to keep them so
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Division of n < 2^31 by a divisor that the launch knows, in five operations
// (T. Granlund and P. Montgomery, Division by invariant integers using
// multiplication, PLDI 1994): the compiler's own for unknown divisors is some
// forty, and short calls are mostly such work.
struct Divisor {
  uint32_t m;
  int32_t s1, s2;
  static Divisor of(int64_t d) {
    int l = 0;
    while ((1ll << l) < d) ++l;
    return Divisor{(uint32_t)((((1ull << l) - (uint64_t)d) << 32) / (uint64_t)d + 1), l < 1 ? l : 1, l < 1 ? 0 : l - 1};
  }
  __device__ __forceinline__ int divide(int n) const {
    const uint32_t t = __umulhi(m, (uint32_t)n);
    return (int)((t + (((uint32_t)n - t) >> s1)) >> s2);
  }
};

// The paged cache (layout: evo.h).  All pages of one head are page_size slots;
// page_size is 1 << page_shift.
struct CacheView {
  void* k;
  void* v;
  float* ks;
  float* vs;
  int n_pages, page_shift, n_kv_heads;
};

// Which rows belong to which sequence; cu == NULL: max_rows each.
struct RowsView {
  const int32_t* cu;
  const int32_t* pages;   // [n_seqs][max_pages]
  int n_seqs, n_rows, max_rows, max_pages;
  Divisor by_max_rows;    // without cu
};

struct HeadsView {
  char* p;
  int64_t row, head;      // strides in elements
};

// One launch over rows: norm and rotation of q and k, k and v into the cache.
struct RowsArgs {
  HeadsView q, k, v, qo, ko;  // ko: keys that do not go to the cache
  int n_heads, n_kv_heads;
  int head_groups;            // workgroups that share a token's heads
  int heads_by_rows;          // heads that go a group of lanes a row: q, k, and v of short calls
  int norm, half, adjacent, n_positions;
  float eps;
  const float* q_gain;
  const float* k_gain;
  const float* table;
  const int32_t* positions;   // NULL: the positions that are written
  const int32_t* starts;
  CacheView cache;
  RowsView rows;
  int wide;                   // every row 16-byte aligned
  int qk_blocks;              // workgroups of the q and k part
  Divisor by_groups, by_kv_heads;
};

// format: EVO_CACHE_*, or -1 with no cache (keys to ko).  dtype: EVO_FP32 / EVO_BF16.
hipError_t launch_rows(int dtype, int format, int head_dim, RowsArgs a, hipStream_t stream);
hipError_t launch_cache_read(int dtype, int format, int head_dim, RowsArgs a, hipStream_t stream);

struct AttArgs {
  HeadsView q, out;
  float* lse;                 // [n_rows][n_heads] or NULL
  CacheView cache;
  RowsView rows;
  const int32_t* lengths;
  const int32_t* starts;      // NULL: lengths - rows
  const int32_t* prefix;      // or NULL
  const float* slopes;        // or NULL
  int n_heads, group;         // group: query heads per key/value head
  int causal, window;
  float scale, cap, inv_cap;  // inv_cap: 0 with no cap
  int wide;                   // rows of q and out 16-byte aligned
  // plan
  int tiles_per_seq;          // 0: a sequence's tiles start at row / tile + sequence
  int n_tiles;                // row tiles over all sequences
  int n_split;                // parts of the keys
  Divisor by_group, by_kv_heads, by_tiles, by_eight, by_split;  // (by_eight: 8 sequences' tiles)
  float* part;                // [n_tiles][n_kv_heads][n_split][tile rows][head_dim] unnormalised outputs
  float* part_ml;             // [n_tiles][n_kv_heads][n_split][tile rows][2]: maximum (log2), sum
  unsigned long long* flags;  // [n_tiles][n_kv_heads][n_split]: `number` where a part is written
  unsigned long long number;  // of this call
};

struct AttPlan {
  int tile_rows, tiles_per_seq, n_tiles, n_split, waves;
  int64_t part_floats, ml_floats, flags;
  bool rest;  // terms of 16 significant bits
};

AttPlan plan_attention(int dtype, int format, int head_dim, int n_heads, int n_kv_heads, const RowsView& r,
                       int max_length, int n_cu);
hipError_t launch_attention(int dtype, int format, int head_dim, const AttPlan& plan, const AttArgs& a,
                            hipStream_t stream);

// The sequence of row n and the row's place in it.
__device__ __forceinline__ void find_row(const RowsView& r, int n, int* seq, int* i) {
  if (!r.cu) {
    const int s = r.by_max_rows.divide(n);
    *seq = s;
    *i = n - s * r.max_rows;
    return;
  }
  int lo = 0, hi = r.n_seqs;  // the last sequence that starts at or before n
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (r.cu[mid] <= n) lo = mid;
    else hi = mid;
  }
  *seq = lo;
  *i = n - r.cu[lo];
}

// The page of a position that lies below max_pages << page_shift.
__device__ __forceinline__ int page_of(const RowsView& r, const CacheView& c, int seq, int page_index) {
  const unsigned pg = (unsigned)r.pages[(int64_t)seq * r.max_pages + page_index];
  return (int)min(pg, (unsigned)(c.n_pages - 1));
}

}  // namespace evo
