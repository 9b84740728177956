// Attention of a chunk of new tokens over the paged cache of keys and values,
// with the softmax's running maximum and sum, in one pass over the cache.
//
// A workgroup takes a tile of 16 R rows (tokens x the query heads that share a
// key/value head) and a part of the keys; its one, four or eight waves take blocks of
// 64 keys in turn and join at the end.  Products are formed transposed, S^T = K
// Q^T and O^T = V^T P^T:
//  * a lane of the first product's result holds one row's scores, so scaling,
//    masks and the running maximum and sum are lane-local, apart from two
//    exchanges over the four lane groups that share a row;
//  * the keys of a block are dealt to the matrix rows in the order (key_of)
//    that leaves each lane with the run of keys that the second product wants
//    from it, so scores become its operand without leaving the lane;
//  * with transposed value pages every operand of K and V is a 16-byte load
//    from memory to registers: nothing but scales goes through LDS in the loop.
// The next block's keys are requested when the first product has taken this
// block's, the next values when the second has.
//
// What bounds it: memory for single tokens (6 over 65001 bf16 positions, 32 heads
// over 8 of 128: 179 us, 5.3 TB/s), waiting and the vector units for chunks over
// 8-bit caches (128 of 32 tokens over 1100 fp8 positions, capped: 44 us; conversions
// and softmax keep the vector units busy for 25 of them, and the 2 waves that a
// SIMD holds on average wait for 40% of their time), latencies for small calls
// (one token over 1000: 8.6 us).
// Longer chunks of more rows share keys and values through LDS (tile_kernel).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "evo.h"
#include "evo_memory.hpp"

namespace evo {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kKeys = 64;     // keys of a block
constexpr int kWaves = 4;
// Least blocks of a part of the keys, for so many workgroups without parts.  A
// part costs its join, which pays where few of the compute units would work: one
// token over 1000 positions (4 workgroups) takes 8.6, 10.9
// and 11.7 us with parts of 4, 8 and 16, over 4000 10.1, 11.4 and 16.5; 24 chunks
// of 16 fp32 rows over 2500 (96) 29.4, 27.0 and 30.8; 32 chunks over 1500 int8
// positions (128) 11.4, 11.2 and 10.4, 64 (256) 15.6 with 8 and 11.7 with 16.
constexpr int part_blocks(int64_t wgs, int n_cu) { return 4 * wgs <= n_cu ? 4 : 2 * wgs < n_cu ? 8 : 16; }
constexpr int kRing = 6;      // operands of a long chunk's products on their way from LDS
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

constexpr int size_of(int f) { return f == EVO_CACHE_FP32 ? 4 : f == EVO_CACHE_BF16 ? 2 : 1; }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Terms are exp2(d), d = x * factor - maximum with the product and the difference
// rounded as one.  The maximum is a rounded product: from 2^24 on it may lie
// whole powers of 2 off the unrounded one, from 2^31 on far enough for terms of 0
// or infinity.  There d is made a difference of rounded products; it is asked for
// where the maximum moves, which costs nothing between (a comparison in every
// block: 2000 causal tokens of 8 sequences, heads of 64, 112 us, so 110).
__device__ __forceinline__ bool is_coarse(float maximum) {
  return __any(fabsf(maximum) >= 0x1p24f && maximum > -kInf);
}
// (maximum: 0 in place of -infinity, of rows that have seen nothing)
__device__ __forceinline__ float coarse_difference(float d, float maximum) {
  const float x = (d + maximum) - maximum;
  return x > 0.f ? 0.f : x;  // (a NaN stays)
}

// The maximum of a row whose scores reach `top`, found for all rows of a wave where
// one outgrows its own.  Over fp4 caches a row that does not keeps its maximum (and a
// maximum that is not coarse its differences), so that no bit of its result depends on
// the rows beside it; the other formats' rows all move.
template <int F> __device__ __forceinline__ float next_maximum(float m, float top) {
  return F == EVO_CACHE_FP4 && top <= m ? m : fmaxf(m, top + 8.f);
}
template <int F> __device__ __forceinline__ float coarse_of_row(float d, float maximum) {
  return F == EVO_CACHE_FP4 && !(fabsf(maximum) >= 0x1p24f) ? d : coarse_difference(d, maximum);
}

// maximum / sum over the four lanes lane % 16 of a wave
__device__ __forceinline__ float over_groups(float x, bool maximum) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float a0 = __builtin_bit_cast(float, (uint32_t)a[0]), a1 = __builtin_bit_cast(float, (uint32_t)a[1]);
  const float y = maximum ? fmaxf(a0, a1) : a0 + a1;
  const uint32_t w = __builtin_bit_cast(uint32_t, y);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  const float b0 = __builtin_bit_cast(float, (uint32_t)b[0]), b1 = __builtin_bit_cast(float, (uint32_t)b[1]);
  return maximum ? fmaxf(b0, b1) : b0 + b1;
}

// two codes of fp4 (byte S of a dword), exact in either type
template <int S> __device__ __forceinline__ uint32_t fp4_bf16(uint32_t v) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 1.f, S));
}
// A dword of a value row in fp4: channels 2 c and 2 c + 1 of 4 keys.  The matrix
// instruction wants neighbouring keys of one channel: half bytes are exchanged
// while they are codes, two operations a channel, which leaves pairs of keys in
// bytes 0 and 2.
// (one instruction, which the compiler does not make of these masks: 128 chunks of 32
// tokens over 1100 positions 38.9 us, else 40.2)
__device__ __forceinline__ uint32_t select_bits(uint32_t mask, uint32_t a, uint32_t b) {
  uint32_t x;
  asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(x) : "s"(mask), "v"(a), "v"(b));
  return x;
}
__device__ __forceinline__ uint32_t even_channel(uint32_t v) { return select_bits(0x000f000fu, v, v >> 4); }
__device__ __forceinline__ uint32_t odd_channel(uint32_t v) { return select_bits(0x000f000fu, v >> 4, v >> 8); }
__device__ __forceinline__ u32x2 channel_bf16(uint32_t v) { return u32x2{fp4_bf16<0>(v), fp4_bf16<2>(v)}; }
// eight codes of fp4 side by side
__device__ __forceinline__ u32x4 row_bf16(uint32_t v) {
  return u32x4{fp4_bf16<0>(v), fp4_bf16<1>(v), fp4_bf16<2>(v), fp4_bf16<3>(v)};
}

// four codes to bf16 (exact: codes have at most 8 significant bits)
template <int F> __device__ __forceinline__ u32x2 codes_bf16(uint32_t v) {
  if (F == EVO_CACHE_FP8)
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, true))};
  return u32x2{pack2((float)(int8_t)v, (float)(int8_t)(v >> 8)), pack2((float)(int8_t)(v >> 16), (float)(int8_t)(v >> 24))};
}
template <int F> __device__ __forceinline__ float code_f32(uint32_t v, int e) {
  if (F == EVO_CACHE_FP4) {
    const auto a = e < 2   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 0)
                   : e < 4 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 1)
                   : e < 6 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 2)
                           : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.f, 3);
    return a[e & 1];
  }
  if (F == EVO_CACHE_FP8) {
    const auto a = e < 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(v, false) : __builtin_amdgcn_cvt_pk_f32_fp8(v, true);
    return a[e & 1];
  }
  return (float)(int8_t)(v >> (8 * e));
}

// How a lane's share of a block lies, by format.  E: consecutive values of a
// key row per load; KG: consecutive keys per load of a value row.  (fp4: a value
// row of the cache is that of two channels, a byte a key.)
template <int F, int DH> struct Lay {
  static constexpr int SZ = size_of(F), PB = per_byte(F);
  static constexpr int E = 16 * PB / SZ < DH / 4 ? 16 * PB / SZ : DH / 4;
  static constexpr int EB = E * SZ / PB;         // bytes of a load of a key row
  static constexpr int KL = DH / (4 * E);        // loads of a key row
  static constexpr int KB = DH * SZ / PB;        // bytes of a key row
  static constexpr int KW = KB / 16;             // dwords of a key row
  static constexpr int KG = 16 / SZ;
  static constexpr int VL = 16 / KG;             // loads of a value row (16 keys)
  static constexpr int VW = 4 * SZ;              // dwords of a value row
  static constexpr int CT = DH / 16;             // tiles of channels
  static constexpr int VT = CT / PB;             // tiles of value rows
  // The first of the four channels that a lane has of tile c.  fp4: tiles 2 i
  // and 2 i + 1 are the even and the odd channels of 32, and are dealt into runs
  // of four (in_runs) after the last block.
  __device__ static constexpr int channel(int c, int g) {
    return PB == 2 ? (c & ~1) * 16 + g * 8 + (c & 1) * 4 : c * 16 + g * 4;
  }
  // the key (in its block) of row 4 g + i of score tile t
  __device__ static constexpr int key_of(int t, int g, int i) {
    constexpr int U = KG / 4;
    return (t / U) * (4 * KG) + g * KG + (t % U) * 4 + i;
  }
};

// The row tile, key/value head and part of the keys of a workgroup.  The tiles
// of a sequence read the same keys: they lie 8 workgroups apart, which puts
// them on one die (workgroup i runs on die i % 8) and its cache; the last, which
// sees most, comes first.
__device__ __forceinline__ bool find_unit(const AttArgs& a, int block, int* tile, int* h, int* split) {
  int unit = block, j = 0;
  if (a.tiles_per_seq > 1) {
    const int eight = a.by_eight.divide(block), rest = block - eight * 8 * a.tiles_per_seq;
    unit = eight * 8 + (rest & 7);
    j = a.tiles_per_seq - 1 - (rest >> 3);
  }
  const int th = a.by_split.divide(unit);
  *split = unit - th * a.n_split;
  *tile = a.by_kv_heads.divide(th);
  *h = th - *tile * a.cache.n_kv_heads;
  if (a.tiles_per_seq > 1) {
    if (*tile >= a.rows.n_seqs) return false;
    *tile = *tile * a.tiles_per_seq + j;
  }
  return true;
}

// A row tile.  Positions of rows lie from -2^30 to below 2^31 - 1, the others and
// the window from 0 to 2^30: sums and differences below stay in 32 bits in the
// order that they are written in.
struct Where {
  int row0, rows, base, p_first, p_last, ctx, start, prefix;
};
constexpr int kFar = 1 << 30;

// The first row of a sequence, inside the call's rows whatever cu_rows holds.
__device__ __forceinline__ int first_row(const RowsView& r, int seq) { return min(max(r.cu[seq], 0), r.n_rows); }

// The row tile of a workgroup; false if it has no rows.
__device__ __forceinline__ bool find_tile(const AttArgs& a, int tile, int tile_rows, int* seq_out, Where* w) {
  int seq, j;
  if (a.tiles_per_seq) {
    seq = a.by_tiles.divide(tile);
    j = tile - seq * a.tiles_per_seq;
  } else {
    int lo = 0, hi = a.rows.n_seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first_row(a.rows, mid) * a.group / tile_rows + mid <= tile) lo = mid;
      else hi = mid;
    }
    seq = lo;
    j = tile - (first_row(a.rows, lo) * a.group / tile_rows + lo);
  }
  int r0, n;
  if (a.rows.cu) {
    r0 = first_row(a.rows, seq);
    n = min(min(max(a.rows.cu[seq + 1], r0), a.rows.n_rows) - r0, a.rows.max_rows);
  } else {
    r0 = seq * a.rows.max_rows;
    n = a.rows.max_rows;
  }
  if (j < 0 || j * tile_rows >= n * a.group) return false;
  w->row0 = r0;
  w->rows = n * a.group;
  w->base = j * tile_rows;
  w->ctx = min(max(a.lengths[seq], 0), a.rows.max_pages << a.cache.page_shift);
  w->start = a.starts ? min(max(a.starts[seq], -kFar), kFar) : w->ctx - n;
  w->prefix = a.prefix ? min(max(a.prefix[seq], 0), w->ctx) : 0;
  w->p_first = w->start + a.by_group.divide(w->base);
  w->p_last = w->start + a.by_group.divide(min(w->base + tile_rows, w->rows) - 1);
  *seq_out = seq;
  return true;
}

// The blocks that some row of the tile sees: the prefix's, then lo .. hi - 1.
struct Blocks {
  int n_prefix, lo, count;
  __device__ int at(int v) const { return v < n_prefix ? v : v - n_prefix + lo; }
};
__device__ __forceinline__ Blocks blocks_of(const AttArgs& a, const Where& w) {
  int hi = w.ctx, lo = 0;
  if (a.causal) hi = min(hi, w.p_last + 1);
  if (a.window) {
    hi = min(hi, min(w.p_last, w.ctx - a.window) + a.window);
    lo = max(0, w.p_first - a.window + 1);
  }
  Blocks b;
  b.n_prefix = (w.prefix + kKeys - 1) / kKeys;
  b.lo = max(lo / kKeys, b.n_prefix);
  b.count = b.n_prefix + (hi > lo ? max(0, (hi + kKeys - 1) / kKeys - b.lo) : 0);
  return b;
}

// The pages of 64 of the blocks v, v + step, .. that a wave comes to: a lane
// holds one, so that no block's load waits for its page's number first.
struct Pages {
  int held;
  __device__ __forceinline__ void load(const AttArgs& a, const Blocks& bl, int seq, int v, int step) {
    const int at = min(v + (int)(threadIdx.x & 63) * step, max(bl.count - 1, 0));
    held = bl.count ? page_of(a.rows, a.cache, seq, (bl.at(at) * kKeys) >> a.cache.page_shift) : 0;
  }
  __device__ __forceinline__ int at(int i) const { return __builtin_amdgcn_readlane(held, i & 63); }
};

// |p - j|, also of a key past the cache's end (without a value that matters)
__device__ __forceinline__ float distance(int p, int j) { return fabsf((float)(int)((unsigned)p - (unsigned)j)); }
__device__ __forceinline__ bool sees(const AttArgs& a, const Where& w, int p, int j) {
  const bool near = (!a.causal || j <= p) && (!a.window || abs(p - j) < a.window);
  return j < w.ctx && (j < w.prefix || near);
}
// The same as a run of positions and the prefix, found once for a row: two
// comparisons a key instead of some ten operations.
struct Seen {
  int lo;
  unsigned span;
  int prefix;
  __device__ __forceinline__ Seen(const AttArgs& a, const Where& w, int p) {
    lo = 0;
    int hi = w.ctx;
    if (a.causal) hi = min(hi, p + 1);
    if (a.window) {
      hi = min(hi, min(p, w.ctx - a.window) + a.window);
      lo = max(0, p - a.window + 1);
    }
    span = (unsigned)max(hi - lo, 0);
    prefix = w.prefix;
  }
  __device__ __forceinline__ bool at(int j) const { return (unsigned)(j - lo) < span || j < prefix; }
};
// Which blocks (by their first key) some row of a tile sees, and which all of
// its rows see whole.
struct Sight {
  int any_lo, any_hi, all_lo, all_hi, prefix;
  __device__ __forceinline__ void set(const AttArgs& a, const Where& w) {
    any_lo = all_lo = -kFar;
    any_hi = kFar;
    all_hi = w.ctx - 1;
    if (a.causal) {
      any_hi = w.p_last;
      all_hi = min(all_hi, w.p_first);
    }
    if (a.window) {
      any_hi = min(any_hi, min(w.p_last, kFar) + (a.window - 1));
      any_lo = max(w.p_first, -1) - a.window + 2 - kKeys;
      all_hi = min(all_hi, min(w.p_first, kFar) + (a.window - 1));
      all_lo = w.p_last - a.window + 1;
    }
    all_hi -= kKeys - 1;
    prefix = w.prefix;
  }
  __device__ __forceinline__ bool any(int kb) const { return (kb >= any_lo && kb <= any_hi) || kb < prefix; }
  __device__ __forceinline__ bool all(int kb) const { return (kb >= all_lo && kb <= all_hi) || kb + kKeys <= prefix; }
};

// tanh from one exponential.  Its error is absolute, up to 2^-22, so a capped
// score is off by up to 2^-22 of the cap however small the score is: behind bf16
// products it is used up to caps of kFastCap, where that is 1.5e-5, and the terms'
// rounding to bf16 is 256 times as much.
constexpr float kFastCap = 64.f;
__device__ __forceinline__ float squash_fast(float x) {
  return 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + exp2_(x * (2.f * kLog2e)));
}
// tanh with an error relative to itself: above kFastCap, where scores may be far
// smaller than the cap.  Near 0 an odd polynomial (Chebyshev interpolation of
// (tanh(x) / x - 1) / x^2 in x^2, off by 1.6 * 2^-24).
template <typename T> __device__ __forceinline__ float squash(float x);
template <> __device__ __forceinline__ float squash<__bf16>(float x) {
  const float y = x * x;
  const float near = fmaf(x * y, fmaf(fmaf(fmaf(0.01799922f, y, -0.05339105f), y, 0.13330514f), y, -0.33333312f), x);
  return fabsf(x) < 0.5f ? near : squash_fast(x);
}
template <> __device__ __forceinline__ float squash<float>(float x) { return tanhf(x); }

template <typename T, int DH> struct Query;
template <int DH> struct Query<__bf16, DH> {
  bf16x8 f[DH / 32];
  __device__ __forceinline__ void negate() {
#pragma unroll
    for (int k = 0; k < DH / 32; ++k) f[k] = -f[k];
  }
};
template <int DH> struct Query<float, DH> {
  float f[DH / 4];
  __device__ __forceinline__ void negate() {
#pragma unroll
    for (int k = 0; k < DH / 4; ++k) f[k] = -f[k];
  }
};

// This lane's share of a query row, in the order of the key loads.
template <int F, int DH>
__device__ __forceinline__ void load_query(Query<__bf16, DH>& q, const __bf16* p, int g, int wide) {
  typedef Lay<F, DH> L;
#pragma unroll
  for (int k = 0; k < DH / 32; ++k) {
    const __bf16* s = p + (k / (L::E / 8)) * (4 * L::E) + g * L::E + (k % (L::E / 8)) * 8;
    if (wide) q.f[k] = *reinterpret_cast<const bf16x8*>(s);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) q.f[k][e] = s[e];
  }
}
template <int F, int DH>
__device__ __forceinline__ void load_query(Query<float, DH>& q, const float* p, int g, int wide) {
  typedef Lay<F, DH> L;
#pragma unroll
  for (int l = 0; l < L::KL; ++l)
#pragma unroll
    for (int e = 0; e < L::E; ++e) q.f[l * L::E + e] = p[l * 4 * L::E + g * L::E + e];
}

// S^T += K Q^T for one tile of 16 keys
template <int F, int DH>
__device__ __forceinline__ f32x4 score_tile(const uint32_t* k, const Query<__bf16, DH>& q) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < DH / 32; ++j) {
    u32x4 w;
    if constexpr (F == EVO_CACHE_FP4) {
      w = row_bf16(k[j]);
    } else if constexpr (is_coded(F)) {
      const u32x2 a = codes_bf16<F>(k[2 * j]), b = codes_bf16<F>(k[2 * j + 1]);
      w = u32x4{a[0], a[1], b[0], b[1]};
    } else {
      w = u32x4{k[4 * j], k[4 * j + 1], k[4 * j + 2], k[4 * j + 3]};
    }
    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), q.f[j], s, 0, 0, 0);
  }
  return s;
}
template <int F, int DH>
__device__ __forceinline__ f32x4 score_tile(const uint32_t* k, const Query<float, DH>& q) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < DH / 4; ++j) {
    float x;
    if constexpr (F == EVO_CACHE_FP4) x = code_f32<F>(k[j / 8], j & 7);
    else if constexpr (is_coded(F)) x = code_f32<F>(k[j / 4], j & 3);
    else x = __builtin_bit_cast(float, k[j]);
    s = __builtin_amdgcn_mfma_f32_16x16x4f32(x, q.f[j], s, 0, 0, 0);
  }
  return s;
}

// The second product's operand made of a row's 16 terms of a block.
template <typename T> struct Terms;
template <> struct Terms<__bf16> {
  bf16x8 f[2];
  __device__ __forceinline__ float at(int t, int i) const { return (float)f[t / 2][t % 2 * 4 + i]; }
  __device__ __forceinline__ void set(const float (&p)[4][4]) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const u32x4 w = {pack2(p[2 * s][0], p[2 * s][1]), pack2(p[2 * s][2], p[2 * s][3]),
                       pack2(p[2 * s + 1][0], p[2 * s + 1][1]), pack2(p[2 * s + 1][2], p[2 * s + 1][3])};
      f[s] = __builtin_bit_cast(bf16x8, w);
    }
  }
};
template <> struct Terms<float> {
  float f[4][4];
  __device__ __forceinline__ float at(int t, int i) const { return f[t][i]; }
  __device__ __forceinline__ void set(const float (&p)[4][4]) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) f[t][i] = p[t][i];
  }
};

// O^T += V^T P^T for one tile of 16 channels
template <int F>
__device__ __forceinline__ f32x4 value_tile(const uint32_t* v, const Terms<__bf16>& p, f32x4 o) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    u32x4 w;
    if constexpr (is_coded(F)) {
      const u32x2 a = codes_bf16<F>(v[2 * s]), b = codes_bf16<F>(v[2 * s + 1]);
      w = u32x4{a[0], a[1], b[0], b[1]};
    } else {
      w = u32x4{v[4 * s], v[4 * s + 1], v[4 * s + 2], v[4 * s + 3]};
    }
    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), p.f[s], o, 0, 0, 0);
  }
  return o;
}
template <int F>
__device__ __forceinline__ f32x4 value_tile(const uint32_t* v, const Terms<float>& p, f32x4 o) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x;
      if constexpr (is_coded(F)) x = code_f32<F>(v[t], i);
      else x = __builtin_bit_cast(float, v[4 * t + i]);
      o = __builtin_amdgcn_mfma_f32_16x16x4f32(x, p.f[t][i], o, 0, 0, 0);
    }
  return o;
}

// The same for the two tiles of a tile of fp4 value rows.  REST: also for what the
// terms' rounding left.
template <bool REST>
__device__ __forceinline__ void value_tiles(const uint32_t* v, const Terms<__bf16>& p, const Terms<__bf16>& rest, f32x4* o) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint32_t a = v[2 * s], b = v[2 * s + 1];
    const u32x2 e0 = channel_bf16(even_channel(a)), e1 = channel_bf16(even_channel(b));
    const u32x2 d0 = channel_bf16(odd_channel(a)), d1 = channel_bf16(odd_channel(b));
    const bf16x8 e = __builtin_bit_cast(bf16x8, u32x4{e0[0], e0[1], e1[0], e1[1]});
    const bf16x8 d = __builtin_bit_cast(bf16x8, u32x4{d0[0], d0[1], d1[0], d1[1]});
    o[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e, p.f[s], o[0], 0, 0, 0);
    o[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(d, p.f[s], o[1], 0, 0, 0);
    if constexpr (REST) {
      o[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e, rest.f[s], o[0], 0, 0, 0);
      o[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(d, rest.f[s], o[1], 0, 0, 0);
    }
  }
}
template <bool REST>
__device__ __forceinline__ void value_tiles(const uint32_t* v, const Terms<float>& p, const Terms<float>&, f32x4* o) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(code_f32<EVO_CACHE_FP4>(v[t], 2 * i + c), p.f[t][i], o[c], 0, 0, 0);
}
// Even and odd channels of 32, four a lane, to eight of them side by side.
__device__ __forceinline__ void in_runs(f32x4* o) {
  const f32x4 e = o[0], d = o[1];
  o[0] = f32x4{e[0], d[0], e[1], d[1]};
  o[1] = f32x4{e[2], d[2], e[3], d[3]};
}

// Values that hold a NaN or an infinity set to 0 (int8 and fp4 codes hold none; a cache
// that was written holds no NaN codes of fp8, unwritten memory may).
template <int F> __device__ __forceinline__ uint32_t finite_only(uint32_t x) {
  if constexpr (F == EVO_CACHE_FP32) return (x & 0x7f800000u) == 0x7f800000u ? 0 : x;
  if constexpr (F == EVO_CACHE_BF16) {
    if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
    if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
  }
  if constexpr (F == EVO_CACHE_FP8) {
    // 0x80 in the bytes that are 0x7f or 0xff; times 255: the whole byte
    const uint32_t nan = ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    x &= ~((nan >> 7) * 255u);
  }
  return x;
}
// The value at an index if it is a NaN or an infinity, else 0.
template <int F> __device__ __forceinline__ float not_finite(const void* v, int64_t at) {
  uint32_t x;
  if constexpr (F == EVO_CACHE_FP32) x = reinterpret_cast<const uint32_t*>(v)[at];
  else if constexpr (F == EVO_CACHE_BF16) x = (uint32_t)reinterpret_cast<const uint16_t*>(v)[at] << 16;
  else x = (reinterpret_cast<const uint8_t*>(v)[at] & 0x7f) == 0x7f ? 0x7fc00000u : 0;
  return (x & 0x7f800000u) == 0x7f800000u ? __builtin_bit_cast(float, x) : 0.f;
}

// Whether a lane's values hold a NaN or an infinity, in two or three operations
// a dword: most masked blocks hold none, and then terms of 0 are enough.
template <int F, int CT, int VW> __device__ __forceinline__ bool any_not_finite(const uint32_t (&v)[CT][VW]) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  uint32_t top = 0;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      const uint32_t x = v[c][i];
      if constexpr (F == EVO_CACHE_FP32) top = max(top, x & 0x7fffffffu);
      if constexpr (F == EVO_CACHE_BF16)
        top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, x & 0x7fff7fffu)));
      if constexpr (F == EVO_CACHE_FP8) top |= (x & 0x7f7f7f7fu) + 0x01010101u;
    }
  if constexpr (F == EVO_CACHE_FP32) return top >= 0x7f800000u;
  if constexpr (F == EVO_CACHE_BF16) return top >= 0x7f800000u || (top & 0xffffu) >= 0x7f80u;
  if constexpr (F == EVO_CACHE_FP8) return top & 0x80808080u;
  return false;
}

// A masked block's values: keys past the cache's length become 0 (a page's
// unused end may hold anything), NaNs and infinities too; returns whether
// there were any.
template <int F, int DH, int CT, int VW>
__device__ __forceinline__ bool clear_tail(uint32_t (&v)[CT][VW], int g, int left) {
  typedef Lay<F, DH> L;
  static_assert(CT == L::CT && VW == L::VW, "a lane's values of a block");
  bool bad = false;
#pragma unroll
  for (int l = 0; l < L::VL; ++l)
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int key = l * (4 * L::KG) + g * L::KG + d * (4 / L::SZ);  // first key of the dword
      uint32_t keep = 0;
#pragma unroll
      for (int e = 0; e < 4 / L::SZ; ++e)
        if (key + e < left) keep |= (L::SZ == 4 ? 0xffffffffu : ((1u << (8 * L::SZ)) - 1) << (8 * L::SZ * e));
#pragma unroll
      for (int c = 0; c < L::CT; ++c) {
        uint32_t& x = v[c][l * 4 + d];
        x &= keep;
        if constexpr (F != EVO_CACHE_INT8) {
          const uint32_t y = finite_only<F>(x);
          bad |= y != x;
          x = y;
        }
      }
    }
  return bad;
}

template <typename T> __device__ __forceinline__ void store4(T* p, int wide, f32x4 x) {
  if (sizeof(T) == 4) {
    if (wide) *reinterpret_cast<f32x4*>(p) = x;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = (T)x[e];
  } else {
    if (wide) *reinterpret_cast<u32x2*>(p) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = (T)x[e];
  }
}

// Parts that another workgroup of the launch reads: loads and stores that go
// past a die's cache (cache policy bit SC1), each die having its own.  Cheaper
// by far than ordinary ones between fences, which write back and empty the
// whole cache: 16 chunks of 16 tokens over 2500 fp8 positions took 51 us so.
constexpr int kCoherent = 16;
struct Parts {
  __amdgpu_buffer_rsrc_t o;  // [n_split][tile_rows][head_dim] of one tile and key/value head
  unsigned long long* ml;
  template <int DH> __device__ __forceinline__ static Parts of(const AttArgs& a, int th, int tile_rows) {
    const int64_t first = (int64_t)th * a.n_split * tile_rows;
    return Parts{__builtin_amdgcn_make_buffer_rsrc(a.part + first * DH, (short)0, a.n_split * tile_rows * DH * 4, 0x00020000),
                 reinterpret_cast<unsigned long long*>(a.part_ml + first * 2)};
  }
};
// The wave's stores so far have landed, and nothing after this has begun.
__device__ __forceinline__ void stores_landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  asm volatile("" ::: "memory");
}

// Joins the parts of four channels of a row, in order; eight parts are
// requested at a time, since a part's load is all latency.
template <typename T, int DH>
__device__ __forceinline__ void join_parts(const AttArgs& a, const Where& wh, int th, int h, int tile_rows, int r, int c) {
  constexpr int AT = 8;
  const int row = wh.base + r;
  const Parts parts = Parts::of<DH>(a, th, tile_rows);
  float M = -kInf, t = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.n_split; s0 += AT) {
    float m[AT], l[AT];
    f32x4 v[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int at = min(s0 + i, a.n_split - 1) * tile_rows + r;
      const unsigned long long ml = __hip_atomic_load(parts.ml + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      m[i] = __builtin_bit_cast(float, (uint32_t)ml);
      l[i] = s0 + i < a.n_split ? __builtin_bit_cast(float, (uint32_t)(ml >> 32)) : 0.f;
      v[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(parts.o, (at * DH + c) * 4, 0, kCoherent));
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < AT; ++i) top = fmaxf(top, m[i]);
    const float base = top == -kInf ? 0.f : top, keep = exp2_(M - base);
    M = top;
    t *= keep;
    o *= keep;
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const float f = exp2_(m[i] - base);
      if (l[i] == 0.f) continue;  // (a part that saw nothing wrote no outputs)
      t += l[i] * f;
      o += v[i] * f;
    }
  }
  const int tok = a.by_group.divide(row), head = h * a.group + row - tok * a.group;
  T* dst = reinterpret_cast<T*>(a.out.p) + (wh.row0 + tok) * a.out.row + head * a.out.head;
  store4(dst + c, a.wide, t == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.f / t));
  if (a.lse && c == 0)
    a.lse[(int64_t)(wh.row0 + tok) * a.n_heads + head] = t == 0.f ? -kInf : (M + __builtin_amdgcn_logf(t)) * kLn2;
}

// Whether all parts of a row tile are written, asked by the wave that has
// written its own.  A part's flag is set to the call's number, which no other
// call of the process has, so that flags need no clearing before; whoever finds
// all set clears them, for a call that is recorded once and replayed.  A flag is
// set once the part has landed, and the others are read once the flag has: the
// writer of the flag that lands last finds all.  Should another find them all
// too, both join the same parts to the same results.  Nobody waits.
__device__ __forceinline__ bool parts_complete(const AttArgs& a, int th, int split) {
  const int lane = threadIdx.x & 63;
  unsigned long long* flags = a.flags + (int64_t)th * a.n_split;
  stores_landed();
  if (lane == 0) __hip_atomic_store(flags + split, a.number, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  stores_landed();
  bool all = true;
  for (int i = lane; i < a.n_split; i += 64)
    all &= __hip_atomic_load(flags + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.number;
  if (!__all(all)) return false;
  for (int i = lane; i < a.n_split; i += 64)
    __hip_atomic_store(flags + i, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

// Workgroup (row tile, key/value head, part of the keys).
// Waves that a SIMD shall hold: what the registers of a wave's block allow.
template <typename T> constexpr int waves_per_simd(int f, int dh, int r, int nw) {
  if (nw == 8) return 2;
  if (sizeof(T) == 4) return dh == 128 || (dh == 64 && r == 2) ? 1 : 2;
  return dh == 128 && f == EVO_CACHE_BF16 ? 1 : r == 2 || dh == 128 ? 2 : 3;
}

// PARTS: the keys are split over workgroups (of its own, because the join's
// code costs the others registers: 32-token chunks over fp8 memories 47 us with
// it and 45 without).
// REST (bf16 over fp4): what the terms' rounding to bf16 leaves is the operand of a
// second product.  Where few keys carry a row, the rounded value scale of one is the error
// of all its outputs: up to 0.0030 without it, 0.0017 with it as a result rounded once.  It
// goes by the rows and positions of a sequence, so that a row's bits do not go by how many
// others share its call: single tokens (one over 1000 positions 7.5 us, else 7.4; 6 over up to
// 65001 54.0, else 52.4; 128 over 2000 38, else 34), and a block of keys for any rows
// (1600 rows of 84 sequences over 27 positions 130 us with and without).  Other
// calls would pay for it in their vector units (128 chunks of 32 over up to 1100 42.5 us, so
// 38.6; 2000 causal rows of 8 sequences 100, so 91), and are 0.0024 off.
template <typename T, int F, int DH, int R, int NW, bool PARTS, bool REST = false>
__global__ void __launch_bounds__(NW * 64, waves_per_simd<T>(F, DH, R, NW)) stream_kernel(AttArgs a) {
  typedef Lay<F, DH> L;
  constexpr int TR = 16 * R;
  __shared__ __attribute__((aligned(16))) float join_o[NW > 1 ? NW / 2 : 1][NW > 1 ? TR * DH : 4];
  __shared__ float join_ml[NW][TR][2];
  // scales of a wave's block, keys' and values'
  __shared__ __attribute__((aligned(16))) float scales[is_coded(F) ? NW : 1][2][is_coded(F) ? kKeys : 4];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, g = lane >> 4;
  int tile, h, split, seq;
  Where wh;
  if (!find_unit(a, blockIdx.x, &tile, &h, &split) || !find_tile(a, tile, TR, &seq, &wh)) return;
  const int th = tile * a.cache.n_kv_heads + h;
  const Blocks bl = blocks_of(a, wh);
  const int per = PARTS ? max(a.by_split.divide(bl.count + a.n_split - 1), NW) : bl.count;
  const int v0 = PARTS ? split * per : 0, v1 = PARTS ? min(v0 + per, bl.count) : bl.count;
  const int ps = a.cache.page_shift;
  Sight sight;
  sight.set(a, wh);
  Pages pages;
  pages.load(a, bl, seq, v0 + w, NW);

  // Scores in units of log2 are off + mul x, mul > 0, with x the products by
  //   plain: one factor, inside the exponential (codes: with the key's scale)
  //   capped: cap tanh(z / cap) = cap + 2 cap x, x = -1 / (1 + exp(2 z / cap))
  //     (squash_fast, folded into the exponential)
  //   else: everything ahead of it; a cap's own factors one after another, because
  //     scale / cap or cap * log2(e) may leave the range of floats
  const bool capped = sizeof(T) == 2 && a.cap > 0.f && a.cap <= kFastCap && !a.slopes;
  const bool plain = a.cap == 0.f && !a.slopes && a.scale != 0.f;
  const float cap_log2 = a.cap * kLog2e, to_log2 = a.scale * kLog2e;
  // (made in vector registers, of which waves of 16 bf16 rows over parts of the keys
  // have none to spare; over codes they stay there: in scalar ones 128 chunks of
  // 32 tokens over fp8 took 45 us, so 43.5)
  const auto kept = [](float x) {
    return F == EVO_CACHE_BF16 ? __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))) : x;
  };
  const float pre = kept(capped ? 2.f * to_log2 * a.inv_cap : a.cap > 0.f ? a.scale : to_log2);
  const float mul = kept(capped ? 2.f * cap_log2 : plain && !is_coded(F) ? fabsf(to_log2) : 1.f);
  const float off = kept(capped ? cap_log2 : 0.f);
  const bool flip = plain && !is_coded(F) && a.scale < 0.f;

  Query<T, DH> q[R];
  int pos[R];
  float slope[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = min(wh.base + r * 16 + lr, wh.rows - 1), tok = a.by_group.divide(row), head = h * a.group + row - tok * a.group;
    pos[r] = wh.start + tok;
    slope[r] = a.slopes ? a.slopes[head] * kLog2e : 0.f;
    load_query<F, DH>(q[r], reinterpret_cast<const T*>(a.q.p) + (wh.row0 + tok) * a.q.row + head * a.q.head, g, a.wide);
  }
  f32x4 o[R][L::CT];
  float m[R], l[R];
  bool coarse[R];  // of the whole wave: some row's maximum is
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -kInf;
    l[r] = 0.f;
    coarse[r] = false;
#pragma unroll
    for (int c = 0; c < L::CT; ++c) o[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // byte offsets of this lane in a block's keys and values
  const uint32_t koff = (uint32_t)(L::key_of(0, lr >> 2, lr & 3) * L::KB + g * L::EB);
  const uint32_t voff = (uint32_t)(((lr << ps) + g * L::KG) * L::SZ);
  uint32_t kr[4][L::KW], vr[L::VT][L::VW];
  const auto load_keys = [&](int kb, int page) {
    const int slot = kb & ((1 << ps) - 1);
    const int64_t b = (int64_t)page * a.cache.n_kv_heads + h;
    const char* p = reinterpret_cast<const char*>(a.cache.k) + ((b << ps) + slot) * L::KB;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < L::KL; ++i) {
        const char* s = p + koff + (L::key_of(t, 0, 0) * L::KB + i * 4 * L::EB);
        if constexpr (L::EB == 4) {
          kr[t][i] = *reinterpret_cast<const uint32_t*>(s);
        } else if constexpr (L::EB == 16) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(s);
#pragma unroll
          for (int e = 0; e < 4; ++e) kr[t][i * 4 + e] = x[e];
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2*>(s);
          kr[t][i * 2] = x[0];
          kr[t][i * 2 + 1] = x[1];
        }
      }
  };
  const auto load_values = [&](int kb, int page) {
    const int slot = kb & ((1 << ps) - 1);
    const int64_t b = (int64_t)page * a.cache.n_kv_heads + h;
    const char* p = reinterpret_cast<const char*>(a.cache.v) + (((b * (DH / L::PB)) << ps) + slot) * L::SZ;
#pragma unroll
    for (int c = 0; c < L::VT; ++c)
#pragma unroll
      for (int i = 0; i < L::VL; ++i) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p + voff + (((c * 16) << ps) + i * 4 * L::KG) * L::SZ);
#pragma unroll
        for (int e = 0; e < 4; ++e) vr[c][i * 4 + e] = x[e];
      }
  };

  // Scales come a key a lane, a block ahead like the keys, and reach the lanes
  // that want them through LDS: asked for in that order, 16 a lane, they were
  // waited for in every block.
  float k_scale = 0.f, v_scale = 0.f;
  const auto load_scales = [&](int kb, int page) {
    if constexpr (is_coded(F)) {
      const int64_t at = (((int64_t)page * a.cache.n_kv_heads + h) << ps) + (kb & ((1 << ps) - 1)) + lane;
      k_scale = a.cache.ks[at];
      v_scale = a.cache.vs[at];
    }
  };

  int v = v0 + w;
  int page = pages.at(0);
  if (v < v1) {
    load_scales(bl.at(v) * kKeys, page);
    load_keys(bl.at(v) * kKeys, page);
    load_values(bl.at(v) * kKeys, page);
  }
  if (flip) {  // (here: no load waits for the query)
#pragma unroll
    for (int r = 0; r < R; ++r) q[r].negate();
  }
  for (int it = 1; v < v1; v += NW, ++it) {
    const int kb = bl.at(v) * kKeys, next = v + NW < v1 ? bl.at(v + NW) * kKeys : -1;
    const int64_t b = (int64_t)page * a.cache.n_kv_heads + h;
    const int slot = kb & ((1 << ps) - 1);
    if ((it & 63) == 0) pages.load(a, bl, seq, v + NW, NW);
    page = pages.at(it);
    const bool masked = !sight.all(kb);
    if constexpr (is_coded(F)) {
      wave_sync();
      scales[w][0][lane] = k_scale * pre;
      scales[w][1][lane] = v_scale;
      wave_sync();
    }
    const auto scale_of = [&](int which, int t) { return *reinterpret_cast<const f32x4*>(&scales[w][which][L::key_of(t, g, 0)]); };
    f32x4 s[R][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) s[r][t] = score_tile<F, DH>(kr[t], q[r]);
    __builtin_amdgcn_sched_barrier(0);
    if (next >= 0) {
      load_scales(next, page);
      load_keys(next, page);
    }
    __builtin_amdgcn_sched_barrier(0);

    Terms<T> terms[R], rests[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float x[4][4];
      const auto each = [&](auto f) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) f(x[t][i], t, i);
      };
      each([&](float& x, int t, int i) { x = s[r][t][i]; });
      const auto times = [&](int which) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const f32x4 y = scale_of(which, t);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[t][i] *= y[i];
        }
      };
      if constexpr (is_coded(F)) times(0);
      if (capped) {
        each([&](float& x, int, int) { x = __builtin_amdgcn_rcpf(-1.f - exp2_(is_coded(F) ? x : x * pre)); });
      } else if (!plain) {
        if (!is_coded(F)) each([&](float& x, int, int) { x *= pre; });
        if (a.cap > 0.f) each([&](float& x, int, int) { x = a.cap * squash<T>(x * a.inv_cap) * kLog2e; });
        if (a.slopes)
          each([&](float& x, int t, int i) { x = fmaf(-slope[r], distance(pos[r], kb + L::key_of(t, g, i)), x); });
      }
      const Seen seen(a, wh, pos[r]);
      if (masked) each([&](float& x, int t, int i) { x = seen.at(kb + L::key_of(t, g, i)) ? x : -kInf; });
      float top = x[0][0];
      each([&](float& x, int, int) { top = fmaxf(top, x); });
      top = over_groups(fmaf(top, mul, off), true);
      // the maximum is set 2^8 ahead when scores outgrow it: terms are at most 1,
      // so they take no value out of range, and the outputs are seldom rescaled
      if (__any(!(top <= m[r]))) {
        const float m_new = next_maximum<F>(m[r], top);
        const float f = exp2_(m[r] - (m_new == -kInf ? 0.f : m_new));
        m[r] = m_new;
        l[r] *= f;
#pragma unroll
        for (int c = 0; c < L::CT; ++c) o[r][c] *= f;
        if constexpr (!is_coded(F)) coarse[r] = is_coarse(m_new);  // (codes: scaled ahead, the factor is 1)
      }
      const float base = m[r] == -kInf ? 0.f : m[r], shift = off - base;
      float sum = 0.f;
      each([&](float& x, int, int) { x = fmaf(x, mul, shift); });
      if (__builtin_expect(coarse[r], 0)) each([&](float& x, int, int) { x = coarse_difference(x, base); });
      each([&](float& x, int, int) { x = exp2_(x); sum += x; });
      l[r] += sum;
      if constexpr (is_coded(F)) {
        // (an unseen key's scale may be a NaN)
        times(1);
        if (masked) each([&](float& x, int t, int i) { x = seen.at(kb + L::key_of(t, g, i)) ? x : 0.f; });
      }
      terms[r].set(x);
      if constexpr (REST) {
        each([&](float& x, int t, int i) { x -= terms[r].at(t, i); });
        rests[r].set(x);
      }
    }
    bool bad = false;
    if constexpr (holds_nan(F)) {
      if (masked && __any(any_not_finite<F>(vr))) {
        // What a row does not see must not reach it, but 0 times a NaN or an
        // infinity is NaN: those are taken out of the operand, and added below
        // to the rows that see them.
        bad = clear_tail<F, DH>(vr, g, wh.ctx - kb);
      }
    }
#pragma unroll
    for (int c = 0; c < L::VT; ++c)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (F == EVO_CACHE_FP4) value_tiles<REST>(vr[c], terms[r], rests[r], &o[r][2 * c]);
        else o[r][c] = value_tile<F>(vr[c], terms[r], o[r][c]);
      }
    if constexpr (holds_nan(F)) {
      if (__builtin_expect(__any(bad), 0)) {
#pragma unroll 1
        for (int j = 0; j < min(kKeys, wh.ctx - kb); ++j) {
          int64_t at = ((b * DH + 4 * g) << ps) + slot + j;
          asm volatile("" : "+v"(at));  // the addresses are made here, not kept over the loop
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const bool see = sees(a, wh, pos[r], kb + j);
#pragma unroll
            for (int c = 0; c < L::CT; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float x = not_finite<F>(a.cache.v, at + ((c * 16 + e) << ps));
                if (see) o[r][c][e] += x;
                __builtin_amdgcn_sched_barrier(0);
              }
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (next >= 0) load_values(next, page);
    __builtin_amdgcn_sched_barrier(0);
  }

  if constexpr (F == EVO_CACHE_FP4) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < L::CT; c += 2) in_runs(&o[r][c]);
  }

  // ---- the waves' results, in pairs: w and w + NW / 2, then w and w + NW / 4, .. ----
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l[r] = over_groups(l[r], false);
    if (g == 0) {
      join_ml[w][r * 16 + lr][0] = m[r];
      join_ml[w][r * 16 + lr][1] = l[r];
    }
  }
  __syncthreads();
  float total[R], top[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float M = -kInf;
    for (int i = 0; i < NW; ++i) M = fmaxf(M, join_ml[i][r * 16 + lr][0]);
    const float base = M == -kInf ? 0.f : M;
    float t = 0.f;
    for (int i = 0; i < NW; ++i) t += join_ml[i][r * 16 + lr][1] * exp2_(join_ml[i][r * 16 + lr][0] - base);
    total[r] = t;
    top[r] = M;
    const float f = exp2_(m[r] - base);
#pragma unroll
    for (int c = 0; c < L::CT; ++c) o[r][c] *= f;
  }
  const auto put = [&](float* dst) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < L::CT; ++c) *reinterpret_cast<f32x4*>(dst + ((r * L::CT + c) * 64 + lane) * 4) = o[r][c];
  };
  const auto add = [&](const float* src) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < L::CT; ++c) o[r][c] += *reinterpret_cast<const f32x4*>(src + ((r * L::CT + c) * 64 + lane) * 4);
  };
  if constexpr (NW > 1) {
    if (w >= NW / 2) put(join_o[w - NW / 2]);
    __syncthreads();
    if (w < NW / 2) add(join_o[w]);
  }
#pragma unroll
  for (int k = NW / 4; k >= 1; k /= 2) {  // waves k .. 2 k - 1 use the place that they have just read
    if (w >= k && w < 2 * k) put(join_o[w]);
    __syncthreads();
    if (w < k) add(join_o[w + k]);
  }

  if constexpr (PARTS) {
    const Parts parts = Parts::of<DH>(a, th, TR);
    if (w == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (wh.base + r * 16 + lr >= wh.rows) continue;
        const int part = split * TR + r * 16 + lr;
        if (g == 0)
          __hip_atomic_store(parts.ml + part, __builtin_bit_cast(uint32_t, top[r]) | (unsigned long long)__builtin_bit_cast(uint32_t, total[r]) << 32,
                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (v0 < v1) {
          // (the whole offset in a vector register: with a scalar part the wait
          // states before the data's next change are left out)
#pragma unroll
          for (int c = 0; c < L::CT; ++c)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o[r][c]), parts.o, (part * DH + L::channel(c, g)) * 4, 0, kCoherent);
        }
      }
      const bool complete = parts_complete(a, th, split);
      if (lane == 0) join_ml[0][0][0] = complete ? 1.f : 0.f;
    }
    __syncthreads();
    if (join_ml[0][0][0] == 0.f) return;
    for (int x = threadIdx.x; x < min(TR, wh.rows - wh.base) * (DH / 4); x += NW * 64)
      join_parts<T, DH>(a, wh, th, h, TR, x / (DH / 4), x % (DH / 4) * 4);
    return;
  }
  if (w != 0) return;

#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = wh.base + r * 16 + lr;
    if (row >= wh.rows) continue;
    const int tok = a.by_group.divide(row), head = h * a.group + row - tok * a.group;
    const float inv = total[r] == 0.f ? 0.f : 1.f / total[r];
    T* dst = reinterpret_cast<T*>(a.out.p) + (wh.row0 + tok) * a.out.row + head * a.out.head;
#pragma unroll
    for (int c = 0; c < L::CT; ++c)
      store4(dst + L::channel(c, g), a.wide, total[r] == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[r][c] * inv);
    if (a.lse && g == 0)
      a.lse[(int64_t)(wh.row0 + tok) * a.n_heads + head] =
          total[r] == 0.f ? -kInf : (top[r] + __builtin_amdgcn_logf(total[r])) * kLn2;
  }
}

// ---- long chunks ------------------------------------------------------------
// A workgroup takes 32 rows a wave and shares its keys and values through LDS:
// with hundreds of rows to a key/value head the products are the cost, and a
// block's 64 keys are read from memory once for all waves.  Same transposed
// products, with 32x32 matrix instructions.
//  * LDS holds two blocks as bf16 (codes converted on the way); the next block
//    waits in registers while this one is multiplied, one barrier a block.
//  * 16-byte chunks of an LDS row are exchanged by the row's number (turn_of): a
//    16-byte read serves lanes 0-3, 12-15 and 20-27 together, then 4-11, 16-19
//    and 28-31 (measured), and these 16 rows meet the 16 places of 256 bytes.
//  * The maximum is set 2^8 ahead when a row's scores outgrow it: terms are at
//    most 1, and the outputs are seldom rescaled.
// What bounds it: matrix and vector units in turn (4096 tokens behind 8192, 32
// heads over 8 of 128: 655 to 740 us by card, 1.05 to 0.93 PFLOP/s, a large library
// product's 1.18).
typedef float f32x16 __attribute__((ext_vector_type(16)));

// The LDS row of a block's key that matrix row r of a 32-key tile takes: bits 2
// and 3 exchanged, which leaves a lane with runs of 8 keys.
__device__ __forceinline__ int key_row(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }
// what a row of C chunks of 16 bytes exchanges its chunks by (exclusive or)
template <int C> __device__ __forceinline__ int turn_of(int row) { return (row / (16 / C)) & (C - 1); }

__device__ __forceinline__ float other_half(float x, bool maximum) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float a0 = __builtin_bit_cast(float, (uint32_t)a[0]), a1 = __builtin_bit_cast(float, (uint32_t)a[1]);
  return maximum ? fmaxf(a0, a1) : a0 + a1;
}

// Blocks on their way from memory to LDS: a thread's 16-byte chunks of a block's
// keys and of a block's values.  Where they lie is the same for every block but
// for the block's base, which all threads share: offsets are made once.
template <int F, int DH, int NW> struct Stage {
  static constexpr int SZ = size_of(F), PB = per_byte(F), TH = NW * 64;
  static constexpr int KC = kKeys * DH * SZ / PB / 16;  // chunks of a block's keys, as many of its values
  static constexpr int IT = (KC + TH - 1) / TH;
  static constexpr int KROW = DH * SZ / PB / 16, VROW = kKeys * SZ / 16;
  static constexpr int PER = SZ == 1 ? 2 * PB : 1;      // places of a chunk in LDS, 8 values each
  static constexpr int KB = kKeys * DH * 2;             // bytes of a block's keys in LDS
  // a thread's chunks lie so many rows apart, a multiple of 16, so that they
  // are exchanged alike
  static constexpr int KSTEP = TH / KROW, VSTEP = TH / VROW;
  static_assert(IT == 1 || (KSTEP % 16 == 0 && VSTEP % 16 == 0), "turn_of of a thread's chunks");
  u32x4 k[IT], v[IT];
  float scale;
  uint32_t vat, kto[PER], vto[PER];  // from: values in memory; to: LDS
  bool has_k, has_v;

  __device__ __forceinline__ void init(int ps) {
    // values are dealt from the other end, so that few chunks still meet all waves
    const uint32_t kc = threadIdx.x, vc = threadIdx.x ^ (TH / 2);
    has_k = KC % TH == 0 || kc < (uint32_t)KC;
    has_v = KC % TH == 0 || vc < (uint32_t)KC;
    vat = ((vc / VROW) << ps) * SZ + vc % VROW * 16;
    constexpr int VP = PER / PB;                        // of a chunk of one channel's values
#pragma unroll
    for (int b = 0; b < PER; ++b) {
      kto[b] = kc / KROW * (DH * 2) + ((kc % KROW * PER + b) ^ turn_of<DH / 8>(kc / KROW)) * 16;
      const uint32_t row = vc / VROW * PB + b / VP;
      vto[b] = row * (kKeys * 2) + ((vc % VROW * VP + b % VP) ^ turn_of<kKeys / 8>(row)) * 16;
    }
  }
  // p, ks, vs: the block's base, the same for all threads
  __device__ __forceinline__ void load_keys(const char* p, const float* ks, const float* vs) {
#pragma unroll
    for (int i = 0; i < IT; ++i)
      if (has_k) k[i] = *reinterpret_cast<const u32x4*>(p + (uint32_t)(threadIdx.x * 16 + i * (TH * 16)));
    if constexpr (is_coded(F))
      if (threadIdx.x < 128) scale = (threadIdx.x < 64 ? ks : vs - 64)[threadIdx.x];
  }
  __device__ __forceinline__ void load_values(const char* p, int ps) {
#pragma unroll
    for (int i = 0; i < IT; ++i)
      if (has_v) v[i] = *reinterpret_cast<const u32x4*>(p + (size_t)((uint32_t)(i * VSTEP) << ps) * SZ + vat);
  }
  __device__ __forceinline__ static void put(char* lds, const uint32_t (&to)[PER], u32x4 x) {
    if constexpr (F == EVO_CACHE_FP4) {
#pragma unroll
      for (int b = 0; b < 4; ++b) *reinterpret_cast<u32x4*>(lds + to[b]) = row_bf16(x[b]);
    } else if constexpr (is_coded(F)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const u32x2 lo = codes_bf16<F>(x[2 * b]), hi = codes_bf16<F>(x[2 * b + 1]);
        *reinterpret_cast<u32x4*>(lds + to[b]) = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    } else {
      *reinterpret_cast<u32x4*>(lds + to[0]) = x;
    }
  }
  __device__ __forceinline__ void store_keys(char* lds, float* scales) const {
#pragma unroll
    for (int i = 0; i < IT; ++i)
      if (has_k) put(lds + i * KSTEP * (DH * 2), kto, k[i]);
    if constexpr (is_coded(F))
      if (threadIdx.x < 128) scales[threadIdx.x] = scale;
  }
  __device__ __forceinline__ void store_values(char* lds) const {
#pragma unroll
    for (int i = 0; i < IT; ++i)
      if (has_v) {
        char* to = lds + i * VSTEP * PB * (kKeys * 2);
        if constexpr (F == EVO_CACHE_FP4) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const u32x2 e0 = channel_bf16(even_channel(v[i][2 * b])), e1 = channel_bf16(even_channel(v[i][2 * b + 1]));
            const u32x2 d0 = channel_bf16(odd_channel(v[i][2 * b])), d1 = channel_bf16(odd_channel(v[i][2 * b + 1]));
            *reinterpret_cast<u32x4*>(to + vto[b]) = u32x4{e0[0], e0[1], e1[0], e1[1]};
            *reinterpret_cast<u32x4*>(to + vto[2 + b]) = u32x4{d0[0], d0[1], d1[0], d1[1]};
          }
        } else {
          put(to, vto, v[i]);
        }
      }
  }
  // Values of a block that some row does not see all of: past the `left` keys
  // that the cache holds they become 0; NaNs and infinities too, and *bad is set.
  // (fp4: finite whatever the codes are, so that terms of 0 are enough.)
  __device__ __forceinline__ void clear_values(int left, int* bad) {
    if constexpr (F == EVO_CACHE_FP4) return;
    bool found = false;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int key = (int)((threadIdx.x ^ (TH / 2)) % VROW) * (16 / SZ);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint32_t x = v[i][d];
#pragma unroll
        for (int e = 0; e < 4 / SZ; ++e)
          if (key + d * (4 / SZ) + e >= left) x &= ~(((1u << (8 * SZ)) - 1) << (8 * SZ * e));
        if constexpr (holds_nan(F)) {
          const uint32_t y = finite_only<F>(x);
          found |= y != x;
          x = y;
        }
        v[i][d] = x;
      }
    }
    if (found && has_v) *bad = 1;
  }
};

// Workgroup (row tile of 32 NW rows, key/value head, part of the keys).
//
// Half of the waves run half a block behind the others: while one half of them
// multiplies (the scores of block i, then the outputs of block i - 1), the other
// does the softmax of its scores, with a barrier between the halves of a block.
// Waves w and w + NW / 2 share a SIMD where NW is 8, so that its matrix and
// vector units work side by side.  In units of barriers, wave half `late` (0 or
// 1) multiplies for block i at 2 i + late and takes its softmax at 2 i + 1 +
// late.  There it also stores its share of the keys of block i + 1 + late and
// of the values of block i + late: both places were last read at 2 i - 1 + 2
// late at most, and are first read at 2 i + 2 + 2 late.  (Scales are stored with
// the keys by the first two waves, at 2 i - 1 for block i; the softmax of block
// i - 2 has read their place at 2 i - 2.)// With the products instead, a
// 4096-token chunk behind 8192 tokens took 707 us; here 689 us.
//
// FAR_CAP: a cap above kFastCap (of its own, because its code costs the others
// registers: 100 tokens over 2000 bf16 positions, cap 30, 98 us with it and 82
// without).
template <int F, int DH, int NW, bool FAR_CAP>
__global__ void __launch_bounds__(NW * 64, 2) tile_kernel(AttArgs a) {
  typedef Stage<F, DH, NW> S;
  constexpr int TR = 32 * NW, CT = DH / 32;
  __shared__ __attribute__((aligned(16))) char lds_k[2][S::KB], lds_v[2][S::KB];
  __shared__ __attribute__((aligned(16))) float scales[is_coded(F) ? 2 : 1][is_coded(F) ? 128 : 1];
  // of the values of block i at i & 3; cleared at 2 i - 4, set at 2 i and 2 i + 1, read at 2 i + 2 and 2 i + 3
  __shared__ int bad[4];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, half = lane >> 5, late = w >= NW / 2 ? 1 : 0;
  int tile, h, split, seq;
  Where wh;
  if (!find_unit(a, blockIdx.x, &tile, &h, &split) || !find_tile(a, tile, TR, &seq, &wh)) return;
  const Blocks bl = blocks_of(a, wh);
  const int per = max(a.by_split.divide(bl.count + a.n_split - 1), 1);
  const int v0 = min(split * per, bl.count), n = min(v0 + per, bl.count) - v0;
  const int ps = a.cache.page_shift;

  const int row = min(wh.base + w * 32 + lr, wh.rows - 1), tok = a.by_group.divide(row), head = h * a.group + row - tok * a.group;
  const int pos = wh.start + tok;
  const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.f;
  // what this wave's rows see, to skip masks and whole blocks
  Sight sight, tile_sight;
  {
    Where ww = wh;
    const int r0 = wh.base + w * 32;
    ww.p_first = wh.start + a.by_group.divide(min(r0, wh.rows - 1));
    ww.p_last = wh.start + a.by_group.divide(min(r0 + 31, wh.rows - 1));
    sight.set(a, ww);
    tile_sight.set(a, wh);
  }
  // scores in units of log2: with no cap or bias by one factor inside the
  // exponential (its sign moved to the query, so that the largest product is
  // the largest score), else ahead of it
  const bool plain = a.cap == 0.f && !a.slopes && a.scale != 0.f;
  const float factor = plain ? fabsf(a.scale) * kLog2e : 1.f;
  const float to_cap = a.scale * a.inv_cap, cap_log2 = a.cap * kLog2e, to_log2 = a.scale * kLog2e;
  bf16x8 q[DH / 16];
  {
    const __bf16* p = reinterpret_cast<const __bf16*>(a.q.p) + (wh.row0 + tok) * a.q.row + head * a.q.head + half * 8;
    const uint32_t flip = plain && a.scale < 0.f ? 0x80008000u : 0;
#pragma unroll
    for (int k = 0; k < DH / 16; ++k) {
      if (a.wide) q[k] = *reinterpret_cast<const bf16x8*>(p + k * 16);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) q[k][e] = p[k * 16 + e];
      u32x4 x = __builtin_bit_cast(u32x4, q[k]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] ^= flip;
      q[k] = __builtin_bit_cast(bf16x8, x);
    }
  }
  f32x16 o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[c][e] = 0.f;
  float m = -kInf, l = 0.f;
  bool coarse = false;  // of the whole wave: some row's maximum is

  const int krow = key_row(lr) * (DH * 2), kturn = turn_of<DH / 8>(key_row(lr)) ^ half;
  const int vrow = lr * (kKeys * 2), vturn = turn_of<kKeys / 8>(lr) ^ half;

  S next;
  next.init(ps);
  // Where block i of this part lies: first element of its page and head, slot.
  // Keys are asked for a block ahead of values, which use what was found then.
  struct Place {
    int64_t first;
    int slot;
  };
  Pages pages;
  pages.load(a, bl, seq, v0, 1);
  int paged = 64;  // blocks below it are in `pages`
  const auto place = [&](int i) {
    if (i >= paged) {
      pages.load(a, bl, seq, v0 + i, 1);
      paged += 64;
    }
    const int head_page = pages.at(i) * a.cache.n_kv_heads + h;  // (pages * heads stay below 2^31, see the checks)
    return Place{(int64_t)head_page * (DH << ps), bl.at(v0 + i) * kKeys & ((1 << ps) - 1)};
  };
  Place at_keys = {}, at_values = {};
  const auto fetch_keys = [&](int i) {
    if (i >= n) return;
    at_keys = place(i);
    const int64_t key = at_keys.first + at_keys.slot * DH, row = at_keys.first / DH + at_keys.slot;
    next.load_keys(reinterpret_cast<const char*>(a.cache.k) + key * S::SZ / S::PB, is_coded(F) ? a.cache.ks + row : nullptr,
                   is_coded(F) ? a.cache.vs + row : nullptr);
  };
  const auto fetch_values = [&](int i) {
    if (i >= n) return;
    next.load_values(reinterpret_cast<const char*>(a.cache.v) + (at_values.first / S::PB + at_values.slot) * S::SZ, ps);
  };
  const auto put_keys = [&](int i) {
    if (i < n) next.store_keys(lds_k[i & 1], scales[is_coded(F) ? i & 1 : 0]);
  };
  const auto put_values = [&](int i) {
    if (i >= n) return;
    const int kb = bl.at(v0 + i) * kKeys;
    if (!tile_sight.all(kb)) next.clear_values(wh.ctx - kb, &bad[i & 3]);
    next.store_values(lds_v[i & 1]);
  };

  // (values that no terms meet yet, finite all the same)
  for (int x = threadIdx.x * 16; x < S::KB; x += NW * 64 * 16) *reinterpret_cast<u32x4*>(lds_v[1] + x) = u32x4{0, 0, 0, 0};
  if (threadIdx.x < 4) bad[threadIdx.x] = 0;
  __syncthreads();
  fetch_keys(0);
  at_values = at_keys;
  put_keys(0);
  if (late) {
    fetch_values(0);
    fetch_keys(1);
    at_values = at_keys;
    put_values(0);
    put_keys(1);
  }
  fetch_values(late);
  fetch_keys(1 + late);
  __syncthreads();
  if (late) __syncthreads();

  // The products of a block: its scores, and the outputs of the block before.
  // kRing operands are on their way from LDS at any time; left to itself the
  // compiler keeps one, and every matrix instruction waits for its read.
  // (Always both, also where the terms are zeros or the scores of no use: a
  // second path would cost a second set of accumulators, and the other half of
  // the waves would be waited for all the same.)
  const auto products = [&](f32x16(&s)[2], const bf16x8(&p)[4], const char* keys, const char* values) {
    constexpr int NK = DH / 8, N = NK + 4 * CT;
    const auto read = [&](int x) {
      if (x < NK) return *reinterpret_cast<const bf16x8*>(keys + krow + (x & 1) * (32 * DH * 2) + (((x & ~1) ^ kturn) * 16));
      const int y = x - NK;
      return *reinterpret_cast<const bf16x8*>(values + vrow + y % CT * (32 * kKeys * 2) + (((2 * (y / CT)) ^ vturn) * 16));
    };
    bf16x8 ring[kRing];
#pragma unroll
    for (int x = 0; x < kRing; ++x) ring[x] = read(x);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < N; ++x) {
      if (x < NK) s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[x % kRing], q[x / 2], s[x & 1], 0, 0, 0);
      else o[(x - NK) % CT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[x % kRing], p[(x - NK) / CT], o[(x - NK) % CT], 0, 0, 0);
      if (x + kRing < N) ring[x % kRing] = read(x + kRing);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  bf16x8 p[4];  // the terms of the block before
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  for (int i = 0; i <= n; ++i) {
    const int kb = i < n ? bl.at(v0 + i) * kKeys : 0;
    const bool any = i < n && sight.any(kb);
    if (late == 0 && threadIdx.x == 0) bad[(i + 2) & 3] = 0;
    // ---- products ----
    f32x16 s[2];
    products(s, p, lds_k[i & 1], lds_v[(i - 1) & 1]);
    if (i > 0) {
      if constexpr (holds_nan(F)) {
        if (__builtin_expect(bad[(i - 1) & 3], 0)) {
          // the values that store_values() took out, for the rows that see them
          const int kl = bl.at(v0 + i - 1) * kKeys, s0 = kl & ((1 << ps) - 1);
          const int64_t b = (int64_t)page_of(a.rows, a.cache, seq, kl >> ps) * a.cache.n_kv_heads + h;
#pragma unroll 1
          for (int j = 0; j < min(kKeys, wh.ctx - kl); ++j) {
            const bool see = sees(a, wh, pos, kl + j);
            int64_t at = ((b * DH + 4 * half) << ps) + s0 + j;
            asm volatile("" : "+v"(at));  // 64 addresses are made here, not kept over the loop
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float x = not_finite<F>(a.cache.v, at + ((c * 32 + 8 * (e >> 2) + (e & 3)) << ps));
                if (see) o[c][e] += x;
                __builtin_amdgcn_sched_barrier(0);
              }
          }
        }
      }
    }
    if (i == n) break;
    __syncthreads();
    // ---- softmax, and the next blocks ----
    put_values(i + late);
    put_keys(i + 1 + late);
    at_values = at_keys;
    fetch_values(i + 1 + late);
    fetch_keys(i + 2 + late);
    if (any) {
      const bool masked = !sight.all(kb);
      // element e of tile t is key 32 t + 16 (e / 8) + 8 half + e % 8
      const auto key_at = [&](int t, int e) { return kb + 32 * t + 16 * (e >> 3) + 8 * half + (e & 7); };
      const auto times = [&](const float* by) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(by + 32 * t + 16 * (e >> 3) + 8 * half + (e & 7));
#pragma unroll
            for (int d = 0; d < 4; ++d) s[t][e + d] *= x[d];
          }
      };
      if constexpr (is_coded(F)) times(scales[i & 1]);
      if (!plain) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float z = s[t][e];
            if constexpr (FAR_CAP) z = a.cap * squash<__bf16>(z * a.scale * a.inv_cap) * kLog2e;
            else z = a.cap > 0.f ? cap_log2 * squash_fast(z * to_cap) : z * to_log2;
            if (a.slopes) z = fmaf(-slope, distance(pos, key_at(t, e)), z);
            s[t][e] = z;
          }
      }
      if (masked) {
        const Seen seen(a, wh, pos);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!seen.at(key_at(t, e))) s[t][e] = -kInf;
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
      top = other_half(top, true) * factor;
      if (__any(!(top <= m))) {
        const float m_new = next_maximum<F>(m, top);
        const float f = exp2_(m - (m_new == -kInf ? 0.f : m_new));
        m = m_new;
        l *= f;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[c][e] *= f;
        coarse = is_coarse(m_new);
      }
      const float base = m == -kInf ? 0.f : m;
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = fmaf(s[t][e], factor, -base);
      if (__builtin_expect(coarse, 0)) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[t][e] = coarse_of_row<F>(s[t][e], base);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[t][e] = exp2_(s[t][e]);
          sum += s[t][e];
        }
      l += sum;
      if constexpr (is_coded(F)) {
        times(scales[i & 1] + 64);
        if (masked) {
          const Seen seen(a, wh, pos);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!seen.at(key_at(t, e))) s[t][e] = 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = pack2(s[j >> 1][(j & 1) * 8 + 2 * e], s[j >> 1][(j & 1) * 8 + 2 * e + 1]);
        p[j] = __builtin_bit_cast(bf16x8, x);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    }
    __syncthreads();
  }
  if (!late) __syncthreads();  // (as many barriers in both halves)

  l = other_half(l, false);
  const int r = w * 32 + lr;
  if (wh.base + r >= wh.rows) return;
  if (a.n_split > 1) {
    const int64_t part = (((int64_t)tile * a.cache.n_kv_heads + h) * a.n_split + split) * TR + r;
    if (half == 0) {
      a.part_ml[part * 2] = m;
      a.part_ml[part * 2 + 1] = l;
    }
    if (n <= 0) return;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4*>(a.part + part * DH + c * 32 + 2 * e + 4 * half) = f32x4{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]};
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  __bf16* dst = reinterpret_cast<__bf16*>(a.out.p) + (wh.row0 + tok) * a.out.row + head * a.out.head;
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      store4(dst + c * 32 + 2 * e + 4 * half, a.wide,
             l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : f32x4{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]} * inv);
  if (a.lse && half == 0)
    a.lse[(int64_t)(wh.row0 + tok) * a.n_heads + head] = l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Joins the parts of a launch of tile_kernel, a thread four channels of a row.
template <int DH>
__global__ void __launch_bounds__(256) join_kernel(AttArgs a, int tile_rows) {
  const int wgs = tile_rows * (DH / 4) / 256;  // of a tile: tile_rows is 128 or 256
  const int th = blockIdx.x / wgs, x = (blockIdx.x - th * wgs) * 256 + threadIdx.x;
  const int tile = a.by_kv_heads.divide(th), h = th - tile * a.cache.n_kv_heads;
  int seq;
  Where wh;
  if (tile >= a.n_tiles || !find_tile(a, tile, tile_rows, &seq, &wh)) return;
  const int r = x / (DH / 4);
  if (wh.base + r < wh.rows) join_parts<__bf16, DH>(a, wh, th, h, tile_rows, r, x % (DH / 4) * 4);
}

// Which formats take two row blocks to a wave, and what leaves a SIMD the
// registers for two waves (200 fp32 rows, which do not fit, 24 us with four waves
// to a workgroup and 32 with eight).
constexpr bool two_row_blocks(int f, int dh) { return !is_coded(f) && !(f == EVO_CACHE_FP32 && dh == 128); }
constexpr bool eight_waves(int f, int dh, int tile_rows) {
  return !(tile_rows == 32 && dh * size_of(f) >= 256) && !(f == EVO_CACHE_FP32 && dh == 128);
}

// Rows of a sequence and key/value head from which keys and values go through
// LDS (measured at tile_rows_of).
constexpr int64_t kNever = 1ll << 40;
constexpr int64_t lds_rows(int f, int dh) {
  if (f == EVO_CACHE_FP32) return kNever;
  if (dh == 128) return f == EVO_CACHE_BF16 ? 33 : 97;
  if (f == EVO_CACHE_BF16) return dh == 64 ? 65 : 1025;
  return f == EVO_CACHE_INT8 && dh == 64 ? 2049 : kNever;
}

template <typename T, int F, int DH, int R, int NW>
void launch_stream(int64_t wgs, const AttPlan& p, const AttArgs& a, hipStream_t stream) {
  if constexpr (F == EVO_CACHE_FP4 && sizeof(T) == 2 && R == 1) {
    if (p.rest) {
      if constexpr (NW == 1)
        hipLaunchKernelGGL((stream_kernel<T, F, DH, R, 1, false, true>), dim3(wgs), dim3(64), 0, stream, a);
      else
        hipLaunchKernelGGL((a.n_split > 1 ? stream_kernel<T, F, DH, R, NW, true, true> : stream_kernel<T, F, DH, R, NW, false, true>),
                           dim3(wgs), dim3(NW * 64), 0, stream, a);
      return;
    }
  }
  if constexpr (NW == 1)  // (not in parts)
    hipLaunchKernelGGL((stream_kernel<T, F, DH, R, 1, false>), dim3(wgs), dim3(64), 0, stream, a);
  else if constexpr (NW == 4 || eight_waves(F, DH, 16 * R))
    hipLaunchKernelGGL((a.n_split > 1 ? stream_kernel<T, F, DH, R, NW, true> : stream_kernel<T, F, DH, R, NW, false>),
                       dim3(wgs), dim3(NW * 64), 0, stream, a);
}

template <typename T, int F, int DH>
hipError_t launch_as(const AttPlan& p, const AttArgs& a, hipStream_t stream) {
  const int64_t blocks = (int64_t)p.n_tiles * a.cache.n_kv_heads;
  int64_t wgs = blocks * p.n_split;
  if (p.tiles_per_seq > 1) wgs = (wgs / p.tiles_per_seq + 7) / 8 * 8 * p.tiles_per_seq;  // (see find_unit)
  constexpr int R2 = two_row_blocks(F, DH) ? 2 : 1;
  if (p.tile_rows == 16) {
    if (p.waves == 1) launch_stream<T, F, DH, 1, 1>(wgs, p, a, stream);
    else if (p.waves == 8) launch_stream<T, F, DH, 1, 8>(wgs, p, a, stream);
    else launch_stream<T, F, DH, 1, 4>(wgs, p, a, stream);
  } else if (p.tile_rows == 32) {
    if (p.waves == 1) launch_stream<T, F, DH, R2, 1>(wgs, p, a, stream);
    else if (p.waves == 8) launch_stream<T, F, DH, R2, 8>(wgs, p, a, stream);
    else launch_stream<T, F, DH, R2, 4>(wgs, p, a, stream);
  } else if constexpr (sizeof(T) == 2 && lds_rows(F, DH) != kNever) {
    const bool far = a.cap > kFastCap;
    if (p.tile_rows == 128)
      hipLaunchKernelGGL((far ? tile_kernel<F, DH, 4, true> : tile_kernel<F, DH, 4, false>), dim3(wgs), dim3(256), 0, stream, a);
    else if constexpr (DH == 128)
      hipLaunchKernelGGL((far ? tile_kernel<F, DH, 8, true> : tile_kernel<F, DH, 8, false>), dim3(wgs), dim3(512), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_split == 1) return e;
    hipLaunchKernelGGL((join_kernel<DH>), dim3(blocks * (p.tile_rows * (DH / 4) / 256)), dim3(256), 0, stream, a, p.tile_rows);
  }
  return hipGetLastError();
}

// Rows of a tile, by the rows that a sequence has for a key/value head.
// Measured, us of a call:
//  * 8-bit caches take 16 rows to a wave: the registers then hold three waves to
//    a SIMD, which hide the conversions (two row blocks to a wave: 32-token
//    chunks over fp8 memories 51, one 45).
//  * others take two row blocks, which halves the reads (12 heads of 64 over 4000
//    bf16 positions of 16 sequences: 64 rows 72, one block 88; 32 rows 51 and 50;
//    32 rows of 128, grouped by four over 8000, 109 and 137; fp32, 64 rows 158
//    and 201, but 32 rows 126 and 114: there one block would be the faster).  Two
//    row blocks of fp32 keys of 128 do not fit.
//  * LDS pays from lds_rows() on, where a sequence's rows share enough: heads of
//    128, bf16: 32 rows 109, LDS 113, 64 rows 140 and 119; 8-bit: 96 rows 78 and
//    91, 128 rows 96 and 76.  Heads of 64, bf16: 64 rows 45 and 46, 80 rows 50 and
//    46 (2000 positions); int8: 800 rows 250 and 278, 2000 rows of 8 sequences 307
//    and 280, causal 181 and 208, 4096 rows of one over 12288 586 and 461; fp8 448
//    and 472 there.  Heads of 32, bf16: 800 rows 96 and 101, 2000 rows 116 and 102,
//    causal 81 and 85; int8 over 8000 270 and 347.
//  * through LDS, heads of 128 take tiles of 256 (4096 rows behind 8192 659,
//    tiles of 128 746; 64 rows, 256 to a head, 57 and 64), the others of 128
//    (1024 rows behind 1024, 4 sequences, 51, tiles of 256 59, which then are fewer
//    than compute units; larger calls were not compared).
//  * fp4 takes the other codes' choices, which were not measured over it, but for a
//    single block of keys, which does not go through LDS (32 over 8 heads of 128: 4000
//    rows of 4 sequences over 64 positions 76, LDS 118; 1000 rows of 8 30 and 55).
int tile_rows_of(int dtype, int format, int head_dim, int64_t rows, bool rest) {
  if (dtype == EVO_BF16 && rows >= lds_rows(format, head_dim) && !rest) return head_dim == 128 && rows > 128 ? 256 : 128;
  return rows <= 16 || !two_row_blocks(format, head_dim) ? 16 : 32;
}

}  // namespace

// (By the lengths alone: what masks hide is not considered, so parts of the keys
// that no row sees may have workgroups that find no block.)
AttPlan plan_attention(int dtype, int format, int head_dim, int n_heads, int n_kv_heads, const RowsView& r,
                       int max_length, int n_cu) {
  AttPlan p = {};
  const int group = n_heads / n_kv_heads;
  const int64_t rows = (int64_t)r.max_rows * group;  // of one sequence and key/value head
  const int64_t blocks = ((int64_t)max_length + kKeys - 1) / kKeys;
  p.rest = dtype == EVO_BF16 && format == EVO_CACHE_FP4 && (rows <= 8 || blocks <= 1);
  p.tile_rows = tile_rows_of(dtype, format, head_dim, rows, p.rest);
  // row tiles: as many for every sequence, or packed by the rows before
  const int64_t even = (rows + p.tile_rows - 1) / p.tile_rows;
  const int64_t packed = (int64_t)r.n_rows * group / p.tile_rows + r.n_seqs;
  if (!r.cu || even * r.n_seqs <= packed) {
    p.tiles_per_seq = (int)even;
    p.n_tiles = (int)(even * r.n_seqs);
  } else {
    p.n_tiles = (int)packed;
  }
  const int64_t wgs = (int64_t)p.n_tiles * n_kv_heads;
  // parts of the keys: two workgroups for every compute unit (one of eight
  // waves), each with a few blocks for every wave (part_blocks)
  int64_t each = p.tile_rows == 256 ? 1 : 2, most = blocks / part_blocks(wgs, n_cu);
  // Over fp4, where a block's bytes are a quarter and a part's join weighs more: three,
  // and no more parts than a part has blocks (one token over 65536 positions, 8 heads of
  // 128, 27.0 us with 64 parts, 22.0 with 32; 12 heads of 64 over 16384 16.6 with 42,
  // 11.4 with 16; 6 ragged sequences of up to 65001 65 with two, 54 with three, 59 with
  // four; 6 equally long ones 113, 90 and 104; all with bf16 queries).
  if (format == EVO_CACHE_FP4 && p.tile_rows <= 32) {
    each = 3;
    most = std::min(most, (int64_t)std::ceil(std::sqrt((double)blocks)));
  }
  const int64_t want = wgs ? (each * n_cu + wgs - 1) / wgs : 1;
  p.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(want, most));
  // a workgroup that has its compute unit to itself brings eight waves, unless its
  // part has fewer blocks than that
  p.waves = wgs * p.n_split <= n_cu && (p.n_split == 1 || blocks / p.n_split >= 8) && eight_waves(format, head_dim, p.tile_rows) ? 8 : kWaves;
  // where tiles alone give every SIMD a wave and their keys are few, a wave takes a
  // tile of its own: no wave without a block, no join (84 chunks of 1600 fp32 rows
  // over 27 positions 491 us with four waves and 129 with one, int8 136 and 48;
  // over 250 93 and 52, int8 27 and 20; over 1000 126 and 111, int8 35 and 43)
  if (p.tile_rows <= 32 && p.n_split == 1 && wgs >= 4 * (int64_t)n_cu && blocks <= 8) p.waves = 1;
  if (p.n_split > 1) {
    p.ml_floats = wgs * p.n_split * p.tile_rows * 2;
    p.part_floats = wgs * p.n_split * p.tile_rows * head_dim;
    // few rows are joined by the workgroup that ends last, which saves a launch;
    // long chunks' tiles by a launch of its own, over all compute units
    if (p.tile_rows <= 32) p.flags = wgs * p.n_split;
  }
  return p;
}

hipError_t launch_attention(int dtype, int format, int head_dim, const AttPlan& plan, const AttArgs& a,
                            hipStream_t stream) {
#define X(D, T, F, DH) \
  if (dtype == D && format == F && head_dim == DH) return launch_as<T, F, DH>(plan, a, stream);
#define Y(DH)                             \
  X(EVO_FP32, float, EVO_CACHE_FP32, DH)  \
  X(EVO_FP32, float, EVO_CACHE_INT8, DH)  \
  X(EVO_FP32, float, EVO_CACHE_FP8, DH)   \
  X(EVO_FP32, float, EVO_CACHE_FP4, DH)   \
  X(EVO_BF16, __bf16, EVO_CACHE_BF16, DH) \
  X(EVO_BF16, __bf16, EVO_CACHE_INT8, DH) \
  X(EVO_BF16, __bf16, EVO_CACHE_FP8, DH)  \
  X(EVO_BF16, __bf16, EVO_CACHE_FP4, DH)
  Y(32) Y(64) Y(128)
#undef Y
#undef X
  return hipErrorInvalidValue;
}

}  // namespace evo
