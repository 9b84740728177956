// Rows of queries, keys and values around the paged cache: norm for each head
// and rotation by position in one pass, quantising as the cache is written,
// and reading it back.
//
// What bounds it: memory.  Every value is read once and written once; norm,
// rotation and quantising are a few operations a value (65537 tokens of 40 heads
// of 128: 309 us, 4.35 TB/s of a copy's 4.92; 8 memories of 8191 fp8 tokens written
// and read back: 160 us, 3.7 TB/s).
//  * Queries and keys: a row of head_dim values lies over head_dim / 8 lanes,
//    8 values a lane (16 bytes of bf16), so that the row's sum of squares or
//    maximum takes 2 to 4 lane exchanges.  A group of lanes keeps its token's
//    (cos, sin) and works through several heads, because the table's 8 bytes
//    a pair would otherwise be four times the row's own traffic.
//  * Values go to a transposed page: a lane takes a whole row (its maximum
//    then needs no exchange) and a wave 64 consecutive tokens, so that each of
//    the head_dim stores of a wave is a run of neighbouring slots.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "evo.h"
#include "evo_memory.hpp"

namespace evo {
namespace {

constexpr int kNone = -1;
constexpr int kThreads = 256;
constexpr int kAhead = 4;     // heads whose rows a lane requests ahead
constexpr int kFill = 2048;   // workgroups that fill the device (8 a compute unit)
constexpr int kValueWaves = 1024;

template <int F> struct Held;
template <> struct Held<EVO_CACHE_FP32> { typedef float type; };
template <> struct Held<EVO_CACHE_BF16> { typedef __bf16 type; };
template <> struct Held<EVO_CACHE_INT8> { typedef int8_t type; };
template <> struct Held<EVO_CACHE_FP8> { typedef uint8_t type; };
template <> struct Held<kNone> { typedef uint8_t type; };

__device__ __forceinline__ float low(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }

// 8 consecutive values
__device__ __forceinline__ void load8(const float* p, int wide, float* x) {
  if (wide) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[e];
  }
}
__device__ __forceinline__ void load8(const __bf16* p, int wide, float* x) {
  if (wide) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = low(a[e]); x[2 * e + 1] = high(a[e]); }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)p[e];
  }
}
__device__ __forceinline__ void store8(float* p, int wide, const float* x) {
  if (wide) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = x[e];
  }
}
__device__ __forceinline__ void store8(__bf16* p, int wide, const float* x) {
  if (wide) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = (__bf16)x[e];
  }
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// How a row whose largest magnitude has the bits `top` is coded: code =
// round(x / s).  The quotient comes from s's reciprocal and one residual step,
// which gives the correctly rounded x / s in 32 bits.  (Values halfway between two
// codes, frequent with bf16 inputs, may fall to either: s is a rounded quotient
// itself.  200000 rows of 64 in int8: all codes but those are the exact
// quotient's.)  Rows near the smallest floats are lifted first (lift), to keep the
// reciprocal finite.
struct Coding {
  float s, r, d, lift;
};
template <int F> __device__ __forceinline__ Coding coding_of(uint32_t top) {
  constexpr float M = F == EVO_CACHE_INT8 ? 127.f : 448.f;
  const float amax = __builtin_bit_cast(float, top);
  Coding c;
  if (top >= 0x7f800000u) {  // a NaN or an infinity in the row
    c.s = __builtin_nanf("");
    c.r = c.d = c.lift = 0.f;
    return c;
  }
  c.s = amax / M;
  c.lift = amax < 0x1p-60f ? 0x1p64f : 1.f;
  c.d = c.s * c.lift;
  c.r = c.d > 0.f ? 1.f / c.d : 0.f;
  return c;
}
template <int F> __device__ __forceinline__ float quotient(float x, const Coding& c) {
  constexpr float M = F == EVO_CACHE_INT8 ? 127.f : 448.f;
  if (c.r == 0.f) return 0.f;
  x *= c.lift;
  const float q = x * c.r;
  return __builtin_amdgcn_fmed3f(fmaf(fmaf(-q, c.d, x), c.r, q), -M, M);
}
// four codes, the first in the lowest byte
template <int F> __device__ __forceinline__ uint32_t code4(const float* y) {
  if (F == EVO_CACHE_FP8) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
  }
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) v |= ((uint32_t)(int)rintf(y[e]) & 0xffu) << (8 * e);
  return v;
}
template <int F> __device__ __forceinline__ void decode4(uint32_t v, float* y) {
  if (F == EVO_CACHE_FP8) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(v, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(v, true);
    y[0] = a[0]; y[1] = a[1]; y[2] = b[0]; y[3] = b[1];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)(int8_t)(v >> (8 * e));
  }
}

// Slot of position `pos` of a sequence: index of its (page, head) block, or -1
// where there is none.
__device__ __forceinline__ int64_t block_of(const RowsArgs& a, int seq, int pos, int head) {
  if (pos < 0 || (pos >> a.cache.page_shift) >= a.rows.max_pages) return -1;
  return (int64_t)page_of(a.rows, a.cache, seq, pos >> a.cache.page_shift) * a.cache.n_kv_heads + head;
}

// (selected as numbers: a choice between two members of the arguments would put
// them into memory)
__device__ __forceinline__ float* scales_of(const RowsArgs& a, bool value) {
  const uint64_t k = (uint64_t)a.cache.ks, v = (uint64_t)a.cache.vs;
  return reinterpret_cast<float*>(value ? v : k);
}

// The lane's 8 values of a row into the cache: keys side by side, values a page
// row each.
template <int F, int DH>
__device__ __forceinline__ void store_held(const RowsArgs& a, int64_t block, int slot, bool value, int lane, const float* y,
                                           const Coding& c) {
  typedef typename Held<F>::type H;
  const int ps = a.cache.page_shift;
  H* k = reinterpret_cast<H*>(a.cache.k) + ((block << ps) + slot) * DH + lane * 8;
  H* v = reinterpret_cast<H*>(a.cache.v) + ((block * DH + lane * 8) << ps) + slot;
  if constexpr (is_coded(F)) {
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = quotient<F>(y[e], c);
    const u32x2 w = {code4<F>(z), code4<F>(z + 4)};
    if (!value) {
      *reinterpret_cast<u32x2*>(k) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[(int64_t)e << ps] = (H)(w[e / 4] >> (8 * (e & 3)));
    }
    if (lane == 0) scales_of(a, value)[(block << ps) + slot] = c.s;
  } else if constexpr (F != kNone) {
    if (!value) {
      store8(k, 1, y);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[(int64_t)e << ps] = (H)y[e];
    }
  }
}

// A row's 8 values of a lane as they lie in memory.
template <typename T> struct Raw { u32x4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Raw<T> load_raw(const T* p, int wide) {
  Raw<T> r;
  if (wide) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const u32x4*>(p)[i];
  } else {
    T* d = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = p[e];
  }
  return r;
}
__device__ __forceinline__ void unpack(const Raw<__bf16>& r, float* x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[2 * e] = low(r.w[0][e]); x[2 * e + 1] = high(r.w[0][e]); }
}
__device__ __forceinline__ void unpack(const Raw<float>& r, float* x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(float, (uint32_t)r.w[e / 4][e % 4]);
}

template <typename T, int F, int DH>
__device__ __forceinline__ void qk_rows(const RowsArgs& a, int block) {
  constexpr int LPR = DH / 8;  // lanes a row
  const int heads = a.heads_by_rows, groups = a.head_groups;
  const int lane = threadIdx.x % LPR;
  const int at = a.by_groups.divide(block), h0 = block - at * groups;
  const int tok = at * (kThreads / LPR) + (int)threadIdx.x / LPR;
  // whole waves stay for the exchanges; rows past the end repeat the last one
  // and are not stored
  const bool live = tok < a.rows.n_rows;
  const int n = live ? tok : a.rows.n_rows - 1;
  const auto source = [&](int h) {
    const int hk = h - a.n_heads, hv = hk - a.n_kv_heads;
    const T* p = hk < 0 ? reinterpret_cast<const T*>(a.q.p) + n * a.q.row + h * a.q.head
                 : hv < 0 ? reinterpret_cast<const T*>(a.k.p) + n * a.k.row + hk * a.k.head
                          : reinterpret_cast<const T*>(a.v.p) + n * a.v.row + hv * a.v.head;
    return p + lane * 8;
  };
  Raw<T> next[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (h0 + u * groups < heads) next[u] = load_raw(source(h0 + u * groups), a.wide);
  int seq = 0, i = 0, pos = 0;
  if constexpr (F != kNone) {
    find_row(a.rows, n, &seq, &i);
    pos = a.starts[seq] + i;
  }
  const int turn = a.positions ? a.positions[n] : pos;
  float cs[8], sn[8];
  bool rotated = false;
  if (a.half) {
    // halves: the lane's 8 values meet pairs 8 lane' .. + 7; adjacent: 4 pairs
    const bool in = turn >= 0 && turn < a.n_positions;
    const float* t = a.table + (int64_t)(in ? turn : 0) * (2 * a.half);
    rotated = lane * 8 < 2 * a.half;
    if (rotated) {
      if (a.adjacent) {
        const f32x4 u = *reinterpret_cast<const f32x4*>(t + lane * 8), w = *reinterpret_cast<const f32x4*>(t + lane * 8 + 4);
        cs[0] = cs[1] = u[0]; cs[2] = cs[3] = u[2]; cs[4] = cs[5] = w[0]; cs[6] = cs[7] = w[2];
        sn[0] = -u[1]; sn[1] = u[1]; sn[2] = -u[3]; sn[3] = u[3];
        sn[4] = -w[1]; sn[5] = w[1]; sn[6] = -w[3]; sn[7] = w[3];
      } else {
        const bool second = lane * 8 >= a.half;
        const float* tt = t + 2 * (lane * 8 - (second ? a.half : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 u = *reinterpret_cast<const f32x4*>(tt + 4 * e);
          cs[2 * e] = u[0]; cs[2 * e + 1] = u[2];
          sn[2 * e] = second ? u[1] : -u[1];
          sn[2 * e + 1] = second ? u[3] : -u[3];
        }
      }
    }
    if (!in) {
      rotated = true;
#pragma unroll
      for (int e = 0; e < 8; ++e) cs[e] = sn[e] = __builtin_nanf("");
    }
  }
  float qg[8], kg[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    qg[e] = a.norm && a.q_gain ? a.q_gain[lane * 8 + e] : 1.f;
    kg[e] = a.norm && a.k_gain ? a.k_gain[lane * 8 + e] : 1.f;
  }
  const int half_lanes = a.half / 8;
  const int partner = (threadIdx.x & 63) + (lane < half_lanes ? half_lanes : lane < 2 * half_lanes ? -half_lanes : 0);

  const auto one = [&](int h, const Raw<T>& raw) {
    const bool is_q = h < a.n_heads, is_v = F != kNone && h >= a.n_heads + a.n_kv_heads;
    const int hk = h - a.n_heads - (is_v ? a.n_kv_heads : 0);
    float x[8];
    unpack(raw, x);
    if (a.norm && !is_v) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int d = 1; d < LPR; d *= 2) ss += __shfl_xor(ss, d);
      const float r = 1.f / sqrtf(ss * (1.f / DH) + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * r * (is_q ? qg[e] : kg[e]);
    }
    if (a.half && !is_v) {
      float o[8];
      if (a.adjacent) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = x[e ^ 1];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = __shfl(x[e], partner);
      }
      if (rotated) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(o[e], sn[e], x[e] * cs[e]);
      }
    }
    if (is_q || F == kNone) {
      T* dst = is_q ? reinterpret_cast<T*>(a.qo.p) + n * a.qo.row + h * a.qo.head
                    : reinterpret_cast<T*>(a.ko.p) + n * a.ko.row + hk * a.ko.head;
      if (live) store8(dst + lane * 8, a.wide, x);
      return;
    }
    Coding c = {};
    if constexpr (is_coded(F)) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, magnitude(x[e]));
#pragma unroll
      for (int d = 1; d < LPR; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      c = coding_of<F>(top);
    }
    const int64_t b = block_of(a, seq, pos, hk);
    if (live && b >= 0) store_held<F, DH>(a, b, pos & ((1 << a.cache.page_shift) - 1), is_v, lane, x, c);
  };
  for (int h = h0; h < heads; h += kAhead * groups) {
    Raw<T> now[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      now[u] = next[u];
      const int hn = h + (kAhead + u) * groups;
      if (hn < heads) next[u] = load_raw(source(hn), a.wide);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (h + u * groups < heads) one(h + u * groups, now[u]);
  }
}

// A wave's 64 rows of values pass through LDS a slice of kSlice bytes at a time,
// because a lane that reads (or writes) a row of its own touches a cache line 16
// bytes at a time: staged, P lanes take a row's part of a slice, RP rows at once.
constexpr int kSlice = 128, kPitch = kSlice + 16;
template <typename T, int DH> struct Slices {
  static constexpr int N = kSlice / (int)sizeof(T);
  static constexpr int V = N < DH ? N : DH;            // values of a row in a slice
  static constexpr int P = V * (int)sizeof(T) / 16;
  static constexpr int RP = 64 / P;
  static constexpr int C = DH / V;                     // slices
};
// the address that lane r holds
__device__ __forceinline__ char* address_of(char* p, int r) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)u, r), hi = (uint32_t)__shfl((int)(uint32_t)(u >> 32), r);
  return reinterpret_cast<char*>(lo | (uint64_t)hi << 32);
}
__device__ __forceinline__ uint32_t top_of(u32x4 w, __bf16) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max(m, max((w[e] << 16) & 0x7fffffffu, w[e] & 0x7fff0000u));
  return m;
}
__device__ __forceinline__ uint32_t top_of(u32x4 w, float) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max(m, w[e] & 0x7fffffffu);
  return m;
}

// The wave's 64 rows of values and where they lie: lane l has row l.
struct ValueRow {
  int n, h, slot;
  int64_t block;  // -1: the row has no slot
  bool live;
};
__device__ __forceinline__ ValueRow value_row(const RowsArgs& a, int block) {
  const int w = __builtin_amdgcn_readfirstlane(block * (kThreads / 64) + (int)(threadIdx.x >> 6));
  ValueRow r;
  const int tile = a.by_kv_heads.divide(w);
  r.h = w - tile * a.n_kv_heads;
  const int64_t n = (int64_t)tile * 64 + (threadIdx.x & 63);
  r.live = n < a.rows.n_rows;
  r.n = r.live ? (int)n : a.rows.n_rows - 1;
  int seq, i;
  find_row(a.rows, r.n, &seq, &i);
  const int pos = a.starts[seq] + i;
  r.block = block_of(a, seq, pos, r.h);
  r.slot = pos & ((1 << a.cache.page_shift) - 1);
  return r;
}

template <typename T, int F, int DH>
__device__ __forceinline__ void v_rows(const RowsArgs& a, int block, char* lds, uint32_t* tops) {
  typedef typename Held<F>::type H;
  typedef Slices<T, DH> S;
  const int lane = threadIdx.x & 63;
  const ValueRow r = value_row(a, block);
  const bool live = r.live && r.block >= 0;
  char* src = a.v.p + (r.n * a.v.row + r.h * a.v.head) * (int64_t)sizeof(T);
  u32x4 w[S::C][S::P];
#pragma unroll
  for (int i = 0; i < S::P; ++i) {
    const char* p = address_of(src, i * S::RP + lane / S::P) + (lane % S::P) * 16;
#pragma unroll
    for (int c = 0; c < S::C; ++c) {
      if (a.wide) {
        w[c][i] = *reinterpret_cast<const u32x4*>(p + c * kSlice);
      } else {
        T* d = reinterpret_cast<T*>(&w[c][i]);
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) d[e] = reinterpret_cast<const T*>(p + c * kSlice)[e];
      }
    }
  }
  Coding cd = {};
  if constexpr (is_coded(F)) {
#pragma unroll
    for (int i = 0; i < S::P; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int c = 0; c < S::C; ++c) m = max(m, top_of(w[c][i], T()));
#pragma unroll
      for (int d = 1; d < S::P; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
      if (lane % S::P == 0) tops[i * S::RP + lane / S::P] = m;
    }
    wave_sync();
    cd = coding_of<F>(tops[lane]);
    if (live) a.cache.vs[(r.block << a.cache.page_shift) + r.slot] = cd.s;
  }
  H* dst = reinterpret_cast<H*>(a.cache.v) + ((r.block * DH) << a.cache.page_shift) + r.slot;
#pragma unroll
  for (int c = 0; c < S::C; ++c) {
    wave_sync();
#pragma unroll
    for (int i = 0; i < S::P; ++i)
      *reinterpret_cast<u32x4*>(lds + (i * S::RP + lane / S::P) * kPitch + (lane % S::P) * 16) = w[c][i];
    wave_sync();
    if (live) {
#pragma unroll
      for (int j = 0; j < S::V; j += 8) {
        float x[8];
        load8(reinterpret_cast<const T*>(lds + lane * kPitch) + j, 1, x);
        if constexpr (is_coded(F)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = quotient<F>(x[e], cd);
          const uint32_t v[2] = {code4<F>(x), code4<F>(x + 4)};
#pragma unroll
          for (int e = 0; e < 8; ++e)
            dst[(int64_t)(c * S::V + j + e) << a.cache.page_shift] = (H)(v[e / 4] >> (8 * (e & 3)));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[(int64_t)(c * S::V + j + e) << a.cache.page_shift] = (H)x[e];
        }
      }
    }
  }
}

template <typename T, int F, int DH>
__global__ void __launch_bounds__(kThreads) rows_kernel(RowsArgs a) {
  __shared__ __attribute__((aligned(16))) char stage[F == kNone ? 1 : kThreads / 64][F == kNone ? 16 : 64 * kPitch];
  __shared__ uint32_t tops[F == kNone ? 1 : kThreads];
  const int w = threadIdx.x >> 6;
  if ((int)blockIdx.x < a.qk_blocks) qk_rows<T, F, DH>(a, blockIdx.x);
  else if constexpr (F != kNone) v_rows<T, F, DH>(a, blockIdx.x - a.qk_blocks, stage[w], tops + w * 64);
}

// ---- reading back: keys a group of lanes a token, values a lane a row ------
template <typename T, int F, int DH>
__device__ __forceinline__ void read_keys(const RowsArgs& a, int block) {
  typedef typename Held<F>::type H;
  constexpr int LPR = DH / 8;
  const int ps = a.cache.page_shift, groups = a.head_groups;
  const int lane = threadIdx.x % LPR;
  const int at = a.by_groups.divide(block);
  const int n = at * (kThreads / LPR) + (int)threadIdx.x / LPR;
  if (n >= a.rows.n_rows) return;
  int seq, i;
  find_row(a.rows, n, &seq, &i);
  const int pos = a.starts[seq] + i;
  const int64_t b = block_of(a, seq, pos, 0);
  for (int h = block - at * groups; h < a.heads_by_rows; h += groups) {
    const bool is_v = h >= a.n_kv_heads;
    const int hk = is_v ? h - a.n_kv_heads : h;
    float x[8] = {};
    if (b >= 0) {
      const int64_t row = ((b + hk) << ps) + (pos & ((1 << ps) - 1));
      const H* k = reinterpret_cast<const H*>(a.cache.k) + row * DH + lane * 8;
      const H* v = reinterpret_cast<const H*>(a.cache.v) + (((b + hk) * DH + lane * 8) << ps) + (pos & ((1 << ps) - 1));
      if constexpr (is_coded(F)) {
        u32x2 w = {0, 0};
        if (!is_v) {
          w = *reinterpret_cast<const u32x2*>(k);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(uint8_t)v[(int64_t)e << ps] << (8 * (e & 3));
        }
        const float s = scales_of(a, is_v)[row];
        decode4<F>(w[0], x);
        decode4<F>(w[1], x + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= s;
      } else if (!is_v) {
        load8(k, 1, x);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[(int64_t)e << ps];
      }
    }
    T* dst = is_v ? reinterpret_cast<T*>(a.v.p) + n * a.v.row + hk * a.v.head
                  : reinterpret_cast<T*>(a.ko.p) + n * a.ko.row + hk * a.ko.head;
    store8(dst + lane * 8, a.wide, x);
  }
}

template <typename T, int F, int DH>
__device__ __forceinline__ void read_values(const RowsArgs& a, int block, char* lds) {
  typedef typename Held<F>::type H;
  typedef Slices<T, DH> S;
  const int ps = a.cache.page_shift, lane = threadIdx.x & 63;
  const ValueRow r = value_row(a, block);
  const uint64_t rows = __ballot(r.live);
  char* dst = a.v.p + (r.n * a.v.row + r.h * a.v.head) * (int64_t)sizeof(T);
  const H* src = reinterpret_cast<const H*>(a.cache.v) + ((r.block * DH) << ps) + r.slot;
  float s = 0.f;
  if constexpr (is_coded(F)) s = r.block >= 0 ? a.cache.vs[(r.block << ps) + r.slot] : 0.f;
#pragma unroll
  for (int c = 0; c < S::C; ++c) {
    wave_sync();
#pragma unroll
    for (int j = 0; j < S::V; j += 8) {
      float x[8] = {};
      if (r.block >= 0) {
        const H* p = src + ((int64_t)(c * S::V + j) << ps);
        if constexpr (is_coded(F)) {
          uint32_t v[2] = {0, 0};
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e / 4] |= (uint32_t)(uint8_t)p[(int64_t)e << ps] << (8 * (e & 3));
          decode4<F>(v[0], x);
          decode4<F>(v[1], x + 4);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= s;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = (float)p[(int64_t)e << ps];
        }
      }
      store8(reinterpret_cast<T*>(lds + lane * kPitch) + j, 1, x);
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < S::P; ++i) {
      const int row = i * S::RP + lane / S::P;
      const u32x4 w = *reinterpret_cast<const u32x4*>(lds + row * kPitch + (lane % S::P) * 16);
      char* p = address_of(dst, row) + c * kSlice + (lane % S::P) * 16;
      if (!(rows >> row & 1)) continue;
      if (a.wide) {
        *reinterpret_cast<u32x4*>(p) = w;
      } else {
        const T* d = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) reinterpret_cast<T*>(p)[e] = d[e];
      }
    }
  }
}

template <typename T, int F, int DH>
__global__ void __launch_bounds__(kThreads) read_kernel(RowsArgs a) {
  __shared__ __attribute__((aligned(16))) char stage[kThreads / 64][64 * kPitch];
  // values first: what a write left last is read first, from the caches (two
  // bf16 memories written and read back 120 us, else 124; 8 in fp8 161 and 164)
  const int nv = (int)gridDim.x - a.qk_blocks;
  if ((int)blockIdx.x >= nv) read_keys<T, F, DH>(a, blockIdx.x - nv);
  else read_values<T, F, DH>(a, blockIdx.x, stage[threadIdx.x >> 6]);
}

// How a launch is divided.  Values go the way of keys, a group of lanes a row,
// where the waves of 64 rows of their own would not fill the device.
// Else the part that takes a token's heads in turn: as few groups of heads as
// still fill the device.
template <int DH> int divide(RowsArgs* a, bool values) {
  constexpr int per = kThreads / (DH / 8);  // tokens of a workgroup
  const int64_t waves = values ? ((int64_t)a->rows.n_rows + 63) / 64 * a->n_kv_heads : 0;
  const bool by_rows = values && waves < kValueWaves;
  a->heads_by_rows = a->n_heads + a->n_kv_heads + (by_rows ? a->n_kv_heads : 0);
  const int64_t blocks = ((int64_t)a->rows.n_rows + per - 1) / per;
  a->head_groups = (int)std::max<int64_t>(1, std::min<int64_t>(a->heads_by_rows, (kFill + blocks - 1) / blocks));
  a->qk_blocks = (int)(blocks * a->head_groups);
  a->by_groups = Divisor::of(a->head_groups);
  a->by_kv_heads = Divisor::of(std::max(a->n_kv_heads, 1));
  return a->qk_blocks + (by_rows ? 0 : (int)((waves + kThreads / 64 - 1) / (kThreads / 64)));
}

template <typename T, int F, int DH>
hipError_t launch_rows_as(RowsArgs a, hipStream_t stream) {
  const int blocks = divide<DH>(&a, F != kNone);
  hipLaunchKernelGGL((rows_kernel<T, F, DH>), dim3(blocks), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int F, int DH>
hipError_t launch_read_as(RowsArgs a, hipStream_t stream) {
  const int blocks = divide<DH>(&a, true);
  hipLaunchKernelGGL((read_kernel<T, F, DH>), dim3(blocks), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

#define EVO_ROW_TYPES(X, DH)      \
  X(EVO_FP32, float, EVO_CACHE_FP32, DH)  \
  X(EVO_FP32, float, EVO_CACHE_INT8, DH)  \
  X(EVO_FP32, float, EVO_CACHE_FP8, DH)   \
  X(EVO_BF16, __bf16, EVO_CACHE_BF16, DH) \
  X(EVO_BF16, __bf16, EVO_CACHE_INT8, DH) \
  X(EVO_BF16, __bf16, EVO_CACHE_FP8, DH)

}  // namespace

hipError_t launch_rows(int dtype, int format, int head_dim, RowsArgs a, hipStream_t stream) {
#define X(D, T, F, DH) \
  if (dtype == D && format == F && head_dim == DH) return launch_rows_as<T, F, DH>(a, stream);
#define Y(DH)                                   \
  EVO_ROW_TYPES(X, DH)                          \
  X(EVO_FP32, float, kNone, DH)                 \
  X(EVO_BF16, __bf16, kNone, DH)
  Y(32) Y(64) Y(128)
#undef Y
#undef X
  return hipErrorInvalidValue;
}

hipError_t launch_cache_read(int dtype, int format, int head_dim, RowsArgs a, hipStream_t stream) {
#define X(D, T, F, DH) \
  if (dtype == D && format == F && head_dim == DH) return launch_read_as<T, F, DH>(a, stream);
  EVO_ROW_TYPES(X, 32) EVO_ROW_TYPES(X, 64) EVO_ROW_TYPES(X, 128)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace evo
