// Products of rows with 4-bit weights that have a power-of-two scale for each 32
// values (evo_coded_linear).
//
// The matrix instruction takes a tile of 16 weight rows and of 16 rows of x; a
// lane's share of a weight row is a whole group of 32 codes (16 bytes), with its
// scale, and becomes operands by one conversion for two values: a code times a power
// of two is exact in bf16.  Its 32 values meet the same 32 of x, so that neither side
// is rearranged.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "evo.h"
#include "evo_layers.hpp"

namespace evo {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// eight codes times 2^e as the operand of a bf16 product
__device__ __forceinline__ bf16x8 operand(uint32_t v, float scale) {
  const u32x4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 3))};
  return __builtin_bit_cast(bf16x8, w);
}

// 16 bytes of a row of x from value k on, of any alignment (one load on this
// hardware); of a row's last values, 0 behind its end
template <typename T> __device__ __forceinline__ u32x4 load16(const T* row, int k) {
  struct __attribute__((packed, aligned(sizeof(T)))) Any { u32x4 v; };
  return reinterpret_cast<const Any*>(row + k)->v;
}
template <typename T> __device__ __forceinline__ u32x4 load_last(const T* row, int k, int n_in) {
  constexpr int N = 16 / (int)sizeof(T);
  u32x4 v = {0, 0, 0, 0};
  if (n_in < N) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (k + e < n_in) {
        if (sizeof(T) == 4) v[e % 4] = reinterpret_cast<const uint32_t*>(row)[k + e];
        else v[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[k + e] << (16 * (e & 1));
      }
    return v;
  }
  // the row's last 16 bytes, moved down by what lies before k
  const int off = min(max(k - (n_in - N), 0), N), d = off * (int)sizeof(T) / 4;
  v = load16(row, min(k, n_in - N));
  if (d & 1) v = u32x4{v[1], v[2], v[3], 0};
  if (d & 2) v = u32x4{v[2], v[3], 0, 0};
  if (d & 4) v = u32x4{0, 0, 0, 0};
  if (sizeof(T) == 2 && (off & 1))
    v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  return v;
}

// Activations of results that are rounded to T.  In bf16 (half a step: 2^-8 of the
// value) they come from the hardware's exponential and reciprocal, and the normal
// distribution's tail, 1/2 erfc(z), z = |x| / sqrt(2), from exp(-z^2) t P(t), t = 1 / (1 +
// 0.44 z), P a least-squares fit of degree 5 to the scaled complement over z to 10.5:
// off by 2^-17 of the tail, and by 2^-16 with the exponential's (2049 rows of 4096
// features, GELU: 78 us, with the library's functions 86).
template <typename T> __device__ __forceinline__ float activate(float x, int act);
template <> __device__ __forceinline__ float activate<float>(float x, int act) {
  if (act == EVO_ACT_SILU) return x / (1.f + expf(-x));
  if (act == EVO_ACT_GELU) return 0.5f * x * erfcf(x * -0.70710678f);  // (no cancellation below 0)
  return x;
}
template <> __device__ __forceinline__ float activate<__bf16>(float x, int act) {
  if (act == EVO_ACT_SILU) return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504f));
  if (act == EVO_ACT_GELU) {
    const float a = fminf(fabsf(x), 14.f);  // (the tail is 0 from there on; an infinite x stays outside)
    const float t = __builtin_amdgcn_rcpf(fmaf(a, 0.44f * 0.70710678f, 1.f));
    float p = fmaf(-0.14610105f, t, 0.35063967f);
    p = fmaf(p, t, 0.04074476f);
    p = fmaf(p, t, 0.26357940f);
    p = fmaf(p, t, 0.24257124f);
    p = fmaf(p, t, 0.24856086f);
    const float tail = 0.5f * t * p * __builtin_amdgcn_exp2f(a * a * (-0.5f * 1.44269504f));
    return x * (x > 0.f ? 1.f - tail : tail);
  }
  return x;
}
__device__ __forceinline__ float scale_of(uint8_t e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }

// four outputs of a row from channel n on
template <typename T>
__device__ __forceinline__ void put(const LinearArgs& a, int row, int n, f32x4 o) {
  T* dst = reinterpret_cast<T*>(a.out.p) + row * a.out.row + n;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = activate<T>(o[e] + (a.bias && n + e < a.n_out ? a.bias[n + e] : 0.f), a.act);
  if (a.wide_out && n + 4 <= a.n_out) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(dst) = u32x2{pack2(y[0], y[1]), pack2(y[2], y[3])};
    else *reinterpret_cast<f32x4*>(dst) = f32x4{y[0], y[1], y[2], y[3]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.n_out) dst[e] = (T)y[e];
}

// ---- few rows ---------------------------------------------------------------
// A lane's 32 codes of a weight row against as many values of a row of x: 16 by 16
// products over a chunk of 128.
__device__ __forceinline__ f32x4 multiply_chunk(u32x4 codes, float scale, const u32x4 (&x)[4], f32x4 o) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(codes[j], scale), __builtin_bit_cast(bf16x8, x[j]), o, 0, 0, 0);
  return o;
}
__device__ __forceinline__ f32x4 multiply_chunk(u32x4 codes, float scale, const u32x4 (&x)[8], f32x4 o) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t v = codes[j / 2];
    const auto a = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, scale, 2) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, scale, 0);
    const auto b = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, scale, 3) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, scale, 1);
    const float w[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
    for (int e = 0; e < 4; ++e) o = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], __builtin_bit_cast(float, (uint32_t)x[j][e]), o, 0, 0, 0);
  }
  return o;
}

// Workgroup (16 C weight rows, 16 rows of x): its eight waves take chunks of 128
// values in turn, straight from memory to registers, and join their sums through LDS,
// in order.  What bounds it: memory (one row, 8192 to 8192 features: 13 us with weights
// that come from memory, 12 where the last cache has them, of the 7.2 that the codes take
// at a copy's rate and the 2.8 of the smallest launch).  C is 2
// where that leaves a workgroup for each compute unit, because x is then read half as
// often (16 rows, 8192 to 8192: 19.6 us, so 27), else 1 (one row, 4096 to 4096: 5.6,
// so 7.2).  Requesting two or four chunks at once changes nothing: three to four
// workgroups share a compute unit.
template <typename T, int C>
__global__ void __launch_bounds__(512) few_rows_kernel(LinearArgs a, int weight_tiles) {
  constexpr int NW = 8, XL = 2 * (int)sizeof(T), V = 16 / (int)sizeof(T);  // loads of a row's chunk, their values
  __shared__ __attribute__((aligned(16))) f32x4 sums[NW][C][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, g = lane >> 4;
  const int rt = blockIdx.x / weight_tiles, n0 = (blockIdx.x - rt * weight_tiles) * (16 * C), row = rt * 16 + lr;
  const uint8_t* codes[C];
  const uint8_t* scales[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int64_t n = min(n0 + c * 16 + lr, a.n_out - 1);
    codes[c] = a.codes + n * a.chunks * 64 + g * 16;
    scales[c] = a.scales + n * a.chunks * 4 + g;
  }
  const T* const x = reinterpret_cast<const T*>(a.x.p) + min(row, a.n_rows - 1) * a.x.row;
  f32x4 o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int whole = a.n_in / 128;
  for (int k = w; k < a.chunks; k += NW) {
    u32x4 v[C], xv[XL];
    uint8_t e[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      v[c] = *reinterpret_cast<const u32x4*>(codes[c] + k * 64);
      e[c] = scales[c][k * 4];
    }
#pragma unroll
    for (int j = 0; j < XL; ++j)
      xv[j] = k < whole ? load16(x, k * 128 + g * 32 + j * V) : load_last(x, k * 128 + g * 32 + j * V, a.n_in);
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = multiply_chunk(v[c], scale_of(e[c]), xv, o[c]);
  }
#pragma unroll
  for (int c = 0; c < C; ++c) sums[w][c][lane] = o[c];
  __syncthreads();
  if (w >= C) return;
  f32x4 s = sums[0][w][lane];
#pragma unroll
  for (int j = 1; j < NW; ++j) s += sums[j][w][lane];
  if (row < a.n_rows) put<T>(a, row, n0 + w * 16 + g * 4, s);
}

// ---- more rows ---------------------------------------------------------------
// Workgroup (32 CW WW weight rows, 32 RW WR rows of x): its eight waves are KS groups
// of WW by WR, each with a tile of CW by RW matrix products of 32 by 32.  A stage
// holds KS chunks of 128 values, a group's each, of rows, codes and scales in LDS.
// 16-byte pieces of an LDS row are exchanged by the row's number, so that the 16 rows of
// a reading step meet all places of 256 bytes (no bank conflicts).
//  * Codes stay codes in LDS, a quarter of the bytes of operands, and every wave
//    converts those it multiplies: two conversions to a product of 32 clocks.
//  * A stage's loads, its way to LDS, the conversions and the reading of the next step's
//    operands lie between the products of the stage two before it (2048 rows of 4096 to
//    4096 features: a stage put whole between two barriers 83 us, piece by piece 68).
//  * Results pass through LDS, so that rows are stored side by side (3 us less).
// What bounds it: 2048 rows of 4096 to 4096 features, bf16, take 64 us on inputs that
// stay in the caches, 1075 TFLOP/s, and 72 on others (a
// library product with bf16 weights 62 to 66); 4096 rows of 8192 to 8192 446 us, 1232 TFLOP/s.
// Of a round's time 12 us are start and end; the rest runs at 78% of the matrix units'
// rate where one workgroup works alone, and at 50% where all do, when the card's power
// bounds it (with rows of zeros 348 us instead of 446).
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A step of a chunk's product: 16 bytes of a row of x against as many values of a
// weight row.  A lane's half of the wave takes a group of 32 values at a time, the
// first and second groups in the first half of the steps.
template <typename T> struct Step;
template <> struct Step<__bf16> {
  static constexpr int kSteps = 8, kValues = 8;
  typedef bf16x8 X;
  typedef bf16x8 W;
  static __device__ __forceinline__ W weights(u32x4 v, int j, float scale) { return operand(v[j & 3], scale); }
  static __device__ __forceinline__ f32x16 multiply(const W& w, const X& x, f32x16 o) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x, o, 0, 0, 0);
  }
};
template <> struct Step<float> {
  static constexpr int kSteps = 16, kValues = 4;
  typedef f32x4 X;
  typedef f32x4 W;
  static __device__ __forceinline__ W weights(u32x4 v, int j, float scale) {
    const uint32_t u = v[j / 2 & 3];
    const auto a = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 2) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 0);
    const auto b = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 3) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, scale, 1);
    return W{a[0], a[1], b[0], b[1]};
  }
  static __device__ __forceinline__ f32x16 multiply(const W& w, const X& x, f32x16 o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o = __builtin_amdgcn_mfma_f32_32x32x2f32(w[e], x[e], o, 0, 0, 0);
    return o;
  }
};

constexpr int kBand = 4;
template <typename T, int CW, int RW, int WW, int WR, int KS> struct Tile {
  static constexpr int W = 32 * CW * WW, R = 32 * RW * WR;
  static constexpr int RC = 128 * (int)sizeof(T) / 16;            // pieces of a row's chunk
  static constexpr int NX = KS * R * RC, NW = KS * W * 4, NS = KS * W;
  static constexpr int X = 0, C = X + NX * 16, S = C + NW * 16, kBytes = S + NS * 4;  // a stage
  static constexpr int kJoin = (KS - 1) * WW * WR * CW * RW * 4096;
  static constexpr int kLds = 3 * kBytes > kJoin ? 3 * kBytes : kJoin;
};

template <typename T, int CW, int RW, int WW, int WR, int KS>
__global__ void __launch_bounds__(64 * WW * WR * KS, WW * WR * KS / 4) tile_kernel(LinearArgs a, int row_tiles, int tiles) {
  typedef Tile<T, CW, RW, WW, WR, KS> L;
  typedef Step<T> P;
  constexpr int ST = P::kSteps, TH = 64 * WW * WR * KS;
  static_assert(L::NX % TH == 0 && TH % (KS * L::RC) == 0, "every thread has the same piece of its rows");
  constexpr int IX = L::NX / TH, IW = (L::NW + TH - 1) / TH, IS = (L::NS + TH - 1) / TH;
  __shared__ __attribute__((aligned(16))) char lds[L::kLds];
  // A die takes neighbouring tiles (workgroup i runs on die i % 8), kBand of the rows by
  // as many of the weights as it holds at a time, so that its cache serves both (4096
  // rows of 8192 to 8192 features 446 us, with all rows first 463).
  const int per = (int)gridDim.x / 8, tile = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if (tile >= tiles) return;
  const int weight_tiles = tiles / row_tiles, band = tile / (kBand * weight_tiles), in_band = tile - band * (kBand * weight_tiles);
  const int high = min(kBand, row_tiles - band * kBand), ct = in_band / high;
  const int row0 = (band * kBand + in_band - ct * high) * L::R, n0 = ct * L::W;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, half = lane >> 5;
  const int group = w / (WW * WR), wn = w % (WW * WR) / WR * (32 * CW), wr = w % WR * (32 * RW);

  const T* x_from[IX];
  const uint8_t* w_from[IW];
  const uint8_t* s_from[IS];
  int x_to[IX], w_to[IW];
#pragma unroll
  for (int i = 0; i < IX; ++i) {
    const int at = threadIdx.x + i * TH, row = at / (KS * L::RC), p = at % (KS * L::RC);
    x_from[i] = reinterpret_cast<const T*>(a.x.p) + min(row0 + row, a.n_rows - 1) * a.x.row;
    x_to[i] = L::X + (((p / L::RC) * L::R + row) * L::RC + ((p ^ row) & (L::RC - 1))) * 16;
  }
  const int x_k = threadIdx.x % (KS * L::RC) * (16 / (int)sizeof(T));  // (the same for all of them: TH is a multiple)
#pragma unroll
  for (int i = 0; i < IW; ++i) {
    const int at = threadIdx.x + i * TH, row = at / (KS * 4), p = at % (KS * 4);
    w_from[i] = a.codes + (int64_t)min(n0 + row, a.n_out - 1) * a.chunks * 64;
    w_to[i] = L::C + (((p / 4) * L::W + row) * 4 + ((p ^ (row / 4)) & 3)) * 16;
  }
#pragma unroll
  for (int i = 0; i < IS; ++i) {
    const int at = threadIdx.x + i * TH;
    s_from[i] = a.scales + (int64_t)min(n0 + at / KS, a.n_out - 1) * a.chunks * 4;
  }
  const int w_k = threadIdx.x % (KS * 4) / 4, w_p = threadIdx.x % 4, s_k = threadIdx.x % KS;
  struct Pieces {
    u32x4 x[IX], w[IW];
    uint32_t s[IS];
  };
  const int stages = (a.chunks + KS - 1) / KS;
  // a stage's pieces, one at a time: of x, codes and scales (chunks past the last are
  // not multiplied; `full`: all values of the stage lie in the rows)
  constexpr int N = IX + IW + IS;
  const auto fetch = [&](Pieces& to, int s, int i, bool full) {
    if (i < IX) {
      to.x[i] = full ? load16(x_from[i], s * KS * 128 + x_k) : load_last(x_from[i], s * KS * 128 + x_k, a.n_in);
    } else if (i < IX + IW) {
      to.w[i - IX] = *reinterpret_cast<const u32x4*>(w_from[i - IX] + min(s * KS + w_k, a.chunks - 1) * 64 + w_p * 16);
    } else {
      struct __attribute__((packed)) Any { uint32_t v; };
      to.s[i - IX - IW] = reinterpret_cast<const Any*>(s_from[i - IX - IW] + min(s * KS + s_k, a.chunks - 1) * 4)->v;
    }
  };
  const auto put_piece = [&](char* to, const Pieces& from, int i) {
    if (i < IX) {
      *reinterpret_cast<u32x4*>(to + x_to[i]) = from.x[i];
    } else if (i < IX + IW) {
      if (L::NW % TH == 0 || (int)threadIdx.x + (i - IX) * TH < L::NW) *reinterpret_cast<u32x4*>(to + w_to[i - IX]) = from.w[i - IX];
    } else {
      const int at = threadIdx.x + (i - IX - IW) * TH;
      if (L::NS % TH == 0 || at < L::NS) *reinterpret_cast<uint32_t*>(to + L::S + ((at % KS) * L::W + at / KS) * 4) = from.s[i - IX - IW];
    }
  };
  const auto fetch_all = [&](Pieces& to, int s) {
    const bool full = (s + 1) * KS * 128 <= a.n_in;
#pragma unroll
    for (int i = 0; i < N; ++i) fetch(to, s, i, full);
  };
  const auto put_all = [&](char* to, const Pieces& from) {
#pragma unroll
    for (int i = 0; i < N; ++i) put_piece(to, from, i);
  };
  f32x16 o[CW][RW];
#pragma unroll
  for (int c = 0; c < CW; ++c)
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[c][r][e] = 0.f;

  // What a lane multiplies next: operands of two steps, and the codes and scales of
  // a chunk's halves that weights are made of.
  typename P::X x[2][RW];
  typename P::W wt[2][CW];
  u32x4 codes[2][CW];
  uint32_t exponents[2][CW];
  const int x_row = L::X + (group * L::R + wr + lr) * (L::RC * 16), w_row = group * L::W + wn + lr;
  // (the tiles' rows lie a multiple of 32 apart)
  const int turn = lr & (L::RC - 1), w_turn = (lr / 4) & 3;
  const auto read_x = [&](const char* at, int j, int r) {
    const int piece = (j / (ST / 2) * 2 + half) * (ST / 2) + j % (ST / 2);
    x[j & 1][r] = *reinterpret_cast<const typename P::X*>(at + x_row + r * 32 * (L::RC * 16) + ((piece ^ turn) * 16));
  };
  const auto read_codes = [&](const char* at, int b, int c) {
    codes[b][c] = *reinterpret_cast<const u32x4*>(at + L::C + (w_row + c * 32) * 64 + (((b * 2 + half) ^ w_turn) * 16));
    exponents[b][c] = *reinterpret_cast<const uint8_t*>(at + L::S + (w_row + c * 32) * 4 + b * 2 + half);
  };
  const auto make_weights = [&](int j, int c) {
    wt[j & 1][c] = P::weights(codes[j / (ST / 2)][c], j % (ST / 2), scale_of((uint8_t)exponents[j / (ST / 2)][c]));
  };

  // Three stages lie in LDS: stage s is multiplied, s + 1 is complete (its first
  // operands are read at the end of s) and s + 2 is put, piece by piece between
  // the products, while s + 3 is on its way to registers.
  Pieces next;
  char *now = lds, *then = lds + L::kBytes, *after = lds + 2 * L::kBytes;
  const auto stage = [&](int s, bool full) {
    const int ahead = min(s + 3, stages - 1);
    const bool mine = KS == 1 || s * KS + group < a.chunks;
#pragma unroll
    for (int j = 0; j < ST; ++j) {
      const int j1 = (j + 1) % ST;  // of the next stage at the end
      const char* const at = j + 1 < ST ? now : then;
      // work beside a step's products
      const int pieces = N > j ? (N - j + ST - 1) / ST : 0, halves = j == 0 || j == ST / 2 ? CW : 0;
      const int all = RW + CW + halves + pieces;
      const auto beside = [&](int k) {
        if (k < RW) {
          read_x(at, j1, k);
        } else if (k < RW + CW) {
          make_weights(j1, k - RW);
        } else if (k < RW + CW + halves) {
          if (j) read_codes(then, 0, k - RW - CW);
          else read_codes(now, 1, k - RW - CW);
        } else {
          const int i = j + (k - RW - CW - halves) * ST;
          put_piece(after, next, i);
          fetch(next, ahead, i, full);
        }
      };
#pragma unroll
      for (int k = 0; k < all; ++k) beside(k);
      if (mine) {
#pragma unroll
        for (int r = 0; r < RW; ++r)
#pragma unroll
          for (int c = 0; c < CW; ++c) o[c][r] = P::multiply(wt[j & 1][c], x[j & 1][r], o[c][r]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    char* const t = now;
    now = then;
    then = after;
    after = t;
  };
  {
    Pieces p0, p1;
    fetch_all(p0, 0);
    fetch_all(p1, min(1, stages - 1));
    fetch_all(next, min(2, stages - 1));
    put_all(now, p0);
    put_all(then, p1);
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CW; ++c) read_codes(now, 0, c);
#pragma unroll
  for (int r = 0; r < RW; ++r) read_x(now, 0, r);
#pragma unroll
  for (int c = 0; c < CW; ++c) make_weights(0, c);
  int s = 0;
  for (; (s + 4) * KS * 128 <= a.n_in; ++s) stage(s, true);
  for (; s < stages; ++s) stage(s, (min(s + 3, stages - 1) + 1) * KS * 128 <= a.n_in);
  if constexpr (KS > 1) {
    // the groups' sums, joined in order
    __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);
    constexpr int M = CW * RW * 4;
    if (group) {
#pragma unroll
      for (int c = 0; c < CW; ++c)
#pragma unroll
        for (int r = 0; r < RW; ++r)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            sums[((w - WW * WR) * M + (c * RW + r) * 4 + q) * 64 + lane] = f32x4{o[c][r][4 * q], o[c][r][4 * q + 1], o[c][r][4 * q + 2], o[c][r][4 * q + 3]};
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int g = 0; g < KS - 1; ++g)
#pragma unroll
        for (int c = 0; c < CW; ++c)
#pragma unroll
          for (int r = 0; r < RW; ++r)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 v = sums[((g * WW * WR + w) * M + (c * RW + r) * 4 + q) * 64 + lane];
#pragma unroll
              for (int e = 0; e < 4; ++e) o[c][r][4 * q + e] += v[e];
            }
    }
  }
  // results through LDS, so that a row's lie side by side as they are stored
  constexpr int kPitch = L::W * (int)sizeof(T) + 16, kPieces = L::W * (int)sizeof(T) / 16, V = 16 / (int)sizeof(T);
  static_assert(L::R * kPitch <= L::kLds && TH % kPieces == 0, "the results fit");
  __syncthreads();
  if (group == 0) {
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
      for (int c = 0; c < CW; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = wn + c * 32 + q * 8 + half * 4;
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = activate<T>(o[c][r][4 * q + e] + (a.bias ? a.bias[min(n0 + n + e, a.n_out - 1)] : 0.f), a.act);
          char* const to = lds + (wr + r * 32 + lr) * kPitch + n * (int)sizeof(T);
          if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to) = u32x2{pack2(y[0], y[1]), pack2(y[2], y[3])};
          else *reinterpret_cast<f32x4*>(to) = f32x4{y[0], y[1], y[2], y[3]};
        }
  }
  __syncthreads();
  const int n = threadIdx.x % kPieces * V, left = a.n_out - (n0 + n);
#pragma unroll
  for (int row = threadIdx.x / kPieces; row < L::R; row += TH / kPieces) {
    if (row0 + row >= a.n_rows) break;
    T* const dst = reinterpret_cast<T*>(a.out.p) + (row0 + row) * a.out.row + n0 + n;
    const char* const from = lds + row * kPitch + n * (int)sizeof(T);
    if (a.wide_out && left >= V) {
      *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(from);
    } else {
      for (int e = 0; e < V; ++e)
        if (e < left) dst[e] = reinterpret_cast<const T*>(from)[e];
    }
  }
}

template <typename T, int CW, int RW, int WW, int WR, int KS> void launch_tiles(const LinearArgs& a, hipStream_t stream) {
  typedef Tile<T, CW, RW, WW, WR, KS> L;
  const int rt = (a.n_rows + L::R - 1) / L::R, tiles = rt * ((a.n_out + L::W - 1) / L::W);
  hipLaunchKernelGGL((tile_kernel<T, CW, RW, WW, WR, KS>), dim3((tiles + 7) / 8 * 8), dim3(64 * WW * WR * KS), 0, stream, a, rt, tiles);
}

template <typename T, int C> void launch_few(const LinearArgs& a, hipStream_t stream) {
  const int wt = (a.n_out + 16 * C - 1) / (16 * C), tiles = wt * ((a.n_rows + 15) / 16);
  hipLaunchKernelGGL((few_rows_kernel<T, C>), dim3(tiles), dim3(512), 0, stream, a, wt);
}

// Which kernel takes a call's rows: the one whose tiles cost least, from times
// measured over 1 to 4000 rows of 100 to 8192 features (us: of a round of tiles, one
// to a compute unit, and of each of its chunks of 128 values).  The smallest tiles that
// fill the device win while rows are few, the largest where rounds are many: 64 rows
// of 4096 to 4096 features, bf16, take 24.4, 17.4, 11.9, 16.0, 22.4, 30.6 and 45.8 us in
// the order below, 1000 rows 330, 223, 85, 69, 51, 46 and 51, 4000 rows 1307, 872, 316,
// 242, 192, 171 and 131.
struct Shape {
  int rows, weights, parts;  // parts: of K in a workgroup
  float start, chunk;
  float least;  // what a round of one tile takes of that; 0: a compute unit holds several workgroups
  void (*launch)(const LinearArgs&, hipStream_t);
};
template <typename T> struct Shapes;
template <> struct Shapes<__bf16> {
  static constexpr Shape of[] = {{16, 16, 8, 0.02f, 0.168f, 0.f, launch_few<__bf16, 1>},
                                 {16, 32, 8, 0.05f, 0.225f, 0.f, launch_few<__bf16, 2>},
                                 {32, 64, 4, 4.6f, 0.18f, 0.95f, launch_tiles<__bf16, 1, 1, 2, 1, 4>},
                                 {32, 128, 2, 3.2f, 0.375f, 0.88f, launch_tiles<__bf16, 1, 1, 4, 1, 2>},
                                 {64, 128, 2, 4.8f, 0.595f, 0.8f, launch_tiles<__bf16, 2, 1, 2, 2, 2>},
                                 {128, 128, 1, 4.f, 1.16f, 0.65f, launch_tiles<__bf16, 1, 2, 4, 2, 1>},
                                 {128, 256, 1, 10.f, 1.7f, 0.68f, launch_tiles<__bf16, 2, 2, 4, 2, 1>}};
};
template <> struct Shapes<float> {
  static constexpr Shape of[] = {{16, 16, 8, 0.05f, 0.36f, 0.f, launch_few<float, 1>},
                                 {16, 32, 8, 0.3f, 0.375f, 0.f, launch_few<float, 2>},
                                 {32, 128, 2, 5.f, 2.15f, 0.97f, launch_tiles<float, 1, 1, 4, 1, 2>},
                                 {64, 256, 1, 6.f, 7.85f, 0.97f, launch_tiles<float, 2, 1, 4, 2, 1>}};
};
constexpr float kLaunch = 2.f;
float cost(const Shape& s, int64_t rows, const LinearArgs& a, int n_cu) {
  const int64_t tiles = ((rows + s.rows - 1) / s.rows) * ((a.n_out + s.weights - 1) / s.weights);
  float rounds = (float)tiles / (float)n_cu;
  if (s.least > 0.f) {
    const float whole = floorf(rounds), rest = rounds - whole;
    rounds = whole + (rest > 0.f ? s.least + (1.f - s.least) * rest : 0.f);
  } else {
    rounds = std::max(rounds, 1.f);
  }
  return kLaunch + rounds * (s.start + s.chunk * (float)a.chunks);
}
template <typename T> const Shape* cheapest(int64_t rows, const LinearArgs& a, int n_cu, float* least) {
  const Shape* best = nullptr;
  for (const Shape& s : Shapes<T>::of) {
    const float c = cost(s, rows, a, n_cu);
    if (!best || c < *least) { best = &s; *least = c; }
  }
  return best;
}

// The launches of a call: `rest` takes what `first` (or NULL) leaves.
struct Launches {
  const Shape* first;
  int first_rows;
  const Shape* rest;
};
template <typename T> Launches plan(const LinearArgs& a, int n_cu) {
  // Rows that fill whole rounds may go before the rest, in a launch of their own:
  // 2049 rows of 4096 to 4096 features in tiles of 128 by 256 alone 109 us, split 75.
  float least;
  Launches p = {nullptr, 0, cheapest<T>(a.n_rows, a, n_cu, &least)};
  for (const Shape& s : Shapes<T>::of) {
    if (s.least == 0.f) continue;
    const int64_t wt = (a.n_out + s.weights - 1) / s.weights, rt = a.n_rows / s.rows;
    for (int64_t n : {rt * wt / n_cu * n_cu / wt, rt}) {
      const int64_t rows = n * s.rows;
      if (!rows || rows >= a.n_rows) continue;
      float c;
      const Shape* other = cheapest<T>(a.n_rows - rows, a, n_cu, &c);
      c += cost(s, rows, a, n_cu);
      if (c < least) { least = c; p = {&s, (int)rows, other}; }
    }
  }
  return p;
}

template <typename T> hipError_t launch_as(const LinearArgs& a, int n_cu, hipStream_t stream) {
  const Launches p = plan<T>(a, n_cu);
  LinearArgs b = a;
  if (p.first) {
    b.n_rows = p.first_rows;
    p.first->launch(b, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    b = a;
    b.n_rows -= p.first_rows;
    b.x.p += p.first_rows * b.x.row * (int64_t)sizeof(T);
    b.out.p += p.first_rows * b.out.row * (int64_t)sizeof(T);
  }
  p.rest->launch(b, stream);
  return hipGetLastError();
}

template <typename T> int describe_as(const LinearArgs& a, int n_cu, int32_t* out) {
  const Launches p = plan<T>(a, n_cu);
  constexpr int kinds = sizeof(Shapes<T>::of) / sizeof(Shape);
  *out++ = kinds;
  int n = 0;
  const auto add = [&](const Shape* s, int rows) {
    for (int v : {(int)(s - Shapes<T>::of), rows, s->rows, s->weights, s->parts}) *out++ = v;
    ++n;
  };
  if (p.first) add(p.first, p.first_rows);
  add(p.rest, a.n_rows - p.first_rows);
  return n;
}

}  // namespace

hipError_t launch_linear4(int dtype, int n_cu, const LinearArgs& a, hipStream_t stream) {
  return dtype == EVO_BF16 ? launch_as<__bf16>(a, n_cu, stream) : launch_as<float>(a, n_cu, stream);
}

int describe_linear4(int dtype, int n_cu, const LinearArgs& a, int32_t* out) {
  return dtype == EVO_BF16 ? describe_as<__bf16>(a, n_cu, out) : describe_as<float>(a, n_cu, out);
}

}  // namespace evo
