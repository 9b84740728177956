// Norms after a block and before the next, with the block's gate and the residual
// between them, in one pass over the rows (evo_block_norm).
//
// A row lies over LPR lanes (a part of a wave, a wave, or up to 16 of them), 8 values
// a lane and chunk, and stays in registers from its load to its stores: sums
// of squares, and for layer norms sums first, are lane exchanges (and a word of LDS for
// each wave where several share a row).
//
// What bounds it: memory (65537 rows of 1024, fp32 stream and bf16 blocks, each with its
// modulation: 148 us, 5.4 TB/s, where a copy has 4.92), latencies for few rows (16 rows of
// 256: 4.3 us in a recorded graph; requesting gains and modulation with the row saved 5%
// and cost wide rows their registers).  Where d is no multiple of 8 or some row does not lie
// at 16 bytes, all of a call's arrays go value by value, which the memory's transactions
// bound (4099 bf16 rows of 1021 37 us, of 1016 11; 65537 of 1023, fp32 stream, 550, of 1016
// 163).
#include <hip/hip_runtime.h>

#include "evo.h"
#include "evo_layers.hpp"

namespace evo {
namespace {

constexpr int kThreads = 256;
constexpr int kFewRows = 1500;

// 8 values from index `at` of a row of d; those behind its end are `fill`
template <bool WIDE> __device__ __forceinline__ void load8(const float* p, int at, int d, float fill, float* x) {
  if (WIDE) {
    if (at >= d) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fill;
      return;
    }
    const f32x4 a = *reinterpret_cast<const f32x4*>(p + at), b = *reinterpret_cast<const f32x4*>(p + at + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at + e < d ? p[at + e] : fill;
  }
}
template <bool WIDE> __device__ __forceinline__ void load8(const __bf16* p, int at, int d, float fill, float* x) {
  if (WIDE) {
    if (at >= d) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fill;
      return;
    }
    const u32x4 a = *reinterpret_cast<const u32x4*>(p + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __builtin_bit_cast(float, a[e] << 16);
      x[2 * e + 1] = __builtin_bit_cast(float, a[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at + e < d ? (float)p[at + e] : fill;
  }
}
template <bool WIDE> __device__ __forceinline__ void store8(float* p, int at, int d, const float* x) {
  if (WIDE) {
    if (at >= d) return;
    *reinterpret_cast<f32x4*>(p + at) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + at + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < d) p[at + e] = x[e];
  }
}
template <bool WIDE> __device__ __forceinline__ void store8(__bf16* p, int at, int d, const float* x) {
  if (WIDE) {
    if (at >= d) return;
    *reinterpret_cast<u32x4*>(p + at) = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < d) p[at + e] = (__bf16)x[e];
  }
}

// threads of a workgroup whose rows take so many lanes
constexpr int threads_of(int lpr) { return lpr > kThreads ? lpr : kThreads; }

// The row's sum over its lanes.  `sums`: a word for each of its waves that no other
// sum of the workgroup uses.
template <int LPR> __device__ __forceinline__ float row_sum(float x, float* sums) {
#pragma unroll
  for (int s = 1; s < (LPR < 64 ? LPR : 64); s *= 2) x += __shfl_xor(x, s);
  if constexpr (LPR > 64) {
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
    __syncthreads();
    float y[LPR / 64];
#pragma unroll
    for (int w = 0; w < LPR / 64; ++w) y[w] = sums[w];
#pragma unroll
    for (int n = LPR / 128; n >= 1; n /= 2)
#pragma unroll
      for (int w = 0; w < n; ++w) y[w] = y[2 * w] + y[2 * w + 1];
    x = y[0];
  }
  return x;
}

template <int LPR, int C, bool WIDE>
__device__ __forceinline__ void norm_row(const NormArgs& a, int kind, const float* gain, const float* bias, int lane,
                                         float (&x)[C][8], float* sums) {
  if (kind == EVO_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[c][e];
    const float mean = row_sum<LPR>(s, sums) * a.inv_d;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = (c * LPR + lane) * 8 + e < a.d ? x[c][e] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[c][e], x[c][e], s);
  const float r = 1.f / sqrtf(fmaf(row_sum<LPR>(s, sums + (LPR > 64 ? LPR / 64 : 0)), a.inv_d, a.eps));
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float g[8], b[8];
    if (gain) load8<WIDE>(gain, (c * LPR + lane) * 8, a.d, 0.f, g);
    if (bias) load8<WIDE>(bias, (c * LPR + lane) * 8, a.d, 0.f, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[c][e] *= r;
      if (gain) x[c][e] *= g[e];
      if (bias) x[c][e] += b[e];
    }
  }
}

template <typename TS, typename TB, int LPR, int C, bool WIDE>
__global__ void __launch_bounds__(threads_of(LPR)) norm_kernel(NormArgs a) {
  __shared__ float sums[LPR > 64 ? LPR / 16 : 1];
  const int lane = threadIdx.x % LPR;
  const int64_t at_row = (int64_t)blockIdx.x * (threads_of(LPR) / LPR) + threadIdx.x / LPR;
  // whole waves stay for the exchanges; rows past the end repeat the last one
  // and are not stored
  const bool live = at_row < a.n_rows;
  const int n = live ? (int)at_row : a.n_rows - 1;
  int mod = 0;
  bool known = true;
  if (a.n_mods) {
    mod = a.mod_rows ? a.mod_rows[n] : a.by_mod.divide(n);
    known = mod >= 0 && mod < a.n_mods;
    if (!known) mod = 0;
  }
  const TB* const gate = a.gate.p ? reinterpret_cast<const TB*>(a.gate.p) + mod * a.gate.row : nullptr;
  const TB* const scale = a.scale.p ? reinterpret_cast<const TB*>(a.scale.p) + mod * a.scale.row : nullptr;
  const TB* const shift = a.shift.p ? reinterpret_cast<const TB*>(a.shift.p) + mod * a.shift.row : nullptr;
  float x[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) load8<WIDE>(reinterpret_cast<const TS*>(a.x.p) + n * a.x.row, (c * LPR + lane) * 8, a.d, 0.f, x[c]);
  if (a.y.p) {
    float y[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) load8<WIDE>(reinterpret_cast<const TB*>(a.y.p) + n * a.y.row, (c * LPR + lane) * 8, a.d, 0.f, y[c]);
    if (a.post) norm_row<LPR, C, WIDE>(a, a.post, a.post_gain, a.post_bias, lane, y, sums);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float g[8];
      if (gate) load8<WIDE>(gate, (c * LPR + lane) * 8, a.d, 0.f, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = fmaf(x[c][e], a.alpha, gate ? g[e] * y[c][e] : y[c][e]);
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] *= a.alpha;
  }
  if (!known) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = __builtin_nanf("");
  }
  if (a.x_out.p && live) {
#pragma unroll
    for (int c = 0; c < C; ++c) store8<WIDE>(reinterpret_cast<TS*>(a.x_out.p) + n * a.x_out.row, (c * LPR + lane) * 8, a.d, x[c]);
  }
  if (!a.pre) return;
  norm_row<LPR, C, WIDE>(a, a.pre, a.pre_gain, a.pre_bias, lane, x, sums + (LPR > 64 ? LPR / 32 : 0));
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float m[8], t[8];
    if (scale) load8<WIDE>(scale, (c * LPR + lane) * 8, a.d, 0.f, m);
    if (shift) load8<WIDE>(shift, (c * LPR + lane) * 8, a.d, 0.f, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (scale) x[c][e] = fmaf(x[c][e], m[e], x[c][e]);
      if (shift) x[c][e] += t[e];
    }
    if (live) store8<WIDE>(reinterpret_cast<TB*>(a.h.p) + n * a.h.row, (c * LPR + lane) * 8, a.d, x[c]);
  }
}

template <typename TS, typename TB, int LPR, int C>
hipError_t launch_as(bool wide, const NormArgs& a, hipStream_t stream) {
  constexpr int rows = threads_of(LPR) / LPR;
  const dim3 grid((unsigned)(((int64_t)a.n_rows + rows - 1) / rows));
  hipLaunchKernelGGL((wide ? norm_kernel<TS, TB, LPR, C, true> : norm_kernel<TS, TB, LPR, C, false>), grid, dim3(threads_of(LPR)), 0,
                     stream, a);
  return hipGetLastError();
}

// Lanes of a row, and 8 values each so many times: as few values a lane as a workgroup
// allows (8000 rows of 8192, bf16, 134 us over 1024 lanes, 183 over 256; of 16384 318 and
// 782; 301 rows of 5120 7.4 and 8.3; one row of 8192 5.8 and 8.8).  At 1024 values two a
// lane spare the exchange between waves, which pays where rows fill the device (3000 rows
// 9.3 us, else 11.2; 1500 7.1 and 7.2; 300 6.2 and 4.9).
template <typename TS, typename TB> hipError_t launch_types(bool wide, const NormArgs& a, hipStream_t stream) {
  if (a.d <= 128) return launch_as<TS, TB, 16, 1>(wide, a, stream);
  if (a.d <= 256) return launch_as<TS, TB, 32, 1>(wide, a, stream);
  if (a.d <= 512) return launch_as<TS, TB, 64, 1>(wide, a, stream);
  if (a.d <= 1024 && a.n_rows > kFewRows) return launch_as<TS, TB, 64, 2>(wide, a, stream);
  if (a.d <= 2048) return launch_as<TS, TB, 256, 1>(wide, a, stream);
  if (a.d <= 4096) return launch_as<TS, TB, 512, 1>(wide, a, stream);
  if (a.d <= 8192) return launch_as<TS, TB, 1024, 1>(wide, a, stream);
  return launch_as<TS, TB, 1024, 2>(wide, a, stream);
}

}  // namespace

hipError_t launch_block_norm(int stream_dtype, int block_dtype, bool wide, const NormArgs& a, hipStream_t stream) {
  if (stream_dtype == EVO_BF16) return launch_types<__bf16, __bf16>(wide, a, stream);
  if (block_dtype == EVO_BF16) return launch_types<float, __bf16>(wide, a, stream);
  return launch_types<float, float>(wide, a, stream);
}

}  // namespace evo
