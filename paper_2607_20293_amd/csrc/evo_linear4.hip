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

// the 8 values of a row of x that a lane multiplies at a time
template <typename T> struct Part;
template <> struct Part<__bf16> { bf16x8 v; };
template <> struct Part<float> { float v[8]; };

__device__ __forceinline__ f32x4 multiply(uint32_t codes, float scale, const Part<__bf16>& x, f32x4 o) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(codes, scale), x.v, o, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(uint32_t codes, float scale, const Part<float>& x, f32x4 o) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
             c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  const float w[8] = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#pragma unroll
  for (int e = 0; e < 8; ++e) o = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x.v[e], o, 0, 0, 0);
  return o;
}

// values k .. k + 7 of a row of x, 0 behind its end
__device__ __forceinline__ void load_part(const __bf16* row, int k, int n_in, int wide, Part<__bf16>& x) {
  if (wide && k + 8 <= n_in) {
    x.v = *reinterpret_cast<const bf16x8*>(row + k);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = k + e < n_in ? row[k + e] : (__bf16)0.f;
}
__device__ __forceinline__ void load_part(const float* row, int k, int n_in, int wide, Part<float>& x) {
  if (wide && k + 8 <= n_in) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(row + k), b = *reinterpret_cast<const f32x4*>(row + k + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x.v[e] = a[e]; x.v[4 + e] = b[e]; }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = k + e < n_in ? row[k + e] : 0.f;
}

__device__ __forceinline__ float activate(float x, int act) {
  if (act == EVO_ACT_SILU) return x / (1.f + expf(-x));
  if (act == EVO_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678f));
  return x;
}
__device__ __forceinline__ float scale_of(uint8_t e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }

// four outputs of a row from channel n on
template <typename T>
__device__ __forceinline__ void put(const LinearArgs& a, int row, int n, f32x4 o) {
  T* dst = reinterpret_cast<T*>(a.out.p) + row * a.out.row + n;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = activate(o[e] + (a.bias && n + e < a.n_out ? a.bias[n + e] : 0.f), a.act);
  if (a.wide_out && n + 4 <= a.n_out) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(dst) = u32x2{pack2(y[0], y[1]), pack2(y[2], y[3])};
    else *reinterpret_cast<f32x4*>(dst) = f32x4{y[0], y[1], y[2], y[3]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.n_out) dst[e] = (T)y[e];
}

// Workgroup (16 weight rows, 16 R rows of x): its NW waves take chunks of 128
// values in turn and join their sums through LDS, in order.
template <typename T, int R, int NW>
__global__ void __launch_bounds__(NW * 64) few_rows_kernel(LinearArgs a) {
  __shared__ __attribute__((aligned(16))) f32x4 sums[NW][R][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, row0 = blockIdx.y * (16 * R);
  const int64_t n = min(n0 + lr, a.n_out - 1);
  const uint8_t* const codes = a.codes + n * a.chunks * 64 + g * 16;
  const uint8_t* const scales = a.scales + n * a.chunks * 4 + g;
  const T* x[R];
#pragma unroll
  for (int r = 0; r < R; ++r) x[r] = reinterpret_cast<const T*>(a.x.p) + min(row0 + r * 16 + lr, a.n_rows - 1) * a.x.row;
  f32x4 o[R];
#pragma unroll
  for (int r = 0; r < R; ++r) o[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int c = w; c < a.chunks; c += NW) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(codes + (int64_t)c * 64);
    const float scale = scale_of(scales[c * 4]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        Part<T> p;
        load_part(x[r], c * 128 + g * 32 + j * 8, a.n_in, a.wide_x, p);
        o[r] = multiply(v[j], scale, p, o[r]);
      }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) sums[w][r][lane] = o[r];
  __syncthreads();
  for (int r = w; r < R; r += NW) {
    f32x4 s = sums[0][r][lane];
    for (int i = 1; i < NW; ++i) s += sums[i][r][lane];
    const int row = row0 + r * 16 + lr;
    if (row < a.n_rows) put<T>(a, row, n0 + g * 4, s);
  }
}

template <typename T> hipError_t launch_as(const LinearArgs& a, hipStream_t stream) {
  const unsigned tiles = (unsigned)((a.n_out + 15) / 16);
  if (a.n_rows <= 16)
    hipLaunchKernelGGL((few_rows_kernel<T, 1, 8>), dim3(tiles, (a.n_rows + 15) / 16), dim3(512), 0, stream, a);
  else
    hipLaunchKernelGGL((few_rows_kernel<T, 4, 8>), dim3(tiles, (a.n_rows + 63) / 64), dim3(512), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear4(int dtype, int n_cu, const LinearArgs& a, hipStream_t stream) {
  (void)n_cu;
  return dtype == EVO_BF16 ? launch_as<__bf16>(a, stream) : launch_as<float>(a, stream);
}

}  // namespace evo
