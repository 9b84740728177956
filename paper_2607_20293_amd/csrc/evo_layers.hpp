// Interface between the entry points of the layers around the attention
// (evo_layers.hip) and their kernels: products with 4-bit weights (evo_linear4.hip)
// and norms around a block (evo_block_norm.hip).
#pragma once

#include "evo_memory.hpp"

namespace evo {

struct MatrixView {
  char* p;
  int64_t row;  // stride in elements
};

struct NormArgs {
  MatrixView x, y, x_out, h;  // y, x_out, h: p NULL where there is none
  MatrixView gate, scale, shift;
  const float* post_gain;
  const float* post_bias;
  const float* pre_gain;
  const float* pre_bias;
  const int32_t* mod_rows;
  int n_rows, d, n_mods;
  int post, pre;
  float alpha, eps, inv_d;
  Divisor by_mod;             // rows of a modulation row, without mod_rows
};
// wide: every row of every matrix 16-byte aligned, d a multiple of 8
hipError_t launch_block_norm(int stream_dtype, int block_dtype, bool wide, const NormArgs& a, hipStream_t stream);

struct LinearArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  MatrixView x, out;
  const float* bias;
  int n_rows, n_in, n_out, chunks;  // chunks: of 128 values of a weight row
  int act;
  int wide_out;                     // rows of out 16-byte aligned
};
hipError_t launch_linear4(int dtype, int n_cu, const LinearArgs& a, hipStream_t stream);
// Its launches, as evo_debug_linear_plan tells them.
int describe_linear4(int dtype, int n_cu, const LinearArgs& a, int32_t* out);

}  // namespace evo
