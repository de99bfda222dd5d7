// Products of a few rows with bf16 or e4m3 matrices (a decode step's): the forms of ffn.cu and product.cu below
// THIN_ROWS rows in all.
#pragma once
#include "row.cuh"

namespace deamoe {

constexpr int THIN_ROWS = 16;

struct ThinArgs {
  const void *x, *w;
  int64_t xs;              // row stride of x in values
  int M, K;                // columns of the output (rows of w; DUAL: features, w has 2 M rows); length of a row
  int n_rows, groups;
  const int32_t* off;      // [groups + 1] rows of the groups, or null
  __nv_bfloat16* out;
  int64_t os;
  const float *x_scale, *w_scale;
  const void *bias, *residual;
  int64_t rs;
  int bias_f32, act;
};

// dual: w's first M rows are the gate, the others the up projection, out = silu(gate) up
cudaError_t thin_launch(bool e4m3, bool dual, const ThinArgs& a, cudaStream_t s, bool chained);

}  // namespace deamoe
