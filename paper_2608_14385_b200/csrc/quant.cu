// Products with 4-bit matrices of group scales: out[r] = W[e(r)] x[src(r)], optionally through SwiGLU.
//
//   W[i, c] = s[i, c / G] (q[i, c] - z[i, c / G])   =>   (W x)[i] = sum_g s[i, g] sum_{c in g} (q - z) x[c]
//
// so the group scale multiplies an fp32 sum and no weight is ever rounded.  A decode step has a few rows per matrix:
// the codes (half a byte a weight, read once) bound it.
#include <climits>

#include "row.cuh"

namespace deamoe {

struct QuantArgs {
  const uint8_t* codes;
  const void* scales;
  const uint8_t* zeros;
  const void* x;
  int64_t xs;
  const int32_t *expert_off, *row_pair;
  void* out;
  int64_t os;
  int n_expert, n_out, n_in, group, groups, n_token, ppt, n_rows, swiglu, scale_f32;
};

static __device__ __forceinline__ float quant_scale(const QuantArgs& A, size_t i) {
  return A.scale_f32 ? reinterpret_cast<const float*>(A.scales)[i]
                     : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(A.scales)[i]);
}

// One warp per value of the output, 8 columns a lane and step.
template <typename T> __global__ void __launch_bounds__(256) k_quant_simple(QuantArgs A) {
  const int lane = threadIdx.x & 31;
  const int width = A.swiglu ? A.n_out / 2 : A.n_out;
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t r = blockIdx.y;
  if (i >= width) return;
  int e = 0;
  if (A.expert_off) {
    int lo = 0, hi = A.n_expert;  // the last e with expert_off[e] <= r
    while (hi - lo > 1) {
      const int m = (lo + hi) / 2;
      if (A.expert_off[m] <= r) lo = m; else hi = m;
    }
    e = lo;
    if (r < A.expert_off[e] || r >= A.expert_off[e + 1]) return;
  }
  const int64_t src = A.row_pair ? A.row_pair[r] / A.ppt : r;
  const bool have = src >= 0 && src < A.n_token && (!A.row_pair || A.row_pair[r] >= 0);
  float v[2] = {0.f, 0.f};
  for (int half = 0; half < (A.swiglu ? 2 : 1); ++half) {
    const size_t row = (size_t)e * A.n_out + i + (half ? width : 0);
    const uint32_t* q = reinterpret_cast<const uint32_t*>(A.codes + row * (A.n_in / 2));
    for (int w = lane; have && w < A.n_in / 8; w += 32) {
      const uint32_t word = q[w];
      const size_t g = row * A.groups + (size_t)w * 8 / A.group;
      const int z = A.zeros ? A.zeros[g] & 15 : 8;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        s = fmaf((float)((int)((word >> (4 * j)) & 15) - z), to_f<T>(reinterpret_cast<const T*>(A.x)[src * A.xs + w * 8 + j]), s);
      v[half] = fmaf(quant_scale(A, g), s, v[half]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[half] += __shfl_xor_sync(0xffffffffu, v[half], o);
  }
  if (lane == 0)
    reinterpret_cast<T*>(A.out)[r * A.os + i] = from_f<T>(A.swiglu ? silu_f(v[0]) * v[1] : v[0]);
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_quant_workspace(int32_t dtype, int32_t n_token, int32_t n_in) {
  (void)dtype; (void)n_token; (void)n_in;
  return 0;
}

deamoe_status_t deamoe_quant_product(void* cuda_stream, int32_t dtype, const uint8_t* codes, int32_t scale_dtype,
                                     const void* scales, const uint8_t* zeros, int32_t n_expert, int32_t n_out,
                                     int32_t n_in, int32_t group, const void* x, int64_t x_stride, int32_t n_token,
                                     const int32_t* expert_off, const int32_t* row_pair, int32_t pairs_per_token,
                                     int32_t n_rows, int32_t swiglu, void* out, int64_t out_stride, void* workspace,
                                     uint64_t workspace_bytes) {
  if (!known_type(dtype) || !known_type(scale_dtype) || n_expert <= 0 || n_out <= 0 || n_in <= 0 || pairs_per_token <= 0 ||
      (swiglu != 0 && swiglu != 1) || (group != 32 && group != 64 && group != 128) || (!expert_off && n_expert != 1))
    return DEAMOE_ERR_INVALID_ARG;
  if (n_in % 32 != 0 || (swiglu && n_out % 2 != 0) || n_expert > DEAMOE_MAX_EXPERTS || n_in > DEAMOE_MAX_WIDTH ||
      n_out > DEAMOE_MAX_WIDTH)
    return DEAMOE_ERR_UNSUPPORTED;
  if (n_rows < 0 || n_token < 0) return DEAMOE_ERR_BATCH;
  if (n_rows == 0) return DEAMOE_OK;
  const size_t es = type_bytes(dtype);
  const int width = swiglu ? n_out / 2 : n_out;
  if (!codes || !aligned16(codes) || !scales || !aligned_to(scales, type_bytes(scale_dtype)) ||
      (n_token > 0 && (!x || !aligned_to(x, es) || x_stride < n_in)) || !out || !aligned_to(out, es) || out_stride < width ||
      out == x || !aligned_to(expert_off, 4) || !aligned_to(row_pair, 4))
    return DEAMOE_ERR_INVALID_ARG;
  const uint64_t need = deamoe_quant_workspace(dtype, n_token, n_in);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return DEAMOE_ERR_INVALID_ARG;
  QuantArgs A;
  A.codes = codes; A.scales = scales; A.zeros = zeros; A.x = x; A.xs = x_stride; A.expert_off = expert_off;
  A.row_pair = row_pair; A.out = out; A.os = out_stride; A.n_expert = n_expert; A.n_out = n_out; A.n_in = n_in;
  A.group = group; A.groups = (n_in + group - 1) / group; A.n_token = n_token; A.ppt = pairs_per_token; A.n_rows = n_rows;
  A.swiglu = swiglu; A.scale_f32 = scale_dtype == DEAMOE_F32;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (n_rows > 65535) return DEAMOE_ERR_BATCH;
  const dim3 grid((width + 7) / 8, n_rows);
  if (dtype == DEAMOE_F32) k_quant_simple<float><<<grid, 256, 0, s>>>(A);
  else k_quant_simple<__nv_bfloat16><<<grid, 256, 0, s>>>(A);
  return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA;
}

}  // extern "C"
