// The second half of a product whose tiles were too few to fill the device and were dealt along k (matmul.cu): the parts' fp32
// sums are added in their order and go through the epilogue.  A thread takes 8 columns of a row; the parts come from the L2,
// where the kernel before has just left them.
#include "matmul.cuh"

namespace deamoe {

namespace {

constexpr int JT = 256;

template <bool DUAL> __global__ void __launch_bounds__(JT) k_join(const __grid_constant__ JoinArgs A) {
  pdl_trigger();
  const int packs = (A.M + 7) / 8, width = packs * (DUAL ? 16 : 8);
  const int64_t i = (int64_t)blockIdx.x * JT + threadIdx.x;
  const int64_t row = i / packs;
  const int m = (int)(i % packs) * 8, n = min(8, A.M - m);
  bool mine = row < A.n_rows;
  if (A.off) {
    bool falls = false;
    for (int e = threadIdx.x; e < A.groups; e += JT) falls |= A.off[e + 1] < A.off[e];
    if (__syncthreads_or(falls)) mine = false;
    mine = mine && row >= A.off[0] && row < A.off[A.groups];
  }
  pdl_wait();
  if (!mine) return;
  const int64_t step = (int64_t)A.n_rows * width;
  const float* p = A.part + row * width + (DUAL ? 2 * m : m);
  float v[8], up[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = up[j] = 0.f;
#pragma unroll 4
  for (int s = 0; s < A.splits; ++s, p += step) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    if constexpr (DUAL) {
      const float4 c = __ldcg(reinterpret_cast<const float4*>(p) + 2), d = __ldcg(reinterpret_cast<const float4*>(p) + 3);
      up[0] += c.x; up[1] += c.y; up[2] += c.z; up[3] += c.w; up[4] += d.x; up[5] += d.y; up[6] += d.z; up[7] += d.w;
    }
  }
  if constexpr (DUAL) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = silu_f(v[j]) * up[j];
  } else {
    const float xs = A.x_scale ? A.x_scale[row] : 1.f;
    const __nv_bfloat16* add = reinterpret_cast<const __nv_bfloat16*>(A.residual) + row * A.rs + m;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) {
        if (A.x_scale) v[j] *= xs * A.w_scale[m + j];
        if (A.bias)
          v[j] += A.bias_f32 ? reinterpret_cast<const float*>(A.bias)[m + j] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(A.bias)[m + j]);
        v[j] = sigma_f(A.act, v[j]);
        if (A.residual) v[j] += __bfloat162float(add[j]);
      }
  }
  __nv_bfloat16* out = A.out + row * A.os + m;
  if (A.wide && n == 8) {
    Pack<__nv_bfloat16, 8> o;
    o.narrow(v);
    store_pack(out, o);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) out[j] = __float2bfloat16_rn(v[j]);
  }
}

}  // namespace

cudaError_t join_launch(const JoinArgs& a, cudaStream_t s) {
  const int64_t work = (int64_t)a.n_rows * ((a.M + 7) / 8);
  const dim3 grid((unsigned)((work + JT - 1) / JT));
  return a.dual ? launch_pdl(k_join<true>, grid, dim3(JT), 0, s, a) : launch_pdl(k_join<false>, grid, dim3(JT), 0, s, a);
}

}  // namespace deamoe
