// Matrix products with bias, activation and residual in their epilogue, from bf16 or from e4m3 values with a scale a row, and
// the gradients of the bf16 form.
//
//   out = act(z) + residual,  z = x W^T (sx sw) + b
//   dz = dout act'(z),  dx = dz W,  dW = dz^T x,  db = sum over tokens of dz
//
// Per-row scales of both operands leave the sum as one factor a token and one a column, so the 8-bit product is the bf16
// one with operands half as wide.  Gradients: z is recomputed from the forward's inputs in fp32; dz is rounded to bf16 as an
// operand of the two products behind it, db is summed from the unrounded dz.  Without an activation dz is dout itself and no
// product but dx and dW runs.
#include "matmul.cuh"
#include "thin.cuh"

namespace deamoe {

constexpr int BIAS_ROWS = 64;  // rows of dout that one block adds up

// Column sums of bf16 rows: a block adds BIAS_ROWS rows of 256 columns (8 a thread, 8 threads along the rows), part[block row][column].
__global__ void __launch_bounds__(256) k_bias_sums(const __nv_bfloat16* __restrict__ d, int64_t stride, int T, int n, float* __restrict__ part) {
  __shared__ float buf[8][256];
  pdl_trigger();
  const int q = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int c = blockIdx.y * 256 + q * 8;
  const int64_t t0 = (int64_t)blockIdx.x * BIAS_ROWS;
  float s[8] = {};
  if (c < n)
#pragma unroll
    for (int i = 0; i < BIAS_ROWS / 8; ++i) {
      const int64_t t = t0 + r + 8 * i;
      if (t < T) {
        float f[8];
        load_pack<__nv_bfloat16, 8>(d + t * stride + c).widen(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += f[j];
      }
    }
#pragma unroll
  for (int j = 0; j < 8; ++j) buf[r][q * 8 + j] = s[j];
  __syncthreads();
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v += buf[i][threadIdx.x];
  const int col = blockIdx.y * 256 + threadIdx.x;
  if (col < n) part[(int64_t)blockIdx.x * n + col] = v;
}
// Partial sums added in their order: 32 columns a block, 8 threads a column.  late: as in matmul.cu.
__global__ void __launch_bounds__(256) k_add_parts(const float* part, int parts, int n, float* __restrict__ out, int late) {
  __shared__ float buf[8][32];
  const int q = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + q;
  if (!late) pdl_wait();
  pdl_trigger();
  float s = 0.f;
  if (c < n)
    for (int i = r; i < parts; i += 8) s += __ldcg(part + (int64_t)i * n + c);
  buf[r][q] = s;
  __syncthreads();
  if (r == 0 && c < n) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += buf[i][q];
    out[c] = s;
  }
  if (late) pdl_wait();
}

static uint64_t ceil256(uint64_t v) { return (v + 255) / 256 * 256; }

static MatmulCall product_call(int M, int K, int N, int chunk, bool whole) {
  MatmulCall c = {};
  c.args.M = M; c.args.K = K; c.args.N = N; c.args.groups = 1; c.args.chunk = chunk;
  c.args.splits = 1;
  c.args.tile_n = matmul_tile_n(N, (M + MM_M - 1) / MM_M, whole);
  return c;
}

static int product_splits(const MatmulArgs& a) {
  return matmul_splits((int64_t)((a.M + MM_M - 1) / MM_M) * ((a.N + a.tile_n - 1) / a.tile_n), (a.K + a.chunk - 1) / a.chunk, a.N, a.M);
}

// Forward: bytes of the parts' sums, and of those of contractions of more than one stretch
static uint64_t parts_bytes(const MatmulArgs& a) {
  const int splits = product_splits(a);
  return splits > 1 ? (uint64_t)splits * a.N * ((a.M + 7) / 8 * 8) * 4 : 0;
}
static uint64_t product_sums(const MatmulArgs& a) { return matmul_sums(a.K, a.chunk, product_splits(a)); }
// Backward, for each of the two that can overlap (dx and dW)
static uint64_t backward_sums(int T, int n_out, int n_in) {
  const int k = n_out > n_in ? n_out : n_in;
  return matmul_sums(k > T ? k : T, 64, 1);
}

static deamoe_status_t check_product(int dtype, int T, int n_out, int n_in, int act, int bias_dtype, const void* bias) {
  if ((dtype != DEAMOE_BF16 && dtype != DEAMOE_E4M3) || n_out <= 0 || n_in <= 0 || act < DEAMOE_SIGMA_NONE || act > DEAMOE_SIGMA_GELU ||
      !known_type(bias_dtype) || !aligned_to(bias, type_bytes(bias_dtype)))
    return DEAMOE_ERR_INVALID_ARG;
  if (n_in % (dtype == DEAMOE_E4M3 ? 16 : 8) || n_in > DEAMOE_MAX_WIDTH || n_out > DEAMOE_MAX_WIDTH) return DEAMOE_ERR_UNSUPPORTED;
  const int64_t tiles = ((int64_t)T / 32 + 1) * ((n_out > n_in ? n_out : n_in) / MM_M + 1);  // counted in 32 bits
  if (T < 0 || T > MM_MAX_ROWS || tiles > INT32_MAX) return DEAMOE_ERR_BATCH;
  return DEAMOE_OK;
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

deamoe_status_t deamoe_product(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, const float* x_scale, int32_t n_token,
                               const void* weight, const float* weight_scale, int32_t n_out, int32_t n_in, int32_t bias_dtype,
                               const void* bias, int32_t act, const void* residual, int64_t residual_stride, void* out,
                               int64_t out_stride, void* workspace, uint64_t workspace_bytes) {
  deamoe_status_t st = check_product(dtype, n_token, n_out, n_in, act, bias_dtype, bias);
  if (st != DEAMOE_OK || n_token == 0) return st;
  const bool e4m3 = dtype == DEAMOE_E4M3;
  if (!x || !weight || !out || !aligned16(x) || !aligned16(weight) || x_stride < n_in || x_stride % (e4m3 ? 16 : 8) ||
      (e4m3 ? !x_scale || !weight_scale || !aligned_to(x_scale, 4) || !aligned_to(weight_scale, 4) : x_scale || weight_scale) ||
      !aligned_to(out, 2) || out_stride < n_out || out == x || out == weight || !aligned_to(residual, 2) ||
      (residual && residual_stride < n_out) || (residual == out && residual && residual_stride != out_stride))
    return DEAMOE_ERR_INVALID_ARG;
  const uint64_t need = deamoe_product_workspace(dtype, n_token, n_out, n_in, act, 0);
  if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return DEAMOE_ERR_INVALID_ARG;
  if (n_token <= THIN_ROWS) {
    ThinArgs a = {};
    a.x = x; a.xs = x_stride; a.w = weight; a.M = n_out; a.K = n_in; a.n_rows = n_token; a.groups = 1;
    a.out = reinterpret_cast<__nv_bfloat16*>(out); a.os = out_stride; a.x_scale = x_scale; a.w_scale = weight_scale;
    a.bias = bias; a.bias_f32 = bias_dtype == DEAMOE_F32; a.act = act; a.residual = residual; a.rs = residual_stride;
    if (thin_launch(e4m3, false, a, reinterpret_cast<cudaStream_t>(cuda_stream), false) == cudaSuccess) return DEAMOE_OK;
    cudaGetLastError();
    return DEAMOE_ERR_CUDA;
  }
  MatmulCall c = product_call(n_out, n_in, n_token, e4m3 ? 128 : 64, true);
  c.args.out = out; c.args.os = out_stride; c.args.wide = wide_rows(out, out_stride, n_token, 2);
  c.args.bias = bias; c.args.bias_f32 = bias_dtype == DEAMOE_F32; c.args.act = act;
  c.args.residual = residual; c.args.rs = residual_stride; c.args.wide_in = wide_rows(residual, residual_stride, n_token, 2);
  c.args.x_scale = x_scale; c.args.w_scale = weight_scale;
  const int es = e4m3 ? 1 : 2;
  if (!map_rows(&c.maps.a, weight, es, n_in, n_out, n_in, 1, n_in, 128) || !map_b(&c, x, es, n_in, n_token, x_stride)) return DEAMOE_ERR_CUDA;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  const int splits = product_splits(c.args);
  if (product_sums(c.args)) c.args.sums = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + ceil256(parts_bytes(c.args)));
  if (splits > 1) {  // few tiles: dealt along k, the parts' sums joined by a kernel of their own
    JoinArgs j = {};
    j.part = reinterpret_cast<float*>(workspace); j.splits = splits; j.n_rows = n_token; j.M = n_out; j.groups = 1;
    j.out = reinterpret_cast<__nv_bfloat16*>(out); j.os = out_stride; j.x_scale = x_scale; j.w_scale = weight_scale; j.bias = bias;
    j.residual = residual; j.rs = residual_stride; j.bias_f32 = c.args.bias_f32; j.act = act; j.wide = c.args.wide;
    c.args.splits = splits; c.args.out = workspace; c.args.os = (n_out + 7) / 8 * 8; c.args.out_group = c.args.os * n_token;
    if (matmul_launch(e4m3 ? MF_PART_E4M3 : MF_PART, c, s) == cudaSuccess && join_launch(j, s) == cudaSuccess) return DEAMOE_OK;
  } else if (matmul_launch(e4m3 ? MF_PRODUCT_E4M3 : MF_PRODUCT, c, s) == cudaSuccess) {
    return DEAMOE_OK;
  }
  cudaGetLastError();
  return DEAMOE_ERR_CUDA;
}

static uint64_t bias_parts(int64_t T, int n_out, int act) {
  // with an activation two rows of sums a tile of tokens, else one a block of rows
  return (uint64_t)(act == DEAMOE_SIGMA_NONE ? (T + BIAS_ROWS - 1) / BIAS_ROWS : MM_PARTS * ((T + MM_N_LEAST - 1) / MM_N_LEAST)) * n_out * 4;
}

static uint64_t dz_bytes(int T, int n_out, int act) { return act == DEAMOE_SIGMA_NONE ? 0 : ceil256((uint64_t)T * n_out * 2); }

uint64_t deamoe_product_workspace(int32_t dtype, int32_t n_token, int32_t n_out, int32_t n_in, int32_t act, int32_t backward) {
  if (n_token <= 0 || n_out <= 0 || n_in <= 0) return 0;
  if (!backward) {
    if (n_token <= THIN_ROWS) return 0;
    const MatmulArgs a = product_call(n_out, n_in, n_token, dtype == DEAMOE_E4M3 ? 128 : 64, true).args;
    return ceil256(parts_bytes(a)) + product_sums(a);
  }
  return ceil256(bias_parts(n_token, n_out, act)) + dz_bytes(n_token, n_out, act) + 2 * backward_sums(n_token, n_out, n_in);
}

deamoe_status_t deamoe_product_backward(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, int32_t n_token,
                                        const void* weight, int32_t n_out, int32_t n_in, int32_t bias_dtype, const void* bias,
                                        int32_t act, const void* dout, int64_t dout_stride, void* dx, int64_t dx_stride,
                                        void* dweight, float* dbias, void* workspace, uint64_t workspace_bytes) {
  deamoe_status_t st = check_product(dtype, n_token, n_out, n_in, act, bias_dtype, bias);
  if (st != DEAMOE_OK) return st;
  if (dtype != DEAMOE_BF16 || n_out % 8) return DEAMOE_ERR_UNSUPPORTED;
  if (!weight || !aligned16(weight) || !dweight || !aligned16(dweight) || dweight == weight || !aligned_to(dbias, 4))
    return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (n_token == 0)  // sums over no tokens
    return cudaMemsetAsync(dweight, 0, (size_t)n_out * n_in * 2, s) == cudaSuccess &&
                   (!dbias || cudaMemsetAsync(dbias, 0, (size_t)n_out * 4, s) == cudaSuccess)
               ? DEAMOE_OK : DEAMOE_ERR_CUDA;
  if (!x || !aligned16(x) || x_stride < n_in || x_stride % 8 || !dout || !aligned16(dout) || dout_stride < n_out || dout_stride % 8 ||
      !dx || !aligned16(dx) || dx_stride < n_in || dx_stride % 8 || dx == x || dx == dout || dx == weight)
    return DEAMOE_ERR_INVALID_ARG;
  const uint64_t need = deamoe_product_workspace(dtype, n_token, n_out, n_in, act, 1);
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return DEAMOE_ERR_INVALID_ARG;
  float* part = reinterpret_cast<float*>(workspace);
  const bool plain = act == DEAMOE_SIGMA_NONE;
  void* dz = reinterpret_cast<char*>(workspace) + ceil256(bias_parts(n_token, n_out, act));
  const void* g = plain ? dout : dz;  // gradient of z as an operand
  const int64_t gs = plain ? dout_stride : n_out;
  MatmulCall a = product_call(n_out, n_in, n_token, 64, false), b = product_call(n_in, n_out, n_token, 64, false),
             c = product_call(n_out, n_token, n_in, 64, false);
  a.args.out = dz; a.args.os = n_out; a.args.wide = 1; a.args.bias = bias; a.args.bias_f32 = bias_dtype == DEAMOE_F32; a.args.act = act;
  a.args.dout = dout; a.args.rs = dout_stride; a.args.wide_in = 1; a.args.part = dbias ? part : nullptr;
  b.args.out = dx; b.args.os = dx_stride; b.args.wide = 1;
  if ((!plain && (!map_rows(&a.maps.a, weight, 2, n_in, n_out, n_in, 1, n_in, 128) || !map_b(&a, x, 2, n_in, n_token, x_stride))) ||
      !map_rows(&b.maps.a, weight, 2, n_in, n_out, n_in, 1, n_in, 64) || !map_b(&b, g, 2, n_out, n_token, gs) ||
      !map_rows(&c.maps.a, g, 2, n_out, n_token, gs, 1, gs, 64) || !map_b_rows_inner(&c, x, n_in, n_token, x_stride) ||
      !map_out(&c, dweight, n_in, n_out, n_in, 1, (int64_t)n_out * n_in))
    return DEAMOE_ERR_CUDA;
  // What depends on nothing but what is already there runs beside the rest.  With an activation: dz, dx, the sums of the bias
  // gradient's parts and dW, of which the last two need dz as dx does, which waits for it.  Without one: the parts of the bias
  // gradient, dx and dW beside them, and their sums at the end.
  c.args.late = 1;
  b.args.late = plain && dbias;
  if (const uint64_t each = backward_sums(n_token, n_out, n_in)) {  // (b waits for a, c may run beside b)
    char* sums = reinterpret_cast<char*>(dz) + dz_bytes(n_token, n_out, act);
    a.args.sums = b.args.sums = reinterpret_cast<float*>(sums);
    c.args.sums = reinterpret_cast<float*>(sums + each);
  }
  const int parts = plain ? (n_token + BIAS_ROWS - 1) / BIAS_ROWS : MM_PARTS * ((n_token + a.args.tile_n - 1) / a.args.tile_n);
  auto add_parts = [&](int late) {
    return launch_pdl(k_add_parts, dim3((n_out + 31) / 32), dim3(256), 0, s, (const float*)part, parts, (int)n_out, dbias, late) == cudaSuccess;
  };
  bool ok = true;
  if (!plain) {
    ok = matmul_launch(MF_PRODUCT_GRAD, a, s) == cudaSuccess;
  } else if (dbias) {
    k_bias_sums<<<dim3(parts, (n_out + 255) / 256), 256, 0, s>>>(reinterpret_cast<const __nv_bfloat16*>(dout), dout_stride, n_token, n_out, part);
    ok = cudaGetLastError() == cudaSuccess;
  }
  ok = ok && matmul_launch(MF_STORE_TRANSPOSED, b, s) == cudaSuccess;
  if (ok && dbias && !plain) ok = add_parts(1);
  ok = ok && matmul_launch(MF_WEIGHT_GRAD, c, s) == cudaSuccess;
  if (ok && dbias && plain) ok = add_parts(0);
  if (ok) return DEAMOE_OK;
  cudaGetLastError();
  return DEAMOE_ERR_CUDA;
}

}  // extern "C"
