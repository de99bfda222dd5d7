// Norms around a layer: RMSNorm before it, and after it the residual sum with the gate, the norm of the layer's
// output and the norm of the sum (the next block's input) in one pass; and the gradients.
//
//   rms(v) = sqrt(mean(v^2) + eps)
//   norm:           u = x / rms(x) * w
//   norm_residual:  out = a x + b g (y / rms(y) * w),   u = out / rms(out) * wn     (out unrounded inside u)
// Gradients.  For n = v / rms(v) with gradient d:  dv = r d - v r^3 mean(d v),  r = 1 / rms(v).  So
//   D    = dout + [gradient of u through out] = dout + ro du wn - out ro^3 mean(du wn out)
//   dx   = a D,   dgate = b D (y ry w),   dv = b g D,   dw = sum_t dv (y ry),   dwn = sum_t du (out ro),
//   dy   = ry dv w - y ry^3 mean(dv w y)
// The backward pass takes x and y (not out), so that out is recomputed in fp32 and nothing rounded enters it; the
// row statistics are recomputed too, they cost nothing next to the loads.  All sums are fp32; each output is rounded
// once.
//
// Every operator is a few passes of HBM traffic over [T, h] rows, nothing else: bytes bound it.  Sums over the tokens
// (dw, dwn, a per-channel dgate) are kept per thread block and added by a second kernel in block order: no atomics,
// equal calls give equal bits.
#include "row.cuh"

namespace deamoe {

constexpr int NORM_CTAS = 296;  // thread blocks of the backward kernels: partial sums of the columns, one row each

struct Rows {  // a [T, h] matrix with a row stride (elements), or a null pointer
  const void* p;
  int64_t stride;
};

struct NormArgs {
  int64_t T;
  int h;
  int wdt;                 // type of the weights
  float eps, next_eps, a, b;
  int gate_kind;           // deamoe_gate_t
  int post_norm, next_norm;
  Rows x, y, gate, dout, du, dadd;
  const void *w, *wn;      // gains, or null (ones)
  void *out, *u, *dx, *dy, *dgate;
  int64_t out_s, u_s, dx_s, dy_s, dgate_s;
  float* part;             // [3][NORM_CTAS][h]: partial column sums of dw, dwn, dgate
  float* dgate_token;      // [T]
};

static __device__ __forceinline__ float load_gain(const void* w, int wdt, int64_t i) {
  if (!w) return 1.f;
  return wdt == DEAMOE_F32 ? reinterpret_cast<const float*>(w)[i]
                           : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(w)[i]);
}
template <typename T> static __device__ __forceinline__ float at(const Rows& m, int64_t t, int i) {
  return to_f<T>(reinterpret_cast<const T*>(m.p)[t * m.stride + i]);
}
template <typename T> static __device__ __forceinline__ void put(void* p, int64_t stride, int64_t t, int i, float v) {
  reinterpret_cast<T*>(p)[t * stride + i] = from_f<T>(v);
}
template <typename T> static __device__ __forceinline__ float gate_at(const NormArgs& A, int64_t t, int i) {
  switch (A.gate_kind) {
    case DEAMOE_GATE_CHANNEL: return to_f<T>(reinterpret_cast<const T*>(A.gate.p)[i]);
    case DEAMOE_GATE_TOKEN: return to_f<T>(reinterpret_cast<const T*>(A.gate.p)[t]);
    case DEAMOE_GATE_FULL: return at<T>(A.gate, t, i);
  }
  return 1.f;
}
static __device__ __forceinline__ float inv_rms(float ss, int h, float eps) { return rsqrtf(ss / (float)h + eps); }

// ---------------------------------------------------------------- any width, any alignment: one block a row

constexpr int ANY_THREADS = 256;

template <typename T> __global__ void __launch_bounds__(ANY_THREADS) k_norm_any(NormArgs A) {
  __shared__ float buf[32];
  const int64_t t = blockIdx.x;
  float ss[1] = {0.f};
  for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
    const float v = at<T>(A.x, t, i);
    ss[0] = fmaf(v, v, ss[0]);
  }
  block_sums<1>(ss, buf);
  const float r = inv_rms(ss[0], A.h, A.eps);
  for (int i = threadIdx.x; i < A.h; i += ANY_THREADS)
    put<T>(A.u, A.u_s, t, i, at<T>(A.x, t, i) * r * load_gain(A.w, A.wdt, i));
}

template <typename T> __global__ void __launch_bounds__(ANY_THREADS) k_norm_grad_any(NormArgs A) {
  __shared__ float buf[2][64];
  float* part = A.part + (size_t)blockIdx.x * A.h;
  int flip = 0;
  bool first = true;
  for (int64_t t = blockIdx.x; t < A.T; t += gridDim.x) {
    float s[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
      const float v = at<T>(A.x, t, i);
      s[0] = fmaf(v, v, s[0]);
      s[1] = fmaf(at<T>(A.du, t, i) * load_gain(A.w, A.wdt, i), v, s[1]);
    }
    block_sums<2>(s, buf[flip]);
    flip ^= 1;
    const float r = inv_rms(s[0], A.h, A.eps);
    const float c = r * r * r * (s[1] / (float)A.h);
    for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
      const float v = at<T>(A.x, t, i), d = at<T>(A.du, t, i);
      float dx = r * d * load_gain(A.w, A.wdt, i) - v * c;
      if (A.dadd.p) dx += at<T>(A.dadd, t, i);
      const float dw = d * v * r;
      part[i] = first ? dw : part[i] + dw;
      put<T>(A.dx, A.dx_s, t, i, dx);
    }
    first = false;
  }
}

template <typename T> __global__ void __launch_bounds__(ANY_THREADS) k_residual_any(NormArgs A) {
  __shared__ float buf[2][32];
  const int64_t t = blockIdx.x;
  float ry = 1.f;
  if (A.post_norm) {
    float ss[1] = {0.f};
    for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
      const float v = at<T>(A.y, t, i);
      ss[0] = fmaf(v, v, ss[0]);
    }
    block_sums<1>(ss, buf[0]);
    ry = inv_rms(ss[0], A.h, A.eps);
  }
  auto sum = [&](int i) {
    const float v = at<T>(A.y, t, i) * ry * load_gain(A.w, A.wdt, i);
    return fmaf(A.a, at<T>(A.x, t, i), A.b * gate_at<T>(A, t, i) * v);
  };
  float ro = 1.f;
  if (A.next_norm) {
    float ss[1] = {0.f};
    for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
      const float o = sum(i);
      ss[0] = fmaf(o, o, ss[0]);
    }
    block_sums<1>(ss, buf[1]);
    ro = inv_rms(ss[0], A.h, A.next_eps);
  }
  for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
    const float o = sum(i);
    put<T>(A.out, A.out_s, t, i, o);
    if (A.next_norm) put<T>(A.u, A.u_s, t, i, o * ro * load_gain(A.wn, A.wdt, i));
  }
}

template <typename T> __global__ void __launch_bounds__(ANY_THREADS) k_residual_grad_any(NormArgs A) {
  __shared__ float buf[4][64];  // the last sum alternates: it may be the only one of a row
  int flip = 2;
  float* part_w = A.part + (size_t)blockIdx.x * A.h;
  float* part_n = part_w + (size_t)NORM_CTAS * A.h;
  float* part_g = part_n + (size_t)NORM_CTAS * A.h;
  bool first = true;
  for (int64_t t = blockIdx.x; t < A.T; t += gridDim.x) {
    float ry = 1.f;
    if (A.post_norm) {
      float ss[1] = {0.f};
      for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
        const float v = at<T>(A.y, t, i);
        ss[0] = fmaf(v, v, ss[0]);
      }
      block_sums<1>(ss, buf[0]);
      ry = inv_rms(ss[0], A.h, A.eps);
    }
    auto branch = [&](int i) { return at<T>(A.y, t, i) * ry * load_gain(A.w, A.wdt, i); };
    auto sum = [&](int i) { return fmaf(A.a, at<T>(A.x, t, i), A.b * gate_at<T>(A, t, i) * branch(i)); };
    float ro = 1.f, co = 0.f;
    if (A.next_norm) {
      float s[2] = {0.f, 0.f};
      for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
        const float o = sum(i);
        s[0] = fmaf(o, o, s[0]);
        s[1] = fmaf(at<T>(A.du, t, i) * load_gain(A.wn, A.wdt, i), o, s[1]);
      }
      block_sums<2>(s, buf[1]);
      ro = inv_rms(s[0], A.h, A.next_eps);
      co = ro * ro * ro * (s[1] / (float)A.h);
    }
    auto total = [&](int i) {  // gradient of the sum
      float d = at<T>(A.dout, t, i);
      if (A.next_norm) d += ro * at<T>(A.du, t, i) * load_gain(A.wn, A.wdt, i) - sum(i) * co;
      return d;
    };
    float s[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
      const float d = total(i);
      s[0] = fmaf(A.b * gate_at<T>(A, t, i) * d * load_gain(A.w, A.wdt, i), at<T>(A.y, t, i), s[0]);
      s[1] = fmaf(A.b * d, branch(i), s[1]);
    }
    block_sums<2>(s, buf[flip]);
    flip ^= 1;
    const float cy = A.post_norm ? ry * ry * ry * (s[0] / (float)A.h) : 0.f;
    if (A.gate_kind == DEAMOE_GATE_TOKEN && threadIdx.x == 0) A.dgate_token[t] = s[1];
    for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
      const float d = total(i), y = at<T>(A.y, t, i), w = load_gain(A.w, A.wdt, i);
      const float dv = A.b * gate_at<T>(A, t, i) * d;
      const float dy = ry * dv * w - y * cy;
      if (A.w) part_w[i] = (first ? 0.f : part_w[i]) + dv * y * ry;
      if (A.wn) part_n[i] = (first ? 0.f : part_n[i]) + at<T>(A.du, t, i) * sum(i) * ro;
      const float dg = A.b * d * y * ry * w;
      if (A.gate_kind == DEAMOE_GATE_CHANNEL) part_g[i] = (first ? 0.f : part_g[i]) + dg;
      if (A.gate_kind == DEAMOE_GATE_FULL) put<T>(A.dgate, A.dgate_s, t, i, dg);
      put<T>(A.dx, A.dx_s, t, i, A.a * d);
      put<T>(A.dy, A.dy_s, t, i, dy);
    }
    first = false;
  }
}

// ---------------------------------------------------------------- sums over the blocks' partial rows

struct ColumnSums {
  const float* part[3];
  float* out[3];
};
// A block adds 32 columns of one array: 8 row groups side by side, then the groups in order.
__global__ void __launch_bounds__(256) k_column_sums(ColumnSums S, int rows, int h) {
  __shared__ float acc[8][33];
  pdl_wait();
  const float* p = S.part[blockIdx.y];
  float* out = S.out[blockIdx.y];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
  float s = 0.f;
  if (c < h)
    for (int r = g; r < rows; r += 8) s += p[(size_t)r * h + c];
  acc[g][threadIdx.x & 31] = s;
  __syncthreads();
  if (g == 0 && c < h) {
    for (int i = 1; i < 8; ++i) s += acc[i][threadIdx.x & 31];
    out[c] = s;
  }
}

// ---------------------------------------------------------------- host side

static deamoe_status_t check_norm(int32_t dtype, int32_t wdtype, int32_t tokens, int32_t h, float eps) {
  if (!known_type(dtype) || !known_type(wdtype) || h <= 0 || !(eps >= 0.f)) return DEAMOE_ERR_INVALID_ARG;
  if (h > DEAMOE_MAX_WIDTH) return DEAMOE_ERR_UNSUPPORTED;
  if (tokens < 0) return DEAMOE_ERR_BATCH;
  return DEAMOE_OK;
}
static bool bad_rows(const void* p, int64_t stride, int32_t h, size_t es) { return !p || !aligned_to(p, es) || stride < h; }

static deamoe_status_t launch_sums(const ColumnSums& S, int arrays, int rows, int h, cudaStream_t s) {
  if (arrays == 0) return DEAMOE_OK;
  if (launch_pdl(k_column_sums, dim3((h + 31) / 32, arrays), dim3(256), 0, s, S, rows, h) != cudaSuccess) {
    cudaGetLastError();
    return DEAMOE_ERR_CUDA;
  }
  return DEAMOE_OK;
}

template <typename T> static deamoe_status_t norm_t(const NormArgs& A, cudaStream_t s) {
  k_norm_any<T><<<(unsigned)A.T, ANY_THREADS, 0, s>>>(A);
  return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA;
}
static int grad_ctas(int64_t T) { return (int)(T < NORM_CTAS ? T : NORM_CTAS); }

template <typename T> static deamoe_status_t norm_grad_t(const NormArgs& A, cudaStream_t s) {
  k_norm_grad_any<T><<<grad_ctas(A.T), ANY_THREADS, 0, s>>>(A);
  return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA;
}
template <typename T> static deamoe_status_t residual_t(const NormArgs& A, cudaStream_t s) {
  k_residual_any<T><<<(unsigned)A.T, ANY_THREADS, 0, s>>>(A);
  return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA;
}
template <typename T> static deamoe_status_t residual_grad_t(const NormArgs& A, cudaStream_t s) {
  k_residual_grad_any<T><<<grad_ctas(A.T), ANY_THREADS, 0, s>>>(A);
  return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA;
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_norm_workspace(int32_t n_token, int32_t hidden) {
  if (n_token <= 0 || hidden <= 0) return 0;
  return (uint64_t)3 * NORM_CTAS * hidden * sizeof(float);
}

deamoe_status_t deamoe_norm(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, int32_t n_token,
                            int32_t hidden, int32_t weight_dtype, const void* weight, float eps, void* out,
                            int64_t out_stride) {
  deamoe_status_t st = check_norm(dtype, weight_dtype, n_token, hidden, eps);
  if (st != DEAMOE_OK || n_token == 0) return st;
  const size_t es = type_bytes(dtype);
  if (bad_rows(x, x_stride, hidden, es) || bad_rows(out, out_stride, hidden, es) ||
      !aligned_to(weight, type_bytes(weight_dtype)) || (x == out && x_stride != out_stride))
    return DEAMOE_ERR_INVALID_ARG;
  NormArgs A = {};
  A.T = n_token; A.h = hidden; A.wdt = weight_dtype; A.eps = eps; A.w = weight;
  A.x = {x, x_stride}; A.u = out; A.u_s = out_stride;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32 ? norm_t<float>(A, s) : norm_t<__nv_bfloat16>(A, s);
}

deamoe_status_t deamoe_norm_backward(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, int32_t n_token,
                                     int32_t hidden, int32_t weight_dtype, const void* weight, float eps, const void* du,
                                     int64_t du_stride, const void* dadd, int64_t dadd_stride, void* dx,
                                     int64_t dx_stride, float* dweight, void* workspace, uint64_t workspace_bytes) {
  deamoe_status_t st = check_norm(dtype, weight_dtype, n_token, hidden, eps);
  if (st != DEAMOE_OK) return st;
  if (!dweight || !aligned_to(dweight, 4)) return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (n_token == 0)
    return cudaMemsetAsync(dweight, 0, (size_t)hidden * 4, s) == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA;
  const size_t es = type_bytes(dtype);
  if (bad_rows(x, x_stride, hidden, es) || bad_rows(du, du_stride, hidden, es) || bad_rows(dx, dx_stride, hidden, es) ||
      (dadd && bad_rows(dadd, dadd_stride, hidden, es)) || !aligned_to(weight, type_bytes(weight_dtype)))
    return DEAMOE_ERR_INVALID_ARG;
  if (dx == x || dx == du || (dx == dadd && dx_stride != dadd_stride)) return DEAMOE_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) || workspace_bytes < deamoe_norm_workspace(n_token, hidden))
    return DEAMOE_ERR_INVALID_ARG;
  NormArgs A = {};
  A.T = n_token; A.h = hidden; A.wdt = weight_dtype; A.eps = eps; A.w = weight;
  A.x = {x, x_stride}; A.du = {du, du_stride}; A.dadd = {dadd, dadd_stride}; A.dx = dx; A.dx_s = dx_stride;
  A.part = reinterpret_cast<float*>(workspace);
  st = dtype == DEAMOE_F32 ? norm_grad_t<float>(A, s) : norm_grad_t<__nv_bfloat16>(A, s);
  if (st != DEAMOE_OK) return st;
  ColumnSums S = {};
  S.part[0] = A.part; S.out[0] = dweight;
  return launch_sums(S, 1, grad_ctas(n_token), hidden, s);
}

static deamoe_status_t check_block(int32_t gate_kind, const void* gate, int64_t gate_stride, int32_t hidden, size_t es,
                                   int32_t normalise, const void* weight, float a, float b) {
  if (gate_kind < DEAMOE_GATE_NONE || gate_kind > DEAMOE_GATE_FULL) return DEAMOE_ERR_INVALID_ARG;
  if ((gate_kind == DEAMOE_GATE_NONE) != (gate == nullptr) || !aligned_to(gate, es)) return DEAMOE_ERR_INVALID_ARG;
  if (gate_kind == DEAMOE_GATE_FULL && gate_stride < hidden) return DEAMOE_ERR_INVALID_ARG;
  if ((normalise != 0 && normalise != 1) || (!normalise && weight)) return DEAMOE_ERR_INVALID_ARG;
  if (!(a == a) || !(b == b)) return DEAMOE_ERR_INVALID_ARG;
  return DEAMOE_OK;
}

deamoe_status_t deamoe_norm_residual(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, const void* y,
                                     int64_t y_stride, int32_t n_token, int32_t hidden, int32_t normalise,
                                     int32_t weight_dtype, const void* weight, float eps, int32_t gate_kind,
                                     const void* gate, int64_t gate_stride, float residual_scale, float branch_scale,
                                     void* out, int64_t out_stride, const void* next_weight, float next_eps, void* next,
                                     int64_t next_stride) {
  deamoe_status_t st = check_norm(dtype, weight_dtype, n_token, hidden, eps);
  if (st == DEAMOE_OK && !(next_eps >= 0.f)) st = DEAMOE_ERR_INVALID_ARG;
  if (st != DEAMOE_OK || n_token == 0) return st;
  const size_t es = type_bytes(dtype), ws = type_bytes(weight_dtype);
  if (bad_rows(x, x_stride, hidden, es) || bad_rows(y, y_stride, hidden, es) || bad_rows(out, out_stride, hidden, es) ||
      (next && bad_rows(next, next_stride, hidden, es)) || !aligned_to(weight, ws) || !aligned_to(next_weight, ws) ||
      (next_weight && !next))
    return DEAMOE_ERR_INVALID_ARG;
  if ((out == x && out_stride != x_stride) || out == y || next == x || next == y || next == out)
    return DEAMOE_ERR_INVALID_ARG;
  st = check_block(gate_kind, gate, gate_stride, hidden, es, normalise, weight, residual_scale, branch_scale);
  if (st != DEAMOE_OK) return st;
  NormArgs A = {};
  A.T = n_token; A.h = hidden; A.wdt = weight_dtype; A.eps = eps; A.next_eps = next_eps;
  A.a = residual_scale; A.b = branch_scale; A.gate_kind = gate_kind; A.post_norm = normalise; A.next_norm = next ? 1 : 0;
  A.x = {x, x_stride}; A.y = {y, y_stride}; A.gate = {gate, gate_stride}; A.w = weight; A.wn = next_weight;
  A.out = out; A.out_s = out_stride; A.u = next; A.u_s = next_stride;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32 ? residual_t<float>(A, s) : residual_t<__nv_bfloat16>(A, s);
}

deamoe_status_t deamoe_norm_residual_backward(
    void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, const void* y, int64_t y_stride, int32_t n_token,
    int32_t hidden, int32_t normalise, int32_t weight_dtype, const void* weight, float eps, int32_t gate_kind,
    const void* gate, int64_t gate_stride, float residual_scale, float branch_scale, const void* dout,
    int64_t dout_stride, const void* next_weight, float next_eps, const void* dnext, int64_t dnext_stride, void* dx,
    int64_t dx_stride, void* dy, int64_t dy_stride, void* dgate, int64_t dgate_stride, float* dweight,
    float* dnext_weight, void* workspace, uint64_t workspace_bytes) {
  deamoe_status_t st = check_norm(dtype, weight_dtype, n_token, hidden, eps);
  if (st == DEAMOE_OK && !(next_eps >= 0.f)) st = DEAMOE_ERR_INVALID_ARG;
  if (st != DEAMOE_OK) return st;
  const size_t es = type_bytes(dtype), ws = type_bytes(weight_dtype);
  // a gradient is given back exactly for what the call has: the gains, the gate
  if ((weight == nullptr) != (dweight == nullptr) || (next_weight == nullptr) != (dnext_weight == nullptr) ||
      !aligned_to(dweight, 4) || !aligned_to(dnext_weight, 4))
    return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (n_token == 0) {  // sums over no tokens
    if (gate_kind < DEAMOE_GATE_NONE || gate_kind > DEAMOE_GATE_FULL || !aligned_to(dgate, 4)) return DEAMOE_ERR_INVALID_ARG;
    bool ok = true;
    for (void* p : {(void*)dweight, (void*)dnext_weight, gate_kind == DEAMOE_GATE_CHANNEL ? dgate : nullptr})
      if (p) ok &= cudaMemsetAsync(p, 0, (size_t)hidden * 4, s) == cudaSuccess;
    return ok ? DEAMOE_OK : DEAMOE_ERR_CUDA;
  }
  st = check_block(gate_kind, gate, gate_stride, hidden, es, normalise, weight, residual_scale, branch_scale);
  if (st != DEAMOE_OK) return st;
  if (next_weight && !dnext) return DEAMOE_ERR_INVALID_ARG;
  const size_t gs = gate_kind == DEAMOE_GATE_FULL ? es : 4;
  if ((gate_kind == DEAMOE_GATE_NONE) != (dgate == nullptr) || !aligned_to(dgate, gs) ||
      (gate_kind == DEAMOE_GATE_FULL && dgate_stride < hidden))
    return DEAMOE_ERR_INVALID_ARG;
  if (bad_rows(x, x_stride, hidden, es) || bad_rows(y, y_stride, hidden, es) || bad_rows(dout, dout_stride, hidden, es) ||
      (dnext && bad_rows(dnext, dnext_stride, hidden, es)) || bad_rows(dx, dx_stride, hidden, es) ||
      bad_rows(dy, dy_stride, hidden, es) || !aligned_to(weight, ws) || !aligned_to(next_weight, ws))
    return DEAMOE_ERR_INVALID_ARG;
  const void* ins[5] = {x, y, dout, dnext, gate_kind == DEAMOE_GATE_FULL ? gate : nullptr};
  for (const void* in : ins)
    if (in && (dx == in || dy == in || dgate == in)) return DEAMOE_ERR_INVALID_ARG;
  if (dx == dy || dgate == dx || dgate == dy) return DEAMOE_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) || workspace_bytes < deamoe_norm_workspace(n_token, hidden))
    return DEAMOE_ERR_INVALID_ARG;
  NormArgs A = {};
  A.T = n_token; A.h = hidden; A.wdt = weight_dtype; A.eps = eps; A.next_eps = next_eps;
  A.a = residual_scale; A.b = branch_scale; A.gate_kind = gate_kind; A.post_norm = normalise; A.next_norm = dnext ? 1 : 0;
  A.x = {x, x_stride}; A.y = {y, y_stride}; A.gate = {gate, gate_stride}; A.w = weight; A.wn = next_weight;
  A.dout = {dout, dout_stride}; A.du = {dnext, dnext_stride};
  A.dx = dx; A.dx_s = dx_stride; A.dy = dy; A.dy_s = dy_stride; A.dgate = dgate; A.dgate_s = dgate_stride;
  A.dgate_token = gate_kind == DEAMOE_GATE_TOKEN ? reinterpret_cast<float*>(dgate) : nullptr;
  A.part = reinterpret_cast<float*>(workspace);
  st = dtype == DEAMOE_F32 ? residual_grad_t<float>(A, s) : residual_grad_t<__nv_bfloat16>(A, s);
  if (st != DEAMOE_OK) return st;
  ColumnSums S = {};
  int n = 0;
  const size_t step = (size_t)NORM_CTAS * hidden;
  if (dweight) { S.part[n] = A.part; S.out[n++] = dweight; }
  if (dnext_weight) { S.part[n] = A.part + step; S.out[n++] = dnext_weight; }
  if (gate_kind == DEAMOE_GATE_CHANNEL) { S.part[n] = A.part + 2 * step; S.out[n++] = reinterpret_cast<float*>(dgate); }
  return launch_sums(S, n, grad_ctas(n_token), hidden, s);
}

}  // extern "C"
