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
// Every operator is one pass of HBM traffic over [T, h] rows: bytes bound the forward calls (8192 x 7168 bf16: norm 38 us,
// norm_residual with a channel gate and the next norm 81 us, 6.2 and 5.8 TB/s) and norm_backward (67 us, 80 with dadd:
// 5.3 and 5.8 TB/s); norm_residual_backward (170 us, 4.1 TB/s) is held by a row's latency, see there.  Sums over the
// tokens (dw, dwn, a per-channel dgate) are kept per thread block and added by a second kernel in block order: no
// atomics, equal calls give equal bits.
#include <cuda_fp8.h>

#include <atomic>

#include "row.cuh"

namespace deamoe {

// Thread blocks of the backward kernels, each of which leaves one row of partial column sums: 16 columns a thread (a
// row's fixed work -- addresses, the reduction -- is spread over more values than with 8, and 128 registers hold the
// columns' constants and sums), 512 threads an SM or the 8 blocks that they come in for rows below 1024 values (rows of up
// to 8192 values; else two blocks an SM).
constexpr int NORM_SMS = 148;
constexpr int GRAD_COLUMNS = 16, GRAD_MAX_WIDTH = 8192;
constexpr int GRAD_ODD_COLUMNS = 8;  // of rows that are read value by value
static int grad_threads(int h, int columns = GRAD_COLUMNS) { return ((h + columns - 1) / columns + 31) / 32 * 32; }
static int grad_blocks_per_sm(int h) {
  if (h > GRAD_MAX_WIDTH) return 2;
  const int n = 512 / grad_threads(h);
  return n > 8 ? 8 : n;
}
static int grad_ctas(int64_t T, int h) {
  const int most = NORM_SMS * grad_blocks_per_sm(h);
  return T < most ? (int)T : most;
}

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
  uint8_t* codes;          // [T, h] e4m3 of the quantised norms, and their rows' scales
  int64_t codes_s;
  float* scale;
  float* part;             // [3][grad_ctas][h]: partial column sums of dw, dwn, dgate
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
// r^3 m for a mean m of values of size 1 / r: r^3 alone leaves fp32's range for rows beyond 1e13 or below 1e-13
static __device__ __forceinline__ float cube_times(float r, float m) { return (r * r) * (r * m); }

// ---------------------------------------------------------------- any width, any alignment: one block a row

constexpr int ANY_THREADS = 256;
// An SM's 228 KB of shared memory go to its blocks: each has its ring, 2 KB for the sums' buffers and 1 KB that the device keeps.
constexpr int SM_SMEM = 228 * 1024, BLOCK_SMEM = 3 * 1024;
constexpr int RING_BYTES = SM_SMEM - BLOCK_SMEM;  // of one block alone (two fp32 rows of 4 x 7168 values)

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
    const float c = cube_times(r, s[1] / (float)A.h);
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

template <typename T> __global__ void __launch_bounds__(ANY_THREADS) k_residual_grad_any(NormArgs A, size_t part_step) {
  __shared__ float buf[4][64];  // the last sum alternates: it may be the only one of a row
  int flip = 2;
  float* part_w = A.part + (size_t)blockIdx.x * A.h;
  float* part_n = part_w + part_step;
  float* part_g = part_n + part_step;
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
      co = cube_times(ro, s[1] / (float)A.h);
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
    const float cy = A.post_norm ? cube_times(ry, s[0] / (float)A.h) : 0.f;
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

// ---------------------------------------------------------------- rows held in registers

// VE gains at column i (null = ones)
template <int VE> static __device__ __forceinline__ void load_gains(const void* w, int wdt, int64_t i, float (&f)[VE]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = 1.f;
  } else if constexpr (VE == 1) {
    f[0] = load_gain(w, wdt, i);
  } else if (wdt == DEAMOE_F32) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(w) + i);
#pragma unroll
    for (int j = 0; j < VE / 4; ++j) {
      const float4 v = p[j];
      f[4 * j] = v.x; f[4 * j + 1] = v.y; f[4 * j + 2] = v.z; f[4 * j + 3] = v.w;
    }
  } else {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(w) + i);
    uint32_t u[VE / 2];
    if constexpr (VE == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      u[0] = v.x; u[1] = v.y; u[2] = v.z; u[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      u[0] = v.x; u[1] = v.y;
    }
#pragma unroll
    for (int j = 0; j < VE / 2; ++j) {
      f[2 * j] = __uint_as_float(u[j] << 16);
      f[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
    }
  }
}

template <typename T> static __device__ __forceinline__ const T* row_at(const Rows& m, int64_t t) {
  return reinterpret_cast<const T*>(m.p) + t * m.stride;
}
template <typename T, int VE> static __device__ __forceinline__ void load_row(const Rows& m, int64_t t, int c, float (&f)[VE]) {
  load_once<T, VE>(row_at<T>(m, t) + (int64_t)c * VE).widen(f);
}
template <typename T, int VE>
static __device__ __forceinline__ void store_row(void* p, int64_t stride, int64_t t, int c, const float (&f)[VE]) {
  Pack<T, VE> o;
  o.narrow(f);
  store_pack<T, VE>(reinterpret_cast<T*>(p) + t * stride + (int64_t)c * VE, o);
}
template <typename T, int VE> static __device__ __forceinline__ void load_gate(const NormArgs& A, int64_t t, int c, float (&g)[VE]) {
  if (A.gate_kind == DEAMOE_GATE_FULL) {
    load_row<T, VE>(A.gate, t, c, g);
  } else if (A.gate_kind == DEAMOE_GATE_CHANNEL) {
    load_pack<T, VE>(reinterpret_cast<const T*>(A.gate.p) + (int64_t)c * VE).widen(g);
  } else {
    const float v = A.gate_kind == DEAMOE_GATE_TOKEN ? to_f<T>(reinterpret_cast<const T*>(A.gate.p)[t]) : 1.f;
#pragma unroll
    for (int j = 0; j < VE; ++j) g[j] = v;
  }
}

// Forward kernels: one block a row, NV packs of VE values a thread, the row read once.  Rows in flight hide each
// other's two reductions.
template <typename T, int VE, int NV, int MAXT> __global__ void __launch_bounds__(MAXT) k_norm_rows(NormArgs A, int packs) {
  __shared__ float buf[32];
  const int64_t t = blockIdx.x;
  Pack<T, VE> x[NV];
  float ss[1] = {0.f};
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c < packs) x[n] = load_once<T, VE>(row_at<T>(A.x, t) + (int64_t)c * VE);
  }
#pragma unroll
  for (int n = 0; n < NV; ++n)
    if ((int)(threadIdx.x + n * blockDim.x) < packs) {
      float f[VE];
      x[n].widen(f);
#pragma unroll
      for (int j = 0; j < VE; ++j) ss[0] = fmaf(f[j], f[j], ss[0]);
    }
  block_sums<1>(ss, buf);
  const float r = inv_rms(ss[0], A.h, A.eps);
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
    float f[VE], w[VE];
    x[n].widen(f);
    load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, w);
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] *= r * w[j];
    store_row<T, VE>(A.u, A.u_s, t, c, f);
  }
}

template <typename T, int VE, int NV, int MAXT> __global__ void __launch_bounds__(MAXT) k_residual_rows(NormArgs A, int packs) {
  __shared__ float buf[2][32];
  const int64_t t = blockIdx.x;
  Pack<T, VE> x[NV], y[NV];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c < packs) {
      y[n] = load_once<T, VE>(row_at<T>(A.y, t) + (int64_t)c * VE);
      x[n] = load_once<T, VE>(row_at<T>(A.x, t) + (int64_t)c * VE);
    }
  }
  float ry = 1.f;
  if (A.post_norm) {
    float ss[1] = {0.f};
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if ((int)(threadIdx.x + n * blockDim.x) < packs) {
        float f[VE];
        y[n].widen(f);
#pragma unroll
        for (int j = 0; j < VE; ++j) ss[0] = fmaf(f[j], f[j], ss[0]);
      }
    block_sums<1>(ss, buf[0]);
    ry = inv_rms(ss[0], A.h, A.eps);
  }
  float s[NV][VE], ss[1] = {0.f};
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
    float f[VE], w[VE], g[VE];
    load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, w);
    load_gate<T, VE>(A, t, c, g);
    y[n].widen(f);
    x[n].widen(s[n]);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      s[n][j] = fmaf(A.a, s[n][j], A.b * g[j] * (f[j] * ry * w[j]));
      ss[0] = fmaf(s[n][j], s[n][j], ss[0]);
    }
    store_row<T, VE>(A.out, A.out_s, t, c, s[n]);
  }
  if (!A.next_norm) return;
  block_sums<1>(ss, buf[1]);
  const float ro = inv_rms(ss[0], A.h, A.next_eps);
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
    float w[VE];
    load_gains<VE>(A.wn, A.wdt, (int64_t)c * VE, w);
#pragma unroll
    for (int j = 0; j < VE; ++j) s[n][j] *= ro * w[j];
    store_row<T, VE>(A.u, A.u_s, t, c, s[n]);
  }
}

// ---------------------------------------------------------------- norms with an output in 8 bits
//
//   u = s / rms(s) * w,   scale = max |u| / 448,   code = e4m3(u / scale)            (s: x, or the sum after the block)
//
// With m = max |s w| the code is e4m3(s w * 448 / m) and the scale m / rms(s) / 448: the sum of squares and the maximum
// come from one reduction, and the codes do not wait for the root.  Rows whose m is below 2^-110 (a row of zeros among
// them) take 2^-110 for it.  A NaN stays the maximum, so that the row's scale (and all its codes) are NaN even where the sum of squares
// is not used or does not see it (a gain of NaN).  The row stays in registers; HBM bounds it: 5 bytes a value without a sum, 7 with
// one (bf16).
constexpr int CODES_THREADS = 512;  // of an SM, in the persistent form: 128 registers each
constexpr float E4M3_MAX = 448.f, QUANT_LEAST = 0x1p-110f;

// the larger one, or NaN if either is (with its sign bit clear)
static __device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// the maximum of v[0] and the sums of the others over a block, to every thread; buf: 32 N floats, as for block_sums
template <int N> static __device__ __forceinline__ void block_max_sums(float (&v)[N], float* buf) {
  auto join = [&](int o) {
    v[0] = max_or_nan(v[0], __shfl_xor_sync(0xffffffffu, v[0], o));
#pragma unroll
    for (int i = 1; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  };
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) join(o);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) buf[i * 32 + w] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane < warps ? buf[i * 32 + lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) join(o);
}
// The same for a maximum m >= 0 and two sums over at most 16 warps, in a third of the instructions: non-negative floats order as
// integers (NaN of a clear sign bit above infinity), for which a warp has a reduction of its own, and half a warp each adds one of the
// sums.  Fixed order; buf: 96 floats.
static __device__ __forceinline__ void block_max_two_sums(float& m, float& a, float& b, float* buf) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const bool up = lane >= 16;
  const float send = up ? a : b;
  m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
  float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, send, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (warps > 1) {
    if ((lane & 15) == 0) {
      buf[(up ? 64 : 32) + w] = v;
      if (lane == 0) buf[w] = m;
    }
    __syncthreads();
    const int i = lane & 15;
    m = __uint_as_float(__reduce_max_sync(0xffffffffu, i < warps ? __float_as_uint(buf[i]) : 0u));
    v = i < warps ? buf[(up ? 64 : 32) + i] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  a = __shfl_sync(0xffffffffu, v, 0);
  b = __shfl_sync(0xffffffffu, v, 16);
}
// scale of a row into memory; returns what its values are multiplied by (to 2 units; 2^-8 keeps the reciprocal a normal number
// up to the largest m)
static __device__ __forceinline__ float row_scale(const NormArgs& A, int64_t t, float ss, float m) {
  m = max_or_nan(m, QUANT_LEAST);
  if (threadIdx.x == 0) A.scale[t] = (A.next_norm ? inv_rms(ss, A.h, A.next_eps) : 1.f) * m * (1.f / E4M3_MAX);
  return (E4M3_MAX * 0x1p-8f) * __fdividef(1.f, m * 0x1p-8f);
}
template <int VE> static __device__ __forceinline__ void store_codes(uint8_t* p, const float (&f)[VE]) {
  if constexpr (VE == 1) {
    *p = __nv_cvt_float_to_fp8(f[0], __NV_SATFINITE, __NV_E4M3);
  } else {
    uint32_t u[VE / 4];
#pragma unroll
    for (int i = 0; i < VE / 4; ++i)
      u[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[4 * i], f[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
             (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2], f[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
    if constexpr (VE == 8) *reinterpret_cast<uint2*>(p) = make_uint2(u[0], u[1]);
    else *reinterpret_cast<uint32_t*>(p) = u[0];
  }
}

// y.p null: s = x, nothing but the codes is written
template <typename T> __global__ void __launch_bounds__(ANY_THREADS) k_codes_any(NormArgs A) {
  __shared__ float buf[2][64];
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
    const float x = at<T>(A.x, t, i);
    return A.y.p ? fmaf(A.a, x, A.b * gate_at<T>(A, t, i) * (at<T>(A.y, t, i) * ry * load_gain(A.w, A.wdt, i))) : x;
  };
  float v[2] = {0.f, 0.f};
  for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
    const float s = sum(i);
    v[0] = max_or_nan(v[0], fabsf(s * load_gain(A.wn, A.wdt, i)));
    v[1] = fmaf(s, s, v[1]);
  }
  block_max_sums<2>(v, buf[1]);
  const float f = row_scale(A, t, v[1], v[0]);
  for (int i = threadIdx.x; i < A.h; i += ANY_THREADS) {
    const float s = sum(i);
    if (A.y.p) put<T>(A.out, A.out_s, t, i, s);
    const float c[1] = {s * load_gain(A.wn, A.wdt, i) * f};
    store_codes<1>(A.codes + t * A.codes_s + i, c);
  }
}

template <typename T, int VE, int NV, int MAXT> __global__ void __launch_bounds__(MAXT) k_codes_rows(NormArgs A, int packs) {
  __shared__ float buf[2][64];
  const int64_t t = blockIdx.x;
  Pack<T, VE> x[NV], y[NV];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c < packs) {
      if (A.y.p) y[n] = load_once<T, VE>(row_at<T>(A.y, t) + (int64_t)c * VE);
      x[n] = load_once<T, VE>(row_at<T>(A.x, t) + (int64_t)c * VE);
    }
  }
  float ry = 1.f;
  if (A.post_norm) {
    float ss[1] = {0.f};
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if ((int)(threadIdx.x + n * blockDim.x) < packs) {
        float f[VE];
        y[n].widen(f);
#pragma unroll
        for (int j = 0; j < VE; ++j) ss[0] = fmaf(f[j], f[j], ss[0]);
      }
    block_sums<1>(ss, buf[0]);
    ry = inv_rms(ss[0], A.h, A.eps);
  }
  float s[NV][VE], v[2] = {0.f, 0.f};
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
    float f[VE], w[VE], g[VE];
    x[n].widen(s[n]);
    if (A.y.p) {
      load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, w);
      load_gate<T, VE>(A, t, c, g);
      y[n].widen(f);
#pragma unroll
      for (int j = 0; j < VE; ++j) s[n][j] = fmaf(A.a, s[n][j], A.b * g[j] * (f[j] * ry * w[j]));
      store_row<T, VE>(A.out, A.out_s, t, c, s[n]);
    }
    load_gains<VE>(A.wn, A.wdt, (int64_t)c * VE, w);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      v[1] = fmaf(s[n][j], s[n][j], v[1]);
      s[n][j] *= w[j];
      v[0] = max_or_nan(v[0], fabsf(s[n][j]));
    }
  }
  block_max_sums<2>(v, buf[1]);
  const float scale = row_scale(A, t, v[1], v[0]);
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
#pragma unroll
    for (int j = 0; j < VE; ++j) s[n][j] *= scale;
    store_codes<VE>(A.codes + t * A.codes_s + (int64_t)c * VE, s[n]);
  }
}

// Two fp32 values in one register pair: the backward kernels are bound by instruction issue, and sm_100a has multiply
// and multiply-add on such pairs, each value rounded as by itself.
struct F2 { unsigned long long v; };
static __device__ __forceinline__ F2 pair(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
static __device__ __forceinline__ float low(F2 a) { return __uint_as_float((uint32_t)a.v); }
static __device__ __forceinline__ float high(F2 a) { return __uint_as_float((uint32_t)(a.v >> 32)); }
static __device__ __forceinline__ F2 fma_(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
static __device__ __forceinline__ F2 mul_(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
static __device__ __forceinline__ float fma_(float a, float b, float c) { return fmaf(a, b, c); }
static __device__ __forceinline__ float mul_(float a, float b) { return a * b; }
static __device__ __forceinline__ float total(F2 a) { return low(a) + high(a); }
static __device__ __forceinline__ float total(float a) { return a; }
template <typename P> static __device__ __forceinline__ P splat(float a);
template <> __device__ __forceinline__ float splat<float>(float a) { return a; }
template <> __device__ __forceinline__ F2 splat<F2>(float a) { return pair(a, a); }
// VE values as VE / 2 pairs (or the one value)
template <int VE> struct Lanes {
  using P = F2;
  static constexpr int N = VE / 2;
  static __device__ __forceinline__ void from(const float (&f)[VE], P (&p)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = pair(f[2 * i], f[2 * i + 1]);
  }
  static __device__ __forceinline__ void to(const P (&p)[N], float (&f)[VE]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f[2 * i] = low(p[i]);
      f[2 * i + 1] = high(p[i]);
    }
  }
};
template <> struct Lanes<1> {
  using P = float;
  static constexpr int N = 1;
  static __device__ __forceinline__ void from(const float (&f)[1], P (&p)[1]) { p[0] = f[0]; }
  static __device__ __forceinline__ void to(const P (&p)[1], float (&f)[1]) { f[0] = p[0]; }
};

// Backward kernels: persistent blocks, a block walks its rows with the column sums of its threads' columns in
// registers.  A thread copies its own packs of the rows to come into shared memory (asynchronously, `stages` rows ahead)
// and is the only one to read them back, so the loads of later rows run under a row's reductions without any barrier.
template <int N> static __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
static __device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
static __device__ __forceinline__ void copies_wait_for(int stages) {  // all but the stages - 1 youngest groups are there
  if (stages >= 4) copies_wait<3>();
  else if (stages == 3) copies_wait<2>();
  else if (stages == 2) copies_wait<1>();
  else copies_wait<0>();
}

// NIN row-wise inputs of the rows to come: through the ring (VE > 1) or straight from memory when they are used.
template <typename T, int VE, int NV, int NIN> struct RowFeed {
  const Rows (&in)[NIN];
  int64_t rows;
  int packs, stages;
  uint32_t mine, pitch;  // shared address of this thread's first pack; bytes from one input's packs to the next's
  uint32_t row_bytes;    // ... and from one row's to the next's

  __device__ __forceinline__ RowFeed(const Rows (&m)[NIN], int64_t T_, int packs_, int stages_, int nin, uint4* ring)
      : in(m), rows(T_), packs(packs_), stages(stages_) {
    mine = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    pitch = NV * blockDim.x * 16;
    row_bytes = nin * pitch;
  }
  __device__ __forceinline__ uint32_t next(uint32_t at) const { return at + row_bytes == stages * row_bytes ? 0 : at + row_bytes; }
  // `at`: byte offset of the row's slot in the ring
  __device__ __forceinline__ void request(int64_t t, uint32_t at) const {
    if constexpr (VE > 1) {
      if (t < rows)
#pragma unroll
        for (int i = 0; i < NIN; ++i) {
          if (!in[i].p) continue;
          const char* row = reinterpret_cast<const char*>(row_at<T>(in[i], t));
#pragma unroll
          for (int n = 0; n < NV; ++n) {
            const uint32_t c = threadIdx.x + n * blockDim.x;
            if ((int)c < packs)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + at + i * pitch + n * blockDim.x * 16), "l"(row + c * 16u)
                           : "memory");
          }
        }
      copies_commit();
    }
  }
  // until the oldest `n` rows of the ring are there
  __device__ __forceinline__ void wait_for(int n) const {
    if constexpr (VE > 1) copies_wait_for(stages - n + 1);
  }
  __device__ __forceinline__ Pack<T, VE> get(int i, int64_t t, uint32_t at, int n) const {
    if constexpr (VE > 1) {
      Pack<T, VE> v;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v.r.x), "=r"(v.r.y), "=r"(v.r.z), "=r"(v.r.w) : "r"(mine + at + i * pitch + n * blockDim.x * 16) : "memory");
      return v;
    } else {
      return load_once<T, VE>(row_at<T>(in[i], t) + (int64_t)(threadIdx.x + n * blockDim.x) * VE);
    }
  }
  __device__ __forceinline__ void get(int i, int64_t t, uint32_t at, int n, typename Lanes<VE>::P (&p)[Lanes<VE>::N]) const {
    float f[VE];
    get(i, t, at, n).widen(f);
    Lanes<VE>::from(f, p);
  }
};
template <typename T, int VE>
static __device__ __forceinline__ void store_lanes(void* p, int64_t stride, int64_t t, int c, const typename Lanes<VE>::P (&v)[Lanes<VE>::N]) {
  float f[VE];
  Lanes<VE>::to(v, f);
  store_row<T, VE>(p, stride, t, c, f);
}

// The 8-bit norms of many rows.  Done as k_codes_rows does them they are bound by instruction issue (so 72 us for
// 8192 x 7168 bf16, 5.7 TB/s).  So persistent blocks, whose threads hold their columns' gains (with the branch's factor and a gate per
// channel in them) as pairs of fp32 in registers and work on pairs; whose next rows are on their way meanwhile; and one reduction a row,
// which brings the branch's sum of squares of the row to come with it.
//   TWO: the sum of x and a branch; FULL: with a gate per value
template <typename T, int VE, int NV, int MAXT, bool TWO, bool FULL>
__global__ void __launch_bounds__(MAXT, NV == 2 ? 2 : 1) k_codes_feed(NormArgs A, int packs, int stages) {
  extern __shared__ uint4 ring[];
  __shared__ float buf[3][96];  // one reduction a row, its buffers in turn
  using L = Lanes<VE>;
  using P = typename L::P;
  constexpr int N = L::N, NIN = FULL ? 3 : TWO ? 2 : 1;
  const Rows in[3] = {A.x, TWO ? A.y : Rows{nullptr, 0}, FULL ? A.gate : Rows{nullptr, 0}};
  const RowFeed<T, VE, NV, 3> F(in, A.T, packs, stages, NIN, ring);
  P wy[NV][N], wn[NV][N];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    float f[VE], g[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = g[j] = 0.f;
    if (c < packs) load_gains<VE>(A.wn, A.wdt, (int64_t)c * VE, f);
    L::from(f, wn[n]);
    if constexpr (TWO) {
      if (c < packs) {
        load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, f);
        if (A.gate_kind == DEAMOE_GATE_CHANNEL) load_gate<T, VE>(A, 0, c, g);
      }
#pragma unroll
      for (int j = 0; j < VE; ++j) f[j] *= A.gate_kind == DEAMOE_GATE_CHANNEL ? A.b * g[j] : A.b;
      L::from(f, wy[n]);
    }
  }
  uint32_t at = 0, to = 0;
  int64_t ahead = blockIdx.x;
  for (int i = 0; i < stages; ++i, ahead += gridDim.x) {
    F.request(ahead, to);
    to = F.next(to);
  }
  auto squares = [&](int64_t t, uint32_t slot) {  // of this thread's columns of a row's branch
    P sq = splat<P>(0.f);
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if ((int)(threadIdx.x + n * blockDim.x) < packs) {
        P y[N];
        F.get(1, t, slot, n, y);
#pragma unroll
        for (int j = 0; j < N; ++j) sq = fma_(y[j], y[j], sq);
      }
    return total(sq);
  };
  const bool post = TWO && A.post_norm;
  const float per_value = 1.f / (float)A.h;
  float ry = 1.f;  // of the row to come: its sum goes with the reduction of the row before it
  if (post) {
    F.wait_for(1);
    float ss[1] = {squares(blockIdx.x, 0)};
    block_sums<1>(ss, buf[0]);
    ry = inv_rms(ss[0], A.h, A.eps);
  }
  int flip = 1;
  for (int64_t t = blockIdx.x; t < A.T; t += gridDim.x, ahead += gridDim.x) {
    F.wait_for(post ? 2 : 1);
    P s[NV][N];
    float cy = ry;
    if (TWO && A.gate_kind == DEAMOE_GATE_TOKEN) cy *= to_f<T>(reinterpret_cast<const T*>(A.gate.p)[t]);
    const P cy2 = splat<P>(cy), a2 = splat<P>(A.a);
    P sq = splat<P>(0.f);
    float m = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = threadIdx.x + n * blockDim.x;
      if (c >= packs) continue;
      F.get(0, t, at, n, s[n]);
      if constexpr (TWO) {
        P y[N];
        F.get(1, t, at, n, y);
        if constexpr (FULL) {
          P g[N];
          F.get(2, t, at, n, g);
#pragma unroll
          for (int j = 0; j < N; ++j) y[j] = mul_(y[j], g[j]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) s[n][j] = fma_(a2, s[n][j], mul_(cy2, mul_(y[j], wy[n][j])));
        store_lanes<T, VE>(A.out, A.out_s, t, c, s[n]);
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        sq = fma_(s[n][j], s[n][j], sq);
        s[n][j] = mul_(s[n][j], wn[n][j]);
        m = max_or_nan(max_or_nan(m, fabsf(low(s[n][j]))), fabsf(high(s[n][j])));
      }
    }
    float v[3] = {m, total(sq), 0.f};
    if (post && t + gridDim.x < A.T) v[2] = squares(t + gridDim.x, F.next(at));
    F.request(ahead, at);  // the row has been read: its slot takes the one `stages` further
    at = F.next(at);
    block_max_two_sums(v[0], v[1], v[2], buf[flip]);
    flip = 3 - flip;
    if (post) ry = rsqrtf(fmaf(v[2], per_value, A.eps));
    const P f2 = splat<P>(row_scale(A, t, v[1], v[0]));
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = threadIdx.x + n * blockDim.x;
      if (c >= packs) continue;
      float f[VE];
#pragma unroll
      for (int j = 0; j < N; ++j) s[n][j] = mul_(s[n][j], f2);
      L::to(s[n], f);
      store_codes<VE>(A.codes + t * A.codes_s + (int64_t)c * VE, f);
    }
  }
}

template <typename T, int VE, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT, 1) k_norm_grad_rows(NormArgs A, int packs, int stages) {
  extern __shared__ uint4 ring[];
  __shared__ float buf[2][64];  // taken in turn: a sum's buffer is free again after the next sum's barrier
  const Rows in[3] = {A.x, A.du, A.dadd};
  const RowFeed<T, VE, NV, 3> F(in, A.T, packs, stages, A.dadd.p ? 3 : 2, ring);
  const bool add = A.dadd.p != nullptr;
  using L = Lanes<VE>;
  using P = typename L::P;
  constexpr int N = L::N;
  P acc[NV][N], w[NV][N];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    float f[VE] = {};
    if (c < packs) load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, f);
    L::from(f, w[n]);
#pragma unroll
    for (int j = 0; j < N; ++j) acc[n][j] = splat<P>(0.f);
  }
  const float inv_h = 1.f / (float)A.h;
  for (int i = 0; i < stages; ++i) F.request(blockIdx.x + (int64_t)i * gridDim.x, i * F.row_bytes);
  uint32_t stage = 0;
  int flip = 0;
  for (int64_t t = blockIdx.x; t < A.T; t += gridDim.x) {
    Pack<T, VE> px[NV], pd[NV];
    P s0 = splat<P>(0.f), s1 = s0;
    F.wait_for(1);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if ((int)(threadIdx.x + n * blockDim.x) >= packs) continue;
      float f[VE];
      P x[N], d[N];
      px[n] = F.get(0, t, stage, n);
      pd[n] = F.get(1, t, stage, n);
      px[n].widen(f);
      L::from(f, x);
      pd[n].widen(f);
      L::from(f, d);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        s0 = fma_(x[j], x[j], s0);
        s1 = fma_(mul_(d[j], w[n][j]), x[j], s1);
      }
    }
    float s[2] = {total(s0), total(s1)};
    block_sums_many<2, 2>(s, buf[flip]);
    flip ^= 1;
    const float r = inv_rms(s[0], A.h, A.eps);
    const P r2 = splat<P>(r), c2 = splat<P>(-cube_times(r, s[1] * inv_h));
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = threadIdx.x + n * blockDim.x;
      if (c >= packs) continue;
      float f[VE];
      P x[N], d[N];
      px[n].widen(f);
      L::from(f, x);
      pd[n].widen(f);
      L::from(f, d);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        d[j] = mul_(r2, d[j]);
        acc[n][j] = fma_(d[j], x[j], acc[n][j]);
        d[j] = fma_(d[j], w[n][j], mul_(x[j], c2));
      }
      if (add) {
        P e[N];
        F.get(2, t, stage, n, e);
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] = fma_(splat<P>(1.f), e[j], d[j]);
      }
      store_lanes<T, VE>(A.dx, A.dx_s, t, c, d);
    }
    F.request(t + (int64_t)stages * gridDim.x, stage);
    stage = F.next(stage);
  }
  float* part = A.part + (size_t)blockIdx.x * A.h;
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
    float f[VE];
    L::to(acc[n], f);
#pragma unroll
    for (int j = 0; j < VE; ++j) part[(size_t)c * VE + j] = f[j];
  }
}

// With p = b g w (a column's constant unless the gate is full), gt the token's gate (or 1) and gr = gt ry:
//   s = a x + gr p y,   D = dout + ro du wn - co s,   dx = a D,   sum3 = sum p D y,
//   dy = gr p D - y gr ry^2 sum3 / h,   dgate_token = ry sum3,   E = gr D y,
//   dw = b g sum_t E,   dgate_channel = b w sum_t E   -- one accumulator a column for both.
// sum3 = sum p y dout + ro sum p y du wn - co sum p y s, so all of a row's sums are taken before ro and co are known,
// and the sum of the next row's y^2 with them: one reduction and one barrier a row, not three in turn.  That one is still
// what a row waits for (4096 x 7168 bf16: 100 us, of which some 45 are issue): the column constants p and q and the sums
// take the registers that a second block would need to work meanwhile.
template <typename T, int VE, int NV, int MAXT, bool FULL>
__global__ void __launch_bounds__(MAXT, 1) k_residual_grad_rows(NormArgs A, int packs, int stages, size_t part_step) {
  extern __shared__ uint4 ring[];
  __shared__ float buf[2][256];
  const Rows in[5] = {A.x, A.y, A.dout, A.du, {FULL ? A.gate.p : nullptr, A.gate.stride}};
  const RowFeed<T, VE, NV, 5> F(in, A.T, packs, stages, FULL ? 5 : 4, ring);
  using L = Lanes<VE>;
  using P = typename L::P;
  constexpr int N = L::N;
  P acc_e[NV][N], acc_n[NV][N], p[NV][N], q[NV][N];
  auto channel_gate = [&](int c, float (&g)[VE]) {
#pragma unroll
    for (int j = 0; j < VE; ++j) g[j] = 1.f;
    if (A.gate_kind == DEAMOE_GATE_CHANNEL) load_pack<T, VE>(reinterpret_cast<const T*>(A.gate.p) + (int64_t)c * VE).widen(g);
  };
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    float w[VE] = {}, wn[VE] = {}, g[VE];
    if (c < packs) {
      channel_gate(c, g);
      load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, w);
      load_gains<VE>(A.wn, A.wdt, (int64_t)c * VE, wn);
#pragma unroll
      for (int j = 0; j < VE; ++j) w[j] *= A.b * g[j];
    }
    L::from(w, p[n]);
    L::from(wn, q[n]);
#pragma unroll
    for (int j = 0; j < N; ++j) acc_e[n][j] = acc_n[n][j] = splat<P>(0.f);
  }
  auto squares = [&](int64_t t, uint32_t stage) {  // of y
    P ss = splat<P>(0.f);
    if (A.post_norm && t < A.T)
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const int c = threadIdx.x + n * blockDim.x;
        if (c >= packs) continue;
        P y[N];
        if (stages > 1) {
          F.get(1, t, stage, n, y);
        } else {  // no room for two rows
          float f[VE];
          load_pack<T, VE>(row_at<T>(A.y, t) + (int64_t)c * VE).widen(f);
          L::from(f, y);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) ss = fma_(y[j], y[j], ss);
      }
    return total(ss);
  };
  const float inv_h = 1.f / (float)A.h;
  const P a2 = splat<P>(A.a);
  for (int i = 0; i < stages; ++i) F.request(blockIdx.x + (int64_t)i * gridDim.x, i * F.row_bytes);
  uint32_t stage = 0;
  int flip = 0;
  float s[6];
  F.wait_for(1);
  s[0] = squares(blockIdx.x, 0);
  block_sums_many<1, 2>(reinterpret_cast<float(&)[1]>(s), buf[flip]);
  flip ^= 1;
  for (int64_t t = blockIdx.x; t < A.T; t += gridDim.x) {
    const float gt = A.gate_kind == DEAMOE_GATE_TOKEN ? to_f<T>(reinterpret_cast<const T*>(A.gate.p)[t]) : 1.f;
    const float ry = A.post_norm ? inv_rms(s[0], A.h, A.eps) : 1.f;
    const float gr = gt * ry;
    const P gr2 = splat<P>(gr);
    const uint32_t later = F.next(stage);
    F.wait_for(2);  // this row and the next
    P s1 = splat<P>(0.f), s2 = s1, s3 = s1, s4 = s1, s5 = s1;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if ((int)(threadIdx.x + n * blockDim.x) >= packs) continue;
      P x[N], y[N], u[N], o[N], g[N];
      F.get(1, t, stage, n, y);
      F.get(2, t, stage, n, o);
      if constexpr (FULL) F.get(4, t, stage, n, g);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        y[j] = mul_(FULL ? mul_(p[n][j], g[j]) : p[n][j], y[j]);  // p y
        s3 = fma_(y[j], o[j], s3);
      }
      if (A.next_norm) {
        F.get(0, t, stage, n, x);
        F.get(3, t, stage, n, u);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const P sum = fma_(gr2, y[j], mul_(a2, x[j])), uq = mul_(u[j], q[n][j]);
          s1 = fma_(sum, sum, s1);
          s2 = fma_(uq, sum, s2);
          s4 = fma_(y[j], uq, s4);
          s5 = fma_(y[j], sum, s5);
        }
      }
    }
    s[0] = squares(t + gridDim.x, later);
    s[1] = total(s1); s[2] = total(s2); s[3] = total(s3); s[4] = total(s4); s[5] = total(s5);
    block_sums_many<6, 8>(s, buf[flip]);
    flip ^= 1;
    const float ro = A.next_norm ? inv_rms(s[1], A.h, A.next_eps) : 0.f;
    const float co = cube_times(ro, s[2] * inv_h);
    const float sum3 = s[3] + ro * s[4] - co * s[5];
    const float cy = A.post_norm ? (gr * ry) * (ry * (sum3 * inv_h)) : 0.f;
    if (A.dgate_token && threadIdx.x == 0) A.dgate_token[t] = ry * sum3;
    const P ro2 = splat<P>(ro), co2 = splat<P>(-co), cy2 = splat<P>(-cy);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = threadIdx.x + n * blockDim.x;
      if (c >= packs) continue;
      P o[N], y[N], g[N], dx[N];
      F.get(2, t, stage, n, o);
      F.get(1, t, stage, n, y);
      if constexpr (FULL) F.get(4, t, stage, n, g);
      if (A.next_norm) {
        P x[N], u[N];
        F.get(0, t, stage, n, x);
        F.get(3, t, stage, n, u);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const P sum = fma_(gr2, mul_(FULL ? mul_(p[n][j], g[j]) : p[n][j], y[j]), mul_(a2, x[j])), ru = mul_(ro2, u[j]);
          acc_n[n][j] = fma_(ru, sum, acc_n[n][j]);
          o[j] = fma_(ru, q[n][j], fma_(co2, sum, o[j]));
        }
      }
#pragma unroll
      for (int j = 0; j < N; ++j) dx[j] = mul_(a2, o[j]);
      store_lanes<T, VE>(A.dx, A.dx_s, t, c, dx);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const P gd = mul_(gr2, o[j]), yc = mul_(y[j], cy2);
        if constexpr (FULL) {
          dx[j] = mul_(mul_(p[n][j], gd), y[j]);  // dgate
          const P gg = mul_(g[j], gd);
          acc_e[n][j] = fma_(gg, y[j], acc_e[n][j]);
          o[j] = fma_(p[n][j], gg, yc);
        } else {
          acc_e[n][j] = fma_(gd, y[j], acc_e[n][j]);
          o[j] = fma_(p[n][j], gd, yc);
        }
      }
      if constexpr (FULL) store_lanes<T, VE>(A.dgate, A.dgate_s, t, c, dx);
      store_lanes<T, VE>(A.dy, A.dy_s, t, c, o);
    }
    F.request(t + (int64_t)stages * gridDim.x, stage);
    stage = later;
  }
  float* part = A.part + (size_t)blockIdx.x * A.h;
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = threadIdx.x + n * blockDim.x;
    if (c >= packs) continue;
    float w[VE], g[VE], ae[VE], an[VE];
    channel_gate(c, g);
    load_gains<VE>(A.w, A.wdt, (int64_t)c * VE, w);
    L::to(acc_e[n], ae);
    L::to(acc_n[n], an);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const size_t i = (size_t)c * VE + j;
      if (A.w) part[i] = A.b * g[j] * ae[j];
      if (A.wn) part[part_step + i] = an[j];
      if (A.gate_kind == DEAMOE_GATE_CHANNEL) part[2 * part_step + i] = A.b * w[j] * ae[j];
    }
  }
}

// ---------------------------------------------------------------- sums over the blocks' partial rows

struct ColumnSums {
  const float* part[3];
  float* out[3];
};
// A block adds 32 CE columns of one array: 8 row groups side by side, then the groups in order.  CE: columns a thread, 4
// where rows start on 16-byte boundaries.
template <int CE> __global__ void __launch_bounds__(256) k_column_sums(ColumnSums S, int rows, int h) {
  __shared__ float acc[8][32 * CE];
  pdl_wait();
  const float* p = S.part[blockIdx.y];
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * CE;
  float s[CE] = {};
  if (c < h) {
#pragma unroll 8
    for (int r = g; r < rows; r += 8) {
      float v[CE];
      if constexpr (CE == 4) load_pack<float, 4>(p + (size_t)r * h + c).widen(v);
      else v[0] = p[(size_t)r * h + c];
#pragma unroll
      for (int j = 0; j < CE; ++j) s[j] += v[j];
    }
  }
#pragma unroll
  for (int j = 0; j < CE; ++j) acc[g][j * 32 + lane] = s[j];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * CE; i += 256) {
    const int col = (blockIdx.x * 32 + (i & 31)) * CE + (i >> 5);
    if (col >= h) continue;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) t += acc[k][i];
    S.out[blockIdx.y][col] = t;
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
  const cudaError_t e = h % 4 == 0 ? launch_pdl(k_column_sums<4>, dim3((h + 127) / 128, arrays), dim3(256), 0, s, S, rows, h)
                                   : launch_pdl(k_column_sums<1>, dim3((h + 31) / 32, arrays), dim3(256), 0, s, S, rows, h);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return DEAMOE_ERR_CUDA;
  }
  return DEAMOE_OK;
}

static deamoe_status_t ran() { return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA; }

// Lets a kernel use the SM's whole shared memory; once per kernel and device.
template <typename K> static bool whole_smem(K* fn, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  if (done.load(std::memory_order_acquire) >> dev & 1) return true;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_BYTES) != cudaSuccess) return false;
  done.fetch_or(1ull << dev, std::memory_order_release);
  return true;
}

// Whether all of a call's rows and gains can be read 16 bytes at a time.
template <typename T> static bool wide_call(const NormArgs& A) {
  bool ok = A.h % (16 / sizeof(T)) == 0;
  for (const Rows& m : {A.x, A.y, A.dout, A.du, A.dadd})
    if (m.p) ok = ok && wide_rows(m.p, m.stride, A.T, sizeof(T));
  if (A.gate_kind == DEAMOE_GATE_FULL) ok = ok && wide_rows(A.gate.p, A.gate.stride, A.T, sizeof(T));
  if (A.gate_kind == DEAMOE_GATE_CHANNEL) ok = ok && aligned16(A.gate.p);
  ok = ok && aligned16(A.w) && aligned16(A.wn) && wide_rows(A.out, A.out_s, A.T, sizeof(T)) &&
       wide_rows(A.u, A.u_s, A.T, sizeof(T)) && wide_rows(A.dx, A.dx_s, A.T, sizeof(T)) &&
       wide_rows(A.dy, A.dy_s, A.T, sizeof(T));
  if (A.gate_kind == DEAMOE_GATE_FULL) ok = ok && wide_rows(A.dgate, A.dgate_s, A.T, sizeof(T));
  // the codes of 16 bytes of values: 8 bytes, or 4
  if (A.codes) ok = ok && aligned_to(A.codes, 16 / sizeof(T)) && (A.T == 1 || A.codes_s % (16 / sizeof(T)) == 0);
  return ok;
}

static unsigned warps_of(int packs, int nv) { return (unsigned)(((packs + nv - 1) / nv + 31) / 32 * 32); }
// Few rows: one pack a thread, the shortest way through a row (norm of 8 rows of 7168 bf16 values: 2.2 us, 2.8 with four;
// 296 rows 3.0 / 3.8).  Many: four, so that the rows in flight on an SM are enough bytes to keep HBM busy (592 rows 4.3
// us, 4.8 with one; 8192 rows 37 / 67).
static bool few_rows(int64_t T) { return T <= 2 * NORM_SMS; }

#define DEAMOE_ROW_FORMS(KERNEL, ANY)                                                                                   \
  constexpr int VE = 16 / sizeof(T);                                                                                     \
  const unsigned grid = (unsigned)A.T;                                                                                   \
  if (wide_call<T>(A)) {                                                                                                 \
    const int packs = A.h / VE;                                                                                          \
    if (packs <= 1024 && (few_rows(A.T) || packs < 128)) {                                                               \
      KERNEL<T, VE, 1, 1024><<<grid, warps_of(packs, 1), 0, s>>>(A, packs);                                              \
      return ran();                                                                                                      \
    }                                                                                                                    \
    if (packs <= 2048) {                                                                                                 \
      KERNEL<T, VE, 4, 512><<<grid, warps_of(packs, 4), 0, s>>>(A, packs);                                               \
      return ran();                                                                                                      \
    }                                                                                                                    \
  } else if (A.h <= 2048) {                                                                                              \
    KERNEL<T, 1, 4, 512><<<grid, warps_of(A.h, 4), 0, s>>>(A, A.h);                                                      \
    return ran();                                                                                                        \
  } else if (A.h <= 8192) {                                                                                              \
    KERNEL<T, 1, 16, 512><<<grid, warps_of(A.h, 16), 0, s>>>(A, A.h);                                                    \
    return ran();                                                                                                        \
  }                                                                                                                      \
  ANY<T><<<grid, ANY_THREADS, 0, s>>>(A);                                                                                \
  return ran()

template <typename T> static deamoe_status_t norm_t(const NormArgs& A, cudaStream_t s) {
  DEAMOE_ROW_FORMS(k_norm_rows, k_norm_any);
}
template <typename T> static deamoe_status_t residual_t(const NormArgs& A, cudaStream_t s) {
  DEAMOE_ROW_FORMS(k_residual_rows, k_residual_any);
}
template <typename T> static deamoe_status_t codes_rows_t(const NormArgs& A, cudaStream_t s) {
  DEAMOE_ROW_FORMS(k_codes_rows, k_codes_any);
}
#undef DEAMOE_ROW_FORMS

// Rows ahead in the ring: what the blocks of an SM can share of its shared memory, four at most.  All of an SM's blocks have
// to be resident: one that waits for another's end makes the grid twice as long (4096 x 3584 bf16, where two blocks miss
// it by 2 KB if their own needs are not counted: 83 us, 64 with one stage less).
static constexpr int grad_stages(int blocks_per_sm, size_t stage_bytes) {
  const size_t n = (SM_SMEM / blocks_per_sm - BLOCK_SMEM) / stage_bytes;
  return n > 4 ? 4 : (n < 1 ? 1 : (int)n);
}
static constexpr bool grad_blocks_fit() {
  for (int threads = 32; threads <= 512; threads += 32)
    for (int blocks = 1; blocks <= 8 && blocks * threads <= 512; ++blocks)
      for (int inputs = 2; inputs <= 5; ++inputs)
        for (int value_bytes = 2; value_bytes <= 4; value_bytes += 2) {
          const size_t stage = (size_t)inputs * GRAD_COLUMNS * value_bytes * threads;
          if (blocks * (stage * grad_stages(blocks, stage) + BLOCK_SMEM) > SM_SMEM) return false;
        }
  return true;
}
static_assert(grad_blocks_fit(), "an SM's blocks of the gradient kernels do not fit its shared memory");
template <typename K, typename... Rest>
static deamoe_status_t run_grad(K* kernel, std::atomic<uint64_t>& done, const NormArgs& A, int ctas, int threads, int packs,
                                size_t stage_bytes, cudaStream_t s, Rest... rest) {
  int stages = 1;
  if (stage_bytes) {
    if (!whole_smem(kernel, done)) return DEAMOE_ERR_CUDA;
    stages = grad_stages((ctas + NORM_SMS - 1) / NORM_SMS, stage_bytes);
  }
  kernel<<<ctas, threads, stage_bytes * stages, s>>>(A, packs, stages, rest...);
  return ran();
}

template <typename T> static deamoe_status_t codes_t(const NormArgs& A, cudaStream_t s) {
  constexpr int VE = 16 / sizeof(T), NV = 4;
  const int packs = A.h / VE;
  // (a sum of narrow rows leaves the persistent blocks too few columns beside a row's fixed work: 16384 x 1024 25.8 us, 23.4 with a block a
  // row; without a sum 9.0, 13.0)
  if (few_rows(A.T) || !wide_call<T>(A) || packs < 128 || packs > 2048 || (A.y.p && A.gate_kind != DEAMOE_GATE_FULL && packs <= 256))
    return codes_rows_t<T>(A, s);
  const int nin = A.gate_kind == DEAMOE_GATE_FULL ? 3 : A.y.p ? 2 : 1;
  auto run = [&](auto kernel, std::atomic<uint64_t>& done, int nv, int sm_threads) {
    const int threads = (int)warps_of(packs, nv);
    const size_t stage = (size_t)nin * nv * threads * 16;
    int blocks = sm_threads / threads;
    while (blocks > 1 && grad_stages(blocks, stage) < 2) --blocks;  // a row and the one to come
    const int stages = grad_stages(blocks, stage);
    const int64_t most = (int64_t)NORM_SMS * blocks;
    if (!whole_smem(kernel, done)) return DEAMOE_ERR_CUDA;
    kernel<<<(unsigned)(A.T < most ? A.T : most), threads, stage * stages, s>>>(A, packs, stages);
    return ran();
  };
  static std::atomic<uint64_t> done[5];
  // Sums of rows of 513 to 896 packs: twice the threads with half the columns, two blocks an SM (448 threads are what two of them can have
  // registers for).  With this and with four packs a thread, us: bf16 14115 x 4160 79 and 86, 11468 x 5120 77 and 76, 8340 x 7040 73 and 81,
  // 8192 x 7168 72 and 80, with a gate of its own 84 and 95; fp32 14115 x 2080 72 and 70, 11468 x 2560 65 and 68, 8192 x 3584 69 and 68.
  if (nin > 1 && packs > 512 && packs <= 896)
    return nin == 3 ? run(k_codes_feed<T, VE, 2, 448, true, true>, done[0], 2, 896) : run(k_codes_feed<T, VE, 2, 448, true, false>, done[1], 2, 896);
  return nin == 3 ? run(k_codes_feed<T, VE, NV, CODES_THREADS, true, true>, done[2], NV, CODES_THREADS)
       : nin == 2 ? run(k_codes_feed<T, VE, NV, CODES_THREADS, true, false>, done[3], NV, CODES_THREADS)
                  : run(k_codes_feed<T, VE, NV, CODES_THREADS, false, false>, done[4], NV, CODES_THREADS);
}
// (rows of up to 2048 packs with a gate of their own take 96 KB a stage: two fit one block's ring)
static_assert(2 * 3 * 4 * 512 * 16 <= RING_BYTES, "two rows in a ring");

template <typename T> static deamoe_status_t norm_grad_t(const NormArgs& A, cudaStream_t s) {
  constexpr int VE = 16 / sizeof(T), NV = GRAD_COLUMNS / VE;
  const int ctas = grad_ctas(A.T, A.h), threads = grad_threads(A.h);
  static std::atomic<uint64_t> done[2];
  if (A.h > GRAD_MAX_WIDTH) {
    k_norm_grad_any<T><<<ctas, ANY_THREADS, 0, s>>>(A);
    return ran();
  }
  if (!wide_call<T>(A)) return run_grad(k_norm_grad_rows<T, 1, GRAD_ODD_COLUMNS, 1024>, done[0], A, ctas, grad_threads(A.h, GRAD_ODD_COLUMNS), A.h, 0, s);
  return run_grad(k_norm_grad_rows<T, VE, NV, 512>, done[1], A, ctas, threads, A.h / VE,
                  (size_t)(A.dadd.p ? 3 : 2) * NV * threads * 16, s);
}

template <typename T> static deamoe_status_t residual_grad_t(const NormArgs& A, cudaStream_t s) {
  constexpr int VE = 16 / sizeof(T), NV = GRAD_COLUMNS / VE;
  const int ctas = grad_ctas(A.T, A.h), threads = grad_threads(A.h), odd = grad_threads(A.h, GRAD_ODD_COLUMNS);
  const size_t step = (size_t)ctas * A.h;
  static std::atomic<uint64_t> done[4];
  if (A.h > GRAD_MAX_WIDTH) {
    k_residual_grad_any<T><<<ctas, ANY_THREADS, 0, s>>>(A, step);
    return ran();
  }
  const bool full = A.gate_kind == DEAMOE_GATE_FULL, wide = wide_call<T>(A);
  const size_t stage = wide ? (size_t)(full ? 5 : 4) * NV * threads * 16 : 0;
  const int packs = wide ? A.h / VE : A.h;
  if (!wide)
    return full ? run_grad(k_residual_grad_rows<T, 1, GRAD_ODD_COLUMNS, 1024, true>, done[0], A, ctas, odd, packs, stage, s, step)
                : run_grad(k_residual_grad_rows<T, 1, GRAD_ODD_COLUMNS, 1024, false>, done[1], A, ctas, odd, packs, stage, s, step);
  return full ? run_grad(k_residual_grad_rows<T, VE, NV, 512, true>, done[2], A, ctas, threads, packs, stage, s, step)
              : run_grad(k_residual_grad_rows<T, VE, NV, 512, false>, done[3], A, ctas, threads, packs, stage, s, step);
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_norm_workspace(int32_t n_token, int32_t hidden) {
  if (n_token <= 0 || hidden <= 0) return 0;
  return (uint64_t)3 * grad_ctas(n_token, hidden) * hidden * sizeof(float);
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
  return launch_sums(S, 1, grad_ctas(n_token, hidden), hidden, s);
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

deamoe_status_t deamoe_norm_quant(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, int32_t n_token, int32_t hidden,
                                  int32_t normalise, int32_t weight_dtype, const void* weight, float eps, void* codes,
                                  int64_t codes_stride, float* scale) {
  deamoe_status_t st = check_norm(dtype, weight_dtype, n_token, hidden, eps);
  if (st == DEAMOE_OK && normalise != 0 && normalise != 1) st = DEAMOE_ERR_INVALID_ARG;
  if (st != DEAMOE_OK || n_token == 0) return st;
  if (bad_rows(x, x_stride, hidden, type_bytes(dtype)) || bad_rows(codes, codes_stride, hidden, 1) || !scale || !aligned_to(scale, 4) ||
      !aligned_to(weight, type_bytes(weight_dtype)) || codes == x)
    return DEAMOE_ERR_INVALID_ARG;
  NormArgs A = {};
  A.T = n_token; A.h = hidden; A.wdt = weight_dtype; A.next_eps = eps; A.next_norm = normalise; A.wn = weight;
  A.x = {x, x_stride}; A.codes = reinterpret_cast<uint8_t*>(codes); A.codes_s = codes_stride; A.scale = scale;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32 ? codes_t<float>(A, s) : codes_t<__nv_bfloat16>(A, s);
}

deamoe_status_t deamoe_norm_residual_quant(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, const void* y,
                                           int64_t y_stride, int32_t n_token, int32_t hidden, int32_t normalise,
                                           int32_t weight_dtype, const void* weight, float eps, int32_t gate_kind,
                                           const void* gate, int64_t gate_stride, float residual_scale, float branch_scale,
                                           void* out, int64_t out_stride, const void* next_weight, float next_eps, void* codes,
                                           int64_t codes_stride, float* scale) {
  deamoe_status_t st = check_norm(dtype, weight_dtype, n_token, hidden, eps);
  if (st == DEAMOE_OK && !(next_eps >= 0.f)) st = DEAMOE_ERR_INVALID_ARG;
  if (st != DEAMOE_OK || n_token == 0) return st;
  const size_t es = type_bytes(dtype), ws = type_bytes(weight_dtype);
  if (bad_rows(x, x_stride, hidden, es) || bad_rows(y, y_stride, hidden, es) || bad_rows(out, out_stride, hidden, es) ||
      bad_rows(codes, codes_stride, hidden, 1) || !scale || !aligned_to(scale, 4) || !aligned_to(weight, ws) ||
      !aligned_to(next_weight, ws))
    return DEAMOE_ERR_INVALID_ARG;
  if ((out == x && out_stride != x_stride) || out == y || codes == x || codes == y || codes == out) return DEAMOE_ERR_INVALID_ARG;
  st = check_block(gate_kind, gate, gate_stride, hidden, es, normalise, weight, residual_scale, branch_scale);
  if (st != DEAMOE_OK) return st;
  NormArgs A = {};
  A.T = n_token; A.h = hidden; A.wdt = weight_dtype; A.eps = eps; A.next_eps = next_eps;
  A.a = residual_scale; A.b = branch_scale; A.gate_kind = gate_kind; A.post_norm = normalise; A.next_norm = 1;
  A.x = {x, x_stride}; A.y = {y, y_stride}; A.gate = {gate, gate_stride}; A.w = weight; A.wn = next_weight;
  A.out = out; A.out_s = out_stride; A.codes = reinterpret_cast<uint8_t*>(codes); A.codes_s = codes_stride; A.scale = scale;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32 ? codes_t<float>(A, s) : codes_t<__nv_bfloat16>(A, s);
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
  const size_t step = (size_t)grad_ctas(n_token, hidden) * hidden;
  if (dweight) { S.part[n] = A.part; S.out[n++] = dweight; }
  if (dnext_weight) { S.part[n] = A.part + step; S.out[n++] = dnext_weight; }
  if (gate_kind == DEAMOE_GATE_CHANNEL) { S.part[n] = A.part + 2 * step; S.out[n++] = reinterpret_cast<float*>(dgate); }
  return launch_sums(S, n, grad_ctas(n_token, hidden), hidden, s);
}

}  // extern "C"
