// Shared pieces of the operators around a layer (tokens.cu, norm.cu, quant.cu): rows of fp32 or bf16 values with a
// row stride, read and written 16 bytes or one value at a time, and sums over a thread block.
#pragma once
#include "deamoe_internal.cuh"

namespace deamoe {

template <typename T> static __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> static __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// VE consecutive values of a row as one register group: VE = 16 bytes of them where base and stride allow, else 1.
template <typename T, int VE> struct Pack;
template <> struct Pack<__nv_bfloat16, 8> {
  uint4 r;
  __device__ __forceinline__ void widen(float (&f)[8]) const {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void narrow(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    r = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <> struct Pack<float, 4> {
  uint4 r;
  __device__ __forceinline__ void widen(float (&f)[4]) const {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  }
  __device__ __forceinline__ void narrow(const float (&f)[4]) {
    r = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <typename T> struct Pack<T, 1> {
  T r;
  __device__ __forceinline__ void widen(float (&f)[1]) const { f[0] = to_f<T>(r); }
  __device__ __forceinline__ void narrow(const float (&f)[1]) { r = from_f<T>(f[0]); }
};

template <typename T, int VE> static __device__ __forceinline__ Pack<T, VE> load_pack(const T* p) {
  Pack<T, VE> v;
  if constexpr (VE == 1) v.r = *p;
  else v.r = *reinterpret_cast<const uint4*>(p);
  return v;
}
// the same for data read once: not kept in the L1
template <typename T, int VE> static __device__ __forceinline__ Pack<T, VE> load_once(const T* p) {
  Pack<T, VE> v;
  if constexpr (VE == 1) {
    v.r = *p;
  } else {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.r.x), "=r"(v.r.y), "=r"(v.r.z), "=r"(v.r.w) : "l"(p));
  }
  return v;
}
template <typename T, int VE> static __device__ __forceinline__ void store_pack(T* p, const Pack<T, VE>& v) {
  if constexpr (VE == 1) *p = v.r;
  else *reinterpret_cast<uint4*>(p) = v.r;
}

// Sums of N values over a block of at most 1024 threads, returned to every thread.  The order of the additions is
// fixed by the block's shape.  `buf`: N * 32 floats of shared memory, free again when every thread has returned and
// the block has passed one more barrier.
template <int N> static __device__ __forceinline__ void block_sums(float (&v)[N], float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
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
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

// Sums of N <= P values (P a power of two up to 8) over a block, to every thread, with one barrier: a warp halves the
// number of values it carries while it halves the lanes (P / 2 + P / 4 + ... shuffles instead of 5 P), and a group of
// 32 / P lanes adds one value's partials of the warps.  Fixed order.  `buf`: 32 * P floats, as for block_sums.
template <int N, int P> static __device__ __forceinline__ void block_sums_many(float (&out)[N], float* buf) {
  static_assert(N <= P && P <= 8 && (P & (P - 1)) == 0, "");
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, warps = blockDim.x >> 5;
  float v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = i < N ? out[i] : 0.f;
  int o = 16;
#pragma unroll
  for (int half = P / 2; half >= 1; half /= 2, o /= 2)
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const bool up = (lane & o) != 0;
      const float send = up ? v[i] : v[i + half], keep = up ? v[i + half] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  constexpr int G = 32 / P;  // lanes that now hold the same value
  float s = v[0];
#pragma unroll
  for (int d = G / 2; d >= 1; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
  if (warps > 1) {
    const int which = lane / G, sub = lane % G;
    if (sub == 0) buf[w * P + which] = s;
    __syncthreads();
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32 / G; ++i)
      if (i * G + sub < warps) s += buf[(i * G + sub) * P + which];
#pragma unroll
    for (int d = G / 2; d >= 1; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = __shfl_sync(0xffffffffu, s, i * G);
}

// Exclusive prefix sums of tot[0..n) in place, tot[n] = the total.  All threads of the block; ends with a barrier.
static __device__ void block_exclusive_scan(int* tot, int n, int* warp_sums) {
  const int nt = blockDim.x, per = (n + nt - 1) / nt;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, warps = nt >> 5;
  const int lo = min(n, (int)threadIdx.x * per), hi = min(n, lo + per);
  int s = 0;
  for (int i = lo; i < hi; ++i) s += tot[i];
  int x = s;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  int base = 0, all = 0;
  for (int i = 0; i < warps; ++i) {
    if (i < w) base += warp_sums[i];
    all += warp_sums[i];
  }
  int run = base + x - s;
  for (int i = lo; i < hi; ++i) {
    const int c = tot[i];
    tot[i] = run;
    run += c;
  }
  if (threadIdx.x == 0) tot[n] = all;
  __syncthreads();
}

// ---------------------------------------------------------------- argument checks shared by the entry points

static inline size_t type_bytes(int dtype) { return dtype == DEAMOE_F32 ? 4 : 2; }
static inline bool known_type(int dtype) { return dtype == DEAMOE_F32 || dtype == DEAMOE_BF16; }
static inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// a matrix of `rows` rows whose rows may be read 16 bytes at a time
static inline bool wide_rows(const void* p, int64_t stride, int64_t rows, size_t bytes) {
  return aligned16(p) && (rows <= 1 || (stride * (int64_t)bytes) % 16 == 0);
}

}  // namespace deamoe
