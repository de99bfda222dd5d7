// Few rows: every matrix is read once and the bytes bound it.  A block takes 16 rows of a matrix (DUAL: 8 of gate and the same 8
// of up) and all of a group's rows of x, 8 or 16 at a time; its four or eight warps split the columns and add up in a fixed order.
//
// The products run on mma.sync with the matrix rows as M and the rows of x as N (the tcgen05 kernel would leave most SMs
// without a tile: 4096 rows are 16 tiles of 256).  Its operands come from registers, and since the order of k is free as long as
// both operands agree, a thread's 16 bytes of a row are its operands of two instructions as they lie: columns 8 t .. 8 t + 7
// of a step of 32 (e4m3: 16 t .. of 64) belong to thread t of a row's four, no staging and no shuffles.
// Four steps of loads are in flight a warp.  A kernel launched behind another one of the call loads its first weights before
// it waits for that one's results.  Early launch: one token's block 22.2 -> 20.6 us, 8 x 7168 x 7168 in 8 bits 14.2 -> 13.7.
#include "thin.cuh"

namespace deamoe {

namespace {

constexpr int T_AHEAD = 4; // steps of loads in flight
constexpr int T_SMS = 148;
// The instruction's sums are cut at every step, as the tensor-core kernel's are (matmul.cuh): a warp adds its sums up in fp32 proper after so many turns
// of its loop, 32768 columns (e4m3: 65536).
constexpr int T_STRETCH = 256;

template <bool FP8> __device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (FP8)
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_stream(const char* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// NT: groups of 8 rows of x in a pass; TW: warps of a block.  (One block an SM is all that the bounds ask for: without that the
// compiler keeps to 64 - 93 registers, and fewer loads are in flight: 16 rows of 7168 x 7168 in 30 us, 22 with 112.)
// LONG: a warp has more than a stretch (by itself, for the registers: rows of up to 131072 columns never have).
template <bool FP8, bool DUAL, int NT, int TW, bool LONG> __global__ void __launch_bounds__(TW * 32, 1) k_thin(const __grid_constant__ ThinArgs A, int behind) {
  constexpr int ES = FP8 ? 1 : 2, VE = 16 / ES, STEP = 4 * VE, COLS = 8 * NT, ROWS = DUAL ? 8 : 16;
  __shared__ float part[TW][16][COLS + 1];
  __shared__ int found, counts[TW * 32 + 1], warp_sums[32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
  const int m0 = blockIdx.x * ROWS;
  // Launched early behind whatever is before it in the stream: nothing is read until that has ended.  Behind another kernel of its
  // own call (`behind`), which has waited so, only x has to wait.
  if (!behind) pdl_wait();
  pdl_trigger();
  // the blockIdx.y-th group that has rows
  int e = 0, row0 = 0, row1 = A.n_rows;
  if (A.off) {
    auto at = [&](int i) { return min(max(A.off[i], 0), A.n_rows); };
    const int per = (A.groups + TW * 32 - 1) / (TW * 32), lo = min(A.groups, tid * per), hi = min(A.groups, lo + per);
    int n = 0;
    bool falls = false;
    for (int i = lo; i < hi; ++i) {
      falls |= A.off[i + 1] < A.off[i];
      n += at(i + 1) > at(i);
    }
    counts[tid] = n;
    if (tid == 0) found = -1;
    if (__syncthreads_or(falls)) {
      pdl_wait();
      return;
    }
    block_exclusive_scan(counts, TW * 32, warp_sums);
    int left = (int)blockIdx.y - counts[tid];
    if (left >= 0 && left < n)
      for (int i = lo; i < hi; ++i)
        if (at(i + 1) > at(i) && left-- == 0) found = i;
    __syncthreads();
    e = found;
    if (e < 0) {
      pdl_wait();
      return;
    }
    row0 = at(e);
    row1 = at(e + 1);
  }
  const int64_t row_bytes = (int64_t)A.K * ES;
  // rows past the matrix repeat its last one; what they give is not stored
  const char* w = reinterpret_cast<const char*>(A.w) + (int64_t)e * (DUAL ? 2 : 1) * A.M * row_bytes;
  const char* wa = w + min(m0 + g, A.M - 1) * row_bytes + q * 16;
  const char* wb = w + (DUAL ? A.M + min(m0 + g, A.M - 1) : min(m0 + g + 8, A.M - 1)) * row_bytes + q * 16;
  const int steps = (A.K + STEP - 1) / STEP;

  for (int r0 = row0; r0 < row1; r0 += COLS) {
    const char* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
      x[n] = reinterpret_cast<const char*>(A.x) + (int64_t)min(r0 + n * 8 + g, row1 - 1) * A.xs * ES + q * 16;
    float acc[NT][4] = {}, before[LONG ? NT : 1][4] = {};
    for (int s0 = warp; s0 < steps; s0 += TW * T_AHEAD) {
      if constexpr (LONG)
        if ((s0 - warp) % (TW * T_AHEAD * T_STRETCH) == 0)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              before[n][j] += acc[n][j];
              acc[n][j] = 0.f;
            }
      uint4 a[T_AHEAD], b[T_AHEAD], v[T_AHEAD][NT];
#pragma unroll
      for (int u = 0; u < T_AHEAD; ++u) {
        const int s = s0 + u * TW;
        const bool in = s * STEP + q * VE < A.K;  // (rows are whole 16-byte pieces)
        a[u] = in ? load_stream(wa + (int64_t)s * 64) : make_uint4(0, 0, 0, 0);
        b[u] = in ? load_stream(wb + (int64_t)s * 64) : make_uint4(0, 0, 0, 0);
      }
      if (r0 == row0 && s0 == warp) pdl_wait();  // x may be what the kernel before this one writes
#pragma unroll
      for (int u = 0; u < T_AHEAD; ++u) {
        const int s = s0 + u * TW;
        const bool in = s * STEP + q * VE < A.K;
#pragma unroll
        for (int n = 0; n < NT; ++n) v[u][n] = in ? *reinterpret_cast<const uint4*>(x[n] + (int64_t)s * 64) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < T_AHEAD; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma16<FP8>(acc[n], a[u].x, b[u].x, a[u].y, b[u].y, v[u][n].x, v[u][n].y);
          mma16<FP8>(acc[n], a[u].z, b[u].z, a[u].w, b[u].w, v[u][n].z, v[u][n].w);
        }
    }
    pdl_wait();  // (a warp without a step of columns has not waited yet)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) part[warp][g + 8 * (j >> 1)][n * 8 + 2 * q + (j & 1)] = acc[n][j] + (LONG ? before[LONG ? n : 0][j] : 0.f);
    __syncthreads();
    for (int o = tid; o < ROWS * COLS; o += TW * 32) {
      const int m = o % ROWS, c = o / ROWS;
      if (r0 + c >= row1 || m0 + m >= A.M) continue;
      const int64_t row = r0 + c;
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < TW; ++i) v += part[i][m][c];
      if constexpr (DUAL) {
        float up = 0.f;
#pragma unroll
        for (int i = 0; i < TW; ++i) up += part[i][m + 8][c];
        v = silu_f(v) * up;
      } else {
        if constexpr (FP8) v *= A.x_scale[row] * A.w_scale[m0 + m];
        if (A.bias)
          v += A.bias_f32 ? reinterpret_cast<const float*>(A.bias)[m0 + m] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(A.bias)[m0 + m]);
        v = sigma_f(A.act, v);
        if (A.residual) v += __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(A.residual)[row * A.rs + m0 + m]);
      }
      A.out[row * A.os + m0 + m] = __float2bfloat16_rn(v);
    }
    __syncthreads();
  }
}

template <bool FP8, bool DUAL> cudaError_t launch(const ThinArgs& a, cudaStream_t s, bool chained) {
  const int rows = DUAL ? 8 : 16;
  const dim3 grid((a.M + rows - 1) / rows, a.off ? (a.groups < a.n_rows ? a.groups : a.n_rows) : 1);
  // With three blocks an SM and more, blocks of four warps are all resident at once (7168 x 7168: 448 blocks, where 444 of eight
  // warps fit; one row 20.8 us, 21.2 - 25.4 with eight; 16 rows over 13 of 32 experts 201 us, 239); with fewer, eight keep
  // more loads in flight (4096 x 4096: 9.0 us, 11.7 with four).
  const bool many = (int64_t)grid.x * grid.y >= 3 * T_SMS;
  const int threads = many ? 128 : 256;
  constexpr int TURN = (FP8 ? 64 : 32) * T_AHEAD;  // columns of a warp's turn
  const bool wide = (a.K - 1) / (TURN * T_STRETCH) >= threads / 32;
  auto kernel = a.n_rows <= 8 ? (many ? k_thin<FP8, DUAL, 1, 4, false> : k_thin<FP8, DUAL, 1, 8, false>)
                              : (many ? k_thin<FP8, DUAL, 2, 4, false> : k_thin<FP8, DUAL, 2, 8, false>);
  if (wide)
    kernel = a.n_rows <= 8 ? (many ? k_thin<FP8, DUAL, 1, 4, true> : k_thin<FP8, DUAL, 1, 8, true>)
                           : (many ? k_thin<FP8, DUAL, 2, 4, true> : k_thin<FP8, DUAL, 2, 8, true>);
  return launch_pdl(kernel, grid, dim3(threads), 0, s, a, (int)chained);
}

}  // namespace

cudaError_t thin_launch(bool e4m3, bool dual, const ThinArgs& a, cudaStream_t s, bool chained) {
  if (e4m3) return launch<true, false>(a, s, chained);
  return dual ? launch<false, true>(a, s, chained) : launch<false, false>(a, s, chained);
}

}  // namespace deamoe
