// Products with 4-bit matrices of group scales: out[r] = W[e(r)] x[src(r)], optionally through SwiGLU.
//
//   W[i, c] = s[i, c / G] (q[i, c] - z[i, c / G])   =>   (W x)[i] = sum_g s[i, g] sum_{c in g} (q - z) x[c]
//
// so the group scale multiplies an fp32 sum and no weight is ever rounded.  A decode step has a few rows per matrix:
// the codes (half a byte a weight, read once) bound it, and the work beside them is to widen 2 weights a byte.
//
// Tensor cores: mma.m16n8k16 with 16 matrix rows as M and up to 8 tokens as N (legacy path: with this few tokens the
// instruction rate it needs is a fraction of what it has, and its A operand comes from registers, where the codes
// have to be widened anyway).  q - z is a whole number of at most 15, exact in any 16-bit type; fp16 is used because
// its 10 mantissa bits let two nibbles of a 16-bit half be widened in place (1024 + q and 1024 + 16 q), one shift
// less per pair than bf16's 7 bits.  x therefore becomes fp16 as well, in a kernel of its own: each row scaled by a
// power of two to a largest magnitude of 2^14..2^15, so that fp16's range costs nothing (values below 2^-39 of the
// row's largest lose bits, far under fp32's own resolution of the sum); bf16 values fit exactly, fp32 values as two
// parts (2^-23 relative).
#include <atomic>
#include <climits>
#include <cuda_fp16.h>

#include "row.cuh"

namespace deamoe {

constexpr int QW = 8;        // warps of a block
constexpr int QCOLS = 128;   // columns of a step: 64 bytes of a row
constexpr int Q_GRID = 296;  // two blocks on each of the 148 SMs

struct QuantArgs {
  const uint8_t* codes;
  const void* scales;
  const uint8_t* zeros;
  const void* x;
  int64_t xs;
  const int32_t *expert_off, *row_pair;
  void* out;
  int64_t os;
  int n_expert, n_out, n_in, groups, n_token, ppt, n_rows, swiglu, scale_f32;
  int steps;        // column steps of a row
  int wk;           // warps that share a row tile's columns (the others of the block take other tiles)
  int tile_groups;  // blocks of QW / wk row tiles a matrix
  __half* xh;       // [n_rows][planes][steps * QCOLS]
  int32_t* xe;      // [n_rows] exponent the row was scaled by
};

static __device__ __forceinline__ float quant_scale(const QuantArgs& A, size_t i) {
  return A.scale_f32 ? reinterpret_cast<const float*>(A.scales)[i]
                     : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(A.scales)[i]);
}

// x in the order of the rows, as fp16 scaled by 2^-exponent, 8 columns in the order 0 4 1 5 2 6 3 7 (the order in
// which the codes of a 32-bit word are widened).  One block a row; a row without a source is zero.
template <typename T, int PLANES> __global__ void __launch_bounds__(256) k_quant_x(QuantArgs A) {
  __shared__ float buf[32];
  const int64_t r = blockIdx.x;
  int64_t src = r;
  if (A.row_pair) src = A.row_pair[r] >= 0 ? A.row_pair[r] / A.ppt : -1;
  const bool have = src >= 0 && src < A.n_token;
  const T* x = reinterpret_cast<const T*>(A.x) + (have ? src : 0) * A.xs;
  pdl_trigger();
  float top = 0.f;
  for (int c = threadIdx.x; have && c < A.n_in; c += 256) {
    const float v = fabsf(to_f<T>(x[c]));
    if (v <= 3.4028234663852886e38f) top = fmaxf(top, v);  // infinities and NaN stay what they are
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = top;
  __syncthreads();
  for (int i = 0; i < 8; ++i) top = fmaxf(top, buf[i]);
  const int e = top > 0.f ? ilogbf(top) - 14 : 0;
  if (threadIdx.x == 0) A.xe[r] = e;
  const int width = A.steps * QCOLS;
  __half* out = A.xh + r * PLANES * width;
  for (int c = threadIdx.x; c < width / 8; c += 256) {
    union { __half h[8]; uint4 u; } hi, lo;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int col = c * 8 + (p >> 1) + (p & 1) * 4;
      const float v = have && col < A.n_in ? scalbnf(to_f<T>(x[col]), -e) : 0.f;
      hi.h[p] = __float2half_rn(v);
      const float rest = v - __half2float(hi.h[p]);
      lo.h[p] = __float2half_rn(isfinite(v) ? rest : 0.f);
    }
    *reinterpret_cast<uint4*>(out + c * 8) = hi.u;
    if constexpr (PLANES == 2) *reinterpret_cast<uint4*>(out + width + c * 8) = lo.u;
  }
}

static __device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
static __device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
static __device__ __forceinline__ __half2 bits_half2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
static __device__ __forceinline__ uint32_t pick(uint32_t w, uint32_t mask) { return (w & mask) | 0x64006400u; }  // one LOP3

// The 8 codes of a word minus the zero point, as four half pairs: columns (0 4) (1 5) (2 6) (3 7).
// low = 1024 + z, high = -(64 + z): 1024 + q - (1024 + z) and (1024 + 16 q) / 16 - (64 + z), both exact.
static __device__ __forceinline__ void widen(uint32_t w, __half2 low, __half2 high, uint32_t (&p)[4]) {
  const __half2 sixteenth = __float2half2_rn(0.0625f);
  const uint32_t v = w >> 8;
  p[0] = half2_bits(__hsub2(bits_half2(pick(w, 0x000f000fu)), low));
  p[1] = half2_bits(__hfma2(bits_half2(pick(w, 0x00f000f0u)), sixteenth, high));
  p[2] = half2_bits(__hsub2(bits_half2(pick(v, 0x000f000fu)), low));
  p[3] = half2_bits(__hfma2(bits_half2(pick(v, 0x00f000f0u)), sixteenth, high));
}

// A block takes a contiguous share of the items (expert, group of row tiles, pass of 8 NT rows); its warps split an
// item's columns (wk of them a tile).  Every warp streams its own codes, `DEPTH` steps of 16 rows x 128 columns ahead
// and across items, into its own part of shared memory; nothing is shared between warps but the sums at an item's end.
template <typename T, int PLANES, int NT, int NG, int DEPTH>
__global__ void __launch_bounds__(QW * 32, 2) k_quant(QuantArgs A) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int warp_sums[QW];
  uint8_t* ring = smem + (threadIdx.x >> 5) * (DEPTH * 1024);
  float4* sums = reinterpret_cast<float4*>(smem + QW * DEPTH * 1024);     // [2][QW][NT][32]
  int* first = reinterpret_cast<int*>(sums + 2 * QW * NT * 32);           // [n_expert + 1] first item of each expert
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int g = lane >> 2, j = lane & 3;
  const int R = A.n_rows;
  auto row_begin = [&](int e) { return A.expert_off ? min(max(A.expert_off[e], 0), R) : 0; };
  auto row_end = [&](int e) { return A.expert_off ? min(max(A.expert_off[e + 1], 0), R) : R; };
  for (int e = threadIdx.x; e < A.n_expert; e += QW * 32) {
    const int rows = max(row_end(e) - row_begin(e), 0);
    first[e] = (rows + 8 * NT - 1) / (8 * NT) * A.tile_groups;
  }
  __syncthreads();
  block_exclusive_scan(first, A.n_expert, warp_sums);
  const int total = first[A.n_expert];
  const int i0 = (int)((int64_t)total * blockIdx.x / gridDim.x), i1 = (int)((int64_t)total * (blockIdx.x + 1) / gridDim.x);
  const int wr = w / A.wk, wkk = w - wr * A.wk, tiles_per = QW / A.wk;
  const int c0 = A.steps * wkk / A.wk, c1 = A.steps * (wkk + 1) / A.wk;
  const int width = A.swiglu ? A.n_out / 2 : A.n_out;
  const int tile_rows = A.swiglu ? 8 : 16;  // output columns of a tile

  int e_start = 0;
  {
    int lo = 0, hi = A.n_expert;  // the last e with first[e] <= i0
    while (hi - lo > 1) {
      const int m = (lo + hi) / 2;
      if (first[m] <= i0) lo = m; else hi = m;
    }
    e_start = lo;
  }
  auto tile_of = [&](int item, int e, int& pass) {
    const int local = item - first[e], passes = (first[e + 1] - first[e]) / A.tile_groups;
    const int tg = passes == 1 ? local : local / passes;
    pass = local - tg * passes;
    return tg * tiles_per + wr;
  };
  // matrix row of tile row r, or -1
  auto matrix_row = [&](int tile, int r) {
    if (A.swiglu) {
      const int i = tile * 8 + (r & 7);
      return i < width ? (r < 8 ? i : width + i) : -1;
    }
    const int i = tile * 16 + r;
    return i < width ? i : -1;
  };

  // -- the codes' cursor
  int p_item = i0, p_e = e_start, p_c = c0, p_slot = 0;
  const uint8_t *p_lo = nullptr, *p_hi = nullptr;  // this lane's 16-byte piece of rows g and g + 8, or null
  auto p_enter = [&]() {
    if (p_item >= i1 || c0 == c1) return;
    while (p_item >= first[p_e + 1]) ++p_e;
    int pass;
    const int tile = tile_of(p_item, p_e, pass);
    const int lo = matrix_row(tile, g), hi = matrix_row(tile, g + 8);
    const size_t base = (size_t)p_e * A.n_out, half = A.n_in / 2;
    p_lo = lo >= 0 ? A.codes + (base + lo) * half + j * 16 : nullptr;
    p_hi = hi >= 0 ? A.codes + (base + hi) * half + j * 16 : nullptr;
  };
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  const uint32_t put_at = ring_at + g * 64 + ((j ^ ((g >> 1) & 3)) * 16);
  auto p_request = [&]() {
    if (p_item < i1 && c0 < c1) {
      const bool in = p_c * QCOLS + j * 32 < A.n_in;
      const uint32_t to = put_at + p_slot * 1024;
      const uint8_t* lo = in && p_lo ? p_lo + (size_t)p_c * 64 : A.codes;
      const uint8_t* hi = in && p_hi ? p_hi + (size_t)p_c * 64 : A.codes;
      const int nlo = in && p_lo ? 16 : 0, nhi = in && p_hi ? 16 : 0;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(lo), "r"(nlo) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + 512), "l"(hi), "r"(nhi) : "memory");
      if (++p_c == c1) {
        p_c = c0;
        ++p_item;
        p_enter();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    p_slot = p_slot + 1 == DEPTH ? 0 : p_slot + 1;
  };
  p_enter();
#pragma unroll 1
  for (int i = 0; i < DEPTH; ++i) p_request();
  pdl_wait();  // x in fp16

  // -- the items
  const uint32_t get_at = ring_at + (lane & 7) * 64 + (((lane >> 3) ^ (((lane & 7) >> 1) & 3)) * 16);
  const int xw = A.steps * QCOLS;
  int slot = 0, flip = 0, e = e_start;
  for (int item = i0; item < i1; ++item, flip ^= 1) {
    while (item >= first[e + 1]) ++e;
    int pass;
    const int tile = tile_of(item, e, pass);
    const int r_lo = max(matrix_row(tile, g), 0), r_hi = max(matrix_row(tile, g + 8), 0);
    const size_t s_lo = ((size_t)e * A.n_out + r_lo) * A.groups, s_hi = ((size_t)e * A.n_out + r_hi) * A.groups;
    const int row0 = row_begin(e) + pass * 8 * NT, rows = min(row_end(e) - row0, 8 * NT);
    const __half* xp = A.xh + (size_t)(row0 + g) * PLANES * xw + j * 8;
    float acc[NT][4] = {};
    for (int c = c0; c < c1; ++c) {
      // scales and zero points of the step's groups (the last step may have fewer)
      float sl[NG], sh[NG];
      int zl[NG], zh[NG];
#pragma unroll
      for (int k = 0; k < NG; ++k) {
        const int grp = c * NG + k;
        const bool in = grp < A.groups;
        sl[k] = in ? quant_scale(A, s_lo + grp) : 0.f;
        sh[k] = in ? quant_scale(A, s_hi + grp) : 0.f;
        zl[k] = in && A.zeros ? A.zeros[s_lo + grp] & 15 : 8;
        zh[k] = in && A.zeros ? A.zeros[s_hi + grp] & 15 : 8;
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
      __syncwarp();
      uint32_t lo[4], hi[4];
      const uint32_t from = get_at + slot * 1024;
      asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                   : "=r"(lo[0]), "=r"(lo[1]), "=r"(lo[2]), "=r"(lo[3]) : "r"(from) : "memory");
      asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                   : "=r"(hi[0]), "=r"(hi[1]), "=r"(hi[2]), "=r"(hi[3]) : "r"(from + 512) : "memory");
      __syncwarp();
      p_request();  // the slot just read
      slot = slot + 1 == DEPTH ? 0 : slot + 1;
      float grp[NT][4] = {};
      const __half* xc = xp + (size_t)c * QCOLS;
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int k = m * NG / 4;
        uint32_t pl[4], ph[4];
        widen(lo[m], __half2half2(__ushort_as_half(0x6400 | zl[k])), __half2half2(__ushort_as_half(0xd400 | zl[k] << 4)), pl);
        widen(hi[m], __half2half2(__ushort_as_half(0x6400 | zh[k])), __half2half2(__ushort_as_half(0xd400 | zh[k] << 4)), ph);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (NT > 1 && t * 8 >= rows) break;
#pragma unroll
          for (int p = 0; p < PLANES; ++p) {
            uint4 b = make_uint4(0, 0, 0, 0);
            if (t * 8 + g < rows)
              b = *reinterpret_cast<const uint4*>(xc + (size_t)(t * 8 * PLANES + p) * xw + m * 32);
            mma_f16(grp[t], pl[0], ph[0], pl[1], ph[1], b.x, b.y);
            mma_f16(grp[t], pl[2], ph[2], pl[3], ph[3], b.z, b.w);
          }
        }
        if ((m + 1) * NG % 4 == 0 && c * NG + k < A.groups) {  // a group ends
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            acc[t][0] = fmaf(sl[k], grp[t][0], acc[t][0]);
            acc[t][1] = fmaf(sl[k], grp[t][1], acc[t][1]);
            acc[t][2] = fmaf(sh[k], grp[t][2], acc[t][2]);
            acc[t][3] = fmaf(sh[k], grp[t][3], acc[t][3]);
            grp[t][0] = grp[t][1] = grp[t][2] = grp[t][3] = 0.f;
          }
        }
      }
    }
    // join the warps' column shares, in order; the other buffer is still being read by slower warps
    float4* mine = sums + ((size_t)flip * QW + w) * NT * 32 + lane;
#pragma unroll
    for (int t = 0; t < NT; ++t) mine[t * 32] = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
    __syncthreads();
    // a thread: one token, one tile row g and its partner g + 8
    for (int i = threadIdx.x; i < tiles_per * NT * 64; i += QW * 32) {
      const int h = i & 1, l = (i >> 1) & 31, t = (i >> 6) % NT, tr = (i >> 6) / NT;
      const int token = t * 8 + (l & 3) * 2 + h;
      if (token >= rows) continue;
      float a = 0.f, b = 0.f;
      for (int k = 0; k < A.wk; ++k) {
        const float* v = reinterpret_cast<const float*>(sums + ((size_t)flip * QW + tr * A.wk + k) * NT * 32 + t * 32 + l);
        a += v[h];
        b += v[h + 2];
      }
      const int64_t r = row0 + token;
      const int ex = A.xe[r];
      a = scalbnf(a, ex);
      b = scalbnf(b, ex);
      T* out = reinterpret_cast<T*>(A.out) + r * A.os;
      const int i_tile = (tile - wr + tr) * tile_rows + (l >> 2);
      if (A.swiglu) {
        if (i_tile < width) out[i_tile] = from_f<T>(a / (1.f + expf(-a)) * b);
      } else {
        if (i_tile < width) out[i_tile] = from_f<T>(a);
        if (i_tile + 8 < width) out[i_tile + 8] = from_f<T>(b);
      }
    }
  }
}

template <typename T, int NG> static deamoe_status_t quant_t(const QuantArgs& A, cudaStream_t s) {
  constexpr int PLANES = sizeof(T) == 4 ? 2 : 1;
  auto run = [&](auto kernel, int nt, int depth, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!(done.load(std::memory_order_acquire) >> dev & 1)) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 112 * 1024);
      if (e != cudaSuccess) return e;
      done.fetch_or(1ull << dev, std::memory_order_release);
    }
    const size_t smem = (size_t)QW * depth * 1024 + 2 * QW * nt * 512 + (size_t)(A.n_expert + 1) * 4;
    k_quant_x<T, PLANES><<<A.n_rows, 256, 0, s>>>(A);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_pdl(kernel, dim3(Q_GRID), dim3(QW * 32), smem, s, A);
  };
  static std::atomic<uint64_t> done[2];
  const cudaError_t e = A.n_rows <= 8 ? run(k_quant<T, PLANES, 1, NG, 10>, 1, 10, done[0])
                                      : run(k_quant<T, PLANES, 4, NG, 8>, 4, 8, done[1]);
  if (e == cudaSuccess) return DEAMOE_OK;
  cudaGetLastError();
  return DEAMOE_ERR_CUDA;
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_quant_workspace(int32_t dtype, int32_t n_rows, int32_t n_in) {
  if (n_rows <= 0 || n_in <= 0) return 0;
  const uint64_t width = ((uint64_t)n_in + QCOLS - 1) / QCOLS * QCOLS;
  return (uint64_t)n_rows * (width * (dtype == DEAMOE_F32 ? 4 : 2) + sizeof(int32_t));
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
  const uint64_t need = deamoe_quant_workspace(dtype, n_rows, n_in);
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return DEAMOE_ERR_INVALID_ARG;
  QuantArgs A;
  A.codes = codes; A.scales = scales; A.zeros = zeros; A.x = x; A.xs = x_stride; A.expert_off = expert_off;
  A.row_pair = row_pair; A.out = out; A.os = out_stride; A.n_expert = n_expert; A.n_out = n_out; A.n_in = n_in;
  A.groups = (n_in + group - 1) / group; A.n_token = n_token; A.ppt = pairs_per_token; A.n_rows = n_rows;
  A.swiglu = swiglu; A.scale_f32 = scale_dtype == DEAMOE_F32;
  A.steps = (n_in + QCOLS - 1) / QCOLS;
  A.wk = QW;
  while (A.wk > A.steps) A.wk /= 2;
  const int tiles = swiglu ? (width + 7) / 8 : (width + 15) / 16;
  A.tile_groups = (tiles + QW / A.wk - 1) / (QW / A.wk);
  // items are counted in 32 bits (an expert's last pass may be short, hence one more each)
  if ((int64_t)A.tile_groups * ((int64_t)n_rows / 8 + n_expert) > INT_MAX) return DEAMOE_ERR_BATCH;
  A.xh = reinterpret_cast<__half*>(workspace);
  A.xe = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(workspace) +
                                    (size_t)n_rows * A.steps * QCOLS * (dtype == DEAMOE_F32 ? 4 : 2));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (dtype == DEAMOE_F32)
    return group == 128 ? quant_t<float, 1>(A, s) : group == 64 ? quant_t<float, 2>(A, s) : quant_t<float, 4>(A, s);
  return group == 128 ? quant_t<__nv_bfloat16, 1>(A, s)
                      : group == 64 ? quant_t<__nv_bfloat16, 2>(A, s) : quant_t<__nv_bfloat16, 4>(A, s);
}

}  // extern "C"
