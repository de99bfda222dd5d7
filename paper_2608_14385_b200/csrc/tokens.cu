// Tokens sorted by expert and back: the (token, slot) pairs of a routing decision in expert order, rows of tokens
// copied into that order, rows summed back with the gate weights of Eq. (3), and the gradients of both.
//
// Everything is a permutation plus at most one multiply-add per value, so HBM bounds it (launch latency for a few
// tokens).  Both directions go token by token: a token's row is read or written once and its k expert rows once each,
// whatever order the experts put them in, so the traffic is the least there is (T h + P h values) and does not lean
// on the caches.  No atomics: sums over a token's rows are taken in slot order, and equal calls give equal bits.
#include <climits>

#include "row.cuh"

namespace deamoe {

// ---------------------------------------------------------------- sorting

// Pairs go to warps in contiguous stretches; a warp ranks 32 pairs at a time among the lanes that hold the same
// expert (match_any) and counts on in its own column of counters, so the order within an expert is the pair order
// (a stable sort) without any atomics.
// Up to here one block sorts everything: 4.4 us for 512 pairs of 256 experts where the three kernels take 6.2, but 7.7 us
// for 2048 and 11.4 for 4096 where they take 7.3.
constexpr int SORT_SMALL_PAIRS = 1536;
constexpr int SORT_COUNTERS = 16384;  // 16-bit counters of one block (warps x experts)
constexpr int SORT_SMALL_ITERS = SORT_SMALL_PAIRS / 32 / (SORT_COUNTERS / DEAMOE_MAX_EXPERTS);
constexpr int SORT_SEG = 1024;             // pairs of one block in the three-kernel form
constexpr int SORT_SEG_WARPS = 8;          // (8 warps x 2048 experts fit the counters)
constexpr int SORT_SEG_ITERS = SORT_SEG / 32 / SORT_SEG_WARPS;

static __device__ __forceinline__ int sort_key(const int32_t* idx, int p, int end, int n) {
  if (p >= end) return n;
  const int e = idx[p];
  return (unsigned)e < (unsigned)n ? e : n;  // out of range: dropped
}

// Rank of the lane's pair among the warp's earlier pairs of expert e; advances the warp's counters.
static __device__ __forceinline__ int warp_rank(unsigned short* cnt, int e, int n) {
  const int lane = threadIdx.x & 31;
  const unsigned peers = __match_any_sync(0xffffffffu, e);
  const int before = __popc(peers & ((1u << lane) - 1u));
  int old = 0;
  if (e < n) old = cnt[e];
  __syncwarp();
  if (e < n && before == 0) cnt[e] = (unsigned short)(old + __popc(peers));
  __syncwarp();
  return old + before;
}

__global__ void __launch_bounds__(1024) k_sort_small(const int32_t* __restrict__ idx, int P, int n, int warps,
                                                     int32_t* __restrict__ expert_off, int32_t* __restrict__ pair_row,
                                                     int32_t* __restrict__ row_pair) {
  __shared__ unsigned short cnt[SORT_COUNTERS];
  __shared__ int tot[DEAMOE_MAX_EXPERTS + 1];
  __shared__ int warp_sums[32];
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < warps * n; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  const int seg = ((P + warps * 32 - 1) / (warps * 32)) * 32;
  const int begin = w * seg, end = min(P, begin + seg);
  int key[SORT_SMALL_ITERS], rank[SORT_SMALL_ITERS];
  if (w < warps) {
#pragma unroll
    for (int i = 0; i < SORT_SMALL_ITERS; ++i) {
      if (i * 32 >= seg) break;
      key[i] = sort_key(idx, begin + i * 32 + lane, end, n);
    }
#pragma unroll
    for (int i = 0; i < SORT_SMALL_ITERS; ++i) {
      if (i * 32 >= seg) break;
      rank[i] = warp_rank(cnt + w * n, key[i], n);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += blockDim.x) {  // counters -> first rank of each warp; totals
    int run = 0;
    for (int j = 0; j < warps; ++j) {
      const int c = cnt[j * n + e];
      cnt[j * n + e] = (unsigned short)run;
      run += c;
    }
    tot[e] = run;
  }
  __syncthreads();
  block_exclusive_scan(tot, n, warp_sums);
  for (int e = threadIdx.x; e <= n; e += blockDim.x) expert_off[e] = tot[e];
  for (int r = tot[n] + threadIdx.x; r < P; r += blockDim.x) row_pair[r] = -1;
  if (w < warps) {
#pragma unroll
    for (int i = 0; i < SORT_SMALL_ITERS; ++i) {
      if (i * 32 >= seg) break;
      const int p = begin + i * 32 + lane;
      if (p >= end) continue;
      int row = -1;
      if (key[i] < n) {
        row = tot[key[i]] + cnt[w * n + key[i]] + rank[i];
        row_pair[row] = p;
      }
      pair_row[p] = row;
    }
  }
}

// Three kernels for more pairs (32768 pairs of 256 experts: 8.1 us, all of it latency; the lists are 0.4 MB).
// 1: every block ranks its stretch and counts its experts.
__global__ void __launch_bounds__(SORT_SEG_WARPS * 32) k_sort_count(const int32_t* __restrict__ idx, int P, int n,
                                                                   int32_t* __restrict__ hist,
                                                                   unsigned short* __restrict__ rank_out) {
  __shared__ unsigned short cnt[SORT_COUNTERS];
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < SORT_SEG_WARPS * n; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  const int64_t begin = (int64_t)blockIdx.x * SORT_SEG + w * (SORT_SEG / SORT_SEG_WARPS);
  int key[SORT_SEG_ITERS], rank[SORT_SEG_ITERS];
#pragma unroll
  for (int i = 0; i < SORT_SEG_ITERS; ++i) {
    const int64_t p = begin + i * 32 + lane;
    key[i] = p < P ? sort_key(idx, (int)p, P, n) : n;
  }
#pragma unroll
  for (int i = 0; i < SORT_SEG_ITERS; ++i) rank[i] = warp_rank(cnt + w * n, key[i], n);
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += blockDim.x) {
    int run = 0;
    for (int j = 0; j < SORT_SEG_WARPS; ++j) {
      const int c = cnt[j * n + e];
      cnt[j * n + e] = (unsigned short)run;
      run += c;
    }
    hist[(size_t)blockIdx.x * n + e] = run;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SORT_SEG_ITERS; ++i) {
    const int64_t p = begin + i * 32 + lane;
    if (p < P && key[i] < n) rank_out[p] = (unsigned short)(cnt[w * n + key[i]] + rank[i]);
  }
}

// 2: for 32 experts a block, the counts of all stretches become first ranks (exclusive sums over the stretches).
__global__ void __launch_bounds__(1024) k_sort_scan(int32_t* __restrict__ hist, int G, int n, int32_t* __restrict__ total) {
  __shared__ int part[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int e = blockIdx.x * 32 + lane;
  const int per = (G + 31) / 32, lo = min(G, w * per), hi = min(G, lo + per);
  int s = 0;
  if (e < n)
    for (int g = lo; g < hi; ++g) s += hist[(size_t)g * n + e];
  part[w][lane] = s;
  __syncthreads();
  int run = 0, all = 0;
  for (int i = 0; i < 32; ++i) {
    if (i < w) run += part[i][lane];
    all += part[i][lane];
  }
  if (e >= n) return;
  for (int g = lo; g < hi; ++g) {
    const int c = hist[(size_t)g * n + e];
    hist[(size_t)g * n + e] = run;
    run += c;
  }
  if (w == 0) total[e] = all;
}

// 3: first row of every expert (each block for itself), then every pair to its place.
__global__ void __launch_bounds__(SORT_SEG_WARPS * 32) k_sort_place(const int32_t* __restrict__ idx, int P, int n,
                                                                   const int32_t* __restrict__ hist,
                                                                   const int32_t* __restrict__ total,
                                                                   const unsigned short* __restrict__ rank,
                                                                   int32_t* __restrict__ expert_off,
                                                                   int32_t* __restrict__ pair_row,
                                                                   int32_t* __restrict__ row_pair) {
  __shared__ int tot[DEAMOE_MAX_EXPERTS + 1];
  __shared__ int warp_sums[32];
  constexpr int THREADS = SORT_SEG_WARPS * 32, PER = SORT_SEG / THREADS;
  const int64_t begin = (int64_t)blockIdx.x * SORT_SEG + threadIdx.x;
  int e[PER], base[PER], rk[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) e[i] = begin + i * THREADS < P ? sort_key(idx, (int)(begin + i * THREADS), P, n) : n;
  pdl_wait();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    base[i] = e[i] < n ? hist[(size_t)blockIdx.x * n + e[i]] : 0;
    rk[i] = e[i] < n ? rank[begin + i * THREADS] : 0;
  }
  for (int k = threadIdx.x; k < n; k += THREADS) tot[k] = total[k];
  __syncthreads();
  block_exclusive_scan(tot, n, warp_sums);
  if (blockIdx.x == 0)
    for (int k = threadIdx.x; k <= n; k += THREADS) expert_off[k] = tot[k];
  const int filled = tot[n];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int64_t p = begin + i * THREADS;
    if (p >= P) break;
    int row = -1;
    if (e[i] < n) {
      row = tot[e[i]] + base[i] + rk[i];
      row_pair[row] = (int)p;
    }
    pair_row[p] = row;
    if (p >= filled) row_pair[p] = -1;
  }
}

static size_t sort_hist_bytes(int64_t P, int n) { return (size_t)((P + SORT_SEG - 1) / SORT_SEG) * n * sizeof(int32_t); }

// ---------------------------------------------------------------- moving rows

// Measured (4096 tokens, top-8, 7168 bf16 values a row): dispatch 85 us, combine 85 us, dispatch_backward 83 us
// (6.2 - 6.4 TB/s on 0.53 GB), combine_backward 168 us (5.9 TB/s on 1.0 GB): HBM bounds all four.  16 tokens: 2 us
// each, launch latency.
//
// A block covers `by` tokens with `bx` threads each (bx * by = 256), a thread one pack of columns; rows wider than
// bx packs take several blocks in y.
struct RowGrid { dim3 grid, block; };
static RowGrid row_grid(int64_t tokens, int64_t packs) {
  int bx = 8;
  while (bx < 256 && bx < packs) bx *= 2;
  const int by = 256 / bx;
  return {dim3((unsigned)((tokens + by - 1) / by), (unsigned)((packs + bx - 1) / bx)), dim3(bx, by)};
}

template <typename T, int VE>
__global__ void __launch_bounds__(256) k_dispatch(const T* __restrict__ x, int64_t xs, const int32_t* __restrict__ pair_row,
                                                  int64_t tokens, int k, int packs, T* __restrict__ rows, int64_t rs,
                                                  unsigned n_rows) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int c = blockIdx.y * blockDim.x + threadIdx.x;
  if (t >= tokens || c >= packs) return;
  const Pack<T, VE> v = load_once<T, VE>(x + t * xs + (int64_t)c * VE);
  const int32_t* pr = pair_row + t * k;
  for (int q = 0; q < k; ++q) {
    const unsigned r = (unsigned)pr[q];  // -1 (dropped) is beyond every n_rows
    if (r < n_rows) store_pack<T, VE>(rows + r * rs + (int64_t)c * VE, v);
  }
}

// out[t] = sum_q w[t, q] rows[pair_row[t, q]] in slot order, fp32, rounded once; w == nullptr: every weight 1 (the
// gradient of k_dispatch).
template <typename T, int VE, bool W>
__global__ void __launch_bounds__(256) k_collect(const T* __restrict__ rows, int64_t rs, unsigned n_rows,
                                                 const int32_t* __restrict__ pair_row, const float* __restrict__ w,
                                                 int64_t tokens, int k, int packs, T* __restrict__ out, int64_t os) {
  constexpr int Q = 8;  // rows in flight
  const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int c = blockIdx.y * blockDim.x + threadIdx.x;
  if (t >= tokens || c >= packs) return;
  const int32_t* pr = pair_row + t * k;
  float acc[VE] = {};
  for (int q0 = 0; q0 < k; q0 += Q) {
    Pack<T, VE> v[Q];
    unsigned r[Q];
    float g[Q];
#pragma unroll
    for (int j = 0; j < Q; ++j) {
      r[j] = q0 + j < k ? (unsigned)pr[q0 + j] : 0xffffffffu;
      if constexpr (W) g[j] = q0 + j < k ? w[t * k + q0 + j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < Q; ++j)
      if (r[j] < n_rows) v[j] = load_once<T, VE>(rows + r[j] * rs + (int64_t)c * VE);
#pragma unroll
    for (int j = 0; j < Q; ++j)
      if (r[j] < n_rows) {
        float f[VE];
        v[j].widen(f);
#pragma unroll
        for (int i = 0; i < VE; ++i) acc[i] = W ? fmaf(g[j], f[i], acc[i]) : acc[i] + f[i];
      }
  }
  Pack<T, VE> o;
  o.narrow(acc);
  store_pack<T, VE>(out + t * os + (int64_t)c * VE, o);
}

// drows[r] = w dout[t] and dw = <dout[t], rows[r]> for every pair's row r: one pass over dout and rows.  `bx` threads
// (whole warps) walk a token's columns, eight rows at a time; the dot products are summed over the warp, then over
// the token's warps in order.
template <typename T, int VE>
__global__ void __launch_bounds__(256) k_collect_grad(const T* __restrict__ dout, int64_t ds, const T* __restrict__ rows,
                                                      int64_t rs, unsigned n_rows, const int32_t* __restrict__ pair_row,
                                                      const float* __restrict__ w, int64_t tokens, int k, int packs,
                                                      T* __restrict__ drows, int64_t drs, float* __restrict__ dw) {
  constexpr int Q = 8;
  __shared__ float part[8][Q];  // per warp of the block
  const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const bool live = t < tokens;
  const int lane = threadIdx.x & 31, wpt = blockDim.x >> 5, wx = threadIdx.x >> 5;
  for (int q0 = 0; q0 < k; q0 += Q) {
    unsigned r[Q];
    float g[Q], acc[Q];
#pragma unroll
    for (int j = 0; j < Q; ++j) {
      const bool in = live && q0 + j < k;
      r[j] = in ? (unsigned)pair_row[t * k + q0 + j] : 0xffffffffu;
      g[j] = in ? w[t * k + q0 + j] : 0.f;
      acc[j] = 0.f;
    }
    if (live)
      for (int c = threadIdx.x; c < packs; c += blockDim.x) {
        float d[VE];
        load_pack<T, VE>(dout + t * ds + (int64_t)c * VE).widen(d);
        Pack<T, VE> v[Q];
        if (dw) {
#pragma unroll
          for (int j = 0; j < Q; ++j)
            if (r[j] < n_rows) v[j] = load_once<T, VE>(rows + r[j] * rs + (int64_t)c * VE);
        }
        if (drows) {
#pragma unroll
          for (int j = 0; j < Q; ++j)
            if (r[j] < n_rows) {
              float f[VE];
#pragma unroll
              for (int i = 0; i < VE; ++i) f[i] = g[j] * d[i];
              Pack<T, VE> o;
              o.narrow(f);
              store_pack<T, VE>(drows + r[j] * drs + (int64_t)c * VE, o);
            }
        }
        if (dw) {
#pragma unroll
          for (int j = 0; j < Q; ++j)
            if (r[j] < n_rows) {
              float f[VE];
              v[j].widen(f);
#pragma unroll
              for (int i = 0; i < VE; ++i) acc[j] = fmaf(d[i], f[i], acc[j]);
            }
        }
      }
    if (!dw) continue;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int j = 0; j < Q; ++j) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
    __syncthreads();  // the previous eight have been read
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < Q; ++j) part[threadIdx.y * wpt + wx][j] = acc[j];
    __syncthreads();
    if (live && threadIdx.x < Q && q0 + (int)threadIdx.x < k) {
      float s = 0.f;
      for (int i = 0; i < wpt; ++i) s += part[threadIdx.y * wpt + i][threadIdx.x];
      dw[t * k + q0 + threadIdx.x] = s;  // a dropped pair has no row: 0
    }
  }
}

// ---------------------------------------------------------------- host side

static deamoe_status_t check_pairs(int32_t dtype, int32_t tokens, int32_t k, int32_t h) {
  if (!known_type(dtype) || k <= 0 || h <= 0) return DEAMOE_ERR_INVALID_ARG;
  if (k > DEAMOE_MAX_TOPK || h > DEAMOE_MAX_WIDTH) return DEAMOE_ERR_UNSUPPORTED;
  if (tokens < 0 || (int64_t)tokens * k > INT_MAX) return DEAMOE_ERR_BATCH;
  return DEAMOE_OK;
}
static bool bad_matrix(const void* p, int64_t stride, int32_t h, size_t es) {
  return !p || !aligned_to(p, es) || stride < h;
}
static deamoe_status_t launched() { return cudaGetLastError() == cudaSuccess ? DEAMOE_OK : DEAMOE_ERR_CUDA; }

template <typename T>
static deamoe_status_t dispatch_t(cudaStream_t s, const void* x, int64_t xs, const int32_t* pr, int32_t tokens, int k,
                                  int h, void* rows, int64_t rs, int64_t n_rows) {
  constexpr int VE = 16 / sizeof(T);
  const bool wide = h % VE == 0 && wide_rows(x, xs, tokens, sizeof(T)) && wide_rows(rows, rs, n_rows, sizeof(T));
  const int packs = wide ? h / VE : h;
  const RowGrid g = row_grid(tokens, packs);
  if (wide)
    k_dispatch<T, VE><<<g.grid, g.block, 0, s>>>((const T*)x, xs, pr, tokens, k, packs, (T*)rows, rs, (unsigned)n_rows);
  else
    k_dispatch<T, 1><<<g.grid, g.block, 0, s>>>((const T*)x, xs, pr, tokens, k, packs, (T*)rows, rs, (unsigned)n_rows);
  return launched();
}

template <typename T>
static deamoe_status_t collect_t(cudaStream_t s, const void* rows, int64_t rs, int64_t n_rows, const int32_t* pr,
                                 const float* w, int32_t tokens, int k, int h, void* out, int64_t os) {
  constexpr int VE = 16 / sizeof(T);
  const bool wide = h % VE == 0 && wide_rows(out, os, tokens, sizeof(T)) && wide_rows(rows, rs, n_rows, sizeof(T));
  const int packs = wide ? h / VE : h;
  const RowGrid g = row_grid(tokens, packs);
  auto fn = wide ? (w ? k_collect<T, VE, true> : k_collect<T, VE, false>) : (w ? k_collect<T, 1, true> : k_collect<T, 1, false>);
  fn<<<g.grid, g.block, 0, s>>>((const T*)rows, rs, (unsigned)n_rows, pr, w, tokens, k, packs, (T*)out, os);
  return launched();
}

template <typename T>
static deamoe_status_t collect_grad_t(cudaStream_t s, const void* dout, int64_t ds, const void* rows, int64_t rs,
                                      int64_t n_rows, const int32_t* pr, const float* w, int32_t tokens, int k, int h,
                                      void* drows, int64_t drs, float* dw) {
  constexpr int VE = 16 / sizeof(T);
  const bool wide = h % VE == 0 && wide_rows(dout, ds, tokens, sizeof(T)) &&
                    (!dw || wide_rows(rows, rs, n_rows, sizeof(T))) && (!drows || wide_rows(drows, drs, n_rows, sizeof(T)));
  const int packs = wide ? h / VE : h;
  int bx = 32;
  while (bx < 256 && bx < packs) bx *= 2;
  const dim3 block(bx, 256 / bx), grid((unsigned)(((int64_t)tokens + block.y - 1) / block.y));
  auto fn = wide ? k_collect_grad<T, VE> : k_collect_grad<T, 1>;
  fn<<<grid, block, 0, s>>>((const T*)dout, ds, (const T*)rows, rs, (unsigned)n_rows, pr, w, tokens, k, packs, (T*)drows,
                            drs, dw);
  return launched();
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_sort_workspace(int32_t n_token, int32_t top_k, int32_t n_expert) {
  const int64_t P = (int64_t)n_token * top_k;
  if (n_token < 0 || top_k <= 0 || n_expert <= 0 || P <= SORT_SMALL_PAIRS) return 0;
  return sort_hist_bytes(P, n_expert) + (uint64_t)n_expert * sizeof(int32_t) + (uint64_t)P * sizeof(unsigned short);
}

deamoe_status_t deamoe_sort_pairs(void* cuda_stream, const int32_t* topk_idx, int32_t n_token, int32_t top_k,
                                  int32_t n_expert, int32_t* expert_off, int32_t* pair_row, int32_t* row_pair,
                                  void* workspace, uint64_t workspace_bytes) {
  if (n_expert <= 0) return DEAMOE_ERR_INVALID_ARG;
  if (n_expert > DEAMOE_MAX_EXPERTS) return DEAMOE_ERR_UNSUPPORTED;
  deamoe_status_t st = check_pairs(DEAMOE_F32, n_token, top_k, 1);
  if (st != DEAMOE_OK) return st;
  if (!expert_off || (n_token > 0 && (!topk_idx || !pair_row || !row_pair))) return DEAMOE_ERR_INVALID_ARG;
  if (!aligned_to(topk_idx, 4) || !aligned_to(expert_off, 4) || !aligned_to(pair_row, 4) || !aligned_to(row_pair, 4))
    return DEAMOE_ERR_INVALID_ARG;
  const int P = n_token * top_k, n = n_expert;
  const uint64_t need = deamoe_sort_workspace(n_token, top_k, n_expert);
  if (need > 0 && (!workspace || !aligned_to(workspace, 4) || workspace_bytes < need)) return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (P <= SORT_SMALL_PAIRS) {
    int warps = (P + 31) / 32;
    if (warps > 32) warps = 32;
    if (warps > SORT_COUNTERS / n) warps = SORT_COUNTERS / n;
    if (warps < 1) warps = 1;
    const int threads = warps > 8 || n > 512 ? 1024 : 256;
    k_sort_small<<<1, threads, 0, s>>>(topk_idx, P, n, warps, expert_off, pair_row, row_pair);
    return launched();
  }
  const int G = (int)(((int64_t)P + SORT_SEG - 1) / SORT_SEG);
  int32_t* hist = reinterpret_cast<int32_t*>(workspace);
  int32_t* total = hist + sort_hist_bytes(P, n) / sizeof(int32_t);
  unsigned short* rank = reinterpret_cast<unsigned short*>(total + n);
  k_sort_count<<<G, SORT_SEG_WARPS * 32, 0, s>>>(topk_idx, P, n, hist, rank);
  if (launched() != DEAMOE_OK) return DEAMOE_ERR_CUDA;
  if (launch_pdl(k_sort_scan, dim3((n + 31) / 32), dim3(1024), 0, s, hist, G, n, total) != cudaSuccess ||
      launch_pdl(k_sort_place, dim3(G), dim3(SORT_SEG_WARPS * 32), 0, s, topk_idx, P, n, hist, total, rank, expert_off,
                 pair_row, row_pair) != cudaSuccess) {
    cudaGetLastError();
    return DEAMOE_ERR_CUDA;
  }
  return DEAMOE_OK;
}

deamoe_status_t deamoe_dispatch(void* cuda_stream, int32_t dtype, const void* x, int64_t x_stride, const int32_t* pair_row,
                                int32_t n_token, int32_t top_k, int32_t hidden, void* rows, int64_t rows_stride,
                                int64_t n_rows) {
  deamoe_status_t st = check_pairs(dtype, n_token, top_k, hidden);
  if (st != DEAMOE_OK) return st;
  if (n_rows < 0 || n_rows > INT_MAX) return DEAMOE_ERR_INVALID_ARG;
  if (n_token == 0 || n_rows == 0) return DEAMOE_OK;
  const size_t es = type_bytes(dtype);
  if (bad_matrix(x, x_stride, hidden, es) || bad_matrix(rows, rows_stride, hidden, es) || x == rows || !pair_row ||
      !aligned_to(pair_row, 4))
    return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32
             ? dispatch_t<float>(s, x, x_stride, pair_row, n_token, top_k, hidden, rows, rows_stride, n_rows)
             : dispatch_t<__nv_bfloat16>(s, x, x_stride, pair_row, n_token, top_k, hidden, rows, rows_stride, n_rows);
}

static deamoe_status_t collect_impl(void* cuda_stream, int32_t dtype, const void* rows, int64_t rows_stride,
                                    int64_t n_rows, const int32_t* pair_row, const float* w, int32_t n_token,
                                    int32_t top_k, int32_t hidden, void* out, int64_t out_stride) {
  deamoe_status_t st = check_pairs(dtype, n_token, top_k, hidden);
  if (st != DEAMOE_OK) return st;
  if (n_rows < 0 || n_rows > INT_MAX) return DEAMOE_ERR_INVALID_ARG;
  if (n_token == 0) return DEAMOE_OK;
  const size_t es = type_bytes(dtype);
  if ((n_rows > 0 && bad_matrix(rows, rows_stride, hidden, es)) || bad_matrix(out, out_stride, hidden, es) ||
      rows == out || !pair_row || !aligned_to(pair_row, 4) || !aligned_to(w, 4))
    return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32
             ? collect_t<float>(s, rows, rows_stride, n_rows, pair_row, w, n_token, top_k, hidden, out, out_stride)
             : collect_t<__nv_bfloat16>(s, rows, rows_stride, n_rows, pair_row, w, n_token, top_k, hidden, out, out_stride);
}

deamoe_status_t deamoe_dispatch_backward(void* cuda_stream, int32_t dtype, const void* drows, int64_t drows_stride,
                                         int64_t n_rows, const int32_t* pair_row, int32_t n_token, int32_t top_k,
                                         int32_t hidden, void* dx, int64_t dx_stride) {
  return collect_impl(cuda_stream, dtype, drows, drows_stride, n_rows, pair_row, nullptr, n_token, top_k, hidden, dx,
                      dx_stride);
}

deamoe_status_t deamoe_combine(void* cuda_stream, int32_t dtype, const void* rows, int64_t rows_stride, int64_t n_rows,
                               const int32_t* pair_row, const float* topk_w, int32_t n_token, int32_t top_k,
                               int32_t hidden, void* out, int64_t out_stride) {
  if (n_token > 0 && !topk_w) return DEAMOE_ERR_INVALID_ARG;
  return collect_impl(cuda_stream, dtype, rows, rows_stride, n_rows, pair_row, topk_w, n_token, top_k, hidden, out,
                      out_stride);
}

deamoe_status_t deamoe_combine_backward(void* cuda_stream, int32_t dtype, const void* dout, int64_t dout_stride,
                                        const void* rows, int64_t rows_stride, int64_t n_rows, const int32_t* pair_row,
                                        const float* topk_w, int32_t n_token, int32_t top_k, int32_t hidden, void* drows,
                                        int64_t drows_stride, float* dw) {
  deamoe_status_t st = check_pairs(dtype, n_token, top_k, hidden);
  if (st != DEAMOE_OK) return st;
  if (n_rows < 0 || n_rows > INT_MAX || (!drows && !dw)) return DEAMOE_ERR_INVALID_ARG;
  if (n_token == 0) return DEAMOE_OK;
  const size_t es = type_bytes(dtype);
  if (bad_matrix(dout, dout_stride, hidden, es) || (dw && n_rows > 0 && bad_matrix(rows, rows_stride, hidden, es)) ||
      (drows && bad_matrix(drows, drows_stride, hidden, es)) || !pair_row || !topk_w)
    return DEAMOE_ERR_INVALID_ARG;
  if (!aligned_to(pair_row, 4) || !aligned_to(topk_w, 4) || !aligned_to(dw, 4)) return DEAMOE_ERR_INVALID_ARG;
  if (drows && (drows == rows || drows == dout)) return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  return dtype == DEAMOE_F32 ? collect_grad_t<float>(s, dout, dout_stride, rows, rows_stride, n_rows, pair_row, topk_w,
                                                     n_token, top_k, hidden, drows, drows_stride, dw)
                             : collect_grad_t<__nv_bfloat16>(s, dout, dout_stride, rows, rows_stride, n_rows, pair_row,
                                                             topk_w, n_token, top_k, hidden, drows, drows_stride, dw);
}

}  // extern "C"
