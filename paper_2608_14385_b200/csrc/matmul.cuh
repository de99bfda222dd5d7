// Products on the fifth-generation tensor cores for the operators around a layer (ffn.cu, product.cu): one persistent
// kernel over 256 x 256 tiles by pairs of CTAs, its operand orders, row groups and epilogues as template parameters.
//
//   D[m, n] = sum_k A[m, k] B[n, k]      stored at out[n][m], weight gradients at out[m][n]
//
// A is the operand whose rows become the outputs' columns (a weight matrix), B the one whose rows become the outputs' rows (tokens).
// With the tokens on the N side a group of any size is a tile of its own width (16 to 256 columns in steps of 16), from a decode step's few rows
// an expert to a prompt's thousands, and the matrix side is always full.
//
// What bounds it.  A bf16 MMA of 256 x 256 x 16 by a pair keeps both SMs' tensor cores busy for 128 cycles; each CTA's
// shared memory then delivers 128 rows of A and 128 of B (8 KB) and takes in as much, 128 bytes a cycle together: a pair
// shares B, a lone CTA with 128 x 256 would need half as much again.  Few rows a group: the matrix's bytes.
//
// Roles of a CTA (1 CTA per SM, clusters of 2, tiles dealt in a fixed order so that equal calls give equal bits):
//   warps 0-7  epilogue, two teams that share a tile's columns: accumulator -> registers -> a warp's transposing buffer -> 16-byte
//              pieces of rows, with the epilogue's arithmetic in fp32
//   warps 8, 9 one thread each issues the TMA copies of A's / B's part of a chunk (128 bytes of k, 128-byte swizzle) into a ring of 5 to 9 stages
//   warp  10   in the pair's first CTA one thread issues the MMAs for both
//   warp  11   ragged contractions (weight gradients: k runs over a group's rows): clears the rows behind the group's end
//              that the last chunk's box brought in, in both operands, before the MMAs may read them
// Two accumulators of 256 columns take turns in tensor memory, so an epilogue runs under the next tile's MMAs.
//
// The tensor cores cut their fp32 sums at every step: terms of one sign lose 6e-9 of their sum a term (bf16, measured: 1.8e-4 over 32768
// terms, 6.6e-3 over 2^20, a third of the sum over 2^26; e4m3 a tenth of that).  So a contraction runs in stretches of MM_STRETCH
// chunks: each is a turn of an accumulator, and the epilogue adds them up in fp32 proper, in their order.
// Every wait is bounded; one that expires ends the CTA's roles and raises the status word that
// deamoe_operator_status reads.
#pragma once
#include <cuda.h>

#include "row.cuh"

namespace deamoe {

enum MatmulEpilogue : int {
  ME_STORE = 0,        // bf16
  ME_STORE_F32 = 1,    // fp32
  ME_SWIGLU = 2,       // A's rows alternate 8 gate, 8 up: silu(gate) up
  ME_SWIGLU_GRAD = 3,  // the same accumulators and the gradient of their product -> gradients of gate and up, and the product
  ME_PRODUCT = 4,      // scales, bias, activation, residual
  ME_PRODUCT_GRAD = 5, // dout times the activation's derivative, and its sums over a tile's rows
  ME_PART = 6,         // fp32 sums of a part of k, [split][row][M rounded up to 8], for join.cu
  ME_PART_DUAL = 7,    // ... of alternating gate and up, [split][row][2 M]
  ME_STORE_ROWS = 8    // bf16, stored at out[m][n] (weight gradients)
};

struct MatmulArgs {
  int M, K;              // rows of A of a group; length of the contraction in values (ragged: the group's rows instead)
  int N;                 // rows of B of one group; grouped rows: the length of the row range
  int groups;
  const int32_t* off;    // [groups + 1] rows of the groups, or null (one group of all rows)
  int tile_n;            // widest tile
  int chunk;             // values of k in 128 bytes
  int splits;            // parts of k that a tile is dealt in (ME_PART, ME_PART_DUAL; else 1)
  int stages, b_bytes;   // of the ring; bytes of a chunk of B's box in a stage (map_b, map_b_rows_inner)
  int late;              // behind another kernel of the call whose results it does not need (see matmul.cu)
  // epilogue
  void* out;
  int64_t os;            // values between out's rows
  int64_t out_group;     // values between splits
  int wide;              // out's rows take 16-byte stores
  const float* dh;       // [N, f]                       (ME_SWIGLU_GRAD)
  void* h_out;           // [N, f] bf16
  int f;
  const void *bias, *residual, *dout;
  const float *x_scale, *w_scale;
  int64_t rs;            // residual's or dout's row stride
  int bias_f32, act, wide_in;
  float* part;           // [2 tiles of N][M] sums of dz    (ME_PRODUCT_GRAD)
  float* sums;           // MM_SUMS_BYTES of matmul_sums(), or null where a contraction is one stretch; no two launches that overlap share them
};

struct MatmulMaps {
  CUtensorMap a, b, out;  // (out: ME_STORE_ROWS)
};

struct MatmulCall {
  MatmulArgs args;
  MatmulMaps maps;
};
enum MatmulForm : int {
  MF_SWIGLU, MF_STORE, MF_STORE_TRANSPOSED, MF_F32_TRANSPOSED, MF_SWIGLU_GRAD, MF_WEIGHT_GRAD, MF_PRODUCT, MF_PRODUCT_E4M3, MF_PRODUCT_GRAD,
  MF_PART, MF_PART_E4M3, MF_PART_SWIGLU
};
cudaError_t matmul_launch(MatmulForm form, const MatmulCall& c, cudaStream_t s);

// Tensor maps.  A matrix of `rows` rows of `cols` values per group, row stride and group stride in values.
bool map_rows(CUtensorMap* m, const void* p, int esize, int64_t cols, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride,
              int box_rows);                       // box: 128 bytes of a row x box_rows rows
bool map_gate_up(CUtensorMap* m, const void* p, int64_t cols, int64_t f, int64_t groups);  // 128 rows: 8 gate, 8 up, ...
// ... of B, with its share of a stage: rows of k as the inner axis (after args.tile_n), or B's rows as the inner axis
bool map_b(MatmulCall* c, const void* p, int esize, int64_t cols, int64_t rows, int64_t stride);
bool map_b_rows_inner(MatmulCall* c, const void* p, int64_t cols, int64_t rows, int64_t stride);

// Tile width of `n` rows in one group for `m_tiles` tiles of A's rows; whole: the product may be split along k.  See matmul.cu
int matmul_tile_n(int64_t n, int64_t m_tiles, bool whole);

// ... of the output of a weight gradient: 32 rows of 64 values
bool map_out(MatmulCall* c, const void* p, int64_t cols, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride);

// Widest tile for `rows` rows in `groups` groups of unknown sizes: four times the average, so that most groups are one tile and a
// stage of the ring holds no more of B than they need, and a 32nd of all rows at least, should they come to one group
int matmul_group_tile_n(int64_t rows, int64_t groups);
// Parts of k for a product of at most `tiles` tiles, `chunks` chunks of k and rows x outputs sums (1: not split): see matmul.cu
int matmul_splits(int64_t tiles, int64_t chunks, int64_t rows, int64_t outputs);

// Adds the splits' sums in their order and applies the epilogue: [splits][n_rows][M rounded up to 8] (dual: [2 M]) -> out.  (join.cu)
struct JoinArgs {
  const float* part;
  int splits, n_rows, M, groups, dual;
  const int32_t* off;    // rows outside [off[0], off[groups]) and rows of falling offsets are left alone; or null
  __nv_bfloat16* out;
  int64_t os;
  const float *x_scale, *w_scale;
  const void *bias, *residual;
  int64_t rs;
  int bias_f32, act, wide;
};
cudaError_t join_launch(const JoinArgs& a, cudaStream_t s);

constexpr int MM_M = 256, MM_N = 256;
constexpr int MM_MAX_ROWS = INT32_MAX - 256;  // so that a tile's end is a number of 32 bits
constexpr int MM_N_LEAST = 64;   // matmul_tile_n gives no less for more rows
constexpr int MM_PARTS = 2;      // rows of sums that a tile leaves in `part`

// Chunks of a stretch: 32768 values (e4m3: 65536), whose loss is a tenth of half a step of bf16 at most.
constexpr int MM_STRETCH = 512;
constexpr uint64_t MM_SUMS_BYTES = 148ull * 128 * MM_N * 4;  // a CTA's half of a tile
// Bytes of `sums` for a contraction over k values in chunks of `chunk`, dealt in `splits` parts.
inline uint64_t matmul_sums(int64_t k, int chunk, int splits) {
  const int64_t chunks = (k + chunk - 1) / chunk;
  return (chunks + splits - 1) / splits > MM_STRETCH ? MM_SUMS_BYTES : 0;
}

}  // namespace deamoe
