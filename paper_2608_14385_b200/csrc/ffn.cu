// Gated feed-forward blocks of experts over rows in expert order (or of one expert), and their gradients.
//
//   g = x Wg^T, u = x Wu^T, h = silu(g) u, y = h Wd^T
//   dh = dy Wd,  dg = dh u s (1 + g (1 - s)),  du = dh silu(g),  s = sigmoid(g)
//   dx = dg Wg + du Wu,  d[Wg; Wu] = [dg du]^T x,  dWd = dy^T h
//
// Two launches forward: gate and up as one product whose epilogue forms h, then the down product.  h is rounded to bf16 between
// them (the tensor cores' operand; half a step of bf16 beside that of the output).  Five launches backward: dh (kept in fp32),
// gate and up once more from the forward's inputs with an epilogue that turns them and dh into dg, du and h (each rounded
// once, as operands), dx, and the two weight gradients.  The backward call takes the forward's inputs and keeps nothing of the
// forward pass: gate and up would cost 4 bytes a value to keep exactly, and recomputing them lets no rounding but the
// operands' into a gradient.
#include "matmul.cuh"
#include "thin.cuh"

namespace deamoe {

static uint64_t ceil256(uint64_t v) { return (v + 255) / 256 * 256; }

struct FfnShape {
  int E, R, h, f;
  const int32_t* off;
};

static MatmulCall ffn_call(const FfnShape& S, int M, int K) {
  MatmulCall c = {};
  c.args.M = M; c.args.K = K; c.args.N = S.R; c.args.groups = S.E; c.args.off = S.off; c.args.tile_n = matmul_group_tile_n(S.R, S.E < S.R ? S.E : S.R); c.args.chunk = 64; c.args.splits = 1;
  c.args.f = S.f; c.args.wide = 1;
  return c;
}

// Few rows, of few experts: from some nine experts on there are tiles enough for the tensor-core kernel, whose copies keep more bytes in
// flight.  9 to 16 rows at random over the experts, us thin and on the tensor cores: 7168 x 2048, 8 experts 100 and 102, 9 experts 131 and
// 120, 32 experts 193 and 167; 4096 x 1536, 8 experts 47 and 50, 16 experts 80 and 74; 2048 x 768, 8 experts 21 and 22, 16 experts 27 and
// 28.  Narrower ones stay bound by their launches, where the line is not the best one (1024 x 384: 8 experts 9.7 and 15, 9 experts
// 11 and 16, 64 experts 15 and 16).
static bool ffn_thin(int E, int R) { return R <= THIN_ROWS && (E <= 8 || R <= 8); }
// A forward product's parts of k: M rows of a matrix (gate and up: of both), K columns.
static int ffn_splits(int E, int R, int64_t M, int64_t K) {
  const int groups = E < R ? E : R;
  const int64_t tiles = (M + MM_M - 1) / MM_M * (R / matmul_group_tile_n(R, groups) + groups);  // no more than that, whatever the offsets
  return matmul_splits(tiles, (K + 63) / 64, R, M);
}
static uint64_t ffn_parts_bytes(int E, int R, int h, int f) {
  const int a = ffn_splits(E, R, 2 * (int64_t)f, h), b = ffn_splits(E, R, h, f);
  const uint64_t up = a > 1 ? (uint64_t)a * R * 2 * f * 4 : 0, down = b > 1 ? (uint64_t)b * R * h * 4 : 0;
  return up > down ? up : down;
}
// Sums of contractions of more than one stretch: the forward products run one after the other.
static uint64_t ffn_sums(int E, int R, int h, int f) {
  const uint64_t up = matmul_sums(h, 64, ffn_splits(E, R, 2 * (int64_t)f, h)), down = matmul_sums(f, 64, ffn_splits(E, R, h, f));
  return up > down ? up : down;
}
// Backward, sums for each of the three that can overlap (dx and both weight gradients).
static uint64_t ffn_backward_sums(int R, int h, int f) {
  const int64_t k = h > 2 * (int64_t)f ? h : 2 * (int64_t)f;
  return matmul_sums(k > R ? k : R, 64, 1);
}

static deamoe_status_t check_ffn(const void* x, int64_t xs, const void* wgu, const void* wd, const int32_t* off, int E, int R, int h, int f) {
  if (E <= 0 || h <= 0 || f <= 0 || (!off && E != 1)) return DEAMOE_ERR_INVALID_ARG;
  if (E > DEAMOE_MAX_EXPERTS || h > DEAMOE_MAX_WIDTH || f > DEAMOE_MAX_WIDTH || h % 8 || f % 8) return DEAMOE_ERR_UNSUPPORTED;
  if (R < 0 || R > MM_MAX_ROWS) return DEAMOE_ERR_BATCH;
  // tiles are counted in 32 bits: a group has at most one tile more than its share of the rows; a matrix's gradient tiles of 256 x 256
  const int64_t most = (int64_t)R / 32 + E, a = h / MM_M + 1, b = 2 * (int64_t)f / MM_N + 1;
  if (most * 2 * (a > b ? a : b) > INT32_MAX || E * a * b > INT32_MAX) return DEAMOE_ERR_BATCH;
  if (!wgu || !wd || !aligned16(wgu) || !aligned16(wd) || !aligned_to(off, 4)) return DEAMOE_ERR_INVALID_ARG;
  if (R > 0 && (!x || !aligned16(x) || xs < h || xs % 8)) return DEAMOE_ERR_INVALID_ARG;
  return DEAMOE_OK;
}
static bool bad_rows8(const void* p, int64_t stride, int h) { return !p || !aligned16(p) || stride < h || stride % 8; }

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_ffn_workspace(int32_t n_expert, int32_t n_rows, int32_t hidden, int32_t ffn, int32_t backward) {
  if (n_expert <= 0 || n_rows <= 0 || hidden <= 0 || ffn <= 0) return 0;
  const uint64_t v = (uint64_t)n_rows * ffn;
  if (backward) return ceil256(4 * v) + ceil256(4 * v) + ceil256(2 * v) + 3 * ffn_backward_sums(n_rows, hidden, ffn);
  if (ffn_thin(n_expert, n_rows)) return ceil256(2 * v);
  return ceil256(2 * v) + ceil256(ffn_parts_bytes(n_expert, n_rows, hidden, ffn)) + ffn_sums(n_expert, n_rows, hidden, ffn);
}

deamoe_status_t deamoe_ffn(void* cuda_stream, const void* x, int64_t x_stride, const void* w_gate_up, const void* w_down,
                           const int32_t* expert_off, int32_t n_expert, int32_t n_rows, int32_t hidden, int32_t ffn, void* out,
                           int64_t out_stride, void* workspace, uint64_t workspace_bytes) {
  deamoe_status_t st = check_ffn(x, x_stride, w_gate_up, w_down, expert_off, n_expert, n_rows, hidden, ffn);
  if (st != DEAMOE_OK || n_rows == 0) return st;
  if (bad_rows8(out, out_stride, hidden) || out == x) return DEAMOE_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) || workspace_bytes < deamoe_ffn_workspace(n_expert, n_rows, hidden, ffn, 0)) return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (ffn_thin(n_expert, n_rows)) {
    ThinArgs a = {};
    a.x = x; a.xs = x_stride; a.w = w_gate_up; a.M = ffn; a.K = hidden; a.n_rows = n_rows; a.groups = n_expert; a.off = expert_off;
    a.out = reinterpret_cast<__nv_bfloat16*>(workspace); a.os = ffn;
    ThinArgs b = a;
    b.x = workspace; b.xs = ffn; b.w = w_down; b.M = hidden; b.K = ffn; b.out = reinterpret_cast<__nv_bfloat16*>(out); b.os = out_stride;
    if (thin_launch(false, true, a, s, false) == cudaSuccess && thin_launch(false, false, b, s, true) == cudaSuccess) return DEAMOE_OK;
    cudaGetLastError();
    return DEAMOE_ERR_CUDA;
  }
  const FfnShape S = {n_expert, n_rows, hidden, ffn, expert_off};
  MatmulCall up = ffn_call(S, ffn, hidden), down = ffn_call(S, hidden, ffn);
  up.args.out = workspace; up.args.os = ffn;
  down.args.out = out; down.args.os = out_stride;
  // few tiles: dealt along k, the parts' sums joined by a kernel of their own
  const int up_splits = ffn_splits(n_expert, n_rows, 2 * (int64_t)ffn, hidden), down_splits = ffn_splits(n_expert, n_rows, hidden, ffn);
  float* part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + ceil256(2 * (uint64_t)n_rows * ffn));
  if (ffn_sums(n_expert, n_rows, hidden, ffn))
    up.args.sums = down.args.sums = reinterpret_cast<float*>(reinterpret_cast<char*>(part) + ceil256(ffn_parts_bytes(n_expert, n_rows, hidden, ffn)));
  auto joined = [&](MatmulCall& c, int splits, bool dual) {
    JoinArgs j = {};
    j.part = part; j.splits = splits; j.n_rows = n_rows; j.M = c.args.M; j.groups = n_expert; j.dual = dual; j.off = expert_off;
    j.out = reinterpret_cast<__nv_bfloat16*>(c.args.out); j.os = c.args.os; j.wide = 1;
    c.args.splits = splits; c.args.out = part; c.args.os = (int64_t)c.args.M * (dual ? 2 : 1); c.args.out_group = c.args.os * n_rows;
    return j;
  };
  if (!map_gate_up(&up.maps.a, w_gate_up, hidden, ffn, n_expert) || !map_b(&up, x, 2, hidden, n_rows, x_stride) ||
      !map_rows(&down.maps.a, w_down, 2, ffn, hidden, ffn, n_expert, (int64_t)hidden * ffn, 128) ||
      !map_b(&down, workspace, 2, ffn, n_rows, ffn))
    return DEAMOE_ERR_CUDA;
  cudaError_t e;
  if (up_splits > 1) {
    const JoinArgs j = joined(up, up_splits, true);
    e = matmul_launch(MF_PART_SWIGLU, up, s);
    if (e == cudaSuccess) e = join_launch(j, s);
  } else {
    e = matmul_launch(MF_SWIGLU, up, s);
  }
  if (e == cudaSuccess && down_splits > 1) {
    const JoinArgs j = joined(down, down_splits, false);
    e = matmul_launch(MF_PART, down, s);
    if (e == cudaSuccess) e = join_launch(j, s);
  } else if (e == cudaSuccess) {
    e = matmul_launch(MF_STORE, down, s);
  }
  if (e == cudaSuccess) return DEAMOE_OK;
  cudaGetLastError();
  return DEAMOE_ERR_CUDA;
}

deamoe_status_t deamoe_ffn_backward(void* cuda_stream, const void* x, int64_t x_stride, const void* w_gate_up, const void* w_down,
                                    const void* dout, int64_t dout_stride, const int32_t* expert_off, int32_t n_expert,
                                    int32_t n_rows, int32_t hidden, int32_t ffn, void* dx, int64_t dx_stride, void* dw_gate_up,
                                    void* dw_down, void* workspace, uint64_t workspace_bytes) {
  deamoe_status_t st = check_ffn(x, x_stride, w_gate_up, w_down, expert_off, n_expert, n_rows, hidden, ffn);
  if (st != DEAMOE_OK) return st;
  if (!dw_gate_up || !dw_down || !aligned16(dw_gate_up) || !aligned16(dw_down) || dw_gate_up == w_gate_up || dw_down == w_down ||
      dw_gate_up == dw_down)
    return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  const size_t wd_bytes = (size_t)n_expert * hidden * ffn * 2;
  if (n_rows == 0)  // sums over no rows
    return cudaMemsetAsync(dw_gate_up, 0, 2 * wd_bytes, s) == cudaSuccess && cudaMemsetAsync(dw_down, 0, wd_bytes, s) == cudaSuccess
               ? DEAMOE_OK : DEAMOE_ERR_CUDA;
  if (bad_rows8(dout, dout_stride, hidden) || bad_rows8(dx, dx_stride, hidden) || dx == x || dx == dout) return DEAMOE_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) || workspace_bytes < deamoe_ffn_workspace(n_expert, n_rows, hidden, ffn, 1)) return DEAMOE_ERR_INVALID_ARG;
  const FfnShape S = {n_expert, n_rows, hidden, ffn, expert_off};
  const uint64_t v = (uint64_t)n_rows * ffn;
  char* ws = reinterpret_cast<char*>(workspace);
  float* dh = reinterpret_cast<float*>(ws);
  void* dgu = ws + ceil256(4 * v);
  void* hh = ws + 2 * ceil256(4 * v);
  const int64_t wd_one = (int64_t)hidden * ffn;

  MatmulCall a = ffn_call(S, ffn, hidden);  // dh = dy Wd
  a.args.out = dh; a.args.os = ffn;
  MatmulCall b = ffn_call(S, ffn, hidden);  // gate, up -> dg, du, h
  b.args.out = dgu; b.args.os = 2 * (int64_t)ffn; b.args.dh = dh; b.args.h_out = hh;
  MatmulCall c = ffn_call(S, hidden, 2 * ffn);  // dx = [dg du] [Wg; Wu]
  c.args.out = dx; c.args.os = dx_stride;
  MatmulCall d = ffn_call(S, 2 * ffn, n_rows);  // d[Wg; Wu] = [dg du]^T x
  d.args.tile_n = MM_N; d.args.N = hidden;
  MatmulCall e = ffn_call(S, hidden, n_rows);  // dWd = dy^T h
  e.args.tile_n = MM_N; e.args.N = ffn;
  d.args.late = e.args.late = 1;  // they need b's results as c does, and c waits for those
  // what can run at the same time has sums of its own: b beside a, d beside c, e beside both
  if (const uint64_t each = ffn_backward_sums(n_rows, hidden, ffn)) {
    char* sums = ws + 2 * ceil256(4 * v) + ceil256(2 * v);
    a.args.sums = c.args.sums = reinterpret_cast<float*>(sums);
    b.args.sums = d.args.sums = reinterpret_cast<float*>(sums + each);
    e.args.sums = reinterpret_cast<float*>(sums + 2 * each);
  }
  if (!map_rows(&a.maps.a, w_down, 2, ffn, hidden, ffn, n_expert, wd_one, 64) || !map_b(&a, dout, 2, hidden, n_rows, dout_stride) ||
      !map_gate_up(&b.maps.a, w_gate_up, hidden, ffn, n_expert) || !map_b(&b, x, 2, hidden, n_rows, x_stride) ||
      !map_rows(&c.maps.a, w_gate_up, 2, hidden, 2 * (int64_t)ffn, hidden, n_expert, 2 * wd_one, 64) ||
      !map_b(&c, dgu, 2, 2 * (int64_t)ffn, n_rows, 2 * (int64_t)ffn) ||
      !map_rows(&d.maps.a, dgu, 2, 2 * (int64_t)ffn, n_rows, 2 * (int64_t)ffn, 1, 2 * (int64_t)ffn, 64) ||
      !map_b_rows_inner(&d, x, hidden, n_rows, x_stride) || !map_out(&d, dw_gate_up, hidden, 2 * (int64_t)ffn, hidden, n_expert, 2 * wd_one) ||
      !map_rows(&e.maps.a, dout, 2, hidden, n_rows, dout_stride, 1, dout_stride, 64) || !map_b_rows_inner(&e, hh, ffn, n_rows, ffn) ||
      !map_out(&e, dw_down, ffn, hidden, ffn, n_expert, wd_one))
    return DEAMOE_ERR_CUDA;
  if (matmul_launch(MF_F32_TRANSPOSED, a, s) == cudaSuccess && matmul_launch(MF_SWIGLU_GRAD, b, s) == cudaSuccess &&
      matmul_launch(MF_STORE_TRANSPOSED, c, s) == cudaSuccess && matmul_launch(MF_WEIGHT_GRAD, d, s) == cudaSuccess &&
      matmul_launch(MF_WEIGHT_GRAD, e, s) == cudaSuccess)
    return DEAMOE_OK;
  cudaGetLastError();
  return DEAMOE_ERR_CUDA;
}

}  // extern "C"
