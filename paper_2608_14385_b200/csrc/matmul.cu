// The tensor-core kernel behind the operators around a layer; what it computes and why it is laid out so: matmul.cuh.
#include "matmul.cuh"

#include <atomic>

namespace deamoe {

namespace {

constexpr int MM_RING = 168 * 1024;            // stages of 32 KB (five) to 18 KB (nine), as B's box needs
constexpr int MM_STAGES = 9;                   // at most
constexpr int MM_OPERAND = 16 * 1024;          // one CTA's part of a chunk of A or of B: 128 rows of 128 bytes
constexpr int MM_TEAMS = 2;                    // epilogue teams of 4 warps (a warp reads the 32 lanes of tensor memory of its number mod 4)
constexpr int MM_WARP_A = 4 * MM_TEAMS, MM_WARP_B = MM_WARP_A + 1, MM_WARP_MMA = MM_WARP_A + 2, MM_WARP_CLEAR = MM_WARP_A + 3;
constexpr int MM_THREADS = (MM_WARP_CLEAR + 1) * 32;
constexpr int MM_STEP = 32;                    // accumulator columns of an epilogue step
constexpr int MM_ROW_STEP = 64;                // ... of weight gradients, whose rows are lanes: 128 bytes of a row
constexpr int MM_PITCH = 32 + 4;               // floats of a row of a warp's transposing buffer
constexpr int MM_STAGING = MM_TEAMS * 4 * MM_STEP * MM_PITCH * 4;
constexpr int MM_CONTROL = 512;
// What the copy role says of a tile beside its first stage: its width, the steps of 16 rows of a chunk that has to be cleared behind
// its group's end (0: none), or that there are no more tiles; and its number of chunks.
constexpr uint32_t TILE_END = 1u << 16;
constexpr int TILE_STEPS = 20;
// A chunk to be cleared goes into the ring so many chunks before the tile's end, but is taken last: the MMA role need not wait for
// the clearing.
constexpr int MM_TAIL_LEAD = 2;
__device__ __forceinline__ uint32_t tail_place(uint32_t chunks) { return chunks > MM_TAIL_LEAD ? chunks - 1 - MM_TAIL_LEAD : 0; }
// ... of a whole contraction: in its last stretch
template <bool LONG> __device__ __forceinline__ int tail_of(int chunks) {
  const int before = LONG && chunks > 0 ? (chunks - 1) / MM_STRETCH * MM_STRETCH : 0;
  return before + (int)tail_place(chunks - before);
}
static_assert((MM_STRETCH & (MM_STRETCH - 1)) == 0, "a chunk's place in its stretch");
constexpr int MM_TABLE = (DEAMOE_MAX_EXPERTS + 1) * 8 + 8;  // groups' first tile and first row
constexpr size_t MM_SMEM = (size_t)MM_RING + MM_STAGING + MM_CONTROL + MM_TABLE;
static_assert(MM_RING / (MM_OPERAND + 16 * 128) <= MM_STAGES, "barriers of a stage");
static_assert(MM_SMEM <= 227 * 1024, "shared memory budget");
// One CTA fills more than half of an SM's shared memory, so none of another grid's can be beside it and the
// allocation of all 512 columns of tensor memory never waits.
static_assert(2 * MM_SMEM > 228 * 1024, "tensor-memory allocation must never block");
// After so long without a new stretch among its CTA's copies a wait gives up.  (A stretch takes 0.2 ms at 0.3 us a chunk, but some waits last a
// whole contraction, which over 2^31 rows takes ten seconds, or several tiles.)
constexpr unsigned long long MM_WAIT_NS = 2000000000ull;
constexpr int MM_PAIRS = 74;                   // 148 SMs

__device__ int32_t mm_status;                  // DEAMOE_ERR_TIMEOUT once a wait has expired

// ---------------------------------------------------------------- PTX
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_first(uint32_t addr) {  // the same shared address in the pair's first CTA
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// abort_flag[1]: copies at the last stretch's start.  (Not inlined: each role has its waits, and a small product's time is to a good part that of fetching code.)
__device__ __noinline__ bool bar_wait_longer(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  unsigned long long start = now_ns();
  int copies = abort_flag[1];
  for (unsigned it = 1;; ++it) {
    if (bar_try(bar, parity)) return true;
    if ((it & 63u) == 0 && *abort_flag) return false;
    if ((it & 255u) == 0) {
      const int now = abort_flag[1];
      if (now != copies) start = now_ns();
      else if (now_ns() - start > MM_WAIT_NS) break;
      copies = now;
    }
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return bar_try(bar, parity) || bar_wait_longer(bar, parity, abort_flag);
}
// `bar` may lie in the pair's other CTA
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_5d(uint32_t dst, const CUtensorMap* m, int x, int y, int z, int u, int v, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
// 32 rows of 64 bf16 values of a warp's buffer (128-byte swizzle) to columns x .., rows y .. of group z
__device__ __forceinline__ void store_3d(const CUtensorMap* m, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Shared-memory operand with 128-byte swizzle.  k inner: 8 rows of 128 bytes are a block of 1024 bytes, `sbo` apart.
// Rows inner: a block is 64 values of 8 k's; `sbo` between blocks along k, `lbo` between blocks along the rows.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <bool FP8> __device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  if constexpr (FP8)
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
  else
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// arrives at the barrier of that offset in both CTAs once the MMAs issued so far are done
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
        "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
        "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------- the order of the tiles
struct Tile {
  int group;
  int m0, n0;    // first row of A in the group; first row of B: in all rows (grouped rows) or in the group
  int n, valid;  // width (a multiple of 16), and its columns that exist
  int row0, rows;  // the group's rows (ragged contraction)
  int n_index;   // index of the tile along N in its group
};
// Tiles of a group: its columns are dealt evenly in units of 16 (weight gradients: 64, an epilogue's step), so that one a little above
// a multiple of the widest tile has no sliver.
__device__ __forceinline__ int tiles_along(int n, int widest) { return (n + widest - 1) / widest; }
constexpr int MM_BAND = 8;  // tiles along N that are walked side by side: 74 pairs then share some 8 + 9 operand tiles in the L2

template <bool RAGGED> __device__ __noinline__ Tile find_tile(const MatmulArgs& A, const int* first_tile, const int* first_row, int t,
                                                                 int m_step) {
  int lo = 0, hi = A.groups;  // the group whose range of tiles holds t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_tile[mid] <= t) lo = mid;
    else hi = mid;
  }
  Tile o;
  o.group = lo;
  o.row0 = first_row[lo];
  o.rows = first_row[lo + 1] - o.row0;
  const int cols = RAGGED ? A.N : o.rows;
  const int nt = tiles_along(cols, A.tile_n), mt = (A.M + m_step - 1) / m_step;
  const int r = t - first_tile[lo];
  const int band = r / (MM_BAND * mt), rest = r - band * MM_BAND * mt;
  const int width = min(MM_BAND, nt - band * MM_BAND);
  const int mi = rest / width, ni = band * MM_BAND + rest - mi * width;
  constexpr int UNIT = RAGGED ? MM_ROW_STEP : 16;
  const int units = (cols + UNIT - 1) / UNIT, base = units / nt, more = units - base * nt;  // the first `more` tiles have one more
  const int u0 = ni * base + min(ni, more);
  o.n = (base + (ni < more)) * UNIT;
  o.m0 = mi * m_step;
  o.n_index = ni;
  o.valid = min(o.n, cols - u0 * UNIT);
  o.n0 = u0 * UNIT + (RAGGED ? 0 : o.row0);
  return o;
}

// ---------------------------------------------------------------- epilogue arithmetic
// (The exponential is good to 2 + 1.17 |v| units of fp32 and the division to 2, CUDA's bounds: some ten units at a gate of -4, far below the
// roundings to bf16 behind it, and of the order of what the sums of z lose where there is none, in the bias gradient.)
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }
__device__ __forceinline__ float act_grad(int kind, float z) {
  if (kind == DEAMOE_SIGMA_SILU) {
    const float p = sigmoid(z);
    return p * (1.f + z * (1.f - p));
  }
  if (kind == DEAMOE_SIGMA_GELU)
    return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
  return 1.f;
}
// n <= 8 bf16 values at p; wide: all eight, 16 bytes at once
__device__ __forceinline__ void put8(__nv_bfloat16* p, const float (&v)[8], int n, bool wide) {
  if (wide && n == 8) {
    Pack<__nv_bfloat16, 8> o;
    o.narrow(v);
    store_pack(p, o);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = __float2bfloat16_rn(v[j]);
  }
}
__device__ __forceinline__ void put8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void get8(const __nv_bfloat16* p, float (&v)[8], int n) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? __bfloat162float(p[j]) : 0.f;
}
__device__ __forceinline__ void floats8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ float gain(const void* p, int f32, int i) {
  return f32 ? reinterpret_cast<const float*>(p)[i] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
}
// An epilogue warp's part of a contraction in more than one stretch.  Every stretch but the last is added to the CTA's sums, [column / 4]
// [lane of 128][4], where a thread meets nothing but its own values; the last accumulator takes the total, and the epilogue goes on
// from there as from any other (from the accumulator itself where there is one stretch alone).  a: turns of the accumulators so far; returns that of the last one, or ~0 if a wait has expired.
// STEP: columns of an epilogue step.
template <int STEP> __device__ __forceinline__ uint32_t join_stretches(uint32_t a, int chunks, uint32_t lane_base, int n, float* all_sums,
                                                                       uint32_t acc_full, uint32_t acc_empty, volatile int* abort_flag) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = (warp & 3) * 32 + lane;
  const int stretches = (chunks + MM_STRETCH - 1) / MM_STRETCH;
  if (stretches <= 1) return a;
  float* const sums = all_sums + (int64_t)blockIdx.x * (128 * MM_N);
  for (int i = 0;; ++i, ++a) {
    const uint32_t buf = a & 1u;
    const int w = lane == 0 ? bar_wait(acc_full + 8 * buf, (a >> 1) & 1u, abort_flag) : 0;
    if (__shfl_sync(0xffffffffu, w, 0) == 0) return ~0u;
    tc_after();
    const bool last = i + 1 == stretches;
    for (int c0 = (warp >> 2) * STEP; c0 < n; c0 += MM_TEAMS * STEP)
#pragma unroll 1
      for (int c = c0; c < c0 + STEP; c += 32) {
        uint32_t r[32];
        tmem_load(lane_base + buf * MM_N + c, r);
        tmem_load_wait();
        float4* const at = reinterpret_cast<float4*>(sums) + (c / 4) * 128 + row;
        if (i > 0)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float4 v = __ldcg(at + j * 128);
            r[4 * j] = __float_as_uint(v.x + __uint_as_float(r[4 * j]));
            r[4 * j + 1] = __float_as_uint(v.y + __uint_as_float(r[4 * j + 1]));
            r[4 * j + 2] = __float_as_uint(v.z + __uint_as_float(r[4 * j + 2]));
            r[4 * j + 3] = __float_as_uint(v.w + __uint_as_float(r[4 * j + 3]));
          }
        if (last) {
          tmem_store(lane_base + buf * MM_N + c, r);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            __stcg(at + j * 128, make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]), __uint_as_float(r[4 * j + 2]),
                                             __uint_as_float(r[4 * j + 3])));
        }
      }
    if (last) {
      tmem_store_wait();
      return a;
    }
    tc_before();
    __syncwarp();
    if (lane == 0) bar_arrive_cluster(in_first(acc_empty + 8 * buf));
  }
}
// What an epilogue step of a thread takes from memory, asked for a step ahead.
struct Ahead {
  uint4 v[4];
  float scale[4];
};

// ---------------------------------------------------------------- the kernel
// AT / BT: A / B lies with its rows as the inner axis (k outer); RAGGED: the contraction runs over a group's rows; LONG: it may come in
// more than one stretch (by itself, as a small product's time is to a good part that of fetching code: with both in one kernel the gradients of 10 experts
// of 1032 x 344 took 56.3 us, 55.3 without).
template <int EPI, bool AT, bool BT, bool FP8, bool RAGGED, bool LONG>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MM_THREADS, 1)
    k_matmul(const __grid_constant__ MatmulArgs A, const __grid_constant__ MatmulMaps maps) {
  constexpr bool DUAL = EPI == ME_SWIGLU || EPI == ME_SWIGLU_GRAD || EPI == ME_PART_DUAL;  // A's rows alternate gate and up
  constexpr bool SPLIT = EPI == ME_PART || EPI == ME_PART_DUAL;
  static_assert(RAGGED == (EPI == ME_STORE_ROWS), "groups without rows are zeros in that epilogue alone");
  static_assert(MM_PARTS == MM_TEAMS, "a team leaves a row of `part`");
  constexpr int M_STEP = DUAL ? MM_M / 2 : MM_M;                    // in rows of A as the caller counts them (DUAL: features)
  extern __shared__ __align__(1024) unsigned char smem[];
  float* staging = reinterpret_cast<float*>(smem + MM_RING);
  uint64_t* control = reinterpret_cast<uint64_t*>(smem + MM_RING + MM_STAGING);
  const uint32_t ring = smem_u32(smem), bars = smem_u32(control);
  auto full = [&](int s) { return bars + 8 * s; };
  auto empty = [&](int s) { return bars + 8 * (MM_STAGES + s); };
  auto tail = [&](int s) { return bars + 8 * (2 * MM_STAGES + s); };
  auto cleared = [&](int s) { return bars + 8 * (3 * MM_STAGES + s); };
  auto acc_full = [&](int b) { return bars + 8 * (4 * MM_STAGES + b); };
  auto acc_empty = [&](int b) { return bars + 8 * (4 * MM_STAGES + 2 + b); };
  const uint32_t first_full = in_first(full(0));
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(control + 4 * MM_STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);  // and how far the copies are, see bar_wait
  uint32_t* info = tmem_slot + 3;  // [MM_STAGES][2]: a tile whose first chunk the stage holds
  static_assert((4 * MM_STAGES + 4) * 8 + 12 + MM_STAGES * 8 <= MM_CONTROL, "control region");
  int* first_row = reinterpret_cast<int*>(smem + MM_RING + MM_STAGING + MM_CONTROL);
  int* first_tile = first_row + A.groups + 1;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank(), stages = A.stages, stage_bytes = MM_OPERAND + A.b_bytes;
  if (tid == 0) {
#pragma unroll 1
    for (int s = 0; s < (int)stages; ++s) {
      bar_init(full(s), 1);
      bar_init(empty(s), 1);
      bar_init(tail(s), 1);
      bar_init(cleared(s), 2);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(acc_full(b), 1);
      bar_init(acc_empty(b), 2 * 4 * MM_TEAMS);
    }
    abort_flag[0] = abort_flag[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == MM_WARP_A * 32) prefetch_map(&maps.a);
  if (tid == MM_WARP_B * 32) prefetch_map(&maps.b);
  if (EPI == ME_STORE_ROWS && tid == 0) prefetch_map(&maps.out);
  if (warp == MM_WARP_MMA) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // Launched early behind whatever is before it in the stream, a kernel waits for that here, but for two kinds, which follow another
  // one of their call.  The gradient of gate and up needs that one in its epilogue alone.  A.late: it needs only what was
  // done before that one's own wait, which all its CTAs have passed by now, and waits at its end, so that the stream's order
  // holds for what comes after.
  if (EPI != ME_SWIGLU_GRAD && !A.late) pdl_wait();
  pdl_trigger();
  // groups' rows (offsets outside the range count as its ends) and their tiles; offsets that decrease: no tile at all
  const int mt = (A.M + M_STEP - 1) / M_STEP;
  const int limit = RAGGED ? A.K : A.N;
  if (A.off) {
    bool falls = false;
#pragma unroll 1
    for (int e = tid; e <= A.groups; e += MM_THREADS) {
      const int o = A.off[e];
      if (e > 0) falls |= o < A.off[e - 1];
      first_row[e] = min(max(o, 0), limit);
    }
    falls = __syncthreads_or(falls);
    if (warp == 0) {
      int before = 0;
#pragma unroll 1
      for (int e0 = 0; e0 < A.groups; e0 += 32) {
        const int e = e0 + lane;
        const int n = e < A.groups && !falls ? mt * tiles_along(RAGGED ? A.N : first_row[e + 1] - first_row[e], A.tile_n) : 0;
        int sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += y;
        }
        if (e < A.groups) first_tile[e] = before + sum - n;
        before += __shfl_sync(0xffffffffu, sum, 31);
      }
      if (lane == 0) first_tile[A.groups] = before;
    }
  } else if (tid == 0) {
    first_row[0] = first_tile[0] = 0;
    first_row[1] = limit;
    first_tile[1] = mt * tiles_along(A.N, A.tile_n);
  }
  tc_before();
  cluster_sync();
  tc_after();
  const uint32_t tmem = *tmem_slot;
  const int tiles = first_tile[A.groups] * (SPLIT ? A.splits : 1);  // (SPLIT: parts of tiles)
  const int pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
  auto chunks_of = [&](const Tile& t) { return ((RAGGED ? t.rows : A.K) + A.chunk - 1) / A.chunk; };
  // parts of a tile are dealt evenly, none without a chunk (splits <= chunks)
  auto chunks_in = [&](int it, const Tile& t) {
    const int all = chunks_of(t), base = SPLIT ? all / A.splits : all;
    return SPLIT ? base + (it % A.splits < all - base * A.splits) : all;
  };
  auto tile_at = [&](int it) { return find_tile<RAGGED>(A, first_tile, first_row, SPLIT ? it / A.splits : it, M_STEP); };

  if (warp == MM_WARP_A || warp == MM_WARP_B) {
    // ============================================================ copies
    // A chunk's issue has to fit the 512 cycles of its MMAs here too, and a copy costs its thread some 100: one warp an
    // operand, one box a chunk where the layout allows it, uniform values as in the MMA role.
    const bool is_a = warp == MM_WARP_A, one = elected();
    uint32_t g = 0, s = 0, phase = 1;  // chunks so far; stage, and the phase whose end frees it (a new barrier's phase 1 has ended)
    bool ok = true, free = true;
    const bool rows_inner = is_a ? AT : BT;
    for (int it = pair; ok && it < tiles; it += pairs) {
      const Tile t = tile_at(it);
      const int half = t.n / 2, all = chunks_of(t);
      const int part = SPLIT ? it % A.splits : 0;
      const int base = SPLIT ? all / A.splits : all, more = SPLIT ? all - base * A.splits : 0;
      const int c_begin = part * base + min(part, more), c_end = c_begin + base + (part < more);
      const int at = is_a ? t.m0 + (int)rank * (M_STEP / 2) : t.n0 + (int)rank * half;  // first row of this CTA's part
      const int z = is_a && !RAGGED ? t.group : 0;
      const CUtensorMap* map = is_a ? &maps.a : &maps.b;
      const int left = RAGGED ? t.rows % A.chunk : 0;
      const int tail_at = RAGGED && left ? tail_of<LONG>(all) : -1;
      for (int c = c_begin; c < c_end; ++c) {  // (c: the place in the ring's order)
        if (!free && !bar_wait(empty(s), phase, abort_flag)) { ok = false; break; }
        // rows of the next group come along with the last chunk: this CTA's clearing warp sees them first
        const bool last_rows = RAGGED && c == tail_at;
        const int k0 = (last_rows ? all - 1 : RAGGED && tail_at >= 0 && c > tail_at ? c - 1 : c) * A.chunk;
        const int k = RAGGED ? t.row0 + k0 : k0;
        const uint32_t bar = last_rows ? tail(s) : first_full + 8 * s, dst = ring + s * stage_bytes + (is_a ? 0 : MM_OPERAND);
        if (one) {
          if (is_a && last_rows) bar_expect(tail(s), stage_bytes);
          const bool opens = is_a && (LONG ? ((c - c_begin) & (MM_STRETCH - 1)) == 0 : c == c_begin);
          if (opens) {  // a stretch, to the MMA role a tile of its own
            abort_flag[1] = (int)g;
            const int n = LONG ? min(MM_STRETCH, c_end - c) : c_end - c;
            info[2 * s] = t.n | (RAGGED && c + n == c_end ? (left + 15) / 16 << TILE_STEPS : 0);
            info[2 * s + 1] = n;
          }
          if (is_a && rank == 0) {
            bar_expect(full(s), last_rows ? 0 : 2 * stage_bytes);
          }
          if (DUAL && is_a) {
            load_5d(dst, map, k0, 0, 0, at / 8, z, bar);
          } else if (rows_inner) {
            load_3d(dst, map, at, k, z, bar);
            load_3d(dst + MM_OPERAND / 2, map, at + 64, k, z, bar);
          } else {
            load_3d(dst, map, k, at, z, bar);
          }
        }
        __syncwarp();
        ++g;
        if (++s == stages) {
          s = 0;
          phase ^= 1u;
        }
        free = bar_try(empty(s), phase);
      }
    }
    if (ok && is_a) {  // the end of the list, to the MMA role
      ok = free || bar_wait(empty(s), phase, abort_flag);
      if (ok && rank == 0 && one) {
        info[2 * s] = TILE_END;
        bar_expect(full(s), 0);
      }
      __syncwarp();
      // the last commits must have arrived here before this CTA may end
#pragma unroll 1
      for (uint32_t d = g > stages ? g - stages : 0; ok && d < g; ++d) ok = bar_wait(empty(d % stages), (d / stages) & 1u, abort_flag);
    }
  } else if (warp == MM_WARP_MMA) {
    // ============================================================ MMAs, by the pair's first CTA
    // The issue of a chunk has to fit the 512 cycles of its MMAs, fewer for narrow tiles, so its loop does nothing else.  The whole
    // warp walks it, so that descriptors are warp-uniform values, and one elected thread issues; the next stage is asked for before
    // this one's MMAs are issued; what a tile is the copy role has written beside its first stage.
    if (rank == 0) {
      const bool one = elected();
      const uint64_t da = operand_desc(ring, AT ? MM_OPERAND / 2 : 16, 1024);
      const uint64_t db = operand_desc(ring + MM_OPERAND, BT ? MM_OPERAND / 2 : 16, 1024);
      // fp32 sums of bf16 (or e4m3: type 0) values, 256 rows, both CTAs
      const uint32_t kind = 1u << 4 | (FP8 ? 0u : (1u << 7 | 1u << 10)) | (AT ? 1u << 15 : 0u) | (BT ? 1u << 16 : 0u) | (MM_M >> 4) << 24;
      uint32_t s = 0, phase = 0, a = 0, idesc = 0, d = tmem, cleared_phase = 0;
      auto issue = [&](uint32_t stage, int steps, uint32_t add) {
        if (one) {
          const uint64_t pa = da + (stage * stage_bytes >> 4), pb = db + (stage * stage_bytes >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k)  // 32 bytes of k; rows inner: 16 k's, two blocks of 1024 bytes
            if (!RAGGED || k < steps)
              mma_pair<FP8>(d, pa + (k * (AT ? 2048 : 32) >> 4), pb + (k * (BT ? 2048 : 32) >> 4), idesc, k == 0 ? add : 1u);
          commit_pair(empty(stage));
        }
        __syncwarp();
      };
      bool ready = bar_try(full(0), 0), ok = true;
      while (ok) {
        if (!ready && !bar_wait(full(s), phase, abort_flag)) break;
        const uint32_t what = *(volatile uint32_t*)(info + 2 * s), chunks = *(volatile uint32_t*)(info + 2 * s + 1);
        if (what & TILE_END) break;
        // a chunk to be cleared first comes MM_TAIL_LEAD places before the tile's end, but is taken last
        const int tail_steps = RAGGED ? what >> TILE_STEPS : 0;
        const uint32_t tail_at = RAGGED && tail_steps ? tail_place(chunks) : ~0u;
        uint32_t tail_stage = 0, add = 0;
        idesc = kind | (what & 0x1ffu) >> 3 << 17;
        d = tmem + (a & 1u) * MM_N;
        if (!bar_wait(acc_empty(a & 1u), ((a >> 1) & 1u) ^ 1u, abort_flag)) break;
        tc_after();
        for (uint32_t c = 0; c < chunks; ++c) {
          if (c > 0 && !ready && !bar_wait(full(s), phase, abort_flag)) { ok = false; break; }
          const uint32_t stage = s;
          if (++s == stages) {
            s = 0;
            phase ^= 1u;
          }
          ready = bar_try(full(s), phase);
          if (RAGGED && c == tail_at) {
            tail_stage = stage;
            continue;
          }
          issue(stage, 4, add);
          add = 1;
        }
        if (RAGGED && ok && tail_steps) {
          if (!bar_wait(cleared(tail_stage), (cleared_phase >> tail_stage) & 1u, abort_flag)) break;
          cleared_phase ^= 1u << tail_stage;
          tc_after();
          issue(tail_stage, tail_steps, add);
        }
        if (ok && one) commit_pair(acc_full(a & 1u));
        __syncwarp();
        ++a;
      }
    }
  } else if (warp == MM_WARP_CLEAR) {
    // ============================================================ rows behind a group's end
    if constexpr (RAGGED) {
      uint32_t g = 0, parity = 0;  // bit s: of the next use of tail(s)
      for (int it = pair; it < tiles; it += pairs) {
        const Tile t = tile_at(it);
        const int chunks = chunks_of(t), left = t.rows % A.chunk;
        const int s = (g + tail_of<LONG>(chunks)) % stages;
        g += chunks;
        if (left == 0) continue;
        int ok = lane == 0 ? bar_wait(tail(s), (parity >> s) & 1u, abort_flag) : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        parity ^= 1u << s;
        unsigned char* st = smem + (size_t)s * stage_bytes;
        const int to = (left + 15) / 16 * 128;  // 16-byte pieces of a box's rows of 128 bytes, up to a step of 16 rows
        for (int b = 0; b < 4; ++b)
          for (int i = left * 8 + lane; i < to; i += 32) *reinterpret_cast<uint4*>(st + b * (MM_OPERAND / 2) + i * 16) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_first(cleared(s)));  // both CTAs' parts
      }
    }
  } else {
    // ============================================================ epilogue
    // A warp by itself: its 32 lanes of the accumulator are 32 columns of the output (DUAL: 16 features), which it turns through its own
    // buffer, 32 rows at a time.  The warps of a team share a step's rows; the teams take steps in turn.
    if constexpr (EPI == ME_STORE_ROWS) {
      // The accumulator's lanes are rows of the output and its columns the row's: nothing to turn.  A warp packs 64 columns of its 32
      // rows into its swizzled buffer and TMA takes them from there, whole lines of 128 bytes, cut at the matrix's edges.
      uint32_t a = 0;
      const uint32_t at = smem_u32(staging) + warp * 4096;
      static_assert(MM_TEAMS * 4 * 4096 <= MM_STAGING, "buffers of 32 rows of 128 bytes");
      const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
      const int team = warp >> 2;
      for (int it = pair; it < tiles; it += pairs) {
        const Tile t = tile_at(it);
        const bool none = t.rows == 0;  // a group without rows: zeros
        if constexpr (LONG) {
          a = join_stretches<MM_ROW_STEP>(a, chunks_in(it, t), lane_base, t.n, A.sums, acc_full(0), acc_empty(0), abort_flag);
          if (a == ~0u) break;
        }
        const uint32_t buf = a & 1u;
        if (!none) {
          const int w = lane == 0 ? bar_wait(acc_full(buf), (a >> 1) & 1u, abort_flag) : 0;
          if (__shfl_sync(0xffffffffu, w, 0) == 0) break;
          tc_after();
          ++a;
        }
        auto release = [&] {  // this warp has read its part of the accumulator
          tc_before();
          __syncwarp();
          if (lane == 0) bar_arrive_cluster(in_first(acc_empty(buf)));
        };
        if (!none && team * MM_ROW_STEP >= t.n) release();
        const int row = t.m0 + (int)rank * (MM_M / 2) + (warp & 3) * 32;
        for (int c0 = team * MM_ROW_STEP; c0 < t.n; c0 += MM_TEAMS * MM_ROW_STEP) {
          uint32_t r[2][MM_STEP];
          if (none) {
#pragma unroll
            for (int i = 0; i < MM_STEP; ++i) r[0][i] = r[1][i] = 0;
          } else {
            tmem_load(lane_base + buf * MM_N + c0, r[0]);
            tmem_load(lane_base + buf * MM_N + c0 + MM_STEP, r[1]);
            tmem_load_wait();
            if (c0 + MM_TEAMS * MM_ROW_STEP >= t.n) release();
          }
          asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // (lane 0's: its last store has read the buffer)
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i) {  // 16 bytes of the row's 128; the swizzle: piece ^ row mod 8
            uint32_t p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int k = 8 * (i & 3) + 2 * j;
              const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(r[i >> 2][k]), __uint_as_float(r[i >> 2][k + 1]));
              p[j] = *reinterpret_cast<const uint32_t*>(&v);
            }
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                         ::"r"(at + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3]) : "memory");
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (row < A.M) store_3d(&maps.out, at, t.n0 + c0, row, t.group);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        }
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else {
    if (EPI == ME_SWIGLU_GRAD) pdl_wait();
    uint32_t a = 0;
    bool ok = true;
    const int team = warp >> 2;
    float* const st = staging + warp * (MM_STEP * MM_PITCH);
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    // A thread's part of a step: rows c, c + ITEM_ROWS, ... and 8 columns (DUAL: 8 features).
    constexpr int ITEMS = DUAL ? 2 : 4, ITEM_ROWS = MM_STEP / ITEMS;
    constexpr int OUT_BYTES = EPI == ME_STORE_F32 || SPLIT ? 4 : 2;
    const int q = DUAL ? lane & 1 : lane & 3, c = DUAL ? lane >> 1 : lane >> 2;
    const int64_t out_step = A.os * (ITEM_ROWS * OUT_BYTES);
    const float* const mine = st + c * MM_PITCH + q * (DUAL ? 16 : 8);
    for (int it = pair; ok && it < tiles; it += pairs) {
      const Tile t = tile_at(it);
      if constexpr (LONG) {
        a = join_stretches<MM_STEP>(a, chunks_in(it, t), lane_base, t.n, A.sums, acc_full(0), acc_empty(0), abort_flag);
        if (a == ~0u) break;
      }
      const uint32_t buf = a & 1u;
      const int m = t.m0 + (int)rank * (M_STEP / 2) + (warp & 3) * (M_STEP / 8) + q * 8, n = min(8, A.M - m);
      const int valid = n > 0 ? t.valid : 0;
      const int64_t row0 = t.n0 + team * MM_STEP + c;
      char* out = reinterpret_cast<char*>(A.out) + ((SPLIT ? (int64_t)(it % A.splits) * A.out_group : 0) +
                                                           row0 * A.os + (EPI == ME_PART_DUAL ? 2 : 1) * m) * OUT_BYTES;
      // rows of dh, residual or dout of this thread's items, and x's scales
      const void* const from = EPI == ME_SWIGLU_GRAD ? (const void*)A.dh : EPI == ME_PRODUCT ? A.residual : EPI == ME_PRODUCT_GRAD ? A.dout : nullptr;
      const int64_t in_stride = EPI == ME_SWIGLU_GRAD ? (int64_t)A.f * 4 : A.rs * 2;
      const char* in = reinterpret_cast<const char*>(from) + row0 * in_stride + (int64_t)m * (EPI == ME_SWIGLU_GRAD ? 4 : 2);
      const float* xs = FP8 ? A.x_scale + row0 : nullptr;
      const bool wide_in = EPI == ME_SWIGLU_GRAD || (from && A.wide_in && n == 8);
      auto ask = [&](int at, Ahead& w) {  // `at`: column of the thread's first item
        if constexpr (EPI == ME_SWIGLU_GRAD || EPI == ME_PRODUCT || EPI == ME_PRODUCT_GRAD) {
          const char* p = in;
#pragma unroll
          for (int i = 0; i < ITEMS; ++i, p += in_stride * ITEM_ROWS)
            if (at + i * ITEM_ROWS < valid) {
              if constexpr (EPI == ME_SWIGLU_GRAD) {
                w.v[2 * i] = reinterpret_cast<const uint4*>(p)[0];
                w.v[2 * i + 1] = reinterpret_cast<const uint4*>(p)[1];
              } else if (wide_in) {
                w.v[i] = load_once<__nv_bfloat16, 8>(reinterpret_cast<const __nv_bfloat16*>(p)).r;
              }
              if constexpr (FP8) w.scale[i] = xs[i * ITEM_ROWS];
            }
          in += in_stride * (MM_TEAMS * MM_STEP);
          if constexpr (FP8) xs += MM_TEAMS * MM_STEP;
        }
      };
      float bias[8], scale[8], sums[8];  // of this thread's columns of the output
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sums[j] = bias[j] = 0.f;
        if constexpr (EPI == ME_PRODUCT || EPI == ME_PRODUCT_GRAD)
          if (A.bias && j < n) bias[j] = gain(A.bias, A.bias_f32, m + j);
        if constexpr (EPI == ME_PRODUCT && FP8) scale[j] = j < n ? A.w_scale[m + j] : 0.f;
      }
      float lane_bias = 0.f, lane_scale = 0.f;
      const bool odd_rows = EPI == ME_PRODUCT && (!A.wide || (from && !A.wide_in));
      if (odd_rows) {
        const int col = t.m0 + (int)rank * (M_STEP / 2) + (warp & 3) * 32 + lane;
        if (A.bias && col < A.M) lane_bias = gain(A.bias, A.bias_f32, col);
        if (FP8 && col < A.M) lane_scale = A.w_scale[col];
      }
      // The same where a lane keeps its column: 16 rows of it, from row c0 of the tile on, a register each (packing them would wait for
      // them).  `now` holds a step's first half, `next` its second.
      auto ask_odd = [&](int c0, Ahead& w) {
        const int col = t.m0 + (int)rank * (M_STEP / 2) + (warp & 3) * 32 + lane;
        if (!from || col >= A.M) return;
        const uint16_t* p = reinterpret_cast<const uint16_t*>(from) + (int64_t)(t.n0 + c0) * A.rs + col;
        uint32_t v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i, p += A.rs)
          if (c0 + i < t.valid) v[i] = *p;
#pragma unroll
        for (int i = 0; i < 4; ++i) w.v[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      };
      auto row_scales = [&](int c0) { return FP8 && c0 + lane < t.valid ? A.x_scale[t.n0 + c0 + lane] : 0.f; };
      float scale_now = 0.f, scale_next = 0.f;
      Ahead now, next;
      if (EPI == ME_PRODUCT && odd_rows) {
        ask_odd(team * MM_STEP, now);
        scale_now = row_scales(team * MM_STEP);
      } else {
        ask(team * MM_STEP + c, now);
      }
      const int w = lane == 0 ? bar_wait(acc_full(buf), (a >> 1) & 1u, abort_flag) : 0;
      ok = __shfl_sync(0xffffffffu, w, 0) != 0;
      if (!ok) break;
      tc_after();
      ++a;
      auto release = [&] {  // this warp has read its part of the accumulator
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_first(acc_empty(buf)));
      };
      if (team * MM_STEP >= t.n) release();
      for (int c0 = team * MM_STEP; c0 < t.n; c0 += MM_TEAMS * MM_STEP) {
        uint32_t r[MM_STEP];
        tmem_load(lane_base + buf * MM_N + c0, r);
        if (EPI == ME_PRODUCT && odd_rows) {
          ask_odd(c0 + 16, next);
          scale_next = row_scales(c0 + MM_TEAMS * MM_STEP);  // (past the tile's end: nothing)
        } else {
          ask(c0 + MM_TEAMS * MM_STEP + c, next);
        }
        tmem_load_wait();
        if (c0 + MM_TEAMS * MM_STEP >= t.n) release();
#pragma unroll
        for (int i = 0; i < MM_STEP; ++i) st[i * MM_PITCH + lane] = __uint_as_float(r[i]);
        __syncwarp();
        if constexpr (EPI == ME_PRODUCT) {
          if (odd_rows) {
            // Rows off 16-byte boundaries (an odd number of outputs): a lane keeps its column, and a row's 32 values go as 64 bytes of
            // 32 lanes (eight values a lane, one by one, are 32 pieces a store: 7288 x 880 x 6971 278 us, 92 so; with GeLU and residual 329, 233).
            const int col = t.m0 + (int)rank * (M_STEP / 2) + (warp & 3) * 32 + lane, rows = col < A.M ? min(MM_STEP, t.valid - c0) : 0;
            if (FP8 || A.bias || A.act != DEAMOE_SIGMA_NONE) {
#pragma unroll 4
              for (int i = 0; i < MM_STEP; ++i) {
                float v = st[i * MM_PITCH + lane];
                v = FP8 ? fmaf(v, __shfl_sync(0xffffffffu, scale_now, i) * lane_scale, lane_bias) : v + lane_bias;
                if (A.act != DEAMOE_SIGMA_NONE) v = A.act == DEAMOE_SIGMA_SILU ? v * sigmoid(v) : sigma_f(DEAMOE_SIGMA_GELU, v);
                st[i * MM_PITCH + lane] = v;
              }
            }
            __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(A.out) + (int64_t)(t.n0 + c0) * A.os + col;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const Ahead& w = h ? next : now;
              const uint32_t add[16] = {w.v[0].x, w.v[0].y, w.v[0].z, w.v[0].w, w.v[1].x, w.v[1].y, w.v[1].z, w.v[1].w,
                                        w.v[2].x, w.v[2].y, w.v[2].z, w.v[2].w, w.v[3].x, w.v[3].y, w.v[3].z, w.v[3].w};
#pragma unroll
              for (int i = 0; i < 16; ++i, to += A.os)
                if (16 * h + i < rows) {
                  float v = st[(16 * h + i) * MM_PITCH + lane];
                  if (from) v += __uint_as_float(add[i] << 16);
                  *to = __float2bfloat16_rn(v);
                }
              if (h == 0) ask_odd(c0 + MM_TEAMS * MM_STEP, now);
            }
            scale_now = scale_next;
            __syncwarp();
            continue;
          }
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i, out += out_step) {
          if (c0 + i * ITEM_ROWS + c >= valid) continue;
          const float* from_st = mine + i * (ITEM_ROWS * MM_PITCH);
          __nv_bfloat16* const to = reinterpret_cast<__nv_bfloat16*>(out);
          float v[8];
          floats8(from_st, v);
          if constexpr (DUAL) {  // (f is a multiple of 8)
            float up[8];
            floats8(from_st + 8, up);
            if constexpr (EPI == ME_PART_DUAL) {
              put8(reinterpret_cast<float*>(out), v);
              put8(reinterpret_cast<float*>(out) + 8, up);
            } else if constexpr (EPI == ME_SWIGLU) {
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] *= sigmoid(v[j]) * up[j];
              put8(to, v, 8, true);
            } else {
              const uint32_t d[8] = {now.v[2 * i].x, now.v[2 * i].y, now.v[2 * i].z, now.v[2 * i].w,
                                     now.v[2 * i + 1].x, now.v[2 * i + 1].y, now.v[2 * i + 1].z, now.v[2 * i + 1].w};
              float dg[8], du[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const float p = sigmoid(v[j]), act = v[j] * p, dh = __uint_as_float(d[j]);
                du[j] = dh * act;
                dg[j] = dh * up[j] * (p * (1.f + v[j] * (1.f - p)));
                v[j] = act * up[j];
              }
              put8(to, dg, 8, true);
              put8(to + A.f, du, 8, true);
              put8(reinterpret_cast<__nv_bfloat16*>(A.h_out) + (row0 + c0 - team * MM_STEP + i * ITEM_ROWS) * A.f + m, v, 8, true);
            }
          } else if constexpr (EPI == ME_STORE_F32 || EPI == ME_PART) {
            put8(reinterpret_cast<float*>(out), v);  // (rows of fp32 outputs have room for whole groups of 8)
          } else {
            if constexpr (EPI == ME_PRODUCT || EPI == ME_PRODUCT_GRAD) {
              float add[8];
              if (wide_in) {
                Pack<__nv_bfloat16, 8> w;
                w.r = now.v[i];
                w.widen(add);
              } else if (from) {
                get8(reinterpret_cast<const __nv_bfloat16*>(from) + (row0 + c0 - team * MM_STEP + i * ITEM_ROWS) * A.rs + m, add, n);
              }
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = FP8 ? fmaf(v[j], now.scale[i] * scale[j], bias[j]) : v[j] + bias[j];
              if constexpr (EPI == ME_PRODUCT) {
                if (A.act != DEAMOE_SIGMA_NONE) {
#pragma unroll
                  for (int j = 0; j < 8; ++j) v[j] = A.act == DEAMOE_SIGMA_SILU ? v[j] * sigmoid(v[j]) : sigma_f(DEAMOE_SIGMA_GELU, v[j]);
                }
                if (from) {
#pragma unroll
                  for (int j = 0; j < 8; ++j) v[j] += add[j];
                }
              } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  v[j] = add[j] * act_grad(A.act, v[j]);
                  sums[j] += v[j];
                }
              }
            }
            put8(to, v, EPI == ME_STORE ? 8 : n, EPI == ME_STORE || A.wide);  // (ME_STORE: whole groups of 8)
          }
        }
        out += ITEMS * (MM_TEAMS - 1) * out_step;
        now = next;
        __syncwarp();
      }
      if constexpr (EPI == ME_PRODUCT_GRAD) {
        if (A.part) {  // 8 lanes hold sums of the same columns: added in a fixed order
#pragma unroll
          for (int o = 4; o < 32; o *= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[j] += __shfl_xor_sync(0xffffffffu, sums[j], o);
          if (c == 0)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (j < n) A.part[(int64_t)(MM_TEAMS * t.n_index + team) * A.M + m + j] = sums[j];
        }
      }
    }
    }
  }

  // common end, also after a wait that has expired
  if (A.late) pdl_wait();
  tc_before();
  __syncthreads();
  if (*abort_flag) {
    if (tid == 0) mm_status = DEAMOE_ERR_TIMEOUT;
#pragma unroll 1
    for (int i = 0; i < 64; ++i) __nanosleep(1000);  // copies in flight land before the shared memory is given back
  }
  cluster_sync();
  if (warp == MM_WARP_MMA) {
    tc_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ---------------------------------------------------------------- host
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
  static std::atomic<EncodeFn> found{nullptr};
  EncodeFn f = found.load(std::memory_order_acquire);
  if (!f) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    f = reinterpret_cast<EncodeFn>(p);
    found.store(f, std::memory_order_release);
  }
  return f;
}
bool encode(CUtensorMap* m, const void* p, int esize, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  EncodeFn f = encode_fn();
  if (!f) return false;
  const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
  return f(m, esize == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(p), dims, strides, box,
           ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int EPI, bool AT, bool BT, bool FP8, bool RAGGED, bool LONG>
cudaError_t launch_form(const MatmulCall& c, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  auto kernel = k_matmul<EPI, AT, BT, FP8, RAGGED, LONG>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!(done.load(std::memory_order_acquire) >> dev & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MM_SMEM);
    if (e != cudaSuccess) return e;
    done.fetch_or(1ull << dev, std::memory_order_release);
  }
  // no more pairs than there can be tiles, whatever the offsets
  const MatmulArgs& a = c.args;
  constexpr int m_step = EPI == ME_SWIGLU || EPI == ME_SWIGLU_GRAD || EPI == ME_PART_DUAL ? MM_M / 2 : MM_M;
  const int64_t mt = (a.M + m_step - 1) / m_step;
  const int64_t nt = RAGGED ? (int64_t)a.groups * ((a.N + a.tile_n - 1) / a.tile_n) : a.N / a.tile_n + (a.groups < a.N ? a.groups : a.N);
  const int64_t most = mt * nt * a.splits;
  const dim3 grid(2 * (unsigned)(most < MM_PAIRS ? most : MM_PAIRS));
  return launch_pdl(kernel, grid, dim3(MM_THREADS), MM_SMEM, s, c.args, c.maps);
}
template <int EPI, bool AT, bool BT, bool FP8, bool RAGGED>
cudaError_t launch(const MatmulCall& c, cudaStream_t s) {
  const MatmulArgs& a = c.args;
  if (!matmul_sums(a.K, a.chunk, a.splits)) return launch_form<EPI, AT, BT, FP8, RAGGED, false>(c, s);
  return a.sums ? launch_form<EPI, AT, BT, FP8, RAGGED, true>(c, s) : cudaErrorInvalidValue;
}

}  // namespace

bool map_rows(CUtensorMap* m, const void* p, int esize, int64_t cols, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride,
              int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)groups};
  const cuuint64_t strides[2] = {(cuuint64_t)stride * esize, (cuuint64_t)group_stride * esize};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / esize), (cuuint32_t)box_rows, 1};
  return encode(m, p, esize, 3, dims, strides, box);
}
bool map_gate_up(CUtensorMap* m, const void* p, int64_t cols, int64_t f, int64_t groups) {
  const cuuint64_t dims[5] = {(cuuint64_t)cols, 8, 2, (cuuint64_t)f / 8, (cuuint64_t)groups};
  const cuuint64_t strides[4] = {(cuuint64_t)cols * 2, (cuuint64_t)(f * cols) * 2, (cuuint64_t)cols * 16, (cuuint64_t)(f * cols) * 4};
  const cuuint32_t box[5] = {64, 8, 2, 8, 1};
  return encode(m, p, 2, 5, dims, strides, box);
}
bool map_out(MatmulCall* c, const void* p, int64_t cols, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)groups};
  const cuuint64_t strides[2] = {(cuuint64_t)stride * 2, (cuuint64_t)group_stride * 2};
  const cuuint32_t box[3] = {64, 32, 1};
  return encode(&c->maps.out, p, 2, 3, dims, strides, box);
}
bool map_b(MatmulCall* c, const void* p, int esize, int64_t cols, int64_t rows, int64_t stride) {
  // the lowest box (16, 32, 64 or 128 rows) that holds a CTA's half of the widest tile: one copy a chunk, and what the box does not
  // need of a stage goes to more stages
  const int half = (c->args.tile_n + 15) / 16 * 8;
  int box = 16;
  while (box < half) box *= 2;
  c->args.b_bytes = box * 128;
  c->args.stages = MM_RING / (MM_OPERAND + c->args.b_bytes);
  return map_rows(&c->maps.b, p, esize, cols, rows, stride, 1, stride, box);
}
bool map_b_rows_inner(MatmulCall* c, const void* p, int64_t cols, int64_t rows, int64_t stride) {
  c->args.b_bytes = MM_OPERAND;
  c->args.stages = MM_RING / (2 * MM_OPERAND);
  return map_rows(&c->maps.b, p, 2, cols, rows, stride, 1, stride, 64);
}
int matmul_group_tile_n(int64_t rows, int64_t groups) {
  const int64_t each = (rows + groups - 1) / groups;
  int n = 32;
  while (n < MM_N && (n < 4 * each || n < rows / 32)) n *= 2;
  return n;
}

// The pairs take the tiles in rounds, and a round costs a tile's width and some 100 columns more (2048 x 4096 x 4096: rounds of
// 144, 240 and 256 columns 21, 28 and 30 us), so a narrower tile pays where it saves a part of the last round: 3000 x
// 2000 x 4096 in 18 tiles of 176 48 us, in 12 of 256 57; 1024 x 7168 x 7168 in 5 of 208 98 us, in 4 of 256 107.  Up to 256
// rows A's bytes bound a product that can be split along k, so it reads them once (`whole`).
int matmul_tile_n(int64_t n, int64_t m_tiles, bool whole) {
  int best = MM_N;
  int64_t least = INT64_MAX;
  for (int64_t nt = (n + MM_N - 1) / MM_N, k = 0; k < (whole && n <= MM_N ? 1 : 8); ++nt, ++k) {
    const int64_t width = ((n + nt - 1) / nt + 15) / 16 * 16;
    if (k > 0 && width < MM_N_LEAST) break;
    const int64_t cost = (nt * m_tiles + MM_PAIRS - 1) / MM_PAIRS * (width + 100);
    if (cost < least) {
      least = cost;
      best = (int)width;
    }
  }
  return best;
}
// A decode step's product has fewer tiles than the device has pairs (7168 outputs: 28), and so has one of few outputs: its tiles are
// dealt along k, as evenly over the pairs as some number of parts allows.  In us: a chunk takes a pair some 0.3, a part's sums (4
// bytes a value) are written and read at what is taken as 4 TB/s, mostly in the L2, and joining them takes 3 more.
int matmul_splits(int64_t tiles, int64_t chunks, int64_t rows, int64_t outputs) {
  int best = 1;
  double least = 0.9 * 0.3 * (double)((tiles + MM_PAIRS - 1) / MM_PAIRS) * (double)(chunks + 2);
  for (int s = 2; s <= 16 && s * 4 <= chunks; ++s) {
    const double cost = 0.3 * (double)((tiles * s + MM_PAIRS - 1) / MM_PAIRS) * (double)((chunks + s - 1) / s + 2) + 3 +
                        (double)s * (double)rows * (double)outputs * 8 / 4e6;
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

cudaError_t matmul_launch(MatmulForm form, const MatmulCall& c, cudaStream_t s) {
  switch (form) {
    case MF_SWIGLU: return launch<ME_SWIGLU, false, false, false, false>(c, s);
    case MF_STORE: return launch<ME_STORE, false, false, false, false>(c, s);
    case MF_STORE_TRANSPOSED: return launch<ME_STORE, true, false, false, false>(c, s);
    case MF_F32_TRANSPOSED: return launch<ME_STORE_F32, true, false, false, false>(c, s);
    case MF_SWIGLU_GRAD: return launch<ME_SWIGLU_GRAD, false, false, false, false>(c, s);
    case MF_WEIGHT_GRAD: return launch<ME_STORE_ROWS, true, true, false, true>(c, s);
    case MF_PRODUCT: return launch<ME_PRODUCT, false, false, false, false>(c, s);
    case MF_PRODUCT_E4M3: return launch<ME_PRODUCT, false, false, true, false>(c, s);
    case MF_PART: return launch<ME_PART, false, false, false, false>(c, s);
    case MF_PART_E4M3: return launch<ME_PART, false, false, true, false>(c, s);
    case MF_PART_SWIGLU: return launch<ME_PART_DUAL, false, false, false, false>(c, s);
    case MF_PRODUCT_GRAD: return launch<ME_PRODUCT_GRAD, false, false, false, false>(c, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace deamoe

using namespace deamoe;

extern "C" deamoe_status_t deamoe_operator_status(void* cuda_stream, int32_t* status) {
  if (!status) return DEAMOE_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  int32_t got = 0;
  void* word = nullptr;
  if (cudaGetSymbolAddress(&word, mm_status) != cudaSuccess || cudaMemcpyAsync(&got, word, 4, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaMemsetAsync(word, 0, 4, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
    cudaGetLastError();
    return DEAMOE_ERR_CUDA;
  }
  *status = got;
  return DEAMOE_OK;
}
