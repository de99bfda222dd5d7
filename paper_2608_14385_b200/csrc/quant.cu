// Products with 4-bit matrices of group scales: out[r] = W[e(r)] x[src(r)], optionally through SwiGLU.
//
//   W[i, c] = s[i, c / G] (q[i, c] - z[i, c / G])   =>   (W x)[i] = sum_g s[i, g] sum_{c in g} (q - z) x[c]
//
// so the group scale multiplies an fp32 sum and no weight is ever rounded.  A decode step has a few rows per matrix:
// the codes (half a byte a weight, read once) bound it, and the work beside them is to widen 2 weights a byte.
// Measured: the gate and up matrices (4096 x 7168, groups of 128) of 16 tokens' top-8 of 256 experts, 93 of them active
// (1.4 GB), in 308 us (4.6 TB/s; fp32 tokens 591), of one token's 8 experts in 39 us (3.1 TB/s; 62), one matrix in 11 us
// (14).  Back to back for seconds the first takes a tenth longer: the power limit then holds the clock near 1.75 GHz.  No
// unit is full (issue 56 %, DRAM 52 %, tensor pipe 26 %): four warps a scheduler, which 128 registers a thread allow, do
// not hide the latency of their loads of x and of their own widening.
//
// Tensor cores: mma.m16n8k16 with 16 matrix rows as M and up to 8 tokens as N (legacy path: with this few tokens the
// instruction rate it needs is a fraction of what it has, and its A operand comes from registers, where the codes
// have to be widened anyway).  Widening is a shift, a logical operation and a subtraction a pair: a nibble under the
// exponent of 128 is the bf16 number 128 + q, and 128 + z leaves q - z, exactly (the magic-number conversion of Kim et
// al., 2022, arXiv 2211.10017, there for fp16).  bf16 because x has to stay what it is: bf16 tokens are operands as they
// are, fp32 tokens as three bf16 parts of 8 bits each, which add up to the value.  (As fp16 operands, with a power of two
// a row to bring x into fp16's range and fp32 in two parts, the codes' odd nibbles need no shift and fp32 two thirds of the
// products: 295 us, fp32 468.  But what is 2^-28 of its row's largest value loses bits there, fp32 values from 2^-11 on,
// and that shows where the large value meets a weight of 0.)
#include <atomic>
#include <climits>

#include "row.cuh"

namespace deamoe {

constexpr int QW = 8;        // warps of a block
constexpr int QCOLS = 256;   // columns of a step: 128 bytes of a row
constexpr int QM = QCOLS / 32;  // its parts of 32 columns: two matrix instructions
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
  int vec_scales, vec_zeros;  // a step's scales / zero points of a row can be read as one vector
  int steps;        // column steps of a row
  int wk;           // warps that share a row tile's columns (the others of the block take other tiles)
  int tile_groups;  // blocks of QW / wk warp tiles (16 MT rows) a matrix
  uint16_t* xb;     // [n_rows][planes][steps * QCOLS] bf16
  float* xf;        // [n_rows] factor of the row's products
};

// eight values of a row from column col on, 0 past its end
template <typename T> static __device__ __forceinline__ void eight_of(const T* x, int col, int n_in, bool wide, float (&v)[8]) {
  constexpr int VE = 16 / sizeof(T);
  if (wide && col + 8 <= n_in) {
#pragma unroll
    for (int i = 0; i < 8 / VE; ++i) {
      float f[VE];
      load_pack<T, VE>(x + col + i * VE).widen(f);
#pragma unroll
      for (int k = 0; k < VE; ++k) v[i * VE + k] = f[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < n_in ? to_f<T>(x[col + i]) : 0.f;
  }
}
// the bf16 number of v's sign, exponent and top 8 bits (a NaN stays one)
static __device__ __forceinline__ float top_bits(float v) {
  return __uint_as_float(v == v ? __float_as_uint(v) & 0xffff0000u : 0x7fc00000u);
}
// x in the order of the rows, as bf16 parts that add up to the value (fp32: three, each the top 8 bits of what is left, so
// that no part can round to infinity), 8 columns in the order 0 4 1 5 2 6 3 7 (the order in which the codes of a 32-bit
// word are widened).  One block a row; a row without a source is zero.
// A group's sum of (q - z) x comes before its scale: rows with a value of 2^96 or more are carried times 2^-32, so that the
// sum (below 2^24 times the value) overflows no earlier than the scaled products do.  fp32 rows below 2^-64 are carried
// times 2^24, because a part below 2^-133 is no bf16 number: beside larger ones, that is where a value's bits end.
template <typename T, int PLANES> __global__ void __launch_bounds__(1024) k_quant_x(QuantArgs A, bool wide) {
  const int64_t r = blockIdx.x;
  int64_t src = r;
  if (A.row_pair) src = A.row_pair[r] >= 0 ? A.row_pair[r] / A.ppt : -1;
  const bool have = src >= 0 && src < A.n_token;
  const T* x = reinterpret_cast<const T*>(A.x) + (have ? src : 0) * A.xs;
  pdl_trigger();
  const int width = A.steps * QCOLS;
  float v[8] = {};  // the thread's first eight columns (all of them up to 8192 columns); later ones are read twice
  bool huge = false, tiny = true;
  for (int c = threadIdx.x; have && c < width / 8; c += blockDim.x) {
    float u[8];
    eight_of<T>(x, c * 8, A.n_in, wide, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float m = fabsf(u[i]);
      huge |= m >= 0x1p96f && m <= 0x1.fffffep127f;  // infinities and NaN stay what they are
      tiny &= !(m >= 0x1p-64f && m <= 0x1.fffffep127f);
      if (c == (int)threadIdx.x) v[i] = u[i];
    }
  }
  huge = __syncthreads_or(huge);
  if constexpr (PLANES > 1) tiny = __syncthreads_and(tiny);
  const float f = huge ? 0x1p-32f : PLANES > 1 && tiny ? 0x1p24f : 1.f;
  if (threadIdx.x == 0) A.xf[r] = 1.f / f;
  uint16_t* out = A.xb + r * PLANES * width;
  for (int c = threadIdx.x; c < width / 8; c += blockDim.x) {
    if (c != (int)threadIdx.x && have) eight_of<T>(x, c * 8, A.n_in, wide, v);
    uint32_t part[PLANES][4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {  // columns p and p + 4
      float a = v[p] * f, b = v[p + 4] * f;
#pragma unroll
      for (int k = 0; k < PLANES; ++k) {
        const float ta = top_bits(a), tb = top_bits(b);
        part[k][p] = __float_as_uint(ta) >> 16 | (__float_as_uint(tb) & 0xffff0000u);
        a = isfinite(ta) ? a - ta : 0.f;
        b = isfinite(tb) ? b - tb : 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < PLANES; ++k)
      *reinterpret_cast<uint4*>(out + k * width + c * 8) = make_uint4(part[k][0], part[k][1], part[k][2], part[k][3]);
  }
}

static __device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same with a sum that starts at 0
static __device__ __forceinline__ void mma_bf16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                                     uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Half of a part (16 of its 32 columns); `first`: the sum starts at 0.
static __device__ __forceinline__ void part(float (&d)[4], const uint32_t (&lo)[4], const uint32_t (&hi)[4], const uint4& x, int half,
                                            bool first) {
  if (first) mma_bf16_first(d, lo[0], hi[0], lo[1], hi[1], x.x, x.y);
  else if (half == 0) mma_bf16(d, lo[0], hi[0], lo[1], hi[1], x.x, x.y);
  else mma_bf16(d, lo[2], hi[2], lo[3], hi[3], x.z, x.w);
}
// The 8 codes of a word less the zero point as four pairs: columns (0 4) (1 5) (2 6) (3 7).  z: 128 + the zero point in both
// halves.
static __device__ __forceinline__ uint32_t less(uint32_t a, uint32_t b) {
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
constexpr uint32_t B128 = 0x43004300u;
static __device__ __forceinline__ uint32_t pick(uint32_t w, uint32_t exponent) {  // (w & 0x000f000f) | exponent
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "r"(0x000f000fu), "r"(exponent));
  return d;
}
static __device__ __forceinline__ void widen(uint32_t w, uint32_t b128, uint32_t z, uint32_t (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = less(pick(w >> 4 * i, b128), z);
}
static __device__ __forceinline__ uint4 load_b128(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Where a warp is in the block's items: expert, group of warp tiles, pass of 16 rows (innermost: the passes of a tile
// find its codes in the caches).
struct QuantAt {
  int item, e, tg, pass, passes;
};
static __device__ __forceinline__ void quant_enter(QuantAt& at, const int* first, int tile_groups) {
  while (at.item >= first[at.e + 1]) ++at.e;
  at.passes = (first[at.e + 1] - first[at.e]) / tile_groups;
}
static __device__ __forceinline__ void quant_next(QuantAt& at, int end, const int* first, int tile_groups) {
  ++at.item;
  if (++at.pass < at.passes) return;
  at.pass = 0;
  if (++at.tg < tile_groups) return;
  at.tg = 0;
  if (at.item < end) quant_enter(at, first, tile_groups);
}

// Tokens of a pass.  fp32: what 16 need beside three parts does not fit the registers (16 tokens' top-8 of 64 experts, 4096
// x 7168: 362 us, 409 with 16 a pass; groups of 32 with zero points 578 and 667).
template <int PLANES> constexpr int TOKENS_OF_PASS = PLANES == 1 ? 16 : 8;

// A block takes a contiguous share of the items; its warps split an item's columns (wk of them a tile of 16 MT rows).
// Every warp streams its own codes, DEPTH steps of 16 MT rows x 256 columns ahead and across items, into its own part
// of shared memory; nothing is shared between warps but the sums at an item's end.
template <int PLANES, int MT, int NG, bool Z, bool SF, int DEPTH> struct QuantWarp {
  static constexpr int NTOK = TOKENS_OF_PASS<PLANES> / 8;  // of 8 tokens, in a pass
  static constexpr int NB = 2 * MT;  // blocks of 8 matrix rows in a warp tile
  // a slot of the ring: codes, then every row's scales of the step (fp32), then its zero points (bytes)
  static constexpr int SCALES = MT * 2048, ZEROS = SCALES + 16 * MT * NG * 4, STEP = (ZEROS + (Z ? 16 * MT * NG : 0) + 127) / 128 * 128;
  // Matrices narrower than a warp tile are MT = 1's; else the last tile of a matrix is moved up to its last row, so that
  // every row of every tile exists (the rows that it shares with the tile before are computed twice and written once).
  static constexpr bool NARROW = MT == 1;
  static constexpr int LM = MT == 2 ? 1 : 2;
  const QuantArgs& A;
  const int* first;
  int i1, wr, c0, c1, tiles_per, width, lane, g, j;
  uint32_t ring_at;
  size_t pair_rows, next_rows;  // matrix rows from block 2 m to block 2 m + 1, and to block 2 m + 2
  // the codes' cursor
  QuantAt ahead;
  int p_c, p_out;                // p_out: output column of row g of block 0
  const uint8_t* p_code[NB];     // this lane's 16-byte pieces of row g of the blocks
  // A lane also brings the scales and zero points of one tile row (lane; MT == 1: the first 16 lanes).  They go through
  // registers: a step's are loaded when its codes are requested and written to its slot at the request after, when
  // they have arrived
  bool held, s_exists;
  static constexpr int SW = SF ? NG : NG / 2, ZW = (NG + 3) / 4;  // words of a step's scales (SF: fp32, else bf16) and zero points
  uint32_t held_at, s_raw[SW], z_raw[ZW];
  size_t s_at;                   // index of the row's scales of the next step

  __device__ __forceinline__ QuantWarp(const QuantArgs& a, const int* f, const QuantAt& at, int end, int w, int ln, uint32_t ring)
      : A(a), first(f), i1(end), lane(ln), g(ln >> 2), j(ln & 3), ring_at(ring), ahead(at) {
    tiles_per = QW / A.wk;
    wr = w / A.wk;
    const int share = w - wr * A.wk;
    c0 = A.steps * share / A.wk;
    c1 = A.steps * (share + 1) / A.wk;
    width = A.swiglu ? A.n_out / 2 : A.n_out;
    pair_rows = A.swiglu ? width : 8;
    next_rows = A.swiglu ? 8 : 16;
    p_c = c0;
    held = false;
  }
  // output column of row g of the tile's block 0; block b adds out_of(b)
  __device__ __forceinline__ int out_at(const QuantAt& at) const {
    const int per = MT * (A.swiglu ? 8 : 16), o = (at.tg * tiles_per + wr) * per;
    return (NARROW ? o : max(min(o, width - per), 0)) + g;
  }
  __device__ __forceinline__ int out_of(int b) const { return A.swiglu ? (b >> 1) * 8 : b * 8; }
  __device__ __forceinline__ size_t rows_to(int b) const { return (b >> 1) * next_rows + (b & 1) * pair_rows; }
  __device__ __forceinline__ bool exists(int o, int b) const { return !NARROW || o + out_of(b) < width; }

  __device__ __forceinline__ void aim() {
    p_out = out_at(ahead);
    const size_t row = (size_t)ahead.e * A.n_out + p_out, half = A.n_in / 2;
#pragma unroll
    for (int b = 0; b < NB; ++b) p_code[b] = A.codes + (row + rows_to(b)) * half + (size_t)c0 * (QCOLS / 2) + j * 16;
    const int sb = lane >> 3, sr = lane & 7;
    s_exists = sb < NB && exists(p_out - g + sr, sb);
    s_at = (row - g + sr + rows_to(sb)) * A.groups + (size_t)c0 * NG;
  }
  // what the lane holds, to its slot
  __device__ __forceinline__ void flush() {
    if (!held) return;
#pragma unroll
    for (int k = 0; k < NG; k += 2) {
      const uint32_t a = SF ? s_raw[k] : s_raw[k / 2] << 16, b = SF ? s_raw[(k + 1) % SW] : s_raw[k / 2] & 0xffff0000u;
      asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(held_at + SCALES + (lane * NG + k) * 4), "r"(a), "r"(b) : "memory");
      if constexpr (Z)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(held_at + ZEROS + lane * NG + k), "h"((unsigned short)(z_raw[k / 4] >> (k & 2) * 8))
                     : "memory");
    }
    held = false;
  }
  // the next step's scales and zero points, to be held
  __device__ __forceinline__ void hold(uint32_t slot) {
    held = lane < 16 * MT;
    held_at = ring_at + slot;
    const bool have = held && s_exists;
    const int groups = have ? min(NG, A.groups - p_c * NG) : 0;  // absent ones count as 0: their codes and x are 0 too
#pragma unroll
    for (int k = 0; k < SW; ++k) s_raw[k] = 0;
#pragma unroll
    for (int k = 0; k < ZW; ++k) z_raw[k] = 0;
    const char* s = reinterpret_cast<const char*>(A.scales) + s_at * (SF ? 4 : 2);
    if (A.vec_scales) {
      if (have) {
        if constexpr (SW == 1) {
          s_raw[0] = *reinterpret_cast<const uint32_t*>(s);
        } else {
#pragma unroll
          for (int k = 0; k < SW; k += 2) {
            const uint2 v = reinterpret_cast<const uint2*>(s)[k / 2];
            s_raw[k] = v.x;
            s_raw[k + 1] = v.y;
          }
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < NG; ++k)
        if (k < groups) {
          if constexpr (SF) s_raw[k] = reinterpret_cast<const uint32_t*>(s)[k];
          else s_raw[k / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(s)[k] << (k & 1) * 16;
        }
    }
    if constexpr (Z) {
      const uint8_t* z = A.zeros + s_at;
      if (A.vec_zeros) {
        if (have) {
          if constexpr (NG == 2) {
            z_raw[0] = *reinterpret_cast<const unsigned short*>(z);
          } else {
#pragma unroll
            for (int k = 0; k < ZW; ++k) z_raw[k] = reinterpret_cast<const uint32_t*>(z)[k];
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < NG; ++k)
          if (k < groups) z_raw[k / 4] |= (uint32_t)z[k] << (k & 3) * 8;
      }
    }
    s_at += NG;
  }
  // the next step's codes into the slot at byte `slot` of the ring
  __device__ __forceinline__ void request(uint32_t slot) {
    if (ahead.item < i1) {
      const int left = A.n_in - p_c * QCOLS - j * 32;  // columns from this lane's first piece on; the other is 128 further
      const uint32_t to = ring_at + slot + g * 128 + ((j ^ g) * 16);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const bool have = exists(p_out, b);
        const uint8_t* from = have ? p_code[b] : A.codes;
        // 0 bytes: nothing is read, zeros are written
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to + b * 1024), "l"(from),
                     "r"(have && left > 0 ? 16 : 0) : "memory");
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1 + 64], 16, %2;" ::"r"((to ^ 64) + b * 1024), "l"(from),
                     "r"(have && left > 128 ? 16 : 0) : "memory");
        p_code[b] += QCOLS / 2;
      }
      flush();
      hold(slot);
      if (++p_c == c1) {
        p_c = c0;
        quant_next(ahead, i1, first, A.tile_groups);
        if (ahead.item < i1) aim();
      }
    } else {
      flush();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  // The warp's columns of one item for NT * 8 tokens: acc[mt][t] = this warp's share of the products.
  template <int NT>
  __device__ __forceinline__ void item(const QuantAt& at, int row0, int rows, uint32_t& slot, float (&acc)[MT][NTOK][4]) {
    const int xw = A.steps * QCOLS;
    // tokens past the last take the last one's values: their sums are not looked at
    const uint16_t* xp[NT];
    // parts of x ahead: it comes from the L2, whose latency a whole step (8 parts) hides (16 tokens' top-8 of 256
    // experts, 4096 x 7168 each: 308 us, 336 with 4 parts); where registers do not allow that, two
    constexpr int XB = PLANES * NT == 1 ? 8 : 2;
    uint4 xb[XB][NT][PLANES];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      xp[t] = A.xb + (size_t)(row0 + min(t * 8 + g, rows - 1)) * PLANES * xw + (size_t)c0 * QCOLS + j * 8;
#pragma unroll
      for (int p = 0; p < PLANES; ++p)
#pragma unroll
        for (int m = 0; m < XB; ++m) xb[m][t][p] = load_b128(xp[t] + (size_t)p * xw + m * 32);
    }
    uint32_t b128 = B128;
    asm volatile("" : "+r"(b128));  // in a register: an instruction has room for one constant, the mask
    // the lane's row of the eight matrices an ldmatrix takes: block lane / 8 (MT == 1: block and part)
    const uint32_t lane_at = ring_at + (MT == 2 ? (lane >> 3) : (lane >> 3) & 1) * 1024 + (lane & 7) * 128 +
                             ((lane & 7) ^ (MT == 2 ? 0 : lane >> 4)) * 16;
#pragma unroll 1
    for (int c = c0; c < c1; ++c) {
      const bool more = c + 1 < c1;
      asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
      __syncwarp();
      uint32_t code[NB * LM];  // the codes of LM parts
      const uint32_t from = lane_at + slot, scales = ring_at + slot + SCALES + g * NG * 4, zeros = ring_at + slot + ZEROS + g * NG;
      float grp[MT][NT][4], sc[NB];
      uint32_t z[NB];
#pragma unroll
      for (int m = 0; m < QM; ++m) {
        if (m * NG % QM == 0) {  // a group begins: scale and zero point of the lane's rows
          const int k = m * NG / QM;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(sc[b]) : "r"(scales + (b * 8 * NG + k) * 4) : "memory");
            z[b] = 0x00080008u;
            if constexpr (Z) {
              asm volatile("ld.shared.u8 %0, [%1];" : "=r"(z[b]) : "r"(zeros + b * 8 * NG + k) : "memory");
              z[b] = (z[b] & 15) * 0x00010001u;
            }
          }
        }
        if (m % LM == 0)
          asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                       : "=r"(code[0]), "=r"(code[1]), "=r"(code[2]), "=r"(code[3]) : "r"(from ^ (m * 16)) : "memory");
        if (m == QM - LM) {  // the slot has been read
          __syncwarp();
          request(slot);
          slot = slot + STEP == DEPTH * STEP ? 0 : slot + STEP;
        }
        uint32_t w[NB][4];
#pragma unroll
        for (int b = 0; b < NB; ++b) widen(code[(m % LM) * NB + b], b128, z[b] | B128, w[b]);
        // fp32: the lower parts by themselves, added to the group's sum once.  A matrix step cuts its sum at the largest
        // term's last bit, so each step on the group's sum costs up to a unit of it, each of these 2^-8 of that.
        float low[MT][NT][4];
        if constexpr (PLANES > 1) {
#pragma unroll
          for (int p = PLANES - 1; p > 0; --p)
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                  part(low[mt][t], w[2 * mt], w[2 * mt + 1], xb[m % XB][t][p], half, p == PLANES - 1 && half == 0);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              part(grp[mt][t], w[2 * mt], w[2 * mt + 1], xb[m % XB][t][0], half, m * NG % QM == 0 && half == 0);
        if constexpr (PLANES > 1) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int i = 0; i < 4; ++i) grp[mt][t][i] += low[mt][t][i];
        }
        if (m + XB < QM || more)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int p = 0; p < PLANES; ++p) xb[m % XB][t][p] = load_b128(xp[t] + (size_t)p * xw + (m + XB) * 32);
        if ((m + 1) * NG % QM == 0) {  // a group ends
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float& a = acc[b >> 1][t][(b & 1) * 2 + i];
                a = fmaf(sc[b], grp[b >> 1][t][(b & 1) * 2 + i], a);
              }
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) xp[t] += QCOLS;
    }
  }
};

template <typename T, int PLANES, int MT, int NG, bool Z, bool SF, int DEPTH>
__global__ void __launch_bounds__(QW * 32, 2) k_quant(QuantArgs A) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int warp_sums[QW];
  using Warp = QuantWarp<PLANES, MT, NG, Z, SF, DEPTH>;
  constexpr int TOKENS = TOKENS_OF_PASS<PLANES>;
  float4* sums = reinterpret_cast<float4*>(smem + QW * DEPTH * Warp::STEP);  // [2][QW][MT][32]
  int* first = reinterpret_cast<int*>(sums + 2 * QW * MT * 32);            // [n_expert + 1] first item of each expert
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, R = A.n_rows;
  auto row_begin = [&](int e) { return A.expert_off ? min(max(A.expert_off[e], 0), R) : 0; };
  auto row_end = [&](int e) { return A.expert_off ? min(max(A.expert_off[e + 1], 0), R) : R; };
  bool falling = false;  // ranges that overlap: their items may be more than 32 bits can count
  for (int e = threadIdx.x; e < A.n_expert; e += QW * 32) {
    const int rows = row_end(e) - row_begin(e);
    falling |= rows < 0;
    first[e] = (rows + TOKENS - 1) / TOKENS * A.tile_groups;
  }
  if (__syncthreads_or(falling)) {
    pdl_wait();
    return;
  }
  block_exclusive_scan(first, A.n_expert, warp_sums);
  const int total = first[A.n_expert];
  const int i0 = (int)((int64_t)total * blockIdx.x / gridDim.x), i1 = (int)((int64_t)total * (blockIdx.x + 1) / gridDim.x);
  if (i0 == i1) {  // no share; the grid must not end before the kernel that it was launched beside, even if nobody has one
    pdl_wait();
    return;
  }
  const int tiles_per = QW / A.wk;
  QuantAt at;
  {
    int lo = 0, hi = A.n_expert;  // the last e with first[e] <= i0
    while (hi - lo > 1) {
      const int m = (lo + hi) / 2;
      if (first[m] <= i0) lo = m; else hi = m;
    }
    at.item = i0;
    at.e = lo;
    quant_enter(at, first, A.tile_groups);
    at.tg = (i0 - first[at.e]) / at.passes;
    at.pass = (i0 - first[at.e]) - at.tg * at.passes;
  }
  const int width = A.swiglu ? A.n_out / 2 : A.n_out;
  Warp W(A, first, at, i1, w, lane, (uint32_t)__cvta_generic_to_shared(smem + w * (DEPTH * Warp::STEP)));
  W.aim();
#pragma unroll 1
  for (int i = 0; i < DEPTH; ++i) W.request(i * Warp::STEP);
  pdl_wait();  // x in bf16

  uint32_t slot = 0;
  int flip = 0;
  // a thread: one token, one tile row g and its partner g + 8
  auto join = [&](int t, const QuantAt& at, int row0, int rows, int tile_warp) {
    for (int i = threadIdx.x - tile_warp * 32; i < MT * 64; i += A.wk * 32) {
      const int h = i & 1, l = (i >> 1) & 31, mt = i >> 6;
      const int token = t * 8 + (l & 3) * 2 + h;
      if (token >= rows) continue;
      float a = 0.f, b = 0.f;
      for (int k = 0; k < A.wk; ++k) {
        const float* v = reinterpret_cast<const float*>(sums + ((size_t)(flip * QW + tile_warp + k) * MT + mt) * 32 + l);
        a += v[h];
        b += v[h + 2];
      }
      const int64_t r = row0 + token;
      a *= A.xf[r];
      b *= A.xf[r];
      T* out = reinterpret_cast<T*>(A.out) + r * A.os;
      const int per = A.swiglu ? 8 : 16, o_tile = (at.tg * tiles_per + W.wr) * MT * per;  // its first column, before it was moved up
      const int o = (MT == 1 ? o_tile : max(min(o_tile, width - MT * per), 0)) + mt * per + (l >> 2);
      const bool w0 = o >= o_tile && o < width, w1 = !A.swiglu && o + 8 >= o_tile && o + 8 < width;
      if (A.swiglu) a = a / (1.f + expf(-a)) * b;
      if (w0) out[o] = from_f<T>(a);
      if (w1) out[o + 8] = from_f<T>(b);
    }
  };
  for (; at.item < i1; quant_next(at, i1, first, A.tile_groups)) {
    const int row0 = row_begin(at.e) + at.pass * TOKENS, rows = min(row_end(at.e) - row0, TOKENS);
    float acc[MT][Warp::NTOK][4] = {};
    if (TOKENS == 8 || rows <= 8) W.template item<1>(at, row0, rows, slot, acc);
    else W.template item<Warp::NTOK>(at, row0, rows, slot, acc);
    // join the column shares of the tile's warps, in order, 8 tokens at a time.  Two buffers: one is written while slower
    // warps still read the other, and no warp is two turns ahead of its partners
    const int tile_warp = W.wr * A.wk;  // the tile's first warp
#pragma unroll
    for (int t = 0; t < Warp::NTOK; ++t) {
      if (t * 8 >= rows) break;
      float4* mine = sums + (size_t)(flip * QW + w) * MT * 32 + lane;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) mine[mt * 32] = make_float4(acc[mt][t][0], acc[mt][t][1], acc[mt][t][2], acc[mt][t][3]);
      if (A.wk == 1) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"(1 + W.wr), "r"(A.wk * 32) : "memory");
      join(t, at, row0, rows, tile_warp);
      flip ^= 1;
    }
  }
}

template <typename T, int NG, bool SF> static deamoe_status_t quant_t(QuantArgs& A, cudaStream_t s) {
  constexpr int PLANES = sizeof(T) == 4 ? 3 : 1;
  A.vec_scales = A.groups % NG == 0 && aligned_to(A.scales, NG == 2 && !SF ? 4 : 8);
  A.vec_zeros = A.zeros && A.groups % NG == 0 && aligned_to(A.zeros, NG < 4 ? NG : 4);
  const int tiles16 = A.swiglu ? (A.n_out / 2 + 7) / 8 : (A.n_out + 15) / 16;
  const int active = A.n_expert < A.n_rows ? A.n_expert : A.n_rows;
  // Two row tiles a warp share its x values and loop (16 tokens' top-8 of 256 experts, 4096 x 7168: 308 us, 350 with one
  // tile a warp; fp32 591, 766); one where two would leave blocks without work (one token, one such matrix: 11.4 us, 13.3
  // with two; fp32 14.4, 18.5)
  const int mt = (int64_t)(tiles16 / 2) * active >= Q_GRID && A.n_out >= 32 ? 2 : 1;
  // Warps that share a tile's columns: all, or fewer (longer walks, fewer sums to join) while the blocks keep at least
  // 8 items each, so that their counts differ by little (the same 16 tokens: 308 us with this rule, 335 with all warps on
  // one tile; 4 tokens' top-8 of 64 experts, 7168 x 2048: 56 and 61; fp32 591 and 555, 85 and 90)
  A.wk = QW;
  while (A.wk > A.steps) A.wk /= 2;
  while (A.wk > 1 && (int64_t)((tiles16 + mt - 1) / mt) * (A.wk / 2) / QW * active >= 8 * Q_GRID) A.wk /= 2;
  const int per = QW / A.wk * mt;
  A.tile_groups = (tiles16 + per - 1) / per;
  auto run = [&](auto kernel, int depth, int step, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!(done.load(std::memory_order_acquire) >> dev & 1)) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 112 * 1024);
      if (e != cudaSuccess) return e;
      done.fetch_or(1ull << dev, std::memory_order_release);
    }
    const size_t smem = (size_t)QW * depth * step + (size_t)QW * mt * 1024 + (size_t)(A.n_expert + 1) * 4;
    const int threads = A.steps * (QCOLS / 8) < 1024 ? A.steps * (QCOLS / 8) : 1024;
    const bool wide = aligned16(A.x) && (A.xs * (int64_t)sizeof(T)) % 16 == 0;
    k_quant_x<T, PLANES><<<A.n_rows, threads, 0, s>>>(A, wide);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_pdl(kernel, dim3(Q_GRID), dim3(QW * 32), smem, s, A);
  };
  static std::atomic<uint64_t> done[4];
  cudaError_t e;
  if (mt == 2)
    e = A.zeros ? run(k_quant<T, PLANES, 2, NG, true, SF, 2>, 2, QuantWarp<PLANES, 2, NG, true, SF, 2>::STEP, done[0])
                : run(k_quant<T, PLANES, 2, NG, false, SF, 2>, 2, QuantWarp<PLANES, 2, NG, false, SF, 2>::STEP, done[1]);
  else
    e = A.zeros ? run(k_quant<T, PLANES, 1, NG, true, SF, 4>, 4, QuantWarp<PLANES, 1, NG, true, SF, 4>::STEP, done[2])
                : run(k_quant<T, PLANES, 1, NG, false, SF, 4>, 4, QuantWarp<PLANES, 1, NG, false, SF, 4>::STEP, done[3]);
  if (e == cudaSuccess) return DEAMOE_OK;
  cudaGetLastError();
  return DEAMOE_ERR_CUDA;
}

template <typename T> static deamoe_status_t quant_group(QuantArgs& A, int group, cudaStream_t s) {
  if (A.scale_f32)
    return group == 128 ? quant_t<T, 2, true>(A, s) : group == 64 ? quant_t<T, 4, true>(A, s) : quant_t<T, 8, true>(A, s);
  return group == 128 ? quant_t<T, 2, false>(A, s) : group == 64 ? quant_t<T, 4, false>(A, s) : quant_t<T, 8, false>(A, s);
}

}  // namespace deamoe

using namespace deamoe;

extern "C" {

uint64_t deamoe_quant_workspace(int32_t dtype, int32_t n_rows, int32_t n_in) {
  if (n_rows <= 0 || n_in <= 0) return 0;
  const uint64_t width = ((uint64_t)n_in + QCOLS - 1) / QCOLS * QCOLS;
  return (uint64_t)n_rows * (width * (dtype == DEAMOE_F32 ? 6 : 2) + sizeof(float));
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
  const int tiles = swiglu ? (width + 7) / 8 : (width + 15) / 16;
  // items are counted in 32 bits (an expert's last pass may be short, hence one more each)
  const int64_t passes = (int64_t)n_rows / (dtype == DEAMOE_F32 ? TOKENS_OF_PASS<3> : TOKENS_OF_PASS<1>) + n_expert;
  if (tiles * passes > INT_MAX) return DEAMOE_ERR_BATCH;
  A.xb = reinterpret_cast<uint16_t*>(workspace);
  A.xf = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) +
                                  (size_t)n_rows * A.steps * QCOLS * (dtype == DEAMOE_F32 ? 6 : 2));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (dtype == DEAMOE_F32) return quant_group<float>(A, group, s);
  return quant_group<__nv_bfloat16>(A, group, s);
}

}  // extern "C"
