// Gated feed-forward blocks:  A = X Wg ;  B = X Wu ;  H = act(A) * B ;  Y = H Wd, and their gradients:
//   G = dY Wd^T ;  dA = G * B * act'(A) ;  dB = G * act(A) ;  dX = dA Wg^T + dB Wu^T ;  dWg = X^T dA ;  dWu = X^T dB ;  dWd = H^T dY
//
// All products are fp32 products on the fp16 matrix cores (ht_split.h).  X, dY and the weights are packed into fragments of split values first (weights that few rows meet are not: ht_ffn_stream.h), in one launch that
// reads them twice: 32 rows (of a weight 32 hidden columns) a block, scaled by the largest of each row (of a weight by that of the block); for the
// gradients of weights X and dY also turned, scaled by the largest of the 32 rows.  (A block of zeros has no scale, and what meets it counts in none.)  The hidden columns of Wg and Wu lie interleaved by 32s, so that one product makes A and B of the
// same column in the same lane, and dA and dB are one operand with a reduction over both.  H, dA and dB are kept in fp32, in the order of fragments, and with the largest
// values of their rows and columns; the products that read them split them as they load, with no pass in between: by rows where the reduction is over
// hidden columns, by columns where it is over rows.  A scale that changes along a reduction (of the other operand's 32s) is taken off what is split: a stage of a product is
// 32 values of it.
#include <algorithm>
#include <type_traits>

#include "ht_ffn.h"
#include "ht_split.h"

namespace {

constexpr int HB = 32;                 // hidden columns of a block: [gate, up] of interleaved operands

// ---------------------------------------------------------------- scales

// The exponent of the power of two that brings what has its largest absolute value in these bits to [2^14, 2^15).  (NONE: there is nothing, or only zeros.)
constexpr int NONE = 1 << 20;
__device__ __forceinline__ int scale_exp(uint32_t bits) {
  if (bits == 0) return NONE;
  const int e = 141 - (int)(bits >> 23);
  return e > 126 ? 126 : e;            // (values below 2^-112 come to less)
}
__device__ __forceinline__ int exp_or_0(int e) { return e >= NONE ? 0 : e; }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)((e < -126 ? -126 : e > 126 ? 126 : e) + 127) << 23); }
// What a block of zeros (its exponent is NONE) meets is scaled by 0: it adds nothing, and takes no bits off what the other blocks meet.  (What is not finite becomes NaN there, as 0 times it is.
// ldexp takes NONE as it is: sums of zeros stay 0, and largest values less it are 0.)
__device__ __forceinline__ float pow2_or_0(int e) { return e < -NONE / 4 ? 0.f : pow2(e); }
// Of an operand the largest value is that of what is finite: the rest becomes NaN in its split, and takes no bits off the others.
__device__ __forceinline__ uint32_t size_bits(float x) {
  const uint32_t b = __float_as_uint(fabsf(x));
  return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t max4(V4 x) { return max(max(size_bits(x[0]), size_bits(x[1])), max(size_bits(x[2]), size_bits(x[3]))); }

// ---------------------------------------------------------------- operands

// Fragments of a matrix: 32 of its own rows a block (or, turned, of its own columns: `own` and `run` are its rows and columns, or the other way round), zeros behind the last.
struct Pack {
  const float* p;
  int64_t ld, own, run;
  int turned;
  int *e_own, *e_block;                // exponents: of each of the own (null: they have the block's), of the block (NONE where it is all zeros)
  _Float16* F;                         // by own rows, reduction along run: row block b is number b mul + add, KS steps
  int64_t KS;
  int mul, add;
  _Float16* T;                         // (nullable) by run, scaled by blocks, KS_t steps; own as the reduction
  int64_t KS_t;
  int tiles;                           // of PACK_RUN along run
  int steps, blocks_t;                 // of F and of T that are written: whole pairs of stages of a reduction; what a tile has beyond its operand's rows reaches no sum that is kept
  unsigned blocks, share;              // (of so many own rows' blocks each takes a part of the tiles, all of them look for the largest values)
};
constexpr int PACKS = 5, PACK_RUN = 128;
constexpr int64_t PACK_BLOCKS = 1024;  // where there are fewer, tiles are shared out
struct Packs {
  unsigned first[PACKS + 1];           // blocks before each, and before those that clear words (side by side: one trip to the arguments)
  Pack pack[PACKS];
  int n = 0;
  uint32_t* zero;                      // words that become 0, by the blocks behind
  int64_t zeros;
};
constexpr unsigned ZEROS = 4096;       // a block
__global__ void __launch_bounds__(256) k_ffn_pack(Packs packs) {
  __shared__ float sh[HB][PACK_RUN + 1];
  __shared__ uint32_t top[HB];
  int i = 0;
#pragma unroll
  for (int k = 1; k <= PACKS; ++k) i += blockIdx.x >= packs.first[k];
  unsigned block = blockIdx.x - packs.first[i];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;
  if (i == PACKS) {
    for (int64_t k = (int64_t)block * ZEROS + tid; k < packs.zeros && k < (int64_t)(block + 1) * ZEROS; k += 256) packs.zero[k] = 0;
    return;
  }
  const Pack& a = packs.pack[i];
  const unsigned part = block % a.share;
  block /= a.share;
  const int64_t own0 = (int64_t)block * HB, left = a.own - own0;               // (left may be <= 0: zeros)
  if (tid < HB) top[tid] = 0;
  __syncthreads();
  // What is there at (row, c .. c + 3); the others are 0.  Loads have no condition (rows and columns behind the last are the last again), so that they go together: with one each, 128 x
  // 1,024 rows took 17 us.  whole: all of the columns that the block looks at are there.
  auto four = [&](int64_t row, int64_t c, int64_t rows, int64_t cols, bool whole) __attribute__((always_inline)) {
    const float* from = a.p + (row < rows ? row : rows - 1) * a.ld;
    V4 x;
    if (whole) {
      x = *reinterpret_cast<const V4u*>(from + c);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = from[c + k < cols ? c + k : cols - 1];
    }
    return x;
  };
  auto there = [&](V4 x, int64_t row, int64_t c, int64_t rows, int64_t cols) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = row < rows && c + k < cols ? x[k] : 0.f;
    return x;
  };
  if (!a.turned) {
    // a wave eight rows
    uint32_t m[8] = {};
    auto look = [&](int64_t c0, bool whole) __attribute__((always_inline)) {
      V4 x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = four(own0 + wave * 8 + q, c0 + lane * 4, a.own, a.run, whole);
#pragma unroll
      for (int q = 0; q < 8; ++q) m[q] = max(m[q], max4(x[q]));                // (the last column again is no larger)
    };
    int64_t c0 = 0;
#pragma unroll 2
    for (; c0 + 256 <= a.run; c0 += 256) look(c0, true);
    if (c0 < a.run) look(c0, false);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      for (int o = 32; o > 0; o >>= 1) m[q] = max(m[q], (uint32_t)__shfl_xor((int)m[q], o, 64));
      if (lane == 0) top[wave * 8 + q] = wave * 8 + q < left ? m[q] : 0;
    }
  } else {
    // eight lanes a row of 32 columns
    uint32_t m = 0;
    auto look = [&](int64_t r0, bool whole) __attribute__((always_inline)) {
      V4 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = four(r0 + q * 32 + (tid >> 3), own0 + (tid & 7) * 4, a.run, a.own, whole);
#pragma unroll
      for (int q = 0; q < 4; ++q) m = max(m, max4(x[q]));
    };
    const bool whole = left >= HB;
    if (whole) {
#pragma unroll 2
      for (int64_t r0 = 0; r0 < a.run; r0 += 128) look(r0, true);
    } else if (left > 0) {
      for (int64_t r0 = 0; r0 < a.run; r0 += 128) look(r0, false);
    }
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if (lane == 0) top[wave] = m;      // (the others stay 0)
  }
  __syncthreads();
  uint32_t all = top[l32];
  for (int o = 16; o > 0; o >>= 1) all = max(all, (uint32_t)__shfl_xor((int)all, o, 64));
  const int e_all = scale_exp(all), eb = exp_or_0(e_all), eo = a.e_own ? exp_or_0(scale_exp(top[l32])) : eb;
  if (tid < HB && a.e_own && part == 0) a.e_own[own0 + tid] = eo;
  if (tid == 0 && a.e_block && part == 0) a.e_block[(int64_t)block * a.mul + a.add] = e_all;
  const float fb = pow2(eb), fo = pow2(eo);
  auto put = [&](_Float16* to, int64_t frag, const float (&x)[8]) {
    v8h hi, lo;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      _Float16 u, v;
      split2(x[t], &u, &v);
      hi[t] = u;
      lo[t] = v;
    }
    *reinterpret_cast<v8h*>(to + frag * 2 * FRAG + lane * 8) = hi;
    *reinterpret_cast<v8h*>(to + frag * 2 * FRAG + FRAG + lane * 8) = lo;
  };
  for (int tile = part; tile < a.tiles; tile += a.share) {
    const int64_t run0 = (int64_t)tile * PACK_RUN;
    V4 y[4];
    // 32 lanes a row of PACK_RUN, or eight a row of 32
    const int64_t rows = a.turned ? a.run : a.own, cols = a.turned ? a.own : a.run;
    auto fetch = [&](bool whole) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = a.turned ? q * 32 + (tid >> 3) : q * 8 + (tid >> 5), c4 = a.turned ? (tid & 7) * 4 : (tid & 31) * 4;
        y[q] = four((a.turned ? run0 : own0) + r, (a.turned ? own0 : run0) + c4, rows, cols, whole);
      }
      if (whole && left >= HB && run0 + PACK_RUN <= a.run) return;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = a.turned ? q * 32 + (tid >> 3) : q * 8 + (tid >> 5), c4 = a.turned ? (tid & 7) * 4 : (tid & 31) * 4;
        y[q] = there(y[q], (a.turned ? run0 : own0) + r, (a.turned ? own0 : run0) + c4, rows, cols);
      }
    };
    if (a.turned ? left >= HB : run0 + PACK_RUN <= a.run) fetch(true);
    else fetch(false);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = a.turned ? q * 32 + (tid >> 3) : q * 8 + (tid >> 5), c4 = a.turned ? (tid & 7) * 4 : (tid & 31) * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (a.turned) sh[c4 + k][r] = y[q][k];
        else sh[r][c4 + k] = y[q][k];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int ks = wave * 2 + u, k = ks * 16 + half * 4;
      float x[8];
      if (run0 / 16 + ks < a.steps) {
#pragma unroll
        for (int t = 0; t < 8; ++t) x[t] = sh[l32][k + (t >> 2) * 8 + (t & 3)] * fo;
        put(a.F, ((int64_t)block * a.mul + a.add) * a.KS + run0 / 16 + ks, x);
      }
      if (!a.T || run0 / 32 + wave >= a.blocks_t) continue;
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = sh[u * 16 + half * 4 + (t >> 2) * 8 + (t & 3)][wave * 32 + l32] * fb;
      put(a.T, (run0 / 32 + wave) * a.KS_t + (int64_t)block * 2 + u, x);
    }
  }
}

// ---------------------------------------------------------------- products

// PROJECT  A's rows: the interleaved hidden columns, B's the rows of X: A and B of the block, H and its largest values
// BACK     A's rows: hidden columns of Wd, B's 64 the rows of dY: G, from that and A and B all of H, dA, dB and their largest values
// ROWS     A: H or [dA dB] by rows, B: a weight turned: Y, dX
// COLS     A: X or dY by columns, B: [dA dB] or H turned: gradients of weights
// PROJECT_SMALL  PROJECT by 64 rows a block, for calls whose tiles are fewer than there is room for, and three blocks a CU
// COLS_SMALL     COLS of at most 128 rows of A
enum { PROJECT, BACK, ROWS, COLS, PROJECT_SMALL, COLS_SMALL };
constexpr bool is_cols(int mode) { return mode == COLS || mode == COLS_SMALL; }

struct Out {                           // value (m, n) at m ms + n ns, split_part floats apart
  float* p;
  int64_t ms, ns, split_part;
};
struct Args {
  const _Float16 *A, *B;               // fragments; row blocks KSA, KSB steps apart (B turned: of its own)
  int64_t KSA, KSB;
  int64_t mt, nt;                      // tiles
  int64_t pairs;                       // of stages, of the reduction
  int splits;                          // parts of it
  int two;                             // an operand is [dA dB]
  // exponents: PROJECT of Wg and Wu by hidden blocks, interleaved, BACK of Wd; ROWS, COLS: of the other operand by stages of the reduction
  const int* e_w;
  const int* e_in;                     // PROJECT, BACK: of the rows of X, of dY
  // largest values of what is made, less the exponents of what it will meet: by rows of H (Wd's: e_d), of dA and dB together (Wg's and Wu's), by columns of H (the rows'
  // of dY by 32s: e_y), of dA and dB (of X: e_x)
  uint32_t *h_row, *d_row, *h_col, *a_col, *b_col;
  const int *e_d, *e_x, *e_y;
  int64_t n, f;                        // rows, hidden columns that there are
  float *H, *D;                        // in the order of fragments (null: not wanted)
  int64_t KSH, KSD;
  float *gate, *up;                    // [n x f]
  int64_t ld_gate, ld_up;
  Out out[2];                          // ROWS: [0]; COLS of [dA dB]: gate's and up's (null: not wanted)
  int64_t m_end, n_end;                // (n_end: of hidden columns, for COLS)
  int add;
};

// Eight values (t = 0 .. 3 and 4 .. 7 where the planes will be), times `all` and each times its factor, powers of two.  Two instructions a value: the compiler rounds each value twice where it
// is left to itself (a pair's halves once more for themselves).
template <class F>
__device__ __forceinline__ void split8(v8h& p0, v8h& p1, float all, F&& factor) {
  typedef uint32_t v4i __attribute__((ext_vector_type(4)));
  const V4 x = __builtin_bit_cast(V4, p0) * all, y = __builtin_bit_cast(V4, p1) * all;
  v4i hi, lo;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = k < 2 ? x[2 * k] : y[2 * k - 4], b = k < 2 ? x[2 * k + 1] : y[2 * k - 3], fa = factor(2 * k), fb = factor(2 * k + 1);
    uint32_t h, l;
    asm("v_fma_mixlo_f16 %0, %2, %3, 0 op_sel_hi:[0,0,0]\n\t"
        "v_fma_mixhi_f16 %0, %4, %5, 0 op_sel_hi:[0,0,0]\n\t"
        "v_fma_mixlo_f16 %1, %2, %3, -%0 op_sel_hi:[0,0,1]\n\t"
        "v_fma_mixhi_f16 %1, %4, %5, -%0 op_sel:[0,0,1] op_sel_hi:[0,0,1]"
        : "=&v"(h), "=&v"(l)
        : "v"(a), "v"(fa), "v"(b), "v"(fb));
    hi[k] = h, lo[k] = l;
  }
  p0 = __builtin_bit_cast(v8h, hi), p1 = __builtin_bit_cast(v8h, lo);
}

// The largest of each of four over l32: the e-th in the lanes with l32 / 8 = e.
__device__ __forceinline__ float max_over_32(const float (&x)[4]) {
  const bool up16 = threadIdx.x & 16, up8 = threadIdx.x & 8;
  float y[2], v;
#pragma unroll
  for (int k = 0; k < 2; ++k) y[k] = fmaxf(up16 ? x[k + 2] : x[k], __shfl_xor(up16 ? x[k] : x[k + 2], 16, 64));
  v = fmaxf(up8 ? y[1] : y[0], __shfl_xor(up8 ? y[0] : y[1], 8, 64));
  for (int o = 4; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// acc += A B^T of fragments: NI row blocks of A a wave, NJ of B, which the four waves of a block share.  A wave reads its own rows of A straight into registers,
// a stage ahead (FAR) or a step, and B goes through LDS, which is filled a stage ahead.
//   Ap   the wave's first row block, the lane's place in it; a_rows halfs from one row block to the next
//   Bp   the tile's first row block (TURN: the tile's first 16 of the reduction's first row block); b_rows from one to the next
//   in_a(x, i, e)  what is done to a step's planes of row block i before they are used, in_b(rb, e): to what a wave brings of B; e: the stage's exponent, of e_stage (TURN)
template <bool TURN, bool FAR, int NI, int NJ, class InA, class InB>
__device__ __forceinline__ void multiply(v16f (&acc)[NI][NJ], const _Float16* Ap, const int64_t a_rows, const _Float16* B, const int64_t b_rows, const int* e_stage, int todo, _Float16* Bs, InA&& in_a,
                                         InB&& in_b) {
  static_assert(!TURN || NJ == 4, "a stage of a turned operand is 32 x 128");
  constexpr int STAGE = stage_halfs(TURN), RB = TURN ? 4 : NJ * KT * 2 / 4, AHEAD = FAR ? 2 * KT : 2;
  static_assert(FAR || KT == 2, "steps take turns");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  // a wave brings NJ of the fragments (row block, step, plane) of a stage, or two of the eight 16s
  int64_t b_at[RB];
#pragma unroll
  for (int u = 0; u < RB; ++u) {
    const int q = wave * RB + u;
    b_at[u] = TURN ? (int64_t)q * FRAG : (int64_t)(q / (KT * 2)) * b_rows + q % (KT * 2) * FRAG;
  }
  const _Float16* Bp = B + lane * 8;
  const int64_t b_step = TURN ? b_rows : KT * 2 * FRAG;
  v8h ra[AHEAD][NI][2], rb[RB];
  int e = 0, e_next = 0;
  auto fetch_a = [&](int to) {        // the next step
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int p = 0; p < 2; ++p) ra[to][i][p] = *reinterpret_cast<const v8h*>(Ap + i * a_rows + p * FRAG);
    Ap += 2 * FRAG;
  };
  auto fetch_b = [&]() {              // the next stage
#pragma unroll
    for (int u = 0; u < RB; ++u) rb[u] = *reinterpret_cast<const v8h*>(Bp + b_at[u]);
    Bp += b_step;
    if (TURN) e_next = *e_stage++;
  };
  auto stash = [&](int to) {
    in_b(rb, e_next);
    e = e_next;
#pragma unroll
    for (int u = 0; u < RB; ++u)
      *reinterpret_cast<v8h*>(Bs + to * STAGE + (TURN ? ((wave * 4 + u) * 2 + half) * TURN_HALF + l32 * 8 : (wave * RB + u) * FRAG + lane * 8)) = rb[u];
  };
  auto read_b = [&](v8h* b, int cur, int k) {          // k: step * NJ + row block
    const int u = k / NJ, j = k % NJ;
    if (TURN) {
      const int i = lane & 15, sixteen = j * 2 + ((lane >> 4) & 1);
      const _Float16* f = Bs + cur * STAGE + (sixteen * 4 + (i & 1)) * TURN_HALF + (u * 16 + half * 4 + (i >> 2)) * 8 + ((i >> 1) & 1) * 4;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const v4h lo = turned(f + p * 2 * TURN_HALF), hi = turned(f + p * 2 * TURN_HALF + 64);
        b[p] = v8h{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      }
      return;
    }
    const _Float16* f = Bs + cur * STAGE + (j * KT * 2 + u * 2) * FRAG + lane * 8;
    b[0] = *reinterpret_cast<const v8h*>(f);
    b[1] = *reinterpret_cast<const v8h*>(f + FRAG);
  };
  // (Loads have no condition, so that waits count only the loads that they wait for: the last stage fetches itself again.  The barriers to scheduling
  // keep them where they stand; they would be moved down to where they are used.)
  auto stage = [&](int cur, bool more) {
    if (!more) Bp -= b_step, e_stage -= TURN;
    if (FAR && !more) Ap -= KT * 2 * FRAG;
    v8h b[2][2];
    read_b(b[0], cur, 0);
    fetch_b();
    if (FAR) {
#pragma unroll
      for (int u = 0; u < KT; ++u) fetch_a((cur ^ 1) * KT + u);
    }
#pragma unroll
    for (int k = 0; k < NJ * KT; ++k) {
      const int u = k / NJ, j = k % NJ;
      v8h (&x)[NI][2] = ra[FAR ? cur * KT + u : u];
      const v8h (&y)[2] = b[k & 1];
      if (j == 0) {
        if (!FAR) {
          if (u == KT - 1 && !more) Ap -= KT * 2 * FRAG;
          fetch_a(u ^ 1);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) in_a(x[i], i, e);
      }
      if (k + 1 < NJ * KT) read_b(b[(k + 1) & 1], cur, k + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][1], y[0], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[1], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[0], acc[i][j], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    stash(cur ^ 1);
    __syncthreads();
  };
  if (todo <= 0) return;
  fetch_b();
#pragma unroll
  for (int u = 0; u < (FAR ? KT : 1); ++u) fetch_a(u);
  stash(0);
  __syncthreads();
  do {
    stage(0, true);
    stage(1, --todo > 0);
  } while (todo > 0);
}

__device__ __forceinline__ void raise(uint32_t* word, uint32_t m) {       // (most find a word as large as it need be)
  if (__hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < m) atomicMax(word, m);
}
// Where a block's tile is: each XCD takes a contiguous part of the tiles, eight tiles of A over all of B after eight others.
struct Tile {
  int64_t split, m, n;                 // m < 0: none
  __device__ __forceinline__ Tile(unsigned block, int64_t mt, int64_t nt, int splits) {
    const int64_t tiles = mt * nt, per = (tiles * splits + 7) / 8, ts = (int64_t)(block & 7) * per + (block >> 3);
    m = -1;
    if ((int64_t)(block >> 3) >= per || ts >= tiles * splits) return;
    split = ts / tiles;
    const int64_t t = ts - split * tiles, g = t / (8 * nt), gm = mt - g * 8 < 8 ? mt - g * 8 : 8, q = t - g * 8 * nt;
    m = g * 8 + q % gm, n = q / gm;
  }
};
template <int NI, int NJ>
__device__ __forceinline__ void clear(v16f (&acc)[NI][NJ]) {
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
}

// Hidden values as they are stored.  Lane l32 + 32 half of a 32 x 32 tile of sums has column l32, a row of X, and the rows 8 k + 4 half + 0 .. 3, hidden columns c .. c + 3.
struct Hidden {
  const Args& a;
  int lane, half;
  __device__ __forceinline__ Hidden(const Args& args) : a(args), lane(threadIdx.x & 63), half((threadIdx.x & 63) >> 5) {}
  // four values of hidden columns c .. c + 3 of a row of gate or up; whole: there are all of the block's
  __device__ __forceinline__ void put(float* p, int64_t c, V4 x, bool whole) const {
    if (whole) {
      *reinterpret_cast<V4*>(p + c) = x;
      return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < a.f) p[c + k] = x[k];
  }
  __device__ __forceinline__ V4 get(const float* p, int64_t c, bool whole) const {      // (behind the last column: the last one again)
    if (whole) return *reinterpret_cast<const V4*>(p + c);
    V4 x;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = p[c + k < a.f ? c + k : a.f - 1];
    return x;
  }
  // four values of a row, in the order of fragments: the k-th four of 16 columns by half
  __device__ __forceinline__ void put_frag(float* p, int64_t KS, int64_t row_block, int64_t step, int k, V4 x) const {
    // (past the caches, which have the operands to keep: 232,965 x 256 x 1,024 backward 4.16 -> 4.08 ms)
    __builtin_nontemporal_store(x, reinterpret_cast<V4*>(p + ((row_block * KS + step) * 2 + k) * (FRAG / 2) + lane * 4));
  }
  // H, dA and dB of NJ row blocks from row block b0 on, of the hidden block hb.  Largest values, less the exponents of what they will meet: of the rows of dA and dB
  // together in md, of the columns (of H, dA, dB, 32 each) to cols.  (An infinite one may be the largest: what is scaled by it is not finite in any case.)  get(j, k, x, y): A
  // and B of four hidden columns of a row, fetched four columns ahead; sums(j, k, e): G of one.  Behind the last row and column G is 0, and with it dA and dB; H is 0
  // behind the last row, and behind the last column what get() gives there, which nothing reads that is kept.
  template <int ACT, int NJ, class Get, class Sums>
  __device__ __forceinline__ void back(int64_t b0, int64_t hb, float (&md)[NJ], float* cols, Get&& get, Sums&& sums) const {
    const int64_t c0 = hb * HB;
    float fx[NJ], fy[NJ], ma[NJ] = {}, mb[NJ] = {};
#pragma unroll
    for (int j = 0; j < NJ; ++j) fx[j] = pow2_or_0(-a.e_x[b0 + j]), fy[j] = pow2_or_0(-a.e_y[b0 + j]);
    const int eg = a.e_d[hb * 2], eu = a.e_d[hb * 2 + 1];
    const int l32 = lane & 31;
    V4 x[2][NJ], y[2][NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) get(j, 0, x[0][j], y[0][j]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k < 3) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) get(j, k + 1, x[(k + 1) & 1][j], y[(k + 1) & 1][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
      const int64_t step = c0 / 16 + (k >> 1), step_d = c0 / 8 + (k >> 1);
      float ch[4] = {}, ca[4] = {}, cb[4] = {};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        V4 h, da, db;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Act s = act_of<ACT>(x[k & 1][j][e]);
          const float u = y[k & 1][j][e], g = sums(j, k, e);
          h[e] = s.v * u, da[e] = g * u * s.s, db[e] = g * s.v;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ch[e] = fmaxf(ch[e], fabsf(h[e] * fy[j])), ca[e] = fmaxf(ca[e], fabsf(da[e] * fx[j])), cb[e] = fmaxf(cb[e], fabsf(db[e] * fx[j]));
          ma[j] = fmaxf(ma[j], fabsf(da[e])), mb[j] = fmaxf(mb[j], fabsf(db[e]));
        }
        put_frag(a.H, a.KSH, b0 + j, step, k & 1, h);
        put_frag(a.D, a.KSD, b0 + j, step_d, k & 1, da);
        put_frag(a.D, a.KSD, b0 + j, step_d + 2, k & 1, db);
        __builtin_amdgcn_sched_barrier(0);      // (one after the other: together they need more registers than there are)
      }
      const float th = max_over_32(ch), ta = max_over_32(ca), tb = max_over_32(cb);
      if (!(l32 & 7)) {
        float* to = cols + k * 8 + half * 4 + (l32 >> 3);
        to[0] = th, to[32] = ta, to[64] = tb;
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) md[j] = fmaxf(__builtin_amdgcn_ldexpf(ma[j], -eg), __builtin_amdgcn_ldexpf(mb[j], -eu));
  }
  // What the four waves found, to where it is kept: cols, of HBS hidden blocks from hidden column c0 on, and md by way of top (4 NJ 32 words of LDS).  All words are
  // looked at together: each takes a trip to memory.
  template <int NJ, int HBS>
  __device__ __forceinline__ void back_tops(int64_t b0, int64_t c0, const float (&md)[NJ], const float* cols, float* top) const {
    constexpr int R = NJ * 32, N = R + HBS * 96, U = (N + 255) / 256;
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float x = fmaxf(md[j], __shfl_xor(md[j], 32, 64));
      if (half == 0) top[wave * R + j * 32 + lane] = x;
    }
    __syncthreads();
    uint32_t *word[U], is[U], was[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = u * 256 + threadIdx.x;
      word[u] = nullptr;
      float m = 0.f;
      if (i < R) {
        m = fmaxf(fmaxf(top[i], top[R + i]), fmaxf(top[2 * R + i], top[3 * R + i]));
        if (b0 * 32 + i < a.n) word[u] = a.d_row + b0 * 32 + i;
      } else if (i < N) {
        const int q = i - R, which = q / 32 % 3;
        const int64_t c = c0 + q / 96 * 32 + q % 32;
        m = cols[q];
        if (c < a.f) word[u] = (which == 0 ? a.h_col : which == 1 ? a.a_col : a.b_col) + c;
      }
      is[u] = __float_as_uint(m);
      was[u] = word[u] ? __hip_atomic_load(word[u], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0xffffffffu;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (was[u] < is[u]) atomicMax(word[u], is[u]);
  }
};

template <int MODE, int ACT>
__device__ __forceinline__ void ffn_split(const Args& a, unsigned block, _Float16* Bs) {
  constexpr bool BY_COLS = is_cols(MODE), TURN = MODE == ROWS || BY_COLS;
  const Tile tile(block, a.mt, a.nt, a.splits);
  if (tile.m < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
  constexpr int NI = MODE == COLS_SMALL ? 1 : 2, NJ = MODE == PROJECT_SMALL || MODE == BACK ? 2 : 4;       // row blocks of A a wave, and of B (BACK has much to do with each sum)
  constexpr int NR = NJ * 32, MT = NI * 128;
  const int64_t split = tile.split, m0 = tile.m * MT, n0 = tile.n * NR, mw = m0 + wave * (NI * 32);
  const int64_t s0 = a.pairs * split / a.splits * 2;                 // its first stage
  const int todo = __builtin_amdgcn_readfirstlane((int)(a.pairs * (split + 1) / a.splits - s0 / 2));

  // exponents of a row of H or [dA dB] (ROWS), and of a column (COLS); hidden column of column n of B
  auto row_exp = [&](int64_t v) { return exp_or_0(scale_exp((a.two ? a.d_row : a.h_row)[v])); };
  auto hidden = [&](int64_t n) { return a.two ? n / (2 * HB) * HB + n % HB : n; };
  auto col_exp = [&](int64_t n) {
    const int64_t c = hidden(n);
    return c >= a.f ? 0 : exp_or_0(scale_exp(!a.two ? a.h_col[c] : (n / HB) & 1 ? a.b_col[c] : a.a_col[c]));
  };
  // exponents of the rows or columns of the sums, a thread each, for the end (looked up there they would be two trips to memory)
  int end = 0;
  if constexpr (MODE == ROWS) end = m0 + tid < a.m_end ? row_exp(m0 + tid) : 0;
  if constexpr (BY_COLS) end = tid < TN ? col_exp(n0 + tid) : 0;
  v16f acc[NI][NJ];
  clear(acc);
  const _Float16* Ap = a.A + (mw / 32 * a.KSA + s0 * KT) * 2 * FRAG + lane * 8;
  const _Float16* B = a.B + (TURN ? s0 * a.KSB + n0 / 16 : n0 / 32 * a.KSB + s0 * KT) * 2 * FRAG;
  const int64_t a_rows = a.KSA * 2 * FRAG, b_rows = a.KSB * 2 * FRAG;
  const auto a_as_it_is = [](v8h (&)[2], int, int) {};
  const auto b_as_it_is = [](v8h (&)[NJ], int) {};
  if constexpr (MODE == ROWS) {
    int er[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) er[i] = row_exp(mw + i * 32 + l32);
    multiply<true, true>(acc, Ap, a_rows, B, b_rows, a.e_w + s0, todo, Bs, [&](v8h (&x)[2], int i, int e) {
      // (in two powers: the row's exponent has the weights' in it, and less this stage's it may lie outside the range of floats)
      const int t = er[i] - e, u = t >> 1;
      const float f = pow2_or_0(t - u);
      split8(x[0], x[1], pow2(u), [&](int) { return f; });
    }, b_as_it_is);
  } else if constexpr (BY_COLS) {
    float fc[2][8];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int k = 0; k < 8; ++k) fc[u][k] = pow2(col_exp(n0 + wave * 32 + u * 16 + (k >> 2) * 8 + half * 4 + (k & 3)));
    multiply<true, true>(acc, Ap, a_rows, B, b_rows, a.e_w + s0, todo, Bs, a_as_it_is, [&](v8h (&rb)[4], int e) {
      const float f = pow2_or_0(-e);
#pragma unroll
      for (int u = 0; u < 2; ++u) split8(rb[u * 2], rb[u * 2 + 1], f, [&](int t) { return fc[u][t]; });
    });
  } else {
    multiply<false, NJ == 4>(acc, Ap, a_rows, B, b_rows, nullptr, todo, Bs, a_as_it_is, b_as_it_is);
  }

  // lane l32 + 32 half of a 32 x 32 tile has column l32 and the rows 8 (e / 4) + 4 half + e % 4
  if constexpr (TURN) {
    // Exponents of the rows or columns of sums, all of them looked up at once (where they are used, one after the other, each would be a trip to memory).  Sums go by way of LDS, 32
    // columns at a time, so that what writes them is a short loop: unrolled it is 4,000 instructions a wave (1,003 x 301 x 1,213, Y: 16.2 -> 15.3 us, 8,192 x 1,024 x 4,096, dX: 463 -> 447).
    int* ends = reinterpret_cast<int*>(Bs);
    float* sums = reinterpret_cast<float*>(Bs) + TM;
    constexpr int P = MT + 4;
    static_assert((TM + 32 * P) * 4 <= 2 * stage_halfs(true) * 2, "sums of 32 columns beside the exponents");
    ends[tid] = end;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool up = BY_COLS && a.two && (j & 1);
      float* out = up ? a.out[1].p : a.out[0].p;
      const int64_t ms = up ? a.out[1].ms : a.out[0].ms, ns = up ? a.out[1].ns : a.out[0].ns, part = up ? a.out[1].split_part : a.out[0].split_part;
      if (!out) continue;
      const int64_t c0 = BY_COLS && a.two ? n0 / 2 + j / 2 * HB : n0 + j * 32;      // its first column
      if (c0 >= a.n_end) continue;
      if (j > 0) __syncthreads();
      const int en = BY_COLS ? ends[j * 32 + l32] : 0;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = wave * (NI * 32) + i * 32 + k * 8 + half * 4;
          const int4 em = MODE == ROWS ? *reinterpret_cast<const int4*>(ends + r) : make_int4(0, 0, 0, 0);
          *reinterpret_cast<V4*>(sums + l32 * P + r) =
              V4{__builtin_amdgcn_ldexpf(acc[i][j][k * 4], -(em.x + en)), __builtin_amdgcn_ldexpf(acc[i][j][k * 4 + 1], -(em.y + en)),
                 __builtin_amdgcn_ldexpf(acc[i][j][k * 4 + 2], -(em.z + en)), __builtin_amdgcn_ldexpf(acc[i][j][k * 4 + 3], -(em.w + en))};
        }
      __syncthreads();
      // fours of neighbours: of a row 32 columns by eight lanes, or of a column all rows by a wave or half of one
      const bool along = ns == 1;
      constexpr int LANES = MT / 4, COLUMNS = 256 / LANES, TIMES = MT / 32;      // of a column, columns at a time, how often
      const int m = along ? tid >> 3 : (tid % LANES) * 4, n = along ? (tid & 7) * 4 : tid / LANES, m_step = along ? 32 : 0, n_step = along ? 0 : COLUMNS;
      float* to = out + split * part + (m0 + m) * ms + (c0 + n) * ns;
      const int64_t step = along ? 32 * ms : COLUMNS * ns;
      auto four = [&](int it) {
        const float* from = sums + (n + it * n_step) * P + m + it * m_step;
        return along ? V4{from[0], from[P], from[2 * P], from[3 * P]} : *reinterpret_cast<const V4*>(from);
      };
      if (m0 + MT <= a.m_end && c0 + HB <= a.n_end) {
        V4 x[TIMES];
#pragma unroll
        for (int it = 0; it < TIMES; ++it) x[it] = four(it);
        if (a.add) {
#pragma unroll
          for (int it = 0; it < TIMES; ++it) x[it] += *reinterpret_cast<const V4u*>(to + it * step);
        }
#pragma unroll
        for (int it = 0; it < TIMES; ++it) *reinterpret_cast<V4u*>(to + it * step) = x[it];
        continue;
      }
#pragma unroll 1
      for (int it = 0; it < TIMES; ++it, to += step) {
        V4 x = four(it);
        const int64_t m_left = a.m_end - (m0 + m + it * m_step), n_left = a.n_end - (c0 + n + it * n_step), left = along ? n_left : m_left;
        if (m_left <= 0 || n_left <= 0) continue;
        if (left >= 4) {
          if (a.add) x += *reinterpret_cast<const V4u*>(to);
          *reinterpret_cast<V4u*>(to) = x;
        } else {
          for (int k = 0; k < left; ++k) {
            const float v = k == 0 ? x[0] : k == 1 ? x[1] : x[2];
            to[k] = a.add ? to[k] + v : v;
          }
        }
      }
    }
    return;
  }
  float* top = reinterpret_cast<float*>(Bs);
  const Hidden at(a);
  if constexpr (MODE == PROJECT || MODE == PROJECT_SMALL) {
    const int64_t c0 = mw / 2;                          // the wave's 32 hidden columns
    int exps[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) exps[j] = a.e_in[n0 + j * 32 + l32];
    const int e0 = a.e_w[c0 / HB * 2], e1 = a.e_w[c0 / HB * 2 + 1], ed = a.e_d[c0 / HB];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t v = n0 + j * 32 + l32;
      const bool there = v < a.n;
      const int ex = exps[j];
      float m = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t c = c0 + k * 8 + half * 4;
        V4 x, y, h;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = __builtin_amdgcn_ldexpf(acc[0][j][k * 4 + e], -(ex + e0)), y[e] = __builtin_amdgcn_ldexpf(acc[1][j][k * 4 + e], -(ex + e1));
          h[e] = act_of<ACT>(x[e]).v * y[e];
          m = fmaxf(m, fabsf(h[e]));
        }
        if (a.gate && there) at.put(a.gate + v * a.ld_gate, c, x, c0 + HB <= a.f), at.put(a.up + v * a.ld_up, c, y, c0 + HB <= a.f);
        at.put_frag(a.H, a.KSH, n0 / 32 + j, c0 / 16 + (k >> 1), k & 1, h);
      }
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      if (half == 0) top[wave * NR + j * 32 + l32] = __builtin_amdgcn_ldexpf(m, -ed);
    }
    __syncthreads();
    if (tid < NR && n0 + tid < a.n) raise(a.h_row + n0 + tid, __float_as_uint(fmaxf(fmaxf(top[tid], top[NR + tid]), fmaxf(top[2 * NR + tid], top[3 * NR + tid]))));
  }
  if constexpr (MODE == BACK) {
    float md[NJ] = {};
    float* cols = top + 4 * NR;
    int ey[NJ];
    const float *gate[NJ], *up[NJ];
    const bool last = n0 + NR > a.n;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t v = n0 + j * 32 + l32, row = v < a.n ? v : a.n - 1;
      ey[j] = a.e_in[v];
      gate[j] = a.gate + row * a.ld_gate, up[j] = a.up + row * a.ld_up;
    }
    auto part = [&](const v16f (&sums)[NJ], int i) __attribute__((always_inline)) {
      const int64_t c0 = mw + i * HB;
      const int e0 = a.e_w[c0 / HB];
      float m[NJ];
      at.back<ACT, NJ>(n0 / 32, c0 / HB, m, cols + (wave * 2 + i) * 96, [&](int j, int k, V4& x, V4& y) {
        const int64_t c = c0 + k * 8 + half * 4;
        x = at.get(gate[j], c, c0 + HB <= a.f), y = at.get(up[j], c, c0 + HB <= a.f);
        if (last && n0 + j * 32 + l32 >= a.n) x = y = V4{0.f, 0.f, 0.f, 0.f};
      }, [&](int j, int k, int e) { return __builtin_amdgcn_ldexpf(sums[j][k * 4 + e], -(ey[j] + e0)); });
#pragma unroll
      for (int j = 0; j < NJ; ++j) md[j] = fmaxf(md[j], m[j]);
    };
    part(acc[0], 0);
    part(acc[1], 1);
    at.back_tops<NJ, 8>(n0 / 32, m0, md, cols, top);
  }
}

template <int MODE, int ACT>
__global__ void __launch_bounds__(256, 2) k_ffn_split(Args a) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(MODE == ROWS || is_cols(MODE))];
  ffn_split<MODE, ACT>(a, blockIdx.x, Bs);
}
// By 64 rows.  BACK has 199 registers: three blocks a CU would keep 35 of them in memory (30,000 x 128 x 512 91 -> 117 us, 8,192 x 1,024 x 4,096 341 -> 353); half as many hidden columns
// by 128 rows take as long (356).
template <int MODE, int ACT>
__global__ void __launch_bounds__(256, MODE == BACK ? 2 : 3) k_ffn_narrow(Args a) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(false)];
  ffn_split<MODE, ACT>(a, blockIdx.x, Bs);
}
// dX, and the gradients of the weights, which do not wait for each other, behind each other's blocks where all of them run at once.
struct EndsArgs {
  Args a[3];                           // ROWS, COLS, COLS
  unsigned first[3];                   // blocks before each
};
template <int COLS_D, int COLS_H>
__global__ void __launch_bounds__(256, 2) k_ffn_ends(EndsArgs ends) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(true)];
  if (blockIdx.x < ends.first[1]) return ffn_split<ROWS, 0>(ends.a[0], blockIdx.x, Bs);
  if constexpr (COLS_D == COLS_H) {
    const int k = blockIdx.x < ends.first[2] ? 1 : 2;
    return ffn_split<COLS_D, 0>(ends.a[k], blockIdx.x - ends.first[k], Bs);
  }
  if (blockIdx.x < ends.first[2]) ffn_split<COLS_D, 0>(ends.a[1], blockIdx.x - ends.first[1], Bs);
  else ffn_split<COLS_H, 0>(ends.a[2], blockIdx.x - ends.first[2], Bs);
}

// PROJECT and BACK in one where A and B were not kept: 128 hidden columns by 64 rows, 32 by 64 a wave, first A and B, then G; three blocks a CU, which is what hides their ends.  (Of 96
// rows, two blocks: 232,965 x 256 x 1,024 1,690 -> 1,790 us, 16,384 x 512 x 2,048 417 -> 456, but 8,192 x 1,024 x 4,096 733 -> 702; the sums of 128 would take 192 registers.)
constexpr int REMAKE_ROWS = 64;
static_assert(REMAKE_ROWS % PAIR == 0 && TM % REMAKE_ROWS == 0, "COLS reads whole pairs of stages; pieces are multiples of TM rows");
struct RemakeArgs {
  Args a;                              // A, B, KSA, KSB, pairs, e_w, e_in: the projections'
  const _Float16 *A2, *B2;
  int64_t KS2, pairs2;
  const int *e_w2, *e_in2;
};
template <int ACT>
__global__ void __launch_bounds__(256, 3) k_ffn_remake(RemakeArgs r) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(false)];
  const Args& a = r.a;
  const Tile tile(blockIdx.x, a.mt, a.nt, 1);
  if (tile.m < 0) return;
  constexpr int NJ = REMAKE_ROWS / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t hb = tile.m * 4 + wave, b0 = tile.n * NJ;            // the wave's hidden block, the tile's first row block
  v16f ab[2][NJ], gr[1][NJ];
  const auto a_as_it_is = [](v8h (&)[2], int, int) {};
  const auto b_as_it_is = [](v8h (&)[NJ], int) {};
  clear(ab);
  multiply<false, false>(ab, a.A + hb * 2 * a.KSA * 2 * FRAG + lane * 8, a.KSA * 2 * FRAG, a.B + b0 * a.KSB * 2 * FRAG, a.KSB * 2 * FRAG, nullptr, (int)a.pairs, Bs, a_as_it_is, b_as_it_is);
  clear(gr);
  multiply<false, false>(gr, r.A2 + hb * r.KS2 * 2 * FRAG + lane * 8, 0, r.B2 + b0 * r.KS2 * 2 * FRAG, r.KS2 * 2 * FRAG, nullptr, (int)r.pairs2, Bs, a_as_it_is, b_as_it_is);
  const int e0 = a.e_w[hb * 2], e1 = a.e_w[hb * 2 + 1], e2 = r.e_w2[hb];
  const Hidden at(a);
  float md[NJ];
  float *top = reinterpret_cast<float*>(Bs), *cols = top + 4 * NJ * 32;
  int ex[NJ], ey[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) ex[j] = a.e_in[(b0 + j) * 32 + (lane & 31)], ey[j] = r.e_in2[(b0 + j) * 32 + (lane & 31)];
  at.back<ACT, NJ>(b0, hb, md, cols + wave * 96, [&](int j, int k, V4& x, V4& y) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[e] = __builtin_amdgcn_ldexpf(ab[0][j][k * 4 + e], -(ex[j] + e0)), y[e] = __builtin_amdgcn_ldexpf(ab[1][j][k * 4 + e], -(ex[j] + e1));
  }, [&](int j, int k, int e) { return __builtin_amdgcn_ldexpf(gr[0][j][k * 4 + e], -(ey[j] + e2)); });
  at.back_tops<NJ, 4>(b0, tile.m * 4 * HB, md, cols, top);
}

#include "ht_ffn_stream.h"

constexpr int JOIN_MANY = 32;
__global__ void __launch_bounds__(256) k_ffn_join(FfnJoins joins) {
  int k = 0;
#pragma unroll
  for (int i = 1; i < FFN_JOINS; ++i) k += blockIdx.x >= joins.first[i];
  const unsigned block = blockIdx.x - joins.first[k];
  const FfnJoin& a = joins.join[k];
  // eight lanes a value where there are many parts of few values
  const int sub = a.parts >= JOIN_MANY ? threadIdx.x & 7 : 0, subs = a.parts >= JOIN_MANY ? 8 : 1;
  const int64_t nv = a.pitch / 4, i = ((int64_t)block * 256 + threadIdx.x) / subs, r = i / nv, c = (i - r * nv) * 4;
  if (r >= a.rows || c >= a.cols) return;      // (all eight of them)
  V4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = sub; p < a.parts; p += subs) s += *reinterpret_cast<const V4*>(a.sums + p * a.part + r * a.pitch + c);
  if (subs > 1) {
    for (int o = 1; o < 8; o <<= 1) s += V4{__shfl_xor(s[0], o, 64), __shfl_xor(s[1], o, 64), __shfl_xor(s[2], o, 64), __shfl_xor(s[3], o, 64)};
    if (sub > 0) return;
  }
  float* to = a.out + r * a.ld + c;
  if (c + 4 <= a.cols) {
    if (a.add) s += *reinterpret_cast<const V4u*>(to);
    *reinterpret_cast<V4u*>(to) = s;
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (c + e < a.cols) to[e] = a.add ? to[e] + s[e] : s[e];
}

// ---------------------------------------------------------------- plan

constexpr size_t FFN_BYTES = (size_t)4 << 30, FFN_LEAN = (size_t)64 << 20;     // of what a piece's rows take, at most and where there is no room for more
constexpr int64_t SLOTS = 512;                     // blocks that run together: two a CU
constexpr int64_t LEAST_PAIRS = 4;                 // of a part of a reduction, where a product has a launch for itself

constexpr int64_t SHORT_PAIRS = 8;
// Weights that are read once (ht_ffn_stream.h) against packed ones, us: forward 128 x 1,024 x 4,096 41 | 89, 512 x 512 x 2,048 43 | 53, 1,003 x 301 x 1,213 36 | 44, 2,048 x 256 x 1,024 38 | 42, 1,003 x 512 x 2,048 53 | 60,
// 2,048 x 512 x 1,024 55 | 56, 1,024 x 1,024 x 4,096 142 | 140; with more work, 256 x 2,048 x 8,192 136 | 245, 512 x 1,024 x 4,096 79 | 96, 512 x 2,048 x 8,192 251 | 287, 512 x 4,096 x 16,384
// 1,039 | 1,042; backward 128 x 1,024 x 4,096 90 | 130, 256 x 512 x 2,048 72 | 75, 256 x 256 x 1,024 59 | 52, 384 x 1,024 x 4,096 186 | 160.
constexpr int64_t STREAM_ROWS = 512, STREAM_ROWS_MOST = 2048, STREAM_WORK = (int64_t)7 << 29, STREAM_ROWS_BWD = 256, STREAM_WEIGHTS_BWD = (int64_t)1 << 21;
constexpr int64_t STREAM_BLOCKS = 256;             // of Y or dX, at most: one a CU

// The products behind H, dA and dB: their tiles, pairs of stages of a tile's reduction, and the parts that it is cut into.
struct Ends {
  int64_t tiles[3], pairs[3];
  int parts[3] = {1, 1, 1};
  bool one = false;                                // one launch for all of them
  int64_t blocks(int64_t most) const {             // with parts of at most so many pairs
    int64_t n = 0;
    for (int k = 0; k < 3; ++k) n += tiles[k] * ceil_div64(pairs[k], most);
    return n;
  }
  int64_t fit(int64_t room) const {                // parts that leave no more blocks than that (0: there are none)
    if (tiles[0] + tiles[1] + tiles[2] > room) return 0;
    int64_t most = 1;
    for (int k = 0; k < 3; ++k) most += tiles[k] * pairs[k] / room;
    while (blocks(most) > room) most += (most + 15) / 16;
    return most;
  }
  Ends(int64_t t0, int64_t p0, int64_t t1, int64_t p1, int64_t t2, int64_t p2) : tiles{t0, t1, t2}, pairs{p0, p1, p2} {
    // A CU for each block where its part is short (a block that is alone waits for every stage's loads, but then its sums are few), else two.  us of a call, in one
    // launch | each in its own: 500 x 128 x 512 backward 54 | 103, 2,048 x 256 x 1,024 78 | 120, 4,096 x 768 x 2,048 378 | 442, 16,384 x 512 x 2,048 965 | 967.
    int64_t most = fit(SLOTS / 2);
    if (most == 0 || most > SHORT_PAIRS) most = fit(SLOTS);
    one = most > 0;
    for (int k = 0; k < 3; ++k) {
      const int64_t n = one ? ceil_div64(pairs[k], most) : tiles[k] > 0 ? std::min(SLOTS / tiles[k], pairs[k] / LEAST_PAIRS) : 1;
      parts[k] = (int)std::max<int64_t>(1, std::min<int64_t>(n, 512));
    }
  }
};

template <class F>
void with_act(int act, F&& launch) {   // launch(std::integral_constant<int, act>())
  switch (act) {
    case HT_GATE_SILU: return launch(std::integral_constant<int, HT_GATE_SILU>());
    case HT_GATE_GELU: return launch(std::integral_constant<int, HT_GATE_GELU>());
    case HT_GATE_GELU_TANH: return launch(std::integral_constant<int, HT_GATE_GELU_TANH>());
    case HT_GATE_RELU: return launch(std::integral_constant<int, HT_GATE_RELU>());
    default: return launch(std::integral_constant<int, HT_GATE_SIGMOID>());
  }
}

struct Ffn : FfnCall {
  static int64_t blocks_of(const Args& a) { return up_to(a.mt * a.nt * a.splits, 8); }
  int launch(int mode, const Args& a) const {
    const int64_t blocks = blocks_of(a);
    if (blocks >= (1 << 24)) return ht_set_err(ctx, HT_ESHAPE, "ffn: %lld tiles in one product", (long long)blocks);
    const unsigned grid = (unsigned)blocks;
    switch (mode) {
      case PROJECT: with_act(D->act, [&](auto act) { k_ffn_split<PROJECT, decltype(act)::value><<<grid, 256, 0, ctx->stream>>>(a); }); break;
      case PROJECT_SMALL: with_act(D->act, [&](auto act) { k_ffn_narrow<PROJECT_SMALL, decltype(act)::value><<<grid, 256, 0, ctx->stream>>>(a); }); break;
      case BACK: with_act(D->act, [&](auto act) { k_ffn_narrow<BACK, decltype(act)::value><<<grid, 256, 0, ctx->stream>>>(a); }); break;
      case ROWS: k_ffn_split<ROWS, 0><<<grid, 256, 0, ctx->stream>>>(a); break;
      case COLS: k_ffn_split<COLS, 0><<<grid, 256, 0, ctx->stream>>>(a); break;
      default: k_ffn_split<COLS_SMALL, 0><<<grid, 256, 0, ctx->stream>>>(a);
    }
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  }
  int stream_hidden(const StreamHidden& s) const {
    const unsigned grid = (unsigned)up_to(s.row_tiles * ceil_div64(s.a.f, HB), 8);
    if (dY) (in_out() ? k_stream_hidden<true, true> : k_stream_hidden<false, true>)<<<grid, HIDDEN_WAVES * 64, 0, ctx->stream>>>(s);
    else (in_out() ? k_stream_hidden<true, false> : k_stream_hidden<false, false>)<<<grid, HIDDEN_WAVES * 64, 0, ctx->stream>>>(s);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  }
  int stream_out(const StreamOut& s) const {
    const unsigned grid = (unsigned)up_to(s.row_tiles * ceil_div64(s.width, 32) * s.splits, 8);
    if (dY) (in_out() ? k_stream_out<2, true> : k_stream_out<2, false>)<<<grid, OUT_WAVES * 64, 0, ctx->stream>>>(s);
    else (in_out() ? k_stream_out<1, false> : k_stream_out<1, true>)<<<grid, OUT_WAVES * 64, 0, ctx->stream>>>(s);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  }
  int64_t weights() const { return (int64_t)D->d_hidden * (2 * (int64_t)D->d_in + D->d_out); }
  bool streamed() const {
    if (std::max({Wg->ld, Wu->ld, Wd->ld}) > STREAM_LD) return false;
    const int64_t n = X->rows;
    return dY ? n <= STREAM_ROWS_BWD && weights() >= STREAM_WEIGHTS_BWD : n <= STREAM_ROWS || (n <= STREAM_ROWS_MOST && n * weights() <= STREAM_WORK);
  }
  int run(size_t bytes) const {
    const bool bwd = dY != nullptr, in_out = this->in_out();
    const int64_t n = X->rows, d = D->d_in, f = D->d_hidden, e = D->d_out;
    hipStream_t st = ctx->stream;
    const int64_t fp = up_to(f, 256), dp = up_to(d, TM), ep = up_to(e, TM), KSd = up_to(d, TN) / 16, KSe = up_to(e, TN) / 16, KSH = fp / 16, KSD = fp / 8;
    const bool remake = bwd && !gate, d_w = dWg || dWu;
    // a row's share
    const int64_t own = 4 * (dp + (bwd && d_w ? dp : 0) + (bwd ? ep : 0) + (bwd && dWd ? ep : 0) + fp * (bwd ? 3 : 1));
    const int64_t Rp = std::max<int64_t>(TM, std::min<int64_t>((int64_t)bytes / own / TM * TM, up_to(n, TM)));
    const int64_t KSR = Rp / 16, pieces = ceil_div64(n, Rp);
    // tiles of the products, and parts of their reductions
    const int64_t mt = Rp / TM, nte = up_to(e, TN) / TN, ntd = up_to(d, TN) / TN, ntD = ceil_div64(f, 64), ntH = ceil_div64(f, TN);
    const int64_t pairs_f = ceil_div64(f, PAIR), pairs_2f = ceil_div64(f, HB), pairs_r = ceil_div64(std::min(n, Rp), PAIR);
    const int cols_D = d <= TN ? COLS_SMALL : COLS, cols_H = e <= TN ? COLS_SMALL : COLS;
    const int64_t mtD = cols_D == COLS ? dp / TM : 1, mtH = cols_H == COLS ? ep / TM : 1;
    const bool streamed = this->streamed();
    const Ends ends(streamed ? 0 : Y ? mt * nte : dX ? mt * ntd : 0, Y ? pairs_f : pairs_2f, d_w ? mtD * ntD : 0, pairs_r, dWd ? mtH * ntH : 0, pairs_r);
    const int64_t tiles = ceil_div64(std::min(n, Rp), STREAM_TILE), out_tiles = tiles * ceil_div64(Y ? e : d, 32);
    const int64_t out_parts = std::max<int64_t>(1, std::min(STREAM_BLOCKS / out_tiles, f / (OUT_WAVES * 32)));
    const int sy = streamed ? (int)out_parts : ends.parts[0], sx = sy, sD = ends.parts[1], sH = ends.parts[2];
    const int64_t e4 = up_to(e, 4), d4 = up_to(d, 4), f4 = up_to(f, 4);
    // a weight's gradient as it lies: rows and pitch of its parts
    const int64_t wr = in_out ? d : f, wp = in_out ? f4 : d4, vr = in_out ? f : e, vp = in_out ? e4 : f4;

    OpsBlock m;
    const int64_t n_top = 2 * Rp + 3 * fp;                 // largest values: rows of H, of dA and dB, columns of H, dA, dB
    const auto top = m.add<uint32_t>(n_top);
    const auto ex = m.add<int>(Rp), ey = m.add<int>(Rp), exb = m.add<int>(Rp / HB), eyb = m.add<int>(Rp / HB), ew2 = m.add<int>(2 * fp / HB), ewd = m.add<int>(fp / HB);
    const auto W2 = m.add<_Float16>(streamed ? 0 : 2 * fp * KSd * 32), Wf = m.add<_Float16>(streamed ? 0 : fp * KSe * 32);
    const auto Xr = m.add<_Float16>(Rp * KSd * 32);
    const auto Xt = m.add<_Float16>(d_w ? dp * KSR * 32 : 0);
    const auto Gr = m.add<_Float16>(bwd ? Rp * KSe * 32 : 0);
    const auto Gt = m.add<_Float16>(dWd ? ep * KSR * 32 : 0);
    const auto H = m.add<float>(Rp * fp), Df = m.add<float>(bwd ? Rp * fp * 2 : 0);
    const auto sums_y = m.add<float>(!bwd && sy > 1 ? sy * Rp * e4 : 0), sums_x = m.add<float>(dX && sx > 1 ? sx * Rp * d4 : 0);
    const auto sums_D = m.add<float>(d_w && sD > 1 ? sD * 2 * wr * wp : 0), sums_H = m.add<float>(dWd && sH > 1 ? sH * vr * vp : 0);
    HT_TRY(bytes > FFN_LEAN ? m.take_if_room(ctx) : m.take(ctx));

    uint32_t *h_row = m.at(top), *d_row = h_row + Rp, *h_col = d_row + Rp, *a_col = h_col + fp, *b_col = a_col + fp;
    for (int64_t k = 0; k < pieces; ++k) {
      const int64_t r0 = k * Rp, rows = std::min(Rp, n - r0);
      Packs packs{};
      unsigned blocks = 0;
      auto operand = [&](Pack q, int64_t own) {                         // (zeros up to so many of its own)
        q.tiles = (int)ceil_div64(q.run, PACK_RUN), q.blocks = (unsigned)(own / HB);
        q.steps = (int)(up_to(q.run, PAIR) / 16), q.blocks_t = (int)ceil_div64(q.run, 32);
        blocks += q.blocks;
        packs.pack[packs.n++] = q;
      };
      operand(Pack{X->ptr + r0 * X->ld, X->ld, rows, d, 0, m.at(ex), m.at(exb), m.at(Xr), KSd, 1, 0, d_w ? m.at(Xt) : nullptr, KSR}, up_to(rows, TM));
      if (bwd)
        operand(Pack{dY->ptr + r0 * dY->ld, dY->ld, rows, e, 0, m.at(ey), m.at(eyb), m.at(Gr), KSe, 1, 0, dWd ? m.at(Gt) : nullptr, KSR}, up_to(rows, TM));
      if (k == 0 && !streamed) {
        // by hidden columns: the rows of an OUT_IN Wg, the columns of an IN_OUT one
        operand(Pack{Wg->ptr, Wg->ld, f, d, in_out, nullptr, m.at(ew2), m.at(W2), KSd, 2, 0, nullptr, 0}, fp);
        operand(Pack{Wu->ptr, Wu->ld, f, d, in_out, nullptr, m.at(ew2), m.at(W2), KSd, 2, 1, nullptr, 0}, fp);
        operand(Pack{Wd->ptr, Wd->ld, f, e, !in_out, nullptr, m.at(ewd), m.at(Wf), KSe, 1, 0, nullptr, 0}, fp);
      }
      const unsigned share = (unsigned)std::max<int64_t>(1, PACK_BLOCKS / blocks);
      blocks = 0;
      for (int i = 0; i < packs.n; ++i) {
        Pack& q = packs.pack[i];
        q.share = std::min(share, (unsigned)q.tiles);
        packs.first[i] = blocks;
        blocks += q.blocks *= q.share;
      }
      for (int i = packs.n; i <= PACKS; ++i) packs.first[i] = blocks;
      packs.zero = h_row, packs.zeros = n_top;
      k_ffn_pack<<<blocks + (unsigned)ceil_div64(n_top, ZEROS), 256, 0, st>>>(packs);
      HT_LAUNCH_CHECK(ctx);

      Args base{};
      base.n = rows, base.f = f, base.splits = 1;
      base.h_row = h_row, base.d_row = d_row, base.h_col = h_col, base.a_col = a_col, base.b_col = b_col;
      base.e_x = m.at(exb), base.e_y = m.at(eyb);
      base.KSH = KSH, base.KSD = KSD;
      base.gate = gate ? gate->ptr + r0 * gate->ld : nullptr, base.ld_gate = gate ? gate->ld : 0;
      base.up = up ? up->ptr + r0 * up->ld : nullptr, base.ld_up = up ? up->ld : 0;
      const int64_t row_tiles = ceil_div64(rows, TN);
      Args a = base;
      a.H = m.at(H);
      FfnJoins j{};
      if (streamed) {
        a.D = bwd ? m.at(Df) : nullptr;
        HT_TRY(stream_hidden(StreamHidden{a, {Wg->ptr, Wu->ptr, Wd->ptr}, {Wg->ld, Wu->ld, Wd->ld}, d, e, m.at(Xr), bwd ? m.at(Gr) : nullptr, KSd, KSe, m.at(ex),
                                          m.at(ey), D->act, !gate, (int)ceil_div64(rows, STREAM_TILE)}));
        if (const ht_tensor* to = Y ? Y : dX) {
          const int64_t cols = Y ? e : d, pitch = up_to(cols, 4);
          float *out = to->ptr + r0 * to->ld, *sums = Y ? m.at(sums_y) : m.at(sums_x);
          const bool parts = sy > 1;
          StreamOut o{rows, f, cols, {Y ? Wd->ptr : Wg->ptr, Wu->ptr}, {Y ? Wd->ld : Wg->ld, Wu->ld}, (const _Float16*)(Y ? m.at(H) : m.at(Df)), Y ? KSH : KSD, {h_row, d_row},
                      sy, (int)ceil_div64(rows, STREAM_TILE), parts ? sums : out, parts ? pitch : to->ld, Rp * pitch, !parts && D->accumulate};
          if (parts) j.join[j.n++] = FfnJoin{sums, Rp * pitch, pitch, rows, cols, sy, D->accumulate, out, to->ld};
          HT_TRY(stream_out(o));
        }
      } else if (!bwd || remake) {
        a.A = m.at(W2), a.KSA = KSd, a.B = m.at(Xr), a.KSB = KSd;
        a.mt = ceil_div64(f, TN), a.nt = row_tiles, a.pairs = ceil_div64(d, PAIR);
        a.e_w = m.at(ew2), a.e_in = m.at(ex);
        a.e_d = m.at(ewd);
        if (!bwd) {
          // (half tiles where whole ones fill less than half of the places, us of whole ones -> of half ones: 128 tiles, 1,024 x 1,024 x 2,048 101 -> 89, 4,096 x 512 x 512 62 -> 56, 4,096 x 128 x
          // 512 41 -> 38; 192, 4,096 x 512 x 768 67.2 -> 66.7; 216, 2,304 x 512 x 1,536 68.6 -> 68.4; 240, 1,024 x 1,024 x 3,840 123 -> 126.  Of more tiles they only read more: 16,384 x 1,024 x
          // 4,096 1,114 -> 1,192)
          const bool small = a.mt * a.nt < SLOTS / 2;
          if (small) a.nt = ceil_div64(rows, TN / 2);
          HT_TRY(launch(small ? PROJECT_SMALL : PROJECT, a));
        }
      }
      if (bwd) a.D = m.at(Df), a.e_d = m.at(ew2);
      if (streamed) {
      } else if (remake) {
        a.nt = ceil_div64(rows, REMAKE_ROWS);
        const RemakeArgs r{a, m.at(Wf), m.at(Gr), KSe, ceil_div64(e, PAIR), m.at(ewd), m.at(ey)};
        with_act(D->act, [&](auto act) { k_ffn_remake<decltype(act)::value><<<(unsigned)up_to(a.mt * a.nt, 8), 256, 0, st>>>(r); });
        HT_LAUNCH_CHECK(ctx);
      } else if (bwd) {
        a.A = m.at(Wf), a.KSA = KSe, a.B = m.at(Gr), a.KSB = KSe;
        a.mt = ceil_div64(f, TM), a.nt = ceil_div64(rows, TN / 2), a.pairs = ceil_div64(e, PAIR);
        a.e_w = m.at(ewd), a.e_in = m.at(ey);
        HT_TRY(launch(BACK, a));
      }
      // Y, or dX; their parts' sums are added up behind each piece, those of the weights' gradients behind the last
      auto by_rows = [&](const ht_tensor* to, const float* P, int64_t KSP, bool two, const _Float16* W, int64_t KSW, const int* e_w, int64_t cols, int64_t nt,
                         int64_t pairs, int splits, float* sums, int64_t pitch) {
        Args a = base;
        a.A = (const _Float16*)P, a.KSA = KSP, a.B = W, a.KSB = KSW;
        a.mt = ceil_div64(rows, TM), a.nt = nt, a.pairs = pairs, a.splits = splits, a.two = two, a.e_w = e_w;
        a.m_end = rows, a.n_end = cols;
        float* out = to->ptr + r0 * to->ld;
        a.out[0] = splits > 1 ? Out{sums, pitch, 1, Rp * pitch} : Out{out, to->ld, 1, 0};
        a.add = splits == 1 && D->accumulate;
        if (splits > 1) j.join[j.n++] = FfnJoin{sums, Rp * pitch, pitch, rows, cols, splits, D->accumulate, out, to->ld};
        return a;
      };
      auto by_cols = [&](const _Float16* At, const int* e_rows, int64_t m_end, const float* P, int64_t KSP, bool two, int64_t tiles_m, int64_t nt, int splits, float* sums,
                         int64_t r, int64_t pitch, const ht_tensor* o0, const ht_tensor* o1, bool m_is_row) {
        Args a = base;
        a.A = At, a.KSA = KSR, a.B = (const _Float16*)P, a.KSB = KSP;
        a.mt = tiles_m, a.nt = nt, a.pairs = ceil_div64(rows, PAIR), a.splits = splits, a.two = two, a.e_w = e_rows;
        a.m_end = m_end, a.n_end = f;
        const ht_tensor* o[2] = {o0, o1};
        for (int i = 0; i < 2; ++i) {
          if (!o[i]) continue;
          const int64_t ld = splits > 1 ? pitch : o[i]->ld;
          a.out[i] = Out{splits > 1 ? sums + i * r * pitch : o[i]->ptr, m_is_row ? ld : 1, m_is_row ? 1 : ld, splits > 1 ? (two ? 2 : 1) * r * pitch : 0};
          if (splits > 1 && k + 1 == pieces)
            j.join[j.n++] = FfnJoin{sums + i * r * pitch, (two ? 2 : 1) * r * pitch, pitch, o[i]->rows, o[i]->cols, splits, D->accumulate_dW, o[i]->ptr, o[i]->ld};
        }
        a.add = k > 0 || (splits == 1 && D->accumulate_dW);
        return a;
      };
      if (Y && !streamed) HT_TRY(launch(ROWS, by_rows(Y, m.at(H), KSH, false, m.at(Wf), KSe, m.at(ewd), e, nte, pairs_f, sy, m.at(sums_y), e4)));
      Args ax{}, ad{}, ah{};                             // (no tiles: not asked for)
      if (dX && !streamed) ax = by_rows(dX, m.at(Df), KSD, true, m.at(W2), KSd, m.at(ew2), d, ntd, pairs_2f, sx, m.at(sums_x), d4);
      if (d_w) ad = by_cols(m.at(Xt), m.at(exb), d, m.at(Df), KSD, true, mtD, ntD, sD, m.at(sums_D), wr, wp, dWg, dWu, in_out);
      if (dWd) ah = by_cols(m.at(Gt), m.at(eyb), e, m.at(H), KSH, false, mtH, ntH, sH, m.at(sums_H), vr, vp, dWd, nullptr, !in_out);
      const int64_t bx = blocks_of(ax), bd = blocks_of(ad), bh = blocks_of(ah);
      if (bwd && ends.one) {
        const auto kernel = cols_D == COLS ? (cols_H == COLS ? k_ffn_ends<COLS, COLS> : k_ffn_ends<COLS, COLS_SMALL>)
                                           : (cols_H == COLS ? k_ffn_ends<COLS_SMALL, COLS> : k_ffn_ends<COLS_SMALL, COLS_SMALL>);
        if (bx + bd + bh > 0) kernel<<<(unsigned)(bx + bd + bh), 256, 0, st>>>(EndsArgs{{ax, ad, ah}, {0, (unsigned)bx, (unsigned)(bx + bd)}});
        HT_LAUNCH_CHECK(ctx);
      } else {
        if (bx) HT_TRY(launch(ROWS, ax));
        if (bd) HT_TRY(launch(cols_D, ad));
        if (bh) HT_TRY(launch(cols_H, ah));
      }
      HT_TRY(ht_ffn_join(ctx, j));
    }
    return HT_OK;
  }
  int call() const {
    if (X->rows == 0) {                // nothing to add up
      FfnJoins w{};
      for (const ht_tensor* t : {dWg, dWu, dWd})
        if (t && !D->accumulate_dW) w.join[w.n++] = FfnJoin{nullptr, 0, up_to(t->cols, 4), t->rows, t->cols, 0, 0, t->ptr, t->ld};
      return ht_ffn_join(ctx, w);
    }
    if (X->rows <= (weights() < FEW_WEIGHTS || !streamed() ? HT_FFN_FEW : 16)) return ht_ffn_few(*this);
    // Half as large pieces as long as there is no room for larger ones (nothing has been launched by a call that is refused memory): with 1 GB to spend 232,965 x 256 x 1,024 backward
    // takes 3.79 ms, of pieces of 64 MiB 5.85, with all it needs 3.76.
    int rc = HT_ENOMEM;
    for (size_t bytes = FFN_BYTES; rc == HT_ENOMEM && bytes >= FFN_LEAN; bytes /= 2) rc = run(bytes);
    return rc;
  }
};

struct Named {
  const ht_tensor* t;
  const char* name;
};
// Outputs that are there share no memory with inputs and with each other.
int check_apart(ht_ctx* ctx, const char* call, std::initializer_list<Named> in, std::initializer_list<Named> out) {
  for (auto o = out.begin(); o != out.end(); ++o) {
    if (!o->t) continue;
    for (const Named& i : in)
      if (i.t && ht_shares(o->t, i.t)) return ht_set_err(ctx, HT_EINVAL, "%s: %s shares memory with %s", call, o->name, i.name);
    for (auto p = out.begin(); p != o; ++p)
      if (p->t && ht_shares(o->t, p->t)) return ht_set_err(ctx, HT_EINVAL, "%s: %s shares memory with %s", call, o->name, p->name);
  }
  return HT_OK;
}

int check_block(ht_ctx* ctx, const char* call, const ht_ffn_desc* D, const ht_tensor* X, const ht_tensor* Wg, const ht_tensor* Wu, const ht_tensor* Wd, const ht_tensor* gate,
                const ht_tensor* up, const ht_tensor* Y) {
  if (!D || !X || !Wg || !Wu || !Wd || !Y) return ht_set_err(ctx, HT_EINVAL, "%s: null argument", call);
  for (int32_t w : {D->d_in, D->d_hidden, D->d_out})
    if (w <= 0 || w > HT_FFN_MAX_WIDTH) return ht_set_err(ctx, HT_ESHAPE, "%s: width %d, must be 1 .. %d", call, w, HT_FFN_MAX_WIDTH);
  if (D->act < HT_GATE_SILU || D->act > HT_GATE_SIGMOID) return ht_set_err(ctx, HT_EINVAL, "%s: unknown activation %d", call, D->act);
  if (D->w_form != HT_W_IN_OUT && D->w_form != HT_W_OUT_IN) return ht_set_err(ctx, HT_EINVAL, "%s: unknown form of weights %d", call, D->w_form);
  if (!gate != !up) return ht_set_err(ctx, HT_EINVAL, "%s: gate and up go together", call);
  const std::string c = std::string(call) + ": ";
  HT_TRY(ht_check_rows(ctx, X, X->rows, D->d_in, (c + "X").c_str()));
  const bool in_out = D->w_form == HT_W_IN_OUT;
  const int32_t r = in_out ? D->d_in : D->d_hidden, cols = in_out ? D->d_hidden : D->d_in;
  HT_TRY(ht_check_weights(ctx, Wg, r, cols, (c + "Wg").c_str()));
  HT_TRY(ht_check_weights(ctx, Wu, r, cols, (c + "Wu").c_str()));
  HT_TRY(ht_check_weights(ctx, Wd, in_out ? D->d_hidden : D->d_out, in_out ? D->d_out : D->d_hidden, (c + "Wd").c_str()));
  HT_TRY(ht_check_rows(ctx, Y, X->rows, D->d_out, (c + "Y or dY").c_str()));
  if (gate) {
    HT_TRY(ht_check_rows(ctx, gate, X->rows, D->d_hidden, (c + "gate").c_str()));
    HT_TRY(ht_check_rows(ctx, up, X->rows, D->d_hidden, (c + "up").c_str()));
  }
  return HT_OK;
}

}  // namespace

int ht_ffn_join(ht_ctx* ctx, FfnJoins& j) {
  unsigned grid = 0;
  for (int k = 0; k < j.n; ++k) {
    FfnJoin& a = j.join[k];
    j.first[k] = grid;
    grid += (unsigned)ceil_div64(a.rows * (a.pitch / 4) * (a.parts >= JOIN_MANY ? 8 : 1), 256);
  }
  for (int k = j.n; k < FFN_JOINS; ++k) j.first[k] = grid;
  if (grid == 0) return HT_OK;
  k_ffn_join<<<grid, 256, 0, ctx->stream>>>(j);
  HT_LAUNCH_CHECK(ctx);
  return HT_OK;
}

extern "C" int ht_ffn_fwd(ht_ctx* ctx, const ht_ffn_desc* desc, const ht_tensor* X, const ht_tensor* Wg, const ht_tensor* Wu, const ht_tensor* Wd, ht_tensor* Y, ht_tensor* gate,
                          ht_tensor* up) {
  if (!ctx) return HT_EINVAL;
  HT_TRY(check_block(ctx, "ht_ffn_fwd", desc, X, Wg, Wu, Wd, gate, up, Y));
  HT_TRY(check_apart(ctx, "ht_ffn_fwd", {{X, "X"}, {Wg, "Wg"}, {Wu, "Wu"}, {Wd, "Wd"}}, {{Y, "Y"}, {gate, "gate"}, {up, "up"}}));
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const Ffn op{{ctx, desc, X, Wg, Wu, Wd, gate, up, Y, nullptr, nullptr, nullptr, nullptr, nullptr}};
  return ht_with_room(ctx, [&]() -> int { return op.call(); });
}

extern "C" int ht_ffn_bwd(ht_ctx* ctx, const ht_ffn_desc* desc, const ht_tensor* X, const ht_tensor* Wg, const ht_tensor* Wu, const ht_tensor* Wd, const ht_tensor* gate,
                          const ht_tensor* up, const ht_tensor* dY, ht_tensor* dX, ht_tensor* dWg, ht_tensor* dWu, ht_tensor* dWd) {
  if (!ctx) return HT_EINVAL;
  HT_TRY(check_block(ctx, "ht_ffn_bwd", desc, X, Wg, Wu, Wd, gate, up, dY));
  if (dX) HT_TRY(ht_check_rows(ctx, dX, X->rows, desc->d_in, "ht_ffn_bwd: dX"));
  if (dWg) HT_TRY(ht_check_weights(ctx, dWg, Wg->rows, Wg->cols, "ht_ffn_bwd: dWg"));
  if (dWu) HT_TRY(ht_check_weights(ctx, dWu, Wu->rows, Wu->cols, "ht_ffn_bwd: dWu"));
  if (dWd) HT_TRY(ht_check_weights(ctx, dWd, Wd->rows, Wd->cols, "ht_ffn_bwd: dWd"));
  HT_TRY(check_apart(ctx, "ht_ffn_bwd", {{X, "X"}, {Wg, "Wg"}, {Wu, "Wu"}, {Wd, "Wd"}, {gate, "gate"}, {up, "up"}, {dY, "dY"}},
                     {{dX, "dX"}, {dWg, "dWg"}, {dWu, "dWu"}, {dWd, "dWd"}}));
  HT_HIP(ctx, hipSetDevice(ctx->device));
  if (!dX && !dWg && !dWu && !dWd) return HT_OK;
  const Ffn op{{ctx, desc, X, Wg, Wu, Wd, gate, up, nullptr, dY, dX, dWg, dWu, dWd}};
  return ht_with_room(ctx, [&]() -> int { return op.call(); });
}
