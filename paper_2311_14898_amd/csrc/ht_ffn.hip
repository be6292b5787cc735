// Gated feed-forward blocks:  A = X Wg ;  B = X Wu ;  H = act(A) * B ;  Y = H Wd, and their gradients:
//   G = dY Wd^T ;  dA = G * B * act'(A) ;  dB = G * act(A) ;  dX = dA Wg^T + dB Wu^T ;  dWg = X^T dA ;  dWu = X^T dB ;  dWd = H^T dY
//
// All products are fp32 products on the fp16 matrix cores (ht_split.h).  X, dY and the weights are packed into fragments of split values first: by
// rows, scaled by the largest of each row (of all of a weight); for the gradients of weights also by columns, scaled by the largest of each column.
// The hidden columns of Wg and Wu lie interleaved by 32s, so that one product makes A and B of the same column in the same lane, and dA and dB are one operand
// with a reduction over both.  H, dA and dB are kept in fp32, in the order of fragments, and with the largest values of their rows and columns; the products that
// read them split them as they load: no pass in between, and either scale as the reduction asks for it.
#include <algorithm>

#include "ht_ffn.h"
#include "ht_split.h"

namespace {

constexpr int HB = 32;                 // hidden columns of a block: [gate, up] of interleaved operands

// ---------------------------------------------------------------- scales

// The exponent of the power of two that brings what has its largest absolute value in these bits to [2^14, 2^15).  Largest values are those of
// what is finite: the rest becomes NaN in its split, and takes no bits off the others.  (NONE: there is nothing, or only zeros.)
constexpr int NONE = 1 << 20;
__device__ __forceinline__ int scale_exp(uint32_t bits) {
  if (bits == 0) return NONE;
  const int e = 141 - (int)(bits >> 23);
  return e > 126 ? 126 : e;            // (values below 2^-112 come to less)
}
__device__ __forceinline__ int exp_or_0(int e) { return e >= NONE ? 0 : e; }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)((e < -126 ? -126 : e > 126 ? 126 : e) + 127) << 23); }
__device__ __forceinline__ uint32_t size_bits(float x) {
  const uint32_t b = __float_as_uint(fabsf(x));
  return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ void raise(uint32_t* word, uint32_t m) {       // (most find a word as large as it need be)
  if (__hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < m) atomicMax(word, m);
}

// ---------------------------------------------------------------- operands

// A matrix [rows x cols], pitch ld, of which the largest values are wanted: of each row, of each column, or of all of it (words that hold zeros).
struct Top {
  const float* p;
  int64_t ld, rows, cols;
  uint32_t *rmax, *cmax, *all;         // (null: not wanted)
  unsigned blocks;
};
constexpr int TOPS = 5, TOP_COLS = 256, TOP_UNROLL = 8;
struct Tops {
  Top top[TOPS];
  int n;
};
__host__ __device__ constexpr int top_lanes(int64_t cols) { return cols > 128 ? 64 : cols > 64 ? 32 : 16; }
// Rows of a block at a time, and blocks: each one's words wait for those of the others, so there are not many of them
__host__ __device__ constexpr int top_rows(int64_t cols) { return 4 * TOP_UNROLL * (64 / top_lanes(cols)); }
constexpr int64_t TOP_BLOCKS = 1024;
// lanes of four columns each take a row's TOP_COLS, a wave TOP_UNROLL rows of each of its groups of lanes at a time; columns are joined once a block.
__global__ void __launch_bounds__(256) k_ffn_top(Tops tops) {
  __shared__ __attribute__((aligned(16))) uint32_t sh[4][TOP_COLS];
  unsigned block = blockIdx.x;
  int k = 0;
  while (block >= tops.top[k].blocks) block -= tops.top[k++].blocks;
  const Top& t = tops.top[k];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lpr = top_lanes(t.cols), l = lane & (lpr - 1), groups = 64 / lpr, g = lane / lpr, here = top_rows(t.cols);
  const unsigned cb = (unsigned)((t.cols + TOP_COLS - 1) / TOP_COLS);
  const int64_t c = (int64_t)(block % cb) * TOP_COLS + l * 4;
  uint4 cm = make_uint4(0, 0, 0, 0);
  for (int64_t r0 = (int64_t)(block / cb) * here; r0 < t.rows; r0 += (int64_t)(t.blocks / cb) * here) {
    V4 x[TOP_UNROLL];
#pragma unroll
    for (int q = 0; q < TOP_UNROLL; ++q) {
      const int64_t at = r0 + (wave * TOP_UNROLL + q) * groups + g;
      const float* from = t.p + (at < t.rows ? at : t.rows - 1) * t.ld + c;     // (the last row again, behind it)
      if (c + 4 <= t.cols) {
        x[q] = *reinterpret_cast<const V4u*>(from);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[q][i] = c + i < t.cols ? from[i] : 0.f;
      }
    }
#pragma unroll
    for (int q = 0; q < TOP_UNROLL; ++q) {
      const uint4 b = make_uint4(size_bits(x[q][0]), size_bits(x[q][1]), size_bits(x[q][2]), size_bits(x[q][3]));
      cm = make_uint4(max(cm.x, b.x), max(cm.y, b.y), max(cm.z, b.z), max(cm.w, b.w));
      if (!t.rmax) continue;
      uint32_t m = max(max(b.x, b.y), max(b.z, b.w));
      for (int o = lpr / 2; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
      const int64_t at = r0 + (wave * TOP_UNROLL + q) * groups + g;
      if (l != 0 || at >= t.rows) continue;
      if (cb == 1) t.rmax[at] = m;
      else atomicMax(t.rmax + at, m);
    }
  }
  if (!t.cmax && !t.all) return;
  for (int o = lpr; o < 64; o <<= 1)
    cm = make_uint4(max(cm.x, (uint32_t)__shfl_xor((int)cm.x, o, 64)), max(cm.y, (uint32_t)__shfl_xor((int)cm.y, o, 64)),
                    max(cm.z, (uint32_t)__shfl_xor((int)cm.z, o, 64)), max(cm.w, (uint32_t)__shfl_xor((int)cm.w, o, 64)));
  if (g == 0) *reinterpret_cast<uint4*>(&sh[wave][l * 4]) = cm;
  __syncthreads();
  const int64_t col = (int64_t)(block % cb) * TOP_COLS + threadIdx.x;
  uint32_t m = 0;
  if ((int)threadIdx.x < lpr * 4) m = max(max(sh[0][threadIdx.x], sh[1][threadIdx.x]), max(sh[2][threadIdx.x], sh[3][threadIdx.x]));
  if (t.cmax && (int)threadIdx.x < lpr * 4 && col < t.cols) raise(t.cmax + col, m);
  if (!t.all) return;
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  __syncthreads();
  if (lane == 0) sh[0][wave] = m;
  __syncthreads();
  if (threadIdx.x == 0) raise(t.all, max(max(sh[0][0], sh[0][1]), max(sh[0][2], sh[0][3])));
}

// Fragments of a matrix by rows (R: reduction along columns, KS steps apart) and by columns (T: reduction along rows), zeros behind the last row and column; a
// 64 x 64 tile a block.  Row block b of R is number b mul + add (so of T: its column blocks).
struct Pack {
  const float* p;
  int64_t ld, rows, cols;
  const uint32_t *rmax, *cmax, *all;   // scales: `all` of both, or rows for R and columns for T
  _Float16 *R, *T;
  int64_t KS, KS_t;
  int mul, add;
  unsigned row_tiles, col_tiles;
};
struct Packs {
  Pack pack[TOPS];
  int n;
};
__global__ void __launch_bounds__(256) k_ffn_pack(Packs packs) {
  __shared__ float sh[64][65];
  unsigned block = blockIdx.x;
  int i = 0;
  while (block >= packs.pack[i].row_tiles * packs.pack[i].col_tiles) block -= packs.pack[i].row_tiles * packs.pack[i].col_tiles, ++i;
  const Pack& a = packs.pack[i];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
  const int64_t r0 = (int64_t)(block / a.col_tiles) * 64, c0 = (int64_t)(block % a.col_tiles) * 64;
  const int c4 = (lane & 15) * 4, rq = wave * 16 + (lane >> 4);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t r = r0 + rq + q * 4;
    const float* at = a.p + (r < a.rows ? r : a.rows - 1) * a.ld + c0 + c4;
    V4 y;
    if (c0 + 64 <= a.cols) {
      y = *reinterpret_cast<const V4u*>(at);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = c0 + c4 + k < a.cols ? at[k] : 0.f;
    }
    if (r >= a.rows) y = V4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) sh[rq + q * 4][c4 + k] = y[k];
  }
  __syncthreads();
  auto put = [&](_Float16* to, int64_t frag, const float* x) {
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
  const int b = wave >> 1;                        // row block of the tile; a wave takes two of its four steps
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int ks = (wave & 1) * 2 + u, k = ks * 16 + half * 4;
    float x[8];
    if (a.R && c0 / 16 + ks < a.KS) {
      const int r = b * 32 + l32;
      const float f = pow2(exp_or_0(scale_exp(a.all ? *a.all : r0 + r < a.rows ? a.rmax[r0 + r] : 0u)));
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = sh[r][k + (t >> 2) * 8 + (t & 3)] * f;
      put(a.R, ((r0 / 32 + b) * a.mul + a.add) * a.KS + c0 / 16 + ks, x);
    }
    if (a.T && r0 / 16 + ks < a.KS_t) {
      const int c = b * 32 + l32;
      const float f = pow2(exp_or_0(scale_exp(a.all ? *a.all : c0 + c < a.cols ? a.cmax[c0 + c] : 0u)));
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = sh[k + (t >> 2) * 8 + (t & 3)][c] * f;
      put(a.T, ((c0 / 32 + b) * a.mul + a.add) * a.KS_t + r0 / 16 + ks, x);
    }
  }
}

// ---------------------------------------------------------------- products

// PROJECT  A's rows: the interleaved hidden columns, B's the rows of X: A and B of the block, H and its largest values
// BACK     A's rows: 128 hidden columns of Wd, B's the rows of dY: G, from that and A and B all of H, dA, dB and their largest values
// ROWS     A: H or [dA dB] by rows, B: a weight turned: Y, dX
// COLS     A: X or dY by columns, B: [dA dB] or H turned: gradients of weights
enum { PROJECT, BACK, ROWS, COLS };

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
  Gate act;
  int two;                             // an operand is [dA dB]
  // largest values: of the weights (gate or only one, up), of the rows of X or dY; of what is made or read by rows and by columns (H; or dA and dB)
  const uint32_t *w0, *w1, *rows_in;
  uint32_t *h_row, *a_row, *b_row, *h_col, *a_col, *b_col;
  const uint32_t* m_top;               // COLS: of A's rows
  int64_t n, f;                        // rows, hidden columns that there are
  float *H, *D;                        // in the order of fragments (null: not wanted)
  int64_t KSH, KSD;
  float *gate, *up;                    // [n x f]
  int64_t ld_gate, ld_up;
  Out out[2];                          // ROWS: [0]; COLS of [dA dB]: gate's and up's (null: not wanted)
  int64_t m_end, n_end;                // (n_end: of hidden columns, for COLS)
  int add;
};

// Eight values (t = 0 .. 3 and 4 .. 7 where the planes will be), each times its factor, a power of two.  Two instructions a value: the compiler rounds each value twice where it
// is left to itself (a pair's halves once more for themselves).
template <class F>
__device__ __forceinline__ void split8(v8h& p0, v8h& p1, F&& factor) {
  typedef uint32_t v4i __attribute__((ext_vector_type(4)));
  const V4 x = __builtin_bit_cast(V4, p0), y = __builtin_bit_cast(V4, p1);
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
//   in_a(x, i, cur)  what is done to a step's planes of row block i before they are used (cur: the stage's parity), in_b(rb): to what a wave brings of B
template <bool TURN, bool FAR, int NI, int NJ, class InA, class InB>
__device__ __forceinline__ void multiply(v16f (&acc)[NI][NJ], const _Float16* Ap, const int64_t a_rows, const _Float16* B, const int64_t b_rows, int todo, _Float16* Bs, InA&& in_a, InB&& in_b) {
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
  };
  auto stash = [&](int to) {
    in_b(rb);
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
    if (!more) Bp -= b_step;
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
        for (int i = 0; i < NI; ++i) in_a(x[i], i, cur);
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
  // four values of hidden columns c .. c + 3 of a row of gate or up
  __device__ __forceinline__ void put(float* p, int64_t c, V4 x) const {
    if (c + 4 <= a.f) {
      *reinterpret_cast<V4*>(p + c) = x;
      return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (c + k < a.f) p[c + k] = x[k];
  }
  __device__ __forceinline__ V4 get(const float* p, int64_t c) const {
    if (c + 4 <= a.f) return *reinterpret_cast<const V4*>(p + c);
    V4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (c + k < a.f) x[k] = p[c + k];
    return x;
  }
  // four values of a row, in the order of fragments: the k-th four of 16 columns by half
  __device__ __forceinline__ void put_frag(float* p, int64_t KS, int64_t row_block, int64_t step, int k, V4 x) const {
    // (past the caches, which have the operands to keep: 232,965 x 256 x 1,024 backward 4.16 -> 4.08 ms)
    __builtin_nontemporal_store(x, reinterpret_cast<V4*>(p + ((row_block * KS + step) * 2 + k) * (FRAG / 2) + lane * 4));
  }
  // H, dA and dB of NJ row blocks from row block b0 on, of the hidden columns c0 .. c0 + 31.  Largest values: of the rows join ma and mb, of the columns (of H, dA,
  // dB, 32 each) go to cols.  (An infinite one may be the largest: what is scaled by it is not finite in any case.)  get(j, k, x, y): A and B of four hidden
  // columns of a row, fetched four columns ahead; sums(j, k, e): G of one.
  template <int KIND, int NJ, class Get, class Sums>
  __device__ __forceinline__ void back(int64_t b0, int64_t c0, float (&ma)[NJ], float (&mb)[NJ], float* cols, Get&& get, Sums&& sums) const {
    const int l32 = lane & 31;
    const bool edge = (b0 + NJ) * 32 > a.n || c0 + 32 > a.f;
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
      const int64_t c = c0 + k * 8 + half * 4, step = c0 / 16 + (k >> 1), step_d = c0 / 8 + (k >> 1);
      float ch[4] = {}, ca[4] = {}, cb[4] = {};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int64_t v = (b0 + j) * 32 + l32;
        V4 h, da, db;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Act s = act_of<KIND>(a.act, x[k & 1][j][e]);
          const float u = y[k & 1][j][e], g = sums(j, k, e);
          h[e] = s.v * u, da[e] = g * u * s.s, db[e] = g * s.v;
        }
        if (edge) {                    // what is behind the last row and column is 0, whatever the weights are
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v >= a.n || c + e >= a.f) h[e] = da[e] = db[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ch[e] = fmaxf(ch[e], fabsf(h[e])), ca[e] = fmaxf(ca[e], fabsf(da[e])), cb[e] = fmaxf(cb[e], fabsf(db[e]));
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
  }
  // What the four waves found, to where it is kept: cols, of HBS hidden blocks from hidden column c0 on, and ma and mb by way of top (8 NJ 32 words of LDS).  All words are
  // looked at together: each takes a trip to memory.
  template <int NJ, int HBS>
  __device__ __forceinline__ void back_tops(int64_t b0, int64_t c0, const float (&ma)[NJ], const float (&mb)[NJ], const float* cols, float* top) const {
    constexpr int R = NJ * 32, N = 2 * R + HBS * 96, U = (N + 255) / 256;
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float x = fmaxf(ma[j], __shfl_xor(ma[j], 32, 64)), y = fmaxf(mb[j], __shfl_xor(mb[j], 32, 64));
      top[(wave * 2 + half) * R + j * 32 + (lane & 31)] = half ? y : x;
    }
    __syncthreads();
    uint32_t *word[U], is[U], was[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = u * 256 + threadIdx.x;
      word[u] = nullptr;
      float m = 0.f;
      if (i < 2 * R) {
        const int which = i / R, r = i % R;
        m = fmaxf(fmaxf(top[which * R + r], top[(2 + which) * R + r]), fmaxf(top[(4 + which) * R + r], top[(6 + which) * R + r]));
        if (b0 * 32 + r < a.n) word[u] = (which ? a.b_row : a.a_row) + b0 * 32 + r;
      } else if (i < N) {
        const int q = i - 2 * R, which = q / 32 % 3;
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

template <int MODE, int KIND>
__device__ __forceinline__ void ffn_split(const Args& a, unsigned block, _Float16* Bs) {
  constexpr bool TURN = MODE == ROWS || MODE == COLS;
  const Tile tile(block, a.mt, a.nt, a.splits);
  if (tile.m < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
  constexpr int NI = MODE == BACK ? 1 : 2;               // row blocks of A a wave (BACK has much to do with each sum)
  const int64_t split = tile.split, m0 = tile.m * (NI * 128), n0 = tile.n * TN, mw = m0 + wave * (NI * 32);
  const int64_t s0 = a.pairs * split / a.splits * 2;                 // its first stage
  const int todo = __builtin_amdgcn_readfirstlane((int)(a.pairs * (split + 1) / a.splits - s0 / 2));

  // exponents of the weights; of the rows of A (ROWS), of the columns that are split on the way to LDS (COLS)
  const int e0 = exp_or_0(a.w0 ? scale_exp(*a.w0) : NONE), e1 = exp_or_0(a.w1 ? scale_exp(*a.w1) : NONE);
  // of a row of H or [dA dB], times the weights that it meets: the smallest that its parts allow
  auto row_exp = [&](int64_t v) {
    int e = NONE * 2;
    if (a.two) {
      const int x = scale_exp(a.a_row[v]), y = scale_exp(a.b_row[v]);
      if (x < NONE) e = x + e0;
      if (y < NONE) e = min(e, y + e1);
    } else {
      const int x = scale_exp(a.h_row[v]);
      if (x < NONE) e = x + e0;
    }
    return e >= NONE ? 0 : e;
  };
  // hidden column of column n of B, and which of the two
  auto hidden = [&](int64_t n) { return a.two ? n / (2 * HB) * HB + n % HB : n; };
  auto col_top = [&](int64_t n) -> uint32_t {
    const int64_t c = hidden(n);
    if (c >= a.f) return 0u;
    return !a.two ? a.h_col[c] : (n / HB) & 1 ? a.b_col[c] : a.a_col[c];
  };
  v16f acc[NI][4];
  clear(acc);
  const _Float16* Ap = a.A + (mw / 32 * a.KSA + s0 * KT) * 2 * FRAG + lane * 8;
  const _Float16* B = a.B + (TURN ? s0 * a.KSB + n0 / 16 : n0 / 32 * a.KSB + s0 * KT) * 2 * FRAG;
  const int64_t a_rows = a.KSA * 2 * FRAG, b_rows = a.KSB * 2 * FRAG;
  const auto as_it_is = [](v8h (&)[2], int, int) {};
  if constexpr (MODE == ROWS) {
    float fr[2][2];                    // (a stage's parity is which half of a hidden block [gate, up] it is)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = row_exp(mw + i * 32 + l32);
      fr[i][0] = pow2(e - e0), fr[i][1] = pow2(e - (a.two ? e1 : e0));
    }
    multiply<true, true>(acc, Ap, a_rows, B, b_rows, todo, Bs, [&](v8h (&x)[2], int i, int cur) { split8(x[0], x[1], [&](int) { return fr[i][cur]; }); }, [](v8h (&)[4]) {});
  } else if constexpr (MODE == COLS) {
    float fc[2][8];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int k = 0; k < 8; ++k) fc[u][k] = pow2(exp_or_0(scale_exp(col_top(n0 + wave * 32 + u * 16 + (k >> 2) * 8 + half * 4 + (k & 3)))));
    multiply<true, true>(acc, Ap, a_rows, B, b_rows, todo, Bs, as_it_is, [&](v8h (&rb)[4]) {
#pragma unroll
      for (int u = 0; u < 2; ++u) split8(rb[u * 2], rb[u * 2 + 1], [&](int t) { return fc[u][t]; });
    });
  } else {
    multiply<false, true>(acc, Ap, a_rows, B, b_rows, todo, Bs, as_it_is, [](v8h (&)[4]) {});
  }

  // lane l32 + 32 half of a 32 x 32 tile has column l32 and the rows 8 (e / 4) + 4 half + e % 4
  if constexpr (MODE == ROWS || MODE == COLS) {
    // exponents of the rows and columns of sums, all of them looked up at once (where they are used, one after the other, each would be a trip to memory)
    int* ends = reinterpret_cast<int*>(Bs);
    ends[tid] = m0 + tid < a.m_end ? (MODE == COLS ? exp_or_0(scale_exp(a.m_top[m0 + tid])) : row_exp(m0 + tid)) : 0;
    if (MODE == COLS && tid < TN) ends[TM + tid] = exp_or_0(scale_exp(col_top(n0 + tid)));
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = n0 + j * 32 + l32, c = MODE == COLS ? hidden(n) : n;
      const Out& o = a.out[MODE == COLS && a.two ? j & 1 : 0];
      if (!o.p || c >= a.n_end) continue;
      const int en = MODE == COLS ? ends[TM + j * 32 + l32] : 0;
      float* at = o.p + split * o.split_part + c * o.ns;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = wave * 64 + i * 32 + k * 8 + half * 4;
          const int64_t m = m0 + r;
          const int4 em = *reinterpret_cast<const int4*>(ends + r);
          V4 x{__builtin_amdgcn_ldexpf(acc[i][j][k * 4], -(em.x + en)), __builtin_amdgcn_ldexpf(acc[i][j][k * 4 + 1], -(em.y + en)),
               __builtin_amdgcn_ldexpf(acc[i][j][k * 4 + 2], -(em.z + en)), __builtin_amdgcn_ldexpf(acc[i][j][k * 4 + 3], -(em.w + en))};
          float* to = at + m * o.ms;
          if (o.ms == 1 && m + 4 <= a.m_end) {
            if (a.add) x += *reinterpret_cast<const V4u*>(to);
            *reinterpret_cast<V4u*>(to) = x;
            continue;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m + e < a.m_end) to[e * o.ms] = a.add ? to[e * o.ms] + x[e] : x[e];
        }
    }
    return;
  }
  float* top = reinterpret_cast<float*>(Bs);
  const Hidden at(a);
  if constexpr (MODE == PROJECT) {
    const int64_t c0 = mw / 2;                          // the wave's 32 hidden columns
    int exps[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) exps[j] = exp_or_0(scale_exp(n0 + j * 32 + l32 < a.n ? a.rows_in[n0 + j * 32 + l32] : 0u));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
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
          h[e] = act_of<KIND>(a.act, x[e]).v * y[e];
          m = fmaxf(m, fabsf(h[e]));
        }
        if (a.gate && there) at.put(a.gate + v * a.ld_gate, c, x), at.put(a.up + v * a.ld_up, c, y);
        at.put_frag(a.H, a.KSH, n0 / 32 + j, c0 / 16 + (k >> 1), k & 1, h);
      }
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      if (half == 0) top[wave * TN + j * 32 + l32] = m;
    }
    __syncthreads();
    if (tid < TN && n0 + tid < a.n) raise(a.h_row + n0 + tid, __float_as_uint(fmaxf(fmaxf(top[tid], top[TN + tid]), fmaxf(top[2 * TN + tid], top[3 * TN + tid]))));
  }
  if constexpr (MODE == BACK) {
    float ma[4] = {}, mb[4] = {};
    float* cols = top + 8 * TN;
    int ey[4];
    const float *gate[4], *up[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t v = n0 + j * 32 + l32, row = v < a.n ? v : a.n - 1;
      ey[j] = exp_or_0(scale_exp(a.rows_in[row]));
      gate[j] = a.gate + row * a.ld_gate, up[j] = a.up + row * a.ld_up;
    }
    at.back<KIND, 4>(n0 / 32, mw, ma, mb, cols + wave * 96, [&](int j, int k, V4& x, V4& y) {
      const int64_t c = mw + k * 8 + half * 4;
      x = at.get(gate[j], c), y = at.get(up[j], c);
    }, [&](int j, int k, int e) { return __builtin_amdgcn_ldexpf(acc[0][j][k * 4 + e], -(ey[j] + e0)); });
    at.back_tops<4, 4>(n0 / 32, m0, ma, mb, cols, top);
  }
}

template <int MODE, int KIND>
__global__ void __launch_bounds__(256, 2) k_ffn_split(Args a) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(MODE == ROWS || MODE == COLS)];
  ffn_split<MODE, KIND>(a, blockIdx.x, Bs);
}
// dX, and the gradients of the weights, which do not wait for each other, behind each other's blocks where all of them run at once.
struct Ends {
  Args a[3];                           // ROWS, COLS, COLS
  unsigned first[3];                   // blocks before each
};
__global__ void __launch_bounds__(256, 2) k_ffn_ends(Ends ends) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(true)];
  if (blockIdx.x < ends.first[1]) return ffn_split<ROWS, OTHERS>(ends.a[0], blockIdx.x, Bs);
  const int k = blockIdx.x < ends.first[2] ? 1 : 2;
  ffn_split<COLS, OTHERS>(ends.a[k], blockIdx.x - ends.first[k], Bs);
}

// PROJECT and BACK in one where A and B were not kept: 128 hidden columns by 64 rows, 32 by 64 a wave, first A and B, then G; three blocks a CU, which is what hides their ends.  (Of 96
// rows, two blocks: 232,965 x 256 x 1,024 1,690 -> 1,790 us, 16,384 x 512 x 2,048 417 -> 456, but 8,192 x 1,024 x 4,096 733 -> 702; the sums of 128 would take 192 registers.)
constexpr int REMAKE_ROWS = 64;
static_assert(REMAKE_ROWS % PAIR == 0 && TM % REMAKE_ROWS == 0, "COLS reads whole pairs of stages; pieces are multiples of TM rows");
struct RemakeArgs {
  Args a;                              // A, B, KSA, KSB, pairs, w0, w1, rows_in: the projections'
  const _Float16 *A2, *B2;
  int64_t KS2, pairs2;
  const uint32_t *w2, *rows2;
};
template <int KIND>
__global__ void __launch_bounds__(256, 3) k_ffn_remake(RemakeArgs r) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(false)];
  const Args& a = r.a;
  const Tile tile(blockIdx.x, a.mt, a.nt, 1);
  if (tile.m < 0) return;
  constexpr int NJ = REMAKE_ROWS / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t hb = tile.m * 4 + wave, b0 = tile.n * NJ;            // the wave's hidden block, the tile's first row block
  v16f ab[2][NJ], gr[1][NJ];
  const auto as_it_is = [](v8h (&)[2], int, int) {};
  const auto as_it_comes = [](v8h (&)[NJ]) {};
  clear(ab);
  multiply<false, false>(ab, a.A + hb * 2 * a.KSA * 2 * FRAG + lane * 8, a.KSA * 2 * FRAG, a.B + b0 * a.KSB * 2 * FRAG, a.KSB * 2 * FRAG, (int)a.pairs, Bs, as_it_is, as_it_comes);
  clear(gr);
  multiply<false, false>(gr, r.A2 + hb * r.KS2 * 2 * FRAG + lane * 8, 0, r.B2 + b0 * r.KS2 * 2 * FRAG, r.KS2 * 2 * FRAG, (int)r.pairs2, Bs, as_it_is, as_it_comes);
  const int e0 = exp_or_0(scale_exp(*a.w0)), e1 = exp_or_0(scale_exp(*a.w1)), e2 = exp_or_0(scale_exp(*r.w2));
  const Hidden at(a);
  float ma[NJ] = {}, mb[NJ] = {};
  float *top = reinterpret_cast<float*>(Bs), *cols = top + 8 * NJ * 32;
  int ex[NJ], ey[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t v = (b0 + j) * 32 + (lane & 31), row = v < a.n ? v : a.n - 1;
    ex[j] = exp_or_0(scale_exp(a.rows_in[row])), ey[j] = exp_or_0(scale_exp(r.rows2[row]));
  }
  at.back<KIND, NJ>(b0, hb * HB, ma, mb, cols + wave * 96, [&](int j, int k, V4& x, V4& y) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[e] = __builtin_amdgcn_ldexpf(ab[0][j][k * 4 + e], -(ex[j] + e0)), y[e] = __builtin_amdgcn_ldexpf(ab[1][j][k * 4 + e], -(ex[j] + e1));
  }, [&](int j, int k, int e) { return __builtin_amdgcn_ldexpf(gr[0][j][k * 4 + e], -(ey[j] + e2)); });
  at.back_tops<NJ, 4>(b0, tile.m * 4 * HB, ma, mb, cols, top);
}

__global__ void __launch_bounds__(256) k_ffn_join(FfnJoins joins) {
  unsigned block = blockIdx.x;
  int k = 0;
  while (block >= joins.join[k].blocks) block -= joins.join[k++].blocks;
  const FfnJoin& a = joins.join[k];
  const int64_t nv = a.pitch / 4, i = (int64_t)block * 256 + threadIdx.x, r = i / nv, c = (i - r * nv) * 4;
  if (r >= a.rows || c >= a.cols) return;
  V4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < a.parts; ++p) s += *reinterpret_cast<const V4*>(a.sums + p * a.part + r * a.pitch + c);
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

constexpr size_t FFN_BYTES = (size_t)4 << 30, FFN_LEAN = (size_t)64 << 20;     // of what a piece's rows take
constexpr int64_t SLOTS = 512;                     // blocks that run together: two a CU
constexpr int64_t LEAST_PAIRS = 4;                 // of a part of a reduction

int parts_of(int64_t tiles, int64_t pairs) { return (int)std::max<int64_t>(1, std::min<int64_t>({SLOTS / tiles, pairs / LEAST_PAIRS, 64})); }

struct Ffn : FfnCall {
  static int64_t blocks_of(const Args& a) { return up_to(a.mt * a.nt * a.splits, 8); }
  int launch(int mode, const Args& a) const {
    const int64_t blocks = blocks_of(a);
    if (blocks >= (1 << 24)) return ht_set_err(ctx, HT_ESHAPE, "ffn: %lld tiles in one product", (long long)blocks);
    const unsigned grid = (unsigned)blocks;
    const bool logistic = a.act.logistic();
    if (mode == PROJECT) (logistic ? k_ffn_split<PROJECT, LOGISTIC> : k_ffn_split<PROJECT, OTHERS>)<<<grid, 256, 0, ctx->stream>>>(a);
    else if (mode == BACK) (logistic ? k_ffn_split<BACK, LOGISTIC> : k_ffn_split<BACK, OTHERS>)<<<grid, 256, 0, ctx->stream>>>(a);
    else if (mode == ROWS) k_ffn_split<ROWS, OTHERS><<<grid, 256, 0, ctx->stream>>>(a);
    else k_ffn_split<COLS, OTHERS><<<grid, 256, 0, ctx->stream>>>(a);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
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
    const int sy = parts_of(mt * nte, pairs_f), sx = parts_of(mt * ntd, pairs_2f), sD = parts_of(dp / TM * ntD, pairs_r), sH = parts_of(ep / TM * ntH, pairs_r);
    const int64_t e4 = up_to(e, 4), d4 = up_to(d, 4), f4 = up_to(f, 4);
    // a weight's gradient as it lies: rows and pitch of its parts
    const int64_t wr = in_out ? d : f, wp = in_out ? f4 : d4, vr = in_out ? f : e, vp = in_out ? e4 : f4;

    OpsBlock m;
    const int64_t n_top = 4 + 5 * Rp + dp + ep + 3 * fp;
    const auto top = m.add<uint32_t>(n_top);
    const auto W2 = m.add<_Float16>(2 * fp * KSd * 32), Wf = m.add<_Float16>(fp * KSe * 32);
    const auto Xr = m.add<_Float16>(Rp * KSd * 32);
    const auto Xt = m.add<_Float16>(d_w ? dp * KSR * 32 : 0);
    const auto Gr = m.add<_Float16>(bwd ? Rp * KSe * 32 : 0);
    const auto Gt = m.add<_Float16>(dWd ? ep * KSR * 32 : 0);
    const auto H = m.add<float>(Rp * fp), Df = m.add<float>(bwd ? Rp * fp * 2 : 0);
    const auto sums_y = m.add<float>(!bwd && sy > 1 ? sy * Rp * e4 : 0), sums_x = m.add<float>(dX && sx > 1 ? sx * Rp * d4 : 0);
    const auto sums_D = m.add<float>(d_w && sD > 1 ? sD * 2 * wr * wp : 0), sums_H = m.add<float>(dWd && sH > 1 ? sH * vr * vp : 0);
    HT_TRY(bytes > FFN_LEAN ? m.take_if_room(ctx) : m.take(ctx));

    uint32_t *t_g = m.at(top), *t_u = t_g + 1, *t_d = t_g + 2, *t_x = t_g + 4, *t_y = t_x + Rp, *t_h = t_y + Rp, *t_a = t_h + Rp, *t_b = t_a + Rp, *t_xc = t_b + Rp, *t_yc = t_xc + dp,
             *t_hc = t_yc + ep, *t_ac = t_hc + fp, *t_bc = t_ac + fp;
    for (int64_t k = 0; k < pieces; ++k) {
      const int64_t r0 = k * Rp, rows = std::min(Rp, n - r0);
      HT_TRY(ht_fill_zero(ctx, st, k ? t_x : t_g, (size_t)(k ? n_top - 4 : n_top) * 4));
      Tops tops{};
      Packs packs{};
      unsigned tb = 0, pb = 0;
      auto operand = [&](const float* p, int64_t ld, int64_t r, int64_t c, uint32_t* rm, uint32_t* cm, uint32_t* all, _Float16* R, int64_t KS, _Float16* T, int64_t KS_t, int mul,
                         int add, int64_t row_tile, int64_t col_tile) {
        Top& t = tops.top[tops.n++];
        t = Top{p, ld, r, c, rm, cm, all, (unsigned)(std::min(ceil_div64(r, top_rows(c)), std::max<int64_t>(1, TOP_BLOCKS / ceil_div64(c, TOP_COLS))) * ceil_div64(c, TOP_COLS))};
        tb += t.blocks;
        Pack& q = packs.pack[packs.n++];
        q = Pack{p, ld, r, c, rm, cm, all, R, T, KS, KS_t, mul, add, (unsigned)(up_to(r, row_tile) / 64), (unsigned)(up_to(c, col_tile) / 64)};
        pb += q.row_tiles * q.col_tiles;
      };
      operand(X->ptr + r0 * X->ld, X->ld, rows, d, t_x, d_w ? t_xc : nullptr, nullptr, m.at(Xr), KSd, d_w ? m.at(Xt) : nullptr, KSR, 1, 0, TM, d_w ? TM : TN);
      if (bwd)
        operand(dY->ptr + r0 * dY->ld, dY->ld, rows, e, t_y, dWd ? t_yc : nullptr, nullptr, m.at(Gr), KSe, dWd ? m.at(Gt) : nullptr, KSR, 1, 0, TM, dWd ? TM : TN);
      if (k == 0) {
        // by hidden columns: the rows of an OUT_IN Wg, the columns of an IN_OUT one
        const ht_tensor* w[2] = {Wg, Wu};
        for (int i = 0; i < 2; ++i)
          operand(w[i]->ptr, w[i]->ld, w[i]->rows, w[i]->cols, nullptr, nullptr, t_g + i, in_out ? nullptr : m.at(W2), KSd, in_out ? m.at(W2) : nullptr, KSd, 2, i, in_out ? TN : TM,
                  in_out ? TM : TN);
        operand(Wd->ptr, Wd->ld, Wd->rows, Wd->cols, nullptr, nullptr, t_d, in_out ? m.at(Wf) : nullptr, KSe, in_out ? nullptr : m.at(Wf), KSe, 1, 0, in_out ? TM : TN,
                in_out ? TN : TM);
      }
      k_ffn_top<<<tb, 256, 0, st>>>(tops);
      HT_LAUNCH_CHECK(ctx);
      k_ffn_pack<<<pb, 256, 0, st>>>(packs);
      HT_LAUNCH_CHECK(ctx);

      Args base{};
      base.act = gate_of(D->act), base.n = rows, base.f = f, base.splits = 1;
      base.h_row = t_h, base.a_row = t_a, base.b_row = t_b, base.h_col = t_hc, base.a_col = t_ac, base.b_col = t_bc;
      base.KSH = KSH, base.KSD = KSD;
      base.gate = gate ? gate->ptr + r0 * gate->ld : nullptr, base.ld_gate = gate ? gate->ld : 0;
      base.up = up ? up->ptr + r0 * up->ld : nullptr, base.ld_up = up ? up->ld : 0;
      const int64_t row_tiles = ceil_div64(rows, TN);
      Args a = base;
      a.H = m.at(H);
      if (!bwd || remake) {
        a.A = m.at(W2), a.KSA = KSd, a.B = m.at(Xr), a.KSB = KSd;
        a.mt = ceil_div64(f, TN), a.nt = row_tiles, a.pairs = ceil_div64(d, PAIR);
        a.w0 = t_g, a.w1 = t_u, a.rows_in = t_x;
        if (!bwd) HT_TRY(launch(PROJECT, a));
      }
      if (remake) {
        a.D = m.at(Df);
        a.nt = ceil_div64(rows, REMAKE_ROWS);
        const bool logistic = a.act.logistic();
        (logistic ? k_ffn_remake<LOGISTIC> : k_ffn_remake<OTHERS>)<<<(unsigned)up_to(a.mt * a.nt, 8), 256, 0, st>>>(RemakeArgs{a, m.at(Wf), m.at(Gr), KSe, ceil_div64(e, PAIR), t_d, t_y});
        HT_LAUNCH_CHECK(ctx);
      } else if (bwd) {
        a.A = m.at(Wf), a.KSA = KSe, a.B = m.at(Gr), a.KSB = KSe;
        a.mt = ceil_div64(f, TN), a.nt = row_tiles, a.pairs = ceil_div64(e, PAIR);
        a.w0 = t_d, a.rows_in = t_y;
        a.D = m.at(Df);
        HT_TRY(launch(BACK, a));
      }
      // Y, or dX; their parts' sums are added up behind each piece, those of the weights' gradients behind the last
      FfnJoins j{};
      auto by_rows = [&](const ht_tensor* to, const float* P, int64_t KSP, bool two, const _Float16* W, int64_t KSW, const uint32_t* w0, const uint32_t* w1, int64_t cols, int64_t nt,
                         int64_t pairs, int splits, float* sums, int64_t pitch) {
        Args a = base;
        a.A = (const _Float16*)P, a.KSA = KSP, a.B = W, a.KSB = KSW;
        a.mt = ceil_div64(rows, TM), a.nt = nt, a.pairs = pairs, a.splits = splits, a.two = two, a.w0 = w0, a.w1 = w1;
        a.m_end = rows, a.n_end = cols;
        float* out = to->ptr + r0 * to->ld;
        a.out[0] = splits > 1 ? Out{sums, pitch, 1, Rp * pitch} : Out{out, to->ld, 1, 0};
        a.add = splits == 1 && D->accumulate;
        if (splits > 1) j.join[j.n++] = FfnJoin{sums, Rp * pitch, pitch, rows, cols, splits, D->accumulate, out, to->ld, 0};
        return a;
      };
      auto by_cols = [&](const _Float16* At, const uint32_t* m_top, int64_t m_end, const float* P, int64_t KSP, bool two, int64_t tiles_m, int64_t nt, int splits, float* sums,
                         int64_t r, int64_t pitch, const ht_tensor* o0, const ht_tensor* o1, bool m_is_row) {
        Args a = base;
        a.A = At, a.KSA = KSR, a.B = (const _Float16*)P, a.KSB = KSP;
        a.mt = tiles_m, a.nt = nt, a.pairs = ceil_div64(rows, PAIR), a.splits = splits, a.two = two, a.m_top = m_top;
        a.m_end = m_end, a.n_end = f;
        const ht_tensor* o[2] = {o0, o1};
        for (int i = 0; i < 2; ++i) {
          if (!o[i]) continue;
          const int64_t ld = splits > 1 ? pitch : o[i]->ld;
          a.out[i] = Out{splits > 1 ? sums + i * r * pitch : o[i]->ptr, m_is_row ? ld : 1, m_is_row ? 1 : ld, splits > 1 ? (two ? 2 : 1) * r * pitch : 0};
          if (splits > 1 && k + 1 == pieces)
            j.join[j.n++] = FfnJoin{sums + i * r * pitch, (two ? 2 : 1) * r * pitch, pitch, o[i]->rows, o[i]->cols, splits, D->accumulate_dW, o[i]->ptr, o[i]->ld, 0};
        }
        a.add = k > 0 || (splits == 1 && D->accumulate_dW);
        return a;
      };
      if (Y) HT_TRY(launch(ROWS, by_rows(Y, m.at(H), KSH, false, m.at(Wf), KSe, t_d, nullptr, e, nte, pairs_f, sy, m.at(sums_y), e4)));
      Args ax{}, ad{}, ah{};                             // (no tiles: not asked for)
      if (dX) ax = by_rows(dX, m.at(Df), KSD, true, m.at(W2), KSd, t_g, t_u, d, ntd, pairs_2f, sx, m.at(sums_x), d4);
      if (d_w) ad = by_cols(m.at(Xt), t_xc, d, m.at(Df), KSD, true, dp / TM, ntD, sD, m.at(sums_D), wr, wp, dWg, dWu, in_out);
      if (dWd) ah = by_cols(m.at(Gt), t_yc, e, m.at(H), KSH, false, ep / TM, ntH, sH, m.at(sums_H), vr, vp, dWd, nullptr, !in_out);
      const int64_t bx = blocks_of(ax), bd = blocks_of(ad), bh = blocks_of(ah);
      if (bwd && bx + bd + bh <= SLOTS) {
        k_ffn_ends<<<(unsigned)(bx + bd + bh), 256, 0, st>>>(Ends{{ax, ad, ah}, {0, (unsigned)bx, (unsigned)(bx + bd)}});
        HT_LAUNCH_CHECK(ctx);
      } else {
        if (bx) HT_TRY(launch(ROWS, ax));
        if (bd) HT_TRY(launch(COLS, ad));
        if (bh) HT_TRY(launch(COLS, ah));
      }
      HT_TRY(ht_ffn_join(ctx, j));
    }
    return HT_OK;
  }
  int call() const {
    if (X->rows == 0) {                // nothing to add up
      FfnJoins w{};
      for (const ht_tensor* t : {dWg, dWu, dWd})
        if (t && !D->accumulate_dW) w.join[w.n++] = FfnJoin{nullptr, 0, up_to(t->cols, 4), t->rows, t->cols, 0, 0, t->ptr, t->ld, 0};
      return ht_ffn_join(ctx, w);
    }
    if (X->rows <= HT_FFN_FEW) return ht_ffn_few(*this);
    const int rc = run(FFN_BYTES);
    return rc == HT_ENOMEM ? run(FFN_LEAN) : rc;      // (nothing has been launched by a call that is refused memory)
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
    a.blocks = (unsigned)ceil_div64(a.rows * (a.pitch / 4), 256);
    grid += a.blocks;
  }
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
