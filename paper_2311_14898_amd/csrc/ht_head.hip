// Softmax cross entropy of a linear head over many classes, with its gradients, of whose logits no more are kept than a piece:
//   x_vc = h_v . w_c ;  lse_v = log sum_c exp(x_vc) ;  loss = sum_v u_v (lse_v - x_vy) / N
//   dx_vc = (u_v / N) (exp(x_vc - lse_v) - [c = y_v]) ;  dH = dx W^T ;  dW = H^T dx
// Labelled rows are first listed, and only they are computed with.  Rows go in pieces: a pass over all classes gives lse, and then the gradients of the
// logits, exp(x - lse) - [c = y], are what dH and dW are made of.  Up to 256 classes a tile has all of a row's logits, and one launch leaves their
// gradients.  Of wide rows, and of few logits, the pass keeps its sums, which the gradients take the place of (three products of 2 n d C flops); of others they are
// computed again, class piece by class piece (four).
//
// All products are k_split_nt's: fp32 products on the fp16 matrix cores.  A value is split into two fp16 numbers, x = x0 + x1 (x0 its
// rounding, x1 the rounding of what is left: |x - x0 - x1| <= 2^-22 |x|), after W, each row of H, and each weighted column of H for dW were
// scaled by a power of two that brings the largest value to [2^14, 2^15); x0 y0 + x0 y1 + x1 y0 are added in fp32.  What is left out is at most 3 x 2^-22 of a
// product, typically (the roundings are independent) 2^-24 of it, what fp32 loses in rounding it; values below 2^-17 of the
// largest that they are scaled by keep fewer bits, down to 2^-39 of it.  Three fp16 steps take 96 clocks where an fp32 product takes 512.
//
// Gradients of logits have one scale, 2^15, whatever their class: a row of dW of a class that is no row's label is made of small probabilities alone.  Their
// x1 is held times 2^12, as far as fp16 goes (it is at most 8: scales are powers of two, so that x - m is exact and no p is rounded beyond 1), and y0 is taken times 2^-12 where they meet, in registers: 22 bits down to p = 2^-30, where a class of 2^24 equal
// ones has 2^-24, and 2^-52 (with the x1 y1 that is left out 2^-51) in what is smaller.  Without that factor those are 2^-17 and 2^-39.  What it costs, us with | without: 2,048
// rows x 256 features x 32,768 classes 489 | 485, 2,100 labelled rows of 7,001 x 602 x 50,003 1,468 | 1,448, 8,192 x 256 x 131,072 6,542 | 6,467.
#include <algorithm>

#include "ht_internal.h"

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float V4 __attribute__((ext_vector_type(4)));
typedef float V4u __attribute__((ext_vector_type(4), aligned(4)));      // weights need no alignment

// Operands lie in fragments, what a matrix instruction reads of them: 32 rows x 16 values of the reduction of one plane (x0 or x1), 1 KiB.
// Lane l + 32 h holds row l and the values 8 (t / 4) + 4 h + t % 4, t = 0 .. 7: the order in which a lane of a product's result holds
// its rows, so that results become operands without leaving their lanes (any order will do that both operands have).  Fragment (row block,
// step, plane) is number (block * KS + step) * 2 + plane.
constexpr int FRAG = 512;
constexpr int TM = 256, TN = 128;      // tile of a block: rows of A x rows of B
constexpr float LOG2E = 1.44269504088896340736f;
constexpr int P_EXP = 15;              // gradients of logits are held times 2^15
constexpr int LOW_EXP = 12;            // ... what their rounding leaves times 2^12 more
constexpr size_t HEAD_BYTES = (size_t)6 << 30, HEAD_LEAN = (size_t)64 << 20;   // of what a piece's rows take
// Bytes of a piece's gradients of logits, at most.  ms with pieces of 1 GiB | 2 | 6: 8,192 rows x 256 features x 131,072 classes 6.69 | 6.52 | 6.63, 8,192 x 240 x 60,000 3.02 |
// 2.94 | 2.95, 2,100 labelled rows of 7,001 x 602 x 50,003 1.473 | 1.446 | 1.442.
constexpr size_t HEAD_PIECE = (size_t)2 << 30;
constexpr int64_t HEAD_CLASSES = 8192;             // of a piece at least, where a row's share of the memory is settled

__host__ __device__ constexpr int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// exp(x - m).  (The difference first: products with log2 e of logits of 10^9 are rounded by more than 1.)
__device__ __forceinline__ float exp_less(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * LOG2E); }

// The power of two that brings a row whose largest absolute value has these bits to [2^14, 2^15), and its inverse.
__device__ __forceinline__ uint32_t scale_exp(uint32_t bits) {
  if (bits == 0 || bits >= 0x7f800000u) return 127;
  const uint32_t e = 268 - (bits >> 23);
  return e > 253 ? 253 : e;
}
__device__ __forceinline__ float scale_of(uint32_t bits) { return __uint_as_float(scale_exp(bits) << 23); }
__device__ __forceinline__ float unscale_of(uint32_t bits) { return __uint_as_float((254 - scale_exp(bits)) << 23); }
// What makes a logit of a sum: the inverse of both operands' scales, but never 0 (a sum is below 2^47, so that such a row's logits are below 2^-79, and count as
// 0; the -inf of what lies behind the last class has to stay one).
__device__ __forceinline__ float logit_scale(uint32_t hbits, float ws) { return fmaxf(unscale_of(hbits) * ws, 0x1p-126f); }

// ---------------------------------------------------------------- labelled rows

constexpr int ROW_BLOCKS = 4096;
constexpr int64_t CLEAR_BLOCKS = 8192;

// Labelled rows of the first `blocks` blocks' shares; the other blocks clear n4 fours of words.
__global__ void __launch_bounds__(256) k_head_count(const int32_t* __restrict__ labels, int64_t V, int64_t rpb, int32_t* __restrict__ cnt, unsigned blocks,
                                                    uint4* __restrict__ clear, int64_t n4) {
  __shared__ int sh[4];
  if (blockIdx.x >= blocks) {
    for (int64_t i = (int64_t)(blockIdx.x - blocks) * 256 + threadIdx.x; i < n4; i += (int64_t)(gridDim.x - blocks) * 256) clear[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  int n = 0;
  const int64_t v0 = (int64_t)blockIdx.x * rpb, v1 = v0 + rpb < V ? v0 + rpb : V;
  for (int64_t v = v0 + threadIdx.x; v < v1; v += 256) n += labels[v] >= 0;
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) cnt[blockIdx.x] = sh[0] + sh[1] + sh[2] + sh[3];
}

// idx, lab: the labelled rows in order, and their labels; *total: how many.  Losses of rows without a label are cleared here.
__global__ void __launch_bounds__(256) k_head_place(const int32_t* __restrict__ labels, int64_t V, int64_t rpb, const int32_t* __restrict__ cnt,
                                                    int32_t* __restrict__ idx, int32_t* __restrict__ lab, int64_t* __restrict__ total,
                                                    float* __restrict__ row_loss, float* __restrict__ row_lse) {
  __shared__ int64_t sh64[4];
  __shared__ int sh[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t at = 0;
  for (int b = threadIdx.x; b < (int)blockIdx.x; b += 256) at += cnt[b];
  for (int o = 32; o > 0; o >>= 1) at += __shfl_xor(at, o, 64);
  if (lane == 0) sh64[wave] = at;
  __syncthreads();
  at = sh64[0] + sh64[1] + sh64[2] + sh64[3];
  const int64_t v0 = (int64_t)blockIdx.x * rpb, v1 = v0 + rpb < V ? v0 + rpb : V;
  for (int64_t w0 = v0; w0 < v1; w0 += 256) {
    const int64_t v = w0 + threadIdx.x;
    const int32_t y = v < v1 ? labels[v] : -1;
    const uint64_t mask = __ballot(y >= 0);
    __syncthreads();
    if (lane == 0) sh[wave] = __popcll(mask);
    __syncthreads();
    int before = __popcll(mask & ((1ull << lane) - 1)), all = 0;
    for (int w = 0; w < 4; ++w) before += w < wave ? sh[w] : 0, all += sh[w];
    if (y >= 0) {
      idx[at + before] = (int32_t)v;
      lab[at + before] = y;
    } else if (v < v1) {
      if (row_loss) row_loss[v] = 0.f;
      if (row_lse) row_lse[v] = 0.f;
    }
    at += all;
  }
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *total = at;
}

// All of that in one launch for up to LIST_ROWS rows: blocks of 256 rows, each counting what lies before it, then clear_blocks that clear n4
// fours of words.  Instead of three launches: 6 us of a call less by 80 rows x 256 features x 131,072 classes, 3 by 5,000 x 64 x 500, 4 by 2,048 x 256 x 32,768.
constexpr int64_t LIST_ROWS = 16384;
__global__ void __launch_bounds__(256) k_head_list(const int32_t* __restrict__ labels, int64_t V, unsigned blocks, int32_t* __restrict__ idx, int32_t* __restrict__ lab,
                                                   int64_t* __restrict__ total, float* __restrict__ row_loss, float* __restrict__ row_lse, float* __restrict__ dH,
                                                   int64_t ld, int d, uint4* __restrict__ clear, int64_t n4) {
  __shared__ int sh[4], here[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x >= blocks) {
    for (int64_t i = (int64_t)(blockIdx.x - blocks) * 256 + threadIdx.x; i < n4; i += (int64_t)(gridDim.x - blocks) * 256) clear[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  const int v0 = blockIdx.x * 256;
  int before = 0;
#pragma unroll 8
  for (int v = threadIdx.x; v < v0; v += 256) before += labels[v] >= 0;
  for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
  const int64_t v = v0 + threadIdx.x;
  const int32_t y = v < V ? labels[v] : -1;
  const uint64_t mask = __ballot(y >= 0);
  if (lane == 0) sh[wave] = before, here[wave] = __popcll(mask);
  __syncthreads();
  int at = sh[0] + sh[1] + sh[2] + sh[3], all = 0;
  for (int w = 0; w < 4; ++w) at += w < wave ? here[w] : 0, all += here[w];
  if (y >= 0) {
    const int k = at + __popcll(mask & ((1ull << lane) - 1));
    idx[k] = (int32_t)v;
    lab[k] = y;
  } else if (v < V) {
    if (row_loss) row_loss[v] = 0.f;
    if (row_lse) row_lse[v] = 0.f;
  }
  if (blockIdx.x == blocks - 1 && threadIdx.x == 0) *total = sh[0] + sh[1] + sh[2] + sh[3] + all;
  if (!dH) return;
  uint64_t none = __ballot(y < 0 && v < V);
  while (none) {
    const int r = __builtin_ctzll(none);
    none &= none - 1;
    for (int c = lane * 4; c < d; c += 256) *reinterpret_cast<float4*>(dH + (v0 + wave * 64 + r) * ld + c) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}

// Of more rows: zeros in dH's rows v0 .. v1 - 1 that have no label, by `blocks` blocks behind the first `from` of a launch that has other work.  The first piece's launches
// share them (CLEAR_*: which part of all rows is done after each): where few rows have labels, those launches wait for memory or for each other, and
// writing dH is what there is to do.  us of a call, shared | all of it in the first launch: 1,000,000 rows x 256 features, 1 % of them labelled, 172 classes 268 | 297, 1,000,000 x
// 64 x 100 114 | 130, 200,000 x 100 x 300 (80 MB), 30 % labelled, 252 | 261, 1,000,000 x 256 x 172, 30 % labelled, as fast; dH of less than CLEAR_SHARED bytes, which
// the caches hold, is not shared: 50,000 x 256 x 1,000 (51 MB), 10 % labelled, 124 | 119.
struct Clear {
  const int32_t* labels;
  float* dH;
  int64_t ld;
  int d;
  int64_t v0, v1;
  unsigned from, blocks;
};
// Which share each launch takes matters little: the first 45 % | 30 | 17 | 15 (the others in proportion) 275 | 270 | 264 | 267 us by 1,000,000 x 256 x 172 with 1 % labelled,
// 123 | 116 | 121 | 121 by 1,000,000 x 64 x 100, 351 | 351 | 355 | 352 by 300,000 x 602 x 41 with 10 % (all in the first launch 302, 133, 389); the shares here are
// roughly those of the launches' times where few rows have labels.
constexpr double CLEAR_TOP = 0.3, CLEAR_PACK = 0.4, CLEAR_LOGITS = 0.6, CLEAR_DH = 0.72, CLEAR_DW = 0.85;
constexpr int64_t CLEAR_SHARED = (int64_t)64 << 20;
// A wave 64 rows at a time.
__device__ __forceinline__ void clear_rows(const Clear& a, unsigned block) {
  const int lane = threadIdx.x & 63;
  for (int64_t v0 = a.v0 + ((int64_t)block * 4 + (threadIdx.x >> 6)) * 64; v0 < a.v1; v0 += (int64_t)a.blocks * 256) {
    uint64_t none = __ballot(v0 + lane < a.v1 && a.labels[v0 + lane < a.v1 ? v0 + lane : a.v1 - 1] < 0);
    while (none) {
      const int r = __builtin_ctzll(none);
      none &= none - 1;
      for (int c = lane * 4; c < a.d; c += 256) __builtin_nontemporal_store(V4{0.f, 0.f, 0.f, 0.f}, reinterpret_cast<V4*>(a.dH + (v0 + r) * a.ld + c));
    }
  }
}

// Rows of a piece: what is left of the list from r0 on, at most `most`.
__device__ __forceinline__ int64_t piece_rows(const int64_t* total, int64_t r0, int64_t most) {
  const int64_t left = *total - r0;
  return left < 0 ? 0 : left < most ? left : most;
}

// ---------------------------------------------------------------- operands

// A matrix [rows x cols], pitch ld, its rows as they are or those that idx names, each times weight[idx[r]].
struct Source {
  const float* p;
  int64_t ld, rows, cols;
  const int32_t* idx;            // null: all rows, as they are
  const float* weight;           // (with idx; null: 1)
  const int64_t* total;          // with idx: rows = piece_rows(total, r0, rows)
  int64_t r0;
  __device__ __forceinline__ int64_t n() const { return idx ? piece_rows(total, r0, rows) : rows; }
  __device__ __forceinline__ int64_t row(int64_t r) const { return idx ? (int64_t)idx[r0 + r] : r; }
};

// One launch finds the largest absolute values (as bits; maxima do not depend on their order) that a piece's operands are scaled by: blocks for H, and with the
// first piece blocks for W.
struct HeadTop {
  // H: largest values of rows, and of columns (of weighted rows), into arrays that hold zeros
  Source s;
  uint32_t *rmax, *cmax;
  unsigned gx, gy;               // blocks along rows, along columns
  // W: of all of it
  const float* W;
  int64_t ldw, wrows, wcols;
  uint32_t* wmax;
  unsigned w_blocks;             // (0: it is known)
  Clear clear;
};

// lpr lanes take a row's AMAX_COLS columns, four each, and a wave RW rows of each of its groups of lanes at a time; columns are joined once a block.
constexpr int AMAX_COLS = 256, RW = 8;
__host__ __device__ __forceinline__ int amax_lanes(int64_t cols) { return cols > 128 ? 64 : cols > 64 ? 32 : 16; }
// (Most blocks find a word as large as it need be: requests to one word wait for each other.)
__device__ __forceinline__ void raise(uint32_t* word, uint32_t m) {
  if (__hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < m) atomicMax(word, m);
}
__device__ __forceinline__ uint32_t max4(uint4 x) { return max(max(x.x, x.y), max(x.z, x.w)); }
__device__ __forceinline__ void amax_of_h(const HeadTop& a, int bx, int by) {
  __shared__ __attribute__((aligned(16))) uint32_t sh[4][AMAX_COLS];
  __shared__ uint32_t shr[4 * RW * 4];
  const Source& s = a.s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lpr = amax_lanes(s.cols), l = lane & (lpr - 1), groups = 64 / lpr, g = lane / lpr;
  const int here = 4 * RW * groups;                         // rows of a block at a time
  const int64_t n = s.n(), c = (int64_t)by * AMAX_COLS + l * 4;
  const bool there = c < s.cols;
  uint4 cm = make_uint4(0, 0, 0, 0);
  for (int64_t r0 = (int64_t)bx * here; r0 < n; r0 += (int64_t)a.gx * here) {
    float4 x[RW];
    float w[RW];
#pragma unroll
    for (int q = 0; q < RW; ++q) {
      const int64_t at = r0 + (wave * RW + q) * groups + g, v = s.row(at < n ? at : n - 1);
      x[q] = *reinterpret_cast<const float4*>(s.p + v * s.ld + (there ? c : 0));
      w[q] = s.weight ? s.weight[v] : 1.f;
    }
#pragma unroll
    for (int q = 0; q < RW; ++q) {
      if (c + 1 >= s.cols) x[q].y = x[q].x;                 // (pad columns, and lanes behind the last column: once more what is there)
      if (c + 2 >= s.cols) x[q].z = x[q].x;
      if (c + 3 >= s.cols) x[q].w = x[q].x;
      auto bits = [](float y) { return __float_as_uint(fabsf(y)); };
      uint32_t rm = max4(make_uint4(bits(x[q].x), bits(x[q].y), bits(x[q].z), bits(x[q].w)));
      cm = make_uint4(max(cm.x, bits(x[q].x * w[q])), max(cm.y, bits(x[q].y * w[q])), max(cm.z, bits(x[q].z * w[q])), max(cm.w, bits(x[q].w * w[q])));
      for (int o = lpr / 2; o > 0; o >>= 1) rm = max(rm, (uint32_t)__shfl_xor((int)rm, o, 64));
      if (l == 0) shr[(wave * RW + q) * groups + g] = rm;
    }
    // (one request for the block's rows, not one for each)
    __syncthreads();
    if ((int)threadIdx.x < here && r0 + threadIdx.x < n) {
      if (a.gy == 1) a.rmax[r0 + threadIdx.x] = shr[threadIdx.x];
      else atomicMax(a.rmax + r0 + threadIdx.x, shr[threadIdx.x]);
    }
    __syncthreads();
  }
  for (int o = lpr; o < 64; o <<= 1)
    cm = make_uint4(max(cm.x, (uint32_t)__shfl_xor((int)cm.x, o, 64)), max(cm.y, (uint32_t)__shfl_xor((int)cm.y, o, 64)),
                    max(cm.z, (uint32_t)__shfl_xor((int)cm.z, o, 64)), max(cm.w, (uint32_t)__shfl_xor((int)cm.w, o, 64)));
  if (g == 0) *reinterpret_cast<uint4*>(&sh[wave][l * 4]) = cm;
  __syncthreads();
  const int64_t k = threadIdx.x, col = (int64_t)by * AMAX_COLS + k;
  if (k < lpr * 4 && col < s.cols) raise(a.cmax + col, max(max(sh[0][k], sh[1][k]), max(sh[2][k], sh[3][k])));
}
constexpr int64_t AMAX_BLOCKS = 1024, ABSMAX_BLOCKS = 1024;

__device__ __forceinline__ void amax_of_w(const HeadTop& a, unsigned block) {
  __shared__ uint32_t sh[4];
  constexpr int U = 16;                  // units of 256 columns of a row, at a time
  const uint32_t parts = (uint32_t)((a.wcols + 255) / 256);
  const int64_t n = a.wrows * parts;
  uint32_t m = 0;
  for (int64_t i = (int64_t)block * U; i < n; i += (int64_t)a.w_blocks * U) {
    const int64_t r0 = i / parts;
    const uint32_t q0 = (uint32_t)(i - r0 * parts);
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t q = (q0 + u) / parts;
      const int64_t r = r0 + q, c = (int64_t)(q0 + u - q * parts) * 256 + threadIdx.x;
      x[u] = a.W[(r < a.wrows ? r : a.wrows - 1) * a.ldw + (c < a.wcols ? c : a.wcols - 1)];       // (behind the last ones: those again)
    }
#pragma unroll
    for (int u = 0; u < U; ++u) m = max(m, __float_as_uint(fabsf(x[u])));
  }
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) raise(a.wmax, max(max(sh[0], sh[1]), max(sh[2], sh[3])));
}

__global__ void __launch_bounds__(256) k_head_top(HeadTop a) {
  unsigned block = blockIdx.x;
  if (block < a.gx * a.gy) return amax_of_h(a, (int)(block / a.gy), (int)(block % a.gy));
  block -= a.gx * a.gy;
  if (block < a.w_blocks) return amax_of_w(a, block);
  clear_rows(a.clear, block - a.w_blocks);
}

__device__ __forceinline__ void split2(float x, _Float16* hi, _Float16* lo) {
  *hi = (_Float16)x;
  *lo = (_Float16)(x - (float)*hi);
}
// Of a gradient of a logit, times 2^P_EXP; lo times 2^LOW_EXP.
__device__ __forceinline__ void split_grad(float x, _Float16* hi, _Float16* lo) {
  *hi = (_Float16)x;
  *lo = (_Float16)((x - (float)*hi) * (float)(1 << LOW_EXP));
}
__device__ __forceinline__ v8h lowered(v8h x) { return x * (_Float16)(1.f / (1 << LOW_EXP)); }

// Fragments of the matrix by rows (reduction along columns: KS steps) and by columns (reduction along rows, weighted: KS_t steps), zeros behind
// the last row and column, a 64 x 64 tile a block.
// `all`: the largest value of everything, where it is scaled by one factor.
struct Pack {
  Source s;
  const uint32_t *rmax, *cmax, *all;
  _Float16* R;
  int64_t KS;
  _Float16* T;
  int64_t KS_t, row_tile;
  unsigned col_tiles, blocks;
};
// (H's, in the first blocks, and then W's, with the first piece of rows: W's blocks keep the memory busy that H's few do not)
__global__ void __launch_bounds__(256) k_pack(Pack first, Pack second, Clear clear) {
  if (blockIdx.x >= first.blocks + second.blocks) return clear_rows(clear, blockIdx.x - first.blocks - second.blocks);
  const bool is_first = blockIdx.x < first.blocks;
  const Pack& a = is_first ? first : second;
  const unsigned block = is_first ? blockIdx.x : blockIdx.x - first.blocks;
  const Source s = a.s;
  const uint32_t *__restrict__ rmax = a.rmax, *__restrict__ cmax = a.cmax, *__restrict__ all = a.all;
  _Float16 *__restrict__ R = a.R, *__restrict__ T = a.T;
  const int64_t KS = a.KS, KS_t = a.KS_t, row_tile = a.row_tile;
  const unsigned col_tiles = a.col_tiles;
  __shared__ float sh[64][65];
  __shared__ float wt[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
  const int64_t n = s.n(), tiles = up_to(n, row_tile) / 64 * col_tiles;
  for (int64_t tile = block; tile < tiles; tile += a.blocks) {
    const int64_t r0 = tile / col_tiles * 64, c0 = tile % col_tiles * 64;
    // four rows of 16 lanes at a time
    V4 y[4];
    float w[4];
    const int c4 = (lane & 15) * 4, rq = wave * 16 + (lane >> 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t r = r0 + rq + q * 4, v = s.row(r < n ? r : n - 1);
      const float* at = s.p + v * s.ld + c0 + c4;
      if (c0 + 64 <= s.cols) {
        y[q] = *reinterpret_cast<const V4u*>(at);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) y[q][k] = c0 + c4 + k < s.cols ? at[k] : 0.f;
      }
      w[q] = s.weight ? s.weight[v] : 1.f;
      if (r >= n) y[q] = V4{0.f, 0.f, 0.f, 0.f}, w[q] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int k = 0; k < 4; ++k) sh[rq + q * 4][c4 + k] = y[q][k];
      if ((lane & 15) == 0) wt[rq + q * 4] = w[q];
    }
    __syncthreads();
    auto put = [&](_Float16* to, int64_t frag, const float* x) {
      v8h hi, lo;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        _Float16 a, b;
        split2(x[t], &a, &b);
        hi[t] = a;
        lo[t] = b;
      }
      *reinterpret_cast<v8h*>(to + frag * 2 * FRAG + lane * 8) = hi;
      *reinterpret_cast<v8h*>(to + frag * 2 * FRAG + FRAG + lane * 8) = lo;
    };
    const int b = wave >> 1;                        // row block of the tile; a wave takes two of its four steps
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int ks = (wave & 1) * 2 + u, k = ks * 16 + half * 4;
      float x[8];
      if (R && c0 / 16 + ks < KS) {
        const int r = b * 32 + l32;
        const float f = scale_of(all ? *all : r0 + r < n ? rmax[r0 + r] : 0u);
#pragma unroll
        for (int t = 0; t < 8; ++t) x[t] = sh[r][k + (t >> 2) * 8 + (t & 3)] * f;
        put(R, (r0 / 32 + b) * KS + c0 / 16 + ks, x);
      }
      if (T && r0 / 16 + ks < KS_t) {
        const int c = b * 32 + l32;
        const float f = scale_of(all ? *all : c0 + c < s.cols ? cmax[c0 + c] : 0u);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const int r = k + (t >> 2) * 8 + (t & 3);
          x[t] = sh[r][c] * wt[r] * f;
        }
        put(T, (c0 / 32 + b) * KS_t + r0 / 16 + ks, x);
      }
    }
    __syncthreads();
  }
}
constexpr int64_t PACK_BLOCKS = 16384;

// ---------------------------------------------------------------- products

enum { LOSS, GRAD, SUMS, DIRECT, WHOLE };       // WHOLE: LOSS and GRAD, and what is in between, where one tile has all classes
enum { NEITHER, IS_A, IS_B };                   // which operand are gradients of logits
// The sums of dH: as many parts of the reduction as there are blocks for, by the rows that there are, which the host does not know.
constexpr int64_t LONG_PART = 32, SHORT_PART = 8, ONE_EACH = 256;
struct HeadSplits {
  int64_t blocks;                 // blocks of the launch, tiles of which have room in the sums
  int64_t nt;                     // tiles along the features
  int most, most_short;           // parts of LONG_PART and of SHORT_PART steps
  __device__ __forceinline__ int splits(int64_t rows) const {
    const int64_t tiles = up_to(rows, TM) / TM * nt;
    if (tiles == 0) return 1;
    const int64_t s = blocks / tiles < most ? blocks / tiles : most, t = ONE_EACH / tiles < most_short ? ONE_EACH / tiles : most_short;
    return (int)(s > t ? s : t > 1 ? t : 1);
  }
};
// The sums of dW: at most `most` parts of the rows that there are.
__device__ __forceinline__ int row_parts(int most, int64_t rows) {
  const int64_t s = rows / (SHORT_PART * 16);
  return (int)(s < 1 ? 1 : s < most ? s : most);
}
__device__ __forceinline__ float inv_count(const int64_t* total, int mean) { return mean ? 1.f / (float)(*total > 0 ? *total : 1) : 1.f; }
// Where a piece's dH goes, and what undoes its scales.
struct DhOut {
  float* dH;                      // (null: nowhere)
  int64_t ld;
  int d, mean;
  const int64_t* total;
  int64_t r0;
  const int32_t* idx;
  const float* weight;
  const uint32_t* wmax;
};
struct DhRow {
  float *p, ws, f;
  __device__ __forceinline__ DhRow(const DhOut& o, int64_t v) {
    const int64_t at = o.idx[o.r0 + v];
    p = o.dH + at * o.ld;
    ws = unscale_of(*o.wmax);
    f = inv_count(o.total, o.mean) * (o.weight ? o.weight[at] : 1.f) * (1.f / (1 << P_EXP));
  }
  __device__ __forceinline__ float operator()(float x) const { return x * ws * f; }
};
struct NtArgs {
  Clear clear;
  const _Float16 *A, *B;          // fragments; row blocks KSA, KSB steps apart
  int64_t KSA, KSB;
  int64_t b0;                     // first step of B, or (turned) first row block
  int64_t mt, nt;                 // tiles
  int64_t steps;                  // steps of the reduction (a multiple of 4); < 0: up to the piece's rows
  int splits;                     // parts of it, each with sums of its own
  // the piece
  const int64_t* total;
  int64_t r0, most;
  int rows_are;                   // which operand's rows are the piece's: 0 none, 1 A's, 2 B's
  // LOSS, GRAD: A's rows are classes from c0 on, B's rows of the piece
  int64_t c0, C;
  const uint32_t *wmax, *hmax;    // the largest values of W, of each row of H
  const int32_t* lab;
  float2* part;                   // LOSS: [class tile][most]: largest logit, sum of exponentials less it
  float* xlab;                    // LOSS: the label's logit
  const float2* norm;             // GRAD: of each row the largest logit m and P_EXP - log2 of the sum of exp(x - m): exp(x - lse) without a rounding of lse
  _Float16* P;                    // GRAD: fragments by rows (KSP steps)
  int64_t KSP;
  // WHOLE
  const int32_t* idx;
  const float* weight;
  float *row_loss, *row_lse;
  double* part_loss;              // [row tile]
  // SUMS
  float* out;                     // [split], split_part floats apart; row m of A and row n of B at m ms + n ns
  int64_t split_part, ms, ns;
  int add;
  HeadSplits by_rows;             // rows_are 1: how often the reduction is split follows from the number of rows, and split_part
  DhOut dh;                       // ... and where it is not split (and `add` is 0), its sums go here
  // DIRECT: a part of dW, finished: m_end features by n_end classes
  int64_t m_end, n_end;
  const uint32_t* fmax;           // H's largest values by feature
  int mean;
};

// Of a row's maximum and sum of exponentials: what its probabilities are made of, and its loss.
__device__ __forceinline__ float2 norm_of(float m, float z) { return make_float2(m, P_EXP - log2f(z)); }
__device__ __forceinline__ float row_end(float m, float z, float xlab, int64_t at, float* row_loss, float* row_lse) {
  const float lse = m + logf(z), l = lse - xlab;
  if (row_loss) row_loss[at] = l;
  if (row_lse) row_lse[at] = lse;
  return l;
}

// Column `lane % 16` of four rows of 16, each 16 lanes for themselves, which name four of a row each.
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4h turned(const _Float16* p) {
  return __builtin_bit_cast(v4h, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p));
}

constexpr int KT = 2, PAIR = 32 * KT;   // steps of a stage; values of the reduction in two stages, which go together
// C = A B^T of fragments, 256 x 128 a block, 64 x 128 a wave.  A wave reads its own rows of A straight into registers, a stage ahead, and the four
// waves share B through LDS, which is filled a stage ahead as well; two blocks a CU.
//
// TURN: B is the transpose of what its fragments hold, rows of the reduction by 16s of its own rows (for dH W's classes by features, for dW
// the gradients' rows by classes).  A stage is 32 rows of the reduction by 128, and lies in LDS as in memory; ds_read_tr gives 16 lanes the
// columns of four rows of 16.  (Each half of a fragment starts 640 bytes after the one before, so that what a quarter of the lanes reads
// lies in other banks than what the others do.)
constexpr int TURN_HALF = 320;    // halfs
constexpr int stage_halfs(bool turn) { return turn ? TN / 16 * 4 * TURN_HALF : TN / 32 * KT * 2 * FRAG; }
template <int EPI, int GRADS>
__device__ __forceinline__ void split_nt(const NtArgs& a, const unsigned block, _Float16* Bs) {
  constexpr bool TURN = GRADS != NEITHER;
  constexpr int STAGE = stage_halfs(TURN);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
  if (EPI != GRAD && block >= a.clear.from) return clear_rows(a.clear, block - a.clear.from);
  const int64_t rows = a.total ? piece_rows(a.total, a.r0, a.most) : 0;
  const int64_t mt = a.rows_are == 1 ? up_to(rows, TM) / TM : a.mt, nt = a.rows_are == 2 ? up_to(rows, TN) / TN : a.nt;
  if (EPI == DIRECT && a.r0 > 0 && rows == 0) return;                      // (nothing to add)
  const int splits = a.rows_are == 1 ? a.by_rows.splits(rows) : a.steps < 0 ? row_parts(a.splits, rows) : a.splits;
  // each XCD takes a contiguous part of the tiles, eight tiles of A over all of B after eight others
  const int64_t tiles = mt * nt, per = (tiles * splits + 7) / 8, ts = (int64_t)(block & 7) * per + (block >> 3);
  if ((int64_t)(block >> 3) >= per || ts >= tiles * splits) return;
  const int64_t split = ts / tiles, t = ts - split * tiles;
  const int64_t g = t / (8 * nt), gm = mt - g * 8 < 8 ? mt - g * 8 : 8, q = t - g * 8 * nt;
  const int64_t m0 = (g * 8 + q % gm) * TM, n0 = q / gm * TN;
  const int64_t pairs = (a.steps >= 0 ? a.steps : up_to(rows, PAIR) / 16) / (2 * KT);
  const int64_t s0 = pairs * split / splits * 2;                     // its first stage
  int todo = __builtin_amdgcn_readfirstlane((int)(pairs * (split + 1) / splits - s0 / 2));

  v16f acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const _Float16 *Ap0 = a.A + ((m0 / 32 + wave * 2) * a.KSA + s0 * KT) * 2 * FRAG + lane * 8, *Ap1 = Ap0 + a.KSA * 2 * FRAG;
  // a wave brings one of the four row blocks, or two of the eight 16s
  const _Float16* Bp = a.B + (TURN ? (a.b0 + s0) * a.KSB + n0 / 16 + wave * 2 : (n0 / 32 + wave) * a.KSB + a.b0 + s0 * KT) * 2 * FRAG + lane * 8;
  const int64_t b_step = (TURN ? a.KSB : KT) * 2 * FRAG;
  v8h ra[2][KT][2][2], rb[KT * 2];    // [stage in turn][step][row block][plane]
  auto fetch = [&](int to) {          // of the stage that the pointers have come to
#pragma unroll
    for (int u = 0; u < KT * 2; ++u) rb[u] = *reinterpret_cast<const v8h*>(Bp + u * FRAG);
#pragma unroll
    for (int u = 0; u < KT; ++u)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        ra[to][u][0][p] = *reinterpret_cast<const v8h*>(Ap0 + (u * 2 + p) * FRAG);
        ra[to][u][1][p] = *reinterpret_cast<const v8h*>(Ap1 + (u * 2 + p) * FRAG);
      }
    Ap0 += KT * 2 * FRAG, Ap1 += KT * 2 * FRAG, Bp += b_step;
  };
  auto stash = [&](int to) {
#pragma unroll
    for (int u = 0; u < KT * 2; ++u)
      *reinterpret_cast<v8h*>(Bs + to * STAGE + (TURN ? ((wave * 4 + u) * 2 + half) * TURN_HALF + l32 * 8 : (wave * KT * 2 + u) * FRAG + lane * 8)) = rb[u];
  };
  auto read_b = [&](v8h* b, int cur, int k) {          // k: step * 4 + row block
    if (TURN) {
      const int i = lane & 15, sixteen = (k & 3) * 2 + ((lane >> 4) & 1);
      const _Float16* f = Bs + cur * STAGE + (sixteen * 4 + (i & 1)) * TURN_HALF + ((k >> 2) * 16 + half * 4 + (i >> 2)) * 8 + ((i >> 1) & 1) * 4;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const v4h lo = turned(f + p * 2 * TURN_HALF), hi = turned(f + p * 2 * TURN_HALF + 64);
        b[p] = v8h{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      }
      return;
    }
    const _Float16* f = Bs + cur * STAGE + ((k & 3) * KT * 2 + (k >> 2) * 2) * FRAG + lane * 8;
    b[0] = *reinterpret_cast<const v8h*>(f);
    b[1] = *reinterpret_cast<const v8h*>(f + FRAG);
  };
  // (Loads have no condition, so that waits count only the loads that they wait for: the last stage fetches itself again.  The barriers to scheduling
  // keep them where they stand; they would be moved down to where they are used.)
  auto stage = [&](int cur, bool more) {
    if (!more) Ap0 -= KT * 2 * FRAG, Ap1 -= KT * 2 * FRAG, Bp -= b_step;
    v8h b[2][2];
    read_b(b[0], cur, 0);
    fetch(cur ^ 1);
#pragma unroll
    for (int k = 0; k < 4 * KT; ++k) {
      const v8h (&x)[2][2] = ra[cur][k >> 2];
      const v8h (&y)[2] = b[k & 1];
      if (k + 1 < 4 * KT) read_b(b[(k + 1) & 1], cur, k + 1);
      __builtin_amdgcn_sched_barrier(0);
      const int j = k & 3;
      const v8h y0 = GRADS == IS_A ? lowered(y[0]) : y[0];
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][1], y0, acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(GRADS == IS_B ? lowered(x[i][0]) : x[i][0], y[1], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[0], acc[i][j], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    stash(cur ^ 1);
    __syncthreads();
  };
  if (todo > 0) {
    fetch(0);
    stash(0);
    __syncthreads();
    do {
      stage(0, true);
      stage(1, --todo > 0);
    } while (todo > 0);
  }

  // lane l32 + 32 half of a 32 x 32 tile has column l32 and the rows 8 (e / 4) + 4 half + e % 4
  const int64_t mw = m0 + wave * 64;
  if constexpr (EPI == SUMS) {         // (whole tiles: what lies behind the last row and column is not looked at)
    if (a.dh.dH && splits == 1) {      // nothing to add up: rows of dH
      const int64_t n_end = (a.dh.d + 3) / 4 * 4;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int64_t v = mw + i * 32 + (e >> 2) * 8 + half * 4 + (e & 3);
          if (v >= rows) continue;
          const DhRow to(a.dh, v);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + j * 32 + l32;
            if (n < n_end) to.p[n] = n < a.dh.d ? to(acc[i][j][e]) : 0.f;
          }
        }
      return;
    }
    float* out = a.out + split * (a.rows_are == 1 ? mt * TM * a.ms : a.split_part) + (mw + half * 4) * a.ms + (n0 + l32) * a.ns;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float* o = out + i * 32 * a.ms + j * 32 * a.ns;
        if (a.ms == 1) {               // (fours of a lane's rows are neighbours)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            V4 x{acc[i][j][k * 4], acc[i][j][k * 4 + 1], acc[i][j][k * 4 + 2], acc[i][j][k * 4 + 3]};
            if (a.add) x += *reinterpret_cast<const V4*>(o + k * 8);
            *reinterpret_cast<V4*>(o + k * 8) = x;
          }
          continue;
        }
        float was[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) was[e] = a.add ? o[((e >> 2) * 8 + (e & 3)) * a.ms] : 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) o[((e >> 2) * 8 + (e & 3)) * a.ms] = was[e] + acc[i][j][e];
      }
    return;
  }
  if constexpr (EPI == DIRECT) {       // m: features, n: classes
    const float f = inv_count(a.total, a.mean) * (1.f / (1 << P_EXP));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t m = mw + i * 32 + half * 4, left = a.m_end - m;
      float fs[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {    // (whole tiles of them are there)
        const uint4 x = *reinterpret_cast<const uint4*>(a.fmax + m + k * 8);
        fs[k * 4] = unscale_of(x.x), fs[k * 4 + 1] = unscale_of(x.y), fs[k * 4 + 2] = unscale_of(x.z), fs[k * 4 + 3] = unscale_of(x.w);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + j * 32 + l32;
        if (n >= a.n_end) continue;
        float* o = a.out + m * a.ms + n * a.ns;
        if (a.ms == 1) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            V4 x{acc[i][j][k * 4] * fs[k * 4] * f, acc[i][j][k * 4 + 1] * fs[k * 4 + 1] * f, acc[i][j][k * 4 + 2] * fs[k * 4 + 2] * f, acc[i][j][k * 4 + 3] * fs[k * 4 + 3] * f};
            if (k * 8 + 4 <= left) {
              if (a.add) x += *reinterpret_cast<const V4u*>(o + k * 8);
              *reinterpret_cast<V4u*>(o + k * 8) = x;
            } else {
#pragma unroll
              for (int e = 0; e < 3; ++e)
                if (k * 8 + e < left) o[k * 8 + e] = (a.add ? o[k * 8 + e] : 0.f) + x[e];
            }
          }
        } else if (left >= 28) {
          float was[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) was[e] = a.add ? o[((e >> 2) * 8 + (e & 3)) * a.ms] : 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) o[((e >> 2) * 8 + (e & 3)) * a.ms] = was[e] + acc[i][j][e] * fs[e] * f;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int r = (e >> 2) * 8 + (e & 3);
            if (r < left) o[r * a.ms] = (a.add ? o[r * a.ms] : 0.f) + acc[i][j][e] * fs[e] * f;
          }
        }
      }
    }
    return;
  }
  const float ws = unscale_of(*a.wmax);
  const int64_t left = a.C - a.c0 - mw;                              // classes of the wave's 64
  const int lim = (left >= 64 ? 64 : left < 0 ? 0 : (int)left) - half * 4;
  // rows of the gradients of logits from norm: the gradients times 2^P_EXP, as fragments
  const bool read = a.c0 + mw < up_to(a.C, TN);                             // (nothing reads what is behind the last TN classes)
  auto put_grad = [&](int j, float2 nm) {
    const int64_t v = n0 + j * 32 + l32;
    const bool there = v < rows;
    const float hs = logit_scale(a.hmax[v], ws);
    const int64_t off = there ? a.lab[a.r0 + v] - (a.c0 + mw) : -1;
    const bool mine = off >= 0 && off < 64 && ((off >> 2) & 1) == half;
    const bool any = __ballot(mine);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(fmaf(acc[i][j][e], hs, -nm.x), LOG2E, nm.y));
      if (left < 64 || n0 + TN > rows) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!there || i * 32 + (e >> 2) * 8 + (e & 3) >= lim) p[e] = 0.f;
      }
      if (any) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (mine && off == i * 32 + (e >> 2) * 8 + half * 4 + (e & 3)) p[e] -= (float)(1 << P_EXP);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        v8h hi, lo;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          _Float16 x, y;
          split_grad(p[ks * 8 + u], &x, &y);
          hi[u] = x;
          lo[u] = y;
        }
        _Float16* to = a.P + (((n0 / 32 + j) * a.KSP + (mw + i * 32) / 16 + ks) * 2) * FRAG + lane * 8;
        // (past the caches, which have W and H to keep: 8,192 rows x 131,072 classes 6.80 -> 6.52 ms)
        __builtin_nontemporal_store(hi, reinterpret_cast<v8h*>(to));
        __builtin_nontemporal_store(lo, reinterpret_cast<v8h*>(to + FRAG));
      }
    }
  };
  if constexpr (EPI == LOSS) {
    if (a.P && read) {                 // the sums, for k_head_grad, where the gradients will be
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            _Float16* to = a.P + (((n0 / 32 + j) * a.KSP + (mw + i * 32) / 16 + ks) * 2) * FRAG + lane * 8;
            auto four = [&](int e) { return V4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]}; };
            __builtin_nontemporal_store(four(ks * 8), reinterpret_cast<V4*>(to));
            __builtin_nontemporal_store(four(ks * 8 + 4), reinterpret_cast<V4*>(to + FRAG));
          }
    }
  }
  if constexpr (EPI == LOSS || EPI == WHOLE) {
    float2* red = reinterpret_cast<float2*>(Bs);      // [wave][column]
    float2* norm = red + 4 * TN;                      // WHOLE: [column]
    float* xlab = reinterpret_cast<float*>(norm + TN);
    double* sums = reinterpret_cast<double*>(xlab + TN);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t v = n0 + j * 32 + l32;
      const bool there = v < rows;
      const float hs = logit_scale(a.hmax[v], ws);
      float m = -INFINITY;
      if (left < 64) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (i * 32 + (e >> 2) * 8 + (e & 3) >= lim) acc[i][j][e] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
      m = fmaxf(m, __shfl_xor(m, 32, 64)) * hs;
      const float m1 = m == -INFINITY ? 0.f : m;      // (a wave behind the last class: exp(-inf) throughout)
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) z += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], hs, -m1) * LOG2E);
      z += __shfl_xor(z, 32, 64);
      if (half == 0) red[wave * TN + j * 32 + l32] = make_float2(m, z);
      const int64_t off = there ? a.lab[a.r0 + v] - (a.c0 + mw) : -1;
      const bool mine = off >= 0 && off < 64 && ((off >> 2) & 1) == half;
      if (__ballot(mine)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (mine && off == i * 32 + (e >> 2) * 8 + half * 4 + (e & 3)) (EPI == WHOLE ? xlab[j * 32 + l32] : a.xlab[v]) = acc[i][j][e] * hs;
      }
    }
    __syncthreads();
    float l = 0.f;
    if (tid < TN && n0 + tid < rows) {
      float m = -INFINITY, z = 0.f;
      for (int w = 0; w < 4; ++w) m = fmaxf(m, red[w * TN + tid].x);
      for (int w = 0; w < 4; ++w) {
        const float2 p = red[w * TN + tid];
        z += p.x == -INFINITY ? p.y : p.y * exp_less(p.x, m);
      }
      if constexpr (EPI == LOSS) {
        a.part[m0 / TM * a.most + n0 + tid] = make_float2(m, z);
      } else {
        norm[tid] = norm_of(m, z);
        const int64_t r = a.r0 + n0 + tid, at = a.idx[r];
        l = row_end(m, z, a.lab[r] < a.C ? xlab[tid] : NAN, at, a.row_loss, a.row_lse);
      }
    }
    if constexpr (EPI == WHOLE) {
      // (in 64 bits)
      double mine = 0.0;
      if (tid < TN && n0 + tid < rows) mine = a.weight ? (double)a.weight[a.idx[a.r0 + n0 + tid]] * (double)l : (double)l;
      for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
      if (lane == 0 && wave < 2) sums[wave] = mine;
      __syncthreads();
      if (tid == 0) a.part_loss[n0 / TN] = sums[0] + sums[1];
      if (a.P && read) {
#pragma unroll
        for (int j = 0; j < 4; ++j) put_grad(j, n0 + j * 32 + l32 < rows ? norm[j * 32 + l32] : make_float2(0.f, 0.f));
      }
    }
    return;
  }
  if constexpr (EPI == GRAD) {
    if (!read) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) put_grad(j, n0 + j * 32 + l32 < rows ? a.norm[n0 + j * 32 + l32] : make_float2(0.f, 0.f));
  }
}
template <int EPI, int GRADS>
__global__ void __launch_bounds__(256, 2) k_split_nt(NtArgs a) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(GRADS != NEITHER)];
  split_nt<EPI, GRADS>(a, blockIdx.x, Bs);
}
// dH's and dW's sums, which do not wait for each other, the second behind the first `from` blocks, where those have no more tiles than there are CUs.  us of a call, so |
// in two launches: 100 rows x 64 features x 300 classes 52 | 63, 1,000 x 256 x 1,000 73 | 84, 20,000 x 128 x 300 126 | 131; of more tiles the two take each
// other's place in the caches: 60,000 x 256 x 172 217 | 210, 233,000 x 256 x 41 605 | 580.
__global__ void __launch_bounds__(256, 2) k_split_both(NtArgs first, NtArgs second, unsigned from) {
  __shared__ __attribute__((aligned(16))) _Float16 Bs[2 * stage_halfs(true)];
  if (blockIdx.x < from) return split_nt<SUMS, IS_A>(first, blockIdx.x, Bs);
  split_nt<SUMS, IS_B>(second, blockIdx.x - from, Bs);
}

// ---------------------------------------------------------------- what the products leave

// Blocks of 64 rows, 16 parts of the class tiles each.  part_loss[block] = sum of its rows' weighted losses.
__global__ void __launch_bounds__(1024) k_head_join(const float2* __restrict__ part, int64_t tiles, int64_t most, const int64_t* __restrict__ total, int64_t r0,
                                                    const int32_t* __restrict__ idx, const int32_t* __restrict__ lab, int64_t C,
                                                    const float* __restrict__ weight, const float* __restrict__ xlab, float2* __restrict__ norm,
                                                    float* __restrict__ row_loss, float* __restrict__ row_lse, double* __restrict__ part_loss) {
  __shared__ float2 sh[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t rows = piece_rows(total, r0, most);
  double mine = 0.0;
  for (int64_t v0 = (int64_t)blockIdx.x * 64; v0 < rows; v0 += (int64_t)gridDim.x * 64) {
    const int64_t v = v0 + lane;
    float m = -INFINITY, z = 0.f;
    if (v < rows)
#pragma unroll 4
      for (int64_t t = wave; t < tiles; t += 16) {
        const float2 p = part[t * most + v];
        const float n = fmaxf(m, p.x);
        z = (m == -INFINITY ? z : z * exp_less(m, n)) + (p.x == -INFINITY ? p.y : p.y * exp_less(p.x, n));      // (0 or NaN of what has no maximum)
        m = n;
      }
    sh[wave][lane] = make_float2(m, z);
    __syncthreads();
    if (wave == 0) {
      m = -INFINITY;
      for (int w = 0; w < 16; ++w) m = fmaxf(m, sh[w][lane].x);
      z = 0.f;
      for (int w = 0; w < 16; ++w) z += sh[w][lane].x == -INFINITY ? sh[w][lane].y : sh[w][lane].y * exp_less(sh[w][lane].x, m);
      if (v < rows) {
        norm[v] = norm_of(m, z);
        const int64_t at = idx[r0 + v];
        const float l = row_end(m, z, lab[r0 + v] < C ? xlab[v] : NAN, at, row_loss, row_lse);
        mine += weight ? (double)weight[at] * (double)l : (double)l;
      }
    }
    __syncthreads();
  }
  if (wave != 0) return;
  for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
  if (lane == 0) part_loss[blockIdx.x] = mine;
}

// The gradients of logits whose sums LOSS has kept in their place.  A wave takes fragments of 32 rows, GRAD_FRAGS of them one after the other.
// What this costs is 8 bytes a logit, against the product once more in GRAD: from 193 features on (which are 256 in the product) it is less, and where the sums are
// so few that a product's launch costs more than its work.  us of a call, kept | made again: 2,048 rows x 32,768 classes by 128 features 398 | 384, 256 478 | 497, 602
// 888 | 1,015, 1,024 1,246 | 1,490; 20,000 x 200 x 3,000 467 | 490; 8,192 x 512 x 131,072 10.7 | 11.8 ms; 300 x 128 x 1,000 (1 MB) 69 | 75, 5,000 x 64 x 500 (10 MB)
// 80 | 83, 3,000 x 64 x 5,000 (60 MB) 125 | 120.
constexpr int GRAD_FRAGS = 8;
constexpr int64_t GRAD_BLOCKS = 16384, KEEP_WIDTH = 193, KEEP_BYTES = (int64_t)16 << 20;
__global__ void __launch_bounds__(256) k_head_grad(_Float16* __restrict__ P, int64_t KSP, const int64_t* __restrict__ total, int64_t r0, int64_t most, int64_t C,
                                                   const uint32_t* __restrict__ wmax, const uint32_t* __restrict__ hmax, const int32_t* __restrict__ lab,
                                                   const float2* __restrict__ norm) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int64_t rows = piece_rows(total, r0, most), KS = up_to(C, TN) / 16, per = (KS + GRAD_FRAGS - 1) / GRAD_FRAGS, all = up_to(rows, TN) / 32 * per;
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < all; t += (int64_t)gridDim.x * 4) {
    const int64_t b = t / per, k0 = (t - b * per) * GRAD_FRAGS, v = b * 32 + l32;
    const bool there = v < rows;
    _Float16* at = P + (b * KSP + k0) * 2 * FRAG + lane * 8;
    V4 x[GRAD_FRAGS][2];
#pragma unroll
    for (int k = 0; k < GRAD_FRAGS; ++k) {
      const _Float16* from = at + (k0 + k < KS ? k : 0) * 2 * FRAG;
      x[k][0] = *reinterpret_cast<const V4*>(from), x[k][1] = *reinterpret_cast<const V4*>(from + FRAG);
    }
    const float hs = logit_scale(hmax[v], unscale_of(*wmax));
    const float2 nm = there ? norm[v] : make_float2(0.f, 0.f);
    const int64_t c0 = k0 * 16 + half * 4, off = there ? lab[r0 + v] - c0 : -1, lim = there ? C - c0 : 0;      // (against the classes of the lane: k 16 + u / 4 8 + u % 4)
#pragma unroll
    for (int k = 0; k < GRAD_FRAGS; ++k) {
      if (k0 + k >= KS) break;
      v8h hi, lo;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int c = k * 16 + (u >> 2) * 8 + (u & 3);
        float p = __builtin_amdgcn_exp2f(fmaf(fmaf(x[k][u >> 2][u & 3], hs, -nm.x), LOG2E, nm.y));
        if (c >= lim) p = 0.f;
        if (c == off) p -= (float)(1 << P_EXP);
        _Float16 a, l;
        split_grad(p, &a, &l);
        hi[u] = a, lo[u] = l;
      }
      __builtin_nontemporal_store(hi, reinterpret_cast<v8h*>(at + k * 2 * FRAG));
      __builtin_nontemporal_store(lo, reinterpret_cast<v8h*>(at + k * 2 * FRAG + FRAG));
    }
  }
}

// ---- What comes after a piece's products, in one launch: the loss (a block), dH and dW from the sums of their splits.
struct LossArgs {
  const double* part;
  int64_t n;                     // parts, per_piece of them a piece of `most` rows; the i-th has a value if there is a row i row_step
  int64_t per_piece, most, row_step;
  const int64_t* total;
  int mean;
  float* loss;                   // (null: later)
};
__device__ __forceinline__ void head_loss(const LossArgs& a) {
  __shared__ double sh[256];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < a.n; i += 256) {
    const int64_t k = i / a.per_piece, r = (i - k * a.per_piece) * a.row_step;
    if (r < piece_rows(a.total, k * a.most, a.most)) s += a.part[i];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.loss = *a.total > 0 ? (float)(sh[0] / (a.mean ? (double)*a.total : 1.0)) : 0.f;
}

constexpr int64_t DH_BLOCKS = 8192;
struct DhArgs {
  DhOut to;
  const float* sums;
  HeadSplits by_rows;
  int64_t most, pitch;
  int in_place;                  // what is not split is there already
  unsigned blocks;
};
__device__ __forceinline__ void head_dh(const DhArgs& a, unsigned block) {
  const int64_t rows = piece_rows(a.to.total, a.to.r0, a.most);
  const int nv = (a.to.d + 3) / 4, splits = a.by_rows.splits(rows);
  if (a.in_place && splits == 1) return;
  const int64_t part = up_to(rows, TM) * a.pitch;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < rows * nv; i += (int64_t)a.blocks * 256) {
    const int64_t v = i / nv;
    const int c = (int)(i % nv) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = 0; k < splits; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(a.sums + k * part + v * a.pitch + c);
      s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
    const DhRow to(a.to, v);
    auto out = [&](float x, int k) { return c + k < a.to.d ? to(x) : 0.f; };
    *reinterpret_cast<float4*>(to.p + c) = make_float4(out(s.x, 0), out(s.y, 1), out(s.z, 2), out(s.w, 3));
  }
}

// dW's part [rows x cols] at out (pitch ld): the splits' sums (pitch cols_p, rows_p rows each), scaled by what undoes hmax along rows or columns
struct DwArgs {
  const float* sums;
  int most_parts;
  int64_t most, rows_p, cols_p, rows, cols;
  const uint32_t* hmax;
  int along_rows;
  const int64_t* total;
  int64_t r0;
  int mean, add;
  float* out;
  int64_t ld;
  unsigned blocks;
};
__device__ __forceinline__ void head_dw(const DwArgs& a, unsigned block) {
  if (a.r0 > 0 && *a.total <= a.r0) return;       // (nothing to add)
  const int64_t i = (int64_t)block * 256 + threadIdx.x, r = i / a.cols, c = i - r * a.cols;
  if (r >= a.rows) return;
  const int splits = row_parts(a.most_parts, piece_rows(a.total, a.r0, a.most));
  float s = 0.f;
#pragma unroll 16
  for (int k = 0; k < splits; ++k) s += a.sums[((int64_t)k * a.rows_p + r) * a.cols_p + c];
  // (the inverse scale first: of a feature below 2^-97 it is near the smallest float, and what follows would take it below)
  s = s * unscale_of(a.hmax[a.along_rows ? r : c]) * ((1.f / (1 << P_EXP)) * inv_count(a.total, a.mean));
  float* o = a.out + r * a.ld + c;
  *o = a.add ? *o + s : s;
}

__global__ void __launch_bounds__(256) k_head_end(LossArgs loss, DhArgs dh, DwArgs dw, Clear clear) {
  if (blockIdx.x >= clear.from) return clear_rows(clear, blockIdx.x - clear.from);
  unsigned block = blockIdx.x;
  if (loss.loss) {
    if (block == 0) return head_loss(loss);
    --block;
  }
  if (block < dh.blocks) return head_dh(dh, block);
  head_dw(dw, block - dh.blocks);
}
int head_end(ht_ctx* ctx, hipStream_t st, const LossArgs& loss, const DhArgs& dh, const DwArgs& dw, Clear clear = Clear{}) {
  clear.from = (loss.loss ? 1 : 0) + dh.blocks + dw.blocks;
  if (clear.from + clear.blocks == 0) return HT_OK;
  k_head_end<<<clear.from + clear.blocks, 256, 0, st>>>(loss, dh, dw, clear);
  HT_LAUNCH_CHECK(ctx);
  return HT_OK;
}

struct HeadPlan {
  int64_t Cp, Rp;                    // classes and rows of a piece
  int64_t KSd, steps_d;              // steps over d as operands hold them, and of a reduction
  int64_t Cpad, dpad;
  int splits_w;
  HeadSplits by_rows;
  int64_t sum_rows;                  // of dH's sums
};

HeadPlan head_plan(int64_t V, int64_t d, int64_t C, bool in_out, size_t bytes) {
  HeadPlan p{};
  p.KSd = up_to(d, TN) / 16;
  p.steps_d = up_to(d, PAIR) / 16;
  p.Cpad = up_to(C, TM);
  p.dpad = up_to(d, TM);
  // a row takes 4 bytes a value of its own, by rows and by features, and of its gradient, 4 a class of the piece, and 8 a tile of classes
  const int64_t own = 12 * p.dpad + 8 * (p.Cpad / TM), least = std::min<int64_t>(p.Cpad, HEAD_CLASSES);
  p.Rp = (int64_t)bytes / (4 * least + own) / TM * TM;
  p.Rp = std::max<int64_t>(TM, std::min(p.Rp, up_to(V, TM)));
  if (d >= KEEP_WIDTH && (int64_t)HEAD_PIECE / (4 * p.Cpad) >= 2048) p.Rp = std::min<int64_t>(p.Rp, (int64_t)HEAD_PIECE / (4 * p.Cpad) / TM * TM);
  // ... and as many classes as memory allows: every piece of them reads and writes the sums that dH is made of
  p.Cp = std::max(least, std::min<int64_t>(p.Cpad, (int64_t)std::min(bytes, HEAD_PIECE) / (4 * p.Rp) / TM * TM));
  // Parts of a reduction: for dH of 512 values each at least while there are blocks for two a CU, and of 128 while there are for one (a block that is alone on its CU
  // waits for its loads, 3 us for 64 values); for dW of 128, one block a CU (what is not split needs no sums: 2,048 rows x 32,768 classes 602 | 593 us).  Short
  // parts take 12 us off a call with 100 rows x 64 features x 300 classes, 18 off 1,000 x 256 x 1,000, none off 3,000 x 256 x 5,000 (two short ones a CU: 15 more).
  const int64_t nt = up_to(d, TN) / TN, mt = p.Rp / TM, steps = p.Cp / 16, tiles_w = p.dpad / TM * (p.Cp / TN);
  auto parts = [](int64_t a, int64_t b, int64_t most) { return (int)std::max<int64_t>(1, std::min({a, b, most})); };
  p.splits_w = parts(ONE_EACH / tiles_w, p.Rp / 16 / SHORT_PART, 128);
  const int most = parts(2 * ONE_EACH / nt, steps / LONG_PART, 128), most_short = parts(ONE_EACH / nt, steps / SHORT_PART, 128);       // (of one tile of rows)
  p.by_rows = HeadSplits{std::max<int64_t>(mt * nt, std::min<int64_t>(2 * ONE_EACH / nt, mt * std::max(most, most_short)) * nt), nt, most, most_short};
  p.sum_rows = p.by_rows.blocks / nt * TM;
  return p;
}

// (and sets a->clear.from)
int nt_blocks(ht_ctx* ctx, NtArgs* a, unsigned* grid) {
  const int64_t blocks = up_to(a->rows_are == 1 ? a->by_rows.blocks : a->mt * a->nt * a->splits, 8);
  if (blocks >= (1 << 24)) return ht_set_err(ctx, HT_ESHAPE, "head: %lld tiles in one product", (long long)blocks);
  a->clear.from = (unsigned)blocks;
  *grid = a->clear.from + a->clear.blocks;
  return HT_OK;
}
int split_nt(ht_ctx* ctx, hipStream_t st, int epi, NtArgs a) {
  unsigned grid = 0;
  HT_TRY(nt_blocks(ctx, &a, &grid));
  if (epi == WHOLE) k_split_nt<WHOLE, NEITHER><<<grid, 256, 0, st>>>(a);
  else if (epi == LOSS) k_split_nt<LOSS, NEITHER><<<grid, 256, 0, st>>>(a);
  else if (epi == GRAD) k_split_nt<GRAD, NEITHER><<<grid, 256, 0, st>>>(a);
  else if (epi == DIRECT) k_split_nt<DIRECT, IS_B><<<grid, 256, 0, st>>>(a);
  else if (a.rows_are == 1) k_split_nt<SUMS, IS_A><<<grid, 256, 0, st>>>(a);
  else k_split_nt<SUMS, IS_B><<<grid, 256, 0, st>>>(a);
  HT_LAUNCH_CHECK(ctx);
  return HT_OK;
}
int split_both(ht_ctx* ctx, hipStream_t st, NtArgs a, NtArgs b) {
  unsigned first = 0, second = 0;
  HT_TRY(nt_blocks(ctx, &a, &first));
  HT_TRY(nt_blocks(ctx, &b, &second));
  first = (unsigned)up_to(first, 8);
  k_split_both<<<first + second, 256, 0, st>>>(a, b, first);
  HT_LAUNCH_CHECK(ctx);
  return HT_OK;
}

int head_run(ht_ctx* ctx, const ht_head_desc* D, const ht_tensor* H, const ht_tensor* W, const int32_t* labels, const float* weight,
             float* loss, float* row_loss, float* row_lse, const ht_tensor* dH, const ht_tensor* dW, size_t bytes) {
  const int64_t V = H->rows, d = D->d, C = D->n_classes;
  const bool in_out = D->w_form == HT_W_IN_OUT, grad = dH || dW;
  const int mean = D->reduction == HT_REDUCE_MEAN;
  hipStream_t st = ctx->stream;
  const HeadPlan p = head_plan(V, d, C, in_out, bytes);
  const int64_t pieces = std::max<int64_t>(1, ceil_div64(V, p.Rp)), ct = p.Cpad / TM;
  const int64_t rpb = std::max<int64_t>(256, up_to(ceil_div64(std::max<int64_t>(V, 1), ROW_BLOCKS), 256)), rb = std::max<int64_t>(1, ceil_div64(V, rpb));
  const bool whole = p.Cpad == TM;                         // all classes in one tile
  const bool keep = grad && !whole && p.Cp == p.Cpad && (d >= KEEP_WIDTH || p.Rp * p.Cp * 4 <= KEEP_BYTES);
  const int64_t row_step = whole ? TN : 64, jb = whole ? p.Rp / TN : std::min<int64_t>(p.Rp / 64, 1024);      // a piece's sums of losses
  const int64_t KSR = p.Rp / 16;

  OpsBlock m;
  const auto cnt = m.add<int32_t>(rb);
  const auto idx = m.add<int32_t>(V), lab = m.add<int32_t>(V);
  const auto total = m.add<int64_t>(1);
  const int64_t n_max = 4 + p.Rp + p.dpad;
  const auto mx = m.add<uint32_t>(n_max);                        // the largest values: of W (and three words), of H by row, by feature
  const auto Wf = m.add<_Float16>(p.Cpad * p.KSd * 32);
  const auto Hf = m.add<_Float16>(p.Rp * p.KSd * 32);
  const auto part = m.add<float2>(ct * p.Rp);
  const auto xlab = m.add<float>(p.Rp);
  const auto norm = m.add<float2>(p.Rp);
  const auto ploss = m.add<double>(pieces * jb);
  const auto Ht = m.add<_Float16>(dW ? p.dpad * KSR * 32 : 0);
  const auto P = m.add<_Float16>(grad ? p.Rp * p.Cp * 2 : 0);
  const auto sh = m.add<float>(dH ? p.sum_rows * p.dpad : 0);
  const auto sw = m.add<float>(dW && p.splits_w > 1 ? p.splits_w * p.Cp * p.dpad : 0);
  HT_TRY(bytes > HEAD_LEAN ? m.take_if_room(ctx) : m.take(ctx));

  uint32_t *wmax = m.at(mx), *hmax_v = wmax + 4, *hmax_j = hmax_v + p.Rp;
  const unsigned clear_blocks = (unsigned)std::min<int64_t>(ceil_div64(n_max, 4096), 1024);
  if (V <= LIST_ROWS) {
    const unsigned blocks = (unsigned)std::max<int64_t>(1, ceil_div64(V, 256));
    k_head_list<<<blocks + clear_blocks, 256, 0, st>>>(labels, V, blocks, m.at(idx), m.at(lab), m.at(total), row_loss, row_lse, dH ? dH->ptr : nullptr, dH ? dH->ld : 0,
                                                       (int)d, (uint4*)wmax, n_max / 4);
    HT_LAUNCH_CHECK(ctx);
  } else {
    k_head_count<<<(unsigned)rb + clear_blocks, 256, 0, st>>>(labels, V, rpb, m.at(cnt), (unsigned)rb, (uint4*)wmax, n_max / 4);
    HT_LAUNCH_CHECK(ctx);
    k_head_place<<<(unsigned)rb, 256, 0, st>>>(labels, V, rpb, m.at(cnt), m.at(idx), m.at(lab), m.at(total), row_loss, row_lse);
    HT_LAUNCH_CHECK(ctx);
  }
  const Source w{W->ptr, W->ld, W->rows, W->cols, nullptr, nullptr, nullptr, 0};
  HeadTop t{};
  t.rmax = hmax_v, t.cmax = hmax_j;
  t.gy = (unsigned)ceil_div64(d, AMAX_COLS), t.gx = (unsigned)std::max<int64_t>(1, std::min(ceil_div64(p.Rp, 4 * RW * (64 / amax_lanes(d))), std::max<int64_t>(1, AMAX_BLOCKS / t.gy)));
  t.W = w.p, t.ldw = w.ld, t.wrows = w.rows, t.wcols = w.cols, t.wmax = wmax;
  int64_t cleared = dH && V > LIST_ROWS ? 0 : V;
  auto clear_to = [&](double part) {
    if (V * d * 4 < CLEAR_SHARED) part = 1.0;
    Clear c{labels, dH ? dH->ptr : nullptr, dH ? dH->ld : 0, (int)d, cleared, part >= 1.0 ? V : std::max(cleared, std::min<int64_t>(V, up_to((int64_t)(part * (double)V), 256))), 0, 0};
    c.blocks = (unsigned)std::min(ceil_div64(c.v1 - c.v0, 256), CLEAR_BLOCKS);
    cleared = c.v1;
    return c;
  };
  for (int64_t k = 0; k < pieces; ++k) {
    const int64_t r0 = k * p.Rp;
    if (k > 0) HT_TRY(ht_fill_zero(ctx, st, hmax_v, (size_t)(p.Rp + p.dpad) * 4));
    const Source s{H->ptr, H->ld, p.Rp, d, m.at(idx), weight, m.at(total), r0};
    t.s = s;
    t.w_blocks = k > 0 ? 0 : (unsigned)std::min<int64_t>(ceil_div64(w.rows * ceil_div64(w.cols, 256), 64), ABSMAX_BLOCKS);
    t.clear = clear_to(CLEAR_TOP);
    k_head_top<<<t.gx * t.gy + t.w_blocks + t.clear.blocks, 256, 0, st>>>(t);
    HT_LAUNCH_CHECK(ctx);
    const unsigned hc = (unsigned)ceil_div64(d, 64);
    const Pack ph{s, hmax_v, hmax_j, nullptr, m.at(Hf), p.KSd, dW ? m.at(Ht) : nullptr, KSR, TN, hc, (unsigned)std::min(p.Rp / 64 * hc, PACK_BLOCKS / 2)};
    // by classes: W's rows, or its columns
    const int64_t rt = up_to(w.rows, in_out ? 64 : TM) / 64, wc = up_to(w.cols, in_out ? TM : 64) / 64;
    const Pack pw{w, nullptr, nullptr, wmax, in_out ? nullptr : m.at(Wf), p.KSd, in_out ? m.at(Wf) : nullptr, p.KSd, in_out ? 64 : TM, (unsigned)wc,
                  k > 0 ? 0 : (unsigned)std::min(rt * wc, PACK_BLOCKS)};
    const Clear cp = clear_to(CLEAR_PACK);
    k_pack<<<ph.blocks + pw.blocks + cp.blocks, 256, 0, st>>>(ph, pw, cp);
    HT_LAUNCH_CHECK(ctx);
    NtArgs a{};
    a.total = m.at(total), a.r0 = r0, a.most = p.Rp;
    a.splits = 1;
    a.clear = clear_to(CLEAR_LOGITS);
    a.C = C, a.wmax = wmax, a.hmax = hmax_v, a.lab = m.at(lab), a.part = m.at(part), a.xlab = m.at(xlab), a.norm = m.at(norm);
    a.A = m.at(Wf), a.KSA = p.KSd, a.B = m.at(Hf), a.KSB = p.KSd;
    a.mt = ct, a.nt = p.Rp / TN, a.steps = p.steps_d, a.rows_are = 2;
    if (whole) {
      a.idx = m.at(idx), a.weight = weight, a.row_loss = row_loss, a.row_lse = row_lse, a.part_loss = m.at(ploss) + k * jb;
      a.P = grad ? m.at(P) : nullptr, a.KSP = TM / 16;
      HT_TRY(split_nt(ctx, st, WHOLE, a));
    } else {
      if (keep) a.P = m.at(P), a.KSP = p.Cp / 16;
      HT_TRY(split_nt(ctx, st, LOSS, a));
      k_head_join<<<(unsigned)jb, 1024, 0, st>>>(m.at(part), ct, p.Rp, m.at(total), r0, m.at(idx), m.at(lab), C, weight, m.at(xlab), m.at(norm), row_loss, row_lse,
                                                 m.at(ploss) + k * jb);
      HT_LAUNCH_CHECK(ctx);
    }
    // (with the last piece's)
    const LossArgs last{m.at(ploss), pieces * jb, jb, p.Rp, row_step, m.at(total), mean, k == pieces - 1 ? loss : nullptr};
    if (!grad) {
      HT_TRY(head_end(ctx, st, last, DhArgs{}, DwArgs{}));
      continue;
    }
    const DhOut to{dH ? dH->ptr : nullptr, dH ? dH->ld : 0, (int)d, mean, m.at(total), r0, m.at(idx), weight, wmax};
    DwArgs dw{};
    for (int64_t c0 = 0; c0 < p.Cpad; c0 += p.Cp) {
      const int64_t cp = std::min(p.Cp, p.Cpad - c0), cls = std::min(cp, C - c0);
      NtArgs g = a;
      g.clear = Clear{};
      g.c0 = c0, g.A = m.at(Wf) + c0 * p.KSd * 32, g.mt = cp / TM;
      g.P = m.at(P), g.KSP = p.Cp / 16;
      if (keep) {
        const int64_t waves = p.Rp / 32 * ceil_div64(p.Cpad / 16, GRAD_FRAGS);
        k_head_grad<<<(unsigned)std::min(ceil_div64(waves, 4), GRAD_BLOCKS), 256, 0, st>>>(m.at(P), p.Cp / 16, m.at(total), r0, p.Rp, C, wmax, hmax_v, m.at(lab), m.at(norm));
        HT_LAUNCH_CHECK(ctx);
      } else if (!whole) {
        HT_TRY(split_nt(ctx, st, GRAD, g));
      }
      NtArgs h{};
      const bool both = dH && dW && p.splits_w > 1 && p.Rp / TM * p.by_rows.nt <= ONE_EACH;
      if (dH) {
        h.total = m.at(total), h.r0 = r0, h.most = p.Rp, h.rows_are = 1;
        h.A = m.at(P), h.KSA = p.Cp / 16, h.B = m.at(Wf), h.KSB = p.KSd, h.b0 = c0 / 32;
        h.mt = p.Rp / TM, h.nt = up_to(d, TN) / TN, h.steps = up_to(cls, PAIR) / 16, h.by_rows = p.by_rows;
        h.out = m.at(sh), h.ms = p.dpad, h.ns = 1, h.add = c0 > 0;
        if (p.Cp == p.Cpad) h.dh = to;
        h.clear = clear_to(CLEAR_DH);
        if (!both) HT_TRY(split_nt(ctx, st, SUMS, h));
      }
      if (dW) {
        NtArgs w{};
        w.total = m.at(total), w.r0 = r0, w.most = p.Rp, w.steps = -1, w.splits = p.splits_w;
        w.A = m.at(Ht), w.KSA = KSR, w.B = m.at(P), w.KSB = p.Cp / 16;
        w.mt = p.dpad / TM, w.nt = ceil_div64(cls, TN);
        const int64_t rows = in_out ? d : cls, cols = in_out ? cls : d;
        const int add = k > 0 || D->accumulate_dW;
        w.clear = clear_to(CLEAR_DW);
        float* out = dW->ptr + (in_out ? c0 : c0 * dW->ld);
        if (p.splits_w == 1) {
          w.out = out, w.ms = in_out ? dW->ld : 1, w.ns = in_out ? 1 : dW->ld, w.m_end = d, w.n_end = cls, w.fmax = hmax_j, w.mean = mean, w.add = add;
          HT_TRY(split_nt(ctx, st, DIRECT, w));
          continue;
        }
        const int64_t rows_p = in_out ? p.dpad : p.Cp, cols_p = in_out ? p.Cp : p.dpad;
        w.out = m.at(sw), w.split_part = rows_p * cols_p, w.ms = in_out ? cols_p : 1, w.ns = in_out ? 1 : cols_p;
        HT_TRY(both ? split_both(ctx, st, h, w) : split_nt(ctx, st, SUMS, w));
        const DwArgs part{m.at(sw), p.splits_w, p.Rp, rows_p, cols_p, rows, cols, hmax_j, in_out, m.at(total), r0, mean, add, out, dW->ld, (unsigned)ceil_div64(rows * cols, 256)};
        if (c0 + p.Cp < p.Cpad) HT_TRY(head_end(ctx, st, LossArgs{}, DhArgs{}, part));
        else dw = part;
      }
    }
    const unsigned dh_blocks = dH ? (unsigned)std::min(ceil_div64(p.Rp * ((d + 3) / 4), 256), DH_BLOCKS) : 0;
    HT_TRY(head_end(ctx, st, last, DhArgs{to, m.at(sh), p.by_rows, p.Rp, p.dpad, p.Cp == p.Cpad, dh_blocks}, dw, clear_to(1.0)));
  }
  return HT_OK;
}

}  // namespace

extern "C" int ht_head_loss(ht_ctx* ctx, const ht_head_desc* desc, const ht_tensor* H, const ht_tensor* W, const int32_t* labels,
                            const float* row_weight, float* loss, float* row_loss, float* row_lse, ht_tensor* dH, ht_tensor* dW) {
  if (!ctx) return HT_EINVAL;
  if (!desc || !H || !W || (!labels && H->rows > 0) || !loss) return ht_set_err(ctx, HT_EINVAL, "ht_head_loss: null argument");
  if (desc->d <= 0 || desc->n_classes <= 0) return ht_set_err(ctx, HT_ESHAPE, "ht_head_loss: width and number of classes must be positive");
  if (desc->d > HT_HEAD_MAX_WIDTH || desc->n_classes > HT_HEAD_MAX_CLASSES)
    return ht_set_err(ctx, HT_ESHAPE, "ht_head_loss: %d x %d weights, at most %d x %d", desc->d, desc->n_classes, HT_HEAD_MAX_WIDTH, HT_HEAD_MAX_CLASSES);
  if (desc->w_form != HT_W_IN_OUT && desc->w_form != HT_W_OUT_IN) return ht_set_err(ctx, HT_EINVAL, "ht_head_loss: unknown form of W %d", desc->w_form);
  if (desc->reduction != HT_REDUCE_MEAN && desc->reduction != HT_REDUCE_SUM)
    return ht_set_err(ctx, HT_EINVAL, "ht_head_loss: unknown reduction %d", desc->reduction);
  const int64_t wr = desc->w_form == HT_W_IN_OUT ? desc->d : desc->n_classes;
  const int32_t wcols = desc->w_form == HT_W_IN_OUT ? desc->n_classes : desc->d;
  HT_TRY(ht_check_rows(ctx, H, H->rows, desc->d, "ht_head_loss: H"));
  HT_TRY(ht_check_weights(ctx, W, wr, wcols, "ht_head_loss: W"));
  if (dH) {
    HT_TRY(ht_check_rows(ctx, dH, H->rows, desc->d, "ht_head_loss: dH"));
    if (ht_overlap(dH, H) || ht_overlap(dH, W)) return ht_set_err(ctx, HT_EINVAL, "ht_head_loss: dH shares memory with an input");
  }
  if (dW) {
    HT_TRY(ht_check_weights(ctx, dW, wr, wcols, "ht_head_loss: dW"));
    if (ht_overlap(dW, H) || ht_overlap(dW, W) || (dH && ht_overlap(dW, dH)))
      return ht_set_err(ctx, HT_EINVAL, "ht_head_loss: dW shares memory with another tensor");
  }
  HT_HIP(ctx, hipSetDevice(ctx->device));
  return ht_with_room(ctx, [&]() -> int {
    if (H->rows > 0 && H->rows <= HT_HEAD_FEW) return ht_head_few(ctx, desc, H, W, labels, row_weight, loss, row_loss, row_lse, dH, dW);      // (less memory than either of these)
    auto run = [&](size_t bytes) { return head_run(ctx, desc, H, W, labels, row_weight, loss, row_loss, row_lse, dH, dW, bytes); };
    const int rc = run(HEAD_BYTES);
    return rc == HT_ENOMEM ? run(HEAD_LEAN) : rc;      // (nothing has been launched by a call that is refused memory)
  });
}
