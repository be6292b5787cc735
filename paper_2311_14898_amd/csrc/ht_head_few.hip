// ht_head_loss for at most 64 rows, where all there is to do is read W (twice for dH) and write dW: fp32 matrix instructions on W as it lies, no
// copies of it.  The logits are at most a quarter of W's size and are kept between the launches (64 rows, 256 features): logits with each
// block's maximum and sum | log sum exp, losses | gradients, a part of dH per block | dH.
//
// v_mfma_f32_16x16x4 takes 16 rows of either operand, lane l + 16 q value q of row l.  Which of a reduction's (or of an output's) values are value 0, 1, 2, 3 is
// free as long as both operands agree, so that a lane can load four neighbours at once and use them in four instructions.
#include <algorithm>
#include <type_traits>

#include "ht_internal.h"

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4u __attribute__((ext_vector_type(4), aligned(4)));      // anywhere: weights need no alignment

constexpr int CT = 64, PP = CT + 4;          // classes of a tile of gradients, and its pitch
constexpr int JT = 256;                      // features of a block's gradients
constexpr float LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ float exp_less(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * LOG2E); }

// The labelled rows among V <= 64, found by every wave for itself.
struct FewRows {
  uint64_t mask;
  int n;
  __device__ __forceinline__ FewRows(const int32_t* labels, int64_t V, int* idx, int32_t* lab) {
    const int lane = threadIdx.x & 63;
    const int32_t y = lane < V ? labels[lane] : -1;
    mask = __ballot(y >= 0);
    n = __popcll(mask);
    if (threadIdx.x < 64) {
      idx[lane] = 0, lab[lane] = -1;
      __builtin_amdgcn_wave_barrier();
      if (y >= 0) {
        const int at = __popcll(mask & ((1ull << lane) - 1));
        idx[at] = lane, lab[at] = y;
      }
    }
    __syncthreads();
  }
};

// W's values at p[0 .. 3], of which `left` are there; the others are 0.
__device__ __forceinline__ v4f load4(const float* p, int left) {
  if (left >= 4) return *reinterpret_cast<const v4u*>(p);
  v4f x = {0.f, 0.f, 0.f, 0.f};
  if (left > 0) x[0] = p[0];
  if (left > 1) x[1] = p[1];
  if (left > 2) x[2] = p[2];
  return x;
}
__device__ __forceinline__ void store4(float* p, v4f x, int left, int add) {
  if (left >= 4) {
    v4u* to = reinterpret_cast<v4u*>(p);
    if (add) x += *to;
    *to = x;
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < left) p[i] = add ? p[i] + x[i] : x[i];
}

struct FewArgs {
  const float* H;
  int64_t ldh, V;
  int d, C;
  const float* W;
  int64_t ldw;
  const int32_t* labels;
  float* X;                        // [NB * 16][ldx] logits (null: not wanted)
  int64_t ldx;
  float2* part;                    // [row][blocks]
  int blocks;
  float* xlab;                     // [row]
  unsigned* ticket;
};

// CT classes a block (T = 4), NB * 16 rows, a quarter of the features a wave, in steps of 16: lane l + 16 q has features 4 q .. 4 q + 3 of a step, of row l of H, and of W OUT_IN the
// same features of class t * 16 + l for each tile t, else of those features the classes 4 l + t.  U steps are loaded together; H comes out of the caches.
// T = 1: 16 classes a block, of which lane l + 16 q has class l, for few classes (four times as many blocks).
template <int NB, bool OUT_IN, int T>
__global__ void __launch_bounds__(256) k_few_logits(FewArgs a) {
  constexpr int U = 2;
  constexpr bool BY4 = !OUT_IN && T == 4;  // classes by fours of neighbours
  __shared__ float sums[3][NB][T * 4][64];    // of the waves that do not own the 16 rows
  __shared__ int idx[64];
  __shared__ int32_t lab[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
  const FewRows rows(a.labels, a.V, idx, lab);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
  const int64_t c0 = (int64_t)blockIdx.x * (T * 16);
  v4f acc[T][NB];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[t][b] = v4f{0.f, 0.f, 0.f, 0.f};
  // of a step, OUT_IN: of T classes four features; else of four features four classes, or one
  constexpr int L = OUT_IN ? T : 4;
  const float *Wp[L], *Hp[NB];
  int wleft = 4;                           // (!OUT_IN: classes of the lane that there are)
#pragma unroll
  for (int t = 0; t < L; ++t) {
    const int64_t c = c0 + (OUT_IN ? t * 16 : 0) + l;
    Wp[t] = OUT_IN ? a.W + (c < a.C ? c : a.C - 1) * a.ldw + 4 * q : a.W + (int64_t)(4 * q + t) * a.ldw + (BY4 ? c0 + 4 * l : c < a.C ? c : a.C - 1);
  }
  if (BY4) wleft = a.C - c0 - 4 * l >= 4 ? 4 : (int)(a.C - c0 - 4 * l);
#pragma unroll
  for (int b = 0; b < NB; ++b) Hp[b] = a.H + idx[b * 16 + l] * a.ldh + 4 * q;      // (rows that are not there: the first, whose products nobody looks at)
  const int S = (a.d + 15) / 16, s0 = S * wave / 4, s1 = S * (wave + 1) / 4, whole = a.d / 16;
  auto multiply = [&](const v4f (&w)[L], const v4f (&h)[NB]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(OUT_IN ? w[t][i] : w[i][t], h[b][i], acc[t][b], 0, 0, 0);
  };
  int s = s0;
  const int end = !BY4 || c0 + CT <= a.C ? (s1 < whole ? s1 : whole) : s0;       // (steps without an edge)
  for (; s + U <= end; s += U) {
    v4f w[U][L], h[U][NB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int t = 0; t < L; ++t) {
        const float* at = OUT_IN ? Wp[t] + (s + u) * 16 : Wp[t] + (int64_t)(s + u) * 16 * a.ldw;
        if (OUT_IN || BY4) w[u][t] = *reinterpret_cast<const v4u*>(at);
        else w[u][t] = v4f{*at, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) h[u][b] = *reinterpret_cast<const v4f*>(Hp[b] + (s + u) * 16);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(w[u], h[u]);
  }
  for (; s < s1; ++s) {
    const int left = a.d - s * 16 - 4 * q;           // the lane's features that there are
    v4f w[L], h[NB];
#pragma unroll
    for (int t = 0; t < L; ++t) w[t] = OUT_IN ? load4(Wp[t] + s * 16, left) : load4(Wp[t] + (int64_t)s * 16 * a.ldw, t < left ? (BY4 ? wleft : 1) : 0);
#pragma unroll
    for (int b = 0; b < NB; ++b) h[b] = load4(Hp[b] + s * 16, left);
    multiply(w, h);
  }
  // 16 rows b belong to wave b
#pragma unroll
  for (int b = 0; b < NB; ++b)
    if (b != wave) {
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[(wave - b + 3) & 3][b][t * 4 + r][lane] = acc[t][b][r];
    }
  __syncthreads();
  // a lane has row b * 16 + l and of each tile the classes number 4 q + r
  auto cls = [&](int t, int r) { return BY4 ? c0 + 4 * (4 * q + r) + t : c0 + t * 16 + 4 * q + r; };
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    if (b != wave) continue;
    const int v = b * 16 + l;
    float m = -INFINITY;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = acc[t][b][r];
#pragma unroll
        for (int k = 0; k < 3; ++k) x += sums[k][b][t * 4 + r][lane];
        if (cls(t, r) >= a.C) x = -INFINITY;
        acc[t][b][r] = x;
        m = fmaxf(m, x);
      }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float m1 = m == -INFINITY ? 0.f : m;
    float z = 0.f;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) z += exp_less(acc[t][b][r], m1);
    z += __shfl_xor(z, 16, 64);
    z += __shfl_xor(z, 32, 64);
    if (v >= rows.n) continue;
    if (q == 0) a.part[(int64_t)v * a.blocks + blockIdx.x] = make_float2(m, z);
    const int32_t y = lab[v];
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (cls(t, r) == y) a.xlab[v] = acc[t][b][r];
    if (a.X) {
#pragma unroll
      for (int k = 0; k < T; ++k) {
        v4f x = acc[k][b];
        if constexpr (BY4) x = v4f{acc[0][b][k], acc[1][b][k], acc[2][b][k], acc[3][b][k]};
        *reinterpret_cast<v4f*>(a.X + v * a.ldx + (BY4 ? c0 + 16 * q + 4 * k : c0 + k * 16 + 4 * q)) = x;
      }
    }
  }
}

// A block a row; the last of them to come to an end adds up the losses.  norm (largest logit m, 1 / sum of exp(x - m)), l_of: of the labelled rows in order.
__global__ void __launch_bounds__(256) k_few_join(FewArgs a, const float* __restrict__ weight, int mean, float2* __restrict__ norm, double* __restrict__ l_of,
                                                  float* __restrict__ row_loss, float* __restrict__ row_lse, float* __restrict__ loss) {
  __shared__ int idx[64];
  __shared__ int32_t lab[64];
  __shared__ float2 sh[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = blockIdx.x;
  const FewRows rows(a.labels, a.V, idx, lab);
  if (!((rows.mask >> at) & 1)) {
    if (threadIdx.x == 0) {
      if (row_loss) row_loss[at] = 0.f;
      if (row_lse) row_lse[at] = 0.f;
    }
  } else {
    const int v = __popcll(rows.mask & ((1ull << at) - 1));
    float m = -INFINITY, z = 0.f;
#pragma unroll 8
    for (int t = threadIdx.x; t < a.blocks; t += 256) {
      const float2 p = a.part[(int64_t)v * a.blocks + t];
      const float n = fmaxf(m, p.x);
      z = (m == -INFINITY ? z : z * exp_less(m, n)) + (p.x == -INFINITY ? p.y : p.y * exp_less(p.x, n));
      m = n;
    }
    float all = m;
    for (int o = 32; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor(all, o, 64));
    z = m == -INFINITY ? z : z * exp_less(m, all);
    for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
    if (lane == 0) sh[wave] = make_float2(all, z);
    __syncthreads();
    if (threadIdx.x == 0) {
      m = fmaxf(fmaxf(sh[0].x, sh[1].x), fmaxf(sh[2].x, sh[3].x));
      z = 0.f;
      for (int w = 0; w < 4; ++w) z += sh[w].x == -INFINITY ? sh[w].y : sh[w].y * exp_less(sh[w].x, m);
      const float lse = m + logf(z), l = lab[v] < a.C ? lse - a.xlab[v] : NAN;
      norm[v] = make_float2(m, 1.f / z);
      __hip_atomic_store(l_of + v, weight ? (double)weight[at] * (double)l : (double)l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (row_loss) row_loss[at] = l;
      if (row_lse) row_lse[at] = lse;
    }
  }
  if (wave != 0) return;
  unsigned ended = 0;
  if (lane == 0) ended = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
  if (__builtin_amdgcn_readfirstlane((int)ended) != (int)gridDim.x - 1) return;
  double s = lane < rows.n ? __hip_atomic_load(l_of + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) *loss = rows.n > 0 ? (float)(s / (mean ? (double)rows.n : 1.0)) : 0.f;
}

struct FewGrad {
  const float* weight;
  const float2* norm;
  int mean, add;
  float* dW;                       // (null: not wanted), pitch ldd
  int64_t ldd;
  float* part;                     // [block][NB * 16][d] of dH (null: not wanted)
  int tiles;                       // of CT classes
  int split;                       // blocks that a tile's work is divided among: 1, 2 (dW and dH) or 8 (four each)
};

// Classes in tiles of CT, a contiguous part of them a block; JT features, 64 a wave.
template <int NB, bool OUT_IN, bool CUT>
__global__ void __launch_bounds__(256) k_few_grad(FewArgs a, FewGrad g) {
  __shared__ float Ps[NB * 16][PP];
  __shared__ int idx[64];
  __shared__ int32_t lab[64];
  __shared__ float2 norm[64];
  __shared__ float scale[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
  // CUT: the block's part: quarters w0 .. w1 - 1 of dW's features (OUT_IN: classes), h0 .. h1 - 1 of dH's classes
  const int z = blockIdx.z, each = g.split == 8 ? 1 : 4, parts_h = CUT ? 4 / each : 1;
  const bool for_w = g.dW && (!CUT || z < parts_h), for_h = g.part && (!CUT || z >= parts_h);
  const int w0 = CUT ? z * each : 0, w1 = CUT ? w0 + each : 4, h0 = CUT ? (z - parts_h) * each : 0, h1 = CUT ? h0 + each : 4;
  if (CUT && !for_w && !for_h) return;
  const FewRows rows(a.labels, a.V, idx, lab);
  if (threadIdx.x < 64) {
    const int v = threadIdx.x;
    const bool there = v < rows.n;
    norm[v] = there ? g.norm[v] : make_float2(0.f, 0.f);
    scale[v] = there ? (g.weight ? g.weight[idx[v]] : 1.f) * (g.mean ? 1.f / (float)rows.n : 1.f) : 0.f;
  }
  const int j0 = blockIdx.y * JT + wave * 64, jl = j0 + 4 * l, jleft = a.d - jl;      // the lane's four features, and how many of them there are
  v4f h[NB * 4];                   // row 4 s + q
#pragma unroll
  for (int s = 0; s < NB * 4; ++s) {
    const int v = s * 4 + q;
    h[s] = for_w && v < rows.n ? load4(a.H + idx[v] * a.ldh + jl, jleft) : v4f{0.f, 0.f, 0.f, 0.f};
  }
  v4f sum[4][NB];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) sum[t][b] = v4f{0.f, 0.f, 0.f, 0.f};
  const int t0 = (int)((int64_t)g.tiles * blockIdx.x / gridDim.x), t1 = (int)((int64_t)g.tiles * (blockIdx.x + 1) / gridDim.x);
  // of the next tile: W for dH, OUT_IN four rows of a step of 16 classes, else four columns of a step, of each of four tiles of 16 features; and the logits
  v4f w[4][4], x[NB];
  auto fetch_w = [&](int tile) {
    const int64_t c0 = (int64_t)tile * CT;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (s < h0 || s >= h1) continue;
        if (OUT_IN) {
          const int64_t c = c0 + s * 16 + 4 * q + k;
          w[s][k] = c < a.C ? load4(a.W + c * a.ldw + jl, jleft) : v4f{0.f, 0.f, 0.f, 0.f};
        } else {
          const int j = j0 + k * 16 + l;
          const int64_t c = c0 + s * 16 + 4 * q, left = a.C - c;
          w[s][k] = j < a.d ? load4(a.W + (int64_t)j * a.ldw + c, left >= 4 ? 4 : (int)left) : v4f{0.f, 0.f, 0.f, 0.f};
        }
      }
  };
  auto fetch_x = [&](int tile) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int v = b * 16 + threadIdx.x / 16;
      x[b] = v < rows.n ? *reinterpret_cast<const v4f*>(a.X + v * a.ldx + (int64_t)tile * CT + threadIdx.x % 16 * 4) : v4f{0.f, 0.f, 0.f, 0.f};
    }
  };
  if (t0 < t1) {
    fetch_x(t0);
    if (for_h) fetch_w(t0);
  }
  __syncthreads();                         // (norm, scale)
  for (int tile = t0; tile < t1; ++tile) {
    const int64_t c0 = (int64_t)tile * CT;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int v = b * 16 + threadIdx.x / 16, c = threadIdx.x % 16 * 4;
      v4f p = {0.f, 0.f, 0.f, 0.f};
      if (v < rows.n) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c0 + c + k < a.C) p[k] = (exp_less(x[b][k], norm[v].x) * norm[v].y - (c0 + c + k == lab[v] ? 1.f : 0.f)) * scale[v];
      }
      *reinterpret_cast<v4f*>(&Ps[v][c]) = p;
    }
    __syncthreads();
    if (tile + 1 < t1) fetch_x(tile + 1);
    if (for_w) {
      if (OUT_IN) {
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
          if (ct < w0 || ct >= w1) continue;
          v4f o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < NB * 4; ++s) {
            const float p = Ps[s * 4 + q][ct * 16 + l];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(p, h[s][i], o[i], 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int64_t c = c0 + ct * 16 + 4 * q + r;
            if (c < a.C && jleft > 0) store4(g.dW + c * g.ldd + jl, v4f{o[0][r], o[1][r], o[2][r], o[3][r]}, jleft, g.add);
          }
        }
      } else {
        const int64_t cl = a.C - c0 - 4 * l;
        const int cleft = cl >= 4 ? 4 : (int)cl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {          // features 4 m + i
          if (i < w0 || i >= w1) continue;
          v4f o[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) o[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < NB * 4; ++s) {
            const v4f p = *reinterpret_cast<const v4f*>(&Ps[s * 4 + q][4 * l]);
#pragma unroll
            for (int t = 0; t < 4; ++t) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[s][i], p[t], o[t], 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = j0 + 4 * (4 * q + r) + i;
            if (j < a.d && cleft > 0) store4(g.dW + (int64_t)j * g.ldd + c0 + 4 * l, v4f{o[0][r], o[1][r], o[2][r], o[3][r]}, cleft, g.add);
          }
        }
      }
    }
    if (for_h) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (s < h0 || s >= h1) continue;
          const v4f p = *reinterpret_cast<const v4f*>(&Ps[b * 16 + l][s * 16 + 4 * q]);
#pragma unroll
          for (int k = 0; k < 4; ++k)          // value k of the lane's four classes
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[k], OUT_IN ? w[s][k][t] : w[s][t][k], sum[t][b], 0, 0, 0);
        }
      if (tile + 1 < t1) fetch_w(tile + 1);
    }
    __syncthreads();
  }
  if (!for_h) return;
  // a lane has the rows b * 16 + 4 q + r and a feature of each tile: OUT_IN 4 l + t, else t * 16 + l
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = b * 16 + 4 * q + r;
      if (v >= rows.n) continue;
      float* o = g.part + (((int64_t)blockIdx.x * parts_h + (CUT ? h0 / each : 0)) * (NB * 16) + v) * a.d;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int j = OUT_IN ? jl + t : j0 + t * 16 + l;
        if (j < a.d) o[j] = sum[t][b][r];
      }
    }
}

// dH: rows of 64 features a block, 16 parts of the blocks' sums each
__global__ void __launch_bounds__(1024) k_few_dh(FewArgs a, const float* __restrict__ part, int blocks, int rows16, float* __restrict__ dH, int64_t ld) {
  __shared__ int idx[64];
  __shared__ int32_t lab[64];
  __shared__ float sh[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const FewRows rows(a.labels, a.V, idx, lab);
  const int v = blockIdx.x, j = blockIdx.y * 64 + lane;
  if (!((rows.mask >> v) & 1)) {
    if (wave == 0 && j < a.d) dH[v * ld + j] = 0.f;
    return;
  }
  const int at = __popcll(rows.mask & ((1ull << v) - 1));
  float s = 0.f;
  if (j < a.d)
#pragma unroll 8
    for (int k = blocks * wave / 16; k < blocks * (wave + 1) / 16; ++k) s += part[((int64_t)k * rows16 + at) * a.d + j];
  sh[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && j < a.d) {
    for (int w = 1; w < 16; ++w) s += sh[w][lane];
    dH[v * ld + j] = s;
  }
}

}  // namespace

// Few tiles leave most CUs without a block, and those that have one with a long chain of instructions (64 rows: 512 of 32 clocks a tile for dW and dH).  Up to FEW_TILES tiles the
// logits go by 16 classes a block, and up to SPLIT2 blocks of gradients each is divided, dW from dH, up to SPLIT8 those by quarters.  us of a call, so | not: 64 rows x 64
// features x 500 classes 23 | 34, 40 x 1,000 x 700 37 | 57 (the loss alone 18 | 34), 20 x 180 x 3,600 24 | 28, 64 x 200 x 8,000 37 | 44 (loss 13 | 15); 16 classes a block of 2,048 tiles
// 240 | 213, eighths of 64 blocks 46 | 37 (40 x 1,000 x 700).
constexpr int FEW_TILES = 256, SPLIT8 = 32, SPLIT2 = 128;

int ht_head_few(ht_ctx* ctx, const ht_head_desc* D, const ht_tensor* H, const ht_tensor* W, const int32_t* labels, const float* weight, float* loss, float* row_loss,
                float* row_lse, const ht_tensor* dH, const ht_tensor* dW) {
  const bool out_in = D->w_form == HT_W_OUT_IN, grad = dH || dW;
  const int mean = D->reduction == HT_REDUCE_MEAN, d = D->d, C = D->n_classes;
  const int NB = H->rows <= 16 ? 1 : H->rows <= 32 ? 2 : 4;
  const int tiles = (int)ceil_div64(C, CT);
  const bool narrow = tiles <= FEW_TILES;
  const int blocks = narrow ? (int)ceil_div64(C, 16) : tiles;
  const int64_t ldx = (int64_t)tiles * CT;
  const int gy = (int)ceil_div64(d, JT), gx = (int)std::min<int64_t>(tiles, std::max(64, 512 / gy));
  const int split = (int64_t)gx * gy <= SPLIT8 ? 8 : (int64_t)gx * gy <= SPLIT2 ? 2 : 1, dh_parts = gx * (split == 8 ? 4 : 1);
  hipStream_t st = ctx->stream;
  OpsBlock m;
  const auto X = m.add<float>(grad ? NB * 16 * ldx : 0);
  const auto part = m.add<float2>((int64_t)64 * blocks);
  const auto xlab = m.add<float>(64);
  const auto lrow = m.add<double>(64);
  const auto norm = m.add<float2>(64);
  const auto ticket = m.add<unsigned>(1);
  const auto ph = m.add<float>(dH ? (int64_t)dh_parts * NB * 16 * d : 0);
  HT_TRY(m.take(ctx));
  const FewArgs a{H->ptr, H->ld, H->rows, d, C, W->ptr, W->ld, labels, grad ? m.at(X) : nullptr, ldx, m.at(part), blocks, m.at(xlab), m.at(ticket)};
  const FewGrad g{weight, m.at(norm), mean, D->accumulate_dW, dW ? dW->ptr : nullptr, dW ? dW->ld : 0, dH ? m.at(ph) : nullptr, tiles, split};
  auto run = [&](auto nb, auto form) -> int {
    constexpr int N = decltype(nb)::value;
    constexpr bool F = decltype(form)::value;
    if (narrow) k_few_logits<N, F, 1><<<(unsigned)blocks, 256, 0, st>>>(a);
    else k_few_logits<N, F, 4><<<(unsigned)blocks, 256, 0, st>>>(a);
    HT_LAUNCH_CHECK(ctx);
    k_few_join<<<(unsigned)H->rows, 256, 0, st>>>(a, weight, mean, m.at(norm), m.at(lrow), row_loss, row_lse, loss);
    HT_LAUNCH_CHECK(ctx);
    if (!grad) return HT_OK;
    if (split > 1) k_few_grad<N, F, true><<<dim3((unsigned)gx, (unsigned)gy, (unsigned)split), 256, 0, st>>>(a, g);
    else k_few_grad<N, F, false><<<dim3((unsigned)gx, (unsigned)gy), 256, 0, st>>>(a, g);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  };
  auto with_form = [&](auto nb) { return out_in ? run(nb, std::true_type()) : run(nb, std::false_type()); };
  HT_TRY(NB == 1 ? with_form(std::integral_constant<int, 1>()) : NB == 2 ? with_form(std::integral_constant<int, 2>()) : with_form(std::integral_constant<int, 4>()));
  if (dH) {
    k_few_dh<<<dim3((unsigned)H->rows, (unsigned)ceil_div64(d, 64)), 1024, 0, st>>>(a, m.at(ph), dh_parts, NB * 16, dH->ptr, dH->ld);
    HT_LAUNCH_CHECK(ctx);
  }
  return HT_OK;
}
