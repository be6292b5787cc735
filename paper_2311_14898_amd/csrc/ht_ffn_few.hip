// Gated feed-forward blocks of at most 64 rows (16 of very wide weights), where all there is to do is read the weights (and write their gradients): fp32 matrix instructions on the weights as they lie,
// no copies of them.
//   k_few_hidden  16 hidden columns a block: A and B (and G) over all of the reduction, an eighth a wave; H, or H, dA and dB; and of the gradients of the weights all that these
//                 columns have, which is whole: their reduction is over the rows
//   k_few_out     16 columns of Y or dX by a part of the hidden columns a block; the parts are added up behind it
//
// v_mfma_f32_16x16x4 takes 16 rows of either operand, lane l + 16 q value q of row l; of the result lane l + 16 q has column l (a row of the second operand) and the rows 4 q .. 4 q + 3.
// Which of a reduction's values are value 0, 1, 2, 3 is free as long as both operands agree, so that a lane can load four neighbours at once and use them in four
// instructions.
#include <algorithm>

#include "ht_ffn.h"

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4u __attribute__((ext_vector_type(4), aligned(4)));      // anywhere: weights need no alignment

constexpr int WAVES = 8, OUTS = 16;    // waves of a block, its columns

// Blocks of neighbouring columns run on one XCD: they share cache lines where a weight's rows lie across the columns.
__device__ __forceinline__ int64_t few_tile(int64_t tiles) {
  const int64_t per = (tiles + 7) / 8, t = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  return (int64_t)(blockIdx.x >> 3) < per && t < tiles ? t : -1;
}

// p[0 .. 3], of which `left` are there; the others are 0.
__device__ __forceinline__ v4f load4(const float* p, int64_t left) {
  if (left >= 4) return *reinterpret_cast<const v4u*>(p);
  v4f x = {0.f, 0.f, 0.f, 0.f};
  if (left > 0) x[0] = p[0];
  if (left > 1) x[1] = p[1];
  if (left > 2) x[2] = p[2];
  return x;
}

// acc[m][b] += the products of 16 columns of M weights with rows of x, over the steps s0 .. s1 - 1 of 16 of the reduction (K values).  w[m]: the lane's column; BYK: its reduction lies
// in a row, else k_ld floats apart.  x[b]: row l of the b-th 16.
template <int NB, int M, bool BYK>
__device__ __forceinline__ void few_products(v4f (&acc)[M][NB], const float* const (&w)[M], const int64_t (&k_ld)[M], const float* const (&x)[NB], int64_t K, int s0, int s1) {
  constexpr int U = NB * M <= 4 ? 4 : 2;       // steps loaded together
  const int q = (threadIdx.x & 63) >> 4;
  auto multiply = [&](const v4f (&a)[M], const v4f (&b)[NB]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int c = 0; c < NB; ++c) acc[m][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[m][i], b[c][i], acc[m][c], 0, 0, 0);
  };
  const int whole = (int)(K / 16), end = s1 < whole ? s1 : whole;
  int s = s0;
  for (; s + U <= end; s += U) {
    v4f a[U][M], b[U][NB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = (int64_t)(s + u) * 16 + 4 * q;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        if (BYK) {
          a[u][m] = *reinterpret_cast<const v4u*>(w[m] + k);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) a[u][m][i] = w[m][(k + i) * k_ld[m]];
        }
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) b[u][c] = *reinterpret_cast<const v4f*>(x[c] + k);
    }
    // (all loads before the first product: 24 x 1,024 x 4,096 forward 32 -> 23 us, 1 x 4,096 x 16,384 205 -> 197, backward 682 -> 628; of 64 rows backward 82 -> 85)
    if (NB < 4) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(a[u], b[u]);
  }
  for (; s < s1; ++s) {
    const int64_t k = (int64_t)s * 16 + 4 * q, left = K - k;
    v4f a[M], b[NB];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      if (BYK) {
        a[m] = load4(w[m] + k, left);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[m][i] = i < left ? w[m][(k + i) * k_ld[m]] : 0.f;
      }
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) b[c] = load4(x[c] + k, left);
    multiply(a, b);
  }
}

struct FewArgs {
  int64_t n, d, f, e;
  int act;
  const float *X, *Wg, *Wu, *Wd, *dY;
  int64_t ldx, ldg, ldu, ldd, ldy;
  float *gate, *up;                    // forward: where A and B go (null: nowhere); backward: where they are (null: they are made)
  int64_t ld_gate, ld_up;
  float *H, *A, *B;                    // H; backward: dA and dB (null: not wanted)
  int64_t pitch;
  float *dWg, *dWu, *dWd;              // (null: not wanted)
  int64_t ld_dWg, ld_dWu, ld_dWd;
  int add;
};

// The gradient of a weight: of its 16 columns l from c0 on (of f), for features of P [n x width] by 16s; t: [NB * 16][16] in LDS, 0 behind the last row and column.  A feature's value
// lies at feature ms + column ns.
template <int NB, int M>
__device__ __forceinline__ void few_gradient(const float* P, int64_t ldp, int64_t n, int64_t width, const float* const (&t)[M], float* const (&out)[M], const int64_t (&ms)[M],
                                             const int64_t (&ns)[M], int64_t c, int64_t f, int add) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
  float b[M][NB * 4];
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int s = 0; s < NB * 4; ++s) b[m][s] = t[m][(s * 4 + q) * OUTS + l];
  for (int64_t i0 = wave * 16; i0 < width; i0 += WAVES * 16) {
    const int64_t i = i0 + l < width ? i0 + l : width - 1;
    float a[NB * 4];
#pragma unroll
    for (int s = 0; s < NB * 4; ++s) a[s] = s * 4 + q < n ? P[(s * 4 + q) * ldp + i] : 0.f;
    v4f acc[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      acc[m] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NB * 4; ++s) acc[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[m][s], acc[m], 0, 0, 0);
    }
    if (c >= f) continue;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      if (!out[m]) continue;
      const int64_t j = i0 + 4 * q, left = width - j;
      float* to = out[m] + j * ms[m] + c * ns[m];
      if (ms[m] == 1 && left >= 4) {
        v4f x = acc[m];
        if (add) x += *reinterpret_cast<const v4u*>(to);
        *reinterpret_cast<v4u*>(to) = x;
        continue;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) to[k * ms[m]] = add ? to[k * ms[m]] + acc[m][k] : acc[m][k];
    }
  }
}

template <int NB, bool IN_OUT, bool BWD>
__global__ void __launch_bounds__(WAVES * 64) k_few_hidden(FewArgs a) {
  constexpr int SUMS = BWD ? 3 : 2, N = NB * 256;             // values of each sum
  __shared__ __attribute__((aligned(16))) float sh[WAVES][SUMS][N];
  const int64_t tile = few_tile((a.f + OUTS - 1) / OUTS);
  if (tile < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane & 15;
  const int64_t c0 = tile * OUTS, c = c0 + l < a.f ? c0 + l : a.f - 1;
  const bool make = !BWD || !a.gate;
  auto part = [&](int64_t K, int w) { return (int)((K + 15) / 16 * w / WAVES); };
  {
    v4f ab[2][NB] = {};
    const float* x[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) x[b] = a.X + (b * 16 + l < a.n ? b * 16 + l : a.n - 1) * a.ldx;      // (rows that are not there: the last, whose products nobody looks at)
    const float* const w[2] = {IN_OUT ? a.Wg + c : a.Wg + c * a.ldg, IN_OUT ? a.Wu + c : a.Wu + c * a.ldu};
    const int64_t k_ld[2] = {a.ldg, a.ldu};
    if (make) few_products<NB, 2, !IN_OUT>(ab, w, k_ld, x, a.d, part(a.d, wave), part(a.d, wave + 1));
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int b = 0; b < NB; ++b) *reinterpret_cast<v4f*>(&sh[wave][m][b * 256 + lane * 4]) = ab[m][b];
  }
  if constexpr (BWD) {
    v4f g[1][NB] = {};
    const float* y[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) y[b] = a.dY + (b * 16 + l < a.n ? b * 16 + l : a.n - 1) * a.ldy;
    const float* const w[1] = {IN_OUT ? a.Wd + c * a.ldd : a.Wd + c};
    const int64_t k_ld[1] = {a.ldd};
    few_products<NB, 1, IN_OUT>(g, w, k_ld, y, a.e, part(a.e, wave), part(a.e, wave + 1));
#pragma unroll
    for (int b = 0; b < NB; ++b) *reinterpret_cast<v4f*>(&sh[wave][2][b * 256 + lane * 4]) = g[0][b];
  }
  __syncthreads();
  // the waves' sums, and what is made of them: value 256 b + 64 q + 4 l + i is that of row 16 b + l and column 4 q + i
  constexpr int U = (N + WAVES * 64 - 1) / (WAVES * 64);
  float h[U], da[U], db[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = u * WAVES * 64 + tid;
    h[u] = da[u] = db[u] = 0.f;
    if (k >= N) continue;
    const int64_t v = (k >> 8) * 16 + ((k >> 2) & 15), cc = c0 + ((k >> 6) & 3) * 4 + (k & 3);
    if (v >= a.n || cc >= a.f) continue;
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < SUMS; ++m)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s[m] += sh[w][m][k];
    if (!make) s[0] = a.gate[v * a.ld_gate + cc], s[1] = a.up[v * a.ld_up + cc];
    const Act x = any_act(a.act, s[0]);
    h[u] = x.v * s[1];
    if constexpr (!BWD) {
      if (a.gate) a.gate[v * a.ld_gate + cc] = s[0], a.up[v * a.ld_up + cc] = s[1];
      a.H[v * a.pitch + cc] = h[u];
    } else {
      da[u] = s[2] * s[1] * x.s, db[u] = s[2] * x.v;
      if (a.A) a.A[v * a.pitch + cc] = da[u], a.B[v * a.pitch + cc] = db[u];
    }
  }
  if constexpr (BWD) {
    if (!a.dWg && !a.dWu && !a.dWd) return;
    __syncthreads();
    float* t = &sh[0][0][0];                                  // [H, dA, dB][row][column]
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = u * WAVES * 64 + tid;
      if (k >= N) continue;
      const int at = ((k >> 8) * 16 + ((k >> 2) & 15)) * OUTS + ((k >> 6) & 3) * 4 + (k & 3);
      t[at] = h[u], t[N + at] = da[u], t[2 * N + at] = db[u];
    }
    __syncthreads();
    if (a.dWg || a.dWu) {
      const float* const ts[2] = {t + N, t + 2 * N};
      float* const out[2] = {a.dWg, a.dWu};
      const int64_t ms[2] = {IN_OUT ? a.ld_dWg : 1, IN_OUT ? a.ld_dWu : 1}, ns[2] = {IN_OUT ? 1 : a.ld_dWg, IN_OUT ? 1 : a.ld_dWu};
      few_gradient<NB, 2>(a.X, a.ldx, a.n, a.d, ts, out, ms, ns, c0 + l, a.f, a.add);
    }
    if (a.dWd) {
      const float* const ts[1] = {t};
      float* const out[1] = {a.dWd};
      const int64_t ms[1] = {IN_OUT ? 1 : a.ld_dWd}, ns[1] = {IN_OUT ? a.ld_dWd : 1};
      few_gradient<NB, 1>(a.dY, a.ldy, a.n, a.e, ts, out, ms, ns, c0 + l, a.f, a.add);
    }
  }
}

struct FewOut {
  int64_t n, f, width;                 // rows, reduction, columns
  const float *P[2], *W[2];            // H and Wd; or dA and Wg, dB and Wu
  int64_t pitch, ldw[2];
  int splits;
  float* out;
  int64_t ld, part;                    // of the sums of a part
  int add;
};
// M: how many products.  BYK: a weight's reduction lies in its rows.
template <int NB, int M, bool BYK>
__global__ void __launch_bounds__(WAVES * 64) k_few_out(FewOut a) {
  constexpr int N = NB * 256;
  __shared__ __attribute__((aligned(16))) float sh[WAVES][N];
  const int64_t tiles = (a.width + OUTS - 1) / OUTS, t = few_tile(tiles * a.splits);
  if (t < 0) return;
  const int64_t split = t / tiles, c0 = (t - split * tiles) * OUTS;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane & 15;
  const int64_t c = c0 + l < a.width ? c0 + l : a.width - 1, S = (a.f + 15) / 16, p = split * WAVES + wave;
  const int s0 = (int)(S * p / (a.splits * WAVES)), s1 = (int)(S * (p + 1) / (a.splits * WAVES));
  v4f acc[1][NB] = {};
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const float* x[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) x[b] = a.P[m] + (b * 16 + l < a.n ? b * 16 + l : a.n - 1) * a.pitch;
    const float* const w[1] = {BYK ? a.W[m] + c * a.ldw[m] : a.W[m] + c};
    const int64_t k_ld[1] = {a.ldw[m]};
    few_products<NB, 1, BYK>(acc, w, k_ld, x, a.f, s0, s1);
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) *reinterpret_cast<v4f*>(&sh[wave][b * 256 + lane * 4]) = acc[0][b];
  __syncthreads();
  for (int k = tid; k < N; k += WAVES * 64) {
    const int64_t v = (k >> 8) * 16 + ((k >> 2) & 15), cc = c0 + ((k >> 6) & 3) * 4 + (k & 3);
    if (v >= a.n || cc >= a.width) continue;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += sh[w][k];
    float* to = a.out + split * a.part + v * a.ld + cc;
    *to = a.add ? *to + s : s;
  }
}

constexpr int64_t FEW_BLOCKS = 512;    // of Y or dX, about: two a CU

int splits_of(int64_t width, int64_t f) { return (int)std::max<int64_t>(1, std::min(FEW_BLOCKS / ceil_div64(width, OUTS), f / (WAVES * 16 * 2))); }

template <int NB>
int few(const FfnCall& c) {
  ht_ctx* ctx = c.ctx;
  hipStream_t st = ctx->stream;
  const bool in_out = c.in_out(), bwd = c.dY != nullptr;
  const int64_t n = c.X->rows, d = c.D->d_in, f = c.D->d_hidden, e = c.D->d_out, pitch = (f + 3) / 4 * 4;
  const ht_tensor* to = bwd ? c.dX : c.Y;
  const int64_t width = bwd ? d : e, wp = (width + 3) / 4 * 4;
  const int splits = splits_of(width, f);
  OpsBlock m;
  const auto h = m.add<float>(bwd ? 0 : n * pitch), da = m.add<float>(c.dX ? n * pitch : 0), db = m.add<float>(c.dX ? n * pitch : 0);
  const auto sums = m.add<float>(to && splits > 1 ? splits * n * wp : 0);
  HT_TRY(m.take(ctx));
  FewArgs a{};
  a.n = n, a.d = d, a.f = f, a.e = e, a.act = c.D->act;
  a.X = c.X->ptr, a.ldx = c.X->ld, a.Wg = c.Wg->ptr, a.ldg = c.Wg->ld, a.Wu = c.Wu->ptr, a.ldu = c.Wu->ld, a.Wd = c.Wd->ptr, a.ldd = c.Wd->ld;
  if (bwd) a.dY = c.dY->ptr, a.ldy = c.dY->ld;
  if (c.gate) a.gate = c.gate->ptr, a.ld_gate = c.gate->ld, a.up = c.up->ptr, a.ld_up = c.up->ld;
  a.pitch = pitch;
  if (!bwd) a.H = m.at(h);
  if (c.dX) a.A = m.at(da), a.B = m.at(db);
  if (c.dWg) a.dWg = c.dWg->ptr, a.ld_dWg = c.dWg->ld;
  if (c.dWu) a.dWu = c.dWu->ptr, a.ld_dWu = c.dWu->ld;
  if (c.dWd) a.dWd = c.dWd->ptr, a.ld_dWd = c.dWd->ld;
  a.add = c.D->accumulate_dW;
  const unsigned grid = (unsigned)((ceil_div64(f, OUTS) + 7) / 8 * 8);
  if (bwd) (in_out ? k_few_hidden<NB, true, true> : k_few_hidden<NB, false, true>)<<<grid, WAVES * 64, 0, st>>>(a);
  else (in_out ? k_few_hidden<NB, true, false> : k_few_hidden<NB, false, false>)<<<grid, WAVES * 64, 0, st>>>(a);
  HT_LAUNCH_CHECK(ctx);
  if (!to) return HT_OK;
  FewOut o{};
  o.n = n, o.f = f, o.width = width, o.pitch = pitch, o.splits = splits;
  if (bwd) o.P[0] = m.at(da), o.P[1] = m.at(db), o.W[0] = c.Wg->ptr, o.W[1] = c.Wu->ptr, o.ldw[0] = c.Wg->ld, o.ldw[1] = c.Wu->ld;
  else o.P[0] = m.at(h), o.W[0] = c.Wd->ptr, o.ldw[0] = c.Wd->ld;
  o.out = splits > 1 ? m.at(sums) : to->ptr, o.ld = splits > 1 ? wp : to->ld, o.part = n * wp, o.add = splits == 1 && c.D->accumulate;
  const unsigned blocks = (unsigned)((ceil_div64(width, OUTS) * splits + 7) / 8 * 8);
  if (bwd) (in_out ? k_few_out<NB, 2, true> : k_few_out<NB, 2, false>)<<<blocks, WAVES * 64, 0, st>>>(o);
  else (in_out ? k_few_out<NB, 1, false> : k_few_out<NB, 1, true>)<<<blocks, WAVES * 64, 0, st>>>(o);
  HT_LAUNCH_CHECK(ctx);
  if (splits == 1) return HT_OK;
  FfnJoins j{};
  j.join[j.n++] = FfnJoin{m.at(sums), n * wp, wp, n, width, splits, c.D->accumulate, to->ptr, to->ld};
  return ht_ffn_join(ctx, j);
}

}  // namespace

int ht_ffn_few(const FfnCall& c) {
  switch ((c.X->rows + 15) / 16) {
    case 1: return few<1>(c);
    case 2: return few<2>(c);
    case 3: return few<3>(c);
    default: return few<4>(c);
  }
}
