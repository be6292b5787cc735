// Blocks of more rows than ht_ffn_few.hip has, but not many: most of what there is to read are the weights.  They go as they lie straight from memory into the registers of the block that
// multiplies them (of one for every 64 rows; the others find them in the caches), and are split there; only rows are packed.
//   k_stream_hidden  32 hidden columns and 64 rows a block: A and B (and G) over all of the reduction, a quarter a wave; of their sums H, or H, dA and dB, in the order of
//                    fragments, with their largest values
//   k_stream_out     32 columns of Y or dX and 64 rows, by a part of the hidden columns a block; the parts are added up behind it
// A wave scales the weights by the largest that it has met, and its sums with them where a larger one comes: no pass looks for it before.
#pragma once

// Waves of a block of either; row blocks and rows of a tile.  (k_stream_hidden with eight waves: 1,003 x 512 x 2,048 forward 53 -> 64 us, 256 x 2,048 x 8,192 141 -> 157; with tiles of 128 rows
// 128 x 1,024 x 4,096 51 -> 66, for the rows are read from the caches as often, but by half as many blocks.)
constexpr int HIDDEN_WAVES = 4, OUT_WAVES = 8, NJ = 2, STREAM_TILE = NJ * 32;

// Eight values of a weight's column (lane l32) along the reduction from k0 on, in the order of fragments.  w: the block's first column (the same in all lanes); off: the lane's place
// behind it, floats.  BYK: the reduction lies in a row, else ld floats apart.
template <bool BYK>
__device__ __forceinline__ void raw8(v8h (&x)[2], const float* w, int64_t ld, uint32_t off, int64_t k0) {
  V4 a, b;
  if (BYK) {
    const float* p = w + k0;
    a = *reinterpret_cast<const V4u*>(p + off), b = *reinterpret_cast<const V4u*>(p + 8 + off);
  } else {
    const float* p = w + k0 * ld;
#pragma unroll
    for (int t = 0; t < 4; ++t) a[t] = (p + t * ld)[off], b[t] = (p + (8 + t) * ld)[off];
  }
  x[0] = __builtin_bit_cast(v8h, a), x[1] = __builtin_bit_cast(v8h, b);
}
// The same where the reduction ends `left` values behind k0: zeros there.
template <bool BYK>
__device__ __forceinline__ void raw8_end(v8h (&x)[2], const float* w, int64_t ld, uint32_t off, int64_t k0, int left) {
  const int half = (threadIdx.x & 63) >> 5;
  V4 v[2];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const int k = (t >> 2) * 8 + (t & 3);
    const bool in = half * 4 + k < left;          // (else the column's first value: loads have no condition, so that they go together)
    const float y = w[off - (BYK ? half * 4 : half * 4 * (uint32_t)ld) + (in ? (k0 + half * 4 + k) * (BYK ? 1 : ld) : 0)];
    v[t >> 2][t & 3] = in ? y : 0.f;
  }
  x[0] = __builtin_bit_cast(v8h, v[0]), x[1] = __builtin_bit_cast(v8h, v[1]);
}
template <bool BYK>
__device__ __forceinline__ uint32_t raw_off(int64_t ld, int64_t cols) {      // cols: that there are from the block's first on
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const uint32_t c = (lane & 31) < cols ? lane & 31 : (uint32_t)cols - 1;
  return BYK ? c * (uint32_t)ld + half * 4 : half * 4 * (uint32_t)ld + c;
}
constexpr int64_t STREAM_LD = (int64_t)1 << 25;      // of a weight, at most: places behind a block's first column are 32 bits

// Sums over steps of 16 of the reduction, scaled by the exponent e; what is larger than lim needs another.
struct Scaled {
  v16f acc[NJ];
  int e = 0;
  float lim = 0.f;
  __device__ __forceinline__ Scaled() {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  }
  __device__ __forceinline__ void split(v8h (&x)[2]) {
    const V4 a = __builtin_bit_cast(V4, x[0]), b = __builtin_bit_cast(V4, x[1]);
    float m = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) m = fmaxf(m, fmaxf(fabsf(a[k]), fabsf(b[k])));
    if (__builtin_expect(__ballot(m > lim) != 0, 0)) {
      uint32_t bits = max(max4(a), max4(b));
      for (int o = 32; o > 0; o >>= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, o, 64));
      bits = __builtin_amdgcn_readfirstlane(bits);
      if (__uint_as_float(bits) > lim) {           // (else it was one that is not finite)
        const int next = exp_or_0(scale_exp(bits));
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[j][r] = __builtin_amdgcn_ldexpf(acc[j][r], next - e);
        e = next, lim = pow2(15 - next);
      }
    }
    const float f = pow2(e);
    split8(x[0], x[1], 1.f, [&](int) { return f; });
  }
  __device__ __forceinline__ void add(const v8h (&x)[2], const v8h (&y)[NJ][2]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[1], y[j][0], acc[j], 0, 0, 0);
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0], y[j][1], acc[j], 0, 0, 0);
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0], y[j][0], acc[j], 0, 0, 0);
  }
  __device__ __forceinline__ V4 four(int j, int k, int e_row) const {      // of row j 32 + l32, columns 8 k + 4 half + 0 .. 3
    V4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_ldexpf(acc[j][k * 4 + i], -(e + e_row));
    return x;
  }
};
// Products of the columns of M weights with rows, over the steps s0 .. s1 - 1; a step's operands are fetched two steps ahead: fetch(s, a, b), and what is done to b before it is
// used: in_b(b).  NB = 2: each weight has rows of its own (b[1]).
template <int M, int NB, class Fetch, class InB>
__device__ __forceinline__ void stream(Scaled (&sums)[M], int s0, int s1, Fetch&& fetch, InB&& in_b) {
  if (s0 >= s1) return;
  v8h a[2][M][2], b[2][NB][NJ][2];
  fetch(s0, a[0], b[0]);
  fetch(s0 + 1 < s1 ? s0 + 1 : s0, a[1], b[1]);
  for (int s = s0; s < s1; s += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (s + u < s1) {
        in_b(b[u]);
#pragma unroll
        for (int m = 0; m < M; ++m) {
          sums[m].split(a[u][m]);
          sums[m].add(a[u][m], b[u][NB == 1 ? 0 : m]);
        }
      }
      const int next = s + u + 2 < s1 ? s + u + 2 : s1 - 1;
      __builtin_amdgcn_sched_barrier(0);
      fetch(next, a[u], b[u]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}
// A wave's steps of a reduction of K values, the w-th of W parts: whole ones, and whether the step that the reduction ends in is its own.
struct Steps {
  int s0, s1, left;                    // left: values of step s1 (0: none)
  __device__ __forceinline__ Steps(int64_t K, int w, int W) {
    const int64_t S = (K + 15) / 16;
    s0 = (int)(S * w / W), s1 = (int)(S * (w + 1) / W), left = 0;
    if (s1 > s0 && (int64_t)s1 * 16 > K) --s1, left = (int)(K - (int64_t)s1 * 16);
  }
};
__device__ __forceinline__ void fragments(v8h (&y)[NJ][2], const _Float16* p, int64_t row_block) {      // p: of a step, the lane's place; row_block: halfs
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int q = 0; q < 2; ++q) y[j][q] = *reinterpret_cast<const v8h*>(p + j * row_block + q * FRAG);
}

struct StreamHidden {
  Args a;                              // n, f, H, D, largest values, e_x, e_y, gate, up
  const float* w[3];                   // Wg, Wu, Wd
  int64_t ld[3], d, e;
  const _Float16 *X, *G;               // packed rows of X, dY
  int64_t KSX, KSG;
  const int *ex, *ey;
  int act, make, row_tiles;
};
template <bool IN_OUT, bool BWD>
__global__ void __launch_bounds__(HIDDEN_WAVES * 64, 2) k_stream_hidden(StreamHidden s) {
  constexpr int SUMS = BWD ? 3 : 2;
  __shared__ __attribute__((aligned(16))) float sh[HIDDEN_WAVES][SUMS][1024];
  __shared__ float tops[BWD ? 2 : 1][4][NJ * 32], cols[BWD ? 3 : 1][NJ][32];
  const Args& a = s.a;
  const Tile tile(blockIdx.x, s.row_tiles, (a.f + HB - 1) / HB, 1);
  if (tile.m < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int64_t c0 = tile.n * HB, b0 = tile.m * NJ;
  Scaled ab[2], g[1];
  const auto as_it_is = [](v8h (&)[1][NJ][2]) {};
  if (!BWD || s.make) {
    const float* const w[2] = {IN_OUT ? s.w[0] + c0 : s.w[0] + c0 * s.ld[0], IN_OUT ? s.w[1] + c0 : s.w[1] + c0 * s.ld[1]};
    const uint32_t off[2] = {raw_off<!IN_OUT>(s.ld[0], a.f - c0), raw_off<!IN_OUT>(s.ld[1], a.f - c0)};
    const _Float16* X = s.X + b0 * s.KSX * 2 * FRAG + lane * 8;
    const int64_t rows = s.KSX * 2 * FRAG;
    const Steps at(s.d, wave, HIDDEN_WAVES);
    stream<2, 1>(ab, at.s0, at.s1, [&](int k, v8h (&x)[2][2], v8h (&y)[1][NJ][2]) {
#pragma unroll
      for (int m = 0; m < 2; ++m) raw8<!IN_OUT>(x[m], w[m], s.ld[m], off[m], (int64_t)k * 16);
      fragments(y[0], X + (int64_t)k * 2 * FRAG, rows);
    }, as_it_is);
    if (at.left) {
      v8h x[2][2], y[NJ][2];
#pragma unroll
      for (int m = 0; m < 2; ++m) raw8_end<!IN_OUT>(x[m], w[m], s.ld[m], off[m], (int64_t)at.s1 * 16, at.left);
      fragments(y, X + (int64_t)at.s1 * 2 * FRAG, rows);
#pragma unroll
      for (int m = 0; m < 2; ++m) ab[m].split(x[m]), ab[m].add(x[m], y);
    }
  }
  if constexpr (BWD) {
    const float* const w = IN_OUT ? s.w[2] + c0 * s.ld[2] : s.w[2] + c0;
    const uint32_t off = raw_off<IN_OUT>(s.ld[2], a.f - c0);
    const _Float16* G = s.G + b0 * s.KSG * 2 * FRAG + lane * 8;
    const int64_t rows = s.KSG * 2 * FRAG;
    const Steps at(s.e, wave, HIDDEN_WAVES);
    stream<1, 1>(g, at.s0, at.s1, [&](int k, v8h (&x)[1][2], v8h (&y)[1][NJ][2]) {
      raw8<IN_OUT>(x[0], w, s.ld[2], off, (int64_t)k * 16);
      fragments(y[0], G + (int64_t)k * 2 * FRAG, rows);
    }, as_it_is);
    if (at.left) {
      v8h x[2], y[NJ][2];
      raw8_end<IN_OUT>(x, w, s.ld[2], off, (int64_t)at.s1 * 16, at.left);
      fragments(y, G + (int64_t)at.s1 * 2 * FRAG, rows);
      g[0].split(x), g[0].add(x, y);
    }
  }
  // the waves' sums, a row block after the other: a lane has four columns of a row, 8 k + 4 half + 0 .. 3
  const Hidden at(a);
  static_assert(HIDDEN_WAVES == 4, "a wave for each k");
  const int k = wave;
  int ex[NJ], ey[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) ex[j] = s.ex[(b0 + j) * 32 + l32], ey[j] = BWD ? s.ey[(b0 + j) * 32 + l32] : 0;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (j > 0) __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int m = 0; m < 2; ++m) *reinterpret_cast<V4*>(&sh[wave][m][(q * 64 + lane) * 4]) = ab[m].four(j, q, ex[j]);
      if (BWD) *reinterpret_cast<V4*>(&sh[wave][SUMS - 1][(q * 64 + lane) * 4]) = g[0].four(j, q, ey[j]);
    }
    __syncthreads();
    V4 x[SUMS];
#pragma unroll
    for (int m = 0; m < SUMS; ++m) {
      x[m] = V4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < HIDDEN_WAVES; ++w) x[m] += *reinterpret_cast<const V4*>(&sh[w][m][(k * 64 + lane) * 4]);
    }
    const int64_t block = b0 + j, v = block * 32 + l32, c = c0 + k * 8 + half * 4;
    const bool there = v < a.n, whole = c0 + HB <= a.f;
    if (BWD && !s.make) {
      const int64_t row = there ? v : a.n - 1;
      x[0] = at.get(a.gate + row * a.ld_gate, c, whole), x[1] = at.get(a.up + row * a.ld_up, c, whole);
    }
    if (!BWD && a.gate && there) at.put(a.gate + v * a.ld_gate, c, x[0], whole), at.put(a.up + v * a.ld_up, c, x[1], whole);
    V4 h, da, db;
    float mh = 0.f, ma = 0.f, mb = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = there && c + i < a.f;
      const Act t = any_act(s.act, x[0][i]);
      h[i] = in ? t.v * x[1][i] : 0.f;
      mh = fmaxf(mh, fabsf(h[i]));
      if (BWD) {
        const float r = x[SUMS - 1][i];
        da[i] = in ? r * x[1][i] * t.s : 0.f, db[i] = in ? r * t.v : 0.f;
        ma = fmaxf(ma, fabsf(da[i])), mb = fmaxf(mb, fabsf(db[i]));
      }
    }
    const int64_t step = c0 / 16 + (k >> 1), step_d = c0 / 8 + (k >> 1);
    at.put_frag(a.H, a.KSH, block, step, k & 1, h);
    auto row_top = [&](int which, float m) {
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      if (half == 0) tops[which][k][j * 32 + l32] = m;
    };
    row_top(0, BWD ? ma : mh);
    if constexpr (BWD) {
      at.put_frag(a.D, a.KSD, block, step_d, k & 1, da);
      at.put_frag(a.D, a.KSD, block, step_d + 2, k & 1, db);
      row_top(1, mb);
      const float fx = pow2_or_0(-a.e_x[block]), fy = pow2_or_0(-a.e_y[block]);
      float ch[4], ca[4], cb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) ch[i] = fabsf(h[i] * fy), ca[i] = fabsf(da[i] * fx), cb[i] = fabsf(db[i] * fx);
      const float th = max_over_32(ch), ta = max_over_32(ca), tb = max_over_32(cb);
      const int col = k * 8 + half * 4 + (l32 >> 3);
      if (!(l32 & 7)) cols[0][j][col] = th, cols[1][j][col] = ta, cols[2][j][col] = tb;
    }
  }
  // largest values, to where they are kept: a thread each, so that all of them take one trip to memory
  __syncthreads();
  constexpr int R = NJ * 32, ROWS_OF = BWD ? 2 : 1;
  static_assert(ROWS_OF * R + 96 <= HIDDEN_WAVES * 64, "a thread each");
  if (tid < ROWS_OF * R) {
    const int which = tid / R, r = tid % R;
    const float m = fmaxf(fmaxf(tops[which][0][r], tops[which][1][r]), fmaxf(tops[which][2][r], tops[which][3][r]));
    if (b0 * 32 + r < a.n) raise((which == 0 ? a.h_row : a.d_row) + b0 * 32 + r, __float_as_uint(m));
  } else if (BWD && tid < ROWS_OF * R + 96) {
    const int which = (tid - ROWS_OF * R) >> 5, c = tid & 31;
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) m = fmaxf(m, cols[which][j][c]);
    if (c0 + c < a.f) raise((which == 0 ? a.h_col : which == 1 ? a.a_col : a.b_col) + c0 + c, __float_as_uint(m));
  }
}

struct StreamOut {
  int64_t n, f, width;                 // rows, reduction, columns
  const float* w[2];
  int64_t ld[2];
  const _Float16* P;                   // H or [dA dB] in the order of fragments
  int64_t KS;
  const uint32_t* top[2];              // largest values of its rows (of dA, of dB)
  int splits, row_tiles;
  float* out;
  int64_t pitch, part;                 // of a row, of a part of the sums
  int add;
};
// M: Y's weight, or the two of dX.
template <int M, bool BYK>
__global__ void __launch_bounds__(OUT_WAVES * 64, 2) k_stream_out(StreamOut s) {
  constexpr int GROUP = 32 * 4 + 4, BLOCK = 8 * GROUP;         // floats: four columns of 32 rows, a row block (what a store's lanes read lies in other banks)
  __shared__ __attribute__((aligned(16))) float sh[OUT_WAVES][NJ][BLOCK];
  const Tile tile(blockIdx.x, s.row_tiles, (s.width + 31) / 32, s.splits);
  if (tile.m < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int64_t c0 = tile.n * 32, b0 = tile.m * NJ;
  const float* w[M];
  uint32_t off[M];
  int er[M][NJ];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    w[m] = BYK ? s.w[m] + c0 * s.ld[m] : s.w[m] + c0, off[m] = raw_off<BYK>(s.ld[m], s.width - c0);
#pragma unroll
    for (int j = 0; j < NJ; ++j) er[m][j] = exp_or_0(scale_exp(s.top[m][(b0 + j) * 32 + l32]));
  }
  const _Float16* P = s.P + b0 * s.KS * 2 * FRAG + lane * 8;
  const int64_t rows = s.KS * 2 * FRAG;
  const auto step = [&](int k, int m) { return (int64_t)(M == 1 ? k : (k >> 1) * 4 + (k & 1) + 2 * m) * 2 * FRAG; };
  const auto in_b = [&](v8h (&y)[M][NJ][2]) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const float f = pow2(er[m][j]);
        split8(y[m][j][0], y[m][j][1], 1.f, [&](int) { return f; });
      }
  };
  Scaled sums[M];
  const Steps at(s.f, (int)tile.split * OUT_WAVES + wave, s.splits * OUT_WAVES);
  stream<M, M>(sums, at.s0, at.s1, [&](int k, v8h (&x)[M][2], v8h (&y)[M][NJ][2]) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      raw8<BYK>(x[m], w[m], s.ld[m], off[m], (int64_t)k * 16);
      fragments(y[m], P + step(k, m), rows);
    }
  }, in_b);
  if (at.left) {
    v8h x[M][2], y[M][NJ][2];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      raw8_end<BYK>(x[m], w[m], s.ld[m], off[m], (int64_t)at.s1 * 16, at.left);
      fragments(y[m], P + step(at.s1, m), rows);
    }
    in_b(y);
#pragma unroll
    for (int m = 0; m < M; ++m) sums[m].split(x[m]), sums[m].add(x[m], y[m]);
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      V4 x = sums[0].four(j, k, er[0][j]);
      if (M == 2) x += sums[M - 1].four(j, k, er[M - 1][j]);
      *reinterpret_cast<V4*>(&sh[wave][j][(k * 2 + half) * GROUP + l32 * 4]) = x;
    }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < NJ / 2; ++u) {
    const int i = u * OUT_WAVES * 64 + tid, j = i >> 8, row = (i >> 3) & 31, g = i & 7;
    const int64_t v = (b0 + j) * 32 + row, c = c0 + g * 4;
    if (v >= s.n || c >= s.width) continue;
    V4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < OUT_WAVES; ++q) x += *reinterpret_cast<const V4*>(&sh[q][j][g * GROUP + row * 4]);
    float* to = s.out + tile.split * s.part + v * s.pitch + c;
    if (c + 4 <= s.width) {
      if (s.add) x += *reinterpret_cast<const V4*>(to);
      *reinterpret_cast<V4*>(to) = x;
      continue;
    }
#pragma unroll
    for (int t = 0; t < 3; ++t)
      if (c + t < s.width) to[t] = s.add ? to[t] + x[t] : x[t];
  }
}
