// Gated feed-forward blocks:  A = X Wg ;  B = X Wu ;  H = act(A) * B ;  Y = H Wd, and their gradients:
//   G = dY Wd^T ;  dA = G * B * act'(A) ;  dB = G * act(A) ;  dX = dA Wg^T + dB Wu^T ;  dWg = X^T dA ;  dWu = X^T dB ;  dWd = H^T dY
#include <algorithm>

#include "ht_internal.h"

namespace {

// act(a) and its derivative.  exp(-|a|) gives s(a) and s(-a) = 1 - s(a) without cancellation.
struct Act {
  float v, s;
};
__device__ __forceinline__ Act act_of(int act, float a) {
  if (act == HT_GATE_RELU) return {a < 0.f ? 0.f : a, a > 0.f ? 1.f : a * 0.f};      // (NaN stays NaN)
  if (act == HT_GATE_GELU) {
    const float phi = 0.5f * erfcf(-a * 0.70710678118654752f);
    return {a * phi, fmaf(a * 0.39894228040143268f, expf(-0.5f * a * a), phi)};
  }
  const float k = 1.5957691216057308f;              // 2 sqrt(2 / pi)
  const float u = act == HT_GATE_GELU_TANH ? k * a * fmaf(0.044715f * a, a, 1.f) : a;
  const float e = expf(-fabsf(u)), r = 1.f / (1.f + e), hi = r, lo = e * r;
  const float s = u >= 0.f ? hi : lo, t = u >= 0.f ? lo : hi;
  if (act == HT_GATE_SIGMOID) return {s, s * t};
  const float du = act == HT_GATE_GELU_TANH ? k * fmaf(3.f * 0.044715f * a, a, 1.f) : 1.f;
  return {a * s, fmaf(a * s, t * du, s)};
}

// C[m, n] (+)= sum_k A[m, k] B[k, n], each by its strides; 64 x 64 a block.
struct Product {
  const float *A, *B;
  float* C;
  int64_t am, ak, bk, bn, cm, cn, M, N, K;
  int add;
};
__global__ void __launch_bounds__(256) k_ffn_product(Product p) {
  __shared__ float As[16][65], Bs[16][65];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < p.K; k0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int64_t k = k0 + (i & 15), m = m0 + (i >> 4), n = n0 + (i >> 4);
      As[i & 15][i >> 4] = k < p.K && m < p.M ? p.A[m * p.am + k * p.ak] : 0.f;
      Bs[i & 15][i >> 4] = k < p.K && n < p.N ? p.B[k * p.bk + n * p.bn] : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(As[k][ty * 4 + i], Bs[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= p.M || n >= p.N) continue;
      float* c = p.C + m * p.cm + n * p.cn;
      *c = p.add ? *c + acc[i][j] : acc[i][j];
    }
}

// H = act(A) * B; with dA, dB (G lies in dB): the gradients too.
__global__ void __launch_bounds__(256) k_ffn_gate(int act, const float* A, int64_t lda, const float* B, int64_t ldb, int64_t n, int64_t f, float* H, float* dA, float* dB) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n * f; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / f, c = i - r * f;
    const float a = A[r * lda + c], b = B[r * ldb + c];
    const Act x = act_of(act, a);
    H[i] = x.v * b;
    if (!dA) continue;
    const float g = dB[i];
    dA[i] = g * b * x.s;
    dB[i] = g * x.v;
  }
}

struct Ffn {
  ht_ctx* ctx;
  const ht_ffn_desc* D;
  const ht_tensor *X, *Wg, *Wu, *Wd;
  bool in_out() const { return D->w_form == HT_W_IN_OUT; }
  int product(int64_t M, int64_t N, int64_t K, const float* A, int64_t am, int64_t ak, const float* B, int64_t bk, int64_t bn, float* C, int64_t cm, int64_t cn, int add) const {
    if (M == 0 || N == 0) return HT_OK;
    k_ffn_product<<<dim3((unsigned)ceil_div64(M, 64), (unsigned)ceil_div64(N, 64)), 256, 0, ctx->stream>>>(Product{A, B, C, am, ak, bk, bn, cm, cn, M, N, K, add});
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  }
  // strides of a weight's inputs and outputs
  int64_t by_in(const ht_tensor* W) const { return in_out() ? W->ld : 1; }
  int64_t by_out(const ht_tensor* W) const { return in_out() ? 1 : W->ld; }
  int project(float* A, int64_t lda, float* B, int64_t ldb) const {
    HT_TRY(product(X->rows, D->d_hidden, D->d_in, X->ptr, X->ld, 1, Wg->ptr, by_in(Wg), by_out(Wg), A, lda, 1, 0));
    return product(X->rows, D->d_hidden, D->d_in, X->ptr, X->ld, 1, Wu->ptr, by_in(Wu), by_out(Wu), B, ldb, 1, 0);
  }
  int gate(const float* A, int64_t lda, const float* B, int64_t ldb, float* H, float* dA, float* dB) const {
    const int64_t n = X->rows * D->d_hidden;
    if (n == 0) return HT_OK;
    k_ffn_gate<<<(unsigned)std::min<int64_t>(ceil_div64(n, 256), 65536), 256, 0, ctx->stream>>>(D->act, A, lda, B, ldb, X->rows, D->d_hidden, H, dA, dB);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  }
  int fwd(ht_tensor* Y, ht_tensor* keep_a, ht_tensor* keep_b) const {
    const int64_t n = X->rows, f = D->d_hidden, e = D->d_out;
    OpsBlock m;
    const auto a = m.add<float>(keep_a ? 0 : n * f), b = m.add<float>(keep_b ? 0 : n * f), h = m.add<float>(n * f);
    HT_TRY(m.take(ctx));
    float *A = keep_a ? keep_a->ptr : m.at(a), *B = keep_b ? keep_b->ptr : m.at(b);
    const int64_t lda = keep_a ? keep_a->ld : f, ldb = keep_b ? keep_b->ld : f;
    HT_TRY(project(A, lda, B, ldb));
    HT_TRY(gate(A, lda, B, ldb, m.at(h), nullptr, nullptr));
    return product(n, e, f, m.at(h), f, 1, Wd->ptr, by_in(Wd), by_out(Wd), Y->ptr, Y->ld, 1, D->accumulate);
  }
  int bwd(const ht_tensor* kept_a, const ht_tensor* kept_b, const ht_tensor* dY, ht_tensor* dX, ht_tensor* dWg, ht_tensor* dWu, ht_tensor* dWd) const {
    const int64_t n = X->rows, d = D->d_in, f = D->d_hidden, e = D->d_out;
    OpsBlock m;
    const auto a = m.add<float>(kept_a ? 0 : n * f), b = m.add<float>(kept_b ? 0 : n * f), h = m.add<float>(n * f), da = m.add<float>(n * f), db = m.add<float>(n * f);
    HT_TRY(m.take(ctx));
    if (!kept_a) HT_TRY(project(m.at(a), f, m.at(b), f));
    HT_TRY(product(n, f, e, dY->ptr, dY->ld, 1, Wd->ptr, by_out(Wd), by_in(Wd), m.at(db), f, 1, 0));
    HT_TRY(gate(kept_a ? kept_a->ptr : m.at(a), kept_a ? kept_a->ld : f, kept_b ? kept_b->ptr : m.at(b), kept_b ? kept_b->ld : f, m.at(h), m.at(da), m.at(db)));
    if (dX) {
      HT_TRY(product(n, d, f, m.at(da), f, 1, Wg->ptr, by_out(Wg), by_in(Wg), dX->ptr, dX->ld, 1, D->accumulate));
      HT_TRY(product(n, d, f, m.at(db), f, 1, Wu->ptr, by_out(Wu), by_in(Wu), dX->ptr, dX->ld, 1, 1));
    }
    const int add = D->accumulate_dW;
    if (dWg) HT_TRY(product(d, f, n, X->ptr, 1, X->ld, m.at(da), f, 1, dWg->ptr, by_in(dWg), by_out(dWg), add));
    if (dWu) HT_TRY(product(d, f, n, X->ptr, 1, X->ld, m.at(db), f, 1, dWu->ptr, by_in(dWu), by_out(dWu), add));
    if (dWd) HT_TRY(product(f, e, n, m.at(h), 1, f, dY->ptr, dY->ld, 1, dWd->ptr, by_in(dWd), by_out(dWd), add));
    return HT_OK;
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

extern "C" int ht_ffn_fwd(ht_ctx* ctx, const ht_ffn_desc* desc, const ht_tensor* X, const ht_tensor* Wg, const ht_tensor* Wu, const ht_tensor* Wd, ht_tensor* Y, ht_tensor* gate,
                          ht_tensor* up) {
  if (!ctx) return HT_EINVAL;
  HT_TRY(check_block(ctx, "ht_ffn_fwd", desc, X, Wg, Wu, Wd, gate, up, Y));
  HT_TRY(check_apart(ctx, "ht_ffn_fwd", {{X, "X"}, {Wg, "Wg"}, {Wu, "Wu"}, {Wd, "Wd"}}, {{Y, "Y"}, {gate, "gate"}, {up, "up"}}));
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const Ffn op{ctx, desc, X, Wg, Wu, Wd};
  return ht_with_room(ctx, [&]() -> int { return op.fwd(Y, gate, up); });
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
  const Ffn op{ctx, desc, X, Wg, Wu, Wd};
  return ht_with_room(ctx, [&]() -> int { return op.bwd(gate, up, dY, dX, dWg, dWu, dWd); });
}
