// What the kernels of gated feed-forward blocks share: the activations, a call's tensors, and the sums of what products leave in parts.
#pragma once

#include "ht_internal.h"

// One of ht_ffn_fwd (Y) and ht_ffn_bwd (dY); null: not there, or not asked for.
struct FfnCall {
  ht_ctx* ctx;
  const ht_ffn_desc* D;
  const ht_tensor *X, *Wg, *Wu, *Wd, *gate, *up;
  const ht_tensor *Y, *dY, *dX, *dWg, *dWu, *dWd;
  bool in_out() const { return D->w_form == HT_W_IN_OUT; }
};
// Of 1 .. HT_FFN_FEW rows (ht_ffn_few.hip).
constexpr int HT_FFN_FEW = 64;
int ht_ffn_few(const FfnCall& c);

// out [rows x cols] (+)= the sum of `parts` blocks of [rows x pitch], added up in their order; all of them in one launch.
struct FfnJoin {
  const float* sums;
  int64_t part, pitch, rows, cols;
  int parts, add;
  float* out;
  int64_t ld;
};
constexpr int FFN_JOINS = 4;
struct FfnJoins {
  unsigned first[FFN_JOINS];           // blocks before each (set by ht_ffn_join)
  FfnJoin join[FFN_JOINS];
  int n;
};
int ht_ffn_join(ht_ctx* ctx, FfnJoins& j);

namespace {

// act(a) and its derivative.  Kernels are made for three kinds: s(u) with u = a (k1 + k3 a^2), times a but for the sigmoid itself; the normal distribution; max(a, 0).
enum { LOGISTIC, NORMAL, LINEAR };
struct Gate {
  int act;
  float k1, k3;
  int alone;                           // s(u) itself
  __host__ __device__ int kind() const { return act == HT_GATE_GELU ? NORMAL : act == HT_GATE_RELU ? LINEAR : LOGISTIC; }
};
inline Gate gate_of(int act) {
  const float k = 1.5957691216057308f;             // 2 sqrt(2 / pi)
  return act == HT_GATE_GELU_TANH ? Gate{act, k, 0.044715f * k, 0} : Gate{act, 1.f, 0.f, act == HT_GATE_SIGMOID};
}
struct Act {
  float v, s;
};
template <int KIND>
__device__ __forceinline__ Act act_of(const Gate& g, float a) {
  constexpr float LOG2E = 1.44269504088896340736f;
  if constexpr (KIND == LOGISTIC) {
    // exp(-|u|) gives s(u) and s(-u) = 1 - s(u) without cancellation
    const float q = fminf(a * a, 1e30f), u = a * fmaf(g.k3, q, g.k1), du = fmaf(3.f * g.k3, q, g.k1);
    const float e = __builtin_amdgcn_exp2f(-fabsf(u) * LOG2E), hi = __builtin_amdgcn_rcpf(1.f + e), lo = e * hi;
    const float s = u >= 0.f ? hi : lo, v = a * s;
    return g.alone ? Act{s, lo * hi} : Act{v, fmaf(v, (u >= 0.f ? lo : hi) * du, s)};
  }
  if constexpr (KIND == NORMAL) {
    // Phi(-|a|) = e^(-a^2 / 2) / 2 times exp(z^2) erfc(z), z = |a| / sqrt(2), which is t times a polynomial of t = 1 / (1 + 0.4 z) to 6.2e-9 of itself (a least
    // squares fit to 4,000 values of t in (0, 1], weights raised where it was worst).  A library's erfc takes five times as long: 13 of 28 us of a launch over 1,003 x 1,213.
    constexpr float R[11] = {-0.0292151887f, 0.14044708f, -0.235528022f, 0.13756232f, -0.0468958393f, 0.0839167088f, 0.119008213f, 0.171739295f, 0.207613721f, 0.225675866f, 0.225675836f};
    const float e = __builtin_amdgcn_exp2f(a * a * (-0.5f * LOG2E)), t = __builtin_amdgcn_rcpf(fmaf(0.28284271247461901f, fabsf(a), 1.f));
    float r = R[0];
#pragma unroll
    for (int k = 1; k < 11; ++k) r = fmaf(r, t, R[k]);
    const float tail = 0.5f * e * (t * r), phi = a >= 0.f ? 1.f - tail : tail;
    return {a * phi, fmaf(a * 0.39894228040143268f, e, phi)};
  }
  return {a < 0.f ? 0.f : a, a > 0.f ? 1.f : a * 0.f};      // (NaN stays NaN)
}

}  // namespace
