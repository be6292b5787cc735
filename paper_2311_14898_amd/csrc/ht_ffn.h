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
  unsigned blocks;                     // (set by ht_ffn_join)
};
struct FfnJoins {
  FfnJoin join[4];
  int n;
};
int ht_ffn_join(ht_ctx* ctx, FfnJoins& j);

namespace {

// act(a) and its derivative.  Kernels are made for two kinds: s(u) with u = a (k1 + k3 a^2), times a but for the sigmoid itself, and the others.
enum { LOGISTIC, OTHERS };
struct Gate {
  int act;
  float k1, k3;
  int alone;                           // s(u) itself
  __host__ __device__ bool logistic() const { return act != HT_GATE_GELU && act != HT_GATE_RELU; }
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
  if (g.act == HT_GATE_RELU) return {a < 0.f ? 0.f : a, a > 0.f ? 1.f : a * 0.f};      // (NaN stays NaN)
  const float phi = 0.5f * erfcf(-a * 0.70710678118654752f);
  return {a * phi, fmaf(a * 0.39894228040143268f, __builtin_amdgcn_exp2f(a * a * (-0.5f * LOG2E)), phi)};
}

}  // namespace
