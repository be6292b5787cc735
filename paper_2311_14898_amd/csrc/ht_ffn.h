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
// Of 1 .. HT_FFN_FEW rows (ht_ffn_few.hip); with FEW_WEIGHTS values of weights, of at most 16: more multiply longer there than they read (2,048 x 8,192, us there | with weights split: forward
// of 16 rows 49 | 59, 17 68 | 59, 64 107 | 61, backward 171 | 188, 209 | 192, 313 | 198; 1,024 x 4,096: forward of 48 rows 30 | 36, 64 38 | 36, backward 68 | 77, 81 | 79).
constexpr int HT_FFN_FEW = 64;
constexpr int64_t FEW_WEIGHTS = (int64_t)1 << 24;
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

// act(a) and its derivative; kernels are made for each (HT_GATE_*): what is made of a product's sums takes the vector units as long as the product takes the matrix cores.
struct Act {
  float v, s;
};
template <int ACT>
__device__ __forceinline__ Act act_of(float a) {
  constexpr float LOG2E = 1.44269504088896340736f;
  if constexpr (ACT == HT_GATE_SILU) {
    // s(-a) = 1 - s(a) is off by half a step of 1 where it is small, and so is the derivative, which is near 1 there
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -LOG2E)), v = a * s;
    return {v, fmaf(v, 1.f - s, s)};
  }
  if constexpr (ACT == HT_GATE_GELU_TANH) {        // s(u), u = 2 sqrt(2 / pi) (a + 0.044715 a^3)
    constexpr float K1 = 1.5957691216057308f, K3 = 0.044715f * K1;
    const float q = fminf(a * a, 1e30f), s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * fmaf(q, -LOG2E * K3, -LOG2E * K1))), v = a * s;
    return {v, fmaf(v * (1.f - s), fmaf(q, 3.f * K3, K1), s)};
  }
  if constexpr (ACT == HT_GATE_SIGMOID) {          // exp(-|a|) gives s(a) and s(-a) without cancellation
    const float e = __builtin_amdgcn_exp2f(fabsf(a) * -LOG2E), hi = __builtin_amdgcn_rcpf(1.f + e), lo = e * hi;
    return {a >= 0.f ? hi : lo, lo * hi};
  }
  if constexpr (ACT == HT_GATE_GELU) {
    // Phi(-|a|) = e^(-a^2 / 2) / 2 times exp(z^2) erfc(z), z = |a| / sqrt(2), which is t times a polynomial of t = 1 / (1 + 0.4 z) to 1.4e-8 of itself (a least
    // squares fit to 4,000 values of t in (0, 1], weights raised where it was worst, its coefficients rounded to floats).  The rounding of a^2 in the exponent counts a^2 / 2 fold.  A library's erfc takes five times as long: 13 of 28 us of k_ffn_narrow over 1,003 x 1,213.
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
__device__ __forceinline__ Act any_act(int act, float a) {
  switch (act) {
    case HT_GATE_SILU: return act_of<HT_GATE_SILU>(a);
    case HT_GATE_GELU: return act_of<HT_GATE_GELU>(a);
    case HT_GATE_GELU_TANH: return act_of<HT_GATE_GELU_TANH>(a);
    case HT_GATE_RELU: return act_of<HT_GATE_RELU>(a);
    default: return act_of<HT_GATE_SIGMOID>(a);
  }
}

}  // namespace
