// The norm of many tensors together, and those tensors scaled by what it may be:
//   norm = sqrt(sum of squares) ;  c = max_norm / norm where norm > max_norm, else 1 ;  out (+)= scale c g
// Squares are taken and added up in 64 bits: those of fp32 values neither overflow nor vanish there.  Blocks add up units of the tensors in a fixed
// order, one block their sums, so that the same tensors give the same bits.
#include <algorithm>
#include <new>

#include "ht_internal.h"

namespace {

typedef float V4 __attribute__((ext_vector_type(4)));
typedef float V4u __attribute__((ext_vector_type(4), aligned(4)));      // tensors need no alignment

// A tensor as rows of nv vectors of four (the last may be short); one without gaps between its rows is a single row.  Units are UNIT vectors, rows after rows.
struct Item {
  const float* g;
  float* out;
  int64_t cols, vecs, ld, out_ld;        // vecs: of all rows
};
// Of few values the units are small, so that there are blocks for all CUs (241 tensors of 4.5 M values a norm and a scaling 126 -> 103 us); of many they are large,
// so that few of them have to be looked for in the list.
constexpr int UNIT = 4096, SMALL_UNIT = 1024;
constexpr int64_t SMALL_VECS = (int64_t)2048 * UNIT;
// What is written goes past the caches where the gradients alone fill them (100 M values 246 -> 224 us); of fewer, whoever reads it next finds it there.
constexpr int64_t CACHED_VECS = (int64_t)8 << 20;
constexpr int LIST = 64;                 // tensors of a launch: their descriptions are arguments, so that recorded calls keep them
struct List {
  uint32_t unit0[LIST];                  // the launch's units before each (side by side: all of them are looked at at once)
  Item item[LIST];
  uint32_t units;
  int n, unit;
};
constexpr unsigned NORM_BLOCKS = 2048, END_THREADS = 1024;

// f(vector's place in row r, columns of it that there are) for the unit's vectors of this thread
template <class F>
__device__ __forceinline__ void each_vector(const Item& t, int64_t u, int unit, F&& f) {      // u: of the tensor
  const int64_t v0 = u * unit, nv = (t.cols + 3) / 4;
  const int n = (int)(t.vecs - v0 < unit ? t.vecs - v0 : unit);
  const int64_t r0 = v0 / nv, c0 = v0 - r0 * nv;
  if (c0 + n <= nv) {                    // in one row
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) f(r0, (c0 + i) * 4, t.cols - (c0 + i) * 4);
    return;
  }
  // (nv < 2^29 where there is more than one row)
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 256) {
    const uint32_t k = (uint32_t)(c0 + i), q = k / (uint32_t)nv;
    const int64_t c = (int64_t)(k - q * (uint32_t)nv) * 4;
    f(r0 + q, c, t.cols - c);
  }
}
__device__ __forceinline__ V4 load4(const float* p, int64_t left) {
  if (left >= 4) return *reinterpret_cast<const V4u*>(p);
  return V4{p[0], left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, 0.f};
}
// The tensor that a unit is of, a lane looks at one each, and its number there.
struct UnitOf {
  int i;
  uint32_t u;
  __device__ __forceinline__ UnitOf(const List& list, uint32_t unit) {
    const int lane = threadIdx.x & 63;
    const uint32_t first = lane < list.n ? list.unit0[lane] : 0xffffffffu;
    i = __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= unit)) - 1);
    u = unit - __builtin_amdgcn_readlane(first, i);
  }
};
static_assert(LIST == 64, "a lane each");
template <int N>
__device__ __forceinline__ double block_sum(double s) {
  __shared__ double sh[N / 64];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < N / 64; ++w) s += sh[w];
  return s;
}

__global__ void __launch_bounds__(256) k_grad_squares(List list, double* __restrict__ part) {
  double s = 0.0;
  for (uint32_t u = blockIdx.x; u < list.units; u += gridDim.x) {
    const UnitOf of(list, u);
    const Item& t = list.item[of.i];
    each_vector(t, of.u, list.unit, [&](int64_t r, int64_t c, int64_t left) {
      const V4 x = load4(t.g + r * t.ld + c, left);
      for (int k = 0; k < 4; ++k) s = fma((double)x[k], (double)x[k], s);
    });
  }
  s = block_sum<256>(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// factor (nullable) = scale c
__global__ void __launch_bounds__(END_THREADS) k_grad_end(const double* __restrict__ part, int64_t n, float* __restrict__ norm, float* __restrict__ factor, double max_norm,
                                                          double scale) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += END_THREADS) s += part[i];
  s = block_sum<END_THREADS>(s);
  if (threadIdx.x != 0) return;
  const double all = sqrt(s);
  if (norm) *norm = (float)all;
  if (factor) *factor = (float)(scale * (all <= max_norm ? 1.0 : max_norm / all));
}

// PAST: past the caches.  The tensors' units from their last to their first: what the sums have read last is what the caches still hold.
template <bool PAST>
__global__ void __launch_bounds__(256) k_grad_scale(List list, const float* __restrict__ factor, int add) {
  const float f = *factor;
  for (uint32_t u = blockIdx.x; u < list.units; u += gridDim.x) {
    const UnitOf of(list, u);
    const Item& t = list.item[of.i];
    if (!add && f == 1.f && t.out == t.g) continue;      // (it is there)
    each_vector(t, (t.vecs - 1) / list.unit - of.u, list.unit, [&](int64_t r, int64_t c, int64_t left) {
      V4 x = load4(t.g + r * t.ld + c, left);
      float* to = t.out + r * t.out_ld + c;
      if (add) {
        const V4 y = load4(to, left);
        for (int k = 0; k < 4; ++k) x[k] = fmaf(f, x[k], y[k]);
      } else {
        x *= f;
      }
      if (left >= 4) {
        if (PAST) __builtin_nontemporal_store(x, reinterpret_cast<V4u*>(to));
        else *reinterpret_cast<V4u*>(to) = x;
      } else {
        for (int k = 0; k < 3; ++k)
          if (k < left) to[k] = x[k];
      }
    });
  }
}

int check(ht_ctx* ctx, const char* name, const char* what, int32_t i, const ht_tensor& t) {
  if (t.rows >= 0 && t.rows <= INT32_MAX && t.cols >= 0 && t.ld >= t.cols && t.loc == HT_LOC_DEVICE && ((uintptr_t)t.ptr & 3) == 0 && (t.ptr || t.rows == 0 || t.cols == 0)) return HT_OK;
  char s[96];                          // (a text for each of hundreds of tensors would be most of a call)
  snprintf(s, sizeof s, "%s: %s %d", name, what, i);
  if (t.rows < 0 || t.cols < 0) return ht_set_err(ctx, HT_ESHAPE, "%s: [%lld x %d]", s, (long long)t.rows, t.cols);
  return ht_check_weights(ctx, &t, t.rows, t.cols, s);
}

// No output may share memory with another, or with a gradient that is not the very same view and its own.
int check_shared(ht_ctx* ctx, int32_t n, const ht_tensor* grads, const ht_tensor* out) {
  struct Span {
    const float *a, *b;
    const ht_tensor* t;
    int32_t i;
    bool out;
  };
  std::vector<Span> spans;
  spans.reserve((size_t)n * 2);
  for (int32_t i = 0; i < n; ++i)
    for (int o = 0; o < 2; ++o) {
      const ht_tensor* t = o ? out + i : grads + i;
      if (t->rows > 0 && t->cols > 0) spans.push_back(Span{t->ptr, t->ptr + (t->rows - 1) * t->ld + t->cols, t, i, o == 1});
    }
  std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.a < y.a; });
  for (size_t i = 0; i < spans.size(); ++i)
    for (size_t j = i + 1; j < spans.size() && spans[j].a < spans[i].b; ++j) {
      const Span &x = spans[i], &y = spans[j];
      if (!x.out && !y.out) continue;
      if (x.i == y.i && x.out != y.out && x.t->ptr == y.t->ptr && (x.t->ld == y.t->ld || x.t->rows == 1)) continue;
      if (ht_shares(x.t, y.t))
        return ht_set_err(ctx, HT_EINVAL, "ht_grad_clip: out %d shares memory with %s %d", x.out ? x.i : y.i, x.out && y.out ? "out" : "gradient", x.out ? y.i : x.i);
    }
  return HT_OK;
}

// norm is none of a tensor's values (it may lie between its rows): scaled with them it would be no norm, and the norm written over a gradient would be scaled.
int check_norm(ht_ctx* ctx, const char* name, const char* what, int32_t n, const ht_tensor* t, const float* norm) {
  const uintptr_t p = (uintptr_t)norm;
  if (p & 3) return ht_set_err(ctx, HT_EINVAL, "%s: norm must be 4-byte aligned", name);
  for (int32_t i = 0; norm && i < n; ++i) {
    const uintptr_t a = (uintptr_t)t[i].ptr, row = (uintptr_t)t[i].ld * 4;
    if (p < a || t[i].rows == 0 || t[i].cols == 0 || (p - a) / row >= (uintptr_t)t[i].rows || (p - a) % row >= (uintptr_t)t[i].cols * 4) continue;
    return ht_set_err(ctx, HT_EINVAL, "%s: norm shares memory with %s %d", name, what, i);
  }
  return HT_OK;
}

// Launches over the tensors, LIST of them at a time: launch(list).  With out from the last tensor to the first.
template <class F>
int in_lists(int32_t n, const ht_tensor* grads, const ht_tensor* out, int unit, F&& launch) {
  List list;
  list.n = 0, list.units = 0, list.unit = unit;
  for (int32_t k = 0; k < n; ++k) {
    const int32_t i = out ? n - 1 - k : k;
    const ht_tensor& g = grads[i];
    if (g.rows <= 0 || g.cols <= 0) continue;
    const bool flat = g.rows == 1 || (g.ld == g.cols && (!out || out[i].ld == g.cols));
    const int64_t cols = flat ? g.rows * g.cols : g.cols, vecs = (flat ? 1 : g.rows) * ((cols + 3) / 4);
    list.unit0[list.n] = list.units;
    list.item[list.n++] = Item{g.ptr, out ? out[i].ptr : nullptr, cols, vecs, flat ? 0 : g.ld, out && !flat ? out[i].ld : 0};
    list.units += (uint32_t)((vecs + unit - 1) / unit);
    if (list.n == LIST) {
      HT_TRY(launch(list));
      list.n = 0, list.units = 0;
    }
  }
  return list.n > 0 ? launch(list) : HT_OK;
}

int grads_run(ht_ctx* ctx, int32_t n, const ht_tensor* grads, const ht_tensor* out, double max_norm, double scale, int add, float* norm, bool scaled) {
  hipStream_t st = ctx->stream;
  int64_t parts = 0, vecs = 0;
  for (int32_t i = 0; i < n; ++i)
    if (grads[i].rows > 0 && grads[i].cols > 0) vecs += grads[i].rows * ((grads[i].cols + 3) / 4);
  const int unit = vecs < SMALL_VECS ? SMALL_UNIT : UNIT;
  auto blocks = [](const List& l) { return (unsigned)std::min<uint32_t>(l.units, NORM_BLOCKS); };
  HT_TRY(in_lists(n, grads, nullptr, unit, [&](const List& l) { return parts += blocks(l), (int)HT_OK; }));
  OpsBlock m;
  const auto part = m.add<double>(parts);
  const auto factor = m.add<float>(1);
  HT_TRY(m.take(ctx));
  int64_t at = 0;
  HT_TRY(in_lists(n, grads, nullptr, unit, [&](const List& l) -> int {
    k_grad_squares<<<blocks(l), 256, 0, st>>>(l, m.at(part) + at);
    HT_LAUNCH_CHECK(ctx);
    at += blocks(l);
    return HT_OK;
  }));
  k_grad_end<<<1, END_THREADS, 0, st>>>(m.at(part), parts, norm, scaled ? m.at(factor) : nullptr, max_norm, scale);
  HT_LAUNCH_CHECK(ctx);
  if (!scaled) return HT_OK;
  return in_lists(n, grads, out, unit, [&](const List& l) -> int {
    (vecs > CACHED_VECS ? k_grad_scale<true> : k_grad_scale<false>)<<<(unsigned)std::min<uint32_t>(l.units, 1u << 20), 256, 0, st>>>(l, m.at(factor), add);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  });
}

}  // namespace

extern "C" int ht_grad_norm(ht_ctx* ctx, int32_t n, const ht_tensor* grads, float* norm) {
  if (!ctx) return HT_EINVAL;
  if (n < 0 || (n > 0 && !grads) || !norm) return ht_set_err(ctx, HT_EINVAL, "ht_grad_norm: %s", n < 0 ? "a negative number of tensors" : "null argument");
  for (int32_t i = 0; i < n; ++i) HT_TRY(check(ctx, "ht_grad_norm", "gradient", i, grads[i]));
  HT_TRY(check_norm(ctx, "ht_grad_norm", "gradient", n, grads, norm));
  HT_HIP(ctx, hipSetDevice(ctx->device));
  return ht_with_room(ctx, [&]() -> int { return grads_run(ctx, n, grads, nullptr, 1.0, 1.0, 0, norm, false); });
}

extern "C" int ht_grad_clip(ht_ctx* ctx, int32_t n, const ht_tensor* grads, double max_norm, double scale, int32_t accumulate, ht_tensor* out, float* norm) {
  if (!ctx) return HT_EINVAL;
  if (n < 0 || (n > 0 && !grads)) return ht_set_err(ctx, HT_EINVAL, "ht_grad_clip: %s", n < 0 ? "a negative number of tensors" : "null argument");
  if (!(max_norm > 0.0)) return ht_set_err(ctx, HT_EINVAL, "ht_grad_clip: max_norm %g, must be positive", max_norm);
  const ht_tensor* to = out ? out : grads;
  for (int32_t i = 0; i < n; ++i) {
    HT_TRY(check(ctx, "ht_grad_clip", "gradient", i, grads[i]));
    HT_TRY(check(ctx, "ht_grad_clip", "out", i, to[i]));
    if (to[i].rows != grads[i].rows || to[i].cols != grads[i].cols)
      return ht_set_err(ctx, HT_ESHAPE, "ht_grad_clip: out %d is [%lld x %d], its gradient [%lld x %d]", i, (long long)to[i].rows, to[i].cols, (long long)grads[i].rows,
                        grads[i].cols);
  }
  try {
    HT_TRY(check_shared(ctx, n, grads, to));
  } catch (const std::bad_alloc&) {
    return ht_set_err(ctx, HT_ENOMEM, "ht_grad_clip: no host memory for %d tensors", n);
  }
  HT_TRY(check_norm(ctx, "ht_grad_clip", "gradient", n, grads, norm));
  if (out) HT_TRY(check_norm(ctx, "ht_grad_clip", "out", n, out, norm));
  HT_HIP(ctx, hipSetDevice(ctx->device));
  return ht_with_room(ctx, [&]() -> int { return grads_run(ctx, n, grads, to, max_norm, scale, accumulate, norm, true); });
}
