// Distillation from a teacher's top logits: with q the softmax of a row's entries t_k / T among themselves and p that of the
// student's logits x / T over all classes, l = T^2 sum_k q_k (log q_k - log p_id(k)) and dx_c = u T (p_c - sum of q_k with id(k) = c) / N.
#include "ht_internal.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr int DISTILL_COUNTS = 256, DISTILL_BLOCKS = 4096;

// exp(x / T) = 2^(x f2).  A maximum or a log sum exp is taken from x before the difference is scaled: rows of the type's lowest value, a
// rounded product of which is off by more than 10^30, have differences of 0.
//
// Rows with entries, per block.
__global__ void __launch_bounds__(256) k_distill_count(const int32_t* __restrict__ ids, const float* __restrict__ t, int64_t V, int K, unsigned long long* __restrict__ cnt) {
  __shared__ unsigned long long sh[4];
  unsigned long long n = 0;
  for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < V; v += (int64_t)gridDim.x * 256) {
    bool any = false;
    for (int k = 0; k < K && !any; ++k) any = ids[v * K + k] >= 0 && t[v * K + k] != -INFINITY;
    n += any;
  }
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) cnt[blockIdx.x] = sh[0] + sh[1] + sh[2] + sh[3];
}

// T threads a row (a wave, or a block of 256).
template <int T>
struct Row {
  float* sh;                       // of the block's four waves
  __device__ __forceinline__ void sync() const {
    if (T > 64) __syncthreads();
  }
  template <class F>
  __device__ __forceinline__ float all(float x, F&& f) const {
    for (int o = 32; o > 0; o >>= 1) x = f(x, __shfl_xor(x, o, 64));
    if (T > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
      __syncthreads();
      x = f(f(sh[0], sh[1]), f(sh[2], sh[3]));
    }
    return x;
  }
  __device__ __forceinline__ float max(float x) const { return all(x, [](float a, float b) { return fmaxf(a, b); }); }
  __device__ __forceinline__ float sum(float x) const { return all(x, [](float a, float b) { return a + b; }); }
};

template <int T>
__global__ void __launch_bounds__(256) k_distill(const float* logits, int64_t ld, int64_t V, int C, const int32_t* __restrict__ ids, const float* __restrict__ top,
                                                 int K, float temp, const float* __restrict__ weight, const unsigned long long* __restrict__ cnt, int n_cnt, int mean,
                                                 float* __restrict__ row_loss, float* grad, int64_t ld_g, double* __restrict__ part) {
  constexpr int R = 256 / T, E = HT_DISTILL_MAX_K / T;
  __shared__ float red[4];
  __shared__ double dred[4];
  __shared__ int sid[R][HT_DISTILL_MAX_K];
  __shared__ float sq[R][HT_DISTILL_MAX_K];
  const int r = threadIdx.x / T, l = threadIdx.x % T;
  const Row<T> row{red};
  unsigned long long N = 0;
  for (int i = threadIdx.x & 63; i < n_cnt; i += 64) N += cnt[i];
  for (int o = 32; o > 0; o >>= 1) N += __shfl_xor(N, o, 64);
  const float inv = mean ? 1.f / (float)(N > 0 ? N : 1) : 1.f, f2 = LOG2E / temp;
  double mine = 0.0;
  for (int64_t v0 = (int64_t)blockIdx.x * R; v0 < V; v0 += (int64_t)gridDim.x * R) {
    const int64_t v = v0 + r;
    const bool there = v < V;                      // (the same in all threads of a row)
    const float* x = logits + v * ld;
    float* g = grad ? grad + v * ld_g : nullptr;
    int id[E];
    float t[E], m = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int k = e * T + l;
      id[e] = there && k < K ? ids[v * K + k] : -1;
      t[e] = id[e] >= 0 ? top[v * K + k] : -INFINITY;
      if (t[e] == -INFINITY) id[e] = -1;
      m = fmaxf(m, id[e] >= 0 ? (t[e] != t[e] ? INFINITY : t[e]) : -INFINITY);
    }
    m = row.max(m);
    const bool has = m != -INFINITY;
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) z += id[e] >= 0 ? exp2f((t[e] - m) * f2) : 0.f;
    z = row.sum(z);
    const float mq = m + temp * logf(z);             // (q = exp((t - mq) / T))
    if (!has) {
      if (there && l == 0 && row_loss) row_loss[v] = 0.f;
      if (there && g)
        for (int c = l * 4; c < C; c += T * 4) *reinterpret_cast<float4*>(g + c) = make_float4(0.f, 0.f, 0.f, 0.f);
      if (T == 64) continue;
    }
    if (T > 64 && !has) continue;
    float xm = -INFINITY;
    for (int c = l * 4; c < C; c += T * 4) {
      const float4 a = *reinterpret_cast<const float4*>(x + c);
      xm = fmaxf(xm, a.x);
      if (c + 1 < C) xm = fmaxf(xm, a.y);
      if (c + 2 < C) xm = fmaxf(xm, a.z);
      if (c + 3 < C) xm = fmaxf(xm, a.w);
    }
    xm = row.max(xm);
    float xz = 0.f;
    for (int c = l * 4; c < C; c += T * 4) {
      const float4 a = *reinterpret_cast<const float4*>(x + c);
      xz += exp2f((a.x - xm) * f2);
      if (c + 1 < C) xz += exp2f((a.y - xm) * f2);
      if (c + 2 < C) xz += exp2f((a.z - xm) * f2);
      if (c + 3 < C) xz += exp2f((a.w - xm) * f2);
    }
    xz = row.sum(xz);
    const bool none = xm == -INFINITY;             // no class is possible
    const float lse = none ? 0.f : xm + temp * logf(xz);
    float q[E], xt[E], loss = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[e] = id[e] >= 0 ? exp2f((t[e] - mq) * f2) : 0.f;
      xt[e] = id[e] >= 0 ? (id[e] < C ? x[id[e]] - lse : NAN) : 0.f;
      if (id[e] >= 0 && !(q[e] == 0.f && xt[e] == xt[e])) loss += q[e] * ((t[e] - mq) - xt[e]);
      const int k = e * T + l;
      sid[r][k] = id[e] < C ? id[e] : -1;
      sq[r][k] = q[e];
    }
    loss = row.sum(loss) * temp;
    const float u = weight ? weight[v] : 1.f;
    if (l == 0) {
      if (row_loss) row_loss[v] = loss;
      mine += (double)u * (double)loss;
    }
    if (g) {
      const float w = u * temp * inv;
      for (int c = l * 4; c < C; c += T * 4) {
        const float4 a = *reinterpret_cast<const float4*>(x + c);
        float4 o;
        o.x = none ? 0.f : w * exp2f((a.x - lse) * f2);
        o.y = none ? 0.f : w * exp2f((a.y - lse) * f2);
        o.z = none ? 0.f : w * exp2f((a.z - lse) * f2);
        o.w = none ? 0.f : w * exp2f((a.w - lse) * f2);
        if (c + 1 >= C) o.y = 0.f;
        if (c + 2 >= C) o.z = 0.f;
        if (c + 3 >= C) o.w = 0.f;
        *reinterpret_cast<float4*>(g + c) = o;
      }
      if (T > 64) __syncthreads();
      else __threadfence_block();
      // the entries' classes: an id's first entry subtracts all of its q
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (id[e] < 0 || id[e] >= C) continue;
        const int k = e * T + l;
        bool before = false;
        float s = 0.f;
        for (int j = 0; j < K; ++j) {
          if (sid[r][j] != id[e]) continue;
          before = before || j < k;
          s += sq[r][j];
        }
        if (!before) g[id[e]] = w * ((none ? 0.f : exp2f(xt[e] * f2)) - s);
      }
      row.sync();
    }
  }
  for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) dred[threadIdx.x >> 6] = mine;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (dred[0] + dred[1]) + (dred[2] + dred[3]);
}

__global__ void __launch_bounds__(256) k_distill_loss(const double* __restrict__ part, int n, const unsigned long long* __restrict__ cnt, int n_cnt, int mean,
                                                      float* __restrict__ loss) {
  __shared__ double sh[256];
  __shared__ unsigned long long sc[256];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += part[i];
  sh[threadIdx.x] = s;
  sc[threadIdx.x] = (int)threadIdx.x < n_cnt ? cnt[threadIdx.x] : 0ull;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) {
      sh[threadIdx.x] += sh[threadIdx.x + o];
      sc[threadIdx.x] += sc[threadIdx.x + o];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) *loss = sc[0] > 0 ? (float)(sh[0] / (mean ? (double)sc[0] : 1.0)) : 0.f;
}

}  // namespace

extern "C" int ht_distill_loss(ht_ctx* ctx, const ht_distill_desc* desc, const ht_tensor* logits, const int32_t* top_ids, const float* top_logits,
                               const float* row_weight, float* loss, float* row_loss, ht_tensor* dlogits) {
  if (!ctx) return HT_EINVAL;
  if (!desc || !logits || !loss) return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: null argument");
  if (desc->n_classes <= 0) return ht_set_err(ctx, HT_ESHAPE, "ht_distill_loss: number of classes must be positive");
  if (desc->k < 1 || desc->k > HT_DISTILL_MAX_K) return ht_set_err(ctx, HT_ESHAPE, "ht_distill_loss: %d entries a row, at least 1 and at most %d", desc->k, HT_DISTILL_MAX_K);
  if ((!top_ids || !top_logits) && logits->rows > 0) return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: null argument");
  if (!(desc->temperature > 0.f) || desc->temperature > 3.0e38f) return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: temperature must be positive and finite");
  if (desc->reduction != HT_REDUCE_MEAN && desc->reduction != HT_REDUCE_SUM)
    return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: unknown reduction %d", desc->reduction);
  HT_TRY(ht_check_rows(ctx, logits, logits->rows, desc->n_classes, "ht_distill_loss: logits"));
  if (dlogits) {
    HT_TRY(ht_check_rows(ctx, dlogits, logits->rows, desc->n_classes, "ht_distill_loss: dlogits"));
    if (ht_overlap(dlogits, logits) && (dlogits->ptr != logits->ptr || dlogits->ld != logits->ld))
      return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: dlogits shares memory with logits and is not logits");
  }
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const int64_t V = logits->rows;
  const int C = desc->n_classes, K = desc->k, mean = desc->reduction == HT_REDUCE_MEAN;
  return ht_with_room(ctx, [&]() -> int {
    OpsBlock m;
    const auto cnt = m.add<unsigned long long>(DISTILL_COUNTS);
    const auto part = m.add<double>(DISTILL_BLOCKS);
    HT_TRY(m.take(ctx));
    const unsigned nc = (unsigned)std::max<int64_t>(1, std::min<int64_t>(DISTILL_COUNTS, ceil_div64(V, 256)));
    k_distill_count<<<nc, 256, 0, ctx->stream>>>(top_ids, top_logits, V, K, m.at(cnt));
    HT_LAUNCH_CHECK(ctx);
    const bool wave = C <= 2048;
    const unsigned nb = (unsigned)std::max<int64_t>(1, std::min<int64_t>(DISTILL_BLOCKS, wave ? ceil_div64(V, 4) : V));
    float* g = dlogits ? dlogits->ptr : nullptr;
    const int64_t ld_g = dlogits ? dlogits->ld : 0;
    if (wave)
      k_distill<64><<<nb, 256, 0, ctx->stream>>>(logits->ptr, logits->ld, V, C, top_ids, top_logits, K, desc->temperature, row_weight, m.at(cnt), (int)nc, mean, row_loss,
                                                 g, ld_g, m.at(part));
    else
      k_distill<256><<<nb, 256, 0, ctx->stream>>>(logits->ptr, logits->ld, V, C, top_ids, top_logits, K, desc->temperature, row_weight, m.at(cnt), (int)nc, mean, row_loss,
                                                  g, ld_g, m.at(part));
    HT_LAUNCH_CHECK(ctx);
    k_distill_loss<<<1, 256, 0, ctx->stream>>>(m.at(part), (int)nb, m.at(cnt), (int)nc, mean, loss);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  });
}
