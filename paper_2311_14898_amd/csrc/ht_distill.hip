// Distillation from a teacher's top logits: with q the softmax of a row's entries t_k / T among themselves and p that of the
// student's logits x / T over all classes, l = T^2 sum_k q_k (log q_k - log p_id(k)) and dx_c = u T (p_c - sum of q_k with id(k) = c) / N.
//
// What bounds it is memory: the logits are read and their gradient is written, once each where a row fits its threads' registers (up to 65,536 classes).
#include <type_traits>

#include "ht_internal.h"

namespace {

constexpr int DISTILL_COUNTS = 256, DISTILL_BLOCKS = 4096;
constexpr int FEW_ROWS = 64, FEW_PARTS = 64, FEW_CLASSES = 4096;      // rows up to which a row of more classes is cut among blocks, and into how many parts at most

struct DistillArgs {
  const float* x;                  // (may be grad)
  int64_t ld, V;
  int C;
  const int32_t* ids;
  const float* top;
  int K;
  float temp, f2, f2_low;          // log2 e / temp in two parts
  const float* weight;
  int mean;
  float* row_loss;
  float* grad;
  int64_t ld_g;
};

// exp(d / T) of a difference d <= 0: 2^(d f2) to the last bits (the product's rounding and the rest of f2 are made good: at d f2 = 20 they are 20 half steps).
// What is below 2^-200 is 0, as it would be; NaN stays.
__device__ __forceinline__ float exp_of(float d, const DistillArgs& a) {
  const float y0 = d * a.f2;
  const float e = y0 < -200.f ? 0.f : fmaf(d, a.f2, -y0) + d * a.f2_low;
  const float r = __builtin_amdgcn_exp2f(y0);
  return fmaf(r, e * 0.69314718055994530942f, r);
}

__device__ __forceinline__ bool has_entries(const DistillArgs& a, int64_t v) {
  bool any = false;
  for (int k = 0; k < a.K && !any; ++k) any = a.ids[v * a.K + k] >= 0 && a.top[v * a.K + k] != -INFINITY;
  return any;
}

// How many of at most FEW_ROWS rows have entries, counted by a block for itself; with[v]: whether row v has.
__device__ __forceinline__ int count_few(const DistillArgs& a, int* with) {
  for (int v = threadIdx.x; v < FEW_ROWS; v += blockDim.x) with[v] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < a.V * a.K; i += blockDim.x)
    if (a.ids[i] >= 0 && a.top[i] != -INFINITY) with[i / a.K] = 1;
  __syncthreads();
  static_assert(FEW_ROWS == 64, "a row a lane");
  return __popcll(__ballot(with[threadIdx.x & 63]));
}

// Rows with entries, per block.
__global__ void __launch_bounds__(256) k_distill_count(DistillArgs a, unsigned long long* __restrict__ cnt) {
  __shared__ unsigned long long sh[4];
  unsigned long long n = 0;
  for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < a.V; v += (int64_t)gridDim.x * 256) n += has_entries(a, v);
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) cnt[blockIdx.x] = sh[0] + sh[1] + sh[2] + sh[3];
}

// The value of the lane N further round in the same 16.
template <int N>
__device__ __forceinline__ float turn16(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, false)); }

// T threads of a block that work on one row together.
template <int T>
struct Row {
  static constexpr int W = T > 64 ? T / 64 : 1;
  float2* sh;                      // [W]
  __device__ __forceinline__ void sync() const {
    if (T > 64) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  }
  template <class F>
  __device__ __forceinline__ float2 all(float2 x, F&& f) const {
    // (turned round, the lanes add the same pairs: the same bits in all of them)
    x = f(x, make_float2(turn16<8>(x.x), turn16<8>(x.y)));
    x = f(x, make_float2(turn16<4>(x.x), turn16<4>(x.y)));
    x = f(x, make_float2(turn16<2>(x.x), turn16<2>(x.y)));
    x = f(x, make_float2(turn16<1>(x.x), turn16<1>(x.y)));
    if (T > 16) {
      x = f(x, make_float2(__shfl_xor(x.x, 16, 64), __shfl_xor(x.y, 16, 64)));
      x = f(x, make_float2(__shfl_xor(x.x, 32, 64), __shfl_xor(x.y, 32, 64)));
    }
    if (T > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
      __syncthreads();
      x = sh[0];
      for (int w = 1; w < W; ++w) x = f(x, sh[w]);
    }
    return x;
  }
  __device__ __forceinline__ float2 max(float2 x) const { return all(x, [](float2 a, float2 b) { return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y)); }); }
  __device__ __forceinline__ float2 sum(float2 x) const { return all(x, [](float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }); }
};

// A row's entries in LDS: id (-1: not there), and t, which later becomes q.  Returns the largest t (inf where one is NaN, -inf where none is there).
template <int T>
__device__ __forceinline__ float load_entries(const DistillArgs& a, int64_t v, int l, int* sid, float* sq) {
  float m = -INFINITY;
  for (int k = l; k < a.K; k += T) {
    int id = a.ids[v * a.K + k];
    const float t = id >= 0 ? a.top[v * a.K + k] : -INFINITY;
    if (t == -INFINITY) id = -1;
    sid[k] = id;
    sq[k] = t;
    m = fmaxf(m, t == t ? t : INFINITY);
  }
  return m;
}

// A term of the loss, over T: q ((t - mq) - (x - lse)), 0 where q is.
__device__ __forceinline__ float loss_term(float q, float lq, float lp) { return q == 0.f && lp == lp ? 0.f : q * (lq - lp); }

// What an id's first entry leaves of the gradient: w p less w times all of the id's q, added up in their order.
__device__ __forceinline__ void put_entry(const DistillArgs& a, const int* sid, const float* sq, int k, float* g, float w, float p) {
  const int id = sid[k];
  float s = 0.f;
  for (int j = 0; j < a.K; ++j) {
    if (sid[j] != id) continue;
    if (j < k) return;
    s += sq[j];
  }
  g[id] = w * (p - s);
}

typedef float V4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float4 zero4() { return make_float4(0.f, 0.f, 0.f, 0.f); }

// T threads a row, NV float4 of it in each thread's registers; what goes beyond (MORE) is read once more for the gradient, the last read first, while some of
// it is still in the caches.  Rows of T x NV x 4 classes.  Short rows want waves (at most 72 registers: 100,003 rows x 172 56.7 -> 53.2 us, with three float4s a thread for four 51.3); long rows
// past the caches, loads and stores that are not for them (4,096 x 131,072, where 49,152 classes stay in registers: 1.15 ms, with such stores 1.08, with loads too 1.05).
template <int T, int NV, bool MORE, bool FEW>
__global__ void __launch_bounds__(T < 256 ? 256 : T, T < 256 ? 7 : 1) k_distill(DistillArgs a, unsigned long long* __restrict__ cnt, int n_cnt, double* __restrict__ part) {
  constexpr int B = T < 256 ? 256 : T, R = B / T;
  extern __shared__ float entries[];             // [R][K] ids, [R][K] q
  __shared__ float2 red[B / 64];
  __shared__ double dred[B / 64];
  __shared__ int with[FEW ? FEW_ROWS : 1];
  const int r = threadIdx.x / T, l = threadIdx.x % T;
  const uint32_t C = a.C;                        // (columns are counted in 32 bits without a sign: up to 16,383 behind the last of 2^31 - 1)
  const Row<T> row{red};
  int* sid = reinterpret_cast<int*>(entries) + r * a.K;
  float* sq = entries + R * a.K + r * a.K;
  unsigned long long N = 0;
  if (FEW) {                                     // (at most FEW_ROWS: nobody has counted them, a launch less; k_distill_loss is told)
    N = count_few(a, with);
    if (blockIdx.x == 0 && threadIdx.x == 0) *cnt = N;
  } else {
    for (int i = threadIdx.x & 63; i < n_cnt; i += 64) N += cnt[i];
    for (int o = 32; o > 0; o >>= 1) N += __shfl_xor(N, o, 64);
  }
  const float inv = a.mean ? 1.f / (float)(N > 0 ? N : 1) : 1.f;
  double mine = 0.0;
  for (int64_t v0 = (int64_t)blockIdx.x * R; v0 < a.V; v0 += (int64_t)gridDim.x * R) {
    const int64_t v = v0 + r;
    if (T <= 64 && v >= a.V) continue;           // (larger rows are a block's)
    const float* x = a.x + v * a.ld;
    float* g = a.grad ? a.grad + v * a.ld_g : nullptr;
    float4 keep[NV];
    auto read = [&](int i) {                     // the i-th float4 of the thread; what lies behind the last class counts as -inf
      const uint32_t c = (uint32_t)(i * T + l) * 4;
      float4 y = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (c < C) {
        y = *reinterpret_cast<const float4*>(x + c);
        if (c + 1 >= C) y.y = -INFINITY;
        if (c + 2 >= C) y.z = -INFINITY;
        if (c + 3 >= C) y.w = -INFINITY;
      }
      return y;
    };
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (MORE) {                                // (read once: behind none of it is the last class)
        const V4 y = __builtin_nontemporal_load(reinterpret_cast<const V4*>(x + (u * T + l) * 4));
        keep[u] = make_float4(y.x, y.y, y.z, y.w);
      } else {
        keep[u] = read(u);
      }
    }
    const float tmax = load_entries<T>(a, v, l, sid, sq);
    float xm = -INFINITY, z = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u) xm = fmaxf(xm, fmaxf(fmaxf(keep[u].x, keep[u].y), fmaxf(keep[u].z, keep[u].w)));
    auto sum4 = [&](float4 y, float m) { return (exp_of(y.x - m, a) + exp_of(y.y - m, a)) + (exp_of(y.z - m, a) + exp_of(y.w - m, a)); };
    const int more = MORE ? (int)(((int64_t)a.C + T * 4 - 1) / (T * 4)) : NV;
    float zm = 0.f, mm = -INFINITY;              // of the part beyond: sum less mm
    if (MORE) {
      for (int i = NV; i < more; i += 4) {
        float4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = read(i + u);
        float m = mm;
#pragma unroll
        for (int u = 0; u < 4; ++u) m = fmaxf(m, fmaxf(fmaxf(y[u].x, y[u].y), fmaxf(y[u].z, y[u].w)));
        const float s = m == -INFINITY ? 0.f : m;
        zm *= mm == m ? 1.f : exp_of(mm - s, a);
#pragma unroll
        for (int u = 0; u < 4; ++u) zm += sum4(y[u], s);
        mm = m;
      }
    }
    const float2 top = row.max(make_float2(tmax, fmaxf(xm, mm)));
    if (top.x == -INFINITY) {                    // no teacher
      if (l == 0 && a.row_loss) a.row_loss[v] = 0.f;
      if (g)
        for (uint32_t c = l * 4; c < C; c += T * 4) *reinterpret_cast<float4*>(g + c) = zero4();
      continue;
    }
    xm = top.y == -INFINITY ? 0.f : top.y;
#pragma unroll
    for (int u = 0; u < NV; ++u) z += sum4(keep[u], xm);
    if (MORE && mm != -INFINITY) z += zm * exp_of(mm - xm, a);
    if (MORE && mm == -INFINITY) z += zm;        // (0, or NaN where all that is beyond is)
    float tz = 0.f;
    for (int k = l; k < a.K; k += T)
      if (sid[k] >= 0) tz += exp_of(sq[k] - top.x, a);
    const float2 sums = row.sum(make_float2(tz, z));
    const bool none = top.y == -INFINITY && sums.y == 0.f;             // no class is possible (logits that are all NaN, or NaN and -inf, have no largest either)
    const float mq = a.temp * logf(sums.x), lse = none ? 0.f : a.temp * logf(sums.y), iz = 1.f / sums.x, ip = none ? 0.f : 1.f / sums.y;
    float loss = 0.f;
    for (int k = l; k < a.K; k += T) {
      const int id = sid[k];
      const float d = sq[k] - top.x, q = id >= 0 ? exp_of(d, a) * iz : 0.f;
      sq[k] = q;
      if (id >= 0) loss += loss_term(q, d - mq, id < a.C ? x[id] - xm - lse : NAN);
    }
    loss = row.sum(make_float2(loss, 0.f)).x * a.temp;
    const float u = a.weight ? a.weight[v] : 1.f;
    if (l == 0) {
      if (a.row_loss) a.row_loss[v] = loss;
      mine += (double)u * (double)loss;
    }
    if (!g) continue;
    const float w = u * a.temp * inv, wp = none ? 0.f : w * ip;
    // p of the entries' classes, before a gradient can take the place of their logits
    constexpr int EK = (HT_DISTILL_MAX_K + T - 1) / T;
    float pe[EK];
#pragma unroll
    for (int e = 0; e < EK; ++e) {
      const int k = e * T + l, id = k < a.K ? sid[k] : -1;
      pe[e] = id >= 0 && id < a.C && !none ? exp_of(x[id] - xm, a) * ip : 0.f;
    }
    row.sync();
    auto put = [&](int i, float4 y) {
      const uint32_t c = (uint32_t)(i * T + l) * 4;
      if (c >= C) return;
      float4 o = make_float4(exp_of(y.x - xm, a) * wp, exp_of(y.y - xm, a) * wp, exp_of(y.z - xm, a) * wp, exp_of(y.w - xm, a) * wp);
      if (none) o = zero4();
      if (MORE) __builtin_nontemporal_store(V4{o.x, o.y, o.z, o.w}, reinterpret_cast<V4*>(g + c));     // (or it drives out of the caches what is read again)
      else *reinterpret_cast<float4*>(g + c) = o;
    };
    if (MORE) {
      for (int i = NV + (more - NV + 3) / 4 * 4 - 4; i >= NV; i -= 4) {
        float4 y[4];
#pragma unroll
        for (int u2 = 0; u2 < 4; ++u2) y[u2] = read(i + u2);
#pragma unroll
        for (int u2 = 0; u2 < 4; ++u2) put(i + u2, y[u2]);
      }
    }
#pragma unroll
    for (int u2 = 0; u2 < NV; ++u2) put(u2, keep[u2]);
    row.sync();
    if (l < (-a.C & 3)) g[a.C + l] = 0.f;        // (NaN until here where the row's weight is not finite)
#pragma unroll
    for (int e = 0; e < EK; ++e) {
      const int k = e * T + l;
      if (k < a.K && sid[k] >= 0 && sid[k] < a.C) put_entry(a, sid, sq, k, g, w, pe[e]);
    }
    row.sync();
  }
  for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) dred[threadIdx.x >> 6] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = dred[0];
    for (int w = 1; w < B / 64; ++w) s += dred[w];
    part[blockIdx.x] = s;
  }
}

__global__ void __launch_bounds__(256) k_distill_loss(const double* __restrict__ part, int n, const unsigned long long* __restrict__ cnt, int n_cnt, int mean,
                                                      float* __restrict__ loss) {
  __shared__ double sh[256];
  __shared__ unsigned long long sc[256];
  double s = 0.0;
#pragma unroll 8
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

// ---- few rows of many classes: a row's classes in `gridDim.x` parts.  The first launch leaves each part's maximum and sum, and the entries'
// logits (before a gradient can take their place); in the second every block joins its row's parts, and one more makes the losses.
__device__ __forceinline__ void part_of(int C, int parts, int part, uint32_t* c0, uint32_t* c1) {      // (whole float4s)
  const int64_t n4 = ((int64_t)C + 3) / 4;
  *c0 = (uint32_t)(n4 * part / parts * 4);
  const int64_t e = n4 * (part + 1) / parts * 4;
  *c1 = e < C ? (uint32_t)e : (uint32_t)C;
}

__global__ void __launch_bounds__(256) k_distill_part(DistillArgs a, float2* __restrict__ part, float* __restrict__ xe) {
  __shared__ float2 red[4];
  const Row<256> row{red};
  const int64_t v = blockIdx.y;
  const float* x = a.x + v * a.ld;
  const uint32_t C = a.C;
  uint32_t c0, c1;
  part_of(a.C, gridDim.x, blockIdx.x, &c0, &c1);
  if (blockIdx.x == 0)
    for (int k = threadIdx.x; k < a.K; k += 256) {
      const int id = a.ids[v * a.K + k];
      xe[v * a.K + k] = id >= 0 && id < a.C ? x[id] : NAN;
    }
  float m = -INFINITY, z = 0.f;
  for (uint32_t i = c0 + threadIdx.x * 4; i < c1; i += 4096) {
    float4 y[4];
    float n = m;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t c = i + u * 1024;
      y[u] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (c >= c1) continue;
      y[u] = *reinterpret_cast<const float4*>(x + c);
      if (c + 1 >= C) y[u].y = -INFINITY;
      if (c + 2 >= C) y[u].z = -INFINITY;
      if (c + 3 >= C) y[u].w = -INFINITY;
      n = fmaxf(n, fmaxf(fmaxf(y[u].x, y[u].y), fmaxf(y[u].z, y[u].w)));
    }
    const float s = n == -INFINITY ? 0.f : n;
    z *= m == n ? 1.f : exp_of(m - s, a);
#pragma unroll
    for (int u = 0; u < 4; ++u) z += (exp_of(y[u].x - s, a) + exp_of(y[u].y - s, a)) + (exp_of(y[u].z - s, a) + exp_of(y[u].w - s, a));
    m = n;
  }
  const float all = row.max(make_float2(m, 0.f)).x;
  z = m == -INFINITY ? z : z * exp_of(m - all, a);
  z = row.sum(make_float2(z, 0.f)).x;
  if (threadIdx.x == 0) part[v * FEW_PARTS + blockIdx.x] = make_float2(all, z);
}

// A row's maximum (0 where no class is possible: none) and sum, of its parts, in every lane of a wave.
__device__ __forceinline__ float2 join_parts(const DistillArgs& a, const float2* part, int parts, bool* none) {
  const Row<64> wave{nullptr};
  const int lane = threadIdx.x & 63;
  const float2 p = lane < parts ? part[lane] : make_float2(-INFINITY, 0.f);
  const float m = wave.max(p).x;
  const float z = wave.sum(make_float2(p.x == -INFINITY ? p.y : p.y * exp_of(p.x - m, a), 0.f)).x;
  *none = m == -INFINITY && z == 0.f;
  return make_float2(m == -INFINITY ? 0.f : m, z);
}

__global__ void __launch_bounds__(256) k_distill_apply(DistillArgs a, const float2* __restrict__ part, const float* __restrict__ xe, int parts, float* __restrict__ loss) {
  __shared__ int sid[HT_DISTILL_MAX_K];
  __shared__ float sq[HT_DISTILL_MAX_K];
  __shared__ float2 red[4];
  __shared__ int with[FEW_ROWS];
  __shared__ double dred[4];
  const Row<256> row{red};
  const Row<64> wv{nullptr};
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int N = count_few(a, with);
  if ((int)blockIdx.x < parts) {
    if (!a.grad) return;
    const int64_t v = blockIdx.y;
    float* g = a.grad + v * a.ld_g;
    const uint32_t C = a.C;
    uint32_t c0, c1;
    part_of(a.C, parts, blockIdx.x, &c0, &c1);
    if (!with[v]) {
      for (uint32_t c = c0 + threadIdx.x * 4; c < c1; c += 1024) *reinterpret_cast<float4*>(g + c) = zero4();
    } else {
      const float tmax = row.max(make_float2(load_entries<256>(a, v, threadIdx.x, sid, sq), 0.f)).x;
      bool none;
      const float2 j = join_parts(a, part + v * FEW_PARTS, parts, &none);
      float tz = 0.f;
      for (int k = threadIdx.x; k < a.K; k += 256)
        if (sid[k] >= 0) tz += exp_of(sq[k] - tmax, a);
      tz = row.sum(make_float2(tz, 0.f)).x;
      for (int k = threadIdx.x; k < a.K; k += 256) sq[k] = sid[k] >= 0 ? exp_of(sq[k] - tmax, a) / tz : 0.f;
      const float u = a.weight ? a.weight[v] : 1.f, w = u * a.temp * (a.mean ? 1.f / (float)N : 1.f), ip = none ? 0.f : 1.f / j.y, wp = w * ip;
      const float* x = a.x + v * a.ld;
#pragma unroll 4
      for (uint32_t c = c0 + threadIdx.x * 4; c < c1; c += 1024) {
        const float4 y = *reinterpret_cast<const float4*>(x + c);
        float4 o = make_float4(exp_of(y.x - j.x, a) * wp, exp_of(y.y - j.x, a) * wp, exp_of(y.z - j.x, a) * wp, exp_of(y.w - j.x, a) * wp);
        if (none) o = zero4();
        if (c + 1 >= C) o.y = 0.f;
        if (c + 2 >= C) o.z = 0.f;
        if (c + 3 >= C) o.w = 0.f;
        *reinterpret_cast<float4*>(g + c) = o;
      }
      __syncthreads();
      for (int k = threadIdx.x; k < a.K; k += 256)
        if (sid[k] >= 0 && (uint32_t)sid[k] >= c0 && (uint32_t)sid[k] < c1) put_entry(a, sid, sq, k, g, w, none ? 0.f : exp_of(xe[v * a.K + k] - j.x, a) * ip);
    }
  }
  if ((int)blockIdx.x < parts || blockIdx.y) return;
  // a block behind the parts: the losses, a wave a row
  double all = 0.0;
  for (int64_t v = wave; v < a.V; v += 4) {
    float l = 0.f;
    if (with[v]) {
      bool none;
      const float2 j = join_parts(a, part + v * FEW_PARTS, parts, &none);
      const float lse = none ? 0.f : a.temp * logf(j.y);
      constexpr int E = HT_DISTILL_MAX_K / 64;
      int id[E];
      float t[E], m = -INFINITY, z = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int k = e * 64 + lane;
        id[e] = k < a.K ? a.ids[v * a.K + k] : -1;
        t[e] = id[e] >= 0 ? a.top[v * a.K + k] : -INFINITY;
        if (t[e] == -INFINITY) id[e] = -1;
        m = fmaxf(m, t[e] == t[e] ? t[e] : INFINITY);
      }
      m = wv.max(make_float2(m, 0.f)).x;
#pragma unroll
      for (int e = 0; e < E; ++e) z += id[e] >= 0 ? exp_of(t[e] - m, a) : 0.f;
      z = wv.sum(make_float2(z, 0.f)).x;
      const float mq = a.temp * logf(z);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (id[e] >= 0) l += loss_term(exp_of(t[e] - m, a) / z, t[e] - m - mq, xe[v * a.K + e * 64 + lane] - j.x - lse);
      l = wv.sum(make_float2(l, 0.f)).x * a.temp;
    }
    if (lane == 0 && a.row_loss) a.row_loss[v] = l;
    if (with[v]) all += (double)(a.weight ? a.weight[v] : 1.f) * (double)l;
  }
  if (lane == 0) dred[wave] = all;
  __syncthreads();
  all = (dred[0] + dred[1]) + (dred[2] + dred[3]);
  if (threadIdx.x == 0) *loss = N > 0 ? (float)(all / (a.mean ? (double)N : 1.0)) : 0.f;
}

// f(T, NV, MORE) with the threads a row of C classes takes, and the float4s that each of them keeps
template <class F>
void with_shape(int C, F&& f) {
  auto go = [&](auto t, auto nv) { f(t, nv, std::false_type()); };
  using std::integral_constant;
  if (C <= 64) go(integral_constant<int, 16>(), integral_constant<int, 1>());
  else if (C <= 128) go(integral_constant<int, 16>(), integral_constant<int, 2>());
  else if (C <= 192) go(integral_constant<int, 16>(), integral_constant<int, 3>());
  else if (C <= 256) go(integral_constant<int, 16>(), integral_constant<int, 4>());
  else if (C <= 512) go(integral_constant<int, 64>(), integral_constant<int, 2>());
  else if (C <= 1024) go(integral_constant<int, 64>(), integral_constant<int, 4>());
  else if (C <= 4096) go(integral_constant<int, 256>(), integral_constant<int, 4>());
  else if (C <= 8192) go(integral_constant<int, 256>(), integral_constant<int, 8>());
  else if (C <= 16384) go(integral_constant<int, 1024>(), integral_constant<int, 4>());
  else if (C <= 32768) go(integral_constant<int, 1024>(), integral_constant<int, 8>());
  else if (C <= 65536) go(integral_constant<int, 1024>(), integral_constant<int, 16>());
  else f(integral_constant<int, 1024>(), integral_constant<int, 12>(), std::true_type());
}

}  // namespace

extern "C" int ht_distill_loss(ht_ctx* ctx, const ht_distill_desc* desc, const ht_tensor* logits, const int32_t* top_ids, const float* top_logits,
                               const float* row_weight, float* loss, float* row_loss, ht_tensor* dlogits) {
  if (!ctx) return HT_EINVAL;
  if (!desc || !logits || !loss) return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: null argument");
  if (desc->n_classes <= 0) return ht_set_err(ctx, HT_ESHAPE, "ht_distill_loss: number of classes must be positive");
  if (desc->k < 1 || desc->k > HT_DISTILL_MAX_K) return ht_set_err(ctx, HT_ESHAPE, "ht_distill_loss: %d entries a row, at least 1 and at most %d", desc->k, HT_DISTILL_MAX_K);
  if ((!top_ids || !top_logits) && logits->rows > 0) return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: null argument");
  // (temperature times the logarithm of a sum of up to 2^31 exponentials, below 22, is finite)
  if (!(desc->temperature > 0.f) || desc->temperature > HT_DISTILL_MAX_TEMPERATURE)
    return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: temperature must be positive and at most %g", (double)HT_DISTILL_MAX_TEMPERATURE);
  if (desc->reduction != HT_REDUCE_MEAN && desc->reduction != HT_REDUCE_SUM)
    return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: unknown reduction %d", desc->reduction);
  HT_TRY(ht_check_rows(ctx, logits, logits->rows, desc->n_classes, "ht_distill_loss: logits"));
  if (dlogits) {
    HT_TRY(ht_check_rows(ctx, dlogits, logits->rows, desc->n_classes, "ht_distill_loss: dlogits"));
    if (ht_overlap(dlogits, logits) && (dlogits->ptr != logits->ptr || dlogits->ld != logits->ld))
      return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: dlogits shares memory with logits and is not logits");
  }
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const double f2 = 1.4426950408889634074 / (double)desc->temperature;
  if (!((float)f2 < INFINITY)) return ht_set_err(ctx, HT_EINVAL, "ht_distill_loss: temperature %g is too low", (double)desc->temperature);
  const DistillArgs a{logits->ptr, logits->ld, logits->rows, desc->n_classes, top_ids, top_logits, desc->k, desc->temperature, (float)f2, (float)(f2 - (double)(float)f2),
                      row_weight, desc->reduction == HT_REDUCE_MEAN, row_loss, dlogits ? dlogits->ptr : nullptr, dlogits ? dlogits->ld : 0};
  hipStream_t st = ctx->stream;
  return ht_with_room(ctx, [&]() -> int {
    OpsBlock m;
    if (a.V >= 1 && a.V <= FEW_ROWS && a.C > FEW_CLASSES) {
      const auto part = m.add<float2>(FEW_ROWS * FEW_PARTS);
      const auto xe = m.add<float>((int64_t)FEW_ROWS * HT_DISTILL_MAX_K);
      HT_TRY(m.take(ctx));
      const int parts = (int)std::min<int64_t>(FEW_PARTS, std::max<int64_t>(ceil_div64(a.C, 4096), 1));
      const dim3 grid((unsigned)parts, (unsigned)a.V);
      k_distill_part<<<grid, 256, 0, st>>>(a, m.at(part), m.at(xe));
      HT_LAUNCH_CHECK(ctx);
      k_distill_apply<<<dim3((unsigned)parts + 1, (unsigned)a.V), 256, 0, st>>>(a, m.at(part), m.at(xe), parts, loss);
      HT_LAUNCH_CHECK(ctx);
      return HT_OK;
    }
    const auto cnt = m.add<unsigned long long>(DISTILL_COUNTS);
    const auto part = m.add<double>(DISTILL_BLOCKS);
    HT_TRY(m.take(ctx));
    const unsigned nc = (unsigned)std::max<int64_t>(1, std::min<int64_t>(DISTILL_COUNTS, ceil_div64(a.V, 256)));
    const bool few = a.V <= FEW_ROWS && a.C <= FEW_CLASSES;
    if (!few) {
      k_distill_count<<<nc, 256, 0, st>>>(a, m.at(cnt));
      HT_LAUNCH_CHECK(ctx);
    }
    unsigned nb = 1;
    with_shape(a.C, [&](auto t, auto nv, auto more) {
      constexpr int T = decltype(t)::value, B = T < 256 ? 256 : T, R = B / T;
      nb = (unsigned)std::max<int64_t>(1, std::min<int64_t>(DISTILL_BLOCKS, ceil_div64(a.V, R)));
      constexpr int NV = decltype(nv)::value;
      constexpr bool MORE = decltype(more)::value;
      if constexpr (T * NV * 4 <= FEW_CLASSES && !MORE)
        if (few) return k_distill<T, NV, MORE, true><<<nb, B, (size_t)R * a.K * 8, st>>>(a, m.at(cnt), 0, m.at(part));
      k_distill<T, NV, MORE, false><<<nb, B, (size_t)R * a.K * 8, st>>>(a, m.at(cnt), (int)nc, m.at(part));
    });
    HT_LAUNCH_CHECK(ctx);
    k_distill_loss<<<1, 256, 0, st>>>(m.at(part), (int)nb, m.at(cnt), (int)nc, a.mean, loss);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  });
}
