// Rows of a table by id, and the table's gradient: the rows' gradients summed by id, in a fixed order (no atomics on values).
#include <type_traits>

#include "ht_internal.h"

namespace {

// ---- H[i] = scale * table[ids[i]]: LPR lanes a row, a float4 each, four rows of a group at once.
template <int LPR>
__global__ void __launch_bounds__(256) k_embed(const float* __restrict__ table, int64_t ld, int64_t V, const int32_t* __restrict__ ids, int64_t n, float scale,
                                               float* __restrict__ H, int64_t ld_h, int nv) {
  constexpr int U = 4, G = 256 / LPR;
  const int l = threadIdx.x % LPR;
  const int64_t i0 = ((int64_t)blockIdx.x * G + threadIdx.x / LPR) * U;
  int32_t id[U];
#pragma unroll
  for (int u = 0; u < U; ++u) id[u] = i0 + u < n ? ids[i0 + u] : -1;
  for (int c = l; c < nv; c += LPR) {
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float no = id[u] < 0 ? 0.f : NAN;
      x[u] = make_float4(no, no, no, no);
      if (id[u] >= 0 && id[u] < V) x[u] = *reinterpret_cast<const float4*>(table + id[u] * ld + c * 4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u < n) *reinterpret_cast<float4*>(H + (i0 + u) * ld_h + c * 4) = make_float4(x[u].x * scale, x[u].y * scale, x[u].z * scale, x[u].w * scale);
  }
}

// ---- the gradient.  (id, position) pairs are sorted by id; a tile of TS sorted entries is summed by one group of lanes, in order.  What begins and ends
// in a tile is written; the sums of an id that goes on into other tiles are left, as the tile's first or last, to k_embed_join, which adds
// them in the order of the tiles.
constexpr int TS = 32;

__global__ void __launch_bounds__(256) k_embed_keys(const int32_t* __restrict__ ids, int64_t n, int64_t V, uint64_t* __restrict__ keys) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int32_t id = ids[i];
  keys[i] = (uint64_t)(id >= 0 && id < V ? (uint32_t)id : (uint32_t)V) << 32 | (uint32_t)i;      // (ids of no row: behind the others)
}

struct EmbedOut {
  float* dT;
  int64_t ld, V;
  float scale;
  int add, nv;
  __device__ __forceinline__ void put(uint32_t id, int c, float4 s) const {
    if (id >= (uint32_t)V) return;
    float4* o = reinterpret_cast<float4*>(dT + id * ld + c * 4);
    const float4 was = add ? *o : make_float4(0.f, 0.f, 0.f, 0.f);
    *o = make_float4(was.x + scale * s.x, was.y + scale * s.y, was.z + scale * s.z, was.w + scale * s.w);
  }
};

// edge: [tile][first, last][4 nv] floats
template <int LPR>
__global__ void __launch_bounds__(256) k_embed_sum(const uint64_t* __restrict__ keys, int64_t n, const float* __restrict__ dH, int64_t ld_h, EmbedOut out,
                                                   float4* __restrict__ edge) {
  constexpr int G = 256 / LPR, U = 8;
  const int64_t tile = (int64_t)blockIdx.x * G + threadIdx.x / LPR, p0 = tile * TS;
  const int c = blockIdx.y * LPR + threadIdx.x % LPR;
  if (p0 >= n || c >= out.nv) return;
  const int64_t p1 = p0 + TS < n ? p0 + TS : n;
  const bool goes_on = p1 < n && (uint32_t)(keys[p1] >> 32) == (uint32_t)(keys[p1 - 1] >> 32);
  bool first = p0 > 0 && (uint32_t)(keys[p0 - 1] >> 32) == (uint32_t)(keys[p0] >> 32);      // the run has begun before this tile
  uint32_t id = (uint32_t)(keys[p0] >> 32);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  auto end = [&](bool last) {
    if (first) edge[(tile * 2) * out.nv + c] = s;
    else if (last) edge[(tile * 2 + 1) * out.nv + c] = s;
    else out.put(id, c, s);
    first = false;
  };
  for (int64_t p = p0; p < p1; p += U) {
    uint64_t k[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = keys[p + u < p1 ? p + u : p1 - 1];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const float4*>(dH + (int64_t)(uint32_t)k[u] * ld_h + c * 4);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u >= p1) break;
      const uint32_t t = (uint32_t)(k[u] >> 32);
      if (t != id) {
        end(false);
        id = t;
        s = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      s.x += x[u].x, s.y += x[u].y, s.z += x[u].z, s.w += x[u].w;
    }
  }
  end(goes_on);
}

// A block a tile: if a run begins in it and goes on, its last sum and the first ones of the tiles that the run reaches.
template <int LPR>
__global__ void __launch_bounds__(256) k_embed_join(const uint64_t* __restrict__ keys, int64_t n, EmbedOut out, const float4* __restrict__ edge) {
  constexpr int G = 256 / LPR;
  __shared__ float4 sh[256];
  const int64_t tile = blockIdx.x, p0 = tile * TS, p1 = p0 + TS;
  if (p1 >= n) return;
  const uint32_t id = (uint32_t)(keys[p1 - 1] >> 32);
  if ((uint32_t)(keys[p1] >> 32) != id) return;
  if (p0 > 0 && (uint32_t)(keys[p0 - 1] >> 32) == id) return;       // (sorted: the run has begun before)
  // the run's end, by bisection over the tiles' first entries, then the tiles after this one that it reaches
  int64_t lo = tile + 1, hi = (n + TS - 1) / TS;
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if ((uint32_t)(keys[mid * TS] >> 32) == id) lo = mid;
    else hi = mid;
  }
  const int64_t m = lo - tile;
  const int g = threadIdx.x / LPR;
  for (int c0 = 0; c0 < out.nv; c0 += LPR) {
    const int c = c0 + threadIdx.x % LPR;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < out.nv) {
      if (g == 0) s = edge[(tile * 2 + 1) * out.nv + c];
      const int64_t a = m * g / G, b = m * (g + 1) / G;
#pragma unroll 8
      for (int64_t t = a; t < b; ++t) {
        const float4 x = edge[((tile + 1 + t) * 2) * out.nv + c];
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
      }
    }
    __syncthreads();
    sh[threadIdx.x] = s;
    __syncthreads();
    if (g == 0 && c < out.nv) {
      for (int k = 1; k < G; ++k) {
        const float4 x = sh[k * LPR + threadIdx.x];
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
      }
      out.put(id, c, s);
    }
  }
}

// f(LPR) with the lanes that a row of nv float4s takes
template <class F>
void with_lanes(int nv, F&& f) {
  if (nv <= 4) f(std::integral_constant<int, 4>());
  else if (nv <= 8) f(std::integral_constant<int, 8>());
  else if (nv <= 16) f(std::integral_constant<int, 16>());
  else if (nv <= 32) f(std::integral_constant<int, 32>());
  else f(std::integral_constant<int, 64>());
}

}  // namespace

extern "C" int ht_embed_fwd(ht_ctx* ctx, const ht_tensor* table, const int32_t* ids, float scale, ht_tensor* H) {
  if (!ctx) return HT_EINVAL;
  if (!table || !H || (!ids && H->rows > 0)) return ht_set_err(ctx, HT_EINVAL, "ht_embed_fwd: null argument");
  if (table->cols <= 0) return ht_set_err(ctx, HT_ESHAPE, "ht_embed_fwd: width must be positive");
  HT_TRY(ht_check_rows(ctx, table, table->rows, table->cols, "ht_embed_fwd: table"));
  HT_TRY(ht_check_rows(ctx, H, H->rows, table->cols, "ht_embed_fwd: H"));
  if (ht_overlap(H, table)) return ht_set_err(ctx, HT_EINVAL, "ht_embed_fwd: H shares memory with table");
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const int nv = (table->cols + 3) / 4;
  const int64_t n = H->rows;
  with_lanes(nv, [&](auto lanes) {
    constexpr int LPR = decltype(lanes)::value;
    const int64_t rows = 256 / LPR * 4;
    if (n > 0)
      k_embed<LPR><<<(unsigned)ceil_div64(n, rows), 256, 0, ctx->stream>>>(table->ptr, table->ld, table->rows, ids, n, scale, H->ptr, H->ld, nv);
  });
  HT_LAUNCH_CHECK(ctx);
  return HT_OK;
}

extern "C" int ht_embed_bwd(ht_ctx* ctx, const ht_tensor* dH, const int32_t* ids, float scale, int32_t accumulate, ht_tensor* dT) {
  if (!ctx) return HT_EINVAL;
  if (!dT || !dH || (!ids && dH->rows > 0)) return ht_set_err(ctx, HT_EINVAL, "ht_embed_bwd: null argument");
  if (dT->cols <= 0) return ht_set_err(ctx, HT_ESHAPE, "ht_embed_bwd: width must be positive");
  HT_TRY(ht_check_rows(ctx, dT, dT->rows, dT->cols, "ht_embed_bwd: d_table"));
  HT_TRY(ht_check_rows(ctx, dH, dH->rows, dT->cols, "ht_embed_bwd: dH"));
  if (ht_overlap(dH, dT)) return ht_set_err(ctx, HT_EINVAL, "ht_embed_bwd: d_table shares memory with dH");
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const int nv = (dT->cols + 3) / 4;
  const int64_t n = dH->rows, V = dT->rows, tiles = ceil_div64(n, TS);
  int bits = 1;
  while (((int64_t)1 << bits) <= V) ++bits;
  return ht_with_room(ctx, [&]() -> int {
    OpsBlock m;
    const auto keys = m.add<uint64_t>(n), tmp = m.add<uint64_t>(n);
    const auto edge = m.add<float4>(tiles * 2 * nv);
    size_t rsort = 0, scan = 0;
    ht_radix_wants(n, &rsort, &scan);
    HT_TRY(m.take(ctx, rsort, scan));
    if (!accumulate && V > 0) HT_TRY(ht_fill_zero(ctx, ctx->stream, dT->ptr, (size_t)((V - 1) * dT->ld + dT->cols) * 4));
    if (n == 0 || V == 0) return HT_OK;
    k_embed_keys<<<(unsigned)ceil_div64(n, 256), 256, 0, ctx->stream>>>(ids, n, V, m.at(keys));
    HT_LAUNCH_CHECK(ctx);
    uint64_t* sorted = nullptr;
    HT_TRY(ht_radix_sort_u64(ctx, m.at(keys), m.at(tmp), n, 32, 32 + bits, &sorted));
    const EmbedOut out{dT->ptr, dT->ld, V, scale, accumulate, nv};
    with_lanes(nv, [&](auto lanes) {
      constexpr int LPR = decltype(lanes)::value;
      k_embed_sum<LPR><<<dim3((unsigned)ceil_div64(tiles, 256 / LPR), (unsigned)((nv + LPR - 1) / LPR)), 256, 0, ctx->stream>>>(sorted, n, dH->ptr, dH->ld, out,
                                                                                                                            m.at(edge));
      if (tiles > 1) k_embed_join<LPR><<<(unsigned)tiles, 256, 0, ctx->stream>>>(sorted, n, out, m.at(edge));
    });
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  });
}
