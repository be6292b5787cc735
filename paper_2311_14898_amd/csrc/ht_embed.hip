// Rows of a table by id, and the table's gradient: the rows' gradients summed by id, in a fixed order (no atomics on values).
#include <type_traits>

#include "ht_internal.h"

namespace {

typedef float V4 __attribute__((ext_vector_type(4)));

// ---- H[i] = scale * table[ids[i]]: a float4 a thread and turn, rows one after the other without lanes that idle at their ends, four turns in flight.
// What bounds it is writing H.
constexpr int EMBED_TURNS = 4;
// Bytes of H from which it is written past the L2s, which hold 32 MiB and then keep the table.  Through them | past them: 232,965 rows of 301 floats of a table
// of 60 MB 82 | 57 us, 65,000 of 300 19.5 | 17.7, 35,000 11.5 | 9.7.  Less than that may still be there for whoever reads H next.
constexpr int64_t EMBED_PAST = (int64_t)32 << 20;
template <bool PAST>
__global__ void __launch_bounds__(256) k_embed(const float* __restrict__ table, int64_t ld, int64_t V, const int32_t* __restrict__ ids, int64_t n, float scale,
                                               float* __restrict__ H, int64_t ld_h, uint32_t nv) {
  // a block's first float4 as row and column, in 64 bits once; from there on 32 bits do
  const int64_t first = (int64_t)blockIdx.x * (256 * EMBED_TURNS), r0 = first / nv;
  const uint32_t c0 = (uint32_t)(first - r0 * nv) + threadIdx.x;
  int64_t row[EMBED_TURNS];
  uint32_t c[EMBED_TURNS];
  int32_t id[EMBED_TURNS];
  float4 x[EMBED_TURNS];
#pragma unroll
  for (int u = 0; u < EMBED_TURNS; ++u) {
    const uint32_t at = c0 + u * 256, r = at / nv;
    c[u] = (at - r * nv) * 4;
    row[u] = r0 + r;
    id[u] = row[u] < n ? ids[row[u]] : -1;
  }
#pragma unroll
  for (int u = 0; u < EMBED_TURNS; ++u) {
    const float no = id[u] < 0 ? 0.f : NAN;
    x[u] = make_float4(no, no, no, no);
    if (id[u] >= 0 && id[u] < V) x[u] = *reinterpret_cast<const float4*>(table + id[u] * ld + c[u]);
  }
#pragma unroll
  for (int u = 0; u < EMBED_TURNS; ++u)
    if (row[u] < n) {
      const float f = id[u] < 0 ? 0.f : scale;             // (zeros whatever the scale)
      const V4 y{x[u].x * f, x[u].y * f, x[u].z * f, x[u].w * f};
      V4* to = reinterpret_cast<V4*>(H + row[u] * ld_h + c[u]);
      if (PAST) __builtin_nontemporal_store(y, to);
      else *to = y;
    }
}

// ---- the gradient.  (id, position) pairs are sorted by id; a tile of sorted entries is summed by one group of LPR lanes, in order, and the groups of a
// block join the sums of ids that go on from tile to tile in LDS.  What begins and ends in a block is written; the rest is left, as the
// block's first or last sum, to k_embed_join, which adds it in the order of the blocks.
constexpr int GROUPS = 16;                 // of a block
constexpr int TILE = 32, TILE_FEW = 8;     // entries of a tile

// A table's rows are cleared by blocks of the launch that makes the keys (the first `key_blocks` of it), which leave the memory idle.
struct EmbedClear {
  float* p;                      // 16-byte aligned
  int64_t words;                 // (0: nothing to clear)
  __device__ __forceinline__ void run(int64_t block, int64_t blocks) const {
    const int64_t n4 = words >> 2, stride = blocks * 256;
    for (int64_t i = block * 256 + threadIdx.x; i < n4; i += stride) reinterpret_cast<float4*>(p)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (block == 0 && threadIdx.x < (words & 3)) p[n4 * 4 + threadIdx.x] = 0.f;
  }
};
__device__ __forceinline__ uint64_t embed_key(const int32_t* ids, int64_t i, int64_t V) {      // (ids of no row: behind the others)
  const int32_t id = ids[i];
  return (uint64_t)(id >= 0 && id < V ? (uint32_t)id : (uint32_t)V) << 32 | (uint32_t)i;
}
__global__ void __launch_bounds__(256) k_embed_keys(const int32_t* __restrict__ ids, int64_t n, int64_t V, uint64_t* __restrict__ keys, unsigned key_blocks,
                                                    EmbedClear clear) {
  if (blockIdx.x >= key_blocks) return clear.run(blockIdx.x - key_blocks, gridDim.x - key_blocks);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) keys[i] = embed_key(ids, i, V);
}
// Few entries are put in order in the same launch: an entry's place is the number of entries before it, which it counts.  us, counted | sorted: 6,000 entries
// of 1,000 ids 27 | 32, 10,000 of 131,000 56 | 67, 16,000 of either 95 | 37 and 126 | 68.
constexpr int EMBED_FEW = 8192;
__global__ void __launch_bounds__(256) k_embed_rank(const int32_t* __restrict__ ids, int n, int64_t V, uint64_t* __restrict__ keys, unsigned key_blocks,
                                                    EmbedClear clear) {
  if (blockIdx.x >= key_blocks) return clear.run(blockIdx.x - key_blocks, gridDim.x - key_blocks);
  // 16 lanes an entry, each compares with every 16th four of the others
  extern __shared__ __attribute__((aligned(16))) uint32_t sh[];      // [n, up to the next 4]
  const int n4 = (n + 3) / 4;
  for (int i = threadIdx.x; i < n4 * 4; i += 256) sh[i] = i < n ? (uint32_t)(embed_key(ids, i, V) >> 32) : 0xffffffffu;
  __syncthreads();
  const int l = threadIdx.x & 15, i = blockIdx.x * 16 + (threadIdx.x >> 4);
  const uint32_t mine = i < n ? sh[i] : 0;
  int before = 0;
  for (int q = l; q < n4; q += 16) {
    const uint4 x = *reinterpret_cast<const uint4*>(sh + q * 4);
    const int j = q * 4;
    before += (x.x < mine || (x.x == mine && j < i)) + (x.y < mine || (x.y == mine && j + 1 < i)) + (x.z < mine || (x.z == mine && j + 2 < i)) +
              (x.w < mine || (x.w == mine && j + 3 < i));
  }
  for (int o = 8; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
  if (l == 0 && i < n) keys[before] = (uint64_t)mine << 32 | (uint32_t)i;
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

// edge: [block][first, last][nv]
template <int LPR, int TS>
__global__ void __launch_bounds__(LPR * GROUPS) k_embed_sum(const uint64_t* __restrict__ keys, int64_t n, const float* __restrict__ dH, int64_t ld_h, EmbedOut out,
                                                            float4* __restrict__ edge) {
  constexpr int B = LPR * GROUPS, E = GROUPS * TS, U = 8;
  __shared__ uint32_t id[E + 2], pos[E];   // id[e + 1]: of entry e; before and behind them their neighbours
  __shared__ float4 sums[GROUPS][LPR][2];  // of a tile's first run where it has begun before, of its last where it goes on
  const int64_t e0 = (int64_t)blockIdx.x * E;
  const int here = n - e0 < E ? (int)(n - e0) : E;
  constexpr uint32_t NONE = 0xffffffffu;   // (no id: ids are below 2^31)
  for (int e = (int)threadIdx.x - 1; e < E + 1; e += B) {
    const int64_t p = e0 + e;
    const uint64_t k = p >= 0 && p < n ? keys[p] : (uint64_t)NONE << 32;
    id[e + 1] = (uint32_t)(k >> 32);
    if (e >= 0 && e < E) pos[e] = (uint32_t)k;
  }
  __syncthreads();
  const int g = threadIdx.x / LPR, l = threadIdx.x % LPR, c = blockIdx.y * LPR + l;
  const int a = g * TS, b = a + TS < here ? a + TS : here;
  const bool works = a < here && c < out.nv;
  if (works) {
    bool first = id[a + 1] == id[a];       // the run has begun before this tile
    uint32_t t = id[a + 1];
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    auto end = [&](bool last) {
      if (first) sums[g][l][0] = s;
      else if (last) sums[g][l][1] = s;
      else out.put(t, c, s);
      first = false;
    };
    for (int e = a; e < b; e += U) {
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const float4*>(dH + (int64_t)pos[e + u < b ? e + u : b - 1] * ld_h + c * 4);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (e + u >= b) break;
        const uint32_t i = id[e + u + 1];
        if (i != t) {
          end(false);
          t = i;
          s = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        s.x += x[u].x, s.y += x[u].y, s.z += x[u].z, s.w += x[u].w;
      }
    }
    end(id[b + 1] == t);
  }
  __syncthreads();
  if (!works) return;
  auto goes_on = [&](int k) {              // tile k's last run does
    const int z = (k + 1) * TS < here ? (k + 1) * TS : here;
    return id[z] == id[z + 1];
  };
  auto one_run = [&](int k) {
    const int z = (k + 1) * TS < here ? (k + 1) * TS : here;
    return id[k * TS + 1] == id[z];
  };
  // the sum from tile k's first run on, until the run ends; true: in this block
  auto follow = [&](int k, float4* s) {
    for (; k * TS < here; ++k) {
      const float4 x = sums[k][l][0];
      s->x += x.x, s->y += x.y, s->z += x.z, s->w += x.w;
      if (!one_run(k) || !goes_on(k)) return true;
    }
    return false;
  };
  const bool begun = id[a + 1] == id[a];
  if (g == 0 && begun) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    (void)follow(0, &s);
    edge[(int64_t)blockIdx.x * 2 * out.nv + c] = s;
  }
  if (goes_on(g) && !(begun && one_run(g))) {
    float4 s = sums[g][l][1];
    if (follow(g + 1, &s)) out.put(id[b], c, s);
    else edge[((int64_t)blockIdx.x * 2 + 1) * out.nv + c] = s;
  }
}

// A block each: if a run begins in block `blockIdx.x` of k_embed_sum's (E entries each) and goes on, its last sum and the first ones of those that the run reaches.
template <int LPR>
__global__ void __launch_bounds__(256) k_embed_join(const uint64_t* __restrict__ keys, int64_t n, int E, EmbedOut out, const float4* __restrict__ edge) {
  constexpr int G = 256 / LPR;
  __shared__ float4 sh[256];
  const int64_t block = blockIdx.x, p0 = block * E, p1 = p0 + E;
  const uint32_t id = (uint32_t)(keys[p1 - 1] >> 32);
  if ((uint32_t)(keys[p1] >> 32) != id) return;
  if (p0 > 0 && (uint32_t)(keys[p0 - 1] >> 32) == id) return;       // (sorted: the run has begun before)
  // the last block that the run reaches, by bisection over the blocks' first entries
  int64_t lo = block + 1, hi = (n + E - 1) / E;
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if ((uint32_t)(keys[mid * E] >> 32) == id) lo = mid;
    else hi = mid;
  }
  const int64_t m = lo - block;
  const int g = threadIdx.x / LPR;
  for (int c0 = 0; c0 < out.nv; c0 += LPR) {
    const int c = c0 + threadIdx.x % LPR;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < out.nv) {
      if (g == 0) s = edge[(block * 2 + 1) * out.nv + c];
      const int64_t a = m * g / G, b = m * (g + 1) / G;
#pragma unroll 8
      for (int64_t t = a; t < b; ++t) {
        const float4 x = edge[((block + 1 + t) * 2) * out.nv + c];
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

// Very few entries, all in one launch: a block an entry and 64 float4s of it.  The first entry of an id adds up all of them, each wave those in its share of the
// positions, in order; other blocks clear the rows that none has.  us, so | in order first (three launches): 1,000
// entries of 10,000 ids x 64 7.2 | 13.0, 500 of 131,072 x 256 19 | 29, 1 of 10,000 x 64 7.9 | 11.0, 1,000 of one id 12.5 | 12.6; 2,000 of 10,000 would take 12 | 16, of one id a chain of twice the rows.
constexpr int EMBED_ONCE = 1024, ONCE_ROWS = 1024, ONCE_PARTS = 16, ONCE_WAVES = 8;          // entries; rows that a block clears at a time
__global__ void __launch_bounds__(ONCE_WAVES * 64) k_embed_once(const int32_t* __restrict__ ids, int n, const float* __restrict__ dH, int64_t ld_h, EmbedOut out, unsigned col_blocks) {
  __shared__ int32_t sid[EMBED_ONCE];
  __shared__ uint32_t there[ONCE_ROWS / 32];
  __shared__ float4 sums[ONCE_WAVES][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned sum_blocks = n * col_blocks;
  for (int i = threadIdx.x; i < EMBED_ONCE; i += ONCE_WAVES * 64) sid[i] = i < n ? ids[i] : -1;
  if (blockIdx.x >= sum_blocks) {
    // ONCE_PARTS blocks clear the same ONCE_ROWS rows
    const uint32_t block = (blockIdx.x - sum_blocks) / ONCE_PARTS, part = (blockIdx.x - sum_blocks) % ONCE_PARTS, blocks = (gridDim.x - sum_blocks) / ONCE_PARTS;
    const uint32_t nv = out.nv;
    for (int64_t r0 = (int64_t)block * ONCE_ROWS; r0 < out.V; r0 += (int64_t)blocks * ONCE_ROWS) {
      const int rows = out.V - r0 < ONCE_ROWS ? (int)(out.V - r0) : ONCE_ROWS;
      __syncthreads();
      for (int i = threadIdx.x; i < ONCE_ROWS / 32; i += ONCE_WAVES * 64) there[i] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += ONCE_WAVES * 64) {
        const int64_t r = sid[i] - r0;
        if (sid[i] >= 0 && r >= 0 && r < rows) atomicOr(&there[r >> 5], 1u << (r & 31));
      }
      __syncthreads();
      const uint32_t per = (rows + ONCE_PARTS - 1) / ONCE_PARTS, r1 = part * per, r2 = r1 + per < (uint32_t)rows ? r1 + per : rows;
      // (rows one after the other without lanes that idle at their ends)
      uint32_t r = r1 + threadIdx.x / nv, c = threadIdx.x % nv;
      for (const uint32_t dr = ONCE_WAVES * 64 / nv, dc = ONCE_WAVES * 64 % nv; r < r2;) {
        if (!((there[r >> 5] >> (r & 31)) & 1)) *reinterpret_cast<float4*>(out.dT + (r0 + r) * out.ld + c * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
        r += dr, c += dc;
        if (c >= nv) c -= nv, ++r;
      }
    }
    return;
  }
  __syncthreads();
  const int e = blockIdx.x / col_blocks, id = __builtin_amdgcn_readfirstlane(sid[e]);
  if (id < 0 || id >= out.V) return;
  constexpr int K = EMBED_ONCE / (ONCE_WAVES * 64);      // sets of 64 positions of a wave: every ONCE_WAVES-th
  bool first = true;
  for (int k = 0; k * 64 < e; ++k) {
    const int i = k * 64 + lane;
    first = first && !__ballot(i < e && sid[i] == id);
  }
  if (!first) return;
  uint64_t same[K];
#pragma unroll
  for (int k = 0; k < K; ++k) same[k] = __ballot(sid[(k * ONCE_WAVES + wave) * 64 + lane] == id);
  for (int c0 = blockIdx.x % col_blocks * 64; c0 < out.nv; c0 += col_blocks * 64) {
    const int c = c0 + lane < out.nv ? c0 + lane : out.nv - 1;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      uint64_t left = same[k];
      while (left) {
        constexpr int U = 8;
        float4 x[U];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          at[u] = left ? (k * ONCE_WAVES + wave) * 64 + __builtin_ctzll(left) : -1;
          left &= left - 1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const float4*>(dH + (at[u] < 0 ? at[0] : at[u]) * ld_h + c * 4);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (at[u] >= 0) s.x += x[u].x, s.y += x[u].y, s.z += x[u].z, s.w += x[u].w;
      }
    }
    __syncthreads();
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c0 + lane < out.nv) {
      for (int w = 1; w < ONCE_WAVES; ++w) {
        const float4 x = sums[w][lane];
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
  const int64_t nv = ceil_div64(table->cols, 4), n = H->rows;
  if (n == 0) return HT_OK;
  const bool past = n * nv * 16 >= EMBED_PAST;
  // (a launch takes less than 2^32 threads)
  return ht_in_launches(n, std::max<int64_t>(1, HT_LAUNCH_WAVES * 64 * EMBED_TURNS / nv), [&](int64_t i, int64_t m) {
    const unsigned blocks = (unsigned)ceil_div64(m * nv, 256 * EMBED_TURNS);
    float* to = H->ptr + i * H->ld;
    if (past) k_embed<true><<<blocks, 256, 0, ctx->stream>>>(table->ptr, table->ld, table->rows, ids + i, m, scale, to, H->ld, (uint32_t)nv);
    else k_embed<false><<<blocks, 256, 0, ctx->stream>>>(table->ptr, table->ld, table->rows, ids + i, m, scale, to, H->ld, (uint32_t)nv);
    HT_LAUNCH_CHECK(ctx);
    return (int)HT_OK;
  });
}

extern "C" int ht_embed_bwd(ht_ctx* ctx, const ht_tensor* dH, const int32_t* ids, float scale, int32_t accumulate, ht_tensor* dT) {
  if (!ctx) return HT_EINVAL;
  if (!dT || !dH || (!ids && dH->rows > 0)) return ht_set_err(ctx, HT_EINVAL, "ht_embed_bwd: null argument");
  if (dT->cols <= 0) return ht_set_err(ctx, HT_ESHAPE, "ht_embed_bwd: width must be positive");
  HT_TRY(ht_check_rows(ctx, dT, dT->rows, dT->cols, "ht_embed_bwd: d_table"));
  HT_TRY(ht_check_rows(ctx, dH, dH->rows, dT->cols, "ht_embed_bwd: dH"));
  if (ht_overlap(dH, dT)) return ht_set_err(ctx, HT_EINVAL, "ht_embed_bwd: d_table shares memory with dH");
  HT_HIP(ctx, hipSetDevice(ctx->device));
  const int nv = (int)ceil_div64(dT->cols, 4);
  const int64_t n = dH->rows, V = dT->rows;
  if (n > EMBED_ONCE && ceil_div64(nv, 64) > 65535) return ht_set_err(ctx, HT_ESHAPE, "ht_embed_bwd: %d columns are too many for %lld entries", dT->cols, (long long)n);      // (of a grid)
  int bits = 1;
  while (((int64_t)1 << bits) <= V) ++bits;
  const EmbedOut out{dT->ptr, dT->ld, V, scale, accumulate, nv};
  if (n <= EMBED_ONCE) {
    if (V == 0 || (n == 0 && accumulate)) return HT_OK;
    const unsigned col_blocks = (unsigned)std::min(16, (nv + 63) / 64), clear_blocks = accumulate ? 0 : ONCE_PARTS * (unsigned)std::min<int64_t>(ceil_div64(V, ONCE_ROWS), 4096);
    k_embed_once<<<(unsigned)n * col_blocks + clear_blocks, ONCE_WAVES * 64, 0, ctx->stream>>>(ids, (int)n, dH->ptr, dH->ld, out, col_blocks);
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  }
  return ht_with_room(ctx, [&]() -> int {
    OpsBlock m;
    const bool few = n <= EMBED_FEW;
    const auto keys = m.add<uint64_t>(n), tmp = m.add<uint64_t>(few ? 0 : n);
    const int E = GROUPS * (few ? TILE_FEW : TILE);
    const int64_t blocks = ceil_div64(n, E);
    const auto edge = m.add<float4>(blocks * 2 * nv);
    size_t rsort = 0, scan = 0;
    if (!few) ht_radix_wants(n, &rsort, &scan);
    HT_TRY(m.take(ctx, rsort, scan));
    const EmbedClear clear{dT->ptr, accumulate || V == 0 ? 0 : (V - 1) * dT->ld + dT->cols};
    const unsigned key_blocks = (unsigned)ceil_div64(n, few ? 16 : 256), clear_blocks = (unsigned)std::min<int64_t>(ceil_div64(clear.words, 1024), 4096);
    uint64_t* sorted = m.at(keys);
    if (few) k_embed_rank<<<key_blocks + clear_blocks, 256, (size_t)ceil_div64(n, 4) * 16, ctx->stream>>>(ids, (int)n, V, m.at(keys), key_blocks, clear);
    else k_embed_keys<<<key_blocks + clear_blocks, 256, 0, ctx->stream>>>(ids, n, V, m.at(keys), key_blocks, clear);
    HT_LAUNCH_CHECK(ctx);
    if (V == 0) return HT_OK;
    if (!few) HT_TRY(ht_radix_sort_u64(ctx, m.at(keys), m.at(tmp), n, 32, 32 + bits, &sorted));
    with_lanes(nv, [&](auto lanes) {
      constexpr int LPR = decltype(lanes)::value;
      const dim3 grid((unsigned)blocks, (unsigned)((nv + LPR - 1) / LPR));
      if (few) k_embed_sum<LPR, TILE_FEW><<<grid, LPR * GROUPS, 0, ctx->stream>>>(sorted, n, dH->ptr, dH->ld, out, m.at(edge));
      else k_embed_sum<LPR, TILE><<<grid, LPR * GROUPS, 0, ctx->stream>>>(sorted, n, dH->ptr, dH->ld, out, m.at(edge));
      if (blocks > 1) k_embed_join<LPR><<<(unsigned)(blocks - 1), 256, 0, ctx->stream>>>(sorted, n, E, out, m.at(edge));
    });
    HT_LAUNCH_CHECK(ctx);
    return HT_OK;
  });
}
