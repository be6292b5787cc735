// fp32 products on the fp16 matrix cores: what the operators that multiply so share.  A value is split into two fp16 numbers, x = x0 + x1 (x0 its
// rounding, x1 the rounding of what is left: |x - x0 - x1| <= 2^-22 |x|), after it was scaled by a power of two that brings the largest of what it is
// scaled with to [2^14, 2^15); x0 y0 + x0 y1 + x1 y0 are added in fp32.  Three fp16 steps take 96 clocks where an fp32 product takes 512.
#pragma once

#include "ht_internal.h"

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float V4 __attribute__((ext_vector_type(4)));
typedef float V4u __attribute__((ext_vector_type(4), aligned(4)));      // weights need no alignment

// Operands lie in fragments, what a matrix instruction reads of them: 32 rows x 16 values of the reduction of one plane (x0 or x1), 1 KiB.
// Lane l + 32 h holds row l and the values 8 (t / 4) + 4 h + t % 4, t = 0 .. 7: the order in which a lane of a product's result holds
// its rows, so that results become operands without leaving their lanes (any order will do that both operands have).  Fragment (row block,
// step, plane) is number (block * KS + step) * 2 + plane.
constexpr int FRAG = 512;
constexpr int TM = 256, TN = 128;      // tile of a block: rows of A x rows of B

__host__ __device__ constexpr int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

__device__ __forceinline__ void split2(float x, _Float16* hi, _Float16* lo) {
  *hi = (_Float16)x;
  *lo = (_Float16)(x - (float)*hi);
}

// Column `lane % 16` of four rows of 16, each 16 lanes for themselves, which name four of a row each.
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4h turned(const _Float16* p) {
  return __builtin_bit_cast(v4h, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p));
}

constexpr int KT = 2, PAIR = 32 * KT;   // steps of a stage; values of the reduction in two stages, which go together
// TURN: B is the transpose of what its fragments hold, rows of the reduction by 16s of its own rows.  A stage is 32 rows of the reduction by 128, and
// lies in LDS as in memory; ds_read_tr gives 16 lanes the columns of four rows of 16.  (Each half of a fragment starts 640 bytes after the one before, so
// that what a quarter of the lanes reads lies in other banks than what the others do.)
constexpr int TURN_HALF = 320;    // halfs
constexpr int stage_halfs(bool turn) { return turn ? TN / 16 * 4 * TURN_HALF : TN / 32 * KT * 2 * FRAG; }

}  // namespace
