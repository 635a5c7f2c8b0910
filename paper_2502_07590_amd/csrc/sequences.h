// Sequences packed one behind another by cumulative lengths: which one a tile of rows, or a token, belongs to.
#pragma once

#include "common.h"

namespace dsv {

// Tiles of ROWS rows are numbered without a sum over the sequences before: sequence i's begin at floor(cu[i] * mul / ROWS) + i, which leaves
// ceil(length / ROWS) places at least.  The owner of a place is the last sequence that begins at or before it; 64 candidates a step.
// ROWS = 0: the tokens themselves, no place left empty (the owner of a token).  gap: places more for every sequence instead of one.
__device__ __forceinline__ int first_slot(int cu, int total, int mul, int rows, int i)
{
    const int at = min(max(cu, 0), total) * mul;
    return rows ? (int)((uint32_t)at / (uint32_t)rows) + i : at;
}
__device__ __forceinline__ int find_sequence(const int32_t *__restrict__ cu, int n_seq, int total, int mul, int rows, int slot, int gap = 1)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n_seq;  // lo begins at or before the slot, hi after it
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, at = lo + (lane + 1) * step;
        const bool before = at < hi && first_slot(cu[at], total, mul, rows, at * gap) <= slot;
        lo += __popcll(__ballot(before)) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}
__host__ __device__ __forceinline__ int64_t tile_slots(int64_t total, int mul, int rows, int n_seq) { return total * mul / rows + n_seq; }

}  // namespace dsv
