// Rows grouped by what they chose (flexq_group_rows, flexq_route): how kernels walk them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

struct RowGroup {
    int id, begin, end;   // rows begin .. end - 1 of the order; id < 0: there is none
    int tile;             // number of the piece within the group
};

// Piece number `index`, counting `height` rows of a group at a time (height 0: a group is one piece),
// over groups 0 .. count - 1 and, with `rest`, the rows without a group as group `count`; every
// wavefront finds it for itself, 64 groups a step.  `pieces` (may be null) receives the number of
// pieces in all.  Rows outside 0 .. rows - 1 are never named, whatever the offsets hold.
__device__ __forceinline__ RowGroup find_piece(const int32_t *offsets, int count, int rows, int height, int index,
                                               bool rest = false, int *pieces = nullptr)
{
    const int lane = threadIdx.x & 63, last = rest ? count : count - 1;
    RowGroup g = {-1, 0, 0, 0};
    int before = 0;
    for (int e0 = 0; e0 <= last; e0 += 64) {
        const int e = e0 + lane;
        int begin = 0, end = 0;
        if (e <= last) {
            begin = min(max(offsets[e], 0), rows);
            end = e == count ? rows : min(max(offsets[e + 1], begin), rows);
        }
        const int mine = height == 0 ? (end > begin ? 1 : 0) : (end - begin + height - 1) / height;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d, 64);
            if (lane >= d) sum += up;
        }
        const int first = before + sum - mine;
        const unsigned long long hit = __ballot(index >= first && index < first + mine);
        if (hit) {
            const int l = __ffsll(hit) - 1;
            g.id = e0 + l;
            g.begin = __builtin_amdgcn_readlane(begin, l);
            g.end = __builtin_amdgcn_readlane(end, l);
            g.tile = index - __builtin_amdgcn_readlane(first, l);
        }
        before += __builtin_amdgcn_readlane(sum, 63);
        if (hit && !pieces) break;
    }
    if (pieces) *pieces = before;
    return g;
}

}  // namespace
