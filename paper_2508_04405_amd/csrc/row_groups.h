// Rows grouped by what they chose (flexq_group_rows, flexq_route): how kernels walk them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

struct RowGroup {
    int id, begin, end;   // rows begin .. end - 1 of the order; id < 0: there is none
    int tile;             // number of the piece within the group
};

// Sum over the lanes before this one and itself: DPP shifts within rows of 16, then the rows' totals.
__device__ __forceinline__ int wave_scan(int v)
{
#define FLEXQ_ADD(ctrl, rows, banks) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, banks, true)
    FLEXQ_ADD(0x111, 0xf, 0xf);          // row_shr:1, 2, 4, 8
    FLEXQ_ADD(0x112, 0xf, 0xf);
    FLEXQ_ADD(0x114, 0xf, 0xf);
    FLEXQ_ADD(0x118, 0xf, 0xf);
#undef FLEXQ_ADD
    const int lane = threadIdx.x & 63;
    const int t0 = __builtin_amdgcn_readlane(v, 15), t1 = __builtin_amdgcn_readlane(v, 31), t2 = __builtin_amdgcn_readlane(v, 47);
    return v + (lane >= 16 ? t0 : 0) + (lane >= 32 ? t1 : 0) + (lane >= 48 ? t2 : 0);
}

// Begin and end of group e (of `rest` rows without one: e == count), empty beyond the last.  Rows outside
// 0 .. rows - 1 are never named, whatever the offsets hold.
__device__ __forceinline__ int2 group_rows_of(const int32_t *offsets, int count, int rows, int e, int last)
{
    if (e > last) return make_int2(0, 0);
    const int begin = min(max(offsets[e], 0), rows);
    return make_int2(begin, e == count ? rows : min(max(offsets[e + 1], begin), rows));
}

// Pieces of at most `height` rows of groups 0 .. count - 1, each group cut by itself.
__device__ __forceinline__ int count_pieces(const int32_t *offsets, int count, int rows, int height)
{
    int mine = 0;
    for (int e = threadIdx.x & 63; e < count; e += 64) {
        const int2 r = group_rows_of(offsets, count, rows, e, count - 1);
        mine += (r.y - r.x + height - 1) / height;
    }
    return __builtin_amdgcn_readlane(wave_scan(mine), 63);
}

// Piece number `index` of those (height 0: a group is one piece), with `rest` the rows without a group as
// group `count`; every wavefront finds it for itself, 64 groups a step.
__device__ __forceinline__ RowGroup find_piece(const int32_t *offsets, int count, int rows, int height, int index,
                                               bool rest = false)
{
    const int lane = threadIdx.x & 63, last = rest ? count : count - 1;
    RowGroup g = {-1, 0, 0, 0};
    int before = 0;
    for (int e0 = 0; e0 <= last; e0 += 64) {
        const int2 r = group_rows_of(offsets, count, rows, e0 + lane, last);
        const int mine = height == 0 ? (r.y > r.x ? 1 : 0) : (r.y - r.x + height - 1) / height;
        const int sum = wave_scan(mine), first = before + sum - mine;
        const unsigned long long hit = __ballot(index >= first && index < first + mine);
        if (hit) {
            const int l = __ffsll(hit) - 1;
            g.id = e0 + l;
            g.begin = __builtin_amdgcn_readlane(r.x, l);
            g.end = __builtin_amdgcn_readlane(r.y, l);
            g.tile = index - __builtin_amdgcn_readlane(first, l);
            break;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return g;
}

// Tiles of HIGH rows of a group of n rows, a last one of more than half of that among them (phase 0); the last
// one where it holds no more than half (phase 1).  offsets: all of them, in order, within the rows.
template <int HIGH>
__device__ __forceinline__ int parts_of(int n, int phase)
{
    const int rest = n % HIGH;
    return phase == 0 ? n / HIGH + (rest > HIGH / 2 ? 1 : 0) : (rest > 0 && rest <= HIGH / 2 ? 1 : 0);
}

template <int HIGH>
__device__ __forceinline__ int count_parts(const int *offsets, int count, int phase)
{
    int mine = 0;
    for (int e = threadIdx.x & 63; e < count; e += 64) mine += parts_of<HIGH>(max(offsets[e + 1] - offsets[e], 0), phase);
    return __builtin_amdgcn_readlane(wave_scan(mine), 63);
}

// Number `index` of those: its group, its first row and the group's end.
template <int HIGH>
__device__ __forceinline__ RowGroup find_part(const int *offsets, int count, int phase, int index)
{
    const int lane = threadIdx.x & 63;
    RowGroup g = {0, 0, 1, 0};
    int before = 0;
    for (int e0 = 0; e0 < count; e0 += 64) {
        const int e = min(e0 + lane, count - 1), begin = offsets[e], end = max(offsets[e + 1], begin);
        const int mine = e0 + lane < count ? parts_of<HIGH>(end - begin, phase) : 0;
        const int sum = wave_scan(mine), first = before + sum - mine;
        const unsigned long long hit = __ballot(index >= first && index < first + mine);
        if (hit) {
            const int l = __ffsll(hit) - 1;
            g.id = e0 + l;
            g.end = __builtin_amdgcn_readlane(end, l);
            g.tile = index - __builtin_amdgcn_readlane(first, l);
            const int at = __builtin_amdgcn_readlane(begin, l);
            g.begin = at + (phase == 0 ? g.tile * HIGH : (g.end - at) / HIGH * HIGH);
            break;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return g;
}

}  // namespace
