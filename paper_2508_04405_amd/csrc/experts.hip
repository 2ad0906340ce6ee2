// Linear layers of experts: rows grouped by expert, each group through its own packed weights, and
// the weighted sum over the experts of a token.
//
//   y[r, n] = fp16( sx[i] * sw[e][n] * sum_k xq[i][k] wq[e][n][k] ),   offsets[e] <= r < offsets[e + 1],
//
// i the input row of sorted row r (order[r] / k for token rows, r itself for rows that are sorted
// already), the sum exact in int32 (group-128 scales: per group, then fp32), as in the dense layers.
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "api_internal.h"
#include "flexq_kernels.h"
#include "row_groups.h"
#include <math.h>

namespace {

using flexq::ExpertLinear;

// Few rows an expert: the experts' weights are read once and the products are small change, so a workgroup takes one
// expert and 32 output channels, whose tiles follow each other in memory, its W wavefronts interleave over them, unpack
// in registers and multiply by the rows (the MFMA's other 32, rows that are not there cost nothing), and their sums
// meet in LDS.  More than 32 rows walk the weights again, 32 rows a walk, in the same workgroup and by loads that the caches
// need not keep: an expert far above the others' average holds its workgroups while theirs are done.
// P tiles are asked for ahead, but in branches, so that the compiler waits for all that is on the way at the head of each
// step: there is one tile's time in flight, not P.  Ahead of the first weights lie three trips to memory one after
// the other: offsets, order, token scale.
// Bound by HBM and, below some 30 MB, by launch, ramp-up (those trips) and drain: six experts of 2816 x 2048 for one
// token, 26 MB, 8.2 us (3.2 TB/s), 9.6 with group-128 scales; eight of 4096 x 11008 with those at eight tokens, 250 MB,
// 52 us (4.8).  Activations go straight to registers: staged in LDS they cost a barrier before the first product and
// gained nothing.
template <int GROUP, int P, int W>
__global__ __launch_bounds__(64 * W) void expert_stream_kernel(ExpertLinear a)
{
    __shared__ int red[W][4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row_blocks = a.N / 32, KT = a.K / FLEXQ_TILE_K;
    const int nb = blockIdx.x % row_blocks;
    const RowGroup g = find_piece(a.offsets, a.E, a.slots, 0, blockIdx.x / row_blocks);
    if (g.id < 0) return;
    const uint8_t *base = static_cast<const uint8_t *>(a.packed) + (size_t)g.id * a.expert_bytes;
    const v4i *tiles = reinterpret_cast<const v4i *>(base) + (size_t)nb * KT * (FLEXQ_TILE_BYTES / 16);
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(base + (size_t)a.N * a.K / 4 * 3);

    for (int r0 = g.begin; r0 < g.end; r0 += 32) {
        const int rows = min(32, g.end - r0);
        const int r = r0 + (lane & 31);
        const bool live = (lane & 31) < rows;
        int slot = 0, in = 0;
        if (live) {
            slot = min(max(a.order[r], 0), a.slots - 1);
            in = a.k ? min(slot / a.k, a.x_rows - 1) : r;
        }
        const int8_t *x = a.xq + (size_t)in * a.K + 16 * (lane >> 5);
        const float sx = live ? h2f(a.sx[in]) : 0.0f;

        struct Stage {
            PackedTile w;
            v4i x[4];
            uint16_t gs;
        } st[P];
        auto load = [&](Stage &s, int t) {
            s.w = load_packed_tile(tiles + (size_t)t * (FLEXQ_TILE_BYTES / 16), lane);
            if (live) {
#pragma unroll
                for (int j = 0; j < 4; ++j) s.x[j] = *reinterpret_cast<const v4i *>(x + (size_t)t * FLEXQ_TILE_K + 32 * j);
            }
            if (GROUP) s.gs = scales[((size_t)nb * KT + t) * 32 + (lane & 31)];
        };
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (wave + W * p < KT) load(st[p], wave + W * p);
        v16i acc;
        v16f facc;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            acc[i] = 0;
            facc[i] = 0.0f;
        }
        for (int t = wave; t < KT;) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (t < KT) {
                    if (GROUP) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[i] = 0;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc = mfma_i8(st[p].x[j], unpack_kstep(st[p].w, j), acc);
                    if (GROUP) {
                        const float gs = h2f(st[p].gs);
#pragma unroll
                        for (int i = 0; i < 16; ++i) facc[i] = __builtin_fmaf((float)acc[i], gs, facc[i]);
                    }
                    if (t + W * P < KT) load(st[p], t + W * P);
                    t += W;
                }
            }
        }
        // the wavefronts' sums meet in LDS, eight rows at a time
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (8 * q >= rows) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) red[wave][i][lane] = GROUP ? __float_as_int(facc[4 * q + i]) : acc[4 * q + i];
            __syncthreads();
            for (int i = wave; i < 4; i += W) {
                const int m = mfma_row(4 * q + i, lane);
                const int n = 32 * nb + (lane & 31);
                float v;
                if (GROUP) {
                    float f = 0.0f;
#pragma unroll
                    for (int w = 0; w < W; ++w) f += __int_as_float(red[w][i][lane]);
                    v = f * 0.25f;
                } else {
                    int s = 0;
#pragma unroll
                    for (int w = 0; w < W; ++w) s += red[w][i][lane];
                    v = (float)(s >> 2);
                }
                const float xs = __shfl(sx, m & 31, 64);
                const int to = __shfl(slot, m & 31, 64);
                if (m < rows)
                    a.y[(size_t)(a.scatter ? to : r0 + m) * a.N + n] =
                        f2h(GROUP ? v * xs : v * (xs * h2f(scales[n])));
            }
            __syncthreads();
        }
    }
}

// out[t] = fp16( add[t] + sum_j weights[t][j] * y[t k + j] ), the sum in fp32 in the order of j, eight columns a
// thread.  Bound by memory: 2048 tokens of 6 experts, 2048 wide, 59 MB of which the layer before it has left most in
// the Infinity Cache: 10.4 us.  (Its own launch: added up in the layer's epilogue the sum would need atomics on fp16 rows, in no order.)
__global__ __launch_bounds__(256) void combine_kernel(const uint16_t *y, const int32_t *experts, const float *weights,
                                                      const uint16_t *add, int M, int k, int N, uint16_t *out)
{
    const int chunks = N / 8;
    const long at = (long)blockIdx.x * 256 + threadIdx.x;
    if (at >= (long)M * chunks) return;
    const long m = at / chunks;
    const int c = (int)(at - m * chunks);
    float sum[8];
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (add) v = reinterpret_cast<const uint4 *>(add + m * N)[c];
    auto half = [](const uint4 &q, int i) {
        const unsigned w = i < 2 ? q.x : i < 4 ? q.y : i < 6 ? q.z : q.w;
        return h2f((uint16_t)(w >> (16 * (i & 1))));
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = half(v, i);
    for (int j = 0; j < k; ++j) {
        if (experts[m * k + j] < 0) continue;
        const float w = weights[m * k + j];
        v = reinterpret_cast<const uint4 *>(y + (m * k + j) * N)[c];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(w, half(v, i), sum[i]);
    }
    unsigned o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (unsigned)f2h(sum[2 * i]) | ((unsigned)f2h(sum[2 * i + 1]) << 16);
    reinterpret_cast<uint4 *>(out + m * N)[c] = make_uint4(o[0], o[1], o[2], o[3]);
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline int groups_of(const ExpertLinear &a) { return a.E < a.slots ? a.E : a.slots; }

// Eight wavefronts a workgroup where there are at most two workgroups a CU and rows are long: four leave the
// chip half empty (11008 x 4096 by one token's two experts: 20.8 us with four, 14.6 with eight; with more
// workgroups eight only lengthen the meeting in LDS, 22016 x 4096 26.1 and 27.1, at eight tokens 80.8 and 84.5).
inline int stream_waves(const ExpertLinear &a) { return (long)groups_of(a) * (a.N / 32) <= 512 && a.K >= 4096 ? 8 : 4; }

template <int GROUP>
hipError_t launch_stream(const ExpertLinear &a, hipStream_t st)
{
    const long wgs = (long)groups_of(a) * (a.N / 32);
    if (wgs >= (1L << 31)) return hipErrorInvalidValue;
    if (stream_waves(a) == 8)
        hipLaunchKernelGGL((expert_stream_kernel<GROUP, 2, 8>), dim3((unsigned)wgs), dim3(512), 0, st, a);
    else
        hipLaunchKernelGGL((expert_stream_kernel<GROUP, 2, 4>), dim3((unsigned)wgs), dim3(256), 0, st, a);
    return hipGetLastError();
}

// Which kernel: 1 streaming, 2 .. 5 tiles of 32 x 128 (group-128 scales: 32 x 256), 64 x 128, 128 x 128,
// 128 x 256, 6 persistent tiles of 256 x 256 (128 x 256).
//
// How the rows fall is known on the device only, so by their average over the experts: the kernel that is
// estimated to be fastest.  An estimate is the busiest CU's stages of 128 k at what a stage takes with so many
// workgroups on a CU, something a round and a launch, and no less than the touched experts' weights take from
// memory.  The constants are fitted to 860 random layers (768 .. 12160 deep, 512 .. 22000 wide, 2 .. 128 experts, 16 ..
// 6000 tokens, 1 .. 8 experts each), which they meet to 10 .. 16 %; on 600 others of 1 .. 300 tokens what is chosen takes
// 1.028 times the fastest kernel's time on average, 1.12 or less on nine in ten, 1.48 at most.  All of them were routed
// nearly evenly (experts' scores apart by 0.3 of what they vary by): experts far above the average were not timed, and
// the streaming kernel suffers most there.  Some layers, us by form 1 / 2 / 3 / 4 / 5 / 6:
//   2 experts at 16 rows, K 8576, N 1088     12 / 23 / 27 / 37 / 56 / 49
//   64 at 24 rows, K 2048, N 2816            91 / 50 / 49 / 58 / 56 / -
//   8 at 128 rows, K 11008, N 4096           - / 119 / 97 / 103 / 96 / 103
//   8 at 256 rows, K 11008, N 4096           - / 188 / 144 / 142 / 150 / 122
//   8 at 1024 rows, K 4096, N 22016          - / 1321 / 915 / 776 / 723 / 691
struct TileTimes {
    int height, width, slots;            // of a tile; workgroups on a CU
    double stage[4], round, launch;      // us a stage by workgroups on the CU, a round, a launch
    double rate, least;                  // bytes a us from memory, and what a launch takes beside them
};
constexpr TileTimes kChannelTiles[4] = {
    {32, 128, 4, {0.331, 0.482, 0.716, 0.851}, 1.98, 3.12, 5.55e6, 4.87},
    {64, 128, 4, {0.391, 0.611, 0.958, 1.245}, 2.76, 2.74, 5.58e6, 5.73},
    {128, 128, 3, {0.562, 0.969, 1.488, 0.0}, 3.85, 1.88, 5.20e6, 7.80},
    {128, 256, 2, {0.851, 1.734, 0.0, 0.0}, 6.30, 0.79, 5.05e6, 8.41},
};
constexpr TileTimes kGroupTiles[3] = {
    {32, 256, 2, {0.624, 1.018, 0.0, 0.0}, 2.69, 3.19, 5.39e6, 5.81},
    {64, 128, 2, {0.540, 0.829, 0.0, 0.0}, 2.90, 2.54, 5.07e6, 6.59},
    {128, 128, 2, {0.806, 1.272, 0.0, 0.0}, 3.18, 2.94, 3.81e6, 7.31},
};
struct PersistentTimes {
    double high, low, high_item, low_item;   // us a stage of a tile of either height, and an item
    double uneven, launch, rate, least;      // of an item that the busiest CU has more than the average
};
constexpr PersistentTimes kPersistent[2] = {{1.251, 0.687, 8.50, 5.66, 0.577, 1.86, 4.51e6, 2.68},
                                            {0.993, 0.685, 7.17, 4.08, 0.462, 1.58, 5.36e6, 9.19}};
struct StreamTimes {
    double launch, step, row, wg, rate, least;   // us: a step of a wavefront, more for a row, for a workgroup on the CU
};
constexpr StreamTimes kStream[2] = {{4.77, 0.167, 0.0213, 0.325, 4.61e6, 4.97}, {2.02, 0.334, 0.0526, 0.339, 5.07e6, 5.77}};

int choose_form(const ExpertLinear &a)
{
    const int grouped = a.group != 0, count = groups_of(a);
    const double groups = count, rows = (double)a.slots / groups;
    const double stages = a.K / FLEXQ_TILE_K;
    auto up = [](double v) { return (double)(long)(v + 0.999999); };
    auto most = [](double x, double y) { return x > y ? x : y; };
    // experts with a row, if each slot picked one by itself
    const double touched = a.slots >= 4 * a.E ? a.E : a.E * (1.0 - pow(1.0 - 1.0 / a.E, a.slots));
    const double bytes = touched * 0.75 * (double)a.N * a.K;
    int best = 6;
    double least;
    {
        const PersistentTimes &t = kPersistent[grouped];
        const double height = grouped ? 128.0 : 256.0, across = (a.N + 255) / 256, spread = most(1.0, sqrt(rows));
        double high = 0.0, low = 0.0, sum = 0.0;
        for (int i = -4; i <= 4; ++i) {          // an expert's rows are spread by about their root
            const double weight = exp(-0.125 * i * i), n = most(0.0, rows + 0.5 * i * spread);
            const double whole = (double)(long)(n / height), rest = n - whole * height;
            high += weight * (whole + (rest > height / 2 ? 1.0 : 0.0));
            low += weight * (rest > 0.0 && rest <= height / 2 ? 1.0 : 0.0);
            sum += weight;
        }
        high *= groups * across / sum;
        low *= groups * across / sum;
        const double one = stages * t.high + t.high_item, other = stages * t.low + t.low_item;
        const double longest = high > 0.5 ? one : other;
        least = most((high * one + low * other) / 256.0 + t.uneven * longest, longest) + t.launch;
        least = most(least, bytes / t.rate + t.least);
    }
    for (int f = 0; f < (grouped ? 3 : 4); ++f) {
        const TileTimes &t = grouped ? kGroupTiles[f] : kChannelTiles[f];
        // a tile more than the rows fill, half a one on average
        const double tiles = groups * most(1.0, rows / t.height + 0.5) * ((a.N + t.width - 1) / t.width);
        const long per_cu = (long)up(tiles / 256.0), full = per_cu / t.slots, rest = per_cu % t.slots;
        double us = stages * (full * t.stage[t.slots - 1] + (rest ? t.stage[rest - 1] : 0.0)) +
                    t.round * (double)(full + (rest ? 1 : 0)) + t.launch;
        us = most(us, bytes / t.rate + t.least);
        if (us < least) {
            least = us;
            best = 2 + f;
        }
    }
    if (rows <= 40.0) {
        const StreamTimes &t = kStream[grouped];
        const long wgs = (long)count * (a.N / 32);
        const bool eight = stream_waves(a) == 8;
        const double per_cu = up(wgs / 256.0), steps = up(stages / (eight ? 8.0 : 4.0));
        const double passes = rows > 20.0 ? most(1.0, rows / 32.0 + 0.5) : 1.0, filled = rows < 32.0 ? rows : 32.0;
        double us = t.launch + passes * steps * ((t.step + t.row * filled) * up(per_cu / (eight ? 3.0 : 7.0)) + t.wg * per_cu);
        us = most(us, passes * bytes / t.rate + t.least);
        if (us < least) best = 1;
    }
    return best;
}

}  // namespace

namespace flexq {

flexq_status expert_impl(int form, const void *packed, int E, int group, const int8_t *xq, const uint16_t *sx, int x_rows,
                         const int32_t *order, const int32_t *offsets, int slots, int k, int scatter, int N, int K,
                         uint16_t *y, void *stream, int *dispatched)
{
    if (dispatched) *dispatched = 0;
    if (!packed || !xq || !sx || !order || !offsets || !y) return FLEXQ_EINVAL;
    if (E < 1 || x_rows < 1 || slots < 1 || k < 0 || k > FLEXQ_MAX_EXPERTS_PER_TOKEN || (scatter != 0 && scatter != 1))
        return FLEXQ_EINVAL;
    if (k ? (long)x_rows * k != slots : x_rows != slots) return FLEXQ_EINVAL;
    const size_t bytes = flexq_packed_bytes(N, K, group);
    if (bytes == 0) return N < 1 || K < 1 || (group != 0 && group != 128) ? FLEXQ_EINVAL : FLEXQ_ESHAPE;
    if (E > FLEXQ_MAX_EXPERTS || (long)x_rows * K >= (1L << 32) || (long)N * K / 4 * 3 >= (1L << 32)) return FLEXQ_ESHAPE;
    if (!aligned16(packed) || !aligned16(xq) || !aligned16(y) || !aligned4(order) || !aligned4(offsets)) return FLEXQ_EALIGN;
    ExpertLinear a{};
    a.packed = packed;
    a.expert_bytes = bytes;
    a.xq = xq;
    a.sx = sx;
    a.group = group;
    a.split_k = 1;
    a.order = order;
    a.offsets = offsets;
    a.E = E;
    a.slots = slots;
    a.x_rows = x_rows;
    a.k = k;
    a.scatter = scatter;
    a.N = N;
    a.K = K;
    a.y = y;
    hipStream_t st = (hipStream_t)stream;
    if (form == 0) form = choose_form(a);
    if (dispatched) *dispatched = form;
    hipError_t e;
    if (form == 1)
        e = group ? launch_stream<1>(a, st) : launch_stream<0>(a, st);
    else if (form == 6)
        e = launch_expert_tiles(a, st);
    else
        e = launch_gemm_experts(a, form, st);
    return e == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // namespace flexq

#pragma GCC visibility push(default)
extern "C" {

flexq_status flexq_expert_linear(const void *packed, int E, int group, const int8_t *xq, const uint16_t *sx, int x_rows,
                                 const int32_t *order, const int32_t *offsets, int slots, int k, int scatter, int N,
                                 int K, uint16_t *y, void *stream)
{
    return flexq::expert_impl(0, packed, E, group, xq, sx, x_rows, order, offsets, slots, k, scatter, N, K, y, stream, nullptr);
}

flexq_status flexq_expert_combine(const uint16_t *y, const int32_t *experts, const float *weights, const uint16_t *add,
                                  int M, int k, int N, uint16_t *out, void *stream)
{
    if (!y || !experts || !weights || !out || M < 1 || N < 1 || k < 1 || k > FLEXQ_MAX_EXPERTS_PER_TOKEN) return FLEXQ_EINVAL;
    if (N % 32 != 0 || (long)M * N / 8 > (1L << 32) - 256) return FLEXQ_ESHAPE;     // (threads of a launch)
    if (!aligned16(y) || !aligned16(out) || (add && !aligned16(add)) || !aligned4(experts) || !aligned4(weights))
        return FLEXQ_EALIGN;
    const unsigned blocks = (unsigned)(((long)M * (N / 8) + 255) / 256);
    hipLaunchKernelGGL(combine_kernel, dim3(blocks), dim3(256), 0, (hipStream_t)stream, y, experts, weights, add, M, k, N, out);
    return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
