// Low-rank adapters of many requests beside a projection that all of them share:
//
//   out[m] = fp16( y[m] + scale[l] * B[l] ( A[l] x[m] ) ),   l the adapter of row m,
//
// rows grouped by adapter (row_groups.h), those without one last: out[m] = y[m].
//
// Two launches.  The first makes h = A x in fp32: a workgroup takes 16 rows of one adapter and a
// piece of K, its wavefronts interleave over the piece 32 k at a time, fp16 MFMAs straight from
// memory (a row of x is used once, A lies in L2), and leaves its share of the sums in the workspace
// -- no atomics, so the order of additions is fixed.  The second adds the shares in their order and
// multiplies by B.  h keeps its 32 bits there without fp32 MFMAs (a sixteenth of the rate): scaled per
// row by a power of two that brings its largest value to 2^13 .. 2^14, h is split into hi = fp16(h)
// and lo = fp16(h - hi), which carry 22 bits (or 2^-38 of the row's largest), and both go through one
// MFMA: its 32 k are 16 ranks of hi and the same 16 of lo, against B's 16 ranks twice.  The sum is
// added to y in fp32 and rounded once.
//
// What bounds it: the low ranks' products are nothing (4096 rows of 4096 x 12288, rank 16: 2 GFLOP
// beside 233 MB), so memory, in rows too short for a tile to be used twice: there the first launch
// reads x at 2.3 TB/s, 14 us, the second reads y and writes out at 4.2, 48 us.  Few rows: the two
// launches and their trips to memory, one after the other (one row 3.7 + 4.2 us, 333 rows of
// 5248 x 13664 at rank 32 5.6 + 9.3).  In the second these are offsets (two, where rows without an adapter
// are copied), order, shares of h (a trip for every four splits, added up and split anew by every
// workgroup of a piece), LDS; then each step over columns waits for the loads and the stores of the
// one before.  64 ranks and more with many rows: the loads of A and B from L2, which every 16 or 32 rows
// repeat (4096 x 4096 of rank 64 43 us at 105 MB).
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "row_groups.h"

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
constexpr int kMaxRank = FLEXQ_MAX_RANK;

struct AdapterArgs {
    const uint16_t *a, *b;               // [L, R, K], [L, N, R]
    const float *scale;                  // [L]
    const uint16_t *x, *y;               // [M, K], [M, N]
    const int32_t *order, *offsets;
    uint16_t *out;
    float *h;                            // [splits][M][R], by place in the order
    int L, R, M, N, K, splits, columns;  // columns: of a workgroup of the second launch
};

__device__ __forceinline__ v4f mfma_h(v8h a, v8h b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// RT: tiles of 16 ranks that a workgroup makes; RB: rows of a piece, by 16; grid: pieces x rank chunks x K splits.
// A step is 64 k, a line of every row of x; U steps' loads set out together.
// EXACT: R is a multiple of RT tiles.
template <int RT, int RB, int U, bool EXACT>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs p, int chunks)
{
    constexpr int ROWS = 16 * RB;
    __shared__ float red[4][RT * 16][ROWS + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int id = blockIdx.x;
    const int split = id % p.splits;
    id /= p.splits;
    const int r0 = id % chunks * RT * 16;
    const RowGroup g = find_piece(p.offsets, p.L, p.M, ROWS, id / chunks);
    if (g.id < 0) return;
    const int first = g.begin + ROWS * g.tile, rows = min(ROWS, g.end - first);
    const int steps = p.K / 64;
    const int s0 = (int)((long)split * steps / p.splits), s1 = (int)((long)(split + 1) * steps / p.splits);
    const uint16_t *x[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = min(max(p.order[first + min(16 * b + (lane & 15), rows - 1)], 0), p.M - 1);
        x[b] = p.x + (size_t)row * p.K + 8 * (lane >> 4);
    }
    const uint16_t *a = p.a + ((size_t)g.id * p.R + r0 + (lane & 15)) * p.K + 8 * (lane >> 4);
    const int live = EXACT ? RT : min(RT, (p.R - r0) / 16);
    v4f acc[RT][RB];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[t][b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = s0 + wave; s < s1; s += 4 * U) {
        v8h xv[U][RB][2], av[U][RT][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + 4 * u < s1) {
                const size_t k = (size_t)64 * (s + 4 * u);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < RB; ++b) xv[u][b][h] = *reinterpret_cast<const v8h *>(x[b] + k + 32 * h);
#pragma unroll
                for (int t = 0; t < RT; ++t)
                    if (t < live) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            av[u][t][h] = *reinterpret_cast<const v8h *>(a + (size_t)16 * t * p.K + k + 32 * h);
                    }
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + 4 * u < s1) {
#pragma unroll
                for (int t = 0; t < RT; ++t)
                    if (t < live) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int b = 0; b < RB; ++b) acc[t][b] = mfma_h(av[u][t][h], xv[u][b][h], acc[t][b]);
                    }
            }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[wave][16 * t + 4 * (lane >> 4) + i][16 * b + (lane & 15)] = acc[t][b][i];
    __syncthreads();
    for (int i = tid; i < live * 16 * rows; i += 256) {
        const int m = i / (live * 16), r = i % (live * 16);
        p.h[((size_t)split * p.M + first + m) * p.R + r0 + r] = (red[0][r][m] + red[1][r][m]) + (red[2][r][m] + red[3][r][m]);
    }
}

// Ranks by 32, of which the kernel is laid out for up to F, hi and lo in an MFMA each; 16 that are left over, hi
// and lo, in one.  RB: rows of a piece, by 16.  EXACT: R is 32 F, or 16.
template <int F, int RB, bool EXACT>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs p, int rest)
{
    constexpr int ROWS = 16 * RB;
    constexpr int RT = EXACT && F > 0 ? 2 * F : 2 * F + 1;   // tiles of 16 ranks
    constexpr int STRIDE = RT * 16 + 8;                      // (padded against bank conflicts)
    __shared__ __attribute__((aligned(16))) _Float16 h[2][ROWS][STRIDE];      // hi, lo
    __shared__ float back[ROWS];                             // what undoes a row's power of two, times scale
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int column_blocks = (p.N + p.columns - 1) / p.columns;
    const int c0 = blockIdx.x % column_blocks * p.columns, c1 = min(p.N, c0 + p.columns);
    const RowGroup g = find_piece(p.offsets, p.L, p.M, ROWS, blockIdx.x / column_blocks, rest != 0);
    if (g.id < 0) return;
    const int first = g.begin + ROWS * g.tile, rows = min(ROWS, g.end - first);
    size_t at[RB];                                           // this lane's rows' first columns in y and out
    bool mine[RB];
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        const int m = 16 * k + (lane & 15);
        mine[k] = m < rows;
        const int row = min(max(p.order[first + min(m, rows - 1)], 0), p.M - 1);
        at[k] = (size_t)row * p.N + 16 * (lane >> 4);
    }
    auto load_y = [&](uint4 (&v)[2], int k, int n0) {
        if (mine[k] && n0 + 16 * (lane >> 4) < c1) {
            v[0] = reinterpret_cast<const uint4 *>(p.y + at[k] + n0)[0];
            v[1] = reinterpret_cast<const uint4 *>(p.y + at[k] + n0)[1];
        }
    };
    auto store = [&](const uint4 (&v)[2], int k, int n0) {
        if (mine[k] && n0 + 16 * (lane >> 4) < c1) {
            reinterpret_cast<uint4 *>(p.out + at[k] + n0)[0] = v[0];
            reinterpret_cast<uint4 *>(p.out + at[k] + n0)[1] = v[1];
        }
    };
    if (g.id == p.L) {                   // rows without an adapter
        for (int n0 = c0 + 64 * wave; n0 < c1; n0 += 256)
#pragma unroll
            for (int k = 0; k < RB; ++k)
                if (mine[k] && n0 + 16 * (lane >> 4) < c1) {
                    const uint4 *from = reinterpret_cast<const uint4 *>(p.y + at[k] + n0);
                    uint4 *to = reinterpret_cast<uint4 *>(p.out + at[k] + n0);
                    const uint4 u = from[0], v = from[1];
                    to[0] = u;
                    to[1] = v;
                }
        return;
    }
    const int full = EXACT ? F : p.R / 32, tail = EXACT ? F == 0 : p.R / 16 & 1, live = EXACT ? RT : p.R / 16;
    // MFMA row i of tile t is column 16 (i / 4) + 4 t + i % 4 of 64: a lane's results are 16 in a row
    const int i = lane & 15;
    const uint16_t *b = p.b + (size_t)g.id * p.N * p.R;
    struct Stage {
        v8h full[4][F > 0 ? F : 1], tail[4];
        uint4 y[RB][2];
    };
    auto load = [&](Stage &s, int n0) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint16_t *from = b + (size_t)min(n0 + 16 * (i >> 2) + 4 * t + (i & 3), p.N - 1) * p.R;
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (f < full) s.full[t][f] = *reinterpret_cast<const v8h *>(from + 32 * f + 8 * (lane >> 4));
            if (tail) s.tail[t] = *reinterpret_cast<const v8h *>(from + 32 * full + 8 * ((lane >> 4) & 1));
        }
#pragma unroll
        for (int k = 0; k < RB; ++k) load_y(s.y[k], k, n0);
    };
    Stage st;                            // the first columns' operands set out ahead of h
    int n0 = c0 + 64 * wave;
    if (n0 < c1) load(st, n0);
    {
        const int q = tid & 15;
        float v[RB][RT];
#pragma unroll
        for (int k = 0; k < RB; ++k)
#pragma unroll
            for (int t = 0; t < RT; ++t) v[k][t] = 0.0f;
        // (four splits' shares set out together: one after the other they are most of a small call.  More than sixteen
        // loads the compiler does not gather by itself: rank 128 of 64 x 4096 20.8 us, 12.4 with the array)
        auto share = [&](int s, int k, int t) {
            const int m = min(16 * k + (tid >> 4), rows - 1);         // (rows beyond the last repeat it and are not stored)
            return t < live ? p.h[((size_t)s * p.M + first + m) * p.R + 16 * t + q] : 0.0f;
        };
        if constexpr (RT * RB <= 4) {
#pragma unroll 4
            for (int s = 0; s < p.splits; ++s)
#pragma unroll
                for (int k = 0; k < RB; ++k)
#pragma unroll
                    for (int t = 0; t < RT; ++t) v[k][t] += share(s, k, t);
        } else {
            for (int s = 0; s < p.splits; s += 4) {
                float w[4][RB][RT];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int k = 0; k < RB; ++k)
#pragma unroll
                        for (int t = 0; t < RT; ++t) w[u][k][t] = share(min(s + u, p.splits - 1), k, t);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (s + u < p.splits)
#pragma unroll
                        for (int k = 0; k < RB; ++k)
#pragma unroll
                            for (int t = 0; t < RT; ++t) v[k][t] += w[u][k][t];
            }
        }
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const int m = 16 * k + (tid >> 4);
            float top = 0.0f;
#pragma unroll
            for (int t = 0; t < RT; ++t) top = fmaxf(top, fabsf(v[k][t]));
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
            // an infinite row is what its infinite ranks make of it: the others, finite, stay so, and nothing is taken
            // from an infinity
            const bool infinite = top == INFINITY;
            int e = 0;
            if (top > 0.0f) e = infinite ? -60 : 14 - (__builtin_amdgcn_frexp_expf(top));
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const float w = __builtin_amdgcn_ldexpf(v[k][t], e);
                const _Float16 hi = (_Float16)w;
                h[0][m][16 * t + q] = hi;
                h[1][m][16 * t + q] = infinite ? (_Float16)0.0f : (_Float16)(w - (float)hi);
            }
            if (q == 0) back[m] = __builtin_amdgcn_ldexpf(p.scale[g.id], -e);
        }
    }
    __syncthreads();
    v8h hi[RB][F > 0 ? F : 1], lo[RB][F > 0 ? F : 1], both[RB];
    float undo[RB];
#pragma unroll
    for (int k = 0; k < RB; ++k) {
#pragma unroll
        for (int f = 0; f < F; ++f) {
            hi[k][f] = *reinterpret_cast<const v8h *>(&h[0][16 * k + i][32 * f + 8 * (lane >> 4)]);
            lo[k][f] = *reinterpret_cast<const v8h *>(&h[1][16 * k + i][32 * f + 8 * (lane >> 4)]);
        }
        both[k] = *reinterpret_cast<const v8h *>(&h[lane >> 5][16 * k + i][(tail ? 32 * full : 0) + 8 * ((lane >> 4) & 1)]);
        undo[k] = back[16 * k + i];
    }
    for (; n0 < c1; n0 += 256) {
        v4f acc[RB][4];
#pragma unroll
        for (int k = 0; k < RB; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                acc[k][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int f = 0; f < F; ++f)
                    if (f < full) {
                        acc[k][t] = mfma_h(st.full[t][f], hi[k][f], acc[k][t]);
                        acc[k][t] = mfma_h(st.full[t][f], lo[k][f], acc[k][t]);
                    }
                if (tail) acc[k][t] = mfma_h(st.tail[t], both[k], acc[k][t]);
            }
        uint4 v[RB][2];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const unsigned w[8] = {st.y[k][0].x, st.y[k][0].y, st.y[k][0].z, st.y[k][0].w,
                                   st.y[k][1].x, st.y[k][1].y, st.y[k][1].z, st.y[k][1].w};
            unsigned o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float even = __builtin_fmaf(acc[k][j / 2][2 * (j & 1)], undo[k], h2f((uint16_t)w[j]));
                const float odd = __builtin_fmaf(acc[k][j / 2][2 * (j & 1) + 1], undo[k], h2f((uint16_t)(w[j] >> 16)));
                o[j] = (unsigned)f2h(even) | ((unsigned)f2h(odd) << 16);
            }
            v[k][0] = make_uint4(o[0], o[1], o[2], o[3]);
            v[k][1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
        if (n0 + 256 < c1) load(st, n0 + 256);
#pragma unroll
        for (int k = 0; k < RB; ++k) store(v[k], k, n0);
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Pieces that M rows of `groups` groups can come in, and about how many they will be.
long pieces_bound(int M, int groups, int height) { return M / height + (groups < M ? groups : M); }
long pieces_likely(int M, int groups, int height) { return (M + height - 1) / height + (groups < M ? groups : M) / 2; }

// Rows of a piece, by 16, of either launch (they may differ, h lies by place).  Two read A or B, from L2, half as often,
// but begin dearer and are fewer: they pay where adapters have 24 rows or more on average, in the first launch from
// about 5 million values of x on, whatever the rank, in the second where sixteen rows a piece would read 50 MB of B.  us
// with one / two in both launches: 64 x 4096 x 4096 of rank 64 10.4 / 13.0, 200 x 12288 x 4096 of rank 32 11 / 14, 2000 x
// 4096 x 4096 of rank 64 29.3 / 25.2, 2000 x 8192 x 28672 of rank 128 192 / 132.  (Over 208 shapes of 26 .. 4096 rows
// this takes 1.01 times the best of the four combinations' time on average, two from 24 rows on 1.11.)
int row_blocks(int M, int L, int R, bool enough)
{
    return R <= 128 && M >= 24 * (long)(L < M ? L : M) && enough ? 2 : 1;
}
int down_blocks(int M, int L, int R, int K) { return row_blocks(M, L, R, pieces_likely(M, L, 16) * K >= 300000); }
int up_blocks(int M, int L, int R, int N) { return row_blocks(M, L, R, pieces_likely(M, L, 16) * R * N >= 25000000); }

// K splits of the first launch: until there are about two workgroups a CU -- one, of 32 rows at 64 ranks or more, whose
// loads fill it (4096 x 4096 of rank 64 48 -> 43 us) -- but 1024 k (four steps a wavefront) or more each, 512 where
// even then half the chip is idle (333 x 5248 of rank 32 17.3 -> 16.0 us).  Every split is a share of h that the
// second launch's workgroups read, four at a time: with 32-row pieces no more than 512 ranks' worth (rank 128 of 600 x
// 12288 x 4096 in two 47 us, in four 33, in eight 35), and above four a multiple of four.
int splits_for(int M, int L, int R, int K)
{
    const int blocks = down_blocks(M, L, R, K);
    const long pieces = pieces_likely(M, L, 16 * blocks);
    long s = ((blocks == 2 && R >= 64 ? 256 : 512) + pieces - 1) / pieces;
    const int least = pieces * ((R + 63) / 64) * (K / 1024) <= 128 ? 512 : 1024;
    if (s > K / least) s = K / least;
    if (blocks == 2 && s > 512 / R) s = 512 / R;
    if (s > 4) s -= s % 4;
    return s < 1 ? 1 : s > 64 ? 64 : (int)s;
}

// Columns of a workgroup of the second launch, 256 a step: one step where that gives few workgroups, else 2, 4 ..
// until they are about as many as the chip takes well.  Low ranks are bound by memory and want many in flight
// (us by 1 / 2 / 4 / 8 steps: rank 16 of 4096 x 12288 71 / 64 / 62 / 70, of 4096 x 4096 33 / 31 / 33 / 34); with
// higher ones two workgroups fill a CU's registers and each begins dearer, with its rows, h and first operands
// (rank 64 of 2048 x 8192 81 / 60 / 51 / 51, of 48 x 10240 18.5 / 17.8 / 18.7 / 23.8, 128 of 1024 x 4096 32 / 32 / 38 / 48).
int up_columns(long pieces, int N, int tiles, int blocks)
{
    const long most = tiles <= 2 ? 2100 : blocks == 2 ? 768 : 1024;
    int steps = 1;
    while (steps < 16 && pieces * ((N + 256 * steps - 1) / (256 * steps)) > most) steps *= 2;
    return 256 * steps;
}

size_t workspace_bytes_for(int M, int L, int R, int K)
{
    return ((size_t)splits_for(M, L, R, K) * M * R * 4 + 255) / 256 * 256;
}

bool shape_ok(int L, int R, int M, int K)
{
    return K % 128 == 0 && K <= FLEXQ_MAX_K && L <= FLEXQ_MAX_EXPERTS && R % 16 == 0 && R <= kMaxRank && M <= (1 << 24);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t flexq_adapters_workspace_bytes(int M, int L, int R, int K)
{
    if (M < 1 || L < 1 || R < 1 || K < 1 || !shape_ok(L, R, M, K)) return 0;
    return workspace_bytes_for(M, L, R, K);
}

flexq_status flexq_adapters(const uint16_t *a, const uint16_t *b, const float *scale, int L, int R, const uint16_t *x,
                            const int32_t *order, const int32_t *offsets, int M, int N, int K, const uint16_t *y,
                            uint16_t *out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a || !b || !scale || !x || !order || !offsets || !y || !out) return FLEXQ_EINVAL;
    if (L < 1 || R < 1 || M < 1 || N < 1 || K < 1) return FLEXQ_EINVAL;
    if (!shape_ok(L, R, M, K) || N % 32 != 0) return FLEXQ_ESHAPE;
    if (!aligned16(a) || !aligned16(b) || !aligned16(x) || !aligned16(y) || !aligned16(out) || !aligned4(scale) ||
        !aligned4(order) || !aligned4(offsets))
        return FLEXQ_EALIGN;
    if (!workspace || workspace_bytes < workspace_bytes_for(M, L, R, K)) return FLEXQ_EWORKSPACE;
    if (!aligned16(workspace)) return FLEXQ_EALIGN;
    AdapterArgs p{};
    p.a = a;
    p.b = b;
    p.scale = scale;
    p.x = x;
    p.y = y;
    p.order = order;
    p.offsets = offsets;
    p.out = out;
    p.h = (float *)workspace;
    p.L = L;
    p.R = R;
    p.M = M;
    p.N = N;
    p.K = K;
    p.splits = splits_for(M, L, R, K);
    const int tiles = R / 16, down_by = down_blocks(M, L, R, K), up_by = up_blocks(M, L, R, N);
    // the rows without an adapter need no products, and nothing at all where out is y
    const int rest = out != y ? 1 : 0;
    p.columns = up_columns(pieces_likely(M, L + rest, 16 * up_by), N, tiles, up_by);
    hipStream_t st = (hipStream_t)stream;
    const int rt = tiles == 1 ? 1 : tiles == 2 ? 2 : 4, chunks = (tiles + rt - 1) / rt;
    const long down_grid = pieces_bound(M, L, 16 * down_by) * chunks * p.splits;
    const long up_grid = pieces_bound(M, L + rest, 16 * up_by) * ((N + p.columns - 1) / p.columns);
    if (down_grid >= (1L << 24) || up_grid >= (1L << 24)) return FLEXQ_ESHAPE;      // 256 threads each, 2^32 a launch
    auto down = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)down_grid), dim3(256), 0, st, p, chunks);
        return hipGetLastError();
    };
    auto up = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)up_grid), dim3(256), 0, st, p, rest);
        return hipGetLastError();
    };
    hipError_t e;
    if (down_by == 2)
        e = rt == 1          ? down(adapter_down_kernel<1, 2, 4, true>)
            : rt == 2        ? down(adapter_down_kernel<2, 2, 2, true>)
            : tiles % 4 == 0 ? down(adapter_down_kernel<4, 2, 2, true>)
                             : down(adapter_down_kernel<4, 2, 2, false>);
    else
        e = rt == 1          ? down(adapter_down_kernel<1, 1, 4, true>)
            : rt == 2        ? down(adapter_down_kernel<2, 1, 4, true>)
            : tiles % 4 == 0 ? down(adapter_down_kernel<4, 1, 2, true>)
                             : down(adapter_down_kernel<4, 1, 2, false>);
    if (e != hipSuccess) return FLEXQ_EHIP;
    if (up_by == 2)
        switch (tiles) {
        case 1: e = up(adapter_up_kernel<0, 2, true>); break;
        case 2: e = up(adapter_up_kernel<1, 2, true>); break;
        case 4: e = up(adapter_up_kernel<2, 2, true>); break;
        case 8: e = up(adapter_up_kernel<4, 2, true>); break;
        default: e = up(adapter_up_kernel<3, 2, false>);
        }
    else
        switch (tiles) {
        case 1: e = up(adapter_up_kernel<0, 1, true>); break;
        case 2: e = up(adapter_up_kernel<1, 1, true>); break;
        case 4: e = up(adapter_up_kernel<2, 1, true>); break;
        case 8: e = up(adapter_up_kernel<4, 1, true>); break;
        case 16: e = up(adapter_up_kernel<8, 1, true>); break;
        default: e = tiles < 8 ? up(adapter_up_kernel<3, 1, false>) : up(adapter_up_kernel<7, 1, false>);
        }
    return e == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
