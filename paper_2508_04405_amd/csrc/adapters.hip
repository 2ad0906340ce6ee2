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
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "row_groups.h"

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
constexpr int kRows = 16;                // rows of a piece
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

// RT: tiles of 16 ranks that a workgroup makes; grid: pieces x rank chunks x K splits.
template <int RT>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs p, int chunks)
{
    __shared__ float red[4][RT * 16][kRows + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int id = blockIdx.x;
    const int split = id % p.splits;
    id /= p.splits;
    const int r0 = id % chunks * RT * 16;
    const RowGroup g = find_piece(p.offsets, p.L, p.M, kRows, id / chunks);
    if (g.id < 0) return;
    const int first = g.begin + kRows * g.tile, rows = min(kRows, g.end - first);
    const int row = min(max(p.order[first + min(lane & 15, rows - 1)], 0), p.M - 1);
    const int steps = p.K / 32;
    const int s0 = (int)((long)split * steps / p.splits), s1 = (int)((long)(split + 1) * steps / p.splits);
    const uint16_t *x = p.x + (size_t)row * p.K + 8 * (lane >> 4);
    const uint16_t *a = p.a + ((size_t)g.id * p.R + r0 + (lane & 15)) * p.K + 8 * (lane >> 4);
    const int live = min(RT, (p.R - r0) / 16);
    v4f acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = 0.0f;
    for (int s = s0 + wave; s < s1; s += 4) {
        const v8h xv = *reinterpret_cast<const v8h *>(x + 32 * (size_t)s);
#pragma unroll
        for (int t = 0; t < RT; ++t)
            if (t < live) acc[t] = mfma_h(*reinterpret_cast<const v8h *>(a + (size_t)16 * t * p.K + 32 * (size_t)s), xv, acc[t]);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][16 * t + 4 * (lane >> 4) + i][lane & 15] = acc[t][i];
    __syncthreads();
    for (int i = tid; i < live * 16 * rows; i += 256) {
        const int m = i / (live * 16), r = i % (live * 16);
        p.h[((size_t)split * p.M + first + m) * p.R + r0 + r] = (red[0][r][m] + red[1][r][m]) + (red[2][r][m] + red[3][r][m]);
    }
}

// RT: tiles of 16 ranks, the last ones may be empty.
template <int RT>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs p, int rest)
{
    __shared__ __attribute__((aligned(16))) _Float16 h[kRows][RT * 32 + 8];   // hi 16, lo 16 ranks by turns
    __shared__ float back[kRows];                                             // what undoes a row's power of two, times scale
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int column_blocks = (p.N + p.columns - 1) / p.columns;
    const int c0 = blockIdx.x % column_blocks * p.columns, c1 = min(p.N, c0 + p.columns);
    const RowGroup g = find_piece(p.offsets, p.L, p.M, kRows, blockIdx.x / column_blocks, rest != 0);
    if (g.id < 0) return;
    const int first = g.begin + kRows * g.tile, rows = min(kRows, g.end - first);
    const int row = min(max(p.order[first + min(lane & 15, rows - 1)], 0), p.M - 1);
    const bool mine = (lane & 15) < rows;
    if (g.id == p.L) {                   // rows without an adapter
        for (int n = c0 + 64 * wave + 16 * (lane >> 4); n < c1; n += 256)
            if (mine) {
                const uint4 *from = reinterpret_cast<const uint4 *>(p.y + (size_t)row * p.N + n);
                uint4 *to = reinterpret_cast<uint4 *>(p.out + (size_t)row * p.N + n);
                const uint4 u = from[0], v = from[1];
                to[0] = u;
                to[1] = v;
            }
        return;
    }
    const int live = p.R / 16;
    {
        const int m = tid >> 4, q = tid & 15;
        float v[RT], top = 0.0f;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            v[t] = 0.0f;
            if (t < live && m < rows)
                for (int s = 0; s < p.splits; ++s) v[t] += p.h[((size_t)s * p.M + first + m) * p.R + 16 * t + q];
            top = fmaxf(top, fabsf(v[t]));
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        int e = 0;
        if (top > 0.0f) e = 14 - (__builtin_amdgcn_frexp_expf(top));
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float w = __builtin_amdgcn_ldexpf(v[t], e);
            const _Float16 hi = (_Float16)w;
            h[m][32 * t + q] = hi;
            h[m][32 * t + 16 + q] = (_Float16)(w - (float)hi);
        }
        if (q == 0) back[m] = __builtin_amdgcn_ldexpf(p.scale[g.id], -e);
    }
    __syncthreads();
    v8h hv[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) hv[t] = *reinterpret_cast<const v8h *>(&h[lane & 15][32 * t + 8 * (lane >> 4)]);
    const float undo = back[lane & 15];
    // MFMA row i of tile t is column 16 (i / 4) + 4 t + i % 4 of 64: a lane's results are 16 in a row
    const int i = lane & 15;
    const uint16_t *b = p.b + (size_t)g.id * p.N * p.R + 8 * ((lane >> 4) & 1);
    for (int n0 = c0 + 64 * wave; n0 < c1; n0 += 256) {
        v4f acc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int n = min(n0 + 16 * (i >> 2) + 4 * t + (i & 3), p.N - 1);
            acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < RT; ++r)
                if (r < live) acc[t] = mfma_h(*reinterpret_cast<const v8h *>(b + (size_t)n * p.R + 16 * r), hv[r], acc[t]);
        }
        const int n = n0 + 16 * (lane >> 4);
        if (mine && n < c1) {
            const uint4 *from = reinterpret_cast<const uint4 *>(p.y + (size_t)row * p.N + n);
            uint4 *to = reinterpret_cast<uint4 *>(p.out + (size_t)row * p.N + n);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint4 v = from[u];
                const unsigned w[4] = {v.x, v.y, v.z, v.w};
                unsigned o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float lo = __builtin_fmaf(acc[2 * u + j / 2][2 * (j & 1)], undo, h2f((uint16_t)w[j]));
                    const float hi = __builtin_fmaf(acc[2 * u + j / 2][2 * (j & 1) + 1], undo, h2f((uint16_t)(w[j] >> 16)));
                    o[j] = (unsigned)f2h(lo) | ((unsigned)f2h(hi) << 16);
                }
                to[u] = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Pieces of 16 rows that M rows of L adapters can come in.
long pieces_bound(int M, int L) { return (M + kRows - 1) / kRows + (L < M ? L : M); }

// K splits of the first launch: until there are about two workgroups a CU, but 512 k (four steps a
// wavefront) or more each.
int splits_for(int M, int L, int K)
{
    const long pieces = (M + kRows - 1) / kRows + (L < M ? L : M) / 2;
    long s = 512 / pieces;
    if (s > K / 512) s = K / 512;
    return s < 1 ? 1 : s > 64 ? 64 : (int)s;
}

size_t workspace_bytes_for(int M, int L, int R, int K)
{
    return ((size_t)splits_for(M, L, K) * M * R * 4 + 255) / 256 * 256;
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
    p.splits = splits_for(M, L, K);
    const long pieces = pieces_bound(M, L);
    p.columns = 256;
    while (p.columns < 2048 && pieces * (N / (2 * p.columns)) >= 1024) p.columns *= 2;
    hipStream_t st = (hipStream_t)stream;
    const int tiles = R / 16;
    auto down = [&](auto kern, int rt) {
        const int chunks = (tiles + rt - 1) / rt;
        hipLaunchKernelGGL(kern, dim3((unsigned)(pieces * chunks * p.splits)), dim3(256), 0, st, p, chunks);
        return hipGetLastError();
    };
    hipError_t e = tiles == 1   ? down(adapter_down_kernel<1>, 1)
                   : tiles == 2 ? down(adapter_down_kernel<2>, 2)
                   : tiles <= 4 ? down(adapter_down_kernel<4>, 4)
                                : down(adapter_down_kernel<8>, 8);
    if (e != hipSuccess) return FLEXQ_EHIP;
    // the rows without an adapter need no products, and nothing at all where out is y
    const int rest = out != y ? 1 : 0;
    const unsigned blocks = (unsigned)(pieces_bound(M, L + rest) * ((N + p.columns - 1) / p.columns));
    auto up = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, st, p, rest);
        return hipGetLastError();
    };
    e = tiles == 1   ? up(adapter_up_kernel<1>)
        : tiles == 2 ? up(adapter_up_kernel<2>)
        : tiles <= 4 ? up(adapter_up_kernel<4>)
        : tiles <= 8 ? up(adapter_up_kernel<8>)
                     : up(adapter_up_kernel<16>);
    return e == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
