// Attention of new tokens over the 8-bit cache (cache.hip):
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j),   over the keys j up to token i's own.
//
// Rows of a tile are the tokens of a sequence times the heads that share a key head, 16 RB of them.  A wavefront takes
// two blocks of 16 keys a step, straight from memory: the cache's order is that of its MFMA operands.  S^T = K Q^T, codes
// turned into fp16 exactly (a byte under 0x64 is 1024 + code + 128) and the block's scale taken to the score; in its result
// a lane holds four keys of each block for one row, which is the column operand of O^T = V^T P^T as it is -- the values
// lie in that order of keys -- so that nothing crosses lanes but the running maximum.
//
// The values' scale s_v of a block goes into the exponent, p s_v = exp2(x + log2 s_v - m), m the running maximum of x +
// log2 s_v: the largest product of a row is 1, whatever the scales.  It enters the MFMA in fp16 times 2^14, so that 2^-28 of
// the largest is still normal; the sum of p, in fp32, takes p s_v / s_v unrounded.  Rounding p to fp16 costs a value
// 2^-12 of itself, as much as the output's own rounding, and averages over the keys.
//
// Work is cut evenly: all steps of all tiles of a key head lie in a row, and workgroup i of W takes the i-th part of them,
// whatever sequences it meets there; a tile that several take leaves running maximum, sum and output of each in the
// workspace and a second launch joins them in order.  A step's loads are 2 KiB a block and lane-contiguous.
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "producer_math.h"
#include "row_groups.h"
#include "sequences.h"

namespace {

constexpr int kWaves = 4;
constexpr float kNothing = -1e30f;               // running maximum where no key was seen
constexpr float kShift = 14.0f;                  // p enters the MFMA as p 2^14

struct CachedArgs {
    CacheArgs c;
    const uint16_t *q;
    uint16_t *out;
    size_t q_stride, out_stride;
    float *part;                                 // [kv_heads][parts][2][16 RB rows][D + 4]: output, running maximum, sum
    float scale;                                 // times log2 e
    int group, heads, parts;                     // heads of a key head; workgroups of a key head
    int least;                                   // steps that a workgroup takes at least
};

// Tiles of a sequence and the steps of each (pairs of blocks; every tile counts as many as the last one has).
struct Span {
    int tiles, steps;
};

template <int ROWS>
__device__ __forceinline__ Span span_of(const CachedArgs &a, int begin, int end, int length)
{
    const int n = max(min(end, a.c.M) - max(begin, 0), 0);
    Span s;
    s.tiles = (n * a.group + ROWS - 1) / ROWS;
    s.steps = (length + 2 * kBlock - 1) / (2 * kBlock);
    if (s.steps == 0) s.steps = 1;               // (its rows are zero, and written by someone)
    return s;
}

// The place of step `at` of a key head's steps: whose tile it falls in, and the tile's first step.
struct Place {
    int id, begin, n, length, tile, tiles, steps;
    long tile_first;                             // step of the row of all at which the tile begins
};

template <int ROWS>
__device__ __forceinline__ long all_steps(const CachedArgs &a)
{
    long total = 0;
    for (int s0 = 0; s0 < a.c.count; s0 += 64) {
        const int s = min(s0 + (int)(threadIdx.x & 63), a.c.count - 1);
        const Span w = span_of<ROWS>(a, a.c.starts[s], a.c.starts[s + 1], cached_length(a.c, s));
        long mine = s0 + (int)(threadIdx.x & 63) < a.c.count ? (long)w.tiles * w.steps : 0;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d, 64);
        total += mine;
    }
    return total;
}

template <int ROWS>
__device__ __forceinline__ Place find_step(const CachedArgs &a, long at)
{
    const int lane = threadIdx.x & 63;
    long before = 0;
    for (int s0 = 0; s0 < a.c.count; s0 += 64) {
        const int s = min(s0 + lane, a.c.count - 1);
        const int begin = a.c.starts[s], end = a.c.starts[s + 1], length = cached_length(a.c, s);
        const Span w = span_of<ROWS>(a, begin, end, length);
        const long mine = s0 + lane < a.c.count ? (long)w.tiles * w.steps : 0;
        long sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const long other = __shfl_up(sum, d, 64);
            if (lane >= d) sum += other;
        }
        const long first = before + sum - mine;
        const unsigned long long hit = __ballot(at >= first && at < first + mine);
        if (hit) {
            const int l = __ffsll(hit) - 1;
            Place p;
            p.id = s0 + l;
            p.begin = max(__builtin_amdgcn_readlane(begin, l), 0);
            p.n = min(__builtin_amdgcn_readlane(end, l), a.c.M) - p.begin;
            p.length = __builtin_amdgcn_readlane(length, l);
            p.tiles = __builtin_amdgcn_readlane(w.tiles, l);
            p.steps = __builtin_amdgcn_readlane(w.steps, l);
            const long from = __shfl(first, l, 64);
            p.tile = (int)((at - from) / p.steps);
            p.tile_first = from + (long)p.tile * p.steps;
            return p;
        }
        before += __shfl(sum, 63, 64);
    }
    Place p{};
    p.id = -1;
    return p;
}

// Workgroups that share the steps, and where the part of one begins: part i of n is at / n rounded down.
__device__ __forceinline__ int parts_of_all(const CachedArgs &a, long total)
{
    const long most = (total + a.least - 1) / a.least;
    return (int)(most < a.parts ? most : a.parts);
}

__device__ __forceinline__ v4f mfma_h(v8h a, v8h b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight biased codes -> fp16, exactly.
__device__ __forceinline__ v8h codes_to_half(unsigned lo, unsigned hi)
{
    union {
        unsigned u[4];
        v2h h[4];
        v8h v;
    } x;
    const unsigned top = 0x64646464u;
    x.u[0] = __builtin_amdgcn_perm(top, lo, 0x04010400u);
    x.u[1] = __builtin_amdgcn_perm(top, lo, 0x04030402u);
    x.u[2] = __builtin_amdgcn_perm(top, hi, 0x04010400u);
    x.u[3] = __builtin_amdgcn_perm(top, hi, 0x04030402u);
    const v2h bias = {(_Float16)(1024 + kCodeBias), (_Float16)(1024 + kCodeBias)};
#pragma unroll
    for (int i = 0; i < 4; ++i) x.h[i] = x.h[i] - bias;
    return x.v;
}

__device__ __forceinline__ v8h to_half8(const float (&lo)[4], const float (&hi)[4])
{
    union {
        v2h h[4];
        v8h v;
    } x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x.h[i] = __builtin_convertvector((v2f{lo[2 * i], lo[2 * i + 1]}), v2h);
        x.h[2 + i] = __builtin_convertvector((v2f{hi[2 * i], hi[2 * i + 1]}), v2h);
    }
    return x.v;
}

// Over the four lanes that hold a row's keys: l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float across_max(float v)
{
    auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float across_sum(float v)
{
    auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// What a wavefront holds of its rows.
template <int D, int RB>
struct Running {
    v4f o[RB][D / 16];
    float m[RB], l[RB];
};

// Scores of two blocks of 16 keys, x[b][i] = key 4 g + i of block b (times log2 e, -inf where the row does not see it), go into the
// running state; lv: log2 of the blocks' value scales; values(t): the row operand of channels 16 t .. 16 t + 15.
template <int D, int RB, class Values>
__device__ __forceinline__ void take(Running<D, RB> &r, const float (&x)[RB][2][4], float lv0, float lv1, const Values &values)
{
    v8h p[RB];
    const float inv0 = __builtin_amdgcn_exp2f(-lv0), inv1 = __builtin_amdgcn_exp2f(-lv1);
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        float top = kNothing, e[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[0][i] = x[k][0][i] + lv0;
            e[1][i] = x[k][1][i] + lv1;
            top = fmaxf(top, fmaxf(e[0][i], e[1][i]));
        }
        top = across_max(top);
        if (__any(top > r.m[k])) {
            const float m = fmaxf(r.m[k], top), f = __builtin_amdgcn_exp2f(r.m[k] - m);
            r.m[k] = m;
            r.l[k] *= f;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) r.o[k][t] *= f;
        }
        const float m = r.m[k] - kShift;
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[0][i] = __builtin_amdgcn_exp2f(e[0][i] - m);
            e[1][i] = __builtin_amdgcn_exp2f(e[1][i] - m);
            s0 += e[0][i];
            s1 += e[1][i];
        }
        r.l[k] += s0 * inv0 + s1 * inv1;
        p[k] = to_half8(e[0], e[1]);
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
        const v8h v = values(t);
#pragma unroll
        for (int k = 0; k < RB; ++k) r.o[k][t] = mfma_h(v, p[k], r.o[k][t]);
    }
}

// Four channels of row `row` of a sequence's and key head's rows: o / l, 65504 at most (a scale's own rounding may lead
// beyond); zero where the row sees nothing.
__device__ __forceinline__ void store_row(const CachedArgs &a, int begin, int row, int head, int D, int d, v4f o, float l)
{
    const int token = row / a.group;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    v4f y = o * inv;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i], -65504.0f, 65504.0f);
    uint16_t *out = a.out + (size_t)(begin + token) * a.out_stride + (size_t)(head * a.group + row - token * a.group) * D + d;
    *reinterpret_cast<uint2 *>(out) = make_uint2(pack_h2(y[0], y[1]), pack_h2(y[2], y[3]));
}

template <int D, int RB>
__global__ __launch_bounds__(64 * kWaves) void cached_kernel(CachedArgs a)
{
    typedef CacheBlock<D> B;
    constexpr int ROWS = 16 * RB, P = D / 64;    // P: planes of keys, and of values, of a block
    __shared__ __attribute__((aligned(16))) float red[kWaves][16][D + 4];
    __shared__ float stat[kWaves][2][16];
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i16 = lane & 15;
    const int head = blockIdx.x % c.kv_heads, index = blockIdx.x / c.kv_heads;
    const long total = all_steps<ROWS>(a);
    const int parts = parts_of_all(a, total);
    if (index >= parts) return;
    long at = total * index / parts;
    const long stop = total * (index + 1) / parts;
    while (at < stop) {
        const Place p = find_step<ROWS>(a, at);
        if (p.id < 0) return;
        const long end = min(stop, p.tile_first + p.steps);
        const int first = (int)(at - p.tile_first), last = (int)(end - p.tile_first);    // steps of the tile
        const bool whole = first == 0 && last == p.steps;
        const int rows = min(ROWS, p.n * a.group - p.tile * ROWS);
        // rows of this lane: token, position, query
        int limit[RB];
        v8h q[RB][D / 32];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const int row = p.tile * ROWS + min(16 * k + i16, rows - 1), token = row / a.group;
            limit[k] = p.length - p.n + token;
            const uint16_t *from = a.q + (size_t)(p.begin + token) * a.q_stride + (size_t)(head * a.group + row - token * a.group) * D;
#pragma unroll
            for (int m = 0; m < D / 32; ++m) q[k][m] = *reinterpret_cast<const v8h *>(from + 32 * m + 8 * g);
        }
        Running<D, RB> r;
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            r.m[k] = kNothing;
            r.l[k] = 0.0f;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) r.o[k][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int full = p.length / kBlock;                                  // blocks in pages
        const int seen = (p.length - p.n + (p.tile * ROWS + rows - 1) / a.group) + 1;   // keys that any of the rows sees
        const int blocks = min(full, (max(seen, 0) + kBlock - 1) / kBlock);
        for (int s = first + wave; s < last; s += kWaves) {
            if (2 * s >= blocks) break;
            v4u kw[2][P], vw[2][P];
            float ks[2], lv[2];
            int from[2];                                                     // first key of a block; beyond all where there is none
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int block = min(2 * s + b, blocks - 1);
                const int page = B::page_of(c, p.id, block);
                const uint8_t *codes = B::codes(c, max(page, 0), head, block);
                const unsigned sc = *B::scales(c, max(page, 0), head, block);
                from[b] = page < 0 || 2 * s + b >= blocks ? 0x40000000 : block * kBlock;
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    kw[b][j] = *reinterpret_cast<const v4u *>(codes + 1024 * j + 16 * lane);
                    vw[b][j] = *reinterpret_cast<const v4u *>(codes + kBlock * D + 1024 * j + 16 * lane);
                }
                ks[b] = page < 0 ? 0.0f : h2f((uint16_t)(sc & 0xffffu)) * a.scale;
                lv[b] = page < 0 ? 0.0f : __builtin_amdgcn_logf(h2f((uint16_t)(sc >> 16)));
            }
            float x[RB][2][4];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                v4f acc[RB];
#pragma unroll
                for (int k = 0; k < RB; ++k) acc[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int m = 0; m < D / 32; ++m) {
                    const v8h key = codes_to_half(kw[b][m / 2][2 * (m & 1)], kw[b][m / 2][2 * (m & 1) + 1]);
#pragma unroll
                    for (int k = 0; k < RB; ++k) acc[k] = mfma_h(key, q[k][m], acc[k]);
                }
#pragma unroll
                for (int k = 0; k < RB; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[k][b][i] = from[b] + 4 * g + i <= limit[k] ? acc[k][i] * ks[b] : -INFINITY;
            }
            take(r, x, lv[0], lv[1], [&](int t) { return codes_to_half(vw[0][t / 4][t % 4], vw[1][t / 4][t % 4]); });
        }
        // the unfinished block's tokens, in fp16, with the tile's last step
        const int tail = p.length - full * kBlock;
        if (last == p.steps && tail > 0 && seen > full * kBlock && wave == (p.steps - 1 - first) % kWaves) {
            if (const uint16_t *recent = B::recent(c, p.id, head)) {
                float x[RB][2][4];
                v4f acc[RB];
#pragma unroll
                for (int k = 0; k < RB; ++k) acc[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                const int key = full * kBlock + min(i16, tail - 1);
#pragma unroll
                for (int m = 0; m < D / 32; ++m) {
                    const v8h w = *reinterpret_cast<const v8h *>(recent + B::recent_key(key, 32 * m + 8 * g));
#pragma unroll
                    for (int k = 0; k < RB; ++k) acc[k] = mfma_h(w, q[k][m], acc[k]);
                }
#pragma unroll
                for (int k = 0; k < RB; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[k][0][i] = 4 * g + i < tail && full * kBlock + 4 * g + i <= limit[k] ? acc[k][i] * a.scale : -INFINITY;
                        x[k][1][i] = -INFINITY;
                    }
                take(r, x, 0.0f, 0.0f, [&](int t) {
                    union {
                        uint16_t h[8];
                        v8h v;
                    } w;
                    const uint16_t *from = recent + B::recent_value(full * kBlock + 4 * g, 16 * t + i16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w.h[i] = 4 * g + i < tail ? from[i] : (uint16_t)0;   // (behind the last token anything may lie)
                        w.h[4 + i] = 0;
                    }
                    return w.v;
                });
            }
        }
        // the wavefronts' shares, sixteen rows at a time
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const float l = across_sum(r.l[k]);
            __syncthreads();
            if (g == 0) {
                stat[wave][0][i16] = r.m[k];
                stat[wave][1][i16] = l;
            }
#pragma unroll
            for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(&red[wave][i16][16 * t + 4 * g]) = r.o[k][t];
            __syncthreads();
            for (int u = threadIdx.x; u < min(16, rows - 16 * k) * (D / 4); u += 64 * kWaves) {
                const int row = u / (D / 4), d = u % (D / 4) * 4;
                float m = stat[0][0][row];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) m = fmaxf(m, stat[w][0][row]);
                float sum = 0.0f;
                v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f(stat[w][0][row] - m);
                    sum += f * stat[w][1][row];
                    o += *reinterpret_cast<const v4f *>(&red[w][row][d]) * f;
                }
                if (whole) {
                    store_row(a, p.begin, p.tile * ROWS + 16 * k + row, head, D, d, o, sum);
                } else {
                    float *part =
                        a.part + ((((size_t)head * a.parts + index) * 2 + (first == 0 ? 1 : 0)) * ROWS + 16 * k + row) * (D + 4);
                    *reinterpret_cast<v4f *>(part + d) = o;
                    if (d == 0) {
                        part[D] = m;
                        part[D + 1] = sum;
                    }
                }
            }
        }
        at = end;
    }
}

// Tiles that several workgroups took: their shares in order.  Workgroup (i, r) joins rows r, r + slices, .. of the tile that
// begins in part i and does not end there, if there is one.
template <int D, int RB>
__global__ __launch_bounds__(256) void join_kernel(CachedArgs a, int slices)
{
    constexpr int ROWS = 16 * RB, Q = D / 4;     // Q: threads of a row
    const CacheArgs &c = a.c;
    const int head = blockIdx.x % c.kv_heads, slice = blockIdx.x / c.kv_heads % slices, index = blockIdx.x / c.kv_heads / slices;
    const long total = all_steps<ROWS>(a);
    const int parts = parts_of_all(a, total);
    if (index + 1 >= parts) return;
    const long start = total * index / parts, stop = total * (index + 1) / parts;
    const Place p = find_step<ROWS>(a, stop);
    if (p.id < 0 || p.tile_first >= stop || p.tile_first < start) return;
    const long to = p.tile_first + p.steps;
    int last = index + 1;                        // the last part that has some of the tile
    while (last + 1 < parts && total * (last + 1) / parts < to) ++last;
    const int rows = min(ROWS, p.n * a.group - p.tile * ROWS);
    const int d = threadIdx.x % Q * 4;
    for (int row = slice + slices * (int)(threadIdx.x / Q); row < rows; row += slices * (256 / Q)) {
        float m = kNothing, l = 0.0f;
        v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = index; i <= last; ++i) {
            const float *part = a.part + ((((size_t)head * a.parts + i) * 2 + (i == index ? 1 : 0)) * ROWS + row) * (D + 4);
            const v4f oi = *reinterpret_cast<const v4f *>(part + d);
            const float mi = part[D], li = part[D + 1];
            const float top = fmaxf(m, mi), f = __builtin_amdgcn_exp2f(m - top), fi = __builtin_amdgcn_exp2f(mi - top);
            m = top;
            l = l * f + li * fi;
            o = o * f + oi * fi;
        }
        store_row(a, p.begin, p.tile * ROWS + row, head, D, d, o, l);
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Workgroups of a launch: about four a CU.
int parts_for(int kv_heads)
{
    const int parts = 1024 / kv_heads;
    return parts < 1 ? 1 : parts;
}

// Rows of a tile, by 16: as many as a sequence has on average.
int row_blocks(int M, int count, int group)
{
    const long rows = (long)M * group / count;
    return rows >= 48 ? 4 : rows >= 24 ? 2 : 1;
}

size_t workspace_for(int M, int count, int heads, int kv_heads, int head_dim)
{
    return (size_t)parts_for(kv_heads) * kv_heads * 2 * 16 * row_blocks(M, count, heads / kv_heads) * (head_dim + 4) * 4;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t flexq_cache_attention_workspace_bytes(int M, int sequences, int heads, int kv_heads, int head_dim)
{
    if (M < 1 || sequences < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || (head_dim != 64 && head_dim != 128) ||
        (long)heads * head_dim > FLEXQ_MAX_K)
        return 0;
    return workspace_for(M, sequences, heads, kv_heads, head_dim);
}

flexq_status flexq_cache_attention(const flexq_cache *cache, const flexq_sequences *seqs, int M, int heads, const uint16_t *q,
                                   int q_stride, float scale, uint16_t *out, int out_stride, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    if (!q || !out) return FLEXQ_EINVAL;
    CachedArgs a{};
    if (flexq_status s = flexq::cache_args(cache, seqs, M, a.c); s != FLEXQ_OK) return s;
    const int kv = cache->kv_heads, D = cache->head_dim;
    if (heads < 1 || heads % kv != 0 || !(scale > 0.0f && scale <= 65504.0f)) return FLEXQ_EINVAL;
    if ((long)heads * D > FLEXQ_MAX_K || q_stride < heads * D || out_stride < heads * D || q_stride % 8 != 0 || out_stride % 8 != 0)
        return FLEXQ_ESHAPE;
    if ((long)M * (heads / kv) >= (1L << 30)) return FLEXQ_ESHAPE;
    if (!aligned16(q) || !aligned16(out)) return FLEXQ_EALIGN;
    if (!workspace || workspace_bytes < workspace_for(M, seqs->count, heads, kv, D)) return FLEXQ_EWORKSPACE;
    if (!aligned16(workspace)) return FLEXQ_EALIGN;
    a.q = q;
    a.out = out;
    a.q_stride = (size_t)q_stride;
    a.out_stride = (size_t)out_stride;
    a.part = (float *)workspace;
    a.scale = scale * 1.44269504088896341f;
    a.group = heads / kv;
    a.heads = heads;
    a.parts = parts_for(kv);
    a.least = 8;
    const int rb = row_blocks(M, seqs->count, a.group);
    const int rows = (long)M * a.group < 16 * rb ? M * a.group : 16 * rb, per = 256 / (D / 4);
    const int slices = (rows + per - 1) / per;
    hipStream_t st = (hipStream_t)stream;
    auto run = [&](auto kern, auto join) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(a.parts * kv)), dim3(64 * kWaves), 0, st, a);
        if (hipGetLastError() != hipSuccess) return FLEXQ_EHIP;
        if (a.parts > 1) hipLaunchKernelGGL(join, dim3((unsigned)(a.parts * kv * slices)), dim3(256), 0, st, a, slices);
        return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
    };
    if (D == 128)
        return rb == 4   ? run(cached_kernel<128, 4>, join_kernel<128, 4>)
               : rb == 2 ? run(cached_kernel<128, 2>, join_kernel<128, 2>)
                         : run(cached_kernel<128, 1>, join_kernel<128, 1>);
    return rb == 4   ? run(cached_kernel<64, 4>, join_kernel<64, 4>)
           : rb == 2 ? run(cached_kernel<64, 2>, join_kernel<64, 2>)
                     : run(cached_kernel<64, 1>, join_kernel<64, 1>);
}

}  // extern "C"
#pragma GCC visibility pop
