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
// whatever sequences it meets there; a tile that several take leaves running maximum, sum and output of each in the workspace
// and a second launch joins them in order.  Where there are many tiles of few steps, which would leave a workgroup's wavefronts
// waiting for one another at every tile, each wavefront takes whole tiles of its own instead (`tiles_alone`: 58 sequences of up
// to 394 tokens of 32 key heads 56 -> 26 us, 38 of up to 23 of 8 36 -> 10, 128 of 1000 of 8 63 -> 49).  A step's loads are 2
// KiB a block and lane-contiguous, a step ahead, and non-temporal, since no one reads them again soon (48 sequences of up to
// 8192 tokens, 64 heads over 8: 87 -> 75 us).
//
// Bound by memory where the cache is long: those 413 MB in 75 us, 5.5 TB/s of the 6.5 that reads alone reach, one sequence of
// 131072 tokens, 269 MB, in 50; and the joining launch, 4 to 6 us, which would want a wait between workgroups to go.  A short
// cache takes the trips one after the other: lengths, table, codes, shares (1100 tokens of 32 heads 7.6 + 3.8 us).
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "producer_math.h"
#include "row_groups.h"
#include "sequences.h"

namespace {

constexpr int kWaves = 8;                        // of a workgroup of the streaming kernel
constexpr float kNothing = -1e30f;               // running maximum where no key was seen
constexpr float kShift = 14.0f;                  // p enters the MFMA as p 2^14

struct CachedArgs {
    CacheArgs c;
    const uint16_t *q;
    uint16_t *out;
    size_t q_stride, out_stride;
    float *part;                                 // [kv_heads][parts][2][rows of a tile][D + 4]: output, running maximum, sum
    float scale;                                 // times log2 e
    int group, parts;                            // heads of a key head; workgroups of a key head
    Divider by_group, by_parts;
    int least;                                   // steps that a workgroup takes at least, if a tile has them
};

// Where the steps of a call's tiles lie: those of sequence s follow those of the sequences before it, tile after tile; a
// tile of ROWS rows has as many of KEYS keys as its sequence's length takes (one, if it has none: someone writes its rows).  A lane
// holds one of 64 sequences; where they are more, they are gone through 64 at a time, by a question from where the last one ended.
struct Place {
    int id, begin, n, length, tile, steps;
    int first;                                   // step of all at which the tile begins
};

template <int ROWS, int KEYS>
struct Steps {
    static constexpr int EXTRA = ROWS == 128 ? 1 : kWaves;
    const CachedArgs &a;
    int begin, end, length, tiles, steps, first; // of this lane's sequence; first: of its steps among those of the 64
    int total, tile_total, longest;              // of all: steps, tiles, steps of the longest tile
    int from = 0, before = 0;                    // the 64 in which the last question ended; steps of those before them
    bool alone = false;                          // a tile counts as one step

    __device__ __forceinline__ Steps(const CachedArgs &args) : a(args) {}

    __device__ __forceinline__ int load(int s0)  // -> the steps of all 64
    {
        const int lane = threadIdx.x & 63, s = min(s0 + lane, a.c.count - 1);
        begin = max(a.c.starts[s], 0);
        end = min(a.c.starts[s + 1], a.c.M);
        length = cached_length(a.c, a.c.lengths[s]);
        size(s0);
        return scan();
    }
    __device__ __forceinline__ void size(int s0)
    {
        tiles = s0 + (int)(threadIdx.x & 63) < a.c.count ? (max(end - begin, 0) * a.group + ROWS - 1) / ROWS : 0;
        steps = max((length + KEYS - 1) / KEYS, 1);
    }
    __device__ __forceinline__ int weight() const { return alone ? 1 : steps; }
    __device__ __forceinline__ int scan()
    {
        const int sum = wave_scan(tiles * weight());
        first = sum - tiles * weight();
        return __builtin_amdgcn_readlane(sum, 63);
    }
    __device__ __forceinline__ int all()
    {
        total = tile_total = longest = 0;
        for (int s0 = 0; s0 < a.c.count; s0 += 64) {
            total += load(s0);
            tile_total += __builtin_amdgcn_readlane(wave_scan(tiles), 63);
            longest = max(longest, __builtin_amdgcn_readfirstlane((int)wave_max_bits(tiles ? (unsigned)steps : 0u)));
        }
        return total;
    }
    // (after all()) Whether wavefronts take whole tiles, each its own, and not eight of them a part together.  In half
    // microseconds, a tile costs a wavefront 6 and each of its steps 1, a workgroup 9 and an eighth of them.
    __device__ __forceinline__ bool tiles_alone()
    {
        const int rounds = divide(tile_total + a.parts * kWaves - 1, a.by_parts) / kWaves;
        const float own = (float)rounds * (float)(6 + longest) * (float)a.parts;
        const float together = 9.0f * (float)max(tile_total, a.parts) + 0.125f * (float)total;
        alone = __builtin_amdgcn_readfirstlane(own < together ? 1 : 0) != 0;
        if (alone && a.c.count <= 64) scan();
        return alone;
    }
    // (after all()) Part i of the steps is i * width .. (i + 1) * width - 1.
    __device__ __forceinline__ int width()
    {
        // (quotients by the hardware's reciprocal: a step more or less makes a part longer or shorter, the same for everyone)
        auto over = [](int x, int y) { return (float)x * __builtin_amdgcn_rcpf((float)max(y, 1)); };
        const int even = max(divide(total + a.parts - 1, a.by_parts), min(a.least, (int)(over(total, tile_total) + 0.01f)));
        // where all tiles have as many, parts that begin and end with them, if it takes a step for each wavefront more at most
        // (us without / with: 8 sequences of 700 tokens, 4 rows, 64 heads over 8, 23 / 17, 16 of 300, 9 rows, 25 / 23)
        const int fitting = (int)(over(longest, max((int)(over(longest, even) + 0.01f), 1)) + 0.99f);
        const bool fits = tile_total > 1 && longest * tile_total == total && fitting > even && fitting <= even + EXTRA;
        return __builtin_amdgcn_readfirstlane(fits ? fitting : even);
    }
    __device__ __forceinline__ Place find(int at)        // (after all(); at below it, and rising from one call to the next)
    {
        Place p{};
        p.id = -1;
        for (; from < a.c.count; from += 64) {
            int sum = 0;
            if (a.c.count > 64) {
                sum = load(from);
            } else {
                asm volatile("" : "+v"(begin), "+v"(end), "+v"(length));     // (made again, so that they take no registers meanwhile)
                size(from);
            }
            const unsigned long long hit = __ballot(at - before >= first && at - before < first + tiles * weight());
            if (hit) {
                const int l = __ffsll(hit) - 1;
                p.id = from + l;
                p.begin = __builtin_amdgcn_readlane(begin, l);
                p.n = __builtin_amdgcn_readlane(end, l) - p.begin;
                p.length = __builtin_amdgcn_readlane(length, l);
                p.steps = __builtin_amdgcn_readlane(steps, l);
                const int begins = before + __builtin_amdgcn_readlane(first, l);
                p.tile = alone ? at - begins : (at - begins) / p.steps;
                p.first = alone ? at : begins + p.tile * p.steps;
                return p;
            }
            before += sum;
        }
        return p;
    }
};

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

// Four channels of row `row` of a sequence's and key head's rows: o / l; zero where
// the row sees nothing.
__device__ __forceinline__ void store_row(const CachedArgs &a, int begin, int row, int head, int D, int d, v4f o, float l)
{
    const int token = divide(row, a.by_group);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    v4f y = o * inv;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = within_half(y[i]);
    uint16_t *out = a.out + (size_t)(begin + token) * a.out_stride + (size_t)(head * a.group + row - token * a.group) * D + d;
    *reinterpret_cast<uint2 *>(out) = make_uint2(pack_h2(y[0], y[1]), pack_h2(y[2], y[3]));
}

// Two blocks of 16 keys and values, as a lane has them.
template <int D>
struct Stage {
    v4u k[2][D / 64], v[2][D / 64];
    unsigned scales[2];                          // the key's, the value's << 16
};

template <int D, int RB>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void cached_kernel(CachedArgs a)
{
    typedef CacheBlock<D> B;
    constexpr int ROWS = 16 * RB, P = D / 64;    // P: planes of keys, and of values, of a block
    __shared__ __attribute__((aligned(16))) float red[kWaves][16][D + 4];
    __shared__ float stat[kWaves][2][16];
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i16 = lane & 15;
    const int index = divide(blockIdx.x, c.by_kv), head = blockIdx.x - index * c.kv_heads;
    Steps<ROWS, 2 * kBlock> all(a);
    const int total = all.all(), width = all.width();
    const bool alone = all.tiles_alone();
    const int every = alone ? 1 : kWaves, mine = alone ? 0 : wave;           // of a piece's steps: mine, mine + every, ..
    int at = alone ? index + a.parts * wave : index * width;
    const int stop = alone ? all.tile_total : min(at + width, total);
    while (at < stop) {
        const Place p = all.find(at);
        if (p.id < 0) return;
        const int end = alone ? at + a.parts * kWaves : min(stop, p.first + p.steps);
        const int first = alone ? 0 : at - p.first, last = alone ? p.steps : end - p.first;      // steps of the tile
        const bool whole = first == 0 && last == p.steps;
        const int rows = min(ROWS, p.n * a.group - p.tile * ROWS);
        // rows of this lane: token, position, query
        int limit[RB];
        v8h q[RB][D / 32];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const int row = p.tile * ROWS + min(16 * k + i16, rows - 1), token = divide(row, a.by_group);
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
        const int sees_first = p.length - p.n + divide(p.tile * ROWS, a.by_group);     // last key that the first row sees
        const int seen = p.length - p.n + divide(p.tile * ROWS + rows - 1, a.by_group) + 1;      // keys that any of the rows sees
        const int blocks = min(full, (max(seen, 0) + kBlock - 1) / kBlock);
        const int done = min(last, (blocks + 1) / 2);                        // steps over pages end here
        // pages a step ahead of the loads, loads a step ahead of the products; steps past the end repeat the last block
        auto pages = [&](int (&page)[2], int s) {
#pragma unroll
            for (int b = 0; b < 2; ++b) page[b] = c.table[(size_t)p.id * c.max_pages + (min(2 * s + b, blocks - 1) >> c.shift)];
        };
        auto load = [&](Stage<D> &st, int (&page)[2], int s) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int block = min(2 * s + b, blocks - 1);
                page[b] = __builtin_amdgcn_readfirstlane(page[b]);
                if (page[b] < 0 || page[b] >= c.pages) page[b] = -1;
                const uint8_t *codes = B::codes(c, max(page[b], 0), head, block);
                st.scales[b] = *B::scales(c, max(page[b], 0), head, block);
#pragma unroll
                for (int j = 0; j < P; ++j) st.k[b][j] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(codes + 1024 * j) + lane);
#pragma unroll
                for (int j = 0; j < P; ++j) st.v[b][j] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(codes + kBlock * D + 1024 * j) + lane);
            }
        };
        auto work = [&](const Stage<D> &st, const int (&page)[2], int s) {
            float x[RB][2][4], lv[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int key = 16 * (2 * s + b);
                const float ks = h2f((uint16_t)(st.scales[b] & 0xffffu)) * a.scale;
                lv[b] = __builtin_amdgcn_logf(h2f((uint16_t)(st.scales[b] >> 16)));
                v4f acc[RB];
#pragma unroll
                for (int k = 0; k < RB; ++k) acc[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int m = 0; m < D / 32; ++m) {
                    const v8h w = codes_to_half(st.k[b][m / 2][2 * (m & 1)], st.k[b][m / 2][2 * (m & 1) + 1]);
#pragma unroll
                    for (int k = 0; k < RB; ++k) acc[k] = mfma_h(w, q[k][m], acc[k]);
                }
                const bool there = page[b] >= 0 && 2 * s + b < blocks;
                if (there && key + 15 <= sees_first) {
#pragma unroll
                    for (int k = 0; k < RB; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[k][b][i] = acc[k][i] * ks;
                } else {
                    if (!there) lv[b] = 0.0f;
#pragma unroll
                    for (int k = 0; k < RB; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[k][b][i] = there && key + 4 * g + i <= limit[k] ? acc[k][i] * ks : -INFINITY;
                }
            }
            take(r, x, lv[0], lv[1], [&](int t) { return codes_to_half(st.v[0][t / 4][t % 4], st.v[1][t / 4][t % 4]); });
        };
        int s = first + mine;
        if (s < done) {
            constexpr int N = 2;                         // steps in registers (three or four: no faster)
            Stage<D> st[N];
            int page[N][2], next[2];
#pragma unroll
            for (int u = 0; u < N; ++u) pages(page[u], s + u * every);
#pragma unroll
            for (int u = 0; u < N - 1; ++u) load(st[u], page[u], s + u * every);
            for (bool more = true; more;) {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    pages(next, s + N * every);
                    load(st[(u + N - 1) % N], page[(u + N - 1) % N], s + (N - 1) * every);
                    asm volatile("" ::: "memory");                           // (else the loads sink to their use)
                    __builtin_amdgcn_sched_barrier(0);
                    work(st[u], page[u], s);
                    page[u][0] = next[0];
                    page[u][1] = next[1];
                    s += every;
                    if (s >= done) {
                        more = false;
                        break;
                    }
                }
            }
        }
        // the unfinished block's tokens, in fp16, with the tile's last step
        const int tail = p.length - full * kBlock;
        if (last == p.steps && tail > 0 && seen > full * kBlock && (alone || wave == (p.steps - 1 - first) % kWaves)) {
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
            if (alone) {
                if (16 * k + i16 < rows) {
#pragma unroll
                    for (int t = 0; t < D / 16; ++t)
                        store_row(a, p.begin, p.tile * ROWS + 16 * k + i16, head, D, 16 * t + 4 * g, r.o[k][t], l);
                }
                continue;
            }
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

// Many rows: 128 of a tile, 32 a wavefront, and 64 keys a stage that all of them share.  The codes of the next stage are asked
// for while this one is worked on, and put into LDS as fp16 behind it (two buffers), in the order in which the 32x32x16 MFMAs
// of the prompts' kernel read them, so that a code is turned once for 128 rows.  Heads of 64 take 128 keys a stage, for which
// LDS and registers are there (three chunks of 400 tokens of 30 heads over 6, behind up to 9000: 90 -> 85 us).  A block of 16
// keys is half of a result's registers: its scales are the same in all lanes.  As there, the maximum m that is taken off is
// raised only where a lane's weights of a block add up to more than 2^15.
//
// Bound by the vector unit and the matrix pipe, one after the other in both wavefronts of a SIMD: a stage is 32 matrix instructions
// of 32 cycles a wavefront, beside, with heads of 64 (128 keys), about 470 vector ones -- scores weighed, and codes turned and
// placed, which only 128 rows share -- of four cycles (eight for an exponential): 63 % and 28 % busy there.  With heads of 128
// (64 keys) 0.80 PFLOP/s (512 new tokens each of three sequences of up to 8192, 64 heads over 8, 284 us), against 0.51.  Codes
// put into LDS between the matrix instructions, not behind them: slower (95 -> 103 us, at 64 keys a stage).
constexpr int kStageWaves = 4, kStageRows = 32 * kStageWaves;
constexpr int stage_keys(int D) { return D == 64 ? 128 : 64; }
constexpr float kStageShift = 9.0f, kMost = 32768.0f;

__device__ __forceinline__ v16f mfma_h(v8h a, v8h b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <int D>
__global__ __launch_bounds__(64 * kStageWaves) __attribute__((amdgpu_waves_per_eu(2))) void chunk_kernel(CachedArgs a)
{
    typedef CacheBlock<D> B;
    constexpr int KEYS = stage_keys(D), BLOCKS = KEYS / kBlock;
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    // keys: a line of D channels each; values: a line of KEYS keys for each channel, chunk 2 b + half of 16 bytes holding keys
    // 16 b + 4 half + {0 .. 3, 8 .. 11}; chunks XORed by the line, so that sixteen lines' same chunk meets every bank once
    constexpr int LINE = 2 * D, VLINE = 2 * KEYS, KSTAGE = KEYS * LINE, VSTAGE = D * VLINE;
    constexpr int TASKS = BLOCKS * D / 64 / kStageWaves;           // planes of 1 KiB of a wavefront, of keys and of values
    static_assert(TASKS >= 1, "every wavefront has a plane");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][KSTAGE + VSTAGE];
    __shared__ unsigned tail_top[kStageWaves];                     // of the unfinished block's values: largest magnitudes (bits),
    __shared__ int tail_lift;                                      // and by how many powers of two they are larger in LDS
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, i32 = lane & 31;
    // workgroups 8 apart share an XCD and its L2: each XCD has neighbouring parts, which read the same keys at about the same time
    const int xcd = blockIdx.x % 8, per = gridDim.x / 8, more = gridDim.x % 8;
    const int id = xcd * per + min(xcd, more) + (int)blockIdx.x / 8, head = divide(id, a.by_parts), index = id - head * a.parts;
    auto key_swizzle = [](int line) { return D == 128 ? line & 15 : (line >> 1) & 7; };
    auto value_swizzle = [](int line) { return KEYS == 128 ? line & 15 : (line >> 1) & 7; };
    Steps<kStageRows, KEYS> all(a);
    const int total = all.all(), width = all.width();
    int at = index * width;
    const int stop = min(at + width, total);
    while (at < stop) {
        const Place p = all.find(at);
        if (p.id < 0) return;
        const int end = min(stop, p.first + p.steps);
        const int first = at - p.first, last = end - p.first;            // stages of the tile
        const bool whole = first == 0 && last == p.steps;
        const int row0 = p.tile * kStageRows, rows = min(kStageRows, p.n * a.group - row0);
        const int row = row0 + min(32 * wave + i32, rows - 1), token = divide(row, a.by_group), limit = p.length - p.n + token;
        const bool some = 32 * wave < rows;
        const int w_last = row0 + min(32 * wave + 31, rows - 1);
        const int sees_first = p.length - p.n + divide(row0 + 32 * wave, a.by_group);
        const int sees_last = some ? p.length - p.n + divide(w_last, a.by_group) : -1;
        const int seen = p.length - p.n + divide(row0 + rows - 1, a.by_group) + 1;       // keys that any of the rows sees
        const int full = p.length / kBlock, tail = p.length - full * kBlock;
        const int blocks = min(full, (max(seen, 0) + kBlock - 1) / kBlock);      // in pages
        const bool has_tail = tail > 0 && seen > full * kBlock;
        const int done = min(last, (blocks + (has_tail ? 1 : 0) + BLOCKS - 1) / BLOCKS);
        const uint16_t *recent = B::recent(c, p.id, head);
        v8h q[D / 16];
        {
            const uint16_t *from = a.q + (size_t)(p.begin + token) * a.q_stride + (size_t)(head * a.group + row - token * a.group) * D;
#pragma unroll
            for (int m = 0; m < D / 16; ++m) q[m] = *reinterpret_cast<const v8h *>(from + 16 * m + 8 * half);
        }
        v4u k_codes[TASKS], v_codes[TASKS];
        // lane b, b < BLOCKS: the table's entry and the scales of block b of a stage, and whether the block is there
        int pages = -1;
        unsigned scales = 0u;
        bool there = false;
        const int mine = lane & (BLOCKS - 1);
        // planes of a stage: number n of a wavefront is plane n + TASKS wave, plane j of block b being D / 64 b + j
        auto block_of = [&](int n) { return (TASKS * wave + n) / (D / 64); };
        auto ask_pages = [&](int s) {
            pages = c.table[(size_t)p.id * c.max_pages + (max(min(BLOCKS * s + mine, blocks - 1), 0) >> c.shift)];
        };
        auto fetch = [&](int s) {                    // (after ask_pages of the same stage)
            const bool valid = pages >= 0 && pages < c.pages;
            const int good = valid ? pages : 0;
            there = valid && BLOCKS * s + mine < blocks;
#pragma unroll
            for (int n = 0; n < TASKS; ++n) {
                const int block = min(BLOCKS * s + block_of(n), max(blocks - 1, 0)), plane = (TASKS * wave + n) % (D / 64);
                const uint8_t *codes = B::codes(c, __builtin_amdgcn_readlane(good, block_of(n)), head, block);
                k_codes[n] = reinterpret_cast<const v4u *>(codes + 1024 * plane)[lane];
                v_codes[n] = reinterpret_cast<const v4u *>(codes + kBlock * D + 1024 * plane)[lane];
            }
            scales = *B::scales(c, good, head, there ? BLOCKS * s + mine : 0);
        };
        auto put = [&](int s) {
            uint8_t *ks = lds[s & 1], *vs = ks + KSTAGE;
            const int g = lane >> 4, i = lane & 15;
#pragma unroll
            for (int n = 0; n < TASKS; ++n) {
                const int b = block_of(n), plane = (TASKS * wave + n) % (D / 64), line = kBlock * b + i;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<v8h *>(ks + line * LINE + 16 * ((8 * plane + 4 * h + g) ^ key_swizzle(line))) =
                        codes_to_half(k_codes[n][2 * h], k_codes[n][2 * h + 1]);
#pragma unroll
                for (int t = 0; t < 4; t += 2) {
                    union {
                        v8h v;
                        v2u u[2];
                    } w;
                    w.v = codes_to_half(v_codes[n][t], v_codes[n][t + 1]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int channel = 64 * plane + 16 * (t + h) + i;
                        *reinterpret_cast<v2u *>(vs + channel * VLINE + 16 * ((2 * b + (g & 1)) ^ value_swizzle(channel)) + 8 * (g >> 1)) = w.u[h];
                    }
                }
            }
        };
        // the unfinished block's tokens over what was put in its place
        auto put_tail = [&](int s) {
            uint8_t *ks = lds[s & 1], *vs = ks + KSTAGE;
            const int b = full - BLOCKS * s;
            for (int u = threadIdx.x; u < kBlock * (D / 8); u += 64 * kStageWaves) {
                const int t = u / (D / 8), chunk = u % (D / 8), line = kBlock * b + t;
                v4u w = {0u, 0u, 0u, 0u};
                if (recent && t < tail) w = *reinterpret_cast<const v4u *>(recent + B::recent_key(full * kBlock + t, 8 * chunk));
                *reinterpret_cast<v4u *>(ks + line * LINE + 16 * (chunk ^ key_swizzle(line))) = w;
            }
            // values below 64 larger by a power of two, exactly, which their scale takes back: with a scale of 1 beside the
            // small ones of full blocks, weights of a stage would be taken off a maximum that no product reaches
            constexpr int QUADS = 4 * D / (64 * kStageWaves);                // of a channel's four tokens, a thread
            uint16_t w[QUADS][4];
            unsigned most = 0u;
#pragma unroll
            for (int n = 0; n < QUADS; ++n) {
                const int u = threadIdx.x + 64 * kStageWaves * n, g = u & 3, channel = u >> 2;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[n][e] = 0; // (behind the last token anything may lie)
                if (recent) {
                    const uint16_t *from = recent + B::recent_value(full * kBlock + 4 * g, channel);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (4 * g + e < tail) w[n][e] = from[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) most = max(most, w[n][e] & 0x7fffu);
            }
            most = wave_max_bits(most);
            if (lane == 0) tail_top[wave] = most;
            __syncthreads();
#pragma unroll
            for (int n = 0; n < kStageWaves; ++n) most = max(most, tail_top[n]);
            const int lift = most == 0u ? 0 : max(7 - __builtin_amdgcn_frexp_expf(h2f((uint16_t)most)), 0);
            if (threadIdx.x == 0) tail_lift = lift;
            const float larger = __uint_as_float((unsigned)(127 + lift) << 23);
#pragma unroll
            for (int n = 0; n < QUADS; ++n) {
                const int u = threadIdx.x + 64 * kStageWaves * n, g = u & 3, channel = u >> 2;
                *reinterpret_cast<v2u *>(vs + channel * VLINE + 16 * ((2 * b + (g & 1)) ^ value_swizzle(channel)) + 8 * (g >> 1)) =
                    v2u{pack_h2(h2f(w[n][0]) * larger, h2f(w[n][1]) * larger), pack_h2(h2f(w[n][2]) * larger, h2f(w[n][3]) * larger)};
            }
        };
        v16f o[D / 32];
        float top = kNothing, sum = 0.0f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
        auto prepare = [&](int s) {                  // stage s, asked for, into its buffer
            put(s);
            if (has_tail && full / BLOCKS == s) {
                __syncthreads();
                put_tail(s);
            }
        };
        __syncthreads();                             // (the tile before is done with the buffers)
        if (first < done) {
            ask_pages(first);
            fetch(first);
            ask_pages(first + 1);
            prepare(first);
        }
#pragma unroll
        for (int m = 0; m < D / 16; ++m) asm volatile("" : "+v"(q[m]));  // (they are waited for here, not in the loop)
        for (int s = first; s < done; ++s) {
            const unsigned sc = there ? scales : 0u;
            __syncthreads();                         // the stage is there, and everyone is done with the one before
            if (s + 1 < done) {
                fetch(s + 1);
                ask_pages(s + 2);
            }
            if (some && KEYS * s <= sees_last) {
                const uint8_t *ks = lds[s & 1], *vs = ks + KSTAGE;
                v16f x[BLOCKS / 2];
                {
                    constexpr int AHEAD = 4;         // operands asked for ahead of the instruction that takes them
                    v8h ring[AHEAD];
                    constexpr int U = BLOCKS / 2;
                    auto key_part = [&](int n) {     // n: keys 32 (n % U) .., channels 16 (n / U) ..
                        const int line = 32 * (n % U) + i32;
                        return *reinterpret_cast<const v8h *>(ks + line * LINE + 16 * ((2 * (n / U) + half) ^ key_swizzle(line)));
                    };
#pragma unroll
                    for (int n = 0; n < AHEAD; ++n) ring[n] = key_part(n);
#pragma unroll
                    for (int u = 0; u < BLOCKS / 2; ++u)
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[u][i] = 0.0f;
#pragma unroll
                    for (int n = 0; n < D / 16 * U; ++n) {
                        x[n % U] = mfma_h(ring[n % AHEAD], q[n / U], x[n % U]);
                        if (n + AHEAD < D / 16 * U) ring[n % AHEAD] = key_part(n + AHEAD);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                // the blocks' scales: of keys, with the call's; of values, their logarithm and what takes it back
                float scale[BLOCKS], lv[BLOCKS], back[BLOCKS];
                {
                    const bool code = sc != 0u, ring = has_tail && recent && BLOCKS * s + mine == full;
                    // (a scale is not zero, also where the product is below the smallest number: hidden scores are -inf times it)
                    const float k = code ? fmaxf(h2f((uint16_t)(sc & 0xffffu)) * a.scale, 1e-38f) : a.scale;
                    const float v = code ? __builtin_amdgcn_logf(h2f((uint16_t)(sc >> 16))) : ring ? -(float)tail_lift : -INFINITY;
                    const float inv = code || ring ? __builtin_amdgcn_exp2f(-v) : 0.0f;
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) {
                        scale[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k), b));
                        lv[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), b));
                        back[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(inv), b));
                    }
                }
                if (KEYS * (s + 1) - 1 > sees_first) {
#pragma unroll
                    for (int u = 0; u < BLOCKS / 2; ++u)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (KEYS * s + 32 * u + 8 * (i >> 2) + 4 * half + (i & 3) > limit) x[u][i] = -INFINITY;
                }
                v8h w[BLOCKS / 2][2];
                float part[BLOCKS];
                __builtin_amdgcn_s_setprio(0);
                auto weights = [&] {
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) {
                        const float less = top - kStageShift - lv[b];
                        part[b] = 0.0f;
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b / 2][8 * (b & 1) + i], scale[b], -less));
                            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b / 2][8 * (b & 1) + i + 1], scale[b], -less));
                            part[b] += e0;
                            part[b] += e1;
                            const v2h h = __builtin_convertvector((v2f{e0, e1}), v2h);
                            w[b / 2][b & 1][i] = h[0];
                            w[b / 2][b & 1][i + 1] = h[1];
                        }
                        asm volatile("" : "+v"(w[b / 2][b & 1]));    // (in fp16 from here on, not once all are weighed)
                    }
                };
                bool above = s == first;             // (at the first stage every score is far above m)
                if (!above) {
                    weights();
                    float most = part[0];
#pragma unroll
                    for (int b = 1; b < BLOCKS; ++b) most = fmaxf(most, part[b]);
                    above = __any(most > kMost);
                }
                if (above) {
                    float best = kNothing;
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int i = 0; i < 8; ++i) best = fmaxf(best, x[b / 2][8 * (b & 1) + i] * scale[b] + lv[b]);
                    auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(best), __float_as_uint(best), false, false);
                    const float next = fmaxf(top, fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
                    const float f = __builtin_amdgcn_exp2f(top - next);
                    top = next;
                    sum *= f;
#pragma unroll
                    for (int t = 0; t < D / 32; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[t][i] *= f;
                    weights();
                }
#pragma unroll
                for (int b = 0; b < BLOCKS; b += 2) sum += part[b] * back[b] + part[b + 1] * back[b + 1];
                {
                    __builtin_amdgcn_s_setprio(1);           // (matrix instructions first)
                    constexpr int T = D / 32, AHEAD = 4;
                    v8h ring[AHEAD];
                    auto value_part = [&](int n) {   // n: keys 16 (n / T) .., channels 32 (n % T) ..
                        const int channel = 32 * (n % T) + i32;
                        return *reinterpret_cast<const v8h *>(vs + channel * VLINE + 16 * ((2 * (n / T) + half) ^ value_swizzle(channel)));
                    };
#pragma unroll
                    for (int n = 0; n < AHEAD; ++n) ring[n] = value_part(n);
#pragma unroll
                    for (int n = 0; n < BLOCKS * T; ++n) {
                        o[n % T] = mfma_h(ring[n % AHEAD], w[n / T / 2][n / T & 1], o[n % T]);
                        if (n + AHEAD < BLOCKS * T) ring[n % AHEAD] = value_part(n + AHEAD);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            if (s + 1 < done) prepare(s + 1);
        }
        {
            auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
            sum = __uint_as_float(y[0]) + __uint_as_float(y[1]);
        }
        if (32 * wave + i32 < rows) {
            float *part = a.part + ((((size_t)head * a.parts + index) * 2 + (first == 0 ? 1 : 0)) * kStageRows + 32 * wave + i32) * (D + 4);
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = 32 * t + 8 * i + 4 * half;
                    const v4f y = {o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
                    if (whole)
                        store_row(a, p.begin, row, head, D, d, y, sum);
                    else
                        *reinterpret_cast<v4f *>(part + d) = y;
                }
            if (!whole && half == 0) {
                part[D] = top;
                part[D + 1] = sum;
            }
        }
        at = end;
    }
}

// Tiles that several workgroups took: their shares in order.  Wavefront (i, group) has some rows, one after the other, of
// the tile that begins in part i and does not end there, if there is one: with many rows 256 / D of them, a row of few shares
// each; with few rows one, whose shares its lanes take in turn.
template <int D, int ROWS, int KEYS>
__global__ __launch_bounds__(64) void join_kernel(CachedArgs a, Divider by_groups)
{
    constexpr int Q = D / 4, SHARES = ROWS == kStageRows ? 1 : 64 / Q, HIGH = 64 / Q / SHARES, U = SHARES == 1 ? 4 : 8;    // Q: lanes of a row
    __shared__ __attribute__((aligned(16))) float red[SHARES][D];
    __shared__ float stat[SHARES][2];
    const CacheArgs &c = a.c;
    const int all_groups = divide(blockIdx.x, c.by_kv), head = blockIdx.x - all_groups * c.kv_heads;
    const int index = divide(all_groups, by_groups), group = all_groups - index * (int)by_groups.d;
    Steps<ROWS, KEYS> all(a);
    const int total = all.all(), width = all.width();
    const int start = index * width, stop = start + width;
    if (stop >= total || (ROWS != kStageRows && all.tiles_alone())) return;
    const Place p = all.find(stop);
    if (p.id < 0 || p.first >= stop || p.first < start) return;
    const int rows = p.n * a.group - p.tile * ROWS;
    const int d = threadIdx.x % Q * 4, share = SHARES == 1 ? 0 : threadIdx.x / Q;
    const int row = SHARES == 1 ? HIGH * group + threadIdx.x / Q : group;
    if (HIGH * group >= rows) return;
    const int last = (p.first + p.steps - 1) / width;            // the last part that has some of the tile
    const float *part = a.part + (((size_t)head * a.parts) * 2 * ROWS + min(row, rows - 1)) * (D + 4);
    auto of = [&](int i) { return part + ((size_t)i * 2 + (i == index ? 1 : 0)) * ROWS * (D + 4); };
    float m = kNothing, l = 0.0f;
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](float mi, float li, v4f oi) {
        const float top = fmaxf(m, mi), f = __builtin_amdgcn_exp2f(m - top), fi = __builtin_amdgcn_exp2f(mi - top);
        m = top;
        l = l * f + li * fi;
        o = o * f + oi * fi;
    };
    for (int i = index + share; i <= last; i += U * SHARES) {    // (U loads set out together)
        float mi[U], li[U];
        v4f oi[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float *from = of(min(i + u * SHARES, last));
            oi[u] = *reinterpret_cast<const v4f *>(from + d);
            mi[u] = from[D];
            li[u] = from[D + 1];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * SHARES <= last) add(mi[u], li[u], oi[u]);
    }
    if (SHARES > 1) {
        stat[share][0] = m;                                      // (every lane of a share writes the same)
        stat[share][1] = l;
        *reinterpret_cast<v4f *>(&red[share][d]) = o;
        __syncthreads();
        if (share != 0) return;
#pragma unroll
        for (int i = 1; i < SHARES; ++i) add(stat[i][0], stat[i][1], *reinterpret_cast<const v4f *>(&red[i][d]));
    }
    if (row < rows) store_row(a, p.begin, p.tile * ROWS + row, head, D, d, o, l);
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Rows of a tile: as many as a sequence has on average; 128, which go through LDS, where tiles of 32 would read the cache three
// times, and with heads of 64 twice (us with 32 / 128 a tile: heads of 128, 64 rows, 16 sequences of 1000 tokens of 8 key heads
// 20.5 / 30, of 4000 45 / 53, 8 of 4000 of 32 96 / 85, 72 rows, 16 of 4000 of 8, 85 / 56; heads of 64, 35 rows, 40 of 2000 of
// 6, 42.5 / 34.8, 50 rows, 10 of 3000 of 12, 35 / 32; with 16 / 32 a tile 20 rows, 8 of 4000 of 32 key heads, 86 / 51).
// The host knows the average only, so a batch of unlike sequences has one kind of tile: a chunk of 512 tokens beside 63 single tokens
// (4000 to 8000 tokens cached, 64 heads over 8) takes 277 us, the two apart 104 + 134; a chunk of 256 beside them 225, apart 62 + 134.
int tile_rows(int M, int count, int group, int head_dim)
{
    const long rows = (long)M * group / count;
    return rows > (head_dim == 64 ? 32 : 64) ? kStageRows : rows > 16 ? 32 : 16;
}

// Workgroups of a key head: one a CU in all of the streaming kernel, of eight wavefronts, two of the other.  (Streaming, 1 x 8
// or 2 x 4 wavefronts a CU, us: 8 rows of 8192 tokens of 64 heads over 8 16.6 / 19.2, 16 sequences of 4000 45 / 60, 48 of up to
// 8192 80 / 80; two tiles of 32 rows each, 8 sequences of 4000 of 32 key heads, 99 / 81.)  Counts of key heads that leave CUs
// over lose nothing: 16 sequences of 2000 tokens of 64, 80, 96 and 128 key heads (256, 240, 192 and 256 workgroups) run at 5.9, 5.9,
// 6.5 and 6.5 TB/s.
int parts_for(int kv_heads, int rows)
{
    const int parts = (rows == kStageRows ? 512 : 256) / kv_heads;
    return parts < 1 ? 1 : parts;
}

size_t workspace_for(int M, int count, int heads, int kv_heads, int head_dim)
{
    const int rows = tile_rows(M, count, heads / kv_heads, head_dim);
    return (size_t)parts_for(kv_heads, rows) * kv_heads * 2 * rows * (head_dim + 4) * 4;
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
    // (steps are counted with 32 bits)
    const long tiles = (long)M * (heads / kv) / 16 + seqs->count, steps = (long)seqs->max_pages * cache->page / (2 * kBlock) + 1;
    if ((long)M * (heads / kv) >= (1L << 30) || tiles * steps >= (1L << 31)) return FLEXQ_ESHAPE;
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
    const int rows = tile_rows(M, seqs->count, a.group, D), most = (long)M * a.group < rows ? M * a.group : rows;
    a.parts = parts_for(kv, rows);
    a.by_group = divider(a.group);
    a.by_parts = divider(a.parts);
    // (a part of a few steps costs more in the join than it saves: 11 rows of 8192 tokens 21.5 us, with a step at least 27)
    a.least = rows == kStageRows ? 256 / stage_keys(D) : 8;
    const int groups = rows == kStageRows ? (most + 256 / D - 1) / (256 / D) : most;     // of rows of a tile
    if ((long)a.parts * kv * groups >= (1L << 26)) return FLEXQ_ESHAPE;  // 64 threads each, 2^32 a launch
    hipStream_t st = (hipStream_t)stream;
    auto run = [&](auto kern, int waves, auto join) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(a.parts * kv)), dim3(64 * waves), 0, st, a);
        if (hipGetLastError() != hipSuccess) return FLEXQ_EHIP;
        if (a.parts > 1) hipLaunchKernelGGL(join, dim3((unsigned)(a.parts * kv * groups)), dim3(64), 0, st, a, divider(groups));
        return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
    };
    if (D == 128)
        return rows == kStageRows ? run(chunk_kernel<128>, kStageWaves, join_kernel<128, kStageRows, stage_keys(128)>)
               : rows == 32       ? run(cached_kernel<128, 2>, kWaves, join_kernel<128, 32, 2 * kBlock>)
                                  : run(cached_kernel<128, 1>, kWaves, join_kernel<128, 16, 2 * kBlock>);
    return rows == kStageRows ? run(chunk_kernel<64>, kStageWaves, join_kernel<64, kStageRows, stage_keys(64)>)
           : rows == 32       ? run(cached_kernel<64, 2>, kWaves, join_kernel<64, 32, 2 * kBlock>)
                              : run(cached_kernel<64, 1>, kWaves, join_kernel<64, 16, 2 * kBlock>);
}

}  // extern "C"
#pragma GCC visibility pop
