// Rows that choose their own weights: the choice (scores of the experts -> the k best and their
// weights) and the grouping of rows by what they chose, which the experts' products and the
// adapters of a batch walk.
//
// Mathematics.  Scores s = softmax(l) or sigmoid(l); the choice is by c = s + bias, first (groups
// > 1) among groups by the sum of a group's best one or two c, then among the experts of the kept
// groups; the weights are the chosen s.  Two experts whose c are close must not change places with
// the rounding of an exponential.  Where nothing is added to a score, s grows with l, and l itself,
// exact, is compared (no exponential but the chosen ones').  Else c is made in fp32, good to 2^-21 of
// its size (at least 1), and where two that follow each other come closer than twice that, they are
// made again in 64 bits: of sigmoids the chosen and whoever is that close behind them alone, a lane
// each (one token in a thousand); all, through the same steps, where that does not suffice.
//
// Sixteen lanes a token, four tokens a wavefront, expert e in lane e / V: a tie is won by the lowest
// index.  Values are compared as unsigned keys (the bits of a float or double, so mapped that they
// order like the values, and 0 for what cannot be chosen): a round is each lane's best, the DPP
// maximum over the row, and taking that one out.  (A wavefront a token, with its four keys a lane of
// 256 experts, spent as many instructions a round on one token: 32768 tokens of 256 by logit 35 us
// a call, now 25.)
//
// What bounds it: not the 8 MB of logits (2 us), but the rounds, each a chain that waits for the one
// before and looks at all of a lane's keys.  Sigmoids of 256 experts with a bias, 4 of 8 groups, 8 chosen,
// are four rounds over groups and nine over experts: 14 us for 256 tokens, one pass of every wavefront; 22
// for 8192, where instructions count too, at two wavefronts a SIMD (the second look, inlined, takes the
// registers to 256); 49 for 32768.  333 of 60 by softmax 4.2; one token of 8 3.3 with its grouping, a launch
// and two trips to memory.  More than 256 experts spill registers.
//
// Grouping is a counting sort, stable, so that equal inputs give equal orders: every block counts
// its slots per bucket (bucket `count` holds the rows without one), and a second launch adds up the
// counts of the blocks before it and hands out places -- rank within a wavefront by ballots over the
// bits of the bucket, wavefronts and blocks by their counts.  No atomics but LDS counters, whose sum
// has no order.  Few slots: everything in the one block of one launch.  The second launch takes 9.3 us
// for 65536 slots over 256 experts and 4.9 for 1665 over 60: a chain of barriers and trips to L2 (all
// blocks' counts, 132 KB, are read by every block; bytes to memory 0.8 MB).
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "producer_math.h"
#include "row_groups.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxExperts = FLEXQ_MAX_EXPERTS;          // buckets: one more
constexpr int kMaxBlocks = 256;                          // blocks of a launch over many slots: one a CU
constexpr int kMostRows = 1 << 28;                       // every block reads all blocks' counts: 8192 of them
constexpr int kMostSlots = 32768;                        // of a block: its counts are 16 bits
constexpr int kOneBlock = 1024;                          // slots that one block sorts by itself
constexpr int kRouteThreads = 512, kRouteWaves = 8;      // of a block of the routing kernel
constexpr int kRouteTokens = 4 * kRouteWaves;            // ... and what it takes at a time

struct RouteArgs {
    const void *logits;
    const float *bias;
    int M, E, k, sigmoid, groups, top_groups, group_top, renormalise;
    float scale;
    unsigned long long group_inv;   // e / group size = (e * group_inv) >> 32
    int group_size, group_shift; // 1 << group_shift lanes share a group's scan
    int32_t *experts;
    float *weights;
    int per_block;               // tokens of a block
    int32_t *order, *offsets;    // one block only, or null
    uint16_t *hist;              // [blocks][pairs_of(E + 1) * 2], or null
};

// bytes of the routing kernel's tables in LDS: counts, bases, sums, slots
__host__ __device__ constexpr int route_tables(int buckets)
{
    return (((kRouteWaves + 1) * buckets + kRouteWaves + kRouteThreads) * 4 + 15) / 16 * 16;
}

// place of a token's key e in LDS: a word more in sixteen, so that lanes sixteen or 32 apart meet in no bank
__host__ __device__ constexpr int padded(int e) { return e + (e >> 4); }

// words of a block's counts, two buckets each
__host__ __device__ constexpr int pairs_of(int buckets) { return (buckets + 1) / 2; }

__device__ __forceinline__ unsigned key_of(float v)
{
    const unsigned b = __float_as_uint(v + 0.0f);       // -0 and 0 are one value
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long key_of(double v)
{
    const unsigned long long b = __double_as_longlong(v + 0.0);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double value_of(unsigned long long key)
{
    return __longlong_as_double(key >> 63 ? key ^ 0x8000000000000000ull : ~key);
}
__device__ __forceinline__ float value_of(unsigned key)
{
    return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key);
}

// Over the sixteen lanes of a row, every lane with its row's result.
template <class Op>
__device__ __forceinline__ unsigned row_all(unsigned v, const Op &op)
{
#define FLEXQ_ROW(ctrl) (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false)
    v = op(v, FLEXQ_ROW(0x128));      // row_ror:8, 4, 2, 1
    v = op(v, FLEXQ_ROW(0x124));
    v = op(v, FLEXQ_ROW(0x122));
    v = op(v, FLEXQ_ROW(0x121));
#undef FLEXQ_ROW
    return v;
}
__device__ __forceinline__ unsigned row_best(unsigned k)
{
    return row_all(k, [](unsigned a, unsigned b) { return max(a, b); });
}
template <class Op>
__device__ __forceinline__ float row_all_f(float v, const Op &op)
{
    return __uint_as_float(row_all(__float_as_uint(v), [&](unsigned a, unsigned b) {
        return __float_as_uint(op(__uint_as_float(a), __uint_as_float(b)));
    }));
}
__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// The best of a row's keys: its index l V + v for lane l of the row (ties: the lowest; -1: there is none), its
// key in `wins`.  It is taken out.
template <int V>
__device__ __forceinline__ int pick(unsigned (&key)[V], int lane, unsigned &wins)
{
    unsigned best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    wins = row_best(best);
    const unsigned hits = (unsigned)(__ballot(best == wins) >> (lane & 48)) & 0xffffu;
    const int first = __builtin_ctz(hits | 0x10000u);
    // (its place in the lane by a minimum over all of them and taken out by number: a chain of "found
    // already" through the keys is 16 trips to the scalar unit and back)
    unsigned place[V];
#pragma unroll
    for (int v = 0; v < V; ++v) place[v] = key[v] == wins ? (unsigned)v : (unsigned)V;
#pragma unroll
    for (int w = 1; w < V; w *= 2)
#pragma unroll
        for (int v = 0; v + w < V; v += 2 * w) place[v] = min(place[v], place[v + w]);
    const unsigned at = (lane & 15) == first ? place[0] : (unsigned)V;
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = at == (unsigned)v ? 0u : key[v];
    const unsigned found = row_all(at, [](unsigned a, unsigned b) { return min(a, b); });
    return wins == 0 ? -1 : first * V + (int)found;
}

// Places of a block's slots, at most one a thread, in the order.  id: this thread's slot's bucket, 0 .. count (have:
// it has one); wcount: LDS [WAVES][count + 1]; base[b]: LDS, the next free place of bucket b, moved on.
template <int WAVES>
__device__ __forceinline__ void hand_out(int id, bool have, int slot, int count, int *wcount, int *base, int32_t *order)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, buckets = count + 1;
    for (int i = tid; i < WAVES * buckets; i += 64 * WAVES) wcount[i] = 0;
    __syncthreads();
    unsigned long long same = __ballot(have);
    for (int bit = 1; bit <= count; bit <<= 1) {
        const unsigned long long b = __ballot((id & bit) != 0);
        same &= id & bit ? b : ~b;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    if (have && rank == 0) wcount[wave * buckets + id] = __popcll(same);
    __syncthreads();
    for (int b = tid; b < buckets; b += 64 * WAVES) {
        int c[WAVES], at = base[b];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) c[w] = wcount[w * buckets + b];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            wcount[w * buckets + b] = at;
            at += c[w];
        }
        base[b] = at;
    }
    __syncthreads();
    if (have) order[wcount[wave * buckets + id] + rank] = slot;
    __syncthreads();
}

// base[b] = sum of total[0 .. b - 1] + before[b]; offsets (one block) the sums alone.  total, before: LDS (before
// may be null: 0), two buckets a thread.
template <int WAVES>
__device__ __forceinline__ void begin_buckets(const int *total, const int *before, int count, int *base, int *wave_sums,
                                              int32_t *offsets)
{
    static_assert(2 * 64 * WAVES > kMaxExperts, "two buckets a thread");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int t[2], b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool in = 2 * tid + i <= count;
        t[i] = in ? total[2 * tid + i] : 0;
        b[i] = in && before ? before[2 * tid + i] : 0;
    }
    const int sum = wave_scan(t[0] + t[1]);
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    int ahead = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int s = wave_sums[w];
        if (w < wave) ahead += s;
    }
    int begin = ahead + sum - t[0] - t[1];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (2 * tid + i <= count) {
            base[2 * tid + i] = begin + b[i];
            if (offsets) offsets[2 * tid + i] = begin;   // offsets[count] = the rows that have a bucket
        }
        begin += t[i];
    }
    __syncthreads();
}

constexpr float kLargest = 3.4028234663852886e38f;
constexpr float kClose = 0x1p-20f;       // twice the fp32 scores' error, of their size or 1

__device__ __forceinline__ bool near(unsigned above, unsigned below)
{
    const float x = value_of(above), y = value_of(below);
    return !(x - y > kClose * fmaxf(1.0f, fmaxf(fabsf(x), fabsf(y))));
}

// Keeps the keys of the top_groups best groups.  unsure: set where fp32 does not tell a group left out from one kept: c
// is off by 2^-21 of its size, at least of 1 -- its own, not that of a sum in which two large ones cancel -- so half a
// group's worth lies within 1.5 2^-21 of the larger of the c in it (both of them, and the rounding of the sum and of the
// interval's ends; halves do not overflow).  G: groups a lane of the row keeps (1: up to 16 groups, each scanned by
// as many lanes as there are for it).
template <bool BY_LOGIT, int V, int G>
__device__ __forceinline__ void keep_groups(const RouteArgs &a, unsigned (&key)[V], unsigned *scratch, int lane, bool &unsure)
{
    const int l = lane & 15;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (l * V + v < a.E) scratch[padded(l * V + v)] = key[v];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (a wavefront's own part of LDS: no barrier)
    const int shift = G == 1 ? a.group_shift : 0, P = 1 << shift;     // P lanes a group
    const bool pair = !BY_LOGIT && a.group_top == 2;
    unsigned of_group[G];
    float half[G], off[G];                                   // (off < 0: there is none)
#pragma unroll
    for (int q = 0; q < G; ++q) {
        const int g = G == 1 ? l >> shift : l * G + q;
        unsigned first = 0, second = 0;
        if (g < a.groups)
            for (int i = l & (P - 1); i < a.group_size; i += P) {
                const unsigned c = scratch[padded(g * a.group_size + i)];
                second = max(second, min(first, c));
                first = max(first, c);
            }
        if (G == 1)
            for (int d = 1; d < P; d <<= 1) {
                const unsigned f = __shfl_xor(first, d, 64), s = __shfl_xor(second, d, 64);
                second = max(max(second, s), min(first, f));
                first = max(first, f);
            }
        const float x = value_of(first), y = pair && second != 0 ? value_of(second) : 0.0f;
        of_group[q] = (l & (P - 1)) != 0 || first == 0 ? 0u : pair && second != 0 ? key_of(x + y) : first;
        half[q] = 0.5f * x + 0.5f * y;
        off[q] = first != 0 ? 0.75f * kClose * fmaxf(1.0f, fmaxf(fabsf(x), fabsf(y))) : -1.0f;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read before the next tokens' keys come)
    unsigned long long kept = 0;
    unsigned wins;
    for (int i = 0; i < a.top_groups; ++i) {
        const int g = pick(of_group, lane, wins);
        if (g >= 0) kept |= 1ull << (g >> shift);
    }
    if constexpr (!BY_LOGIT) {
        float low = INFINITY, high = -INFINITY;              // the least that a kept one may be, the most another may
#pragma unroll
        for (int q = 0; q < G; ++q)
            if (off[q] >= 0.0f) {
                if ((kept >> (G == 1 ? l >> shift : l * G + q)) & 1)
                    low = fminf(low, half[q] - off[q]);
                else
                    high = fmaxf(high, half[q] + off[q]);
            }
        low = row_all_f(low, [](float p, float q) { return fminf(p, q); });
        high = row_all_f(high, [](float p, float q) { return fmaxf(p, q); });
        unsure |= !(low > high);
    }
    if ((a.group_size & (V - 1)) == 0) {                     // a lane's experts are of one group
        const unsigned of = (unsigned)(((unsigned)(l * V) * a.group_inv) >> 32);
        const bool in = (kept >> (of & 63)) & 1;
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = in ? key[v] : 0;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const unsigned of = (unsigned)(((unsigned)(l * V + v) * a.group_inv) >> 32);
            if (!((kept >> (of & 63)) & 1)) key[v] = 0;
        }
    }
}
template <bool BY_LOGIT, int V>
__device__ __forceinline__ void keep_groups(const RouteArgs &a, unsigned (&key)[V], unsigned *scratch, int lane, bool &unsure)
{
    if (a.groups <= 16)
        keep_groups<BY_LOGIT, V, 1>(a, key, scratch, lane, unsure);
    else
        keep_groups<BY_LOGIT, V, 4>(a, key, scratch, lane, unsure);
}

// The best of a whole wavefront's 64-bit keys, as pick() above: its index l V + v for lane l.
template <int V>
__device__ __forceinline__ int pick_wide(unsigned long long (&key)[V], int lane, unsigned long long &wins)
{
    unsigned long long best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    const unsigned hi = (unsigned)(best >> 32), top = wave_max_bits(hi);
    const unsigned low = wave_max_bits(hi == top ? (unsigned)best : 0u);
    wins = ((unsigned long long)top << 32) | low;
    if (wins == 0) return -1;
    const int first = __ffsll((unsigned long long)__ballot(best == wins)) - 1;
    int at = 0;
#pragma unroll
    for (int v = V - 1; v >= 0; --v)
        if (key[v] == wins) at = v;
    const int e = first * V + __builtin_amdgcn_readlane(at, first);
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (V * lane == e - v) key[v] = 0;
    return e;
}

// One token's k best by c in 64 bits, a wavefront on it: lane j answers with the j-th.  scratch: the wavefront's
// part of LDS, 8 E bytes of it.
template <int V, class Logit>
__device__ __forceinline__ int choose_exactly(const RouteArgs &a, const Logit &logit, unsigned long long *scratch, int lane)
{
    float x[V], top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        x[v] = lane * V + v < a.E ? logit(lane * V + v) : -INFINITY;
        top = fmaxf(top, x[v]);
    }
    top = wave_max(top);
    double total = 1.0;
    if (!a.sigmoid) {
        total = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (x[v] > -INFINITY) total += exp((double)x[v] - (double)top);
        total = wave_sum(total);
    }
    unsigned long long key[V], wins;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        key[v] = 0;
        if (x[v] > -INFINITY) {
            const double s = a.sigmoid ? 1.0 / (1.0 + exp(-(double)x[v])) : exp((double)x[v] - (double)top) / total;
            const double c = a.bias ? s + (double)a.bias[lane * V + v] : s;
            if (c > -INFINITY) key[v] = key_of(c);
        }
    }
    if (a.top_groups < a.groups) {                           // a lane scans a group
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (lane * V + v < a.E) scratch[lane * V + v] = key[v];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        unsigned long long first = 0, second = 0, worth[1];
        if (lane < a.groups)
            for (int i = 0; i < a.group_size; ++i) {
                const unsigned long long c = scratch[lane * a.group_size + i];
                second = max(second, min(first, c));
                first = max(first, c);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        worth[0] = a.group_top == 2 && second != 0 ? key_of(value_of(first) + value_of(second)) : first;
        unsigned long long kept = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            const int g = pick_wide(worth, lane, wins);
            if (g >= 0) kept |= 1ull << g;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (!((kept >> (((unsigned)(lane * V + v) * a.group_inv >> 32) & 63)) & 1)) key[v] = 0;
    }
    int mine = -1;
    for (int j = 0; j < a.k; ++j) {
        const int e = pick_wide(key, lane, wins);
        if (lane == j) mine = e;
    }
    return mine;
}

// Up to sixteen experts, a lane each (mine; -1: none), put in the order of their c in 64 bits.
__device__ __forceinline__ int order_exactly(const RouteArgs &a, float lv, int mine, int lane)
{
    double c = -INFINITY;
    if (mine >= 0) {
        c = 1.0 / (1.0 + exp(-(double)lv));
        if (a.bias) c += (double)a.bias[mine];
    }
    const long long bits = __double_as_longlong(c);
    int rank = 0;
#pragma unroll
    for (int d = 1; d < 16; ++d) {
        const int from = (lane & 48) | ((lane + d) & 15);
        const unsigned lo = (unsigned)__shfl((int)(unsigned)bits, from, 64), hi = (unsigned)__shfl((int)(bits >> 32), from, 64);
        const double other = __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
        const int e = __shfl(mine, from, 64);
        // (lanes without one stay behind the others, in their order)
        const bool ahead = e >= 0 && (mine < 0 || other > c || (other == c && e < mine));
        rank += ahead || (e < 0 && mine < 0 && (from & 15) < (lane & 15)) ? 1 : 0;
    }
    return __builtin_amdgcn_ds_permute(4 * ((lane & 48) | rank), mine);
}

// e^(x - y), y no less than x, both finite: what the difference lost in rounding, up to 2^-24 of it and so many times
// that of the result, is exact in fp32 and put right to first order.
__device__ __forceinline__ float exp_of_difference(float x, float y)
{
    const float d = x - y, back = d - x;
    const float lost = (x - (d - back)) - (y + back);
    const float e = expf(d);
    return d > -110.0f ? __builtin_fmaf(e, lost, e) : 0.0f;      // (e^-104 is less than any fp32)
}

// BY_LOGIT: the logits are compared; else c.
template <bool BY_LOGIT, int V, bool HALF>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.E, k = a.k, buckets = E + 1;
    const int l = lane & 15, row = lane >> 4;
    int *hist = reinterpret_cast<int *>(lds);                          // [kRouteWaves][buckets] or [buckets]
    int *base = hist + kRouteWaves * buckets;                          // [buckets]
    int *wave_sums = base + buckets;                                   // [kRouteWaves]
    int *ids = wave_sums + kRouteWaves;                                // [kRouteThreads]
    const int stride = padded(E);                                      // words of a token's keys
    unsigned *scratch = reinterpret_cast<unsigned *>(lds + route_tables(buckets)) + (size_t)(4 * wave + row) * stride;
    const bool grouping = a.hist || a.order;
    if (grouping) {
        for (int i = tid; i < buckets; i += kRouteThreads) hist[i] = 0;
        __syncthreads();
    }
    float bias[V];
    if constexpr (!BY_LOGIT) {
#pragma unroll
        for (int v = 0; v < V; ++v) bias[v] = 0.0f;
        if (a.bias)
#pragma unroll
            for (int v = 0; v < V; ++v) bias[v] = a.bias[min(l * V + v, E - 1)];
    }

    const int m0 = blockIdx.x * a.per_block, m1 = min(a.M, m0 + a.per_block);
    for (int step = m0; step < m1; step += kRouteTokens) {
        const int m = step + 4 * wave + row;
        if (step + 4 * wave >= m1) break;                    // (the wavefront's first token: uniform)
        const bool here = m < m1;
        const uint16_t *half = static_cast<const uint16_t *>(a.logits) + (size_t)(here ? m : m0) * E;
        const float *full = static_cast<const float *>(a.logits) + (size_t)(here ? m : m0) * E;
        float x[V], top = -INFINITY;
        // (no branches and no more code than it takes: a wavefront passes here once or twice, and what it waits for
        // is the instructions)
        constexpr int W = V < 4 ? V : 4;
        if (E % W == 0) {                                    // W logits a load (rows begin on a multiple of W)
            typedef float Floats __attribute__((ext_vector_type(W)));
            typedef uint16_t Halves __attribute__((ext_vector_type(W)));
#pragma unroll
            for (int v0 = 0; v0 < V; v0 += W) {
                const int e = min(l * V + v0, E - W);
                if constexpr (HALF) {
                    const Halves h = *reinterpret_cast<const Halves *>(half + e);
#pragma unroll
                    for (int i = 0; i < W; ++i) x[v0 + i] = h2f(h[i]);
                } else {
                    const Floats f = *reinterpret_cast<const Floats *>(full + e);
#pragma unroll
                    for (int i = 0; i < W; ++i) x[v0 + i] = f[i];
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = min(l * V + v, E - 1);
                x[v] = HALF ? h2f(half[e]) : full[e];
            }
        }
        const int valid = here ? E - l * V : 0;              // of this lane's keys
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = v < valid && x[v] > -INFINITY ? fminf(x[v], kLargest) : -INFINITY;   // NaN: cannot be chosen
            top = fmaxf(top, x[v]);
        }
        float total = 1.0f;                                  // of the softmax, where it is needed
        if (!a.sigmoid && (!BY_LOGIT || !a.renormalise)) {
            top = row_all_f(top, [](float p, float q) { return fmaxf(p, q); });
            if constexpr (BY_LOGIT) {
                float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};     // (a sum of 32 by itself would be off by 31 roundings)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v & 3] += x[v] > -INFINITY ? expf(x[v] - top) : 0.0f;
                total = row_all_f((sum[0] + sum[1]) + (sum[2] + sum[3]), [](float p, float q) { return p + q; });
            } else {                     // in 64 bits: the roundings of 512 additions would be more than c may be off by
                double sum = 0.0;
#pragma unroll
                for (int v = 0; v < V; ++v) sum += x[v] > -INFINITY ? (double)expf(x[v] - top) : 0.0;
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
                total = (float)sum;
            }
        }
        unsigned key[V];
        if constexpr (BY_LOGIT) {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = x[v] > -INFINITY ? key_of(x[v]) : 0u;
        } else {
            // (of -inf: a score of 0, and no key)
            constexpr float kLog2e = 1.44269504088896341f;
            float c[V];
            if (a.sigmoid) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    c[v] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[v] * -kLog2e)) + bias[v];
            } else {
                const float part = __builtin_amdgcn_rcpf(total);
#pragma unroll
                for (int v = 0; v < V; ++v) c[v] = __builtin_amdgcn_exp2f((x[v] - top) * kLog2e) * part + bias[v];
            }
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = x[v] > -INFINITY && c[v] > -INFINITY ? key_of(c[v]) : 0u;
        }
        bool unsure = false;                                 // all the experts have to be looked at in 64 bits
        if (a.top_groups < a.groups) keep_groups<BY_LOGIT>(a, key, scratch, lane, unsure);
        int mine = -1;                                       // the expert of slot l
        unsigned last = 0, wins = 0;
        bool close = false;                                  // two that follow each other are
        // the k best and, where c is good to fp32 only, whoever is close behind the last of them
        bool behind = true;
        for (int j = 0;; ++j) {
            if (BY_LOGIT && j == k) break;
            const int e = pick(key, lane, wins);
            if (!BY_LOGIT && j > 0) {
                const bool follows = last != 0 && wins != 0 && near(last, wins);
                if (j >= k) {
                    behind = behind && follows;
                    if (__ballot(behind) == 0) break;
                }
                close |= j >= k ? behind : follows;
                if (j == 16) {
                    unsure |= behind;
                    break;
                }
            }
            if (l == j && (j < k || behind)) mine = e;
            last = wins;
        }
        if constexpr (!BY_LOGIT) {
            unsure |= close && !a.sigmoid;
            if (__ballot(unsure) != 0) {
                for (int r = 0; r < 4; ++r) {                // one token after the other
                    if (!((__ballot(unsure) >> (16 * r)) & 0xffffu)) continue;
                    const int of = step + 4 * wave + r;      // (a token that is there: it had something to choose)
                    const int chosen = choose_exactly<(V + 3) / 4>(
                        a,
                        [&](int e) {
                            const size_t at = (size_t)of * E + e;
                            const float v = HALF ? h2f(static_cast<const uint16_t *>(a.logits)[at]) : static_cast<const float *>(a.logits)[at];
                            return v > -INFINITY ? fminf(v, kLargest) : -INFINITY;
                        },
                        reinterpret_cast<unsigned long long *>(scratch - (size_t)row * stride), lane);
                    const int mine_now = __shfl(chosen, l, 64);
                    if (row == r) mine = mine_now;
                }
                close = close && !unsure;
            }
            if (__ballot(close)) {
                float lv = 0.0f;
                if (mine >= 0) lv = fminf(HALF ? h2f(half[mine]) : full[mine], kLargest);
                const int ordered = order_exactly(a, lv, mine, lane);
                if (close) mine = ordered;
            }
        }

        // weights: renormalised from the largest of the chosen, so that nothing underflows which is not small beside it
        // (sigmoids of negative logits are e^l / (1 + e^l))
        const bool chosen = l < k && mine >= 0;
        float lv = -INFINITY;
        if (chosen) lv = fminf(HALF ? h2f(half[mine]) : full[mine], kLargest);
        const float above = row_all_f(lv, [](float p, float q) { return fmaxf(p, q); });
        float w = 0.0f;
        if (chosen) {
            if (!a.sigmoid) {
                w = a.renormalise ? exp_of_difference(lv, above) : exp_of_difference(lv, top) / total;
            } else if (a.renormalise && above < 0.0f) {
                w = exp_of_difference(lv, above) / (1.0f + expf(lv));
            } else {
                const float t = expf(-fabsf(lv));
                w = (lv < 0.0f ? t : 1.0f) / (1.0f + t);
            }
        }
        if (a.renormalise) {
            const float sum = row_all_f(w, [](float p, float q) { return p + q; });
            w = sum > 0.0f ? w / sum : 0.0f;
        }
        if (here && l < k) {
            a.experts[(size_t)m * k + l] = mine;
            a.weights[(size_t)m * k + l] = w * a.scale;
            if (grouping) {
                const int bucket = mine < 0 ? E : mine;
                if (a.order) ids[(m - m0) * k + l] = bucket;
                atomicAdd(&hist[bucket], 1);
            }
        }
    }
    if (!grouping) return;
    __syncthreads();
    if (a.hist) {
        const int pairs = pairs_of(buckets);
        for (int i = tid; i < pairs; i += kRouteThreads)
            reinterpret_cast<unsigned *>(a.hist)[(size_t)blockIdx.x * pairs + i] =
                (unsigned)hist[2 * i] | (2 * i + 1 < buckets ? (unsigned)hist[2 * i + 1] << 16 : 0u);
        return;
    }
    begin_buckets<kRouteWaves>(hist, nullptr, E, base, wave_sums, a.offsets);
    const bool have = tid < (m1 - m0) * k;
    hand_out<kRouteWaves>(have ? ids[tid] : 0, have, tid, E, hist, base, a.order);
}

// Counts of a block's rows; ids outside 0 .. count - 1 belong to none.
__global__ __launch_bounds__(kThreads) void count_kernel(const int32_t *ids, int rows, int per_block, int count, unsigned *hist)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    int *mine = reinterpret_cast<int *>(lds);
    const int tid = threadIdx.x, buckets = count + 1, pairs = pairs_of(buckets);
    for (int i = tid; i < buckets; i += kThreads) mine[i] = 0;
    __syncthreads();
    const int s0 = blockIdx.x * per_block, n = min(per_block, rows - s0);
    for (int s = tid; s < n; s += kThreads) {
        const int id = ids[s0 + s];
        atomicAdd(&mine[(unsigned)id < (unsigned)count ? id : count], 1);
    }
    __syncthreads();
    for (int i = tid; i < pairs; i += kThreads)
        hist[(size_t)blockIdx.x * pairs + i] =
            (unsigned)mine[2 * i] | (2 * i + 1 < buckets ? (unsigned)mine[2 * i + 1] << 16 : 0u);
}

// Second launch: hist [blocks][pairs] of the same blocks, two buckets a word; with hist null, one block that
// counts by itself.
__global__ __launch_bounds__(kThreads) void place_kernel(const int32_t *ids, int rows, int per_block, int count,
                                                         const unsigned *hist, int32_t *order, int32_t *offsets)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, buckets = count + 1, pairs = pairs_of(buckets);
    int *wcount = reinterpret_cast<int *>(lds);
    int *base = wcount + kWaves * buckets;
    int *wave_sums = base + buckets;
    const int s0 = blockIdx.x * per_block, n = min(per_block, rows - s0);
    int *total = wcount, *before = wcount + 2 * pairs;   // (fit [kWaves][buckets])
    for (int i = tid; i < 4 * pairs; i += kThreads) wcount[i] = 0;
    // the first rows' ids set out ahead of the counts
    int id = tid < n ? ids[s0 + tid] : 0;
    __syncthreads();
    if (hist) {
        // a column of words a thread, the blocks dealt out to as many threads as there are for it
        const int shares = kThreads / pairs, share = tid / pairs, i = tid - share * pairs;
        if (share < shares) {
            unsigned lo = 0, hi = 0, lo_before = 0, hi_before = 0;
            const int blocks = (int)gridDim.x, mine = (int)blockIdx.x;
            auto add = [&](unsigned c, int b) {
                lo += c & 0xffffu;
                hi += c >> 16;
                if (b < mine) {
                    lo_before += c & 0xffffu;
                    hi_before += c >> 16;
                }
            };
            int b = share;
            for (; b + 15 * shares < blocks; b += 16 * shares) {
                unsigned c[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) c[u] = hist[(size_t)(b + u * shares) * pairs + i];
#pragma unroll
                for (int u = 0; u < 16; ++u) add(c[u], b + u * shares);
            }
            for (; b < blocks; b += shares) add(hist[(size_t)b * pairs + i], b);
            atomicAdd(&total[2 * i], (int)lo);
            atomicAdd(&total[2 * i + 1], (int)hi);
            atomicAdd(&before[2 * i], (int)lo_before);
            atomicAdd(&before[2 * i + 1], (int)hi_before);
        }
    } else {
        if (tid < n) atomicAdd(&total[(unsigned)id < (unsigned)count ? id : count], 1);
    }
    __syncthreads();
    begin_buckets<kWaves>(total, before, count, base, wave_sums, blockIdx.x == 0 ? offsets : nullptr);
    for (int c0 = 0; c0 < n; c0 += kThreads) {
        if (c0 > 0) id = c0 + tid < n ? ids[s0 + c0 + tid] : 0;
        hand_out<kWaves>((unsigned)id < (unsigned)count ? id : count, c0 + tid < n, s0 + c0 + tid, count, wcount, base, order);
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Rows of a block, of `unit` slots each (0: ids, one each): spread over at most kMaxBlocks, but no more than
// a block can count.
int rows_per_block(int rows, int unit)
{
    int per = (rows + kMaxBlocks - 1) / kMaxBlocks;
    const int wanted = unit == 0 ? kThreads : kRouteTokens / 2;    // a slot a thread; four wavefronts' tokens
    if (unit == 0) unit = 1;
    per = per > wanted ? per : wanted;
    return per < kMostSlots / unit ? per : kMostSlots / unit;
}

int lds_of(int buckets) { return ((kWaves + 1) * buckets + kWaves + kOneBlock) * 4 + 16; }

hipError_t launch_place(const int32_t *ids, int rows, int per_block, int count, const void *hist, int32_t *order,
                        int32_t *offsets, hipStream_t st)
{
    const unsigned blocks = hist ? (unsigned)((rows + per_block - 1) / per_block) : 1u;
    hipLaunchKernelGGL(place_kernel, dim3(blocks), dim3(kThreads), (size_t)lds_of(count + 1), st, ids, rows,
                       hist ? per_block : rows, count, (const unsigned *)hist, order, offsets);
    return hipGetLastError();
}

template <bool BY_LOGIT, int V>
hipError_t launch_route_v(const RouteArgs &a, bool half, unsigned blocks, hipStream_t st)
{
    // the keys of a block's tokens; four tokens' part holds one's in 64 bits
    const size_t lds = (size_t)(route_tables(a.E + 1) + (a.top_groups < a.groups ? kRouteTokens * padded(a.E) * 4 + 64 : 0));
    static std::atomic<unsigned long long> allowed[2];
    auto kern = half ? route_kernel<BY_LOGIT, V, true> : route_kernel<BY_LOGIT, V, false>;
    constexpr int most = route_tables(kMaxExperts + 1) + kRouteTokens * padded(kMaxExperts) * 4 + 64;
    static_assert(most <= 160 * 1024, "LDS of one CU");
    if (hipError_t e = flexq::allow_dynamic_lds(reinterpret_cast<const void *>(kern), most, allowed[half]); e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kRouteThreads), lds, st, a);
    return hipGetLastError();
}

template <bool BY_LOGIT>
hipError_t launch_route(const RouteArgs &a, bool half, unsigned blocks, hipStream_t st)
{
    if (a.E <= 16) return launch_route_v<BY_LOGIT, 1>(a, half, blocks, st);
    if (a.E <= 32) return launch_route_v<BY_LOGIT, 2>(a, half, blocks, st);
    if (a.E <= 64) return launch_route_v<BY_LOGIT, 4>(a, half, blocks, st);
    if (a.E <= 128) return launch_route_v<BY_LOGIT, 8>(a, half, blocks, st);
    if (a.E <= 256) return launch_route_v<BY_LOGIT, 16>(a, half, blocks, st);
    return launch_route_v<BY_LOGIT, 32>(a, half, blocks, st);
}

size_t hist_bytes(int rows, int unit, int count)
{
    const int per = rows_per_block(rows, unit);
    const size_t blocks = (size_t)((rows + per - 1) / per);
    return (blocks * (size_t)pairs_of(count + 1) * 4 + 255) / 256 * 256;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t flexq_group_rows_workspace_bytes(int rows, int count)
{
    if (rows < 1 || rows > kMostRows || count < 1 || count > kMaxExperts) return 0;
    return hist_bytes(rows, 0, count);
}

flexq_status flexq_group_rows(const int32_t *ids, int rows, int count, int32_t *order, int32_t *offsets,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (!ids || !order || !offsets || rows < 1 || count < 1) return FLEXQ_EINVAL;
    if (count > kMaxExperts || rows > kMostRows) return FLEXQ_ESHAPE;
    if (!aligned4(ids) || !aligned4(order) || !aligned4(offsets)) return FLEXQ_EALIGN;
    if (!workspace || workspace_bytes < hist_bytes(rows, 0, count)) return FLEXQ_EWORKSPACE;
    if (!aligned16(workspace)) return FLEXQ_EALIGN;
    hipStream_t st = (hipStream_t)stream;
    if (rows <= kOneBlock)
        return launch_place(ids, rows, rows, count, nullptr, order, offsets, st) == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
    const int per = rows_per_block(rows, 0);
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), (size_t)(count + 1) * 4, st,
                       ids, rows, per, count, (unsigned *)workspace);
    if (hipGetLastError() != hipSuccess) return FLEXQ_EHIP;
    return launch_place(ids, rows, per, count, workspace, order, offsets, st) == hipSuccess ? FLEXQ_OK
                                                                                                         : FLEXQ_EHIP;
}

size_t flexq_route_workspace_bytes(int M, int E, int k)
{
    if (M < 1 || E < 1 || E > kMaxExperts || k < 1 || k > FLEXQ_MAX_EXPERTS_PER_TOKEN || k > E ||
        (long)M * k > kMostRows)
        return 0;
    return hist_bytes(M, k, E);
}

flexq_status flexq_route(const void *logits, int half, int M, int E, const flexq_routing *R, int32_t *experts,
                         float *weights, int32_t *order, int32_t *offsets, void *workspace, size_t workspace_bytes,
                         void *stream)
{
    if (!logits || !R || !experts || !weights || M < 1 || E < 1 || (half != 0 && half != 1)) return FLEXQ_EINVAL;
    if ((order == nullptr) != (offsets == nullptr)) return FLEXQ_EINVAL;
    if (E > kMaxExperts) return FLEXQ_ESHAPE;
    if (R->k < 1 || R->k > E || R->k > FLEXQ_MAX_EXPERTS_PER_TOKEN) return FLEXQ_EINVAL;
    if (R->score != FLEXQ_SCORE_SOFTMAX && R->score != FLEXQ_SCORE_SIGMOID) return FLEXQ_EINVAL;
    if (R->groups < 1 || R->groups > 64 || E % R->groups != 0) return FLEXQ_EINVAL;
    if (R->top_groups < 1 || R->top_groups > R->groups || R->group_top < 1 || R->group_top > 2) return FLEXQ_EINVAL;
    if ((long)R->k > (long)(E / R->groups) * R->top_groups) return FLEXQ_EINVAL;
    if (!(R->scale > 0.0f) || R->scale > 3.4028234663852886e38f) return FLEXQ_EINVAL;
    if ((long)M * R->k > kMostRows) return FLEXQ_ESHAPE;
    if (!aligned16(logits) || !aligned4(experts) || !aligned4(weights) || !aligned4(R->bias) || !aligned4(order) ||
        !aligned4(offsets))
        return FLEXQ_EALIGN;
    RouteArgs a{};
    a.logits = logits;
    a.bias = R->bias;
    a.M = M;
    a.E = E;
    a.k = R->k;
    a.sigmoid = R->score == FLEXQ_SCORE_SIGMOID;
    a.groups = R->groups;
    a.top_groups = R->top_groups;
    a.group_top = R->group_top;
    a.renormalise = R->renormalise != 0;
    a.scale = R->scale;
    a.group_size = E / R->groups;
    a.group_inv = (1ull << 32) / (unsigned)a.group_size + 1;
    a.group_shift = 4;
    while (a.group_shift > 0 && (16 >> a.group_shift) < R->groups) --a.group_shift;
    a.experts = experts;
    a.weights = weights;
    a.per_block = rows_per_block(M, R->k);
    // what a block takes at a time, and the places, in one launch
    static_assert(kRouteTokens * FLEXQ_MAX_EXPERTS_PER_TOKEN <= kRouteThreads, "a slot a thread");
    const bool one = M <= kRouteTokens;
    if (order) {
        if (!one && (!workspace || workspace_bytes < hist_bytes(M, R->k, E))) return FLEXQ_EWORKSPACE;
        if (!one && !aligned16(workspace)) return FLEXQ_EALIGN;
        if (one) {
            a.per_block = M;
            a.order = order;
            a.offsets = offsets;
        } else {
            a.hist = (uint16_t *)workspace;
        }
    }
    hipStream_t st = (hipStream_t)stream;
    const unsigned blocks = (unsigned)((M + a.per_block - 1) / a.per_block);
    // nothing is added to a score: the logits order like the scores
    const bool by_logit = !a.bias && (a.groups == a.top_groups || a.group_top == 1);
    const hipError_t e = by_logit ? launch_route<true>(a, half != 0, blocks, st) : launch_route<false>(a, half != 0, blocks, st);
    if (e != hipSuccess) return FLEXQ_EHIP;
    if (!order || one) return FLEXQ_OK;
    return launch_place(experts, M * R->k, a.per_block * R->k, E, a.hist, order, offsets, st) == hipSuccess ? FLEXQ_OK
                                                                                                          : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
