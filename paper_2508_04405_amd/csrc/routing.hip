// Rows that choose their own weights: the choice (scores of the experts -> the k best and their
// weights) and the grouping of rows by what they chose, which the experts' products and the
// adapters of a batch walk.
//
// Mathematics.  Scores s = softmax(l) or sigmoid(l); the choice is by c = s + bias, first (groups
// > 1) among groups by the sum of a group's best one or two c, then among the experts of the kept
// groups; the weights are the chosen s.  Two experts whose c are close must not change places with
// the rounding of an exponential.  Where nothing is added to a score, s grows with l, and l itself,
// exact, is compared (no exponential but the chosen ones').  Else c is made in fp32, good to 2^-20 of
// its size (at least 1), and whoever comes next to a chosen one closer than twice that sends the
// token through the same steps again in 64 bits -- one token in some hundreds.
//
// One wavefront a token, expert e in lane e / V: a tie is won by the lowest index.  Values are
// compared as unsigned keys (the bits of a float or double, so mapped that they order like the
// values, and 0 for what cannot be chosen): a round is the DPP maximum over the lanes, its place by
// ballots, on the scalar unit.
//
// Grouping is a counting sort, stable, so that equal inputs give equal orders: every block counts
// its slots per bucket (bucket `count` holds the rows without one), and a second launch adds up the
// counts of the blocks before it and hands out places -- rank within a wavefront by ballots over the
// bits of the bucket, wavefronts and blocks by their counts.  No atomics but LDS counters, whose sum
// has no order.  Few slots: everything in the one block of one launch.
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "producer_math.h"
#include "row_groups.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxExperts = FLEXQ_MAX_EXPERTS;          // buckets: one more
constexpr int kMaxBlocks = 256;                          // blocks of a launch over many slots: one a CU
constexpr int kMostSlots = 32768;                        // of a block: its counts are 16 bits
constexpr int kOneBlock = 1024;                          // slots that one block sorts by itself

struct RouteArgs {
    const void *logits;
    const float *bias;
    int M, E, k, sigmoid, groups, top_groups, group_top, renormalise;
    float scale;
    unsigned long long group_inv;   // e / group size = (e * group_inv) >> 32
    int group_size, group_lanes; // lanes that share a group's scan (a power of two)
    int32_t *experts;
    float *weights;
    int per_block;               // tokens of a block
    int32_t *order, *offsets;    // one block only, or null
    uint16_t *hist;              // [blocks][pairs_of(E + 1) * 2], or null
};

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

__device__ __forceinline__ unsigned wave_best(unsigned k) { return wave_max_bits(k); }
__device__ __forceinline__ unsigned long long wave_best(unsigned long long k)
{
    const unsigned hi = (unsigned)(k >> 32), top = wave_max_bits(hi);
    const unsigned low = wave_max_bits(hi == top ? (unsigned)k : 0u);
    return ((unsigned long long)top << 32) | low;
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Over the sixteen lanes of a row, every lane with its row's result.
template <class Op>
__device__ __forceinline__ float row_all(float v, const Op &op)
{
#define FLEXQ_ROW(ctrl) __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, 0xf, 0xf, false))
    v = op(v, FLEXQ_ROW(0x128));
    v = op(v, FLEXQ_ROW(0x124));
    v = op(v, FLEXQ_ROW(0x4e));
    v = op(v, FLEXQ_ROW(0xb1));
#undef FLEXQ_ROW
    return v;
}

__device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long v)
{
    return ((unsigned long long)uniform((unsigned)(v >> 32)) << 32) | uniform((unsigned)v);
}

// The best of the wavefront's keys: its index (ties: the lowest; -1: there is none), its key in `wins`.
// It is taken out.
template <int V, class Key>
__device__ __forceinline__ int pick(Key (&key)[V], int lane, Key &wins)
{
    Key best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    wins = uniform(wave_best(best));
    if (wins == 0) return -1;
    int e = 64 * V;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const unsigned long long at = __ballot(key[v] == wins);
        if (at) e = min(e, V * (__ffsll(at) - 1) + v);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (V * lane == e - v) key[v] = 0;
    return e;
}

// Places of the n <= kThreads slots of a block in the order.  id: this thread's slot's bucket, 0 .. count (have:
// it has one); wcount: LDS [kWaves][count + 1]; base[b]: LDS, the next free place of bucket b, moved on.
__device__ void hand_out(int id, bool have, int slot, int count, int *wcount, int *base, int32_t *order)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, buckets = count + 1;
    for (int i = tid; i < kWaves * buckets; i += kThreads) wcount[i] = 0;
    __syncthreads();
    unsigned long long same = __ballot(have);
    for (int bit = 1; bit <= count; bit <<= 1) {
        const unsigned long long b = __ballot((id & bit) != 0);
        same &= id & bit ? b : ~b;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    if (have && rank == 0) wcount[wave * buckets + id] = __popcll(same);
    __syncthreads();
    if (tid < buckets) {
        int c[kWaves], at = base[tid];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) c[w] = wcount[w * buckets + tid];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            wcount[w * buckets + tid] = at;
            at += c[w];
        }
        base[tid] = at;
    }
    __syncthreads();
    if (have) order[wcount[wave * buckets + id] + rank] = slot;
    __syncthreads();
}

// base[b] = sum of total[0 .. b - 1] + before[b]; offsets (one block) the sums alone.  One bucket a thread.
__device__ void begin_buckets(int total, int before, int count, int *base, int *wave_sums, int32_t *offsets)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int sum = wave_scan(total);
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    int ahead = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int s = wave_sums[w];
        if (w < wave) ahead += s;
    }
    const int begin = ahead + sum - total;
    if (tid <= count) {
        base[tid] = begin + before;
        if (offsets) offsets[tid] = begin;               // offsets[count] = the rows that have a bucket
    }
    __syncthreads();
}

constexpr float kLargest = 3.4028234663852886e38f;
constexpr float kClose = 0x1p-19f;       // twice the fp32 scores' error, of their size or 1

// What a wavefront needs to choose for a token: the logits, their largest, and what to do with them.
template <int V>
struct Token {
    float l[V], top;
};

// Keeps the keys of the top_groups best groups.  key_of_pair: the key of a group from its best two.  Answers
// whether the first group left out is `near` the last one kept.
template <int V, class Key, class Pair, class Near>
__device__ __forceinline__ bool keep_groups(const RouteArgs &a, Key (&key)[V], Key *scratch, int lane,
                                            const Pair &key_of_pair, const Near &near)
{
    // the wavefront's keys through its own LDS: lane group g x P lanes scans group g
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (lane * V + v < a.E) scratch[lane * V + v] = key[v];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int P = a.group_lanes, g = lane / P;
    Key first = 0, second = 0;
    if (g < a.groups)
        for (int i = lane % P; i < a.group_size; i += P) {
            const Key c = scratch[g * a.group_size + i];
            second = max(second, min(first, c));
            first = max(first, c);
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read before the next token's keys come)
    for (int d = 1; d < P; d <<= 1) {
        const Key f = __shfl_xor(first, d, 64), s = __shfl_xor(second, d, 64);
        second = max(max(second, s), min(first, f));
        first = max(first, f);
    }
    Key of_group[1] = {lane % P == 0 && g < a.groups && first != 0 ? key_of_pair(first, second) : (Key)0};
    unsigned long long kept = 0;
    Key last = 0, next;
    int win = 0;
    for (int i = 0; i < a.top_groups; ++i) {
        win = pick<1>(of_group, lane, next);
        if (win < 0) break;
        kept |= 1ull << (win / P);
        last = next;
    }
    const bool unsure = win >= 0 && pick<1>(of_group, lane, next) >= 0 && near(last, next);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const unsigned of = (unsigned)(((unsigned)(lane * V + v) * a.group_inv) >> 32);
        if (!((kept >> (of & 63)) & 1)) key[v] = 0;
    }
    return unsure;
}

// The k best by c in 64 bits; lane j answers with the j-th.
template <int V>
__device__ __forceinline__ int choose_exactly(const RouteArgs &a, const Token<V> &t, void *scratch, int lane)
{
    double total = 1.0;
    if (!a.sigmoid) {
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (t.l[v] > -INFINITY) sum += exp((double)t.l[v] - (double)t.top);
        total = wave_sum(sum);
    }
    unsigned long long key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        key[v] = 0;
        if (t.l[v] > -INFINITY) {
            const double s = a.sigmoid ? 1.0 / (1.0 + exp(-(double)t.l[v])) : exp((double)t.l[v] - (double)t.top) / total;
            const double c = a.bias ? s + (double)a.bias[lane * V + v] : s;
            if (c > -INFINITY) key[v] = key_of(c);
        }
    }
    if (a.top_groups < a.groups)
        keep_groups(a, key, static_cast<unsigned long long *>(scratch), lane,
                    [&](unsigned long long f, unsigned long long s) {
                        return a.group_top == 2 && s != 0 ? key_of(value_of(f) + value_of(s)) : f;
                    },
                    [](unsigned long long, unsigned long long) { return false; });
    int mine = -1;
    for (int j = 0; j < a.k; ++j) {
        unsigned long long wins;
        const int e = pick(key, lane, wins);
        if (e < 0) break;
        if (lane == j) mine = e;
    }
    return mine;
}

// BY_LOGIT: the logits are compared; else c.
template <bool BY_LOGIT, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.E, k = a.k, buckets = E + 1;
    int *hist = reinterpret_cast<int *>(lds);                          // [kWaves][buckets] or [buckets]
    int *base = hist + kWaves * buckets;                               // [buckets]
    int *wave_sums = base + buckets;                                   // [kWaves]
    int *ids = wave_sums + kWaves;                                     // [kOneBlock]
    unsigned char *scratch = lds + ((size_t)((kWaves + 1) * buckets + kWaves + kOneBlock) * 4 + 15) / 16 * 16 +
                             (size_t)wave * E * (BY_LOGIT ? 4 : 8);
    const bool grouping = a.hist || a.order;
    if (grouping) {
        for (int i = tid; i < buckets; i += kThreads) hist[i] = 0;
        __syncthreads();
    }
    float bias[V];
    if constexpr (!BY_LOGIT) {
#pragma unroll
        for (int v = 0; v < V; ++v) bias[v] = a.bias && lane * V + v < E ? a.bias[lane * V + v] : 0.0f;
    }

    const int m0 = blockIdx.x * a.per_block, m1 = min(a.M, m0 + a.per_block);
    for (int m = m0 + wave; m < m1; m += kWaves) {
        const uint16_t *half = static_cast<const uint16_t *>(a.logits) + (size_t)m * E;
        const float *full = static_cast<const float *>(a.logits) + (size_t)m * E;
        Token<V> t;
        if (E % V == 0) {                                    // (rows begin on a multiple of V)
            typedef float Floats __attribute__((ext_vector_type(V)));
            typedef uint16_t Halves __attribute__((ext_vector_type(V)));
#pragma unroll
            for (int v = 0; v < V; ++v) t.l[v] = -INFINITY;
            if (lane * V < E) {
                if constexpr (HALF) {
                    const Halves h = *reinterpret_cast<const Halves *>(half + lane * V);
#pragma unroll
                    for (int v = 0; v < V; ++v) t.l[v] = h2f(h[v]);
                } else {
                    const Floats f = *reinterpret_cast<const Floats *>(full + lane * V);
#pragma unroll
                    for (int v = 0; v < V; ++v) t.l[v] = f[v];
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                t.l[v] = lane * V + v < E ? (HALF ? h2f(half[lane * V + v]) : full[lane * V + v]) : -INFINITY;
        }
        t.top = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            t.l[v] = t.l[v] > -INFINITY ? fminf(t.l[v], kLargest) : -INFINITY;   // NaN: cannot be chosen
            t.top = fmaxf(t.top, t.l[v]);
        }
        float total = 1.0f;                                  // of the softmax, where it is needed
        if (!a.sigmoid && (!BY_LOGIT || !a.renormalise)) {
            t.top = wave_max(t.top);
            float sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) sum += t.l[v] > -INFINITY ? expf(t.l[v] - t.top) : 0.0f;
            total = wave_sum(sum);
        }
        unsigned key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = 0;
            if (t.l[v] > -INFINITY) {
                if constexpr (BY_LOGIT) {
                    key[v] = key_of(t.l[v]);
                } else {
                    const float s = a.sigmoid ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t.l[v] * -1.44269504088896341f))
                                              : __builtin_amdgcn_exp2f((t.l[v] - t.top) * 1.44269504088896341f) *
                                                    __builtin_amdgcn_rcpf(total);
                    const float c = s + bias[v];
                    if (c > -INFINITY) key[v] = key_of(c);
                }
            }
        }
        auto near = [](unsigned above, unsigned below) {
            const float x = value_of(above), y = value_of(below);
            return !(x - y > kClose * fmaxf(1.0f, fmaxf(fabsf(x), fabsf(y))));
        };
        bool unsure = false;
        if (a.top_groups < a.groups)
            unsure = keep_groups(a, key, reinterpret_cast<unsigned *>(scratch), lane,
                                 [&](unsigned f, unsigned s) {
                                     return !BY_LOGIT && a.group_top == 2 && s != 0 ? key_of(value_of(f) + value_of(s)) : f;
                                 },
                                 [&](unsigned x, unsigned y) { return near(key_of(0.5f * value_of(x)), key_of(0.5f * value_of(y))); });
        int mine = -1;                                       // the expert of slot `lane`, and its key
        unsigned won = 0;
        for (int j = 0; j < (BY_LOGIT ? k : k + 1); ++j) {
            unsigned wins;
            const int e = pick(key, lane, wins);
            if (e < 0) break;
            if (lane == j) {
                mine = e;
                if (!BY_LOGIT) won = wins;
            }
        }
        if constexpr (!BY_LOGIT) {
            const unsigned next = __shfl_down(won, 1, 64);
            unsure |= __ballot(lane < k && next != 0 && near(won, next)) != 0;
            if (unsure) mine = choose_exactly<V>(a, t, scratch, lane);
        }

        // weights, in the lanes of the first row: softmax renormalised from the largest of the chosen, so that
        // nothing underflows; sigmoids that all lie far below 0 are exponentials there
        const bool chosen = lane < k && mine >= 0;
        float lv = -INFINITY;
        if (chosen) lv = fminf(HALF ? h2f(half[mine]) : full[mine], kLargest);
        const float above = row_all(lv, [](float x, float y) { return fmaxf(x, y); });
        float w = 0.0f;
        if (chosen) {
            if (a.renormalise && (!a.sigmoid || above < -60.0f))
                w = expf(lv - above);
            else
                w = a.sigmoid ? 1.0f / (1.0f + expf(-lv)) : expf(lv - t.top) / total;
        }
        if (a.renormalise) {
            const float sum = row_all(w, [](float x, float y) { return x + y; });
            w = sum > 0.0f ? w / sum : 0.0f;
        }
        if (lane < k) {
            a.experts[(size_t)m * k + lane] = mine;
            a.weights[(size_t)m * k + lane] = w * a.scale;
            if (grouping) {
                const int bucket = mine < 0 ? E : mine;
                if (a.order) ids[(m - m0) * k + lane] = bucket;
                atomicAdd(&hist[bucket], 1);
            }
        }
    }
    if (!grouping) return;
    __syncthreads();
    if (a.hist) {
        const int pairs = pairs_of(buckets);
        for (int i = tid; i < pairs; i += kThreads)
            reinterpret_cast<unsigned *>(a.hist)[(size_t)blockIdx.x * pairs + i] =
                (unsigned)hist[2 * i] | (2 * i + 1 < buckets ? (unsigned)hist[2 * i + 1] << 16 : 0u);
        return;
    }
    begin_buckets(tid < buckets ? hist[tid] : 0, 0, E, base, wave_sums, a.offsets);
    const bool have = tid < (m1 - m0) * k;
    hand_out(have ? ids[tid] : 0, have, tid, E, hist, base, a.order);
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
    const int all = tid < buckets ? total[tid] : 0, ahead = tid < buckets ? before[tid] : 0;
    begin_buckets(all, ahead, count, base, wave_sums, blockIdx.x == 0 ? offsets : nullptr);
    for (int c0 = 0; c0 < n; c0 += kThreads) {
        if (c0 > 0) id = c0 + tid < n ? ids[s0 + c0 + tid] : 0;
        hand_out((unsigned)id < (unsigned)count ? id : count, c0 + tid < n, s0 + c0 + tid, count, wcount, base, order);
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Rows of a block, of `unit` slots each (0: ids, one each): spread over at most kMaxBlocks, but no more than
// a block can count.
int rows_per_block(int rows, int unit)
{
    int per = (rows + kMaxBlocks - 1) / kMaxBlocks;
    const int wanted = unit == 0 ? kThreads : kWaves;    // a slot a thread, a token a wavefront
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
    constexpr int bytes = BY_LOGIT ? 4 : 8;              // of a key in LDS
    const size_t lds = (size_t)(lds_of(a.E + 1) + (a.top_groups < a.groups ? kWaves * a.E * bytes : 0));
    static std::atomic<unsigned long long> allowed[2];
    auto kern = half ? route_kernel<BY_LOGIT, V, true> : route_kernel<BY_LOGIT, V, false>;
    constexpr int most = ((kWaves + 1) * (kMaxExperts + 1) + kWaves + kOneBlock) * 4 + 16 + kWaves * kMaxExperts * bytes;
    if (hipError_t e = flexq::allow_dynamic_lds(reinterpret_cast<const void *>(kern), most, allowed[half]); e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), lds, st, a);
    return hipGetLastError();
}

template <bool BY_LOGIT>
hipError_t launch_route(const RouteArgs &a, bool half, unsigned blocks, hipStream_t st)
{
    if (a.E <= 64) return launch_route_v<BY_LOGIT, 1>(a, half, blocks, st);
    if (a.E <= 128) return launch_route_v<BY_LOGIT, 2>(a, half, blocks, st);
    if (a.E <= 256) return launch_route_v<BY_LOGIT, 4>(a, half, blocks, st);
    return launch_route_v<BY_LOGIT, 8>(a, half, blocks, st);
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
    if (rows < 1 || count < 1 || count > kMaxExperts) return 0;
    return hist_bytes(rows, 0, count);
}

flexq_status flexq_group_rows(const int32_t *ids, int rows, int count, int32_t *order, int32_t *offsets,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (!ids || !order || !offsets || rows < 1 || count < 1) return FLEXQ_EINVAL;
    if (count > kMaxExperts) return FLEXQ_ESHAPE;
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
    if (M < 1 || E < 1 || E > kMaxExperts || k < 1 || k > FLEXQ_MAX_EXPERTS_PER_TOKEN || k > E) return 0;
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
    if ((long)M * R->k >= (1L << 31)) return FLEXQ_ESHAPE;
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
    a.group_lanes = 64;
    while (64 / a.group_lanes < R->groups) a.group_lanes /= 2;
    a.experts = experts;
    a.weights = weights;
    a.per_block = rows_per_block(M, R->k);
    // two tokens a wavefront, and the places, in one launch: at 64 tokens 11.4 us, in two 8.9
    static_assert(2 * kWaves * FLEXQ_MAX_EXPERTS_PER_TOKEN <= kOneBlock, "a block's slots");
    const bool one = M <= 2 * kWaves;
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
