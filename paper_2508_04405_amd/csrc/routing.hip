// Rows that choose their own weights: the choice (scores of the experts -> the k best and their
// weights) and the grouping of rows by what they chose, which the experts' products and the
// adapters of a batch walk.
//
// Mathematics.  Scores s = softmax(l) or sigmoid(l); the choice is by c = s + bias, first (groups
// > 1) among groups by the sum of a group's best one or two c, then among the experts of the kept
// groups; the weights are the chosen s.  Two experts whose c are close must not change places with
// the rounding of an exponential, so c is made in 64 bits -- unless nothing is added to a score: s
// grows with l, and l itself, exact, is compared then (no exponential but the chosen ones').
//
// One wavefront a token, expert e in lane e / V: a tie between lanes is won by the lowest lane.
// Values are compared as unsigned keys (the bits of a float or double, so mapped that they order
// like the values, and 0 for what cannot be chosen), 32 bits at a time through the DPP reduction of
// producer_math.h: k rounds of one or two reductions.
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

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxExperts = FLEXQ_MAX_EXPERTS;          // buckets: one more
constexpr int kMaxBlocks = 128;                          // blocks of a launch over many slots
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
    int *hist;                   // [blocks][E + 1], or null
};

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

// Places of the n slots of a block in the order.  ids: LDS, buckets 0 .. count; wcount: LDS
// [kWaves][count + 1]; base[b]: LDS, the next free place of bucket b, moved on.
__device__ void hand_out(const int *ids, int n, int first_slot, int count, int *wcount, int *base, int32_t *order)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, buckets = count + 1;
    for (int s0 = 0; s0 < n; s0 += kThreads) {
        for (int i = tid; i < kWaves * buckets; i += kThreads) wcount[i] = 0;
        __syncthreads();
        const int s = s0 + tid;
        const bool have = s < n;
        const int id = have ? ids[s] : 0;
        unsigned long long same = __ballot(have);
        for (int bit = 1; bit <= count; bit <<= 1) {
            const unsigned long long b = __ballot((id & bit) != 0);
            same &= id & bit ? b : ~b;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1ull));
        if (have && rank == 0) wcount[wave * buckets + id] = __popcll(same);
        __syncthreads();
        for (int b = tid; b < buckets; b += kThreads) {
            int at = base[b];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const int c = wcount[w * buckets + b];
                wcount[w * buckets + b] = at;
                at += c;
            }
            base[b] = at;
        }
        __syncthreads();
        if (have) order[wcount[wave * buckets + id] + rank] = first_slot + s;
        __syncthreads();
    }
}

// base[b] = sum of total[0 .. b - 1] + before[b]; offsets (block 0) the sums alone.  One bucket a thread.
__device__ void begin_buckets(int total, int before, int count, int *base, int *wave_sums, int32_t *offsets)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int sum = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(sum, d, 64);
        if (lane >= d) sum += up;
    }
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    int ahead = 0;
    for (int w = 0; w < wave; ++w) ahead += wave_sums[w];
    const int begin = ahead + sum - total;
    if (tid <= count) {
        base[tid] = begin + before;
        if (offsets) offsets[tid] = begin;               // offsets[count] = the rows that have a bucket
    }
    __syncthreads();
}

// T: what is compared (float: the logits themselves, double: scores with a bias, or group sums).
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a)
{
    using Key = decltype(key_of(T()));
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.E, k = a.k, buckets = E + 1;
    int *hist = reinterpret_cast<int *>(lds);                          // [kWaves][buckets] or [buckets]
    int *base = hist + kWaves * buckets;                               // [buckets]
    int *wave_sums = base + buckets;                                   // [kWaves]
    int *ids = wave_sums + kWaves;                                     // [kOneBlock]
    Key *scratch = reinterpret_cast<Key *>(lds + ((size_t)((kWaves + 1) * buckets + kWaves + kOneBlock) * 4 + 15) / 16 * 16) +
                   (size_t)wave * E;
    const bool grouping = a.hist || a.order;
    if (grouping) {
        for (int i = tid; i < buckets; i += kThreads) hist[i] = 0;
        __syncthreads();
    }

    const int m0 = blockIdx.x * a.per_block, m1 = min(a.M, m0 + a.per_block);
    for (int m = m0 + wave; m < m1; m += kWaves) {
        float l[V];
        Key key[V];
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = lane * V + v;
            l[v] = -INFINITY;
            if (e < E) {
                const size_t at = (size_t)m * E + e;
                l[v] = HALF ? h2f(static_cast<const uint16_t *>(a.logits)[at]) : static_cast<const float *>(a.logits)[at];
                l[v] = l[v] > -INFINITY ? fminf(l[v], 3.4028234663852886e38f) : -INFINITY;   // NaN: cannot be chosen
            }
            top = fmaxf(top, l[v]);
        }
        top = wave_max(top);
        double total = 1.0;                              // of the softmax, where it is needed
        if (!a.sigmoid && (sizeof(T) == 8 || !a.renormalise)) {
            double sum = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (l[v] > -INFINITY)
                    sum += sizeof(T) == 8 ? exp((double)l[v] - (double)top) : (double)expf(l[v] - top);
            total = wave_sum(sum);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = 0;
            if (l[v] > -INFINITY) {
                if constexpr (sizeof(T) == 8) {
                    const double s = a.sigmoid ? 1.0 / (1.0 + exp(-(double)l[v])) : exp((double)l[v] - (double)top) / total;
                    const double c = a.bias ? s + (double)a.bias[lane * V + v] : s;
                    if (c > -INFINITY) key[v] = key_of(c);
                } else {
                    key[v] = key_of(l[v]);
                }
            }
        }
        if (a.top_groups < a.groups) {
            // the wavefront's keys through its own LDS: lane group g x lanes scans group g
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (lane * V + v < E) scratch[lane * V + v] = key[v];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const int P = a.group_lanes, g = lane / P;
            Key first = 0, second = 0;
            if (g < a.groups)
                for (int i = lane % P; i < a.group_size; i += P) {
                    const Key c = scratch[g * a.group_size + i];
                    second = max(second, min(first, c));
                    first = max(first, c);
                }
            for (int d = 1; d < P; d <<= 1) {
                const Key f = __shfl_xor(first, d, 64), s = __shfl_xor(second, d, 64);
                second = max(max(second, s), min(first, f));
                first = max(first, f);
            }
            Key of_group = first;
            if constexpr (sizeof(T) == 8)
                if (a.group_top == 2 && first != 0)
                    of_group = key_of(second != 0 ? value_of(first) + value_of(second) : value_of(first));
            if (lane % P != 0 || g >= a.groups) of_group = 0;
            unsigned long long kept = 0;
            for (int i = 0; i < a.top_groups; ++i) {
                const Key best = wave_best(of_group);
                if (best == 0) break;
                const int win = __ffsll((unsigned long long)__ballot(of_group == best)) - 1;
                kept |= 1ull << (win / P);
                if (lane == win) of_group = 0;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const unsigned of = (unsigned)(((unsigned)(lane * V + v) * a.group_inv) >> 32);
                if (!((kept >> (of & 63)) & 1)) key[v] = 0;
            }
        }
        int mine = -1;                                   // the expert of slot `lane`
        for (int j = 0; j < k; ++j) {
            Key best = key[0];
            int at = 0;
#pragma unroll
            for (int v = 1; v < V; ++v)
                if (key[v] > best) {
                    best = key[v];
                    at = v;
                }
            const Key wins = wave_best(best);
            if (wins == 0) break;
            const int win = __ffsll((unsigned long long)__ballot(best == wins)) - 1;
            const int e = win * V + __builtin_amdgcn_readlane(at, win);
            if (lane == j) mine = e;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (lane == win && at == v) key[v] = 0;
        }
        // weights: the scores of the chosen, in 64 bits (sums of sigmoids far below zero keep their ratio)
        double w = 0.0;
        if (lane < k && mine >= 0) {
            const size_t at = (size_t)m * E + mine;
            float lv = HALF ? h2f(static_cast<const uint16_t *>(a.logits)[at]) : static_cast<const float *>(a.logits)[at];
            lv = fminf(lv, 3.4028234663852886e38f);
            w = a.sigmoid ? 1.0 / (1.0 + exp(-(double)lv)) : exp((double)lv - (double)top) / total;
        }
        if (a.renormalise) {
            const double sum = wave_sum(w);
            w = sum > 0.0 ? w / sum : 0.0;
        }
        if (lane < k) {
            a.experts[(size_t)m * k + lane] = mine;
            a.weights[(size_t)m * k + lane] = (float)(w * (double)a.scale);
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
        for (int i = tid; i < buckets; i += kThreads) a.hist[(size_t)blockIdx.x * buckets + i] = hist[i];
        return;
    }
    begin_buckets(tid < buckets ? hist[tid] : 0, 0, E, base, wave_sums, a.offsets);
    hand_out(ids, (m1 - m0) * k, 0, E, hist, base, a.order);
}

// Counts of a block's rows; ids outside 0 .. count - 1 belong to none.
__global__ __launch_bounds__(kThreads) void count_kernel(const int32_t *ids, int rows, int per_block, int count, int *hist)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    int *mine = reinterpret_cast<int *>(lds);
    const int tid = threadIdx.x;
    for (int i = tid; i <= count; i += kThreads) mine[i] = 0;
    __syncthreads();
    const int s0 = blockIdx.x * per_block, n = min(per_block, rows - s0);
    for (int s = tid; s < n; s += kThreads) {
        const int id = ids[s0 + s];
        atomicAdd(&mine[(unsigned)id < (unsigned)count ? id : count], 1);
    }
    __syncthreads();
    for (int i = tid; i <= count; i += kThreads) hist[(size_t)blockIdx.x * (count + 1) + i] = mine[i];
}

// Second launch: hist [blocks][count + 1] of the same blocks; with hist null, one block that counts by itself.
__global__ __launch_bounds__(kThreads) void place_kernel(const int32_t *ids, int rows, int per_block, int count,
                                                         const int *hist, int32_t *order, int32_t *offsets)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, buckets = count + 1;
    int *wcount = reinterpret_cast<int *>(lds);
    int *base = wcount + kWaves * buckets;
    int *wave_sums = base + buckets;
    int *mine = wave_sums + kWaves;                      // [kThreads]
    const int s0 = blockIdx.x * per_block, n = min(per_block, rows - s0);
    int total = 0, before = 0;
    if (hist) {
        if (tid < buckets)
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const int c = hist[(size_t)b * buckets + tid];
                total += c;
                if (b < (int)blockIdx.x) before += c;
            }
    } else {
        for (int i = tid; i < buckets; i += kThreads) wcount[i] = 0;
        __syncthreads();
        for (int s = tid; s < n; s += kThreads) {
            const int id = ids[s];
            atomicAdd(&wcount[(unsigned)id < (unsigned)count ? id : count], 1);
        }
        __syncthreads();
        if (tid < buckets) total = wcount[tid];
    }
    begin_buckets(total, before, count, base, wave_sums, blockIdx.x == 0 ? offsets : nullptr);
    for (int c0 = 0; c0 < n; c0 += kThreads) {
        const int s = c0 + tid;
        if (s < n) {
            const int id = ids[s0 + s];
            mine[tid] = (unsigned)id < (unsigned)count ? id : count;
        }
        __syncthreads();
        hand_out(mine, min(kThreads, n - c0), s0 + c0, count, wcount, base, order);
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Rows of a block, where `rows` of them (in units of `unit` slots) are spread over at most kMaxBlocks.
int rows_per_block(int rows, int unit)
{
    const int least = (rows + kMaxBlocks - 1) / kMaxBlocks;
    const int wanted = unit == 1 ? kThreads : kWaves;    // a slot a thread, a token a wavefront
    return least > wanted ? least : wanted;
}

int lds_of(int buckets) { return ((kWaves + 1) * buckets + kWaves + kOneBlock) * 4 + 16; }

hipError_t launch_place(const int32_t *ids, int rows, int per_block, int count, const int *hist, int32_t *order,
                        int32_t *offsets, hipStream_t st)
{
    const unsigned blocks = hist ? (unsigned)((rows + per_block - 1) / per_block) : 1u;
    hipLaunchKernelGGL(place_kernel, dim3(blocks), dim3(kThreads), (size_t)lds_of(count + 1), st, ids, rows,
                       hist ? per_block : rows, count, hist, order, offsets);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_route_v(const RouteArgs &a, bool half, unsigned blocks, hipStream_t st)
{
    const size_t lds = (size_t)(lds_of(a.E + 1) + (a.top_groups < a.groups ? kWaves * a.E * (int)sizeof(T) : 0));
    static std::atomic<unsigned long long> allowed[2];
    auto kern = half ? route_kernel<T, V, true> : route_kernel<T, V, false>;
    constexpr int most = ((kWaves + 1) * (kMaxExperts + 1) + kWaves + kOneBlock) * 4 + 16 + kWaves * kMaxExperts * 8;
    if (hipError_t e = flexq::allow_dynamic_lds(reinterpret_cast<const void *>(kern), most, allowed[half]); e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), lds, st, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_route(const RouteArgs &a, bool half, unsigned blocks, hipStream_t st)
{
    if (a.E <= 64) return launch_route_v<T, 1>(a, half, blocks, st);
    if (a.E <= 128) return launch_route_v<T, 2>(a, half, blocks, st);
    if (a.E <= 256) return launch_route_v<T, 4>(a, half, blocks, st);
    return launch_route_v<T, 8>(a, half, blocks, st);
}

size_t hist_bytes(int rows, int unit, int count)
{
    const int per = rows_per_block(rows, unit);
    const size_t blocks = (size_t)((rows + per - 1) / per);
    return (blocks * (size_t)(count + 1) * 4 + 255) / 256 * 256;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t flexq_group_rows_workspace_bytes(int rows, int count)
{
    if (rows < 1 || count < 1 || count > kMaxExperts) return 0;
    return hist_bytes(rows, 1, count);
}

flexq_status flexq_group_rows(const int32_t *ids, int rows, int count, int32_t *order, int32_t *offsets,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (!ids || !order || !offsets || rows < 1 || count < 1) return FLEXQ_EINVAL;
    if (count > kMaxExperts) return FLEXQ_ESHAPE;
    if (!aligned4(ids) || !aligned4(order) || !aligned4(offsets)) return FLEXQ_EALIGN;
    if (!workspace || workspace_bytes < hist_bytes(rows, 1, count)) return FLEXQ_EWORKSPACE;
    if (!aligned16(workspace)) return FLEXQ_EALIGN;
    hipStream_t st = (hipStream_t)stream;
    if (rows <= kOneBlock)
        return launch_place(ids, rows, rows, count, nullptr, order, offsets, st) == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
    const int per = rows_per_block(rows, 1);
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), (size_t)(count + 1) * 4, st,
                       ids, rows, per, count, (int *)workspace);
    if (hipGetLastError() != hipSuccess) return FLEXQ_EHIP;
    return launch_place(ids, rows, per, count, (const int *)workspace, order, offsets, st) == hipSuccess ? FLEXQ_OK
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
    const bool one = (long)M * R->k <= kOneBlock && M <= 4 * kWaves;
    if (order) {
        if (!workspace || workspace_bytes < hist_bytes(M, R->k, E)) return FLEXQ_EWORKSPACE;
        if (!aligned16(workspace)) return FLEXQ_EALIGN;
        if (one) {
            a.per_block = M;
            a.order = order;
            a.offsets = offsets;
        } else {
            a.hist = (int *)workspace;
        }
    }
    hipStream_t st = (hipStream_t)stream;
    const unsigned blocks = (unsigned)((M + a.per_block - 1) / a.per_block);
    // nothing is added to a score: the logits order like the scores
    const bool by_logit = !a.bias && (a.groups == a.top_groups || a.group_top == 1);
    const hipError_t e = by_logit ? launch_route<float>(a, half != 0, blocks, st) : launch_route<double>(a, half != 0, blocks, st);
    if (e != hipSuccess) return FLEXQ_EHIP;
    if (!order || one) return FLEXQ_OK;
    return launch_place(experts, M * R->k, a.per_block * R->k, E, a.hist, order, offsets, st) == hipSuccess ? FLEXQ_OK
                                                                                                          : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
