// The cache of keys and values: new tokens' rows into it, and rows read back.
//
// Sixteen tokens of a sequence, from a multiple of sixteen on, are a block. A block that is full lies in its page as 8-bit
// codes, with one scale for its keys and one for its values of a head: the activation quantizer's codes and scales of the
// 16 D values.  Until then its tokens wait in fp16, in a ring of 32 tokens that every sequence has: so each value is
// rounded once, whatever way its block filled up, and a sequence may be shortened: token t's place is t mod 32, so the ring holds
// the last two blocks up to the furthest token that was written, whatever was cut since -- a block before those is under
// them and does not come back when the sequence is cut a second time.
//
// A workgroup takes one block of a sequence and head, its codes through LDS so that they go out 16 bytes a thread; the one that
// has a sequence's first block -- the only one that reads tokens from the ring -- also writes the new tokens of its last two
// into the ring, after it has read.
//
// Bound by memory where there are many tokens: 4 bytes of rows in and 2 of codes out for each pair of elements; by the launch
// and three dependent trips (starts, lengths, rows) where there are few.  5900 tokens of 40 heads of 128: 47 us in, 3.9 TB/s --
// each workgroup makes its trips for 12 KiB -- and 32 us out, 5.6 TB/s; a token of 32 sequences 4.9 and 3.4 us.
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "producer_math.h"
#include "sequences.h"

namespace {

struct AppendArgs {
    CacheArgs c;
    const uint16_t *k, *v;
    size_t k_stride, v_stride;
};

struct ReadArgs {
    CacheArgs c;
    uint16_t *k, *v;
    size_t k_stride, v_stride;
};

// Four fp16 values of a channel -> four codes with their bias, one to a byte.
__device__ __forceinline__ unsigned code4(const uint16_t (&h)[4], float s, float r)
{
    unsigned out = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float q = __builtin_amdgcn_fmed3f(__builtin_rintf(div_by(h2f(h[i]), s, r)), -128.0f, 127.0f);
        out = __builtin_amdgcn_cvt_pk_u8_f32(q + (float)kCodeBias, i, out);
    }
    return out;
}

template <int D>
__global__ __launch_bounds__(2 * D) void append_kernel(AppendArgs a)
{
    typedef CacheBlock<D> B;
    // the first half of the threads takes values, four tokens of four channels each, the other keys, two times eight elements
    constexpr int THREADS = 2 * D, WAVES = D / 64;               // WAVES: of either half
    __shared__ unsigned top[2 * WAVES];
    __shared__ __attribute__((aligned(16))) uint8_t block[B::kBytes];    // the block's codes as they go out, 16 bytes a thread
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x, index = divide(blockIdx.x, c.by_kv), head = blockIdx.x - index * c.kv_heads;
    const RowRange r = find_rows(c.starts, c.count, c.M, 1, kBlock, 2, index, c.lengths);
    if (r.id < 0 || r.n == 0) return;
    const int length = cached_length(c, r.length), first = first_token(c, r.length, r.n);
    if (first >= length) return;                 // (rows before the first token and behind the table's room are dropped)
    const int b0 = max(first, 0) / kBlock, b = b0 + r.piece, full = length / kBlock;
    const bool leads = r.piece == 0;
    if (b >= full && !leads) return;
    uint16_t *recent = B::recent(c, r.id, head);
    const uint16_t *k = a.k + (size_t)head * D, *v = a.v + (size_t)head * D;
    auto row = [&](int token) { return (size_t)(r.begin + (token - first)); };
    if (b < full) {
        const int page = B::page_of(c, r.id, b);
        const bool values = tid < D;
        const int quad = tid / (D / 4), dv = tid % (D / 4) * 4;              // values: tokens 4 quad .., channels dv ..
        const int token = (tid - D) / (D / 8), dk = tid % (D / 8) * 8;       // keys: tokens token and token + 8, elements dk ..
        uint2 vv[4];
        uint4 kv[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) vv[i] = make_uint2(0u, 0u);
        kv[0] = kv[1] = make_uint4(0u, 0u, 0u, 0u);
        // (whether the block has a page is not waited for: the table is read while the rows are)
        if (values) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = b * kBlock + 4 * quad + i;
                if (t >= first)
                    vv[i] = *reinterpret_cast<const uint2 *>(v + row(t) * a.v_stride + dv);
                else if (recent)
                    vv[i] = make_uint2(recent[B::recent_value(t, dv)] | ((unsigned)recent[B::recent_value(t, dv + 1)] << 16),
                                       recent[B::recent_value(t, dv + 2)] | ((unsigned)recent[B::recent_value(t, dv + 3)] << 16));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = b * kBlock + token + 8 * i;
                if (t >= first)
                    kv[i] = *reinterpret_cast<const uint4 *>(k + row(t) * a.k_stride + dk);
                else if (recent)
                    kv[i] = *reinterpret_cast<const uint4 *>(recent + B::recent_key(t, dk));
            }
        }
        const uint4 half0 = values ? make_uint4(vv[0].x, vv[0].y, vv[1].x, vv[1].y) : kv[0];
        const uint4 half1 = values ? make_uint4(vv[2].x, vv[2].y, vv[3].x, vv[3].y) : kv[1];
        unsigned most = max_bits(half1, max_bits(half0, 0u));
        most = wave_max_bits(most);
        if ((tid & 63) == 0) top[tid >> 6] = most;
        __syncthreads();
        unsigned mv = top[0], mk = top[WAVES];
        if (WAVES == 2) {
            mv = max(mv, top[1]);
            mk = max(mk, top[3]);
        }
        const uint16_t sv = token_scale(h2f((uint16_t)mv), 127.0f), sk = token_scale(h2f((uint16_t)mk), 127.0f);
        if (values) {
            const float s = h2f(sv), inv = 1.0f / s;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint16_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = (uint16_t)((e < 2 ? vv[i].x : vv[i].y) >> 16 * (e & 1));
                *reinterpret_cast<unsigned *>(block + kBlock * D + value_at(4 * quad, dv + e)) = code4(h, s, inv);
            }
        } else {
            const float s = h2f(sk), inv = 1.0f / s;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint2 q = quant8(kv[i], s, inv, -128.0f, 127.0f);
                *reinterpret_cast<uint2 *>(block + key_at(token + 8 * i, dk)) = make_uint2(q.x ^ 0x80808080u, q.y ^ 0x80808080u);
            }
        }
        __syncthreads();
        if (page >= 0) {
            reinterpret_cast<uint4 *>(B::codes(c, page, head, b))[tid] = reinterpret_cast<const uint4 *>(block)[tid];
            if (tid == 0) *B::scales(c, page, head, b) = (unsigned)sk | ((unsigned)sv << 16);
        }
    }
    if (!leads || !recent) return;
    __syncthreads();                             // the ring has been read
    const int begin = max(max(first, 0), (full - 1) * kBlock);
    for (int i = tid; i < (length - begin) * (D / 8); i += THREADS) {
        const int t = begin + i / (D / 8), d = i % (D / 8) * 8;
        *reinterpret_cast<uint4 *>(recent + B::recent_key(t, d)) = *reinterpret_cast<const uint4 *>(k + row(t) * a.k_stride + d);
        const uint4 w = *reinterpret_cast<const uint4 *>(v + row(t) * a.v_stride + d);
        const unsigned w4[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            recent[B::recent_value(t, d + 2 * j)] = (uint16_t)(w4[j] & 0xffffu);
            recent[B::recent_value(t, d + 2 * j + 1)] = (uint16_t)(w4[j] >> 16);
        }
    }
}

// fp16 of a code times its scale.
__device__ __forceinline__ unsigned value2(unsigned lo, unsigned hi, float s)
{
    return pack_h2(within_half((float)((int)lo - kCodeBias) * s), within_half((float)((int)hi - kCodeBias) * s));
}

template <int D>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a)
{
    typedef CacheBlock<D> B;
    constexpr int KEYS = kBlock * D / 8;
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x, index = divide(blockIdx.x, c.by_kv), head = blockIdx.x - index * c.kv_heads;
    const RowRange r = find_rows(c.starts, c.count, c.M, 1, kBlock, 2, index, c.lengths);
    if (r.id < 0 || r.n == 0) return;
    const int length = cached_length(c, r.length), first = first_token(c, r.length, r.n);
    // (first may be negative and the end beyond the table's room: rows of tokens that there are not are zero)
    const int b = (first >> 4) + r.piece, full = length / kBlock, end = first + r.n;
    if (b * kBlock >= end) return;
    uint16_t *ko = a.k + (size_t)head * D, *vo = a.v + (size_t)head * D;
    auto row = [&](int token) { return (size_t)(r.begin + (token - first)); };
    const int token = tid / (D / 8), d = tid % (D / 8) * 8, quad = tid / (D / 2), dv = tid % (D / 2) * 2;
    const bool keys = KEYS == 256 || tid < KEYS, values = D == 128 || quad < 4;
    uint4 kv = make_uint4(0u, 0u, 0u, 0u);
    unsigned vv[4] = {0u, 0u, 0u, 0u};
    if (b >= 0 && b < full) {
        const int page = B::page_of(c, r.id, b);
        if (page >= 0) {
            const uint8_t *codes = B::codes(c, page, head, b);
            const unsigned s = *B::scales(c, page, head, b);
            const float sk = h2f((uint16_t)(s & 0xffffu)), sv = h2f((uint16_t)(s >> 16));
            if (keys) {
                const uint2 q = *reinterpret_cast<const uint2 *>(codes + key_at(token, d));
                kv.x = value2(q.x & 255u, q.x >> 8 & 255u, sk);
                kv.y = value2(q.x >> 16 & 255u, q.x >> 24, sk);
                kv.z = value2(q.y & 255u, q.y >> 8 & 255u, sk);
                kv.w = value2(q.y >> 16 & 255u, q.y >> 24, sk);
            }
            if (values) {
                const unsigned lo = *reinterpret_cast<const unsigned *>(codes + kBlock * D + value_at(4 * quad, dv));
                const unsigned hi = *reinterpret_cast<const unsigned *>(codes + kBlock * D + value_at(4 * quad, dv + 1));
#pragma unroll
                for (int i = 0; i < 4; ++i) vv[i] = value2(lo >> 8 * i & 255u, hi >> 8 * i & 255u, sv);
            }
        }
    } else if (b >= 0 && b * kBlock < length) {
        if (const uint16_t *recent = B::recent(c, r.id, head)) {
            if (keys) kv = *reinterpret_cast<const uint4 *>(recent + B::recent_key(b * kBlock + token, d));
            if (values) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = b * kBlock + 4 * quad + i;
                    vv[i] = recent[B::recent_value(t, dv)] | ((unsigned)recent[B::recent_value(t, dv + 1)] << 16);
                }
            }
        }
    }
    auto mine = [&](int t) { return t >= first && t < end; };
    if (keys && mine(b * kBlock + token)) *reinterpret_cast<uint4 *>(ko + row(b * kBlock + token) * a.k_stride + d) = kv;
    if (values) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = b * kBlock + 4 * quad + i;
            if (mine(t)) *reinterpret_cast<unsigned *>(vo + row(t) * a.v_stride + dv) = vv[i];
        }
    }
}

}  // namespace

namespace flexq {

flexq_status cache_args(const flexq_cache *C, const flexq_sequences *S, int M, CacheArgs &c)
{
    if (!C || !S || M < 1) return FLEXQ_EINVAL;
    if (!C->codes || !C->recent || C->kv_heads < 1 || C->pages < 1 || C->slots < 1) return FLEXQ_EINVAL;
    if (!S->starts || !S->lengths || !S->table || S->count < 1 || S->max_pages < 1) return FLEXQ_EINVAL;
    const size_t page_bytes = flexq_cache_page_bytes(C->kv_heads, C->head_dim, C->page);
    if (page_bytes == 0 || S->count > (1 << 20) || (long)S->max_pages * C->page > (1L << 30)) return FLEXQ_ESHAPE;
    if (M > (1 << 28)) return FLEXQ_ESHAPE;
    if ((reinterpret_cast<uintptr_t>(C->codes) & 15u) || (reinterpret_cast<uintptr_t>(C->recent) & 15u) ||
        (reinterpret_cast<uintptr_t>(S->starts) & 3u) || (reinterpret_cast<uintptr_t>(S->lengths) & 3u) ||
        (reinterpret_cast<uintptr_t>(S->table) & 3u) || (reinterpret_cast<uintptr_t>(S->slots) & 3u))
        return FLEXQ_EALIGN;
    c.codes = (uint8_t *)C->codes;
    c.recent = C->recent;
    c.starts = S->starts;
    c.lengths = S->lengths;
    c.table = S->table;
    c.slots = S->slots;
    c.page_bytes = page_bytes;
    c.kv_heads = C->kv_heads;
    c.by_kv = divider(C->kv_heads);
    c.pages = C->pages;
    c.slot_count = C->slots;
    c.shift = __builtin_ctz((unsigned)C->page / kBlock);
    c.count = S->count;
    c.max_pages = S->max_pages;
    c.M = M;
    return FLEXQ_OK;
}

}  // namespace flexq

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Checks that append and read share; the grid they need.
flexq_status rows_check(const flexq_cache *C, const flexq_sequences *S, int M, const uint16_t *k, int k_stride, const uint16_t *v,
                        int v_stride, CacheArgs &c, long &grid)
{
    if (!k || !v) return FLEXQ_EINVAL;
    if (flexq_status s = flexq::cache_args(C, S, M, c); s != FLEXQ_OK) return s;
    const int width = C->kv_heads * C->head_dim;
    if (k_stride < width || v_stride < width || k_stride % 8 != 0 || v_stride % 8 != 0) return FLEXQ_ESHAPE;
    if (!aligned16(k) || !aligned16(v)) return FLEXQ_EALIGN;
    grid = ((long)M / kBlock + 2L * S->count) * C->kv_heads;
    return grid < (1L << 24) ? FLEXQ_OK : FLEXQ_ESHAPE;          // 256 threads each, 2^32 a launch
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t flexq_cache_page_bytes(int kv_heads, int head_dim, int page)
{
    if (kv_heads < 1 || (head_dim != 64 && head_dim != 128) || (long)kv_heads * head_dim > FLEXQ_MAX_K) return 0;
    if (page < kBlock || page > FLEXQ_CACHE_MAX_PAGE || (page & (page - 1)) != 0) return 0;
    return ((size_t)(page / kBlock) * kv_heads * (2 * kBlock * head_dim + 4) + 255) / 256 * 256;
}

size_t flexq_cache_recent_bytes(int kv_heads, int head_dim)
{
    if (kv_heads < 1 || (head_dim != 64 && head_dim != 128) || (long)kv_heads * head_dim > FLEXQ_MAX_K) return 0;
    return (size_t)kv_heads * 4 * kBlock * head_dim * 2;
}

flexq_status flexq_cache_append(const flexq_cache *cache, const flexq_sequences *seqs, int M, const uint16_t *k, int k_stride,
                                const uint16_t *v, int v_stride, void *stream)
{
    AppendArgs a{};
    long grid = 0;
    if (flexq_status s = rows_check(cache, seqs, M, k, k_stride, v, v_stride, a.c, grid); s != FLEXQ_OK) return s;
    a.k = k;
    a.v = v;
    a.k_stride = (size_t)k_stride;
    a.v_stride = (size_t)v_stride;
    if (cache->head_dim == 128)
        hipLaunchKernelGGL(append_kernel<128>, dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(append_kernel<64>, dim3((unsigned)grid), dim3(128), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

flexq_status flexq_cache_read(const flexq_cache *cache, const flexq_sequences *seqs, int M, uint16_t *k, int k_stride,
                              uint16_t *v, int v_stride, void *stream)
{
    ReadArgs a{};
    long grid = 0;
    if (flexq_status s = rows_check(cache, seqs, M, k, k_stride, v, v_stride, a.c, grid); s != FLEXQ_OK) return s;
    a.k = k;
    a.v = v;
    a.k_stride = (size_t)k_stride;
    a.v_stride = (size_t)v_stride;
    if (cache->head_dim == 128)
        hipLaunchKernelGGL(read_kernel<128>, dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(read_kernel<64>, dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
