// The sequences of a batch whose rows lie one behind the other, and the 8-bit cache of keys and values in pages: how kernels
// walk them.
#pragma once
#include "../../include/flexq.h"
#include "flexq_device.h"

namespace flexq {

// Division by a number that the host knows: floor(2^32 / d) is at most one short in the quotient of x < 2^31.
struct Divider {
    unsigned d, magic;
};
inline Divider divider(int d) { return Divider{(unsigned)d, d == 1 ? 0xffffffffu : (unsigned)(0x100000000ull / (unsigned)d)}; }

// A cache and the sequences of a call, as kernels take them.
struct CacheArgs {
    uint8_t *codes;              // [pages][page_bytes]
    uint16_t *recent;            // [slots][kv_heads][64 D]
    const int32_t *starts, *lengths, *table, *slots;
    size_t page_bytes;
    int kv_heads, pages, slot_count;
    Divider by_kv;
    int shift;                   // blocks of a page: 1 << shift
    int count, max_pages, M;
};

// Checks of a cache and the sequences of a call (host only); fills c.
flexq_status cache_args(const flexq_cache *C, const flexq_sequences *S, int M, CacheArgs &c);

}  // namespace flexq

namespace {

using flexq::CacheArgs;
using flexq::Divider;
using flexq::divider;

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

constexpr int kBlock = FLEXQ_CACHE_BLOCK;    // tokens that share a scale
constexpr int kCodeBias = 128;               // codes are stored as code + 128

__device__ __forceinline__ int divide(int x, Divider by)
{
    const unsigned q = __umulhi((unsigned)x, by.magic);
    return (int)(q + ((unsigned)x - q * by.d >= by.d ? 1u : 0u));
}

// The largest finite fp16 at most: the rounding of weights, or of a scale, may lead a mean of finite values beyond it.
__device__ __forceinline__ float within_half(float y)
{
    return __builtin_amdgcn_fmed3f(y, -65504.0f, 65504.0f);
}

struct RowRange {
    int id, begin, n;    // sequence (-1: none), its first row, its rows
    int piece;           // number of the piece within the sequence
    int length;          // lengths[id], where lengths are given
};

// Sequence s owns pieces place(s) .. place(s + 1) - 1 of a launch, place(s) = floor(starts[s] * mul / div) + extra * s: a
// closed form that leaves every sequence as many as it can need -- ceil(n mul / div) of them with extra = 1 -- so that no
// one adds up the lengths of those before.  Whose piece `index` is, is the last s with place(s) <= index; every wavefront
// finds it for itself, 64 sequences a step.  starts outside 0 .. rows, or falling, never lead outside the rows.
__device__ __forceinline__ RowRange find_rows(const int32_t *starts, int count, int rows, int mul, int div, int extra, int index,
                                              const int32_t *lengths = nullptr)
{
    const int lane = threadIdx.x & 63;
    auto start = [&](int s) { return min(max(starts[s], 0), rows); };
    auto place = [&](int at, int s) { return (int)((unsigned)(at * mul) / (unsigned)div) + extra * s; };
    int lo = 0, span = count;
    while (span > 64) {
        const int step = (span + 63) / 64, s = lo + lane * step;
        const bool before = lane * step < span && place(start(min(s, count)), s) <= index;
        const int hits = __builtin_popcountll(__ballot(before));
        if (hits == 0) return RowRange{-1, 0, 0, 0, 0};
        lo += (hits - 1) * step;
        span = min(step, span - (hits - 1) * step);
    }
    const int s = min(lo + lane, count - 1), a = start(s), b = max(start(s + 1), a);
    const int p = place(a, s), length = lengths ? lengths[s] : 0;
    const int hits = __builtin_popcountll(__ballot(lane < span && p <= index));
    if (hits == 0) return RowRange{-1, 0, 0, 0, 0};
    RowRange r;
    r.id = lo + hits - 1;
    r.begin = __builtin_amdgcn_readlane(a, hits - 1);
    r.n = __builtin_amdgcn_readlane(b, hits - 1) - r.begin;
    r.piece = index - __builtin_amdgcn_readlane(p, hits - 1);
    r.length = __builtin_amdgcn_readlane(length, hits - 1);
    if (r.piece < 0) r.id = -1;                          // (falling starts)
    return r;
}

// A block of one head in its page: 16 D bytes of keys, then as many of values, in the order in which the lanes of a
// wavefront feed them to 16x16x32 MFMAs as the row operand.  Plane j (1 KiB) of the keys gives lane l = (g, i), g = l / 16,
// i = l % 16, sixteen elements of key i: d = 64 j + 8 g + 0 .. 7 and d = 64 j + 32 + 8 g + 0 .. 7.  Plane j of the values
// gives it d = 64 j + 16 t + i, t = 0 .. 3, of keys 4 g .. 4 g + 3.  Behind all blocks of a page follow their scales.
__device__ __forceinline__ int key_at(int token, int d)
{
    return (d >> 6) * 1024 + (((d >> 3) & 3) * 16 + token) * 16 + ((d >> 5) & 1) * 8 + (d & 7);
}
__device__ __forceinline__ int value_at(int token, int d)
{
    return (d >> 6) * 1024 + ((token >> 2) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (token & 3);
}

template <int D>
struct CacheBlock {
    static constexpr int kBytes = 2 * kBlock * D;                // keys and values of a block and head
    static constexpr int kRecent = 4 * kBlock * D;               // halves of a slot and head: two blocks of keys, two of values

    // Page of block b of sequence s, or -1: the table names none there.
    __device__ static __forceinline__ int page_of(const CacheArgs &c, int s, int b)
    {
        const int i = b >> c.shift;
        if (i >= c.max_pages) return -1;
        const int page = c.table[(size_t)s * c.max_pages + i];
        return page >= 0 && page < c.pages ? page : -1;
    }
    __device__ static __forceinline__ uint8_t *codes(const CacheArgs &c, int page, int head, int b)
    {
        return c.codes + (size_t)page * c.page_bytes + (size_t)((head << c.shift) + (b & ((1 << c.shift) - 1))) * kBytes;
    }
    __device__ static __forceinline__ uint32_t *scales(const CacheArgs &c, int page, int head, int b)   // key's, value's << 16
    {
        uint8_t *at = c.codes + (size_t)page * c.page_bytes + (size_t)(c.kv_heads << c.shift) * kBytes;
        return reinterpret_cast<uint32_t *>(at) + (head << c.shift) + (b & ((1 << c.shift) - 1));
    }
    // The recent tokens of a sequence's slot and a head, or null: keys [parity of the block][token][D], values
    // [parity][D][token].
    __device__ static __forceinline__ uint16_t *recent(const CacheArgs &c, int s, int head)
    {
        const int slot = c.slots ? c.slots[s] : s;
        if (slot < 0 || slot >= c.slot_count) return nullptr;
        return c.recent + ((size_t)slot * c.kv_heads + head) * kRecent;
    }
    __device__ static __forceinline__ int recent_key(int token, int d) { return (token & 31) * D + d; }
    __device__ static __forceinline__ int recent_value(int token, int d)
    {
        return 2 * kBlock * D + ((token >> 4) & 1) * (kBlock * D) + d * kBlock + (token & 15);
    }
};

__device__ __forceinline__ int cached_room(const CacheArgs &c) { return c.max_pages << (c.shift + 4); }
__device__ __forceinline__ int cached_length(const CacheArgs &c, int length)
{
    return min(max(length, 0), cached_room(c));
}

// Where the n rows of a sequence go, tokens first .. first + n - 1 (first may be negative): by its length as it is given, also
// where that is beyond the table's room, of which first is the most, so that tokens are counted with 32 bits.
__device__ __forceinline__ int first_token(const CacheArgs &c, int length, int n)
{
    return min(max(length, 0) - n, cached_room(c));
}

}  // namespace
