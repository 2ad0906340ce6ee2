// Causal attention over prompts packed one behind the other:
//
//   out_i = sum_{j <= i} p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j),   j in token i's sequence.
//
// Rows of a tile are the tokens of a sequence times the heads that share a key head, 32 a wavefront, so that grouped heads
// share the keys a workgroup stages and a short prompt fills a tile.  Keys and values come 64 at a time into LDS (direct
// loads, two buffers).  S^T = K Q^T by 32x32x16 MFMAs: a lane holds 32 scores of one row, lane l ^ 32 the row's other 32.  Its
// scores in the order of the registers are the column operand of O^T = V^T P^T for keys {0..3, 8..11} + 4 (l / 32) of every
// sixteen; the row operand is read from LDS transposed, in that order of keys, so that weights never cross lanes.
//
// The maximum that is taken off a score, m, is not the running one but one it was at some time: p = 2^(x - m + 9), and as long as a
// lane's 32 of a stage add up to 2^15 at most -- which the running sum needs anyway -- nothing overflows in fp16.  Where they
// do not (at the first stage, and rarely after it) m becomes the running maximum, and what was added up is scaled down.  So the
// maximum of each stage, a quarter of its vector instructions, is not taken.  p is normal down to 2^-23 of the largest;
// its sum is fp32, unrounded.
//
// What bounds it: power.  16384 tokens of 64 heads over 8 take 4.25 ms, 1.03 PFLOP/s (of what the mask leaves; PyTorch's
// fp16 product of 8192^3 reaches 1.14), the matrix pipe busy 53 % of the cycles at 1.9 GHz.  A form that interleaves exponentials
// with matrix instructions, one block's beside the next one's scores, took 12 % fewer cycles, but at 1.76 GHz, for 1 % of the
// time; without any load of keys and values, at 1.6 GHz, it would take 3.65 ms.  Operands of S four reads ahead of the
// instruction that takes them: 4.31 -> 4.2.  4 wavefronts instead of 8: 4.28, but two workgroups a CU, and so better
// below some thousand tokens (1024 tokens 32 -> 37 us, packed prompts of 300 37 -> 49 with 8).  Heads of 64 have half the matrix
// work to an exponential: the vector unit is 78 % busy, the matrix pipe 55 % (16384 tokens of 24 heads over 6 892 us, 0.92 PFLOP/s).
// Prompts of some thousand tokens wait for the tiles with most stages: with 1024 tokens of 64 heads over 8, 32 us, a CU is busy
// for 59 % of the launch, with 2048, 91 us, for 79 %.  Short prompts are bound by the rows
// themselves and by what a workgroup does before its first stage, about 6000 cycles of trips and 2500 of a first stage (100 of 37
// tokens, 133 MB, 38 us; nine of 3001 in all, heads of 64, 19: the longest one's twelve stages in a row).
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "gemm_common.h"
#include "producer_math.h"
#include "sequences.h"

namespace {

constexpr int kKeys = 64;                        // of a stage
constexpr float kNothing = -1e30f;
constexpr float kShift = 9.0f, kMost = 32768.0f;

struct PromptArgs {
    const uint16_t *q, *k, *v;
    uint16_t *out;
    const int32_t *starts;
    size_t q_stride, k_stride, v_stride, out_stride;
    int M, count, group, kv_heads, pieces;       // pieces: workgroups of a key head
    Divider by_group, by_kv;
    float scale;                                 // times log2 e
};

__device__ __forceinline__ v16f mfma_h(v8h a, v8h b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// A lane's four keys of one channel, of 16 lanes' four channels of one key each.
__device__ __forceinline__ v4h read_transposed(const uint8_t *at)
{
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s *lds_ptr;
    union {
        v4s s;
        v4h h;
    } x;
    x.s = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
    return x.h;
}

// Which chunk of 16 bytes of a staged row lies where: XOR by the row, so that a cycle's lanes (256 bytes) meet every bank
// once -- sixteen keys' same chunk; 32 channels of four keys, read transposed.
template <int D>
__device__ __forceinline__ int key_swizzle(int line)
{
    return D == 128 ? line & 15 : (line >> 1) & 7;
}
template <int D>
__device__ __forceinline__ int value_swizzle(int line)
{
    return D == 128 ? 4 * (line & 3) : 4 * ((line >> 1) & 1);
}

template <int D, int WAVES, int SPLIT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void prompt_kernel(PromptArgs a)
{
    // SPLIT wavefronts share 32 rows, each with its keys of every stage
    constexpr int ROWS = 32 * WAVES / SPLIT, NB = kKeys / 32 / SPLIT;     // NB: blocks of 32 keys of a wavefront
    constexpr int LINE = 2 * D, CH = D / 8;           // LINE: bytes of a staged row; CH: its chunks
    constexpr int STAGE = kKeys * LINE, DMA = STAGE / 1024 / WAVES;      // DMA: loads of a wavefront for keys, or values
    static_assert(STAGE % (1024 * WAVES) == 0, "a stage is whole loads of every wavefront");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][STAGE];  // [buffer][keys, values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, i32 = lane & 31;
    const int group = wave / SPLIT, part = wave % SPLIT * NB;            // its rows and, of a stage, its first block of keys
    const int index = divide(blockIdx.x, a.by_kv), head = blockIdx.x - index * a.kv_heads;
    // the tiles with most keys first
    const RowRange r = find_rows(a.starts, a.count, a.M, a.group, ROWS, 1, a.pieces - 1 - index);
    if (r.id < 0) return;
    const int all = r.n * a.group, row0 = r.piece * ROWS;
    if (row0 >= all) return;
    const int rows = min(ROWS, all - row0);
    const int keys = divide(row0 + rows - 1, a.by_group) + 1;                    // that the last row sees
    const int stages = (keys + kKeys - 1) / kKeys;
    // this lane's row, and what its wavefront sees
    const int row = row0 + min(32 * group + i32, rows - 1), token = divide(row, a.by_group);
    const bool mine = 32 * group + i32 < rows;
    const int w_first = row0 + 32 * group, w_last = row0 + min(32 * group + 31, rows - 1);
    const int sees_all = divide(w_first, a.by_group), sees_any = 32 * group < rows ? divide(w_last, a.by_group) : -1;
    const int q_head = head * a.group + row - token * a.group;
    v8h q[D / 16];
    {
        const uint16_t *from = a.q + (size_t)(r.begin + token) * a.q_stride + (size_t)q_head * D + 8 * half;
#pragma unroll
        for (int m = 0; m < D / 16; ++m) q[m] = *reinterpret_cast<const v8h *>(from + 16 * m);
    }
    // stages: load i of a wavefront fills 1 KiB, lane l 16 bytes at 16 l, and so fetches the chunk that the swizzle keeps there
    // rows past the sequence's end repeat its last one: they are hidden, and p = 0 meets finite values
    const uint16_t *k0 = a.k + (size_t)r.begin * a.k_stride + (size_t)head * D;
    const uint16_t *v0 = a.v + (size_t)r.begin * a.v_stride + (size_t)head * D;
    unsigned k_from[DMA], v_from[DMA];               // of whole stages
    auto from = [&](int i, int most, unsigned line_bytes, bool values) {
        const int at = (wave * DMA + i) * 64 + lane, line = at / CH, swizzle = values ? value_swizzle<D>(line) : key_swizzle<D>(line);
        return (unsigned)min(line, most) * line_bytes + 16u * (unsigned)(at % CH ^ swizzle);
    };
    const unsigned k_line = 2 * (unsigned)a.k_stride, v_line = 2 * (unsigned)a.v_stride;
#pragma unroll
    for (int i = 0; i < DMA; ++i) {
        k_from[i] = from(i, kKeys, k_line, false);
        v_from[i] = from(i, kKeys, v_line, true);
    }
    auto fetch = [&](int stage, int buf) {
        const int most = min(kKeys, r.n - stage * kKeys) - 1;
        const __amdgpu_buffer_rsrc_t kr =
            __builtin_amdgcn_make_buffer_rsrc((void *)(k0 + (size_t)stage * kKeys * a.k_stride), 0, (unsigned)most * k_line + LINE, 0x00020000);
        const __amdgpu_buffer_rsrc_t vr =
            __builtin_amdgcn_make_buffer_rsrc((void *)(v0 + (size_t)stage * kKeys * a.v_stride), 0, (unsigned)most * v_line + LINE, 0x00020000);
#pragma unroll
        for (int i = 0; i < DMA; ++i) {
            uint8_t *dst = &lds[buf][0][(wave * DMA + i) * 1024];
            const unsigned off = most == kKeys - 1 ? k_from[i] : from(i, most, k_line, false);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (void __attribute__((address_space(3))) *)dst, 16, off, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < DMA; ++i) {
            uint8_t *dst = &lds[buf][1][(wave * DMA + i) * 1024];
            const unsigned off = most == kKeys - 1 ? v_from[i] : from(i, most, v_line, true);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (void __attribute__((address_space(3))) *)dst, 16, off, 0, 0, 0);
        }
    };
    v16f o[D / 32];
    float top = kNothing, sum = 0.0f;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    fetch(0, 0);
    for (int stage = 0; stage < stages; ++stage) {
        const int buf = stage & 1;
        wait_vmcnt<0>();
        lds_barrier();                           // everyone's loads of this stage are there, and everyone is done with the last one
        if (stage + 1 < stages) fetch(stage + 1, buf ^ 1);
        const int first = stage * kKeys + 32 * part;
        if (first > sees_any) continue;
        const uint8_t *ks = lds[buf][0] + 32 * part * LINE, *vs = lds[buf][1] + 32 * part * LINE;
        v16f s[NB];
        {
            constexpr int AHEAD = 4;                 // operands asked for ahead of the instruction that takes them
            v8h ring[AHEAD];
            auto key_part = [&](int n) {             // n: block n % NB, channels 16 (n / NB) ..
                const int line = 32 * (n % NB) + i32;
                return *reinterpret_cast<const v8h *>(ks + line * LINE + 16 * ((2 * (n / NB) + half) ^ key_swizzle<D>(line)));
            };
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) ring[n] = key_part(n);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
#pragma unroll
            for (int n = 0; n < D / 16 * NB; ++n) {
                s[n % NB] = mfma_h(ring[n % AHEAD], q[n / NB], s[n % NB]);
                if (n + AHEAD < D / 16 * NB) ring[n % AHEAD] = key_part(n + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (first + 32 * NB - 1 > sees_all) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (first + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3) > token) s[b][i] = -INFINITY;
        }
        v8h p[NB][2];
        float total;
        auto weights = [&] {
            const float less = top - kShift;
            total = 0.0f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.scale, -less));
                    const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i + 1], a.scale, -less));
                    total += e0;
                    total += e1;
                    const v2h h = __builtin_convertvector((v2f{e0, e1}), v2h);
                    p[b][i / 8][i % 8] = h[0];
                    p[b][i / 8][i % 8 + 1] = h[1];
                }
        };
        if (stage != 0) weights();
        if (stage == 0 || __any(total > kMost)) {    // a score far above m: at the first stage, all of them
            float x = s[0][0];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) x = fmaxf(x, s[b][i]);
            auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
            const float next = fmaxf(top, fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])) * a.scale);
            const float f = __builtin_amdgcn_exp2f(top - next);
            top = next;
            sum *= f;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= f;
            weights();
        }
        sum += total;
        // lane (dsub, h) of sixteen lanes each: keys 4 h + 0 .. 3 (and 8 more on) of channels 16 dsub .. + 15
        const int h = lane >> 5, dsub = lane >> 4 & 1, e = lane >> 2 & 3, c4 = lane & 3;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int t = 0; t < D / 32; ++t) {
                    union {
                        v4h h[2];
                        v8h v;
                    } x;
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int line = 32 * b + 16 * u + 8 * w + 4 * h + e;
                        const int c = (4 * t + 2 * dsub + (c4 >> 1)) ^ value_swizzle<D>(line);
                        x.h[w] = read_transposed(vs + line * LINE + 16 * c + 8 * (c4 & 1));
                    }
                    o[t] = mfma_h(x.v, p[b][u], o[t]);
                }
    }
    if constexpr (SPLIT == 2) {                        // the second wavefront's share to the first, lane by lane
        constexpr int UNITS = D / 8, SHARE = (UNITS + 1) * 64;
        v4f *share = reinterpret_cast<v4f *>(&lds[0][0][0]) + group * SHARE + lane;
        static_assert(WAVES / SPLIT * SHARE * 16 <= (int)sizeof(lds), "shares fit into the stages' place");
        lds_barrier();
        if (part != 0) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    share[64 * (4 * t + i)] = v4f{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
            share[64 * UNITS] = v4f{top, sum, 0.0f, 0.0f};
        }
        lds_barrier();
        if (part != 0) return;
        const v4f other = share[64 * UNITS];
        const float next = fmaxf(top, other[0]), f = __builtin_amdgcn_exp2f(top - next), g = __builtin_amdgcn_exp2f(other[0] - next);
        sum = sum * f + other[1] * g;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v4f x = share[64 * (4 * t + i)];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][4 * i + e] = o[t][4 * i + e] * f + x[e] * g;
            }
    }
    {
        auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    if (!mine) return;
    const float inv = 1.0f / sum;
    uint16_t *out = a.out + (size_t)(r.begin + token) * a.out_stride + (size_t)q_head * D + 4 * half;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint2 *>(out + 32 * t + 8 * i) = make_uint2(
                pack_h2(within_half(o[t][4 * i] * inv), within_half(o[t][4 * i + 1] * inv)),
                pack_h2(within_half(o[t][4 * i + 2] * inv), within_half(o[t][4 * i + 3] * inv)));
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

flexq_status flexq_prompt_attention(const uint16_t *q, int q_stride, const uint16_t *k, int k_stride, const uint16_t *v,
                                    int v_stride, const int32_t *starts, int sequences, int M, int heads, int kv_heads,
                                    int head_dim, float scale, uint16_t *out, int out_stride, void *stream)
{
    if (!q || !k || !v || !starts || !out || sequences < 1 || M < 1 || heads < 1 || kv_heads < 1) return FLEXQ_EINVAL;
    if (heads % kv_heads != 0 || !(scale > 0.0f && scale <= 65504.0f)) return FLEXQ_EINVAL;
    if ((head_dim != 64 && head_dim != 128) || (long)heads * head_dim > FLEXQ_MAX_K) return FLEXQ_ESHAPE;
    const int width = heads * head_dim, kv_width = kv_heads * head_dim;
    if (q_stride < width || out_stride < width || k_stride < kv_width || v_stride < kv_width) return FLEXQ_ESHAPE;
    if (q_stride % 8 != 0 || out_stride % 8 != 0 || k_stride % 8 != 0 || v_stride % 8 != 0) return FLEXQ_ESHAPE;
    // (a stage's rows are addressed with 32 bits)
    if (k_stride > (1 << 23) || v_stride > (1 << 23) || sequences > (1 << 20)) return FLEXQ_ESHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned4(starts)) return FLEXQ_EALIGN;
    PromptArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = out;
    a.starts = starts;
    a.q_stride = (size_t)q_stride;
    a.k_stride = (size_t)k_stride;
    a.v_stride = (size_t)v_stride;
    a.out_stride = (size_t)out_stride;
    a.M = M;
    a.count = sequences;
    a.group = heads / kv_heads;
    a.kv_heads = kv_heads;
    a.scale = scale * 1.44269504088896341f;
    if ((long)M * a.group >= (1L << 30)) return FLEXQ_ESHAPE;
    // 256 rows a workgroup instead of 128 where they fill the chip four times over, and heads are of 128 (us with 128 / 256
    // rows: 16384 tokens of 64 heads over 8 4280 / 4200, 8192 of 32 543 / 533, 4096 of 64 over 8 287 / 289; heads of 64, 16384
    // of 24 over 6, 873 / 940)
    const int waves = head_dim == 128 && (long)M * a.group / 256 * kv_heads >= 1024 ? 8 : 4;
    // Two wavefronts to 32 rows where there are too few for the chip and the longest chain of stages counts: a workgroup a CU or
    // two, of long sequences (us with one / two: 512 tokens of 32 heads 14.3 / 12.2, 1500 37 / 34, of 8 heads over 1 5000 99 / 80;
    // heads of 64, 2600 of 24 over 6 42 / 35; but 900 of 64 over 8, 450 workgroups, 28.0 / 29.7, 4 x 200 of 40 12.7 / 15.6)
    const int split = waves == 4 && (long)M * a.group / 128 * kv_heads <= (head_dim == 64 ? 512 : 384) &&
                      M >= (head_dim == 64 ? 256L : 512L) * sequences ? 2 : 1;
    const int rows = 32 * waves / split;
    const long pieces = (long)M * a.group / rows + sequences, grid = pieces * kv_heads;
    if (grid * 64 * waves >= (1L << 32)) return FLEXQ_ESHAPE;            // threads of a launch
    a.pieces = (int)pieces;
    a.by_group = divider(a.group);
    a.by_kv = divider(kv_heads);
    auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(64 * waves), 0, (hipStream_t)stream, a);
    };
    if (head_dim == 64)
        split == 2 ? launch(prompt_kernel<64, 4, 2>) : launch(prompt_kernel<64, 4, 1>);
    else
        waves == 8 ? launch(prompt_kernel<128, 8, 1>) : split == 2 ? launch(prompt_kernel<128, 4, 2>) : launch(prompt_kernel<128, 4, 1>);
    return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
