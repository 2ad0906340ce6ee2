// Queries and keys of fused QKV rows: the RMS norm of each head, if the model has one, and the rotation by position.
//
//   h = x / sqrt(mean(x^2) + eps) * gamma   (or h = x),
//   (y_a, y_b) = (h_a cos t - h_b sin t, h_b cos t + h_a sin t),   t = position * freq[i],
//
// for the pairs (a, b) = (i, i + rot / 2) of a head, or (2 i, 2 i + 1), i < rot / 2; y = h from rot on.  One rounding, to fp16.
//
// A lane takes sixteen elements of a head in two chunks of 16 bytes: both halves of eight pairs, or sixteen that are not
// rotated; D / 16 lanes hold a head and add up its squares.  The angles are the same for all heads of a token: the
// workgroup makes them first, each once, and keeps cosines and sines in LDS.  Turns are counted in 64 bits (position *
// (freq / 2 pi), less the nearest quarter), so that a position of a million is as good as one of ten; what is left, an
// eighth of a turn at most, goes through the Taylor series of sine and cosine, whose next terms are below 2^-28.
//
// Bound by memory (each row read and written once) where there are many, by the launch and two trips where there are few: 4096
// tokens of 64 + 8 heads of 128 take 28 us, 5.3 TB/s, with norms or without, one token 2.1 us.  A token's heads are spread over
// as many workgroups as they fill, each of which makes the angles; four tokens in one workgroup, which makes them once: 512
// tokens 6.0 -> 11.4 us, 4096 25.5 -> 28.7, 8192 50 -> 52.5.
#include "../../include/flexq.h"
#include "flexq_device.h"
#include "flexq_kernels.h"
#include "producer_math.h"
#include "sequences.h"

namespace {

struct RotateArgs {
    const uint16_t *x, *gamma_q, *gamma_k;
    uint16_t *out;
    const int32_t *positions;
    const float *freq;
    size_t x_stride, out_stride;
    int heads, all;                          // all: heads and key heads
    int rot;
    Divider by_chunks;                       // workgroups of a token
    float eps;
};

__device__ __forceinline__ float2 turn(int position, float freq)
{
    const double t = (double)position * ((double)freq * 0.15915494309189533577);
    const double q = rint(4.0 * t);
    const float a = (float)(t - 0.25 * q) * 6.28318530717958647693f, b = a * a;
    const float s = a * (1.0f + b * (-1.0f / 6 + b * (1.0f / 120 + b * (-1.0f / 5040 + b * (1.0f / 362880)))));
    const float c = 1.0f + b * (-0.5f + b * (1.0f / 24 + b * (-1.0f / 720 + b * (1.0f / 40320 + b * (-1.0f / 3628800)))));
    const int quarter = (int)(q - 4.0 * floor(0.25 * q));
    const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;          // up to their signs
    return make_float2(quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y);
}

template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs p)
{
    constexpr int LH = D / 16;               // lanes of a head
    __shared__ float2 angles[D / 2];
    const int m = divide(blockIdx.x, p.by_chunks), chunk = blockIdx.x - m * (int)p.by_chunks.d, half = p.rot / 2;
    const int lane = threadIdx.x % LH, pairs = p.rot / 16;       // the first `pairs` lanes of a head rotate
    const bool rotates = lane < pairs;
    const int a0 = !rotates || INTERLEAVED ? 16 * lane : 8 * lane;
    const int b0 = !rotates || INTERLEAVED ? a0 + 8 : half + 8 * lane;
    const int head = (chunk * 256 + (int)threadIdx.x) / LH;
    const uint16_t *x = p.x + (size_t)m * p.x_stride + (size_t)min(head, p.all - 1) * D;
    // (on their way while the angles are made)
    const uint4 va = *reinterpret_cast<const uint4 *>(x + a0), vb = *reinterpret_cast<const uint4 *>(x + b0);
    if ((int)threadIdx.x < half) angles[threadIdx.x] = turn(p.positions[m], p.freq[threadIdx.x]);
    __syncthreads();
    if (head >= p.all) return;
    const unsigned w[8] = {va.x, va.y, va.z, va.w, vb.x, vb.y, vb.z, vb.w};
    float v[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[2 * i] = h2f((uint16_t)(w[i] & 0xffffu));
        v[2 * i + 1] = h2f((uint16_t)(w[i] >> 16));
    }
    const uint16_t *gamma = head < p.heads ? p.gamma_q : p.gamma_k;
    if (gamma) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss += v[i] * v[i];
#pragma unroll
        for (int d = 1; d < LH; d <<= 1) ss += __shfl_xor(ss, d, 64);
        // (the unit takes numbers below the smallest normal one for zero, whose root's inverse times a head of zeros is NaN)
        const float inv = __builtin_amdgcn_rsqf(fmaxf(ss * (1.0f / D) + p.eps, 0x1p-126f));
        const uint4 ga = *reinterpret_cast<const uint4 *>(gamma + a0), gb = *reinterpret_cast<const uint4 *>(gamma + b0);
        const unsigned g[8] = {ga.x, ga.y, ga.z, ga.w, gb.x, gb.y, gb.z, gb.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[2 * i] = v[2 * i] * inv * h2f((uint16_t)(g[i] & 0xffffu));
            v[2 * i + 1] = v[2 * i + 1] * inv * h2f((uint16_t)(g[i] >> 16));
        }
    }
    if (rotates) {
        const float2 *angle = &angles[8 * lane];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = angle[i].x, s = angle[i].y;
            float &first = v[INTERLEAVED ? 2 * i : i], &second = v[INTERLEAVED ? 2 * i + 1 : 8 + i];
            const float a = first, b = second;
            first = a * c - b * s;
            second = b * c + a * s;
        }
    }
    uint16_t *out = p.out + (size_t)m * p.out_stride + (size_t)head * D;
    *reinterpret_cast<uint4 *>(out + a0) =
        make_uint4(pack_h2(v[0], v[1]), pack_h2(v[2], v[3]), pack_h2(v[4], v[5]), pack_h2(v[6], v[7]));
    *reinterpret_cast<uint4 *>(out + b0) =
        make_uint4(pack_h2(v[8], v[9]), pack_h2(v[10], v[11]), pack_h2(v[12], v[13]), pack_h2(v[14], v[15]));
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

flexq_status flexq_rotate_heads(const uint16_t *x, int x_stride, int M, int heads, int kv_heads, int head_dim,
                                const int32_t *positions, const float *freq, int rot, int interleaved,
                                const uint16_t *gamma_q, const uint16_t *gamma_k, float eps, uint16_t *out, int out_stride,
                                void *stream)
{
    if (!x || !positions || !freq || !out || M < 1 || heads < 1 || kv_heads < 1) return FLEXQ_EINVAL;
    if ((interleaved != 0 && interleaved != 1) || ((gamma_q || gamma_k) && !(eps > 0.0f && eps < INFINITY))) return FLEXQ_EINVAL;
    if ((head_dim != 64 && head_dim != 128) || rot < 16 || rot > head_dim || rot % 16 != 0) return FLEXQ_ESHAPE;
    if (((long)heads + kv_heads) * head_dim > FLEXQ_MAX_K) return FLEXQ_ESHAPE;
    const int width = (heads + kv_heads) * head_dim;
    if (x_stride < width || out_stride < width || x_stride % 8 != 0 || out_stride % 8 != 0) return FLEXQ_ESHAPE;
    if (x == out && x_stride != out_stride && M > 1) return FLEXQ_EINVAL;       // (one row has no next one)
    if (!aligned16(x) || !aligned16(out) || !aligned16(gamma_q) || !aligned16(gamma_k) || !aligned4(positions) || !aligned4(freq))
        return FLEXQ_EALIGN;
    RotateArgs p{};
    p.x = x;
    p.gamma_q = gamma_q;
    p.gamma_k = gamma_k;
    p.out = out;
    p.positions = positions;
    p.freq = freq;
    p.x_stride = (size_t)x_stride;
    p.out_stride = (size_t)out_stride;
    p.heads = heads;
    p.all = heads + kv_heads;
    p.rot = rot;
    p.eps = eps;
    const int chunks = (p.all * (head_dim / 16) + 255) / 256;
    p.by_chunks = divider(chunks);
    const long grid = (long)M * chunks;
    if (grid >= (1L << 24)) return FLEXQ_ESHAPE;                 // 256 threads each, 2^32 a launch
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream, p); };
    if (head_dim == 128)
        interleaved ? launch(rotate_kernel<128, true>) : launch(rotate_kernel<128, false>);
    else
        interleaved ? launch(rotate_kernel<64, true>) : launch(rotate_kernel<64, false>);
    return hipGetLastError() == hipSuccess ? FLEXQ_OK : FLEXQ_EHIP;
}

}  // extern "C"
#pragma GCC visibility pop
