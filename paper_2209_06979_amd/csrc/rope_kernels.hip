// Rotary positions of queries and keys before they are quantised: pair j of a head is turned by position * frequency[j],
//   y1 = m (x1 cos - x2 sin),   y2 = m (x1 sin + x2 cos),
// the pairs (j, j + rot/2) or, interleaved, (2j, 2j + 1); what lies beyond rot is copied.  The gradient is the same with the
// angle reversed.  Memory bounds it: a thread works out the sines of its pairs once and takes them through several heads of its token, 16 bytes at a time, so that
// the double-precision angle is paid by few.  Measured: 134 MB of bf16 in 24.5 us (5.5 TB/s, where a large copy reaches 4.8), 31.5 MB of interleaved fp32, rotated in part,
// in 7.6 us; a step of 1 MB 3.2 us, which is a launch.
#include "decode.h"
#include "rope.h"

namespace {

// VEC: pairs of a thread and head (1: any alignment).  Thread numbers run over the pieces of a head (pairs, then what is copied,
// 2 VEC elements each), the groups that share a token's heads, and tokens, so that neighbours read neighbouring bytes.
template <int TYPE, int VEC, bool INTERLEAVED> __global__ __launch_bounds__(256) void rope_kernel(RopeArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    typedef T Vec __attribute__((ext_vector_type(VEC > 1 ? VEC : 2)));
    const int half = a.rot / 2, turned = half / VEC, rest = a.dim - a.rot;
    const unsigned id = blockIdx.x * 256 + threadIdx.x, pieces = turned + (rest + 2 * VEC - 1) / (2 * VEC); // (threads are counted in 31 bits)
    const unsigned line = id / pieces, token = line / a.groups;
    const int piece = (int)(id - line * pieces), first = (int)(line - token * a.groups);
    if (token >= a.tokens) return;
    const T *x = static_cast<const T *>(a.x) + token * a.x_token_stride;
    T *y = static_cast<T *>(a.y) + token * a.y_token_stride;
    if (piece >= turned) { // copied
        const int at = a.rot + (piece - turned) * 2 * VEC, n = a.dim - at < 2 * VEC ? a.dim - at : 2 * VEC;
        for (int64_t h = first; h < a.heads; h += a.groups) {
            const T *from = x + h * a.x_head_stride + at;
            T *to = y + h * a.y_head_stride + at;
            if (VEC > 1 && n == 2 * VEC) {
                const Vec v1 = reinterpret_cast<const Vec *>(from)[0], v2 = reinterpret_cast<const Vec *>(from)[1];
                reinterpret_cast<Vec *>(to)[0] = v1;
                reinterpret_cast<Vec *>(to)[1] = v2;
            } else {
                for (int e = 0; e < n; ++e) to[e] = from[e];
            }
        }
        return;
    }
    const int j = piece * VEC;
    const double position = (double)a.positions[token];
    float c[VEC], s[VEC];
    double f[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = a.inv_freq[j + e];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const SinCos<float> t = sin_cos_of<float>(position, f[e]);
        c[e] = t.c * (float)a.cos_scale;
        s[e] = t.s * (float)a.sin_scale;
    }
    const int at1 = INTERLEAVED ? 2 * j : j, at2 = INTERLEAVED ? 2 * j + VEC : j + half;
    auto turn = [&](int64_t h) {
        const T *from = x + h * a.x_head_stride;
        T *to = y + h * a.y_head_stride;
        T v[2 * VEC], w[2 * VEC];
        if constexpr (VEC > 1) {
            const Vec v1 = *reinterpret_cast<const Vec *>(from + at1), v2 = *reinterpret_cast<const Vec *>(from + at2);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = v1[e], v[VEC + e] = v2[e];
        } else {
            v[0] = from[at1];
            v[1] = from[at2];
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int i1 = INTERLEAVED ? 2 * e : e, i2 = INTERLEAVED ? 2 * e + 1 : VEC + e;
            const float x1 = (float)v[i1], x2 = (float)v[i2];
            w[i1] = (T)(x1 * c[e] - x2 * s[e]);
            w[i2] = (T)(x1 * s[e] + x2 * c[e]);
        }
        if constexpr (VEC > 1) {
            Vec w1, w2;
#pragma unroll
            for (int e = 0; e < VEC; ++e) w1[e] = w[e], w2[e] = w[VEC + e];
            *reinterpret_cast<Vec *>(to + at1) = w1;
            *reinterpret_cast<Vec *>(to + at2) = w2;
        } else {
            to[at1] = w[0];
            to[at2] = w[1];
        }
    };
    for (int64_t h = first; h < a.heads; h += a.groups) turn(h);
}

// Threads that share a token's heads: as many as fill the device twice over (a thread that takes several heads has its sines for them once).
// With these, a quarter of them and four times as many, 32 heads of 128 bf16: 16384 tokens 43.3, 47.9 and 44.8 us; 2048 tokens 8.2, 7.2, 8.2; 8 tokens 3.0, 3.4, 2.9.
constexpr int64_t THREADS = 2 * 256 * 2048;

template <int TYPE, int VEC> hipError_t launch(const RopeArgs &a, hipStream_t s)
{
    const int64_t pieces = a.rot / 2 / VEC + (a.dim - a.rot + 2 * VEC - 1) / (2 * VEC), threads = a.tokens * a.groups * pieces;
    const dim3 grid((unsigned)((threads + 255) / 256)), block(256);
    if (a.interleaved) return launch_kernel((rope_kernel<TYPE, VEC, true>), grid, block, 0, s, a);
    return launch_kernel((rope_kernel<TYPE, VEC, false>), grid, block, 0, s, a);
}

template <int TYPE> hipError_t launch_type(RopeArgs a, hipStream_t s)
{
    constexpr int VEC = 16 / sizeof(typename RealOf<TYPE>::type);
    const int64_t strides = a.x_token_stride | a.x_head_stride | a.y_token_stride | a.y_head_stride | (a.rot / 2);
    const bool wide = strides % VEC == 0 && ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y)) & 15) == 0;
    const int64_t per_token = a.tokens * ((a.dim + 1) / 2 / (wide ? VEC : 1) + 1), groups = (THREADS + per_token - 1) / per_token;
    a.groups = groups < a.heads ? (int)groups : a.heads;
    return wide ? launch<TYPE, VEC>(a, s) : launch<TYPE, 1>(a, s);
}

} // namespace

hipError_t launch_rope(const RopeArgs &a, mc_type type, hipStream_t s)
{
    if (type == MC_F32) return launch_type<MC_F32>(a, s);
    if (type == MC_F16) return launch_type<MC_F16>(a, s);
    return launch_type<MC_BF16>(a, s);
}
