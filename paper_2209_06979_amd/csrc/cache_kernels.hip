// Keys and values quantised as they are written into a paged cache, and read back:
//   scale = fp32(max |x| / qmax),  code = rint(x / scale), ties to even,  x' = code * scale   (qmax 127 or 7)
// for each vector of dk elements (a token's head).  Both directions stream: 8 elements a lane, a vector's lanes side by side.
// A code is decided as in double precision, from the key as it is after its rotation, which is carried in double precision, too: what lies next to
// a border of rounding goes by the definition and not by a sine's last bit.
#include "decode.h"
#include "rope.h"

namespace {

constexpr int E = 8; // elements of a lane

template <class T> __device__ __forceinline__ void load8(const T *p, float (&v)[E])
{
    typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int q = 0; q < E / N; ++q) {
        const Vec w = reinterpret_cast<const Vec *>(p)[q];
#pragma unroll
        for (int e = 0; e < N; ++e) v[q * N + e] = (float)w[e];
    }
}

template <class T> __device__ __forceinline__ void store8(T *p, const float (&v)[E])
{
    typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int q = 0; q < E / N; ++q) {
        Vec w;
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = (T)v[q * N + e];
        reinterpret_cast<Vec *>(p)[q] = w;
    }
}

// A vector's place in a cache, in vectors; -1 for slots that are none
__device__ __forceinline__ int64_t place_of(const CacheArgs &a, int64_t slot, int head)
{
    if (slot < 0 || slot >= a.slots_end) return -1;
    const int64_t page = slot >> a.page_shift, in_page = slot & (((int64_t)1 << a.page_shift) - 1);
    return ((page * a.kv_heads + head) << a.page_shift) + in_page;
}

// Codes of 8 values (REAL: float as read, or double after a rotation) and their scale; LANES lanes share the vector.
template <class REAL, int BITS, int LANES> __device__ __forceinline__ float codes_of(const REAL (&v)[E], bool there, unsigned (&w)[2])
{
    constexpr int QMAX = BITS == 8 ? 127 : 7;
    REAL m = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const REAL b = __builtin_fabs(v[e]);
        m = b > m || !(b < (REAL)__builtin_inf()) ? ((b < (REAL)__builtin_inf()) ? b : (REAL)__builtin_inf()) : m; // (a NaN counts as infinity)
    }
    if (!there) m = 0;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        const REAL b = __shfl_xor(m, o, 64);
        m = b > m ? b : m;
    }
    const bool finite = m < (REAL)__builtin_inf();
    const float scale = finite ? (float)((double)m / QMAX) : __builtin_nanf("");
    w[0] = w[1] = 0;
    if (finite && scale > 0) {
        const double inv = 1.0 / (double)scale;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const double q = (double)v[e] * inv;
            double c = __builtin_rint(q);
            if (__builtin_fabs(__builtin_fabs(q - c) - 0.5) < 1e-9) c = __builtin_rint((double)v[e] / (double)scale);
            const int code = (int)__builtin_fmin(__builtin_fmax(c, (double)-QMAX), (double)QMAX);
            if (BITS == 8) w[e / 4] |= (unsigned)(code & 255) << (8 * (e % 4));
            else w[0] |= (unsigned)(code & 15) << (4 * e);
        }
    }
    return scale;
}

// Lanes in groups of LANES (a power of two, at least dk / 8) take a token's K and V vectors one after the other.
template <int TYPE, int BITS, int LANES, bool ROPE> __global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    const int64_t line = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES, token = line / a.groups;
    const int first = (int)(line - token * a.groups), lane = threadIdx.x % LANES;
    if (token >= a.tokens) return;
    const int64_t slot = a.slots[token];
    const bool there = lane * E < a.dk;
    const int at = there ? lane * E : 0, half = a.rot / 2;
    double c[E], s[E]; // of each element's pair
    int other[E];      // the pair's other element
    if constexpr (ROPE) {
        const double position = (double)a.positions[token];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = at + e;
            c[e] = 1;
            s[e] = 0;
            other[e] = i;
            if (i < a.rot) {
                const bool second = a.interleaved ? i & 1 : i >= half;
                const SinCos<double> t = sin_cos_of<double>(position, a.inv_freq[a.interleaved ? i / 2 : second ? i - half : i]);
                c[e] = t.c * a.magnitude;
                s[e] = (second ? t.s : -t.s) * a.magnitude;
                other[e] = a.interleaved ? i ^ 1 : second ? i - half : i + half;
            }
        }
    }
    for (int j = first; j < 2 * a.kv_heads; j += a.groups) {
        const int which = j >= a.kv_heads, head = which ? j - a.kv_heads : j;
        const int64_t place = place_of(a, slot, head);
        if (place < 0) continue;
        const T *x = static_cast<const T *>(a.x[which]) + token * a.token_stride[which] + head * a.head_stride[which];
        float v[E];
        unsigned w[2];
        float scale;
        load8(x + at, v);
        if (ROPE && !which) {
            double y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = (double)v[e] * c[e] + (double)(float)x[other[e]] * s[e];
            scale = codes_of<double, BITS, LANES>(y, there, w);
        } else {
            scale = codes_of<float, BITS, LANES>(v, there, w);
        }
        if (!there) continue;
        uint8_t *to = a.codes[which] + (place * a.dk + at) * BITS / 8;
        if (BITS == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<unsigned *>(to) = w[0];
        if (lane == 0) a.scales[which][place] = scale;
    }
}

// A lane takes 8 elements of its token's K and V vectors, one vector after the other.
template <int TYPE, int BITS> __global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    const int pieces = a.dk / E;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, line = id / pieces, token = line / a.groups;
    const int at = (int)(id - line * pieces) * E, first = (int)(line - token * a.groups);
    if (token >= a.tokens) return;
    const int64_t slot = a.slots[token];
    for (int j = first; j < 2 * a.kv_heads; j += a.groups) {
        const int which = j >= a.kv_heads, head = which ? j - a.kv_heads : j;
        const int64_t place = place_of(a, slot, head);
        float v[E] = {};
        if (place >= 0) {
            const float scale = a.scales[which][place];
            const uint8_t *from = a.codes[which] + (place * a.dk + at) * BITS / 8;
            unsigned w[2] = {};
            if (BITS == 8) {
                const uint2 u = *reinterpret_cast<const uint2 *>(from);
                w[0] = u.x;
                w[1] = u.y;
            } else {
                w[0] = *reinterpret_cast<const unsigned *>(from);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int code = BITS == 8 ? (int)(w[e / 4] << (24 - 8 * (e % 4))) >> 24 : (int)(w[0] << (28 - 4 * e)) >> 28;
                v[e] = (float)code * scale;
            }
        }
        store8(static_cast<T *>(a.x[which]) + token * a.token_stride[which] + head * a.head_stride[which] + at, v);
    }
}

template <int TYPE, int BITS, int LANES> hipError_t write(CacheArgs a, hipStream_t s)
{
    a.groups = 2 * a.kv_heads;
    const dim3 grid((unsigned)((a.tokens * a.groups + 256 / LANES - 1) / (256 / LANES))), block(256);
    if (a.rot) return launch_kernel((cache_write_kernel<TYPE, BITS, LANES, true>), grid, block, 0, s, a);
    return launch_kernel((cache_write_kernel<TYPE, BITS, LANES, false>), grid, block, 0, s, a);
}

template <int TYPE, int BITS> hipError_t write_bits(const CacheArgs &a, hipStream_t s)
{
    if (a.dk <= 64) return write<TYPE, BITS, 8>(a, s);
    if (a.dk <= 128) return write<TYPE, BITS, 16>(a, s);
    return write<TYPE, BITS, 32>(a, s);
}

template <int TYPE> hipError_t write_type(const CacheArgs &a, hipStream_t s)
{
    return a.bits == 8 ? write_bits<TYPE, 8>(a, s) : write_bits<TYPE, 4>(a, s);
}

template <int TYPE> hipError_t read_type(CacheArgs a, hipStream_t s)
{
    a.groups = 2 * a.kv_heads;
    const dim3 grid((unsigned)((a.tokens * a.groups * (a.dk / E) + 255) / 256)), block(256);
    if (a.bits == 8) return launch_kernel((cache_read_kernel<TYPE, 8>), grid, block, 0, s, a);
    return launch_kernel((cache_read_kernel<TYPE, 4>), grid, block, 0, s, a);
}

} // namespace

hipError_t launch_cache_write(const CacheArgs &a, mc_type type, hipStream_t s)
{
    if (type == MC_F32) return write_type<MC_F32>(a, s);
    if (type == MC_F16) return write_type<MC_F16>(a, s);
    return write_type<MC_BF16>(a, s);
}

hipError_t launch_cache_read(const CacheArgs &a, mc_type type, hipStream_t s)
{
    if (type == MC_F32) return read_type<MC_F32>(a, s);
    if (type == MC_F16) return read_type<MC_F16>(a, s);
    return read_type<MC_BF16>(a, s);
}
