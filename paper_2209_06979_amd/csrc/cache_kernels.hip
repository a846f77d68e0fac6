// Keys and values quantised as they are written into a paged cache, and read back:
//   scale = fp32(max |x| / qmax),  code = rint(x / scale), ties to even,  x' = code * scale   (qmax 127 or 7)
// for each vector of dk elements (a token's head).  Both directions stream: 8 elements a lane, a vector's lanes side by side.
// A code is decided as in double precision, from the key as it is after its rotation, which is carried in double precision, too: what lies next to
// a border of rounding goes by the definition and not by a sine's last bit.
// Memory bounds both.  16384 tokens of 8 heads of 128 fp16: read 102 MB in 20.4 us (4.9 TB/s, what a large copy reaches), written in 33.6 with keys rotated
// (the rotation and the quotients in double precision were 172 us for both before sines were shared and quotients decided in fp32), in 30 without, 3.4 TB/s.
#include "decode.h"
#include "rope.h"

#include <type_traits>

namespace {

constexpr int E = 8;     // elements of a lane
constexpr int AHEAD = 1; // vectors asked for before they are worked on (with 3, 16384 tokens' write and read took 54.0 us instead of 53.2)

// 8 elements as they lie in memory, and as fp32
template <class T> struct Raw8 {
    typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
    static constexpr int N = 16 / sizeof(T);
    Vec w[E / N];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int q = 0; q < E / N; ++q) w[q] = reinterpret_cast<const Vec *>(p)[q];
    }
    __device__ __forceinline__ float operator[](int e) const { return (float)w[e / N][e % N]; }
};

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

// The place of a token's head 0 in a cache, in vectors (the next heads follow a page's size apart); -1 for slots that are none
__device__ __forceinline__ int64_t place_of(const CacheArgs &a, int64_t slot)
{
    if (slot < 0 || slot >= a.slots_end) return -1;
    return ((slot >> a.page_shift) * a.kv_heads << a.page_shift) + (slot & (((int64_t)1 << a.page_shift) - 1));
}

// The largest over the LANES (8, 16 or 32) lanes that share a vector: rotations within rows of 16 lanes, the halves of 8 mirrored, and a swap of rows
template <int CTRL> __device__ __forceinline__ float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int CTRL> __device__ __forceinline__ double moved(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = (unsigned)__builtin_amdgcn_mov_dpp((int)(unsigned)b, CTRL, 0xF, 0xF, true), hi = (unsigned)__builtin_amdgcn_mov_dpp((int)(unsigned)(b >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, hi << 32 | lo);
}
template <int LANES, class REAL> __device__ __forceinline__ REAL max_of_lanes(REAL m)
{
    auto take = [&](REAL b) { m = b > m ? b : m; };
    take(moved<0xB1>(m));  // quad_perm 1 0 3 2
    take(moved<0x4E>(m));  // quad_perm 2 3 0 1
    take(moved<0x141>(m)); // row_half_mirror
    if (LANES >= 16) take(moved<0x140>(m)); // row_mirror
    if (LANES == 32) take(__shfl_xor(m, 16, 64));
    return m;
}

// m / qmax rounded to fp32 once.  (fp32 division is correctly rounded; in double the product with the inverse is within 2^-51, and only where that leaves the
// rounding open the division is made.)
__device__ __forceinline__ float scale_of(float m, float qmax) { return m / qmax; }
__device__ __forceinline__ float scale_of(double m, float qmax)
{
    const double q = m * (1.0 / qmax);
    const float lo = (float)(q * (1 - 0x1p-50)), hi = (float)(q * (1 + 0x1p-50));
    return lo == hi ? lo : (float)(m / (double)qmax);
}

// Codes of 8 values (REAL: float as read, or double after a rotation) and their scale; LANES lanes share the vector.  finite: all eight are.
// An fp32 quotient decides unless it lies within 1e-4 of a border of rounding (the value rounded to fp32, the inverse scale and their product are each within
// 2^-23: 5e-5 of 127 in all), and only then the division in double precision, for all eight.
template <class REAL, int BITS, int LANES> __device__ __forceinline__ float codes_of(const REAL (&v)[E], bool there, bool finite, unsigned (&w)[2])
{
    constexpr int QMAX = BITS == 8 ? 127 : 7;
    constexpr float MAGIC = 0x1.8p23f; // added, it rounds to whole numbers, ties to even, which then are the low bits
    REAL m = __builtin_elementwise_abs(v[0]);
#pragma unroll
    for (int e = 1; e < E; ++e) m = __builtin_elementwise_max(m, __builtin_elementwise_abs(v[e]));
    if (!finite) m = (REAL)__builtin_inf();
    if (!there) m = 0;
    m = max_of_lanes<LANES>(m);
    const float ratio = scale_of(m, (float)QMAX), scale = ratio < __builtin_inff() ? ratio : __builtin_nanf(""); // (rotated keys can have finite maxima whose ratio is not)
    w[0] = w[1] = 0;
    auto put = [&](int e, unsigned code) {
        if (BITS == 8) w[e / 4] |= (code & 255u) << (8 * (e % 4));
        else w[0] |= (code & 15u) << (4 * e);
    };
    if (scale >= 0x1p-100f) {
        const float inv = __builtin_amdgcn_rcpf(scale);
        float off = 0;
        unsigned code[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float r = (float)v[e] * inv, up = r + MAGIC;
            code[e] = __builtin_bit_cast(unsigned, up);
            off = __builtin_fmaxf(off, __builtin_fabsf(r - (up - MAGIC)));
        }
        if (off > 0.4999f || m > (REAL)__FLT_MAX__) { // (a rotated key beyond fp32 has no fp32 quotient)
#pragma unroll
            for (int e = 0; e < E; ++e) code[e] = (unsigned)(int)__builtin_rint((double)v[e] / (double)scale);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) put(e, code[e]); // (|v| / scale is at most qmax (1 + 2^-24))
    } else if (scale > 0) { // (too small for its inverse; and a subnormal scale can be off by more)
#pragma unroll
        for (int e = 0; e < E; ++e) put(e, (unsigned)(int)__builtin_fmin(__builtin_fmax(__builtin_rint((double)v[e] / (double)scale), (double)-QMAX), (double)QMAX));
    }
    return scale;
}

// How a key's elements find their partners: no rotation, the other element of the pair among the same lane's eight, eight elements side by side (rot / 2 a multiple of
// 8), or anywhere.
enum { PLAIN, PAIRS, HALVES, ANY_HALVES };

// Lanes in groups of LANES (a power of two, at least dk / 8) take a token's K and V vectors one after the other; a key's sines are worked out once.
template <int TYPE, int BITS, int LANES, int ROPE> __global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    const unsigned line = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, token = line / a.groups; // (threads are counted in 31 bits)
    const int first = (int)(line - token * a.groups), lane = threadIdx.x % LANES;
    if (token >= a.tokens) return;
    const int64_t place0 = place_of(a, a.slots[token]);
    if (place0 < 0) return;
    const bool there = lane * E < a.dk;
    const int at = there ? lane * E : 0, half = a.rot / 2;
    double c[E], s[E];       // of each element's pair
    bool turns = true;       // they are finite
    int other = at;          // where the other elements of the pairs are (HALVES)
    if (ROPE != PLAIN && first < a.kv_heads) {
        const double position = (double)a.positions[token];
        if (ROPE == HALVES && at < a.rot) other = at < half ? at + half : at - half;
        double f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) { // (all requests before the first use; elements beyond rot have the first frequency and no use for it)
            const int i = at + e;
            f[e] = a.inv_freq[i >= a.rot ? 0 : ROPE == PAIRS ? i / 2 : i >= half ? i - half : i];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = at + e;
            if (ROPE == PAIRS && e % 2 == 1) {
                c[e] = c[e - 1];
                s[e] = -s[e - 1];
                continue;
            }
            const SinCos<double> t = sin_cos_of<double>(position, f[e]);
            c[e] = i < a.rot ? t.c * a.magnitude : 1.0;
            s[e] = i < a.rot ? (ROPE != PAIRS && i >= half ? t.s : -t.s) * a.magnitude : 0.0;
            turns = turns && __builtin_fabs(c[e]) < __builtin_inf() && __builtin_fabs(s[e]) < __builtin_inf();
        }
    }
    struct Vector { Raw8<T> own, other; };
    // `turned`: keys on their rotation.  Heads from `head` on, `groups` apart; AHEAD of them are on their way while one is worked on.
    auto vectors = [&](auto turned, int which, int head) {
        constexpr bool TURNED = decltype(turned)::value;
        const T *x = static_cast<const T *>(a.x[which]) + token * a.token_stride[which] + head * a.head_stride[which];
        const int64_t step = a.groups * a.head_stride[which], place_step = (int64_t)a.groups << a.page_shift, place = place0 + ((int64_t)head << a.page_shift);
        uint8_t *to = a.codes[which] + (place * a.dk + at) * BITS / 8;
        float *scale_to = a.scales[which] + place;
        auto fetch = [&](Vector &v) {
            v.own.load(x + at);
            if (TURNED && ROPE == HALVES) v.other.load(x + other);
            if (TURNED && ROPE == ANY_HALVES) {
#pragma unroll
                for (int e = 0; e < E; ++e) v.other.w[e / Raw8<T>::N][e % Raw8<T>::N] = x[at + e >= a.rot ? at + e : at + e < half ? at + e + half : at + e - half];
            }
            x += step;
        };
        Vector v[AHEAD + 1];
#pragma unroll
        for (int d = 0; d < AHEAD; ++d)
            if (head + d * a.groups < a.kv_heads) fetch(v[d]);
        for (int h = head; h < a.kv_heads; h += a.groups) {
            if (h + AHEAD * a.groups < a.kv_heads) fetch(v[AHEAD]);
            float own[E];
            unsigned w[2], bits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                own[e] = v[0].own[e];
                const unsigned b = __builtin_bit_cast(unsigned, own[e]) & 0x7fffffffu;
                bits = b > bits ? b : bits;
            }
            const bool finite = bits < 0x7f800000u; // (an element that is not has its rotated pair among the vector's)
            float scale;
            if constexpr (TURNED) {
                double y[E];
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = (double)own[e] * c[e] + (double)(ROPE == PAIRS ? own[e ^ 1] : v[0].other[e]) * s[e];
                if (at + E > a.rot) { // (an infinity beyond rot has no part in its neighbour)
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (at + e >= a.rot) y[e] = (double)own[e];
                }
                scale = codes_of<double, BITS, LANES>(y, there, finite && turns, w);
            } else {
                scale = codes_of<float, BITS, LANES>(own, there, finite, w);
            }
            if (there) {
                if (BITS == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<unsigned *>(to) = w[0];
                if (lane == 0) *scale_to = scale;
            }
            to += place_step * a.dk * BITS / 8;
            scale_to += place_step;
#pragma unroll
            for (int d = 0; d < AHEAD; ++d) v[d] = v[d + 1];
        }
    };
    int j = first;
    if (first < a.kv_heads) {
        vectors(std::integral_constant<bool, ROPE != PLAIN>{}, 0, first);
        j += (a.kv_heads - first + a.groups - 1) / a.groups * a.groups;
    }
    if (j < 2 * a.kv_heads) vectors(std::false_type{}, 1, j - a.kv_heads);
}

// A lane takes 8 elements of its token's K and V vectors, one vector after the other.
template <int TYPE, int BITS> __global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    const unsigned pieces = a.dk / E, id = blockIdx.x * 256 + threadIdx.x, line = id / pieces, token = line / a.groups; // (threads are counted in 31 bits)
    const int at = (int)(id - line * pieces) * E, first = (int)(line - token * a.groups);
    if (token >= a.tokens) return;
    const int64_t place0 = place_of(a, a.slots[token]);
    for (int j = first; j < 2 * a.kv_heads; j += a.groups) {
        const int which = j >= a.kv_heads, head = which ? j - a.kv_heads : j;
        const int64_t place = place0 + ((int64_t)head << a.page_shift);
        float v[E] = {};
        if (place0 >= 0) {
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

// Lanes' groups that share a token's vectors: as many as fill the device (a group that takes several keys has their sines once).
// With these and with four times as many, 8 heads of 128 bf16, rotated: 16384 tokens 33.2 and 43.2 us, 512 tokens 5.8 and 6.0, 8 tokens 4.2 and 4.8.
constexpr int64_t THREADS = 256 * 1024;
int groups_of(const CacheArgs &a, int lanes)
{
    const int64_t per_token = a.tokens * lanes, groups = (THREADS + per_token - 1) / per_token;
    return groups < 2 * a.kv_heads ? (int)groups : 2 * a.kv_heads;
}

template <int TYPE, int BITS, int LANES> hipError_t write(CacheArgs a, hipStream_t s)
{
    a.groups = groups_of(a, LANES);
    const dim3 grid((unsigned)((a.tokens * a.groups + 256 / LANES - 1) / (256 / LANES))), block(256);
    if (a.rot == 0) return launch_kernel((cache_write_kernel<TYPE, BITS, LANES, PLAIN>), grid, block, 0, s, a);
    if (a.interleaved) return launch_kernel((cache_write_kernel<TYPE, BITS, LANES, PAIRS>), grid, block, 0, s, a);
    if (a.rot / 2 % E == 0) return launch_kernel((cache_write_kernel<TYPE, BITS, LANES, HALVES>), grid, block, 0, s, a);
    return launch_kernel((cache_write_kernel<TYPE, BITS, LANES, ANY_HALVES>), grid, block, 0, s, a);
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
