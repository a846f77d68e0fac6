// Log probabilities of given tokens, the entropy of their distributions and the most likely tokens, in one pass over the logits; and
// the gradient in another.  With m a row's largest logit, d = x - m, z = scale d:
//   s = sum e^z,  t = sum e^z d,   log p = z - log s,   entropy = log s - scale t / s,
// kept per thread for the largest x so far and rescaled when a larger one comes (four vectors of 16 bytes at a time).
// The largest `top` logits are kept by each wave as keys in one register pair, sorted over its lanes: a vector whose largest element is below
// the last of them is passed over by one comparison, and an element above it is moved into its place.  The four waves of a workgroup share a
// bound: where each has a quarter of `top` keys that reach it, what is below it is not among the row's `top`.  It comes first from the largest element of
// each lane after the first vectors, sorted, so that only about `top` elements are put in place at the start, and rises with the waves' keys.
// A row is read by one workgroup, or cut into pieces where there are few rows; a second kernel joins these.
// Reading bounds them: fp32 8192 x 50257 272 us, 6.0 TB/s; of 16-bit logits an element's conversion, difference, exponential and sums take most of the time that its bytes do (2048 x 128000 bf16 101 us, 5.2 TB/s;
// with 20 alternatives 116).  The gradient reads and writes as a copy does: 8192 x 50257 bf16 294 us, 5.6 TB/s.
#include "layer.h"

#include "lds_async.h"

namespace {

typedef unsigned long long Key; // an orderable logit, and the complement of its index: larger is earlier

constexpr int THREADS = 256, WAVES = THREADS / 64, UNROLL = 4;
// FAR: what a difference counts as at most: 2^30 times it is finite, and the smallest scale times it has an exponential of 0.
constexpr float LOWEST = -3.402823466e38f, FAR = -1e28f;

template <int TYPE> struct Vector {
    typedef typename RealOf<TYPE>::type T;
    static constexpr int N = 16 / sizeof(T);
    T e[N];
};

// (rows of any width begin anywhere: vectors are loaded and stored at the element's alignment)
template <int TYPE> __device__ __forceinline__ Vector<TYPE> load(const typename RealOf<TYPE>::type *p)
{
    Vector<TYPE> v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// Vector `i` of a row; elements beyond the row's end are -infinity.
template <int TYPE> __device__ __forceinline__ Vector<TYPE> load_guarded(const typename RealOf<TYPE>::type *row, int i, int end, int vocab)
{
    constexpr int N = Vector<TYPE>::N;
    typedef typename RealOf<TYPE>::type T;
    if (i < end && (i + 1) * N <= vocab) return load<TYPE>(row + (int64_t)i * N);
    Vector<TYPE> v;
#pragma unroll
    for (int e = 0; e < N; ++e) v.e[e] = i < end && i * N + e < vocab ? row[i * N + e] : (T)-__builtin_inff();
    return v;
}

// Orders as the logits do, both zeros alike; NaN above all.
__device__ __forceinline__ unsigned ordered(float x)
{
    const int b = __float_as_int(x + 0.0f);
    const unsigned u = b < 0 ? ~(unsigned)b : (unsigned)b | 0x80000000u;
    return x == x ? u : 0xffffffffu;
}
__device__ __forceinline__ float logit_of(Key k)
{
    const unsigned u = (unsigned)(k >> 32);
    return __int_as_float((int)(u & 0x80000000u ? u & 0x7fffffffu : ~u));
}
__device__ __forceinline__ Key larger(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key smaller(Key a, Key b) { return a > b ? b : a; }
__device__ __forceinline__ Key key_of_lane(Key k, int lane)
{
    return (Key)(unsigned)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)k, lane);
}

// The key of the lane before (lane 0: its own)
__device__ __forceinline__ Key key_before(Key k)
{
    const int hi = (int)(k >> 32), lo = (int)k;
    return (Key)(unsigned)__builtin_amdgcn_update_dpp(hi, hi, 0x138, 0xf, 0xf, false) << 32 | (unsigned)__builtin_amdgcn_update_dpp(lo, lo, 0x138, 0xf, 0xf, false);
}

// The 64 largest of two lists that fall from lane 0 on (`other` read backwards): larger elements of both make a bitonic list, which six exchanges sort.
__device__ __forceinline__ Key merged(Key held, Key other_backwards, int lane)
{
    Key k = larger(held, other_backwards);
#pragma unroll
    for (int j = 32; j > 0; j >>= 1) {
        const Key o = __shfl_xor(k, j);
        k = (lane & j) == 0 ? larger(k, o) : smaller(k, o);
    }
    return k;
}

// Lanes' values, falling from lane 0 on.
__device__ __forceinline__ unsigned sorted(unsigned x, int lane)
{
#pragma unroll
    for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const unsigned o = __shfl_xor(x, j);
            const bool falling = (lane & k) == 0 || k == 64, first = (lane & j) == 0;
            x = falling == first ? max(x, o) : min(x, o);
        }
    return x;
}

struct Sums { float m, s, t; };
// (s is 0 where nothing but -infinity was seen; the differences are kept finite so that 0 times them is 0)
__device__ __forceinline__ Sums joined(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m), da = fmaxf(a.m - m, FAR), db = fmaxf(b.m - m, FAR);
    const float fa = __builtin_amdgcn_exp2f(da * c), fb = __builtin_amdgcn_exp2f(db * c);
    return {m, a.s * fa + b.s * fb, (a.t + a.s * da) * fa + (b.t + b.s * db) * fb};
}
// Of all lanes, the same in each (their sums by themselves may differ by a rounding: equal logits would have unequal log probabilities)
__device__ __forceinline__ Sums over_lanes(Sums a, float c)
{
#pragma unroll
    for (int j = 32; j > 0; j >>= 1) a = joined(a, {__shfl_xor(a.m, j), __shfl_xor(a.s, j), __shfl_xor(a.t, j)}, c);
    auto first = [](float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); };
    return {first(a.m), first(a.s), first(a.t)};
}

// One wave writes a row's results.
template <int TYPE> __device__ __forceinline__ void finish(const LogprobArgs &a, int64_t row, Sums z, Key held, int lane)
{
    typedef typename RealOf<TYPE>::type T;
    const bool none = z.s == 0;
    const float log_s = logf(z.s), inf = __builtin_inff();
    if (lane == 0) {
        const int64_t token = a.tokens[row];
        float p = 0;
        if (token >= 0 && token < a.vocab) p = none ? -inf : ((float)static_cast<const T *>(a.logits)[row * a.stride + token] - z.m) * a.scale - log_s;
        a.logprobs[row] = p;
        const float h = none ? 0 : log_s - a.scale * (z.t / z.s);
        a.entropy[row] = h < 0 ? 0 : h;
        if (a.sums) {
            a.sums[2 * row] = none ? 0 : z.m;
            a.sums[2 * row + 1] = none ? inf : log_s; // (infinite: no element has a probability)
        }
    }
    if (lane < a.top) {
        a.top_logprobs[row * a.top + lane] = none ? -inf : (logit_of(held) - z.m) * a.scale - log_s;
        a.top_tokens[row * a.top + lane] = (int64_t)(unsigned)~(unsigned)held;
    }
}

template <int TYPE, bool TOP> __global__ __launch_bounds__(THREADS) void logprob_kernel(LogprobArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int N = Vector<TYPE>::N;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / (unsigned)a.pieces;
    const int piece = (int)(blockIdx.x - row * a.pieces);
    // Vectors begin at whole dwords: of rows that begin between two, behind the first element, which one thread takes by itself.
    // (bf16, 8192 x 50257 184 -> 172 us, 2048 x 128003 115 -> 100; vectors at whole dwords are as fast as at 16 bytes)
    const T *const row_x = static_cast<const T *>(a.logits) + row * a.stride;
    const int lead = sizeof(T) == 2 && a.vocab >= 64 && (reinterpret_cast<uintptr_t>(row_x) & 2) ? 1 : 0;
    const T *const x = row_x + lead;
    const int vocab = a.vocab - lead, vectors = (vocab + N - 1) / N;
    const int first = piece * a.piece_vectors, end = min(first + a.piece_vectors, vectors), whole = min(end, vocab / N);
    const float c = a.scale * 1.4426950408889634f;
    Sums z = {LOWEST, 0, 0};
    const T before_x = row_x[0];
    Key held = 0;                    // of this lane's place
    Key last = 0;                    // the key at place top - 1, of all lanes
    unsigned bound = 0;              // what a key's logit has to reach
    const int quarter = TOP ? (a.top + WAVES - 1) / WAVES - 1 : 0; // place of a wave's key that the bound goes by
    __shared__ unsigned reached[WAVES]; // those keys' logits: they only rise, so that a wave that reads old ones has a lower bound
    auto common = [&] {
        unsigned b = __hip_atomic_load(&reached[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) b = min(b, __hip_atomic_load(&reached[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        bound = max(bound, (unsigned)__builtin_amdgcn_readfirstlane((int)b));
    };
    // Lanes' keys, one after the other, into their places
    auto insert = [&](Key k, bool there) {
        unsigned long long more = __ballot(there && (unsigned)(k >> 32) >= bound && k > last);
        while (more) {
            const int l = __builtin_ctzll(more);
            more &= more - 1;
            const Key fresh = key_of_lane(k, l);
            if (fresh <= last) continue;
            const int place = __builtin_popcountll(__ballot(held > fresh));
            const Key before = key_before(held);
            held = lane < place ? held : lane == place ? fresh : before;
            last = key_of_lane(held, a.top - 1);
            bound = max(bound, (unsigned)(last >> 32));
        }
    };
    for (int at = first; at < end; at += THREADS * UNROLL) {
        Vector<TYPE> v[UNROLL];
        const int i = at + (int)threadIdx.x;
        if (at + THREADS * UNROLL <= whole) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) v[u] = load<TYPE>(x + (int64_t)(i + u * THREADS) * N);
        } else {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) v[u] = load_guarded<TYPE>(x, i + u * THREADS, end, vocab);
        }
        float most[UNROLL]; // (a NaN stays one)
        float m = z.m;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            most[u] = (float)v[u].e[0];
#pragma unroll
            for (int e = 1; e < N; ++e) most[u] = __builtin_elementwise_maximum(most[u], (float)v[u].e[e]);
            m = fmaxf(m, most[u]);
        }
        const float step = fmaxf(z.m - m, FAR), f = __builtin_amdgcn_exp2f(step * c);
        z.t = (z.t + z.s * step) * f;
        z.s *= f;
        z.m = m;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float d = (float)v[u].e[e] - m, p = __builtin_amdgcn_exp2f(d * c);
                z.s += p;
                z.t += p * fmaxf(d, FAR);
            }
        if constexpr (TOP) {
            if (at == first) {
                unsigned o = ordered(most[0]);
#pragma unroll
                for (int u = 1; u < UNROLL; ++u) o = max(o, ordered(most[u]));
                o = sorted(o, lane);
                bound = (unsigned)__builtin_amdgcn_readlane((int)o, a.top - 1); // (at least `top` of this wave's elements reach it)
                if (lane == quarter) reached[wave] = o;
                __syncthreads(); // (every wave comes here once: a piece is no shorter than one batch's first vectors, or its elements are -infinity)
            }
            common();
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float least = logit_of((Key)bound << 32); // (a NaN is not below it)
                if (__ballot(!(most[u] < least)) == 0) continue;
                const int from = (i + u * THREADS) * N;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (__ballot(!((float)v[u].e[e] < least)) == 0) continue;
                    const Key k = (Key)ordered((float)v[u].e[e]) << 32 | (unsigned)~(unsigned)(from + e + lead);
                    insert(k, from + e < vocab);
                    least = logit_of((Key)bound << 32);
                }
            }
            // (a key of 0 stands for none)
            const unsigned mine = (unsigned)(key_of_lane(held, quarter) >> 32);
            if (lane == 0 && mine > __hip_atomic_load(&reached[wave], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP))
                __hip_atomic_store(&reached[wave], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
    }

    __shared__ Sums sums[WAVES];
    __shared__ Key keys[TOP ? WAVES : 1][64];
    if (lead && piece == 0 && wave == 0) {
        const float v = (float)before_x, inf = __builtin_inff();
        if (lane == 0 && v != -inf) z = joined(z, v < inf ? Sums{v, 1, 0} : Sums{LOWEST, __builtin_nanf(""), 0}, c);
        if constexpr (TOP) insert((Key)ordered(v) << 32 | 0xffffffffu, lane == 0);
    }
    z = over_lanes(z, c);
    if (lane == 0) sums[wave] = z;
    if constexpr (TOP) keys[wave][lane] = held;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        z = joined(z, sums[w], c);
        if constexpr (TOP) held = merged(held, keys[w][63 - lane], lane);
    }
    if (a.pieces == 1) return finish<TYPE>(a, row, z, held, lane);
    float *to = a.partial + (row * a.pieces + piece) * logprob_partial(a.top);
    if (lane == 0) to[0] = z.m, to[1] = z.s, to[2] = z.t;
    if (TOP && lane < a.top) reinterpret_cast<Key *>(to + 4)[lane] = held;
}

// A row's pieces, joined: their sums by one wave, a lane each, their keys by all.
template <int TYPE, bool TOP> __global__ __launch_bounds__(THREADS) void logprob_join_kernel(LogprobArgs a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x;
    const float *from = a.partial + row * a.pieces * logprob_partial(a.top);
    const float c = a.scale * 1.4426950408889634f;
    __shared__ Key keys[TOP ? WAVES : 1][64];
    Key held = 0;
    if constexpr (TOP) {
        for (int p = wave; p < a.pieces; p += WAVES) {
            const Key other = 63 - lane < a.top ? reinterpret_cast<const Key *>(from + p * logprob_partial(a.top) + 4)[63 - lane] : 0;
            held = merged(held, other, lane);
        }
        keys[wave][lane] = held;
        __syncthreads();
    }
    if (wave != 0) return;
    Sums z = {LOWEST, 0, 0};
    if (lane < a.pieces) {
        const float *p = from + lane * logprob_partial(a.top);
        z = {p[0], p[1], p[2]};
    }
    z = over_lanes(z, c);
    if constexpr (TOP)
#pragma unroll
        for (int w = 1; w < WAVES; ++w) held = merged(held, keys[w][63 - lane], lane);
    finish<TYPE>(a, row, z, held, lane);
}

// d logits_j = scale (sum of the gradients of what names j - p_j (G + dH (log p_j + H))), G the sum of all gradients of log
// probabilities.  A workgroup takes a stretch of a row; elements that are named again (tokens and alternatives) are written once more at
// the end by the thread that knows all of their terms.
template <int TYPE> __global__ __launch_bounds__(THREADS) void logprob_backward_kernel(LogprobArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int N = Vector<TYPE>::N;
    const int64_t row = blockIdx.x / (unsigned)a.pieces;
    const int piece = (int)(blockIdx.x - row * a.pieces), vectors = (a.vocab + N - 1) / N;
    const int first = piece * (THREADS * UNROLL), end = min(first + THREADS * UNROLL, vectors), whole = min(end, a.vocab / N);
    const T *x = static_cast<const T *>(a.logits) + row * a.stride;
    T *dx = static_cast<T *>(a.dlogits) + row * a.dstride;
    Vector<TYPE> v[UNROLL];
    const int i = first + (int)threadIdx.x;
    const bool all = first + THREADS * UNROLL <= whole;
    if (all) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) v[u] = load<TYPE>(x + (int64_t)(i + u * THREADS) * N);
    } else {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) v[u] = load_guarded<TYPE>(x, i + u * THREADS, end, a.vocab);
    }
    const int64_t token = a.tokens[row];
    const bool none = a.sums[2 * row + 1] == __builtin_inff();
    const bool named = token >= 0 && token < a.vocab && !none;
    const float m = a.sums[2 * row], log_s = a.sums[2 * row + 1], h = a.entropy[row];
    const float dl = named && a.dlogprobs ? a.dlogprobs[row] : 0, dh = a.dentropy ? a.dentropy[row] : 0;
    float g = dl;
    if (a.dtop && !none)
        for (int k = 0; k < a.top; ++k) g += a.dtop[row * a.top + k];
    auto gradient = [&](float l) {
        const float logp = (l - m) * a.scale - log_s, p = __builtin_amdgcn_exp2f(logp * 1.4426950408889634f);
        return p == 0 ? 0.0f : -p * (g + dh * (logp + h));
    };
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int64_t from = (int64_t)(i + u * THREADS) * N;
        Vector<TYPE> d;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float y = gradient((float)v[u].e[e]);
            if (named && from + e == token) y += dl;
            d.e[e] = (T)(y * a.scale);
        }
        if (all) {
            __builtin_memcpy(dx + from, &d, 16);
        } else if (i + u * THREADS < end) {
            asm volatile("" ::: "memory"); // (whole vectors are written as such)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (from + e < a.vocab) dx[from + e] = d.e[e];
            asm volatile("" ::: "memory");
        }
    }
    if (!a.dtop || none) return;
    __syncthreads(); // (the stores above have been made)
    if ((int)threadIdx.x < a.top) {
        const int64_t j = a.chosen[row * a.top + threadIdx.x];
        if (j >= (int64_t)first * N && j < (int64_t)end * N && j < a.vocab) {
            float y = gradient((float)x[j]) + a.dtop[row * a.top + threadIdx.x];
            if (named && j == token) y += dl;
            dx[j] = (T)(y * a.scale);
        }
    }
}

template <int TYPE> hipError_t forward(const LogprobArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows * a.pieces)), block(THREADS);
    const hipError_t e = a.top ? launch_kernel((logprob_kernel<TYPE, true>), grid, block, 0, s, a) : launch_kernel((logprob_kernel<TYPE, false>), grid, block, 0, s, a);
    if (e != hipSuccess || a.pieces == 1) return e;
    const dim3 rows((unsigned)a.rows);
    return a.top ? launch_kernel((logprob_join_kernel<TYPE, true>), rows, block, 0, s, a) : launch_kernel((logprob_join_kernel<TYPE, false>), rows, block, 0, s, a);
}

template <int TYPE> hipError_t backward(LogprobArgs a, hipStream_t s)
{
    constexpr int PER = THREADS * UNROLL * Vector<TYPE>::N;
    a.pieces = (a.vocab + PER - 1) / PER;
    return launch_kernel(logprob_backward_kernel<TYPE>, dim3((unsigned)(a.rows * a.pieces)), dim3(THREADS), 0, s, a);
}

} // namespace

hipError_t launch_token_logprobs(const LogprobArgs &a, hipStream_t s)
{
    return a.type == MC_F32 ? forward<MC_F32>(a, s) : a.type == MC_F16 ? forward<MC_F16>(a, s) : forward<MC_BF16>(a, s);
}

hipError_t launch_token_logprobs_backward(const LogprobArgs &a, hipStream_t s)
{
    return a.type == MC_F32 ? backward<MC_F32>(a, s) : a.type == MC_F16 ? backward<MC_F16>(a, s) : backward<MC_BF16>(a, s);
}
