// The gated feed-forward block, h = act(x Wg^T) (x Wu^T), and its gradient
//   dg = dh u act'(g),   du = dh act(g),   dx = dg Wg + du Wu,   dWg = dg^T x,   dWu = du^T x.
// Three products of matrices, of one tiled kernel: for the first k lies along the rows of both operands, for dx along those of dg and du alone, for dWg and dWu along
// none; operands that have a row for each k are transposed on their way from LDS into registers.
#include "layer.h"

#include "lds_async.h"

namespace {

using mcu::v4f;
using mcu::v4i;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// ---- activations ----------------------------------------------------------------------------------------------------------
// Of 16-bit types: the hardware's exponential and reciprocal, each within a step or two: of a sigmoid some |g| 2^-23 of itself where it is small, far below a rounding
// of h, dg and du.  (With the library's exponential and quotient the activation of a 256 x 128 tile took as long as a seventh of its products.)  fp32 keeps all of its bits.
template <int TYPE> __device__ __forceinline__ float sigmoid(float g)
{
    if constexpr (TYPE == MC_F32) return 1.0f / (1.0f + expf(-g));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}
constexpr float GELU_A = 0.7978845608028654f, GELU_B = 0.044715f;

template <int KIND, int TYPE> __device__ __forceinline__ float activated(float g)
{
    if constexpr (KIND == MC_ACT_SILU) return g * sigmoid<TYPE>(g);
    else if constexpr (KIND == MC_ACT_GELU) return 0.5f * g * (1.0f + erff(g * 0.7071067811865476f));
    else if constexpr (KIND == MC_ACT_GELU_TANH) return g * sigmoid<TYPE>(2.0f * GELU_A * (g + GELU_B * g * g * g)); // ((1 + tanh v) / 2 is sigmoid 2 v)
    else if constexpr (KIND == MC_ACT_RELU) return g > 0 ? g : g != g ? g : 0;
    else return sigmoid<TYPE>(g);
}
// act(g), and its slope
template <int KIND, int TYPE> __device__ __forceinline__ float activated(float g, float &slope)
{
    if constexpr (KIND == MC_ACT_SILU) {
        const float p = sigmoid<TYPE>(g);
        slope = p * (1.0f + g * (1.0f - p));
        return g * p;
    } else if constexpr (KIND == MC_ACT_GELU) {
        const float c = 0.5f * (1.0f + erff(g * 0.7071067811865476f));
        slope = c + g * __builtin_amdgcn_exp2f(g * g * -0.7213475204444817f) * 0.3989422804014327f;
        return g * c;
    } else if constexpr (KIND == MC_ACT_GELU_TANH) {
        const float p = sigmoid<TYPE>(2.0f * GELU_A * (g + GELU_B * g * g * g));
        const float q = p * (1.0f - p); // (0 far from 0, where the cube may be infinite)
        slope = q == 0 ? p : p + q * 2.0f * GELU_A * (g + 3.0f * GELU_B * g * g * g);
        return g * p;
    } else if constexpr (KIND == MC_ACT_RELU) {
        slope = g > 0 ? 1 : g != g ? g : 0;
        return g > 0 ? g : g != g ? g : 0;
    } else {
        const float p = sigmoid<TYPE>(g);
        slope = p * (1.0f - p);
        return p;
    }
}
// f with the activation as a constant
template <class F> __device__ __forceinline__ void with_activation(int kind, F &&f)
{
    switch (kind) {
    case MC_ACT_SILU: return f(std::integral_constant<int, MC_ACT_SILU>{});
    case MC_ACT_GELU: return f(std::integral_constant<int, MC_ACT_GELU>{});
    case MC_ACT_GELU_TANH: return f(std::integral_constant<int, MC_ACT_GELU_TANH>{});
    case MC_ACT_RELU: return f(std::integral_constant<int, MC_ACT_RELU>{});
    default: return f(std::integral_constant<int, MC_ACT_SIGMOID>{});
    }
}

// ---- matrix instructions ----------------------------------------------------------------------------------------------------
// 16 rows of either operand, 16 bytes of each along k: a lane holds piece lane / 16 of row lane % 16.  (fp32: element e of the four pieces are
// the four k of instruction e.)  The result has 4 rows of the first, 4 (lane / 16) + i, for row lane % 16 of the second.
template <int TYPE> __device__ __forceinline__ v4f multiply_one(const v4i &a, const v4i &b, const v4f &c) // (16-bit types)
{
    if constexpr (TYPE == MC_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
template <int TYPE, int N, int M> __device__ __forceinline__ void multiply(const v4i (&a)[N], const v4i (&b)[M], v4f (&c)[N][M])
{
    if constexpr (TYPE == MC_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) // (an instruction's sum is the next one's after all others)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int m = 0; m < M; ++m) c[n][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[n][e]), __int_as_float(b[m][e]), c[n][m], 0, 0, 0);
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int m = 0; m < M; ++m) c[n][m] = multiply_one<TYPE>(a[n], b[m], c[n][m]);
    }
}

// RUN neighbouring elements, `n` of them.
template <class T, int RUN> __device__ __forceinline__ void store_run(T *to, const float (&v)[RUN], int n)
{
    T h[RUN];
#pragma unroll
    for (int e = 0; e < RUN; ++e) h[e] = (T)v[e];
    if (n >= RUN) return (void)__builtin_memcpy(to, h, RUN * sizeof(T));
    asm volatile("" ::: "memory"); // (the compiler would else make some of the stores those of both cases, and write whole runs in parts)
#pragma unroll
    for (int e = 0; e < RUN; ++e)
        if (e < n) to[e] = h[e];
    asm volatile("" ::: "memory");
}

// ---- the tiled product ------------------------------------------------------------------------------------------------------
__device__ const v4i zeros[1] = {};

constexpr int TOGETHER = 8;         // tiles of rows that follow one another for the same columns
enum { PLAIN, GATED, PARTIAL };     // what becomes of a tile: C, act(g) u, or fp32 sums of a piece of k

typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

// One operand's share of the kernel: X of its rows (m or n) to a tile, of which a wave multiplies X / SHARES in FRAGMENTS of 16, STEP bytes of k at a time (64 or 128).
// ROWS false: k along rows.  LDS holds lines of 128 bytes, a row's eight pieces of 16 or two rows' four, at places (piece ^ line % 8): what a read
// addresses at once has different banks.
// ROWS true: a row for each k.  LDS holds the rows, in units of 16 elements at places (unit ^ turned(row)), for the same reason.
template <int TYPE, int X, int SHARES, int WAVES, int STEP, bool ROWS> struct Operand {
    typedef typename RealOf<TYPE>::type T;
    static constexpr int SIZE = sizeof(T), PER = 16 / SIZE, KS = STEP / SIZE, BYTES = X * STEP, COPIES = BYTES / 1024 / WAVES, FRAGMENTS = X / SHARES / 16;
    static constexpr int LINE = X * SIZE, LANES = LINE / 16, UNITS = X / 16; // of a row of the second form
    static constexpr int TO_LINE = 128 / STEP;                              // rows of a line of the first
    static_assert(COPIES * 1024 * WAVES == BYTES && FRAGMENTS * 16 * SHARES == X, "whole copies and fragments");
    unsigned from[COPIES];  // of the lane's pieces, behind the step's address
    unsigned at[FRAGMENTS]; // of the lane's fragments, behind the stage's address

    static __device__ __forceinline__ int turned(int row) { return (SIZE == 4 ? row >> 2 & 3 : (row & 3) | (row >> 3 & 1) << 2) & (UNITS - 1); }
    // of the lane's piece of a copy: its place within the line, its row, and its number along k
    static __device__ __forceinline__ int place(int lane) { return (lane & 7) ^ (lane >> 3); }
    static __device__ __forceinline__ int row_of(int copy, int lane)
    {
        if constexpr (ROWS) return copy * (64 / LANES) + lane / LANES;
        else return (copy * 8 + (lane >> 3)) * TO_LINE + (TO_LINE == 2 ? place(lane) >> 2 : 0);
    }
    static __device__ __forceinline__ int piece(int lane) { return TO_LINE == 2 ? place(lane) & 3 : place(lane); }
    // the tile's rows from `first` on of `count`
    __device__ __forceinline__ void set(int first, int count, int64_t stride, int w, int lane)
    {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int row = row_of(w * COPIES + i, lane);
            if constexpr (ROWS) {
                const int place = lane % LANES, column = (place / SIZE ^ turned(row)) * 16 + place % SIZE * PER;
                from[i] = (unsigned)(row * stride) + (first + column < count ? column * SIZE : 0); // (columns beyond the last are never stored)
            } else {
                from[i] = (unsigned)((min(first + row, count - 1) - first) * stride) + piece(lane) * 16;
            }
        }
    }
    // the wave's share
    __device__ __forceinline__ void fragments(int share, int lane)
    {
        const int i = lane & 15, q = lane >> 4;
#pragma unroll
        for (int f = 0; f < FRAGMENTS; ++f) {
            const int unit = share * FRAGMENTS + f;
            if constexpr (!ROWS && TO_LINE == 2) at[f] = unit * 16 * STEP + (i >> 1) * 128 + ((((i & 1) * 4 + q) ^ (i >> 1)) * 16);
            else if constexpr (!ROWS) at[f] = (unit * 16 + i) * STEP;
            else if constexpr (SIZE == 4) at[f] = 4 * q * LINE + (unit ^ (q & (UNITS - 1))) * 64 + i * 4;
            else at[f] = (8 * q + (i >> 2)) * LINE + (unit ^ turned(8 * q + (i >> 2))) * 32 + (i & 3) * 8;
        }
    }
    // what the lane's piece of copy i begins with along k, of the step's
    static __device__ __forceinline__ int begins(int copy, int lane) { return ROWS ? row_of(copy, lane) : piece(lane) * PER; }
    // Fragment f, 64 bytes of k from 64 h on.
    __device__ __forceinline__ v4i read(const char *stage, int f, int h, int lane) const
    {
        if constexpr (!ROWS) {
            return *reinterpret_cast<const v4i *>(stage + at[f] + (TO_LINE == 2 ? 0 : ((h * 4 + (lane >> 4)) ^ (lane & 7)) * 16));
        } else if constexpr (SIZE == 4) {
            v4i v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const int *>(stage + at[f] + (h * 16 + e) * LINE);
            return v;
        } else { // four rows of 16 elements become four elements of 16 rows, twice
            const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(stage + at[f] + h * 32 * LINE));
            const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(stage + at[f] + (h * 32 + 4) * LINE));
            return __builtin_bit_cast(v4i, (__attribute__((ext_vector_type(8))) short){a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w});
        }
    }
};

// The value, made wide here and not ahead of a loop (the pairs would be spilled).
__device__ __forceinline__ uint64_t here(unsigned x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// What a workgroup multiplies at a time: a tile of one of the products, over all of k or a piece.
struct Work { int m0, n0, z, split, first, steps; };

// The matrix units bound it, and tiles as large as the registers hold (256 x 256 of 16-bit types: 128 accumulators a lane) have the fewest bytes from LDS to a product.  8192 rows of 4096
// bf16: h of 14336 in 1430 .. 1480 us, 1300 .. 1345 Tflop/s (a library's 8192^3 product on the same card 1320); with g and u kept h of 11008 in 1232, dx 1104 (1338 Tflop/s), both weights' gradients 1354 (1091: all operands are
// transposed on their way out of LDS).  fp32, 777 rows of 1001 to 2731: 103, 105 and 90 us, 82 Tflop/s (a library's 4096^3 132): 1118 tiles of 64 x 64 for
// h, 208 of them in six pieces along k for dx, 704 of 128 x 64 for the weights are 4.4, 4.9 and 2.75 to a compute unit, and the slowest unit has five, five and three.  Operands that have to be
// copied first: 777 rows of bf16, 1001 to 2731 28 us where 1000 to 2736 take 19, both passes 87 and 77; 8192 rows of 4095 to 11008, both passes, 4199 and (4096) 3994.
// BM x BN tiles, WM x WN waves, NS stages of STEP bytes of k.  GATED: the rows of B are half gate's, half up's, such that each wave has both of its columns; where it has 32 of
// them, a lane's eight neighbouring ones.
template <int TYPE, int BM, int BN, int WM, int WN, int STEP, int NS, bool AR, bool BR, int MODE> __global__ __launch_bounds__(64 * WM *WN) void product_kernel(ProductArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int W = WM * WN, RM = BM / WM, RN = BN / WN, MF = RM / 16, NF = RN / 16, STAGE = (BM + BN) * STEP;
    constexpr int KS = STEP / sizeof(T), COLUMNS = MODE == GATED ? BN / 2 : BN;
    constexpr bool EIGHT = MODE == GATED && RN % 64 == 0;
    typedef Operand<TYPE, BM, WM, W, STEP, AR> A;
    typedef Operand<TYPE, BN, WN, W, STEP, BR> B;
    constexpr int COPIES = A::COPIES + B::COPIES;
    static_assert(MODE != GATED || (!AR && !BR), "weights lie with k along their rows");
    __shared__ __attribute__((aligned(1024))) char lds[NS][STAGE];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WN, wn = w % WN;

    // Workgroups go to the eight XCDs round-robin: each XCD has a run of the work, in blocks of TOGETHER tiles of rows, and its workgroups take turns.
    const int tiles = a.tiles_m * a.tiles_n, all = tiles * (MODE == GATED ? 1 : a.batch) * (MODE == PARTIAL ? a.splits : 1);
    const int per = (all + 7) / 8, xcd = blockIdx.x & 7, turns = gridDim.x >> 3, end = min(xcd * per + per, all);
    const int each = (a.k + KS - 1) / KS; // steps of one of the products of a sum
    auto work = [&](int u) {
        const int o = u / tiles, t = u - o * tiles, block = t / (TOGETHER * a.tiles_n), high = min(TOGETHER, a.tiles_m - block * TOGETHER), in = t - block * TOGETHER * a.tiles_n;
        const int batch = MODE == GATED ? 1 : a.batch, steps = MODE == GATED ? each : each * a.sum;
        Work v = {(block * TOGETHER + in % high) * BM, in / high * COLUMNS, o % batch, o / batch, 0, steps};
        if constexpr (MODE == PARTIAL) {
            v.first = (int)((int64_t)steps * v.split / a.splits);
            v.steps = (int)((int64_t)steps * (v.split + 1) / a.splits) - v.first;
        }
        return v;
    };

    // What is being asked for
    A oa;
    B ob;
    oa.fragments(wm, lane);
    ob.fragments(wn, lane);
    const char *pa[2], *pb[2], *gated[B::COPIES]; // (pa, pb: of the products of a sum)
    const int64_t a_ahead = AR ? KS * a.a_stride : STEP, b_ahead = BR ? KS * a.b_stride[0] : STEP;
    const unsigned base = mcu::lds_addr_uniform(lds);
    Work asked;
    auto ask_of = [&](int u) {
        asked = work(u);
        oa.set(asked.m0, a.m, a.a_stride, w, lane);
        pa[0] = static_cast<const char *>(asked.z ? a.a[1] : a.a[0]) + (AR ? asked.m0 * (int64_t)sizeof(T) : asked.m0 * a.a_stride);
        pa[1] = static_cast<const char *>(a.a[1]) + (AR ? asked.m0 * (int64_t)sizeof(T) : asked.m0 * a.a_stride);
        if constexpr (MODE == GATED) {
#pragma unroll
            for (int i = 0; i < B::COPIES; ++i) {
                const int first = (w * B::COPIES + i) * 8 * B::TO_LINE, which = first % RN >= RN / 2, in = (first + B::row_of(0, lane)) % (RN / 2);
                // (row 16 f + 4 q + e of 32 holds column 8 q + 4 f + e)
                const int column = first / RN * (RN / 2) + (EIGHT ? (in & ~31) + (in >> 2 & 3) * 8 + (in >> 4 & 1) * 4 + (in & 3) : in);
                const int64_t stride = which ? a.b_stride[1] : a.b_stride[0];
                gated[i] = static_cast<const char *>(which ? a.b[1] : a.b[0]) + asked.n0 * stride;
                ob.from[i] = (unsigned)((min(asked.n0 + column, a.n - 1) - asked.n0) * stride) + B::piece(lane) * 16;
            }
        } else {
            ob.set(asked.n0, a.n, a.b_stride[0], w, lane);
            pb[0] = static_cast<const char *>(a.b[0]) + (BR ? asked.n0 * (int64_t)sizeof(T) : asked.n0 * a.b_stride[0]);
            pb[1] = static_cast<const char *>(a.b[1]) + (BR ? asked.n0 * (int64_t)sizeof(T) : asked.n0 * a.b_stride[0]);
        }
    };
    // A step's copies: their bases, and whether all of the step is there
    struct Step { const char *a, *b; int second; int64_t b_at; int left; };
    auto step_of = [&](int s) {
        const int step = asked.first + s, second = MODE != GATED && step >= each, own = second ? step - each : step;
        return Step{(second ? pa[1] : pa[0]) + own * a_ahead, MODE == GATED ? nullptr : (second ? pb[1] : pb[0]) + own * b_ahead, second, own * b_ahead,
                    s < asked.steps ? a.k - own * KS : 0};
    };
    auto copy = [&](const Step &v, auto i_, int stage) {
        constexpr int i = decltype(i_)::value, j = i - A::COPIES;
        if constexpr (i < A::COPIES) mcu::copy16_to_lds(v.a, oa.from[i], base + stage * STAGE + (w * A::COPIES + i) * 1024);
        else mcu::copy16_to_lds(MODE == GATED ? gated[j] + v.b_at : v.b, ob.from[j], base + stage * STAGE + BM * STEP + (w * B::COPIES + j) * 1024);
    };
    auto request = [&](const Step &v, int stage) {
        if (v.left >= KS) return mcu::static_for<COPIES>([&](auto i) { copy(v, i, stage); });
        // what lies beyond k is zeros of both operands
        const unsigned to = base + stage * STAGE;
#pragma unroll
        for (int i = 0; i < A::COPIES; ++i)
            mcu::copy16_to_lds(A::begins(w * A::COPIES + i, lane) < v.left ? (const void *)(v.a + here(oa.from[i])) : zeros, to + (w * A::COPIES + i) * 1024);
#pragma unroll
        for (int i = 0; i < B::COPIES; ++i)
            mcu::copy16_to_lds(B::begins(w * B::COPIES + i, lane) < v.left ? (const void *)((MODE == GATED ? gated[i] + v.b_at : v.b) + here(ob.from[i])) : zeros,
                               to + BM * STEP + (w * B::COPIES + i) * 1024);
    };

    v4f acc[NF][MF];
    auto clear = [&] {
#pragma unroll
        for (int n = 0; n < NF; ++n)
#pragma unroll
            for (int m = 0; m < MF; ++m) acc[n][m] = (v4f){0, 0, 0, 0};
    };
    // What becomes of a tile
    auto finish = [&](const Work &v) {
        if constexpr (MODE == GATED) {
            constexpr int RUN = EIGHT ? 8 : 4, FS = RUN / 4;
            with_activation(a.activation, [&](auto kind) {
#pragma unroll
                for (int m = 0; m < MF; ++m) {
                    const int row = v.m0 + wm * RM + m * 16 + (lane & 15);
                    if (row >= a.m) continue;
#pragma unroll
                    for (int n = 0; n < NF / 2; n += FS) {
                        const int column = v.n0 + wn * (RN / 2) + n * 16 + RUN * (lane >> 4), count = a.n - column;
                        if (count <= 0) continue;
                        float h[RUN], g[RUN], u[RUN];
#pragma unroll
                        for (int e = 0; e < RUN; ++e) {
                            g[e] = acc[n + e / 4][m][e % 4];
                            u[e] = acc[NF / 2 + n + e / 4][m][e % 4];
                            h[e] = activated<decltype(kind)::value, TYPE>(g[e]) * u[e];
                        }
                        store_run(static_cast<T *>(a.h) + row * a.h_stride + column, h, count);
                        if (a.g) {
                            store_run(a.g + row * a.saved_stride + column, g, count);
                            store_run(a.u + row * a.saved_stride + column, u, count);
                        }
                    }
                }
            });
        } else {
#pragma unroll
            for (int m = 0; m < MF; ++m) {
                const int row = v.m0 + wm * RM + m * 16 + (lane & 15);
                if (row >= a.m) continue;
#pragma unroll
                for (int n = 0; n < NF; ++n) {
                    const int column = v.n0 + wn * RN + n * 16 + 4 * (lane >> 4), count = a.n - column;
                    if (count <= 0) continue;
                    const float c[4] = {acc[n][m][0], acc[n][m][1], acc[n][m][2], acc[n][m][3]};
                    if constexpr (MODE == PARTIAL) store_run(a.partial + ((int64_t)(v.split * a.batch + v.z) * a.m + row) * a.n + column, c, count);
                    else store_run(static_cast<T *>(v.z ? a.c[1] : a.c[0]) + row * (v.z ? a.c_stride[1] : a.c_stride[0]) + column, c, count);
                }
            }
        }
    };

    int u = xcd * per + (int)(blockIdx.x >> 3);
    if (u >= end) return;
    if constexpr (STEP == 64) {
        // The steps of all of a workgroup's tiles are one sequence; copies are asked for NS - 1 steps ahead, those of the next tile before this one's results
        // are written.
        int ask = u, s_asked = 0;      // what is asked for next
        ask_of(ask);
        unsigned came = 0, requested = 0, now = 0; // steps whose own copies have come for certain, that were asked for, and that were multiplied
        constexpr int WHOLE = AR ? 2 : 1;          // a tile's steps are a multiple of this (filled up with zeros)
        auto advance = [&] {
            ++requested;
            if (++s_asked < (asked.steps + WHOLE - 1) / WHOLE * WHOLE) return;
            s_asked = 0;
            ask += turns;
            if (ask < end) ask_of(ask);
        };
        const bool any = asked.steps > 0;
#pragma unroll
        for (int i = 0; i < NS - 1; ++i)
            if (any && ask < end) {
                request(step_of(s_asked), i);
                advance();
            }
        if (requested == NS - 1) mcu::vm_wait<(NS - 2) * COPIES>();
        else mcu::vm_wait<0>();
        asm volatile("s_barrier" ::: "memory");
        if constexpr (AR) {
            // Fragments that are put together from two reads each take too long for a turn of reading: a step's are read while the step before it
            // is multiplied, each of B's as soon as the last product with the one before it is under way, and copies take turns with both.  At a step's
            // barrier the next step has come, and all waves have used the step before.
            constexpr int ALL = NF * MF, APART = ALL / COPIES, AT_ONCE = (MF + NF - 1) / NF; // fragments of A to a row of products
            static_assert(APART * COPIES <= ALL && APART > 1 && MF > 2 * AT_ONCE, "a place for each");
            v4i fa[2][MF], fb[NF];
#pragma unroll
            for (int n = 0; n < NF; ++n) fb[n] = ob.read(lds[0] + BM * STEP, n, 0, lane);
#pragma unroll
            for (int m = 0; m < MF; ++m) fa[0][m] = oa.read(lds[0], m, 0, lane);
            auto turn = [&](auto odd_) {
                constexpr int odd = decltype(odd_)::value;
                if (now + 1 >= came) { // (the step after this one has come: that many copies were asked for behind it)
                    if (requested >= now + NS - 1) mcu::vm_wait<(NS - 3) * COPIES>();
                    else mcu::vm_wait<0>();
                }
                asm volatile("s_barrier" ::: "memory");
                const bool more = any && ask < end;
                const Step v = step_of(s_asked);
                const bool full = more && v.left >= KS;
                const int to = (now + NS - 1) % NS;
                if (more && !full) request(v, to);
                const char *const la = lds[(now + 1) % NS], *const lb = lds[(now + 1) % NS] + BM * STEP; // (behind the last step: read, and not used)
                mcu::static_for<ALL>([&](auto j_) {
                    constexpr int j = decltype(j_)::value, n = j / MF, m = j % MF;
                    acc[n][m] = multiply_one<TYPE>(fb[n], fa[odd][m], acc[n][m]);
                    if constexpr (m % 2 == 1 && m / 2 < AT_ONCE && n * AT_ONCE + m / 2 < MF) fa[odd ^ 1][n * AT_ONCE + m / 2] = oa.read(la, n * AT_ONCE + m / 2, 0, lane);
                    if constexpr (m == MF - 1) fb[n] = ob.read(lb, n, 0, lane);
                    if constexpr (j % APART == APART / 2 && j / APART < COPIES) {
                        if (full) copy(v, std::integral_constant<int, j / APART>{}, to);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
                if (more) advance();
                ++now;
            };
            for (; u < end; u += turns) {
                const Work mine = work(u);
                clear();
                for (int s = 0; s < mine.steps; s += 2) {
                    turn(std::integral_constant<int, 0>{});
                    turn(std::integral_constant<int, 1>{});
                }
                mcu::vm_wait<0>(); // (so that no step of the next tile waits for the stores)
                came = requested;
                finish(mine);
            }
        } else {
            // The waves are two groups, one wave of each to a SIMD, half a step apart: while one group multiplies, the other reads its next fragments and
            // asks for copies.  Two barriers to a step hand the matrix units over.  Before a group leaves its turn of reading, its copies of the step
            // behind have come; a stage is written again when both groups have read it.
            static_assert(W == 8, "two waves to a SIMD");
            const bool late = w >= 4;
            if (late) asm volatile("s_barrier" ::: "memory");
            for (; u < end; u += turns) {
                const Work mine = work(u);
                clear();
                for (int s = 0; s < mine.steps; ++s, ++now) {
                    v4i fa[MF], fb[NF];
                    const char *const la = lds[now % NS], *const lb = lds[now % NS] + BM * STEP;
#pragma unroll
                    for (int n = 0; n < NF; ++n) fb[n] = ob.read(lb, n, 0, lane);
#pragma unroll
                    for (int m = 0; m < MF; ++m) fa[m] = oa.read(la, m, 0, lane);
                    if (any && ask < end) {
                        request(step_of(s_asked), (now + NS - 1) % NS);
                        advance();
                    }
                    if (now + 1 >= came) { // (that many copies were asked for behind the next step's)
                        if (requested >= now + NS) mcu::vm_wait<(NS - 2) * COPIES>();
                        else mcu::vm_wait<0>();
                    }
                    mcu::lgkm_wait();
                    __builtin_amdgcn_sched_barrier(0);
                    asm volatile("s_barrier" ::: "memory");
                    __builtin_amdgcn_sched_barrier(0);
                    multiply<TYPE>(fb, fa, acc);
                    __builtin_amdgcn_sched_barrier(0);
                    asm volatile("s_barrier" ::: "memory");
                    __builtin_amdgcn_sched_barrier(0);
                }
                mcu::vm_wait<0>(); // (so that no step of the next tile waits for the stores)
                came = requested;
                finish(mine);
            }
            if (!late) asm volatile("s_barrier" ::: "memory");
        }
    } else {
        // (a tile to a workgroup: with a loop over tiles the arguments of all that follows were held in scalar registers, more than there are)
        ask_of(u);
        clear();
        const int steps = asked.steps;
#pragma unroll
        for (int s = 0; s < NS - 1; ++s)
            if (s < steps) request(step_of(s), s);
        for (int s = 0; s < steps; ++s) {
            if (s + NS - 1 <= steps) mcu::vm_wait<(NS - 2) * COPIES>(); // (step s has come: that many copies were asked for behind it)
            else mcu::vm_wait<0>();
            asm volatile("s_barrier" ::: "memory"); // for all waves, whose reads of the stage that is written next have returned, too
            if (s + NS - 1 < steps) request(step_of(s + NS - 1), (s + NS - 1) % NS);
            const char *const la = lds[s % NS], *const lb = lds[s % NS] + BM * STEP;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4i fa[MF], fb[NF];
#pragma unroll
                for (int m = 0; m < MF; ++m) fa[m] = oa.read(la, m, h, lane);
#pragma unroll
                for (int n = 0; n < NF; ++n) fb[n] = ob.read(lb, n, h, lane);
                multiply<TYPE>(fb, fa, acc);
            }
            mcu::lgkm_wait();
        }
        finish(asked);
    }
}

// The pieces' sums, four columns to a thread, in the order of the pieces.
template <int TYPE> __global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    const int quads = (a.n + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)a.m * quads;
    if (id >= all * a.batch) return;
    const int z = id >= all;
    const int64_t row = (id - z * all) / quads;
    const int column = (int)(id - z * all - row * quads) * 4, count = a.n - column;
    const float *from = a.partial + ((int64_t)z * a.m + row) * a.n + column;
    float v[4] = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const float *p = from + (int64_t)s * a.batch * a.m * a.n;
        float w[4];
        if (count >= 4) {
            __builtin_memcpy(w, p, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = e < count ? p[e] : 0;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    store_run(static_cast<T *>(z ? a.c[1] : a.c[0]) + row * (z ? a.c_stride[1] : a.c_stride[0]) + column, v, count);
}

// ---- a few rows --------------------------------------------------------------------------------------------------------------
// `count` elements (up to a piece of 16 bytes), zeros behind them, at any alignment
template <class T> __device__ __forceinline__ v4i load_piece(const T *p, int count)
{
    constexpr int PER = 16 / sizeof(T);
    v4i v = {0, 0, 0, 0};
    if (count >= PER) {
        __builtin_memcpy(&v, p, 16);
    } else {
        T e[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) e[i] = i < count ? p[i] : (T)0;
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

constexpr int FEW_WAVES = 4;
// MT tiles of 16 rows of x against 16 rows of either weight, whose pieces go straight into registers: the weights' bytes bound it (1 row of 4096 to 11008 bf16, 180 MB: 31 us, 5.8 TB/s;
// whole calls of fp32, 361 MB: 1 row 73 us, 16 rows 87, 48 rows 116).  The
// waves take turns along k, and their sums meet in LDS.
template <int TYPE, int MT> __global__ __launch_bounds__(64 * FEW_WAVES) void few_rows_kernel(FewRowsArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int PER = 16 / sizeof(T), TAKE = 4 * PER, UNROLL = 4;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, q = lane >> 4, n0 = blockIdx.x * 16;
    const int64_t n = min(n0 + r, a.hidden - 1);
    const T *const pg = static_cast<const T *>(a.gate) + n * a.gate_stride, *const pu = static_cast<const T *>(a.up) + n * a.up_stride;
    const T *px[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) px[m] = static_cast<const T *>(a.x) + (int64_t)min(m * 16 + r, a.rows - 1) * a.x_stride;
    v4f acc[2][MT]; // of gate and up
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[0][m] = acc[1][m] = (v4f){0, 0, 0, 0};
    int k = w * TAKE * UNROLL;
    for (; k + TAKE * UNROLL <= a.dim; k += FEW_WAVES * TAKE * UNROLL) {
        v4i fw[UNROLL][2];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            __builtin_memcpy(&fw[i][0], pg + k + i * TAKE + q * PER, 16);
            __builtin_memcpy(&fw[i][1], pu + k + i * TAKE + q * PER, 16);
        }
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            v4i fx[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) __builtin_memcpy(&fx[m], px[m] + k + i * TAKE + q * PER, 16);
            multiply<TYPE>(fw[i], fx, acc);
        }
    }
    for (int i = 0; i < UNROLL && k + i * TAKE < a.dim; ++i) { // what is left, fewer than UNROLL
        const int at = k + i * TAKE + q * PER, count = a.dim - at;
        const v4i fw[2] = {load_piece(pg + at, count), load_piece(pu + at, count)};
        v4i fx[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) fx[m] = load_piece(px[m] + at, count);
        multiply<TYPE>(fw, fx, acc);
    }
    __shared__ v4f sums[FEW_WAVES][2][MT][64];
#pragma unroll
    for (int m = 0; m < MT; ++m) sums[w][0][m][lane] = acc[0][m], sums[w][1][m][lane] = acc[1][m];
    __syncthreads();
    for (int m = w; m < MT; m += FEW_WAVES) {
        v4f sg = sums[0][0][m][lane], su = sums[0][1][m][lane];
#pragma unroll
        for (int i = 1; i < FEW_WAVES; ++i) sg += sums[i][0][m][lane], su += sums[i][1][m][lane];
        const int row = m * 16 + r, column = n0 + 4 * q, count = a.hidden - column;
        if (row >= a.rows || count <= 0) continue;
        float h[4], gs[4], us[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) gs[e] = sg[e], us[e] = su[e];
        with_activation(a.activation, [&](auto kind) {
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activated<decltype(kind)::value, TYPE>(gs[e]) * us[e];
        });
        store_run(static_cast<T *>(a.h) + row * a.h_stride + column, h, count);
        if (a.g) {
            store_run(a.g + row * a.saved_stride + column, gs, count);
            store_run(a.u + row * a.saved_stride + column, us, count);
        }
    }
}

// ---- the gradient's operands ---------------------------------------------------------------------------------------------------
// dg and du, rounded to the type that the products take: once each, half a step, whose signs the products' sums even out.  (Memory bounds it: 8192 x 11008 bf16, 1.26 GB, 250 us, the rate of a copy.)  Eight elements to a thread; columns from
// hidden to padded_hidden are zeros.
template <int TYPE> __global__ __launch_bounds__(256) void gated_grad_kernel(GatedGradArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    const int octs = (a.padded_hidden + 7) / 8;
    const int64_t all = a.rows * octs;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
        const int64_t row = id / octs;
        const int column = (int)(id - row * octs) * 8, count = a.hidden - column;
        const T *dh = static_cast<const T *>(a.dh) + row * a.dh_stride + column;
        const float *g = a.g + row * a.saved_stride + column, *u = a.u + row * a.saved_stride + column;
        T d[8];
        float gs[8], us[8], dg[8], du[8];
        if (count >= 8) {
            __builtin_memcpy(d, dh, sizeof d);
            __builtin_memcpy(gs, g, 32);
            __builtin_memcpy(us, u, 32);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[e] = e < count ? dh[e] : (T)0;
                gs[e] = e < count ? g[e] : 0;
                us[e] = e < count ? u[e] : 0;
            }
        }
        with_activation(a.activation, [&](auto kind) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float slope;
                const float act = activated<decltype(kind)::value, TYPE>(gs[e], slope);
                du[e] = (float)d[e] * act;
                dg[e] = (float)d[e] * us[e] * slope;
            }
        });
        store_run(static_cast<T *>(a.dg) + row * a.padded_hidden + column, dg, a.padded_hidden - column);
        store_run(static_cast<T *>(a.du) + row * a.padded_hidden + column, du, a.padded_hidden - column);
    }
}

// Matrices whose rows are no whole pieces of 16 bytes, copied into such that are: a piece to a thread.
template <class T> __global__ __launch_bounds__(256) void pad_rows_kernel(PadRowsArgs a)
{
    constexpr int PER = 16 / sizeof(T);
    const PadRowsArgs::Matrix &m = a.matrix[blockIdx.y];
    const unsigned pieces = a.padded / PER, stride = gridDim.x * 256;
    const int64_t all = m.rows * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += stride) {
        const int64_t row = all < 0xffffffffll ? (int64_t)((unsigned)i / pieces) : i / pieces;
        const int column = (int)(i - row * pieces) * PER;
        const v4i v = load_piece(static_cast<const T *>(m.from) + row * m.stride + column, a.width - column);
        __builtin_memcpy(static_cast<T *>(m.to) + row * a.padded + column, &v, 16);
    }
}

// ---- launches --------------------------------------------------------------------------------------------------------------------
template <int TYPE, int BM, int BN, int WM, int WN, int STEP, int NS, bool AR, bool BR, int MODE> hipError_t product(ProductArgs a, hipStream_t s)
{
    constexpr int COLUMNS = MODE == GATED ? BN / 2 : BN;
    a.tiles_m = (a.m + BM - 1) / BM;
    a.tiles_n = (a.n + COLUMNS - 1) / COLUMNS;
    const int64_t all = ((int64_t)a.tiles_m * a.tiles_n * (MODE == GATED ? 1 : a.batch) * (MODE == PARTIAL ? a.splits : 1) + 7) / 8 * 8;
    const dim3 grid((unsigned)(STEP == 64 && all > COMPUTE_UNITS ? COMPUTE_UNITS : all)); // (the large tiles: a workgroup to a compute unit)
    return launch_kernel((product_kernel<TYPE, BM, BN, WM, WN, STEP, NS, AR, BR, MODE>), grid, dim3(64 * WM * WN), 0, s, a);
}

template <int TYPE, bool AR, bool BR, int MODE> hipError_t product_tile(const ProductArgs &a, int tile, hipStream_t s)
{
    switch (tile) {
    case 256: return product<TYPE, 256, 256, 2, 4, TYPE == MC_F32 ? 128 : 64, TYPE == MC_F32 ? 2 : 4, AR, BR, MODE>(a, s);
    case 128: return product<TYPE, 128, 128, 2, 2, 128, 2, AR, BR, MODE>(a, s);
    case 96: return product<TYPE, 128, 64, 2, 2, 128, 3, AR, BR, MODE>(a, s);
    case 64: return product<TYPE, 64, 64, 2, 2, 128, 3, AR, BR, MODE>(a, s);
    default: return product<TYPE, 32, 64, 2, 2, 128, 3, AR, BR, MODE>(a, s);
    }
}

template <int TYPE, bool AR> hipError_t product_plain(ProductArgs a, ProductPlan p, hipStream_t s)
{
    a.splits = p.splits;
    if (p.splits == 1) return product_tile<TYPE, AR, true, PLAIN>(a, p.tile, s);
    const hipError_t e = product_tile<TYPE, AR, true, PARTIAL>(a, p.tile, s);
    if (e != hipSuccess) return e;
    const int64_t threads = (int64_t)a.batch * a.m * ((a.n + 3) / 4);
    return launch_kernel(product_join_kernel<TYPE>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a);
}

template <int TYPE, int MT> hipError_t few_rows(const FewRowsArgs &a, hipStream_t s)
{
    return launch_kernel((few_rows_kernel<TYPE, MT>), dim3((unsigned)((a.hidden + 15) / 16)), dim3(64 * FEW_WAVES), 0, s, a);
}
template <int TYPE> hipError_t few_rows_of(const FewRowsArgs &a, hipStream_t s)
{
    if (a.rows <= 16) return few_rows<TYPE, 1>(a, s);
    if (a.rows <= 32) return few_rows<TYPE, 2>(a, s);
    return few_rows<TYPE, 4>(a, s);
}

} // namespace

hipError_t launch_gated_product(const ProductArgs &a, mc_type type, hipStream_t s)
{
    const int tile = product_plan(a.m, a.n, a.k, 1, type, true).tile;
    return type == MC_F32 ? product_tile<MC_F32, false, false, GATED>(a, tile, s)
         : type == MC_F16 ? product_tile<MC_F16, false, false, GATED>(a, tile, s) : product_tile<MC_BF16, false, false, GATED>(a, tile, s);
}
hipError_t launch_product(const ProductArgs &a, ProductPlan p, bool a_rows, mc_type type, hipStream_t s)
{
    if (a_rows) return type == MC_F32 ? product_plain<MC_F32, true>(a, p, s) : type == MC_F16 ? product_plain<MC_F16, true>(a, p, s) : product_plain<MC_BF16, true>(a, p, s);
    return type == MC_F32 ? product_plain<MC_F32, false>(a, p, s) : type == MC_F16 ? product_plain<MC_F16, false>(a, p, s) : product_plain<MC_BF16, false>(a, p, s);
}
hipError_t launch_few_rows(const FewRowsArgs &a, mc_type type, hipStream_t s)
{
    return type == MC_F32 ? few_rows_of<MC_F32>(a, s) : type == MC_F16 ? few_rows_of<MC_F16>(a, s) : few_rows_of<MC_BF16>(a, s);
}
hipError_t launch_gated_grad(const GatedGradArgs &a, mc_type type, hipStream_t s)
{
    const int64_t blocks = (a.rows * ((a.padded_hidden + 7) / 8) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384)), block(256);
    return type == MC_F32 ? launch_kernel(gated_grad_kernel<MC_F32>, grid, block, 0, s, a)
         : type == MC_F16 ? launch_kernel(gated_grad_kernel<MC_F16>, grid, block, 0, s, a) : launch_kernel(gated_grad_kernel<MC_BF16>, grid, block, 0, s, a);
}
hipError_t launch_pad_rows(const PadRowsArgs &a, mc_type type, hipStream_t s)
{
    int64_t most = 0;
    for (int i = 0; i < a.count; ++i) most = a.matrix[i].rows > most ? a.matrix[i].rows : most;
    const int64_t blocks = (most * (a.padded / (type == MC_F32 ? 4 : 8)) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096), a.count), block(256);
    return type == MC_F32 ? launch_kernel(pad_rows_kernel<uint32_t>, grid, block, 0, s, a) : launch_kernel(pad_rows_kernel<uint16_t>, grid, block, 0, s, a);
}
