// The norms after a block and before the next one, with the block's gate and the residual connection, in one pass:
//   a = post(x),   y = residual_scale r + branch_scale gate a,   n = pre(y),
// a norm being v / sqrt(mean v^2 + eps) weight, or (v - mean v) / sqrt(var v + eps) weight + bias.  Rows are held in registers (eight
// neighbouring elements of a thread to a chunk): a variance is taken around the mean, n from the unrounded y.
// Backward, with hat for normed values, W for an operand times its weight, and r for 1 / deviation:
//   dyt = dy + r2 (W(dn) - mean W(dn) - yhat mean(W(dn) yhat)),   dr = residual_scale dyt,   da = branch_scale gate dyt,
//   dx = r1 (W(da) - mean W(da) - xhat mean(W(da) xhat))          (without the first mean where the norm has none)
// and the parameters' gradients are sums over rows of dn yhat, dn, da xhat, da and branch_scale a dyt.  Nothing is kept from the forward call: y is
// worked out again from x and r, unrounded, for the bytes that reading it would cost.  A workgroup takes consecutive rows, asks for a
// row while it works on the one before, and keeps these sums in registers; a second kernel adds the workgroups' in their order, so that results are the
// same from call to call.
// Memory bounds both: 16384 x 8192 bf16 beside a stream in fp32 284 us, 5.7 TB/s; 16384 x 4096 bf16 104 us, its gradients 180.
#include "layer.h"

#include "lds_async.h"

namespace {

using mcu::v4i;

// Eight elements as they lie in memory
template <int TYPE> struct Raw { v4i v[TYPE == MC_F32 ? 2 : 1]; };

// Element `at` behind element `row`, which is the same in all threads.  SHORT: a thread's share of the address is 32 bits, which takes fewer registers and decides how many rows run at
// once beside a 16-bit stream, and orders the loads worse where it decides nothing (gradients of layer norms, 400 MB of bf16 or 800 of fp32, us with and without: 32552 x 1024 bf16 115, 135, beside
// fp32 191, 161, fp32 233, 205; 16276 x 2048 bf16 108, 128; 2034 x 16384 bf16 359, 388)
template <class T, bool SHORT, class V> __device__ __forceinline__ T *address(V *p, int64_t row, int at)
{
    if constexpr (SHORT) return reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(static_cast<T *>(p) + row) + (uintptr_t)((unsigned)at * (unsigned)sizeof(T)));
    else return static_cast<T *>(p) + (row + at);
}
// Those from element `at` of a row on, at any alignment; of a row of fewer than eight (`dim`), zeros behind them
template <int TYPE, bool SHORT = false> __device__ __forceinline__ Raw<TYPE> load(const void *p, int64_t row, int at, int dim)
{
    typedef typename RealOf<TYPE>::type T;
    const T *from = address<const T, SHORT>(p, row, at);
    Raw<TYPE> r;
    if (dim >= 8) {
        __builtin_memcpy(&r, from, sizeof r);
    } else {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < dim ? from[i] : (T)0;
        __builtin_memcpy(&r, e, sizeof r);
    }
    return r;
}
template <int TYPE> __device__ __forceinline__ void decode(const Raw<TYPE> &r, float (&v)[8])
{
    typename RealOf<TYPE>::type e[8];
    __builtin_memcpy(e, &r, sizeof r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)e[i];
}
// Elements lo .. n - 1
template <int TYPE, bool SHORT = false> __device__ __forceinline__ void store(void *p, int64_t row, int at, int lo, int n, const float (&v)[8])
{
    typedef typename RealOf<TYPE>::type T;
    T *to = address<T, SHORT>(p, row, at), e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = (T)v[i];
    if (lo <= 0 && n >= 8) {
        __builtin_memcpy(to, e, sizeof e);
    } else if (lo < n) {
        asm volatile("" ::: "memory"); // (the compiler would else make some elements' stores those of both cases, and write whole chunks in parts)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= lo && i < n) to[i] = e[i];
        asm volatile("" ::: "memory");
    }
}

// A wave's sum, in all of its lanes: exchanges within 16 lanes, then of the 16s and of the halves.
template <int CONTROL> __device__ __forceinline__ float exchanged(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CONTROL, 0xf, 0xf, true)); }
__device__ __forceinline__ float wave_sum(float x)
{
    x += exchanged<0xb1>(x);  // lanes 1 apart
    x += exchanged<0x4e>(x);  // 2 apart
    x += exchanged<0x141>(x); // mirrored in eights
    x += exchanged<0x140>(x); // and in 16s
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A row over THREADS threads, E chunks of eight elements each: chunk k of thread t begins at element 8 (t + k THREADS).  A last chunk that would reach
// beyond the row is the row's last eight elements, of which the chunk's own follow those of the one before; chunks that begin beyond it have none.  So
// every load is a whole one, without a branch that would wait for it (the gradient of 16384 x 4096 bf16 225 -> 180 us, of 4016 x 1153 fp32, with two sums' barriers less, 55 -> 44).
// Elements that are not the chunk's own are taken for zeros.
template <int THREADS, int E, bool SHORT = false> struct Row {
    static constexpr int WAVES = THREADS / 64;
    int t, dim;
    float inverse;    // 1 / dim
    float *shared;    // 2 x WAVES x 4 floats
    int turn;         // which half of them the next sum uses (one barrier to a sum)

    __device__ __forceinline__ int at(int k) const { return 8 * (t + k * THREADS); }
    __device__ __forceinline__ int place(int k) const { return max(min(at(k), dim - 8), 0); }
    __device__ __forceinline__ int elements() const { return min(dim, 8); }
    __device__ __forceinline__ int first(int k) const { return at(k) - place(k); } // of the chunk's own
    __device__ __forceinline__ bool own(int k, int e) const { return e >= first(k) && (e == 0 || e < dim); }
    __device__ __forceinline__ bool full() const { return E * THREADS * 8 == dim; } // every chunk is whole
    __device__ __forceinline__ void trim(float (&v)[E][8]) const
    {
        if (full()) return;
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = own(k, e) ? v[k][e] : 0;
    }
    template <int N> __device__ __forceinline__ void sums(float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
        if constexpr (WAVES > 1) {
            float *s = shared + turn * 4 * WAVES;
            turn ^= 1;
            if ((t & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) s[4 * (t >> 6) + i] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) { // (a wave's to each lane)
                v[i] = s[4 * (t & (WAVES - 1)) + i];
                v[i] += exchanged<0xb1>(v[i]);
                if constexpr (WAVES > 2) v[i] += exchanged<0x4e>(v[i]);
                if constexpr (WAVES > 4) v[i] += exchanged<0x141>(v[i]);
                if constexpr (WAVES > 8) v[i] += exchanged<0x140>(v[i]);
            }
        }
    }
    // v (zeros beyond the row) becomes its normed values, zeros beyond the row; returns 1 / deviation.
    __device__ __forceinline__ float norm(float (&v)[E][8], int kind, float eps)
    {
        float m;
        return norm(v, kind, eps, m);
    }
    __device__ __forceinline__ float norm(float (&v)[E][8], int kind, float eps, float &m)
    {
        float z[2] = {0, 0}; // of squares, of elements
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) z[0] += v[k][e] * v[k][e], z[1] += v[k][e];
        if (kind == MC_NORM_LAYER) {
            sums(z);
            return centred(v, z[1], z[0], eps, m);
        }
        float q[1] = {z[0]};
        sums(q);
        m = 0;
        const float r = 1.0f / sqrtf(q[0] * inverse + eps);
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] *= r;
        return r;
    }
    // Whether a variance may be taken from the sums of elements and of squares: its error is a rounding times 1 + mean^2 / variance, here at most two.
    __device__ __forceinline__ bool near(float sum, float squares) const
    {
        const float m = sum / dim;
        return __builtin_amdgcn_readfirstlane(m * m <= squares * inverse - m * m);
    }
    // The layer norm, from the sums; around the mean where that is far from 0.
    __device__ __forceinline__ float centred(float (&v)[E][8], float sum, float squares, float eps, float &m)
    {
        m = sum / dim;
        const bool direct = near(sum, squares);
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] -= m;
        trim(v);
        float q[1] = {0};
        if (!direct) {
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) q[0] += v[k][e] * v[k][e];
            sums(q);
        }
        const float r = 1.0f / sqrtf((direct ? squares * inverse - m * m : q[0] * inverse) + eps);
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] *= r;
        return r;
    }
    // Parameters in fp32 (`otherwise` where there are none), zeros beyond the row
    __device__ __forceinline__ void parameters(float (&v)[E][8], const void *p, int type, int64_t from, float otherwise) const
    {
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (!p) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] = otherwise;
            } else if (type == MC_F32) {
                decode(load<MC_F32, SHORT>(p, from, place(k), dim), v[k]);
            } else if (type == MC_F16) {
                decode(load<MC_F16, SHORT>(p, from, place(k), dim), v[k]);
            } else {
                decode(load<MC_BF16, SHORT>(p, from, place(k), dim), v[k]);
            }
        }
        trim(v);
    }
    template <int TYPE> __device__ __forceinline__ void write(void *p, int64_t from, const float (&v)[E][8]) const
    {
#pragma unroll
        for (int k = 0; k < E; ++k) store<TYPE, SHORT>(p, from, place(k), first(k), elements(), v[k]);
    }
    __device__ __forceinline__ void write_parameters(void *p, int type, int64_t from, const float (&v)[E][8]) const
    {
        if (type == MC_F32) write<MC_F32>(p, from, v);
        else if (type == MC_F16) write<MC_F16>(p, from, v);
        else write<MC_BF16>(p, from, v);
    }
};

#define EACH(k, e)                 \
    _Pragma("unroll")              \
    for (int k = 0; k < E; ++k)    \
        _Pragma("unroll") for (int e = 0; e < 8; ++e)

// Parameters as they lie in memory, of a type that is known when the kernel runs
struct RawParameters { v4i lo, hi; };
__device__ __forceinline__ RawParameters load_parameters(const void *p, int type, int64_t row, int at, int dim)
{
    if (type == MC_F32) {
        const Raw<MC_F32> r = load<MC_F32>(p, row, at, dim);
        return {r.v[0], r.v[1]};
    }
    const Raw<MC_F16> r = load<MC_F16>(p, row, at, dim); // (or bf16: bits, and zeros)
    return {r.v[0], r.v[0]};
}
__device__ __forceinline__ void decode_parameters(const RawParameters &r, int type, float (&v)[8])
{
    if (type == MC_F32) decode(Raw<MC_F32>{{r.lo, r.hi}}, v);
    else if (type == MC_F16) decode(Raw<MC_F16>{{r.lo}}, v);
    else decode(Raw<MC_BF16>{{r.lo}}, v);
}

// PACKED: rows of a workgroup, a wave each.  WHOLE: rows are whole chunks.  All operands are asked for before the first is used.  (Without these two, 16384 rows of
// 4096 bf16 took 141 us instead of 101.)
template <int TYPE, int RTYPE, int THREADS, int E, int PACKED, bool WHOLE> __global__ __launch_bounds__(THREADS *PACKED) void block_norm_kernel(NormArgs a)
{
    __shared__ float shared[8 * THREADS / 64];
    const int64_t row = a.first + (int64_t)blockIdx.x * PACKED + (PACKED > 1 ? threadIdx.x / THREADS : 0);
    if (row >= a.rows) return;
    Row<THREADS, E> of = {(int)(PACKED > 1 ? threadIdx.x % THREADS : threadIdx.x), a.dim, 1.0f / a.dim, shared, 0};
    const int loaded = WHOLE ? 8 : a.dim;
    Raw<TYPE> x[E];
    Raw<RTYPE> r[E];
    RawParameters pw[E], g[E], w[E];
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = load<TYPE>(a.x, row * a.x_stride, of.place(k), loaded);
    if (a.r)
#pragma unroll
        for (int k = 0; k < E; ++k) r[k] = load<RTYPE>(a.r, row * a.r_stride, of.place(k), loaded);
    auto ask = [&](RawParameters (&to)[E], const void *p, int64_t from) {
        if (!p) return;
        if (a.p_type == MC_F32) {
#pragma unroll
            for (int k = 0; k < E; ++k) to[k] = load_parameters(p, MC_F32, from, of.place(k), loaded);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) to[k] = load_parameters(p, MC_F16, from, of.place(k), loaded);
        }
    };
    ask(pw, a.post_weight, 0);
    ask(g, a.gate, row / a.gate_rows * a.gate_stride);
    ask(w, a.weight, 0);
    float v[E][8], f[8];
    auto times = [&](const RawParameters (&p)[E], const void *there, const void *bias) {
        if (there)
#pragma unroll
            for (int k = 0; k < E; ++k) {
                decode_parameters(p[k], a.p_type, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] *= f[e];
            }
        if (bias) {
            RawParameters b[E];
            ask(b, bias, 0);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                decode_parameters(b[k], a.p_type, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] += f[e];
            }
        }
    };
#pragma unroll
    for (int k = 0; k < E; ++k) decode(x[k], v[k]);
    of.trim(v);
    if (a.post) {
        of.norm(v, a.post, a.eps);
        times(pw, a.post_weight, a.post_bias);
    }
    times(g, a.gate, nullptr);
#pragma unroll
    for (int k = 0; k < E; ++k) {
        if (a.r) decode(r[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = a.branch_scale * v[k][e] + (a.r ? a.residual_scale * f[e] : 0);
    }
    of.trim(v);
    if (a.y) of.template write<RTYPE>(a.y, row * a.y_stride, v);
    if (!a.pre) return;
    of.norm(v, a.pre, a.eps);
    times(w, a.weight, a.bias);
    of.template write<TYPE>(a.n, row * a.n_stride, v);
}

// LAYER: one of the norms takes means, or there are biases.  With one chunk to a thread parameters stay in registers and the next row is asked for ahead; with two
// parameters are read again for each row (from the caches), where they are used.  SUMS false: the sums over rows, which would not fit into the registers of so wide a row, are left to
// the kernel below, for which a row's means and deviations are written out.
template <int TYPE, int RTYPE, int THREADS, int E, bool LAYER, bool SUMS> __global__ __launch_bounds__(THREADS, THREADS == 1024 ? 4 : THREADS == 512 || (LAYER && RTYPE == MC_F32) ? 2 : 3) void block_norm_backward_kernel(NormArgs a)
{
    __shared__ float shared[8 * THREADS / 64];
    constexpr bool SHORT = RTYPE != MC_F32;
    Row<THREADS, E, SHORT> of = {(int)threadIdx.x, a.dim, 1.0f / a.dim, shared, 0};
    const int64_t first = blockIdx.x * a.per, end = min(first + a.per, a.rows);
    float w[E][8], pw[E][8], pb[LAYER ? E : 1][8], g[E][8]; // (g: times the branch's scale)
    constexpr bool HELD = E == 1, AHEAD = E == 1;
    auto read_here = [] { if constexpr (!HELD) asm volatile("" ::: "memory"); }; // (parameters that are read again are not asked for ahead, into registers that are not there)
    auto post_parameters = [&] {
        of.parameters(pw, a.post_weight, a.p_type, 0, 1);
        if constexpr (LAYER) of.parameters(pb, a.post_bias, a.p_type, 0, 0);
    };
    if constexpr (HELD) {
        of.parameters(w, a.weight, a.p_type, 0, 1);
        post_parameters();
    }
    if (!a.gate) EACH(k, e) g[k][e] = a.branch_scale;
    float sum_g[E][8] = {}, sum_w[E][8] = {}, sum_pw[E][8] = {}, sum_b[LAYER ? E : 1][8] = {}, sum_pb[LAYER ? E : 1][8] = {};
    float *const mine = a.partial + (int64_t)blockIdx.x * 6 * a.dim;
    Raw<TYPE> rx[E], rdn[E] = {};
    Raw<RTYPE> rr[E] = {}, rdy[E] = {};
    auto ask = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
            rx[k] = load<TYPE, SHORT>(a.x, row * a.x_stride, of.place(k), a.dim);
            if (a.r) rr[k] = load<RTYPE, SHORT>(a.r, row * a.r_stride, of.place(k), a.dim);
            if (a.dn) rdn[k] = load<TYPE, SHORT>(a.dn, row * a.dn_stride, of.place(k), a.dim);
            if (a.dy) rdy[k] = load<RTYPE, SHORT>(a.dy, row * a.dy_stride, of.place(k), a.dim);
        }
    };
    if constexpr (AHEAD) ask(first);
    int64_t group = first / a.gate_rows, group_end = (group + 1) * a.gate_rows; // the row's gate, and where its rows end
    bool fresh = true;
    for (int64_t row = first; row < end; ++row) {
        float hat1[E][8], hat2[E][8], d[E][8], dy[E][8];
        if constexpr (!AHEAD) ask(row);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            decode(rx[k], hat1[k]);
            decode(rr[k], hat2[k]);
            decode(rdn[k], d[k]);
            decode(rdy[k], dy[k]);
        }
        of.trim(hat1);
        of.trim(hat2);
        of.trim(d);
        if constexpr (AHEAD) ask(min(row + 1, end - 1));
        if (HELD && a.gate && fresh) {
            of.parameters(g, a.gate, a.p_type, group * a.gate_stride, 1);
            EACH(k, e) g[k][e] *= a.branch_scale;
        }
        float m1 = 0, m2 = 0, r2 = 0, mean2 = 0, dot2 = 0;
        const float r1 = a.post ? of.norm(hat1, a.post, a.eps, m1) : 1;
        if constexpr (HELD) {
            EACH(k, e) {
                float b = hat1[k][e] * pw[k][e];
                if constexpr (LAYER) b += pb[k][e];
                hat2[k][e] = g[k][e] * b + (a.r ? a.residual_scale * hat2[k][e] : 0); // y
            }
        } else {
            float b[E][8], f[E][8];
            read_here();
            of.parameters(b, a.post_weight, a.p_type, 0, 1);
            EACH(k, e) b[k][e] *= hat1[k][e];
            if constexpr (LAYER) {
                read_here();
                of.parameters(f, a.post_bias, a.p_type, 0, 0);
                EACH(k, e) b[k][e] += f[k][e];
            }
            if (a.gate) {
                read_here();
                of.parameters(f, a.gate, a.p_type, group * a.gate_stride, 1);
                EACH(k, e) b[k][e] *= f[k][e];
            }
            EACH(k, e) hat2[k][e] = a.branch_scale * b[k][e] + (a.r ? a.residual_scale * hat2[k][e] : 0);
            read_here();
        }
        if (a.pre && a.dn) {
            float mean, dot;
            if constexpr (!HELD) of.parameters(w, a.weight, a.p_type, 0, 1);
            if constexpr (!SUMS) EACH(k, e) d[k][e] *= w[k][e];
            auto dw = [&](int k, int e) { return SUMS ? d[k][e] * w[k][e] : d[k][e]; };
            // (all sums at once, of y that is not normed yet)
            if (LAYER) {
                float z[4] = {0, 0, 0, 0};
                EACH(k, e) {
                    z[0] += hat2[k][e], z[1] += hat2[k][e] * hat2[k][e], z[2] += dw(k, e), z[3] += dw(k, e) * hat2[k][e];
                }
                of.sums(z);
                if (a.pre != MC_NORM_LAYER) {
                    r2 = 1.0f / sqrtf(z[1] * of.inverse + a.eps);
                    EACH(k, e) hat2[k][e] *= r2;
                    mean = 0, dot = r2 * z[3] * of.inverse;
                } else {
                    const bool direct = of.near(z[0], z[1]);
                    r2 = of.centred(hat2, z[0], z[1], a.eps, m2);
                    if (!direct) {
                        float far[1] = {0};
                        EACH(k, e) far[0] += dw(k, e) * hat2[k][e];
                        of.sums(far);
                        dot = far[0] * of.inverse;
                    } else {
                        dot = r2 * (z[3] - m2 * z[2]) * of.inverse;
                    }
                    mean = z[2] * of.inverse;
                }
            } else {
                float z[2] = {0, 0};
                EACH(k, e) {
                    z[0] += hat2[k][e] * hat2[k][e];
                    z[1] += dw(k, e) * hat2[k][e];
                }
                of.sums(z);
                r2 = 1.0f / sqrtf(z[0] * of.inverse + a.eps);
                mean = 0, dot = z[1] * r2 * of.inverse;
                EACH(k, e) hat2[k][e] *= r2;
            }
            mean2 = mean, dot2 = dot;
            EACH(k, e) {
                if constexpr (SUMS) sum_w[k][e] += d[k][e] * hat2[k][e];
                if constexpr (SUMS && LAYER) sum_b[k][e] += d[k][e];
                dy[k][e] += r2 * (dw(k, e) - mean - hat2[k][e] * dot);
            }
        }
        if (a.dr) {
            EACH(k, e) d[k][e] = a.residual_scale * dy[k][e];
            of.template write<RTYPE>(a.dr, row * a.dr_stride, d);
        }
        if (!SUMS && threadIdx.x == 0) {
            float *to = a.partial + (int64_t)a.workgroups * 6 * a.dim + 8 * row;
            to[0] = m1, to[1] = r1, to[2] = m2, to[3] = r2, to[4] = mean2, to[5] = dot2;
        }
        float z[2] = {0, 0};
        if constexpr (!HELD) {
            read_here();
            post_parameters();
            if (a.gate) {
                of.parameters(g, a.gate, a.p_type, group * a.gate_stride, 1);
                EACH(k, e) g[k][e] *= a.branch_scale;
            }
        }
        EACH(k, e) {
            const float da = g[k][e] * dy[k][e];
            if constexpr (SUMS) {
                float b = hat1[k][e] * pw[k][e];
                if constexpr (LAYER) b += pb[k][e];
                sum_g[k][e] += a.branch_scale * b * dy[k][e];
                sum_pw[k][e] += da * hat1[k][e];
                if constexpr (LAYER) sum_pb[k][e] += da;
            }
            d[k][e] = da * pw[k][e];
            const float mine = of.own(k, e) ? d[k][e] : 0; // (dy is there beyond the row, too)
            z[0] += mine;
            z[1] += mine * hat1[k][e];
        }
        // a row of the gate ends here, or the workgroup does: written out whole, or left for the second kernel in the place of a gate's row that began before (0) or in (1) these rows
        fresh = row + 1 == group_end;
        if (SUMS && a.grads[0] && (fresh || row + 1 == end)) {
            const int64_t begin = group_end - a.gate_rows;
            if (fresh && begin >= first) of.write_parameters(a.grads[0], a.p_type, group * a.dgate_stride, sum_g);
            else of.template write<MC_F32>(mine, begin < first ? 0 : a.dim, sum_g);
            EACH(k, e) sum_g[k][e] = 0;
        }
        if (fresh) ++group, group_end += a.gate_rows;
        if (!a.dx) continue;
        if (a.post) {
            of.sums(z);
            const float mean = LAYER && a.post == MC_NORM_LAYER ? z[0] * of.inverse : 0, dot = z[1] * of.inverse;
            EACH(k, e) d[k][e] = r1 * (d[k][e] - mean - hat1[k][e] * dot);
        }
        of.template write<TYPE>(a.dx, row * a.dx_stride, d);
    }
    if constexpr (!SUMS) return;
    if (a.grads[1]) of.template write<MC_F32>(mine, 2 * a.dim, sum_w);
    if (a.grads[3]) of.template write<MC_F32>(mine, 4 * a.dim, sum_pw);
    if constexpr (LAYER) {
        if (a.grads[2]) of.template write<MC_F32>(mine, 3 * a.dim, sum_b);
        if (a.grads[4]) of.template write<MC_F32>(mine, 5 * a.dim, sum_pb);
    }
}

// The sums over rows, of COLUMNS_EACH columns (eight to a thread) and one workgroup's rows, where the kernel above does not keep them: the same terms again, from the row's
// means and deviations.
constexpr int COLUMN_THREADS = 256, COLUMNS_EACH = 8 * COLUMN_THREADS;
template <int TYPE, int RTYPE> __global__ __launch_bounds__(COLUMN_THREADS) void block_norm_columns_kernel(NormArgs a)
{
    constexpr int E = 1;
    const int64_t first = blockIdx.y * a.per, end = min(first + a.per, a.rows);
    const int left = a.dim - (int)blockIdx.x * COLUMNS_EACH, shift = blockIdx.x * COLUMNS_EACH; // columns from here on
    Row<COLUMN_THREADS, 1> of = {(int)threadIdx.x, left, 0, nullptr, 0};
    const int at = of.place(0);
    auto from = [&](const void *p) { return p ? static_cast<const char *>(p) + (int64_t)shift * (a.p_type == MC_F32 ? 4 : 2) : nullptr; };
    float w[1][8], pw[1][8], pb[1][8], g[1][8];
    of.parameters(w, from(a.weight), a.p_type, 0, 1);
    of.parameters(pw, from(a.post_weight), a.p_type, 0, 1);
    of.parameters(pb, from(a.post_bias), a.p_type, 0, 0);
    if (!a.gate) EACH(k, e) g[k][e] = a.branch_scale;
    float sum_g[1][8] = {}, sum_w[1][8] = {}, sum_pw[1][8] = {}, sum_b[1][8] = {}, sum_pb[1][8] = {};
    float *const mine = a.partial + (int64_t)blockIdx.y * 6 * a.dim + shift;
    int64_t group = first / a.gate_rows, group_end = (group + 1) * a.gate_rows;
    bool fresh = true;
    const bool through = a.pre && a.dn; // (else the gradient does not see y, which may be infinite)
    for (int64_t row = first; row < end; ++row) {
        const float *of_row = a.partial + (int64_t)a.workgroups * 6 * a.dim + 8 * row;
        const float m1 = of_row[0], r1 = of_row[1], m2 = of_row[2], r2 = of_row[3], mean = of_row[4], dot = of_row[5];
        float x[8], r[8], dn[8], dy[8];
        Raw<TYPE> rx = load<TYPE>(a.x, row * a.x_stride + shift, at, left), rdn = {};
        Raw<RTYPE> rr = {}, rdy = {};
        if (a.r) rr = load<RTYPE>(a.r, row * a.r_stride + shift, at, left);
        if (a.dn) rdn = load<TYPE>(a.dn, row * a.dn_stride + shift, at, left);
        if (a.dy) rdy = load<RTYPE>(a.dy, row * a.dy_stride + shift, at, left);
        if (a.gate && fresh) {
            of.parameters(g, from(a.gate), a.p_type, group * a.gate_stride, 1);
            EACH(k, e) g[k][e] *= a.branch_scale;
        }
        decode(rx, x);
        decode(rr, r);
        decode(rdn, dn);
        decode(rdy, dy);
        EACH(k, e) {
            const float hat1 = (x[e] - m1) * r1, b = hat1 * pw[k][e] + pb[k][e], y = g[k][e] * b + (a.r ? a.residual_scale * r[e] : 0), hat2 = through ? (y - m2) * r2 : 0;
            const float dyt = through ? dy[e] + r2 * (dn[e] * w[k][e] - mean - hat2 * dot) : dy[e], da = g[k][e] * dyt;
            sum_w[k][e] += dn[e] * hat2;
            sum_b[k][e] += dn[e];
            sum_g[k][e] += a.branch_scale * b * dyt;
            sum_pw[k][e] += da * hat1;
            sum_pb[k][e] += da;
        }
        fresh = row + 1 == group_end; // (see the kernel above)
        if (a.grads[0] && (fresh || row + 1 == end)) {
            const int64_t begin = group_end - a.gate_rows;
            if (fresh && begin >= first) of.write_parameters(a.grads[0], a.p_type, group * a.dgate_stride + shift, sum_g);
            else of.template write<MC_F32>(mine, begin < first ? 0 : a.dim, sum_g);
            EACH(k, e) sum_g[k][e] = 0;
        }
        if (fresh) ++group, group_end += a.gate_rows;
    }
    if (a.grads[1]) of.template write<MC_F32>(mine, 2 * a.dim, sum_w);
    if (a.grads[2]) of.template write<MC_F32>(mine, 3 * a.dim, sum_b);
    if (a.grads[3]) of.template write<MC_F32>(mine, 4 * a.dim, sum_pw);
    if (a.grads[4]) of.template write<MC_F32>(mine, 5 * a.dim, sum_pb);
}

__device__ __forceinline__ void store_one(void *p, int type, int64_t at, float v)
{
    if (type == MC_F32) static_cast<float *>(p)[at] = v;
    else if (type == MC_F16) static_cast<_Float16 *>(p)[at] = (_Float16)v;
    else static_cast<__bf16 *>(p)[at] = (__bf16)v;
}

constexpr int SUM_COLUMNS = 64, SUM_LINES = 64;
// The workgroups' sums of 64 columns, four to a thread and 64 threads to a column.  blockIdx.y: 0 .. 3 the parameters, from 4 on rows of the gate that several
// workgroups share: by the row's number, or (`by_border`) by the first border between workgroups that lies in it.
__global__ __launch_bounds__(SUM_COLUMNS / 4 * SUM_LINES) void block_norm_sum_kernel(NormArgs a, int by_border)
{
    __shared__ float part[SUM_LINES][SUM_COLUMNS + 4];
    const int quad = threadIdx.x % (SUM_COLUMNS / 4), line = threadIdx.x / (SUM_COLUMNS / 4), column = blockIdx.x * SUM_COLUMNS + 4 * quad;
    int from = 0, to = a.workgroups - 1, slot = 1 + (int)blockIdx.y + 1;
    int64_t group = 0;
    void *out;
    if (blockIdx.y < 4) {
        out = a.grads[1 + blockIdx.y];
        if (!out) return;
    } else {
        const int64_t i = blockIdx.y - 4;
        group = by_border ? ((i + 1) * a.per) / a.gate_rows : i;
        const int64_t begin = group * a.gate_rows, last = begin + a.gate_rows - 1;
        from = (int)(begin / a.per);
        to = (int)(last / a.per);
        if (a.rows > 0 && (from == to || (by_border && from != i))) return;
        out = a.grads[0];
        slot = -1;
    }
    float s[4] = {0, 0, 0, 0};
    const int n = a.dim - column;
    if (n > 0 && a.rows > 0) {
#pragma unroll 4
        for (int w = from + line; w <= to; w += SUM_LINES) {
            const int place = slot >= 0 ? slot : group * a.gate_rows < w * a.per ? 0 : 1;
            const float *p = a.partial + ((int64_t)w * 6 + place) * a.dim + column;
            float v[4];
            if (n >= 4) {
                __builtin_memcpy(v, p, 16);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = e < n ? p[e] : 0;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[e];
        }
    }
    __builtin_memcpy(&part[line][4 * quad], s, 16);
    __syncthreads();
    if (threadIdx.x >= SUM_COLUMNS || (int)(blockIdx.x * SUM_COLUMNS + threadIdx.x) >= a.dim) return;
    float sum = 0;
#pragma unroll 8
    for (int l = 0; l < SUM_LINES; ++l) sum += part[l][threadIdx.x];
    store_one(out, a.p_type, (slot >= 0 ? 0 : group * a.dgate_stride) + blockIdx.x * SUM_COLUMNS + threadIdx.x, sum);
}

template <int TYPE, int RTYPE, int THREADS, int E> hipError_t forward(NormArgs a, hipStream_t s)
{
    constexpr int PACKED = THREADS == 64 ? 4 : 1;
    constexpr int64_t MOST = NORM_LAUNCH_THREADS / (THREADS * PACKED) * PACKED; // rows of a launch
    hipError_t e = hipSuccess;
    for (a.first = 0; a.first < a.rows && e == hipSuccess; a.first += MOST) {
        const int64_t rows = a.rows - a.first < MOST ? a.rows - a.first : MOST;
        const dim3 grid((unsigned)((rows + PACKED - 1) / PACKED)), block(THREADS * PACKED);
        e = a.dim % 8 == 0 ? launch_kernel((block_norm_kernel<TYPE, RTYPE, THREADS, E, PACKED, true>), grid, block, 0, s, a)
                           : launch_kernel((block_norm_kernel<TYPE, RTYPE, THREADS, E, PACKED, false>), grid, block, 0, s, a);
    }
    return e;
}
template <int TYPE, int RTYPE> hipError_t forward_of(const NormArgs &a, hipStream_t s)
{
    if (a.dim <= 512) return forward<TYPE, RTYPE, 64, 1>(a, s);
    if (a.dim <= 1024) return forward<TYPE, RTYPE, 64, 2>(a, s);
    if (a.dim <= 2048) return forward<TYPE, RTYPE, 256, 1>(a, s);
    if (a.dim <= 4096) return forward<TYPE, RTYPE, 256, 2>(a, s);
    if (a.dim <= 8192) return forward<TYPE, RTYPE, 512, 2>(a, s);
    return forward<TYPE, RTYPE, 1024, 2>(a, s);
}

template <int TYPE, int RTYPE, int THREADS, int E, bool LAYER, bool SUMS> hipError_t backward(const NormArgs &a, hipStream_t s)
{
    const hipError_t e = launch_kernel((block_norm_backward_kernel<TYPE, RTYPE, THREADS, E, LAYER, SUMS>), dim3(a.workgroups), dim3(THREADS), 0, s, a);
    if (SUMS || e != hipSuccess || !(a.grads[0] || a.grads[1] || a.grads[2] || a.grads[3] || a.grads[4])) return e;
    return launch_kernel((block_norm_columns_kernel<TYPE, RTYPE>), dim3((a.dim + COLUMNS_EACH - 1) / COLUMNS_EACH, a.workgroups), dim3(COLUMN_THREADS), 0, s, a);
}
// Rows of more than 4096 elements, gradients, us (a copy of their bytes takes 78, 78, 78, 157, 157):
//                                  6510 x 5120 bf16 rms, layer   2712 x 12288 bf16 layer   6510 x 5120 fp32 rms   2034 x 16384 fp32 layer
//   512 threads, sums with the row     194
//   512 threads, sums by columns                  279                     637                       333                    687
//   1024 threads, sums with the row    186        384                                               523
//   1024 threads, sums by columns      201        198                     419                       282                    506
template <int TYPE, int RTYPE, bool LAYER> hipError_t backward_kind(const NormArgs &a, hipStream_t s)
{
    if (a.dim <= 512) return backward<TYPE, RTYPE, 64, 1, LAYER, true>(a, s);
    if (a.dim <= 1024) return backward<TYPE, RTYPE, 128, 1, LAYER, true>(a, s);
    if (a.dim <= 2048) return backward<TYPE, RTYPE, 256, 1, LAYER, true>(a, s);
    if (a.dim <= 4096) return backward<TYPE, RTYPE, 512, 1, LAYER, true>(a, s);
    if (a.dim <= 8192) {
        if constexpr (!LAYER && TYPE != MC_F32) return backward<TYPE, RTYPE, 512, 2, LAYER, true>(a, s);
        else return backward<TYPE, RTYPE, 1024, 1, LAYER, false>(a, s);
    }
    return backward<TYPE, RTYPE, 1024, 2, LAYER, false>(a, s);
}
template <int TYPE, int RTYPE> hipError_t backward_of(const NormArgs &a, hipStream_t s)
{
    const bool layer = a.pre == MC_NORM_LAYER || a.post == MC_NORM_LAYER || a.bias || a.post_bias;
    return layer ? backward_kind<TYPE, RTYPE, true>(a, s) : backward_kind<TYPE, RTYPE, false>(a, s);
}

} // namespace

hipError_t launch_block_norm(const NormArgs &a, hipStream_t s)
{
    if (a.type == MC_F32) return forward_of<MC_F32, MC_F32>(a, s);
    if (a.type == MC_F16) return a.r_type == MC_F16 ? forward_of<MC_F16, MC_F16>(a, s) : forward_of<MC_F16, MC_F32>(a, s);
    return a.r_type == MC_BF16 ? forward_of<MC_BF16, MC_BF16>(a, s) : forward_of<MC_BF16, MC_F32>(a, s);
}

hipError_t launch_block_norm_backward(NormArgs a, hipStream_t s)
{
    const bool params = a.grads[1] || a.grads[2] || a.grads[3] || a.grads[4];
    const dim3 block(SUM_COLUMNS / 4 * SUM_LINES);
    const unsigned columns = (a.dim + SUM_COLUMNS - 1) / SUM_COLUMNS;
    if (a.rows == 0) { // sums over no rows
        a.per = 1;
        a.workgroups = 0;
        return launch_kernel(block_norm_sum_kernel, dim3(columns, (unsigned)(4 + (a.grads[0] ? a.gate_groups : 0))), block, 0, s, a, 0);
    }
    a.workgroups = norm_workgroups(a.rows, a.dim);
    a.per = (a.rows + a.workgroups - 1) / a.workgroups;
    a.workgroups = (int)((a.rows + a.per - 1) / a.per);
    const hipError_t e = a.type == MC_F32 ? backward_of<MC_F32, MC_F32>(a, s)
                       : a.type == MC_F16 ? (a.r_type == MC_F16 ? backward_of<MC_F16, MC_F16>(a, s) : backward_of<MC_F16, MC_F32>(a, s))
                                          : (a.r_type == MC_BF16 ? backward_of<MC_BF16, MC_BF16>(a, s) : backward_of<MC_BF16, MC_F32>(a, s));
    // rows of the gate that no border between workgroups can cut: written by the first kernel
    const bool cut = a.grads[0] && a.workgroups > 1 && a.gate_rows > 1;
    if (e != hipSuccess || (!params && !cut)) return e;
    const int by_border = a.gate_groups > a.workgroups - 1;
    const unsigned gates = cut ? (unsigned)(by_border ? a.workgroups - 1 : a.gate_groups) : 0;
    return launch_kernel(block_norm_sum_kernel, dim3(columns, 4 + gates), block, 0, s, a, by_border);
}
