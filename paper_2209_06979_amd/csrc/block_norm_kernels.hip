// The norms after a block and before the next one, with the block's gate and the residual connection, in one pass:
//   a = post(x),   y = residual_scale r + branch_scale gate a,   n = pre(y),
// a norm being v / sqrt(mean v^2 + eps) weight, or (v - mean v) / sqrt(var v + eps) weight + bias.  Rows are held in registers (eight
// neighbouring elements of a thread to a chunk): a variance is taken around the mean, n from the unrounded y.
// Backward, with hat for normed values, W for an operand times its weight, and r for 1 / deviation:
//   dyt = dy + r2 (W(dn) - mean W(dn) - yhat mean(W(dn) yhat)),   dr = residual_scale dyt,   da = branch_scale gate dyt,
//   dx = r1 (W(da) - mean W(da) - xhat mean(W(da) xhat))          (without the first mean where the norm has none)
// and the parameters' gradients are sums over rows of dn yhat, dn, da xhat, da and branch_scale a dyt.  Nothing is kept from the forward call: y is
// worked out again from x and r, unrounded, for the bytes that reading it would cost.  A workgroup takes consecutive rows and
// keeps these sums in registers; a second kernel adds the workgroups' in their order, so that results are the same from call to call.
#include "layer.h"

#include "lds_async.h"

namespace {

using mcu::v4i;

// Eight elements as they lie in memory, of either width
struct Raw { v4i lo, hi; };

__device__ __forceinline__ Raw load_raw(const void *p, int type, int64_t at)
{
    Raw r;
    if (type == MC_F32) {
        __builtin_memcpy(&r.lo, static_cast<const float *>(p) + at, 16);
        __builtin_memcpy(&r.hi, static_cast<const float *>(p) + at + 4, 16);
    } else {
        __builtin_memcpy(&r.lo, static_cast<const uint16_t *>(p) + at, 16);
        r.hi = r.lo;
    }
    return r;
}
__device__ __forceinline__ float as_float(uint16_t bits, int type)
{
    if (type == MC_BF16) return __int_as_float((int)bits << 16);
    _Float16 h;
    __builtin_memcpy(&h, &bits, 2);
    return (float)h;
}
// `n` elements (fewer than eight), zeros behind them
__device__ __forceinline__ Raw load_part(const void *p, int type, int64_t at, int n)
{
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 0;
    if (type == MC_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) w[e] = static_cast<const uint32_t *>(p)[at + e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) w[e / 2] |= (uint32_t)static_cast<const uint16_t *>(p)[at + e] << (16 * (e % 2));
    }
    return {(v4i){(int)w[0], (int)w[1], (int)w[2], (int)w[3]}, (v4i){(int)w[4], (int)w[5], (int)w[6], (int)w[7]}};
}
__device__ __forceinline__ void decode(const Raw &r, int type, float (&v)[8])
{
    if (type == MC_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __int_as_float(r.lo[e]), v[4 + e] = __int_as_float(r.hi[e]);
    } else if (type == MC_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[2 * e] = __int_as_float(r.lo[e] << 16), v[2 * e + 1] = __int_as_float(r.lo[e] & 0xffff0000);
    } else {
        _Float16 h[8];
        __builtin_memcpy(h, &r.lo, 16);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
    }
}
__device__ __forceinline__ void store(void *p, int type, int64_t at, int n, const float (&v)[8])
{
    if (type == MC_F32) {
        float *to = static_cast<float *>(p) + at;
        if (n >= 8) return (void)__builtin_memcpy(to, v, 32);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) to[e] = v[e];
    } else if (type == MC_BF16) {
        __bf16 h[8], *to = static_cast<__bf16 *>(p) + at;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (__bf16)v[e];
        if (n >= 8) return (void)__builtin_memcpy(to, h, 16);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) to[e] = h[e];
    } else {
        _Float16 h[8], *to = static_cast<_Float16 *>(p) + at;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (_Float16)v[e];
        if (n >= 8) return (void)__builtin_memcpy(to, h, 16);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) to[e] = h[e];
    }
}

// A row over THREADS threads, E chunks of eight elements each: chunk k of thread t begins at element 8 (t + k THREADS).
// WHOLE: the row is whole chunks.
template <int THREADS, int E, bool WHOLE> struct Row {
    static constexpr int WAVES = THREADS / 64;
    int t, dim;
    float *shared;    // 2 x 2 x WAVES floats
    int turn;         // which half of them the next sum uses (one barrier to a sum)

    __device__ __forceinline__ int at(int k) const { return 8 * (t + k * THREADS); }
    __device__ __forceinline__ int count(int k) const { return WHOLE ? (at(k) < dim ? 8 : 0) : min(max(dim - at(k), 0), 8); }
    // (chunks beyond the row: the first elements, which are not used)
    __device__ __forceinline__ void load(Raw (&r)[E], const void *p, int type, int64_t row_at) const
    {
        if (WHOLE) {
            if (type == MC_F32) {
#pragma unroll
                for (int k = 0; k < E; ++k) r[k] = load_raw(p, MC_F32, row_at + (at(k) < dim ? at(k) : 0));
            } else {
#pragma unroll
                for (int k = 0; k < E; ++k) r[k] = load_raw(p, MC_F16, row_at + (at(k) < dim ? at(k) : 0));
            }
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) r[k] = count(k) == 8 ? load_raw(p, type, row_at + at(k)) : load_part(p, type, row_at + at(k), count(k));
        }
    }
    __device__ __forceinline__ void sums(float &a, float &b)
    {
#pragma unroll
        for (int j = 32; j > 0; j >>= 1) {
            a += __shfl_xor(a, j);
            b += __shfl_xor(b, j);
        }
        if constexpr (WAVES > 1) {
            float *s = shared + turn * 2 * WAVES;
            turn ^= 1;
            if ((t & 63) == 0) s[t >> 6] = a, s[WAVES + (t >> 6)] = b;
            __syncthreads();
            a = b = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) a += s[w], b += s[WAVES + w];
        }
    }
    // v becomes its normed values; returns 1 / deviation.
    __device__ __forceinline__ float norm(float (&v)[E][8], int kind, float eps)
    {
        float q = 0, none = 0;
        if (kind == MC_NORM_LAYER) {
            float m = 0;
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) m += e < count(k) ? v[k][e] : 0;
            sums(m, none);
            m /= dim;
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] -= m;
        }
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) q += e < count(k) ? v[k][e] * v[k][e] : 0;
        sums(q, none);
        const float r = 1.0f / sqrtf(q / dim + eps);
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] *= r;
        return r;
    }
    // d becomes the gradient through a norm, from that of the normed values `hat`.
    __device__ __forceinline__ void norm_backward(float (&d)[E][8], const float (&hat)[E][8], float r, int kind)
    {
        float mean = 0, dot = 0;
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                mean += e < count(k) ? d[k][e] : 0;
                dot += e < count(k) ? d[k][e] * hat[k][e] : 0;
            }
        sums(mean, dot);
        mean = kind == MC_NORM_LAYER ? mean / dim : 0;
        dot /= dim;
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) d[k][e] = r * (d[k][e] - mean - hat[k][e] * dot);
    }
    // v = v w + b, either null
    __device__ __forceinline__ void scale(float (&v)[E][8], const Raw (&w)[E], bool has_w, const void *b, int type) const
    {
        float f[8];
        if (has_w)
#pragma unroll
            for (int k = 0; k < E; ++k) {
                decode(w[k], type, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] *= f[e];
            }
        if (b) {
            Raw r[E];
            load(r, b, type, 0);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                decode(r[k], type, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] += f[e];
            }
        }
    }
    __device__ __forceinline__ void write(void *p, int type, int64_t row_at, const float (&v)[E][8]) const
    {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (count(k) > 0) store(p, type, row_at + at(k), count(k), v[k]);
    }
};

// PACKED: rows of a workgroup, a wave each
template <int TYPE, int THREADS, int E, bool WHOLE, int PACKED> __global__ __launch_bounds__(THREADS *PACKED) void block_norm_kernel(NormArgs a)
{
    __shared__ float shared[4 * THREADS / 64];
    const int64_t row = (int64_t)blockIdx.x * PACKED + (PACKED > 1 ? threadIdx.x / THREADS : 0);
    if (row >= a.rows) return;
    Row<THREADS, E, WHOLE> of = {(int)(PACKED > 1 ? threadIdx.x % THREADS : threadIdx.x), a.dim, shared, 0};
    Raw x[E], r[E], w[E], pw[E], g[E];
    of.load(x, a.x, TYPE, row * a.x_stride);
    if (a.r) of.load(r, a.r, a.r_type, row * a.r_stride);
    if (a.post_weight) of.load(pw, a.post_weight, a.p_type, 0);
    if (a.gate) of.load(g, a.gate, a.p_type, row / a.gate_rows * a.gate_stride);
    if (a.weight) of.load(w, a.weight, a.p_type, 0);
    float v[E][8], f[8];
#pragma unroll
    for (int k = 0; k < E; ++k) decode(x[k], TYPE, v[k]);
    if (a.post) {
        of.norm(v, a.post, a.eps);
        of.scale(v, pw, a.post_weight != nullptr, a.post_bias, a.p_type);
    }
    if (a.gate) of.scale(v, g, true, nullptr, a.p_type);
#pragma unroll
    for (int k = 0; k < E; ++k) {
        if (a.r) decode(r[k], a.r_type, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = a.branch_scale * v[k][e] + (a.r ? a.residual_scale * f[e] : 0);
    }
    if (a.y) of.write(a.y, a.r_type, row * a.y_stride, v);
    if (!a.pre) return;
    of.norm(v, a.pre, a.eps);
    of.scale(v, w, a.weight != nullptr, a.bias, a.p_type);
    of.write(a.n, TYPE, row * a.n_stride, v);
}

// LAYER: gradients of biases are asked for, or one of the norms takes means
template <int TYPE, int THREADS, int E, bool WHOLE, bool LAYER> __global__ __launch_bounds__(THREADS) void block_norm_backward_kernel(NormArgs a)
{
    __shared__ float shared[4 * THREADS / 64];
    Row<THREADS, E, WHOLE> of = {(int)threadIdx.x, a.dim, shared, 0};
    const int64_t first = blockIdx.x * a.per, end = min(first + a.per, a.rows);
    Raw w[E], pw[E];
    if (a.weight) of.load(w, a.weight, a.p_type, 0);
    if (a.post_weight) of.load(pw, a.post_weight, a.p_type, 0);
    float sum_g[E][8], sum_w[E][8], sum_pw[E][8], sum_b[LAYER ? E : 1][8], sum_pb[LAYER ? E : 1][8];
#pragma unroll
    for (int k = 0; k < E; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sum_g[k][e] = sum_w[k][e] = sum_pw[k][e] = 0;
            if constexpr (LAYER) sum_b[k][e] = sum_pb[k][e] = 0;
        }
    float *const mine = a.partial + (int64_t)blockIdx.x * 6 * a.dim;
    for (int64_t row = first; row < end; ++row) {
        Raw x[E], r[E], dn[E], dy[E], g[E];
        of.load(x, a.x, TYPE, row * a.x_stride);
        if (a.r) of.load(r, a.r, a.r_type, row * a.r_stride);
        if (a.dn) of.load(dn, a.dn, TYPE, row * a.dn_stride);
        if (a.dy) of.load(dy, a.dy, a.r_type, row * a.dy_stride);
        if (a.gate) of.load(g, a.gate, a.p_type, row / a.gate_rows * a.gate_stride);
        float hat1[E][8], hat2[E][8], d[E][8], f[8], h[8];
#pragma unroll
        for (int k = 0; k < E; ++k) decode(x[k], TYPE, hat1[k]);
        const float r1 = a.post ? of.norm(hat1, a.post, a.eps) : 1;
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!WHOLE || E > 1) hat1[k][e] = e < of.count(k) ? hat1[k][e] : 0; // (what lies beyond the row stays out of all sums)
                d[k][e] = hat1[k][e];
            }
        auto branch = [&](float (&v)[E][8]) { // a from xhat
            if (a.post) of.scale(v, pw, a.post_weight != nullptr, LAYER ? a.post_bias : nullptr, a.p_type);
        };
        branch(d);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (a.r) decode(r[k], a.r_type, f);
            if (a.gate) decode(g[k], a.p_type, h);
#pragma unroll
            for (int e = 0; e < 8; ++e) hat2[k][e] = a.branch_scale * (a.gate ? h[e] * d[k][e] : d[k][e]) + (a.r ? a.residual_scale * f[e] : 0);
        }
        if (a.pre && a.dn) {
            const float r2 = of.norm(hat2, a.pre, a.eps);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                decode(dn[k], TYPE, d[k]);
                if (a.weight) decode(w[k], a.p_type, h);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[k][e] = e < of.count(k) ? d[k][e] : 0;
                    sum_w[k][e] += d[k][e] * hat2[k][e];
                    if constexpr (LAYER) sum_b[k][e] += d[k][e];
                    if (a.weight) d[k][e] *= h[e];
                }
            }
            of.norm_backward(d, hat2, r2, a.pre);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[k][e] = 0;
        }
        if (a.dy)
#pragma unroll
            for (int k = 0; k < E; ++k) {
                decode(dy[k], a.r_type, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[k][e] += e < of.count(k) ? f[e] : 0;
            }
        if (a.dr) {
            float v[E][8];
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] = a.residual_scale * d[k][e];
            of.write(a.dr, a.r_type, row * a.dr_stride, v);
        }
        // the branch's share: d becomes da, the gate's gradient takes a
        if (a.grads[0]) {
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) hat2[k][e] = hat1[k][e];
            branch(hat2);
#pragma unroll
            for (int k = 0; k < E; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum_g[k][e] += a.branch_scale * hat2[k][e] * d[k][e];
            // a row of the gate ends here, or the workgroup does: written out whole, or left for the second kernel in the place of a gate's row that began before (0) or in (1) these rows
            const int64_t group = row / a.gate_rows, begin = group * a.gate_rows;
            const bool last = row + 1 == begin + a.gate_rows;
            if (last || row + 1 == end) {
                if (last && begin >= first) of.write(a.grads[0], a.p_type, group * a.dgate_stride, sum_g);
                else of.write(mine, MC_F32, begin < first ? 0 : a.dim, sum_g);
#pragma unroll
                for (int k = 0; k < E; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum_g[k][e] = 0;
            }
        }
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (a.gate) decode(g[k], a.p_type, h);
            if (a.post_weight) decode(pw[k], a.p_type, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[k][e] *= a.branch_scale;
                if (a.gate) d[k][e] *= h[e];
                sum_pw[k][e] += d[k][e] * hat1[k][e];
                if constexpr (LAYER) sum_pb[k][e] += d[k][e];
                if (a.post_weight) d[k][e] *= f[e];
            }
        }
        if (!a.dx) continue;
        if (a.post) of.norm_backward(d, hat1, r1, a.post);
        of.write(a.dx, TYPE, row * a.dx_stride, d);
    }
    if (a.grads[1]) of.write(mine, MC_F32, 2 * a.dim, sum_w);
    if (a.grads[3]) of.write(mine, MC_F32, 4 * a.dim, sum_pw);
    if constexpr (LAYER) {
        if (a.grads[2]) of.write(mine, MC_F32, 3 * a.dim, sum_b);
        if (a.grads[4]) of.write(mine, MC_F32, 5 * a.dim, sum_pb);
    }
}

__device__ __forceinline__ void store_one(void *p, int type, int64_t at, float v)
{
    if (type == MC_F32) static_cast<float *>(p)[at] = v;
    else if (type == MC_F16) static_cast<_Float16 *>(p)[at] = (_Float16)v;
    else static_cast<__bf16 *>(p)[at] = (__bf16)v;
}

constexpr int SUM_COLUMNS = 64, SUM_LINES = 16;
// The workgroups' sums of 64 columns, 16 threads to a column.  blockIdx.y: 0 .. 3 the parameters, from 4 on rows of the gate that several
// workgroups share: by the row's number, or (`by_border`) by the first border between workgroups that lies in it.
__global__ __launch_bounds__(SUM_COLUMNS *SUM_LINES) void block_norm_sum_kernel(NormArgs a, int by_border)
{
    __shared__ float part[SUM_LINES][SUM_COLUMNS];
    const int column = blockIdx.x * SUM_COLUMNS + threadIdx.x % SUM_COLUMNS, line = threadIdx.x / SUM_COLUMNS;
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
        if (from == to || (by_border && from != i)) return;
        out = a.grads[0];
        slot = -1;
    }
    float s = 0;
    if (column < a.dim)
        for (int w = from + line; w <= to; w += SUM_LINES) {
            const int place = slot >= 0 ? slot : group * a.gate_rows < w * a.per ? 0 : 1;
            s += a.partial[((int64_t)w * 6 + place) * a.dim + column];
        }
    part[line][threadIdx.x % SUM_COLUMNS] = s;
    __syncthreads();
    if (line != 0 || column >= a.dim) return;
#pragma unroll
    for (int l = 1; l < SUM_LINES; ++l) s += part[l][threadIdx.x];
    store_one(out, a.p_type, (slot >= 0 ? 0 : group * a.dgate_stride) + column, s);
}

template <int TYPE, int THREADS, int E, bool WHOLE> hipError_t forward(const NormArgs &a, hipStream_t s)
{
    constexpr int PACKED = THREADS == 64 ? 4 : 1;
    return launch_kernel((block_norm_kernel<TYPE, THREADS, E, WHOLE, PACKED>), dim3((unsigned)((a.rows + PACKED - 1) / PACKED)), dim3(THREADS * PACKED), 0, s, a);
}

template <int TYPE> hipError_t forward_type(const NormArgs &a, hipStream_t s)
{
    if (a.dim % 8 != 0) {
        if (a.dim <= 1024) return forward<TYPE, 64, 2, false>(a, s);
        if (a.dim <= 4096) return forward<TYPE, 256, 2, false>(a, s);
        return forward<TYPE, 1024, 2, false>(a, s);
    }
    if (a.dim <= 512) return forward<TYPE, 64, 1, true>(a, s);
    if (a.dim <= 1024) return forward<TYPE, 64, 2, true>(a, s);
    if (a.dim <= 2048) return forward<TYPE, 256, 1, true>(a, s);
    if (a.dim <= 4096) return forward<TYPE, 256, 2, true>(a, s);
    if (a.dim <= 8192) return forward<TYPE, 512, 2, true>(a, s);
    return forward<TYPE, 1024, 2, true>(a, s);
}

template <int TYPE, int THREADS, int E, bool WHOLE> hipError_t backward(const NormArgs &a, hipStream_t s)
{
    const bool layer = a.pre == MC_NORM_LAYER || a.post == MC_NORM_LAYER || a.bias || a.post_bias || a.grads[2] || a.grads[4];
    const dim3 grid(a.workgroups), block(THREADS);
    return layer ? launch_kernel((block_norm_backward_kernel<TYPE, THREADS, E, WHOLE, true>), grid, block, 0, s, a)
                 : launch_kernel((block_norm_backward_kernel<TYPE, THREADS, E, WHOLE, false>), grid, block, 0, s, a);
}

template <int TYPE> hipError_t backward_type(const NormArgs &a, hipStream_t s)
{
    if (a.dim % 8 != 0) {
        if (a.dim <= 1024) return backward<TYPE, 64, 2, false>(a, s);
        if (a.dim <= 4096) return backward<TYPE, 256, 2, false>(a, s);
        return backward<TYPE, 512, 4, false>(a, s);
    }
    if (a.dim <= 512) return backward<TYPE, 64, 1, true>(a, s);
    if (a.dim <= 1024) return backward<TYPE, 64, 2, true>(a, s);
    if (a.dim <= 2048) return backward<TYPE, 256, 1, true>(a, s);
    if (a.dim <= 4096) return backward<TYPE, 256, 2, true>(a, s);
    if (a.dim <= 8192) return backward<TYPE, 512, 2, true>(a, s);
    return backward<TYPE, 512, 4, true>(a, s);
}

} // namespace

hipError_t launch_block_norm(const NormArgs &a, hipStream_t s)
{
    return a.type == MC_F32 ? forward_type<MC_F32>(a, s) : a.type == MC_F16 ? forward_type<MC_F16>(a, s) : forward_type<MC_BF16>(a, s);
}

hipError_t launch_block_norm_backward(NormArgs a, hipStream_t s)
{
    if (a.rows == 0) { // sums over no rows
        a.per = 1;
        a.workgroups = 0;
        return launch_kernel(block_norm_sum_kernel, dim3((a.dim + SUM_COLUMNS - 1) / SUM_COLUMNS, (unsigned)(4 + (a.grads[0] ? a.gate_groups : 0))), dim3(SUM_COLUMNS * SUM_LINES), 0, s, a, 0);
    }
    a.workgroups = norm_workgroups(a.rows, a.dim);
    a.per = (a.rows + a.workgroups - 1) / a.workgroups;
    a.workgroups = (int)((a.rows + a.per - 1) / a.per);
    const hipError_t e = a.type == MC_F32 ? backward_type<MC_F32>(a, s) : a.type == MC_F16 ? backward_type<MC_F16>(a, s) : backward_type<MC_BF16>(a, s);
    const bool params = a.grads[1] || a.grads[2] || a.grads[3] || a.grads[4];
    // rows of the gate that no border between workgroups can cut: written by the first kernel
    const bool cut = a.grads[0] && a.workgroups > 1 && a.gate_rows > 1;
    if (e != hipSuccess || (!params && !cut)) return e;
    const int64_t groups = a.gate_groups;
    const int by_border = groups > a.workgroups - 1;
    const unsigned gates = cut ? (unsigned)(by_border ? a.workgroups - 1 : groups) : 0;
    return launch_kernel(block_norm_sum_kernel, dim3((a.dim + SUM_COLUMNS - 1) / SUM_COLUMNS, 4 + gates), dim3(SUM_COLUMNS * SUM_LINES), 0, s, a, by_border);
}
