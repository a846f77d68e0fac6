// The gated feed-forward block, h = act(x Wg^T) (x Wu^T), and its gradient
//   dg = dh u act'(g),   du = dh act(g),   dx = dg Wg + du Wu,   dWg = dg^T x,   dWu = du^T x.
// All products have the form C[m][n] = sum of A[m][k] B[n][k] with k along the rows of both (the gradient's operands that lie the other way are written transposed first).
#include "layer.h"

#include "lds_async.h"

namespace {

using mcu::v4f;
using mcu::v4i;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// ---- activations ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float g) { return 1.0f / (1.0f + expf(-g)); }
constexpr float GELU_A = 0.7978845608028654f, GELU_B = 0.044715f;

__device__ __forceinline__ float activated(float g, int kind)
{
    switch (kind) {
    case MC_ACT_SILU: return g / (1.0f + expf(-g));
    case MC_ACT_GELU: return 0.5f * g * (1.0f + erff(g * 0.7071067811865476f));
    case MC_ACT_GELU_TANH: return 0.5f * g * (1.0f + tanhf(GELU_A * (g + GELU_B * g * g * g)));
    case MC_ACT_RELU: return g > 0 ? g : g != g ? g : 0;
    default: return sigmoid(g);
    }
}
// act(g), and its slope
__device__ __forceinline__ float activated(float g, int kind, float &slope)
{
    switch (kind) {
    case MC_ACT_SILU: {
        const float p = sigmoid(g);
        slope = p * (1.0f + g * (1.0f - p));
        return g * p;
    }
    case MC_ACT_GELU: {
        const float c = 0.5f * (1.0f + erff(g * 0.7071067811865476f));
        slope = c + g * expf(-0.5f * g * g) * 0.3989422804014327f;
        return g * c;
    }
    case MC_ACT_GELU_TANH: {
        const float t = tanhf(GELU_A * (g + GELU_B * g * g * g));
        slope = 0.5f * (1.0f + t) + 0.5f * g * (1.0f - t * t) * GELU_A * (1.0f + 3.0f * GELU_B * g * g);
        return 0.5f * g * (1.0f + t);
    }
    case MC_ACT_RELU:
        slope = g > 0 ? 1 : g != g ? g : 0;
        return g > 0 ? g : g != g ? g : 0;
    default: {
        const float p = sigmoid(g);
        slope = p * (1.0f - p);
        return p;
    }
    }
}

// ---- matrix instructions ----------------------------------------------------------------------------------------------------
// 16 rows of either operand, 16 bytes of each along k: a lane holds piece lane / 16 of row lane % 16.  (fp32: element e of the four pieces are
// the four k of instruction e.)  The result has 4 rows of the first, 4 (lane / 16) + i, for row lane % 16 of the second.
template <int TYPE> __device__ __forceinline__ v4f multiply(const v4i &a, const v4i &b, v4f c)
{
    if constexpr (TYPE == MC_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[e]), __int_as_float(b[e]), c, 0, 0, 0);
        return c;
    } else if constexpr (TYPE == MC_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    }
}

// Four neighbouring elements, `n` of them.
template <class T> __device__ __forceinline__ void store4(T *to, const float (&v)[4], int n)
{
    T h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = (T)v[e];
    if (n >= 4) return (void)__builtin_memcpy(to, h, 4 * sizeof(T));
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) to[e] = h[e];
}

// ---- the tiled product ------------------------------------------------------------------------------------------------------
__device__ const v4i zeros[1] = {};

constexpr int STEP = 128;           // bytes of a row that a step takes: eight pieces of 16
constexpr int TOGETHER = 8;         // tiles of rows that follow one another for the same columns

// BM x BN tiles, WM x WN waves.  GATED: the rows of B are half gate's, half up's, such that each wave has both of its columns.
// Pieces lie in LDS at place (piece ^ row % 8) of their row: the rows that a read addresses at once have different banks.
template <int TYPE, int BM, int BN, int WM, int WN, bool GATED> __global__ __launch_bounds__(64 * WM *WN) void product_kernel(ProductArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int W = WM * WN, RM = BM / WM, RN = BN / WN, MF = RM / 16, NF = RN / 16, CA = BM / 8 / W, CB = BN / 8 / W, STAGE = (BM + BN) * STEP;
    constexpr int PER = 16 / sizeof(T), COLUMNS = GATED ? BN / 2 : BN;
    static_assert(CA * 8 * W == BM && CB * 8 * W == BN && RN % 32 == 0, "whole copies");
    __shared__ __attribute__((aligned(1024))) char lds[2][STAGE];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WN, wn = w % WN;

    // Workgroups go to the eight XCDs round-robin: each gets a run of tiles, in blocks of TOGETHER tiles of rows.
    const int tiles = a.tiles_m * a.tiles_n, per = (tiles + 7) / 8, t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || t >= tiles) return;
    const int block = t / (TOGETHER * a.tiles_n), high = min(TOGETHER, a.tiles_m - block * TOGETHER), in = t - block * TOGETHER * a.tiles_n;
    const int m0 = (block * TOGETHER + in % high) * BM, n0 = in / high * COLUMNS, z = blockIdx.y;

    const int piece = (lane & 7) ^ (lane >> 3);
    const char *const pa = static_cast<const char *>(a.a) + z * a.a_batch + m0 * a.a_stride;
    const char *pb[CB];
    unsigned oa[CA], ob[CB];
#pragma unroll
    for (int i = 0; i < CA; ++i) {
        const int row = (w * CA + i) * 8 + (lane >> 3);
        oa[i] = (unsigned)((min(m0 + row, a.m - 1) - m0) * a.a_stride) + piece * 16;
    }
#pragma unroll
    for (int i = 0; i < CB; ++i) {
        const int first = (w * CB + i) * 8;
        int row = first + (lane >> 3), which = 0;
        if constexpr (GATED) {
            which = first % RN >= RN / 2;
            row = first / RN * (RN / 2) + first % (RN / 2) + (lane >> 3);
        }
        const int64_t stride = GATED && which ? a.b_stride[1] : a.b_stride[0];
        pb[i] = static_cast<const char *>(GATED && which ? a.b[1] : a.b[0]) + n0 * stride;
        ob[i] = (unsigned)((min(n0 + row, a.n - 1) - n0) * stride) + piece * 16;
    }
    const unsigned base = mcu::lds_addr_uniform(lds);
    const int steps = (a.k + 8 * PER - 1) / (8 * PER);
    auto request = [&](int step, int buffer) {
        const int64_t at = (int64_t)step * STEP;
        const unsigned to = base + buffer * STAGE;
        if ((step + 1) * 8 * PER <= a.k) {
#pragma unroll
            for (int i = 0; i < CA; ++i) mcu::copy16_to_lds(pa + at, oa[i], to + (w * CA + i) * 1024);
#pragma unroll
            for (int i = 0; i < CB; ++i) mcu::copy16_to_lds(pb[i] + at, ob[i], to + BM * STEP + (w * CB + i) * 1024);
        } else { // pieces beyond k are zeros of both operands
            const bool there = step * 8 * PER + piece * PER < a.k;
#pragma unroll
            for (int i = 0; i < CA; ++i) mcu::copy16_to_lds(there ? (const void *)(pa + at + oa[i]) : zeros, to + (w * CA + i) * 1024);
#pragma unroll
            for (int i = 0; i < CB; ++i) mcu::copy16_to_lds(there ? (const void *)(pb[i] + at + ob[i]) : zeros, to + BM * STEP + (w * CB + i) * 1024);
        }
    };

    v4f acc[NF][MF];
#pragma unroll
    for (int n = 0; n < NF; ++n)
#pragma unroll
        for (int m = 0; m < MF; ++m) acc[n][m] = (v4f){0, 0, 0, 0};
    if (steps > 0) request(0, 0);
    mcu::vm_wait<0>();
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) request(s + 1, (s + 1) & 1); // (its readers passed the last barrier)
        const char *const la = lds[s & 1] + (wm * RM + (lane & 15)) * STEP, *const lb = lds[s & 1] + (BM + wn * RN + (lane & 15)) * STEP;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = ((h * 4 + (lane >> 4)) ^ (lane & 7)) * 16;
            v4i fa[MF], fb[NF];
#pragma unroll
            for (int m = 0; m < MF; ++m) fa[m] = *reinterpret_cast<const v4i *>(la + at + m * 16 * STEP);
#pragma unroll
            for (int n = 0; n < NF; ++n) fb[n] = *reinterpret_cast<const v4i *>(lb + at + n * 16 * STEP);
#pragma unroll
            for (int n = 0; n < NF; ++n)
#pragma unroll
                for (int m = 0; m < MF; ++m) acc[n][m] = multiply<TYPE>(fb[n], fa[m], acc[n][m]);
        }
        mcu::vm_wait<0>();
        __syncthreads();
    }

#pragma unroll
    for (int m = 0; m < MF; ++m) {
        const int row = m0 + wm * RM + m * 16 + (lane & 15);
        if (row >= a.m) continue;
        if constexpr (GATED) {
#pragma unroll
            for (int n = 0; n < NF / 2; ++n) {
                const int column = n0 + wn * (RN / 2) + n * 16 + 4 * (lane >> 4), count = a.n - column;
                if (count <= 0) continue;
                float h[4], g[4], u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    g[e] = acc[n][m][e];
                    u[e] = acc[NF / 2 + n][m][e];
                    h[e] = activated(g[e], a.activation) * u[e];
                }
                store4(static_cast<T *>(a.h) + row * a.h_stride + column, h, count);
                if (a.g) {
                    store4(static_cast<T *>(a.g) + row * a.saved_stride + column, g, count);
                    store4(static_cast<T *>(a.u) + row * a.saved_stride + column, u, count);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < NF; ++n) {
                const int column = n0 + wn * RN + n * 16 + 4 * (lane >> 4), count = a.n - column;
                if (count <= 0) continue;
                const float v[4] = {acc[n][m][0], acc[n][m][1], acc[n][m][2], acc[n][m][3]};
                store4(static_cast<T *>(z ? a.c[1] : a.c[0]) + row * (z ? a.c_stride[1] : a.c_stride[0]) + column, v, count);
            }
        }
    }
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
// MT tiles of 16 rows of x against 16 rows of either weight, whose pieces go straight into registers: the weights' bytes bound it.  The
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
    v4f g[MT], u[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) g[m] = u[m] = (v4f){0, 0, 0, 0};
    int k = w * TAKE * UNROLL;
    for (; k + TAKE * UNROLL <= a.dim; k += FEW_WAVES * TAKE * UNROLL) {
        v4i fg[UNROLL], fu[UNROLL];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            __builtin_memcpy(&fg[i], pg + k + i * TAKE + q * PER, 16);
            __builtin_memcpy(&fu[i], pu + k + i * TAKE + q * PER, 16);
        }
#pragma unroll
        for (int i = 0; i < UNROLL; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                v4i fx;
                __builtin_memcpy(&fx, px[m] + k + i * TAKE + q * PER, 16);
                g[m] = multiply<TYPE>(fg[i], fx, g[m]);
                u[m] = multiply<TYPE>(fu[i], fx, u[m]);
            }
    }
    for (int i = 0; i < UNROLL && k + i * TAKE < a.dim; ++i) { // what is left, fewer than UNROLL
        const int at = k + i * TAKE + q * PER, count = a.dim - at;
        const v4i fg = load_piece(pg + at, count), fu = load_piece(pu + at, count);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const v4i fx = load_piece(px[m] + at, count);
            g[m] = multiply<TYPE>(fg, fx, g[m]);
            u[m] = multiply<TYPE>(fu, fx, u[m]);
        }
    }
    __shared__ v4f sums[FEW_WAVES][2][MT][64];
#pragma unroll
    for (int m = 0; m < MT; ++m) sums[w][0][m][lane] = g[m], sums[w][1][m][lane] = u[m];
    __syncthreads();
    for (int m = w; m < MT; m += FEW_WAVES) {
        v4f sg = sums[0][0][m][lane], su = sums[0][1][m][lane];
#pragma unroll
        for (int i = 1; i < FEW_WAVES; ++i) sg += sums[i][0][m][lane], su += sums[i][1][m][lane];
        const int row = m * 16 + r, column = n0 + 4 * q, count = a.hidden - column;
        if (row >= a.rows || count <= 0) continue;
        float h[4], gs[4], us[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            gs[e] = sg[e];
            us[e] = su[e];
            h[e] = activated(gs[e], a.activation) * us[e];
        }
        store4(static_cast<T *>(a.h) + row * a.h_stride + column, h, count);
        if (a.g) {
            store4(static_cast<T *>(a.g) + row * a.saved_stride + column, gs, count);
            store4(static_cast<T *>(a.u) + row * a.saved_stride + column, us, count);
        }
    }
}

// ---- the gradient's operands ---------------------------------------------------------------------------------------------------
constexpr int TILE = 64;
// A tile of 64 x 64 elements, of which rows x columns are there: written to `to` transposed, with zeros for missing rows up to `padded`
// of them.  Four threads to a line.
template <class T> __device__ __forceinline__ void write_transposed(const T (&tile)[TILE][TILE + 2], T *to, int64_t stride, int columns, int padded)
{
    const int c = threadIdx.x / 4;
    if (c >= columns) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = threadIdx.x % 4 * 16 + i;
        if (r < padded) to[c * stride + r] = tile[r][c];
    }
}

template <class T> __global__ __launch_bounds__(256) void transpose_kernel(const T *from, int64_t from_stride, int64_t rows, int columns, T *to, int64_t to_stride, int64_t padded)
{
    __shared__ T tile[TILE][TILE + 2];
    const int64_t r0 = (int64_t)blockIdx.y * TILE;
    const int c0 = blockIdx.x * TILE, here = min(TILE, columns - c0);
    for (int i = threadIdx.x; i < TILE * TILE; i += 256) {
        const int r = i / TILE, c = i % TILE;
        tile[r][c] = r0 + r < rows && c < here ? from[(r0 + r) * from_stride + c0 + c] : (T)0;
    }
    __syncthreads();
    write_transposed(tile, to + c0 * to_stride + r0, to_stride, here, (int)min((int64_t)TILE, padded - r0));
}

template <class T> __global__ __launch_bounds__(256) void pad_rows_kernel(const T *from, int64_t from_stride, int64_t rows, int width, T *to, int padded)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * padded; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / padded;
        const int c = (int)(i - r * padded);
        to[i] = c < width ? from[r * from_stride + c] : (T)0;
    }
}

// dg and du (rounded to the type that the products take: half a step of each, whose signs the sums over rows and columns even out), written as rows and
// as columns.  What lies between a matrix's end and its padded end is zero.
template <int TYPE> __global__ __launch_bounds__(256) void gated_grad_kernel(GatedGradArgs a)
{
    typedef typename RealOf<TYPE>::type T;
    __shared__ T tg[TILE][TILE + 2], tu[TILE][TILE + 2];
    const int64_t r0 = (int64_t)blockIdx.y * TILE;
    const int c0 = blockIdx.x * TILE;
    const int64_t width = 2 * (int64_t)a.padded_hidden;
    for (int i = threadIdx.x; i < TILE * TILE; i += 256) {
        const int r = i / TILE, c = i % TILE;
        T dg = (T)0, du = (T)0;
        if (r0 + r < a.rows && c0 + c < a.hidden) {
            const float dh = (float)static_cast<const T *>(a.dh)[(r0 + r) * a.dh_stride + c0 + c];
            const float g = (float)static_cast<const T *>(a.g)[(r0 + r) * a.saved_stride + c0 + c], u = (float)static_cast<const T *>(a.u)[(r0 + r) * a.saved_stride + c0 + c];
            float slope;
            du = (T)(dh * activated(g, a.activation, slope));
            dg = (T)(dh * u * slope);
        }
        tg[r][c] = dg;
        tu[r][c] = du;
        if (a.d && r0 + r < a.rows && c0 + c < a.padded_hidden) {
            T *to = static_cast<T *>(a.d) + (r0 + r) * width + c0 + c;
            to[0] = dg;
            to[a.padded_hidden] = du;
        }
    }
    if (!a.dt) return;
    __syncthreads();
    const int columns = min(TILE, a.padded_hidden - c0), padded = (int)min((int64_t)TILE, a.padded_rows - r0);
    T *to = static_cast<T *>(a.dt) + c0 * a.padded_rows + r0;
    write_transposed(tg, to, a.padded_rows, columns, padded);
    write_transposed(tu, to + a.padded_hidden * a.padded_rows, a.padded_rows, columns, padded);
}

// ---- launches --------------------------------------------------------------------------------------------------------------------
template <int TYPE, int BM, int BN, int WM, int WN, bool GATED> hipError_t product(ProductArgs a, hipStream_t s)
{
    a.tiles_m = (a.m + BM - 1) / BM;
    a.tiles_n = (a.n + (GATED ? BN / 2 : BN) - 1) / (GATED ? BN / 2 : BN);
    return launch_kernel((product_kernel<TYPE, BM, BN, WM, WN, GATED>), dim3((unsigned)((a.tiles_m * a.tiles_n + 7) / 8 * 8), GATED ? 1 : a.batch), dim3(64 * WM * WN), 0, s, a);
}

template <int TYPE, bool GATED> hipError_t product_of(const ProductArgs &a, hipStream_t s)
{
    const int64_t tiles = (int64_t)((a.m + 255) / 256) * ((a.n + (GATED ? 127 : 255)) / (GATED ? 128 : 256)) * (GATED ? 1 : a.batch);
    if (tiles >= 192) return product<TYPE, 256, 256, 2, 4, GATED>(a, s);
    return product<TYPE, 128, 128, 2, 2, GATED>(a, s);
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
    return type == MC_F32 ? product_of<MC_F32, true>(a, s) : type == MC_F16 ? product_of<MC_F16, true>(a, s) : product_of<MC_BF16, true>(a, s);
}
hipError_t launch_product(const ProductArgs &a, mc_type type, hipStream_t s)
{
    return type == MC_F32 ? product_of<MC_F32, false>(a, s) : type == MC_F16 ? product_of<MC_F16, false>(a, s) : product_of<MC_BF16, false>(a, s);
}
hipError_t launch_few_rows(const FewRowsArgs &a, mc_type type, hipStream_t s)
{
    return type == MC_F32 ? few_rows_of<MC_F32>(a, s) : type == MC_F16 ? few_rows_of<MC_F16>(a, s) : few_rows_of<MC_BF16>(a, s);
}
hipError_t launch_gated_grad(const GatedGradArgs &a, mc_type type, hipStream_t s)
{
    const dim3 grid((unsigned)((a.padded_hidden + TILE - 1) / TILE), (unsigned)((a.padded_rows + TILE - 1) / TILE)), block(256);
    return type == MC_F32 ? launch_kernel(gated_grad_kernel<MC_F32>, grid, block, 0, s, a)
         : type == MC_F16 ? launch_kernel(gated_grad_kernel<MC_F16>, grid, block, 0, s, a) : launch_kernel(gated_grad_kernel<MC_BF16>, grid, block, 0, s, a);
}
hipError_t launch_pad_rows(const void *from, int64_t from_stride, int64_t rows, int width, void *to, int padded, int size, hipStream_t s)
{
    const int64_t blocks = (rows * padded + 1023) / 1024;
    const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192)), block(256);
    if (size == 4) return launch_kernel(pad_rows_kernel<uint32_t>, grid, block, 0, s, static_cast<const uint32_t *>(from), from_stride, rows, width, static_cast<uint32_t *>(to), padded);
    return launch_kernel(pad_rows_kernel<uint16_t>, grid, block, 0, s, static_cast<const uint16_t *>(from), from_stride, rows, width, static_cast<uint16_t *>(to), padded);
}
hipError_t launch_transpose(const void *from, int64_t from_stride, int64_t rows, int columns, void *to, int64_t to_stride, int64_t padded, int size, hipStream_t s)
{
    const dim3 grid((unsigned)((columns + TILE - 1) / TILE), (unsigned)((padded + TILE - 1) / TILE)), block(256);
    if (size == 4) return launch_kernel(transpose_kernel<uint32_t>, grid, block, 0, s, static_cast<const uint32_t *>(from), from_stride, rows, columns, static_cast<uint32_t *>(to), to_stride, padded);
    return launch_kernel(transpose_kernel<uint16_t>, grid, block, 0, s, static_cast<const uint16_t *>(from), from_stride, rows, columns, static_cast<uint16_t *>(to), to_stride, padded);
}
