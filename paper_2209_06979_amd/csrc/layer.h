// Internal declarations of the operators of a decoder around its attention: norms with gate and residual, the gated feed-forward
// block, log probabilities of tokens.
#pragma once

#include "decode.h"

// ---- norms (block_norm_kernels.hip) -------------------------------------------------------------------------------------
struct NormArgs {
    const void *x, *r;             // block's output, residual (null: none)
    int64_t x_stride, r_stride;    // elements, as all strides here
    const void *weight, *bias, *post_weight, *post_bias; // null: ones, zeros
    const void *gate;              // null: ones
    int64_t gate_stride, gate_rows, gate_groups; // rows that share a row of the gate, rows of the gate
    int64_t rows;
    int dim, type, r_type, p_type; // mc_type of x and n, of r and y, of the parameters
    int pre, post;                 // mc_norm_kind
    float branch_scale, residual_scale, eps;
    void *y, *n;                   // null: not written
    int64_t y_stride, n_stride;
    int64_t first;                 // first row of a launch (filled by the launcher)
    // backward
    const void *dy, *dn;           // null: zeros
    int64_t dy_stride, dn_stride;
    void *dx, *dr;                 // null: not written
    int64_t dx_stride, dr_stride;
    void *grads[5];                // gate, weight, bias, post weight, post bias; null: not asked for
    int64_t dgate_stride;
    int64_t per;                   // rows of a workgroup (filled by the launcher)
    int workgroups;
    float *partial;                // workgroups x (2 for the gate, 4) x dim; rows of more than NORM_SUMS elements, whose sums may be taken by columns: eight floats for each row
};
constexpr int NORM_MOST_DIM = 16384, NORM_SUMS = 4096;
constexpr int64_t NORM_LAUNCH_THREADS = (int64_t)1 << 31; // (a grid's threads are counted in 32 bits: more rows take further launches)
// Workgroups that a backward pass is cut into, at most: as many as run at once
inline int norm_workgroups(int64_t rows, int dim)
{
    const int most = dim <= 512 ? 2048 : dim <= 1024 ? 1536 : dim <= 2048 ? 768 : 256;
    return (int)(rows < most ? rows : most);
}
hipError_t launch_block_norm(const NormArgs &a, hipStream_t s);
hipError_t launch_block_norm_backward(NormArgs a, hipStream_t s);

// ---- log probabilities (logprob_kernels.hip) -----------------------------------------------------------------------------
struct LogprobArgs {
    const void *logits;
    int64_t stride;
    int type;
    int64_t rows;
    int vocab, top;
    float scale;
    const int64_t *tokens;
    float *logprobs, *entropy, *top_logprobs, *sums; // sums: (maximum, log of the sum) of each row, null: not written
    int64_t *top_tokens;
    int pieces;                    // pieces of a row
    int piece_vectors;             // vectors of 16 bytes of a piece
    float *partial;                // rows x pieces x logprob_partial(top) floats
    // backward
    const float *dlogprobs, *dentropy, *dtop; // null: zeros
    const int64_t *chosen;         // rows x top
    void *dlogits;
    int64_t dstride;
};
constexpr int LOGPROB_MOST_TOP = 64;
constexpr float LOGPROB_LEAST_SCALE = 0x1p-64f; // (with smaller ones differences of logits beyond 1e28 would count, which the kernels clamp)
// Floats of a piece: its maximum, sum and weighted sum (and one float more), and its keys of 64 bits (an even number, for their alignment)
constexpr int logprob_partial(int top) { return 4 + 2 * top; }
constexpr int LOGPROB_GROUPS_WANTED = 1024; // workgroups that all rows together are cut into, where they are fewer
constexpr int LOGPROB_LEAST_VECTORS = 1024; // vectors of a piece: four a thread (512, 1024, 2048: 1 x 131072 bf16 with 20 alternatives 17.1, 14.3, 16.8 us; 64 x 32000 with 5 13.6, 12.2, 14.1)
struct LogprobPlan { int pieces, piece_vectors; };
inline LogprobPlan logprob_plan(int64_t rows, int vocab, int type)
{
    const int per = type == MC_F32 ? 4 : 8, vectors = (vocab + per - 1) / per;
    int64_t pieces = (LOGPROB_GROUPS_WANTED + rows - 1) / (rows > 0 ? rows : 1);
    const int most = (vectors + LOGPROB_LEAST_VECTORS - 1) / LOGPROB_LEAST_VECTORS;
    if (pieces > most) pieces = most;
    if (pieces > 64) pieces = 64;
    if (pieces < 1) pieces = 1;
    const int each = (int)((vectors + pieces - 1) / pieces);
    return {(int)((vectors + each - 1) / (each > 0 ? each : 1)), each};
}
hipError_t launch_token_logprobs(const LogprobArgs &a, hipStream_t s);
hipError_t launch_token_logprobs_backward(const LogprobArgs &a, hipStream_t s);

// ---- the gated feed-forward block (gated_ffn_kernels.hip) ------------------------------------------------------------------
// C[m][n] = sum over k of A(m, k) B(n, k).  An operand lies with k along its rows (a row for each m or n), or with a row for each k
// (the gradient's); rows begin at multiples of 16 bytes, and their elements are whole pieces of 16 bytes, zeros behind k where it runs along them.
struct ProductArgs {
    const void *a[2], *b[2];       // gated: x, and gate and up weights.  Else: one, or a sum of two products
    int64_t a_stride, b_stride[2]; // bytes
    int m, n, k;                   // k of each of the products of a sum
    // gated: h, and g and u in fp32 if they are kept (null: not)
    void *h;
    float *g, *u;
    int64_t h_stride, saved_stride; // elements
    int activation;
    // else
    int sum;                       // products of a sum, 1 or 2
    int batch;                     // or 2 products side by side: of a[0] and a[1] with b[0], into c[0] and c[1]
    void *c[2];
    int64_t c_stride[2];           // elements
    float *partial;                // splits x batch x m x n, of products that are cut along k
    // filled by the launcher
    int tiles_m, tiles_n, splits;
};
struct FewRowsArgs { // a few rows of x against both weights
    const void *x, *gate, *up;
    int64_t x_stride, gate_stride, up_stride; // elements
    int rows, dim, hidden, activation;
    void *h;
    float *g, *u;
    int64_t h_stride, saved_stride;
};
struct GatedGradArgs { // dg and du from dh, g and u
    const void *dh;
    const float *g, *u;
    int64_t dh_stride, saved_stride; // elements
    int64_t rows;
    int hidden, activation;
    void *dg, *du;                 // rows x padded hidden, zeros behind hidden
    int padded_hidden;
};
struct PadRowsArgs { // rows of `width` elements into rows of `padded`, zeros behind them; up to three matrices
    struct Matrix { const void *from; int64_t stride, rows; void *to; } matrix[3];
    int count, width, padded;
};
constexpr int FEW_ROWS = 64;
// Few rows go to the kernel that cuts k among waves and copies nothing: up to 64 where weights would have to be copied for the tiles, up to 32 where tiles of 64 x 64 (32 columns of
// h each) would be no more than compute units, up to 4 where they would be no more than 1.5 times as many.  That kernel and the tiles, bf16, us: 16 rows of 4096 to 4096 18.3, 27.8, 64 rows 30.8, 28.6; 16 rows of 1024 to 2816 5.9, 9.2; fp16 1 row of 4096 to 14336 49.5, 47.8,
// 16 rows 57.8, 47.6, 48 rows 85.3, 52.5; bf16 1 row of 4096 to 11008 35.4, 37.2.
inline bool few_rows_best(int64_t rows, int hidden, bool copies)
{
    return rows <= FEW_ROWS && (copies || (rows <= 32 && hidden <= 32 * 256) || (rows <= 4 && hidden <= 32 * 384));
}
hipError_t launch_gated_product(const ProductArgs &a, mc_type type, hipStream_t s);
constexpr int COMPUTE_UNITS = 256;
// Tiles of a product (256, 128, 96 for 128 x 64, 64, or 32 for 32 x 64), and pieces along k
struct ProductPlan { int tile, splits; };
// The shape of tiles and number of pieces along k with the smallest expected time.  A step of 128 bytes of k takes a workgroup `alone` (us) by itself on a compute
// unit, which runs `together` of them at once and spends `busy` on a step of each when it is full; the pieces' sums cost a launch and their bytes.
// Measured, us, tiles of 256 x 256, 128 x 128, 128 x 64, 64 x 64 and 32 x 64 (with the best number of pieces), dx of rows x dim from hidden:
//   bf16  4096 x 4096 from 11008   566, 760, 1148, 1325, 1732        fp32  2048 x 2048 from 5632   698, 669, 682, 730, 808
//         1024 x 4096 from 4096    87, 82, 86, 117, 176                    777 x 1001 from 2731    145, 107, 103, 105, 110
//         128 x 4096 from 14336    80, 62, 65, 79, 98                      100 x 512 from 1400     70, 27, 19, 15, 12
inline ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int batch, mc_type type, bool gated)
{
    struct Shape { int tile, m, n, together; double alone, busy; };
    static constexpr Shape shapes[2][5] = {{{256, 256, 256, 1, 7.3, 7.3}, {128, 128, 128, 2, 2.05, 1.9}, {96, 128, 64, 2, 1.2, 0.97}, {64, 64, 64, 3, 0.8, 0.53}, {32, 32, 64, 4, 0.5, 0.31}},
                                           {{256, 256, 256, 1, 1.45, 1.45}, {128, 128, 128, 2, 0.65, 0.55}, {96, 128, 64, 2, 0.5, 0.4}, {64, 64, 64, 3, 0.375, 0.24}, {32, 32, 64, 4, 0.34, 0.16}}};
    const int64_t size = type == MC_F32 ? 4 : 2, steps = (k * size + 127) / 128;
    ProductPlan best = {256, 1};
    double least = 1e30;
    for (const Shape &s : shapes[type != MC_F32]) {
        const int64_t tiles = (m + s.m - 1) / s.m * ((n * (gated ? 2 : 1) + s.n - 1) / s.n) * batch;
        if (s.tile != 256 && tiles > 1 << 22) continue; // (a grid's threads are counted in 32 bits)
        for (int splits = 1; splits <= (gated ? 1 : 16); ++splits) {
            if (splits > 1 && (steps / splits < 4 || tiles * splits > 4096)) break;
            const int64_t each = (tiles * splits + COMPUTE_UNITS - 1) / COMPUTE_UNITS, rounds = (each + s.together - 1) / s.together;
            const double alone = rounds * s.alone, busy = each * s.busy;
            double us = (alone > busy ? alone : busy) * ((double)(steps + splits - 1) / splits) + 3;
            if (splits > 1) us += 6 + (splits + 1) * (double)(m * n * batch) * 4 / 3.5e6;
            if (us < least) least = us, best = {s.tile, splits};
        }
    }
    return best;
}
// B has a row for each k, and so has A if a_rows
hipError_t launch_product(const ProductArgs &a, ProductPlan p, bool a_rows, mc_type type, hipStream_t s);
hipError_t launch_few_rows(const FewRowsArgs &a, mc_type type, hipStream_t s);
hipError_t launch_gated_grad(const GatedGradArgs &a, mc_type type, hipStream_t s);
hipError_t launch_pad_rows(const PadRowsArgs &a, mc_type type, hipStream_t s);
