// C-ABI entry points of the operators of a decoder around its attention: argument checks on the host, then kernel launches on the
// caller's stream.  See include/magicube.h for the contract of every function.
#include "layer.h"

#include <cmath>

namespace {

inline bool valid_type(int t) { return t == MC_F32 || t == MC_F16 || t == MC_BF16; }
inline int size_of(int t) { return t == MC_F32 ? 4 : 2; }
inline bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

constexpr int64_t MOST_GROUPS = 0x7fffffff / 256; // (a grid's threads are counted in 32 bits)

// rows of `width` elements: any stride that keeps them apart, elements aligned to their size
bool rows_ok(const void *p, int64_t stride, int64_t rows, int width, int type)
{
    return p && aligned(p, size_of(type)) && (rows <= 1 || stride >= width);
}

int check_workspace(const void *p, size_t bytes, size_t needed)
{
    if (needed == 0) return MC_OK;
    if (!p || bytes < needed) return MC_ENOMEM;
    return aligned(p, 256) ? MC_OK : MC_EALIGN;
}

// ---- norms ----------------------------------------------------------------------------------------------------------------
int check_norm(const mc_block_norm_args *n)
{
    if (!n) return MC_EINVAL;
    auto kind = [](int k) { return k == MC_NORM_NONE || k == MC_NORM_RMS || k == MC_NORM_LAYER; };
    auto beside = [&](int t) { return t == (int)n->type || t == MC_F32; };
    if (!valid_type(n->type) || !beside(n->residual_type) || !beside(n->param_type) || !kind(n->pre) || !kind(n->post)) return MC_EUNSUPPORTED;
    if (n->rows < 0 || n->rows > 0x7fffffff || n->dim < 1 || n->dim > NORM_MOST_DIM || !(n->eps >= 0) || !std::isfinite(n->eps) || !std::isfinite(n->branch_scale) ||
        (n->residual_dev && !std::isfinite(n->residual_scale)))
        return MC_EINVAL;
    if ((n->pre == MC_NORM_NONE && (n->weight_dev || n->bias_dev)) || (n->post == MC_NORM_NONE && (n->post_weight_dev || n->post_bias_dev))) return MC_EINVAL;
    if (n->gate_dev ? n->gate_groups < 1 || n->rows % n->gate_groups != 0 : n->gate_groups != 0) return MC_EINVAL;
    if (n->rows == 0) return n->gate_groups > 65535 - 4 ? MC_EINVAL : MC_OK;
    if (!rows_ok(n->x_dev, n->x_stride, n->rows, n->dim, n->type) || (n->residual_dev && !rows_ok(n->residual_dev, n->residual_stride, n->rows, n->dim, n->residual_type)) ||
        (n->gate_dev && !rows_ok(n->gate_dev, n->gate_stride, n->gate_groups, n->dim, n->param_type)))
        return MC_EINVAL;
    for (const void *p : {n->weight_dev, n->bias_dev, n->post_weight_dev, n->post_bias_dev})
        if (!aligned(p, size_of(n->param_type))) return MC_EINVAL;
    return MC_OK;
}

NormArgs norm_args(const mc_block_norm_args *n)
{
    NormArgs a = {};
    a.x = n->x_dev; a.x_stride = n->x_stride; a.r = n->residual_dev; a.r_stride = n->residual_stride;
    a.weight = n->weight_dev; a.bias = n->bias_dev; a.post_weight = n->post_weight_dev; a.post_bias = n->post_bias_dev;
    a.gate = n->gate_dev; a.gate_stride = n->gate_stride; a.gate_groups = n->gate_groups;
    a.gate_rows = n->gate_dev ? n->rows / n->gate_groups : 1;
    a.rows = n->rows; a.dim = n->dim; a.type = n->type; a.r_type = n->residual_type; a.p_type = n->param_type;
    a.pre = n->pre; a.post = n->post; a.branch_scale = n->branch_scale; a.residual_scale = n->residual_scale; a.eps = n->eps;
    return a;
}

// ---- the gated feed-forward block -------------------------------------------------------------------------------------------
constexpr int64_t FFN_MOST_ROWS = (int64_t)1 << 21, FFN_MOST_WIDTH = (int64_t)1 << 20, FFN_MOST = (int64_t)1 << 34, FFN_MOST_LINE = (int64_t)1 << 24;

int check_ffn(const mc_gated_ffn_args *f)
{
    if (!f) return MC_EINVAL;
    if (!valid_type(f->type) || (int)f->activation < MC_ACT_SILU || (int)f->activation > MC_ACT_SIGMOID) return MC_EUNSUPPORTED;
    const int64_t wide = f->dim > f->hidden ? f->dim : f->hidden;
    if (f->rows < 0 || f->rows > FFN_MOST_ROWS || f->dim < 1 || f->hidden < 1 || wide > FFN_MOST_WIDTH || f->rows * wide > FFN_MOST ||
        (int64_t)f->dim * f->hidden > FFN_MOST)
        return MC_EINVAL;
    const int size = size_of(f->type);
    for (const int64_t stride : {f->x_stride, f->gate_stride, f->up_stride})
        if (stride > (FFN_MOST_LINE - 1) / size) return MC_EINVAL;
    if ((f->rows > 0 && !rows_ok(f->x_dev, f->x_stride, f->rows, f->dim, f->type)) || !rows_ok(f->gate_dev, f->gate_stride, f->hidden, f->dim, f->type) ||
        !rows_ok(f->up_dev, f->up_stride, f->hidden, f->dim, f->type))
        return MC_EINVAL;
    return MC_OK;
}

inline int pieces_up(int64_t n, int type)
{
    const int per = 16 / size_of(type);
    return (int)((n + per - 1) / per * per);
}
// The tiled product reads rows in pieces of 16 bytes.
inline bool in_pieces(const void *p, int64_t stride, int64_t rows, int width, int type)
{
    return aligned(p, 16) && (rows <= 1 || stride * size_of(type) % 16 == 0) && width * size_of(type) % 16 == 0;
}

// One more matrix to be copied
void *padded_copy(PadRowsArgs &a, const void *from, int64_t stride, int64_t rows, void *to)
{
    a.matrix[a.count++] = {from, stride, rows, to};
    return to;
}

struct FfnPlan { bool few, pad_x, pad_gate, pad_up; size_t x, gate, up, bytes; }; // offsets of the copies
FfnPlan ffn_plan(const mc_gated_ffn_args *f)
{
    FfnPlan p = {};
    const size_t line = (size_t)pieces_up(f->dim, f->type) * size_of(f->type);
    p.pad_x = !in_pieces(f->x_dev, f->x_stride, f->rows, f->dim, f->type);
    p.pad_gate = !in_pieces(f->gate_dev, f->gate_stride, f->hidden, f->dim, f->type);
    p.pad_up = !in_pieces(f->up_dev, f->up_stride, f->hidden, f->dim, f->type);
    p.few = few_rows_best(f->rows, f->hidden, p.pad_gate || p.pad_up);
    if (p.few) return p;
    p.gate = p.pad_x ? rounded(f->rows * line) : 0;
    p.up = p.gate + (p.pad_gate ? rounded(f->hidden * line) : 0);
    p.bytes = p.up + (p.pad_up ? rounded(f->hidden * line) : 0);
    return p;
}

// The gradient's operands and copies: offsets, and the products' plans
struct FfnGradPlan {
    int hidden;                    // padded
    ProductPlan dx, dw;
    bool pad_x, pad_gate, pad_up;
    size_t dg, du, x, gate, up, partial, bytes;
};
FfnGradPlan ffn_grad_plan(const mc_gated_ffn_args *f)
{
    FfnGradPlan p = {};
    const size_t size = size_of(f->type), line = (size_t)pieces_up(f->dim, f->type) * size;
    p.hidden = pieces_up(f->hidden, f->type);
    p.pad_x = !in_pieces(f->x_dev, f->x_stride, f->rows, f->dim, f->type);
    p.pad_gate = !in_pieces(f->gate_dev, f->gate_stride, f->hidden, f->dim, f->type);
    p.pad_up = !in_pieces(f->up_dev, f->up_stride, f->hidden, f->dim, f->type) || p.pad_gate || (f->hidden > 1 && f->up_stride != f->gate_stride);
    p.pad_gate = p.pad_up;         // (both halves of a sum have one stride)
    p.dx = product_plan(f->rows, f->dim, 2 * (int64_t)f->hidden, 1, f->type, false);
    p.dw = product_plan(f->hidden, f->dim, f->rows, 2, f->type, false);
    p.du = p.dg + rounded((size_t)p.hidden * f->rows * size);
    p.x = p.du + rounded((size_t)p.hidden * f->rows * size);
    p.gate = p.x + (p.pad_x ? rounded(f->rows * line) : 0);
    p.up = p.gate + (p.pad_gate ? rounded(f->hidden * line) : 0);
    p.partial = p.up + (p.pad_up ? rounded(f->hidden * line) : 0);
    const size_t of_dx = p.dx.splits > 1 ? sizeof(float) * p.dx.splits * f->rows * f->dim : 0, of_dw = p.dw.splits > 1 ? sizeof(float) * 2 * p.dw.splits * f->hidden * f->dim : 0;
    p.bytes = p.partial + rounded(of_dx > of_dw ? of_dx : of_dw);
    return p;
}

} // namespace

extern "C" int mc_block_norm(const mc_block_norm_args *args, void *y_dev, int64_t y_stride, void *n_dev, int64_t n_stride, void *stream)
{
    if (const int rc = check_norm(args)) return rc;
    if (args->rows == 0) return MC_OK;
    if ((y_dev && !rows_ok(y_dev, y_stride, args->rows, args->dim, args->residual_type)) ||
        (args->pre ? !rows_ok(n_dev, n_stride, args->rows, args->dim, args->type) : n_dev != nullptr || !y_dev))
        return MC_EINVAL;
    NormArgs a = norm_args(args);
    a.y = y_dev; a.y_stride = y_stride; a.n = n_dev; a.n_stride = n_stride;
    MC_HIP(launch_block_norm(a, static_cast<hipStream_t>(stream)));
    return MC_OK;
}

extern "C" size_t mc_block_norm_backward_workspace(int64_t rows, int dim)
{
    if (rows < 1 || rows > 0x7fffffff || dim < 1 || dim > NORM_MOST_DIM) return 0;
    return ((size_t)norm_workgroups(rows, dim) * 6 * dim + (dim > NORM_SUMS ? 8 * (size_t)rows : 0)) * sizeof(float);
}

extern "C" int mc_block_norm_backward(const mc_block_norm_args *args, const void *dy_dev, int64_t dy_stride, const void *dn_dev, int64_t dn_stride,
                                      const mc_block_norm_grads *grads, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (const int rc = check_norm(args)) return rc;
    if (!grads) return MC_EINVAL;
    if ((dn_dev && !args->pre) || (grads->dresidual_dev && !args->residual_dev) || (grads->dgate_dev && !args->gate_dev) || (grads->dweight_dev && !args->weight_dev) ||
        (grads->dbias_dev && !args->bias_dev) || (grads->dpost_weight_dev && !args->post_weight_dev) || (grads->dpost_bias_dev && !args->post_bias_dev))
        return MC_EINVAL;
    const int64_t rows = args->rows;
    const int dim = args->dim;
    // (the parameters' gradients are written by sums over no rows, too)
    NormArgs a = norm_args(args);
    a.dy = dy_dev; a.dy_stride = dy_stride; a.dn = dn_dev; a.dn_stride = dn_stride;
    a.dx = grads->dx_dev; a.dx_stride = grads->dx_stride; a.dr = grads->dresidual_dev; a.dr_stride = grads->dresidual_stride;
    a.grads[0] = grads->dgate_dev; a.grads[1] = grads->dweight_dev; a.grads[2] = grads->dbias_dev; a.grads[3] = grads->dpost_weight_dev; a.grads[4] = grads->dpost_bias_dev;
    a.dgate_stride = grads->dgate_stride;
    for (void *p : a.grads)
        if (!aligned(p, size_of(args->param_type))) return MC_EINVAL;
    if ((dy_dev && !rows_ok(dy_dev, dy_stride, rows, dim, args->residual_type)) || (dn_dev && !rows_ok(dn_dev, dn_stride, rows, dim, args->type)) ||
        (a.dx && !rows_ok(a.dx, a.dx_stride, rows, dim, args->type)) || (a.dr && !rows_ok(a.dr, a.dr_stride, rows, dim, args->residual_type)) ||
        (a.grads[0] && !rows_ok(a.grads[0], a.dgate_stride, args->gate_groups, dim, args->param_type)))
        return MC_EINVAL;
    if (const int rc = check_workspace(workspace_dev, workspace_bytes, mc_block_norm_backward_workspace(rows, dim))) return rc;
    a.partial = static_cast<float *>(workspace_dev);
    MC_HIP(launch_block_norm_backward(a, static_cast<hipStream_t>(stream)));
    return MC_OK;
}

extern "C" size_t mc_gated_ffn_workspace(const mc_gated_ffn_args *args) { return check_ffn(args) == MC_OK ? ffn_plan(args).bytes : 0; }

extern "C" int mc_gated_ffn(const mc_gated_ffn_args *args, void *h_dev, int64_t h_stride, float *g_dev, float *u_dev, int64_t saved_stride, void *workspace_dev,
                            size_t workspace_bytes, void *stream)
{
    if (const int rc = check_ffn(args)) return rc;
    const mc_gated_ffn_args &f = *args;
    if (f.rows == 0) return MC_OK;
    if (!rows_ok(h_dev, h_stride, f.rows, f.hidden, f.type) || !g_dev != !u_dev ||
        (g_dev && (!rows_ok(g_dev, saved_stride, f.rows, f.hidden, MC_F32) || !rows_ok(u_dev, saved_stride, f.rows, f.hidden, MC_F32))))
        return MC_EINVAL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const FfnPlan p = ffn_plan(args);
    if (p.few) {
        FewRowsArgs a = {};
        a.x = f.x_dev; a.gate = f.gate_dev; a.up = f.up_dev;
        a.x_stride = f.x_stride; a.gate_stride = f.gate_stride; a.up_stride = f.up_stride;
        a.rows = (int)f.rows; a.dim = f.dim; a.hidden = f.hidden; a.activation = f.activation;
        a.h = h_dev; a.g = g_dev; a.u = u_dev; a.h_stride = h_stride; a.saved_stride = saved_stride;
        MC_HIP(launch_few_rows(a, f.type, s));
        return MC_OK;
    }
    if (const int rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
    char *const ws = static_cast<char *>(workspace_dev);
    const int size = size_of(f.type), padded = pieces_up(f.dim, f.type);
    ProductArgs a = {};
    a.a[0] = f.x_dev; a.b[0] = f.gate_dev; a.b[1] = f.up_dev;
    a.a_stride = f.x_stride * size; a.b_stride[0] = f.gate_stride * size; a.b_stride[1] = f.up_stride * size;
    PadRowsArgs pads = {};
    if (p.pad_x) a.a[0] = padded_copy(pads, f.x_dev, f.x_stride, f.rows, ws + p.x), a.a_stride = (int64_t)padded * size;
    if (p.pad_gate) a.b[0] = padded_copy(pads, f.gate_dev, f.gate_stride, f.hidden, ws + p.gate), a.b_stride[0] = (int64_t)padded * size;
    if (p.pad_up) a.b[1] = padded_copy(pads, f.up_dev, f.up_stride, f.hidden, ws + p.up), a.b_stride[1] = (int64_t)padded * size;
    pads.width = f.dim; pads.padded = padded;
    if (pads.count) MC_HIP(launch_pad_rows(pads, f.type, s));
    a.m = (int)f.rows; a.n = f.hidden; a.k = f.dim;
    a.h = h_dev; a.g = g_dev; a.u = u_dev; a.h_stride = h_stride; a.saved_stride = saved_stride; a.activation = f.activation;
    MC_HIP(launch_gated_product(a, f.type, s));
    return MC_OK;
}

extern "C" size_t mc_gated_ffn_backward_workspace(const mc_gated_ffn_args *args) { return check_ffn(args) == MC_OK ? ffn_grad_plan(args).bytes : 0; }

extern "C" int mc_gated_ffn_backward(const mc_gated_ffn_args *args, const void *dh_dev, int64_t dh_stride, const float *g_dev, const float *u_dev, int64_t saved_stride,
                                     void *dx_dev, int64_t dx_stride, void *dgate_dev, int64_t dgate_stride, void *dup_dev, int64_t dup_stride,
                                     void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (const int rc = check_ffn(args)) return rc;
    const mc_gated_ffn_args &f = *args;
    if ((f.rows > 0 && (!rows_ok(dh_dev, dh_stride, f.rows, f.hidden, f.type) || !rows_ok(g_dev, saved_stride, f.rows, f.hidden, MC_F32) ||
                        !rows_ok(u_dev, saved_stride, f.rows, f.hidden, MC_F32))) ||
        (dx_dev && !rows_ok(dx_dev, dx_stride, f.rows, f.dim, f.type)) || (dgate_dev && !rows_ok(dgate_dev, dgate_stride, f.hidden, f.dim, f.type)) ||
        (dup_dev && !rows_ok(dup_dev, dup_stride, f.hidden, f.dim, f.type)))
        return MC_EINVAL;
    const FfnGradPlan p = ffn_grad_plan(args);
    if (const int rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    char *const ws = static_cast<char *>(workspace_dev);
    const int size = size_of(f.type);
    const int padded = pieces_up(f.dim, f.type);
    const bool weights = dgate_dev || dup_dev;
    if (f.rows > 0) {
        GatedGradArgs a = {};
        a.dh = dh_dev; a.g = g_dev; a.u = u_dev; a.dh_stride = dh_stride; a.saved_stride = saved_stride;
        a.rows = f.rows; a.hidden = f.hidden; a.activation = f.activation;
        a.dg = ws + p.dg; a.du = ws + p.du; a.padded_hidden = p.hidden;
        MC_HIP(launch_gated_grad(a, f.type, s));
    }
    ProductArgs a = {};
    a.a[0] = ws + p.dg; a.a[1] = ws + p.du; a.a_stride = (int64_t)p.hidden * size;
    a.n = f.dim; a.partial = reinterpret_cast<float *>(ws + p.partial);
    PadRowsArgs pads = {};
    const void *x = f.x_dev, *gate = f.gate_dev, *up = f.up_dev;
    if (weights && p.pad_x && f.rows > 0) x = padded_copy(pads, x, f.x_stride, f.rows, ws + p.x);
    if (dx_dev && p.pad_gate && f.rows > 0) {
        gate = padded_copy(pads, gate, f.gate_stride, f.hidden, ws + p.gate);
        up = padded_copy(pads, up, f.up_stride, f.hidden, ws + p.up);
    }
    pads.width = f.dim; pads.padded = padded;
    if (pads.count) MC_HIP(launch_pad_rows(pads, f.type, s));
    if (dx_dev && f.rows > 0) { // a sum of two products; the weights have a row for each k
        a.b[0] = gate; a.b[1] = up; a.b_stride[0] = (p.pad_gate ? padded : f.gate_stride) * size;
        a.m = (int)f.rows; a.k = f.hidden; a.sum = 2; a.batch = 1;
        a.c[0] = dx_dev; a.c_stride[0] = dx_stride;
        MC_HIP(launch_product(a, p.dx, false, f.type, s));
    }
    if (weights) { // two products with x; rows of both operands are k
        a.b[0] = x; a.b_stride[0] = (p.pad_x ? padded : f.x_stride) * size;
        if (!dgate_dev) a.a[0] = a.a[1];
        a.m = f.hidden; a.k = (int)f.rows; a.sum = 1; a.batch = dgate_dev && dup_dev ? 2 : 1;
        a.c[0] = dgate_dev ? dgate_dev : dup_dev; a.c_stride[0] = dgate_dev ? dgate_stride : dup_stride; a.c[1] = dup_dev; a.c_stride[1] = dup_stride;
        MC_HIP(launch_product(a, p.dw, true, f.type, s));
    }
    return MC_OK;
}

namespace {
int check_logprobs(mc_type type, int64_t rows, int vocab, int64_t stride, float scale, int top)
{
    if (!valid_type(type)) return MC_EUNSUPPORTED;
    if (rows < 0 || vocab < 1 || vocab > (1 << 30) || !(scale >= LOGPROB_LEAST_SCALE) || !std::isfinite(scale * 1.4426950408889634f) || top < 0 || top > LOGPROB_MOST_TOP || top > vocab ||
        (rows > 1 && stride < vocab) || rows > MOST_GROUPS / ((vocab + 4095) / 4096))
        return MC_EINVAL;
    return MC_OK;
}
} // namespace

extern "C" size_t mc_token_logprobs_workspace(int64_t rows, int vocab, mc_type type, int top)
{
    if (rows < 1 || check_logprobs(type, rows, vocab, vocab, 1, top) != MC_OK) return 0;
    const LogprobPlan p = logprob_plan(rows, vocab, type);
    return p.pieces == 1 ? 0 : (size_t)rows * p.pieces * logprob_partial(top) * sizeof(float);
}

extern "C" int mc_token_logprobs(const void *logits_dev, mc_type type, int64_t rows, int vocab, int64_t stride, const int64_t *tokens_dev, float scale, int top,
                                 float *logprobs_dev, float *entropy_dev, float *top_logprobs_dev, int64_t *top_tokens_dev, float *sums_dev,
                                 void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (const int rc = check_logprobs(type, rows, vocab, stride, scale, top)) return rc;
    if (rows == 0) return MC_OK;
    if (!logits_dev || !aligned(logits_dev, size_of(type)) || !tokens_dev || !logprobs_dev || !entropy_dev || (top > 0 && (!top_logprobs_dev || !top_tokens_dev))) return MC_EINVAL;
    if (const int rc = check_workspace(workspace_dev, workspace_bytes, mc_token_logprobs_workspace(rows, vocab, type, top))) return rc;
    const LogprobPlan p = logprob_plan(rows, vocab, type);
    LogprobArgs a = {};
    a.logits = logits_dev; a.stride = stride; a.type = type; a.rows = rows; a.vocab = vocab; a.top = top; a.scale = scale; a.tokens = tokens_dev;
    a.logprobs = logprobs_dev; a.entropy = entropy_dev; a.top_logprobs = top_logprobs_dev; a.top_tokens = top_tokens_dev; a.sums = sums_dev;
    a.pieces = p.pieces; a.piece_vectors = p.piece_vectors; a.partial = static_cast<float *>(workspace_dev);
    MC_HIP(launch_token_logprobs(a, static_cast<hipStream_t>(stream)));
    return MC_OK;
}

extern "C" int mc_token_logprobs_backward(const void *logits_dev, mc_type type, int64_t rows, int vocab, int64_t stride, const int64_t *tokens_dev, float scale, int top,
                                          const int64_t *top_tokens_dev, const float *sums_dev, const float *entropy_dev, const float *dlogprobs_dev,
                                          const float *dentropy_dev, const float *dtop_dev, void *dlogits_dev, int64_t dlogits_stride, void *stream)
{
    if (const int rc = check_logprobs(type, rows, vocab, stride, scale, top)) return rc;
    if (rows == 0) return MC_OK;
    if (!logits_dev || !aligned(logits_dev, size_of(type)) || !tokens_dev || !sums_dev || !entropy_dev || (dtop_dev && top > 0 && !top_tokens_dev) ||
        !rows_ok(dlogits_dev, dlogits_stride, rows, vocab, type))
        return MC_EINVAL;
    LogprobArgs a = {};
    a.logits = logits_dev; a.stride = stride; a.type = type; a.rows = rows; a.vocab = vocab; a.top = top; a.scale = scale; a.tokens = tokens_dev;
    a.chosen = top_tokens_dev; a.sums = const_cast<float *>(sums_dev); a.entropy = const_cast<float *>(entropy_dev);
    a.dlogprobs = dlogprobs_dev; a.dentropy = dentropy_dev; a.dtop = top > 0 ? dtop_dev : nullptr; a.dlogits = dlogits_dev; a.dstride = dlogits_stride;
    MC_HIP(launch_token_logprobs_backward(a, static_cast<hipStream_t>(stream)));
    return MC_OK;
}
