// C-ABI entry points of the operators around decoding: argument checks on the host, then kernel launches on the caller's stream.
// See include/magicube.h for the contract of every function.
#include "decode.h"

#include <cmath>

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool valid_type(int t) { return t == MC_F32 || t == MC_F16 || t == MC_BF16; }
inline int size_of(mc_type t) { return t == MC_F32 ? 4 : 2; }
// strides of (token, head) tensors: whole 16-byte pieces
inline bool whole_pieces(int64_t a, int64_t b, int size) { return a * size % 16 == 0 && b * size % 16 == 0; }

constexpr int64_t MOST_TOKENS = (int64_t)1 << 31, MOST_CACHED = (int64_t)1 << 30, MOST_GROUPS = 0x7fffffff / 256; // (a grid's threads are counted in 32 bits)

// Checks a cache and that its device is the current one.
int check(const mc_cache *c)
{
    if (!c || !c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return MC_EINVAL;
    if (c->bits != 8 && c->bits != 4) return MC_EUNSUPPORTED;
    if (c->pages < 1 || c->pages > MOST_TOKENS || c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0 ||
        c->kv_heads < 1 || c->kv_heads > 65535 || c->dk < 1 || c->dk > 256 || c->dk % (128 / c->bits) != 0)
        return MC_EINVAL;
    if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->k_scales) || !aligned16(c->v_scales)) return MC_EALIGN;
    int cur = -1;
    MC_HIP(hipGetDevice(&cur));
    if (cur != c->device) {
        note_detail("the cache lives on device %d, the current device is %d", c->device, cur);
        return MC_EINVAL;
    }
    return MC_OK;
}

inline int shift_of(int page_size) { return __builtin_ctz((unsigned)page_size); }

CacheArgs args_of(const mc_cache *c)
{
    CacheArgs a = {};
    a.codes[0] = static_cast<uint8_t *>(c->k_codes); a.codes[1] = static_cast<uint8_t *>(c->v_codes);
    a.scales[0] = c->k_scales; a.scales[1] = c->v_scales;
    a.slots_end = c->pages * c->page_size;
    a.page_shift = shift_of(c->page_size); a.kv_heads = c->kv_heads; a.dk = c->dk; a.bits = c->bits;
    return a;
}

CacheAttnPlan plan_of(const mc_cache *c, int heads, int batch, int max_new, int table_pages)
{
    return cache_attention_plan(c->kv_heads, c->dk, heads / c->kv_heads, batch, max_new, (int64_t)table_pages * c->page_size);
}

// The shape of a call of the attention: what it and its workspace agree on.
int check_shape(const mc_cache *c, int heads, int batch, int max_new, int table_pages)
{
    if (heads < 1 || heads % c->kv_heads != 0 || batch < 0 || batch > 65535 || max_new < 0 || table_pages < 0) return MC_EINVAL;
    const int64_t tokens = (int64_t)table_pages * c->page_size, rows = (int64_t)max_new * (heads / c->kv_heads);
    // (tokens, a few tiles behind them too, and all sequences' tiles, are counted in 31 bits)
    if (tokens > MOST_CACHED || rows > 65535 * 4 || batch * (tokens / CACHE_TILE + 1) > MOST_CACHED) return MC_EINVAL;
    const CacheAttnPlan p = plan_of(c, heads, batch, max_new, table_pages);
    if (((int64_t)p.pieces + batch) * c->kv_heads > (MOST_GROUPS - 4096) / (p.row_tiles > 0 ? p.row_tiles : 1)) return MC_EINVAL;
    return MC_OK;
}

} // namespace

extern "C" int mc_rope_frequencies(int rot, double base, mc_rope_scaling scaling, double factor, double original, double low, double high,
                                   double *inv_freq_host, double *magnitude_host)
{
    if (rot < 2 || rot % 2 != 0 || !(base > 0) || !std::isfinite(base) || !inv_freq_host) return MC_EINVAL;
    if (scaling != MC_ROPE_PLAIN && scaling != MC_ROPE_LINEAR && scaling != MC_ROPE_BASE && scaling != MC_ROPE_PARTS) return MC_EUNSUPPORTED;
    if (scaling != MC_ROPE_PLAIN && (!(factor >= 1) || !std::isfinite(factor))) return MC_EINVAL;
    if (scaling == MC_ROPE_BASE && rot < 4) return MC_EINVAL;
    if (scaling == MC_ROPE_PARTS && (!(original > 0) || !std::isfinite(original) || !(low >= 0) || !(high > low) || !std::isfinite(high))) return MC_EINVAL;
    if (scaling == MC_ROPE_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int j = 0; j < rot / 2; ++j) {
        double f = std::pow(base, -2.0 * j / rot);
        if (scaling == MC_ROPE_LINEAR) f /= factor;
        if (scaling == MC_ROPE_PARTS) {
            const double turns = original * f / (2 * M_PI), mix = (turns - low) / (high - low), keep = mix < 0 ? 0 : mix > 1 ? 1 : mix;
            f = f * keep + f / factor * (1 - keep);
        }
        inv_freq_host[j] = f;
    }
    if (magnitude_host) *magnitude_host = scaling == MC_ROPE_PARTS ? 0.1 * std::log(factor) + 1 : 1;
    return MC_OK;
}

extern "C" int mc_rope(const void *x_dev, mc_type type, int64_t tokens, int heads, int dim, int64_t x_token_stride, int64_t x_head_stride,
                       const int64_t *positions_dev, const double *inv_freq_dev, int rot, int interleaved, float magnitude, int inverse,
                       void *y_dev, int64_t y_token_stride, int64_t y_head_stride, void *stream)
{
    if (!valid_type((int)type)) return MC_EUNSUPPORTED;
    if (tokens < 0 || tokens >= MOST_TOKENS || heads < 1 || heads > 65535 || dim < 1 || dim > 65536 || rot < 0 || rot > dim || rot % 2 != 0 || !std::isfinite(magnitude))
        return MC_EINVAL;
    if (tokens == 0) return MC_OK;
    if (!x_dev || !y_dev || !positions_dev || (!inv_freq_dev && rot > 0)) return MC_EINVAL;
    if (tokens * heads > MOST_GROUPS * 256 / ((dim + 1) / 2)) return MC_EINVAL; // (threads, a pair of elements each)
    RopeArgs a = {};
    a.x = x_dev; a.y = y_dev;
    a.x_token_stride = x_token_stride; a.x_head_stride = x_head_stride; a.y_token_stride = y_token_stride; a.y_head_stride = y_head_stride;
    a.positions = positions_dev; a.inv_freq = inv_freq_dev;
    a.tokens = tokens; a.heads = heads; a.dim = dim; a.rot = rot; a.interleaved = interleaved != 0;
    a.cos_scale = magnitude; a.sin_scale = inverse ? -magnitude : magnitude;
    MC_HIP(launch_rope(a, type, static_cast<hipStream_t>(stream)));
    return MC_OK;
}

extern "C" int mc_cache_write(const mc_cache *cache, const void *k_dev, const void *v_dev, mc_type type, int64_t tokens, int64_t k_token_stride,
                              int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots_dev,
                              const mc_rope_keys *rope, void *stream)
{
    if (const int rc = check(cache)) return rc;
    if (!valid_type((int)type)) return MC_EUNSUPPORTED;
    if (tokens < 0 || tokens >= MOST_TOKENS) return MC_EINVAL;
    if (rope && (rope->rot < 0 || rope->rot > cache->dk || rope->rot % 2 != 0 || !std::isfinite(rope->magnitude))) return MC_EINVAL;
    if (tokens == 0) return MC_OK;
    if (!k_dev || !v_dev || !slots_dev || (rope && rope->rot > 0 && (!rope->positions_dev || !rope->inv_freq_dev))) return MC_EINVAL;
    if (tokens * cache->kv_heads > MOST_GROUPS * 4) return MC_EINVAL; // (threads, 64 for two vectors at most)
    const int size = size_of(type);
    if (!aligned16(k_dev) || !aligned16(v_dev) || !whole_pieces(k_token_stride, k_head_stride, size) || !whole_pieces(v_token_stride, v_head_stride, size))
        return MC_EALIGN;
    CacheArgs a = args_of(cache);
    a.x[0] = const_cast<void *>(k_dev); a.x[1] = const_cast<void *>(v_dev);
    a.token_stride[0] = k_token_stride; a.head_stride[0] = k_head_stride; a.token_stride[1] = v_token_stride; a.head_stride[1] = v_head_stride;
    a.slots = slots_dev; a.tokens = tokens;
    if (rope) {
        a.positions = rope->positions_dev; a.inv_freq = rope->inv_freq_dev;
        a.rot = rope->rot; a.interleaved = rope->interleaved != 0; a.magnitude = rope->magnitude;
    }
    MC_HIP(launch_cache_write(a, type, static_cast<hipStream_t>(stream)));
    return MC_OK;
}

extern "C" int mc_cache_read(const mc_cache *cache, const int64_t *slots_dev, int64_t tokens, mc_type type, void *k_dev, void *v_dev,
                             int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride, void *stream)
{
    if (const int rc = check(cache)) return rc;
    if (!valid_type((int)type)) return MC_EUNSUPPORTED;
    if (tokens < 0 || tokens >= MOST_TOKENS) return MC_EINVAL;
    if (tokens == 0) return MC_OK;
    if (!k_dev || !v_dev || !slots_dev) return MC_EINVAL;
    if (tokens * cache->kv_heads > MOST_GROUPS * 4) return MC_EINVAL; // (threads, 64 for two vectors at most)
    const int size = size_of(type);
    if (!aligned16(k_dev) || !aligned16(v_dev) || !whole_pieces(k_token_stride, k_head_stride, size) || !whole_pieces(v_token_stride, v_head_stride, size))
        return MC_EALIGN;
    CacheArgs a = args_of(cache);
    a.x[0] = k_dev; a.x[1] = v_dev;
    a.token_stride[0] = k_token_stride; a.head_stride[0] = k_head_stride; a.token_stride[1] = v_token_stride; a.head_stride[1] = v_head_stride;
    a.slots = slots_dev; a.tokens = tokens;
    MC_HIP(launch_cache_read(a, type, static_cast<hipStream_t>(stream)));
    return MC_OK;
}

extern "C" size_t mc_cache_attention_workspace(const mc_cache *cache, int heads, int batch, int max_new, int table_pages)
{
    if (!cache || cache->kv_heads < 1 || cache->page_size < 1 || check_shape(cache, heads, batch, max_new, table_pages) != MC_OK) return 0;
    const CacheAttnPlan p = plan_of(cache, heads, batch, max_new, table_pages);
    return (size_t)p.lines * (p.width + 2) * sizeof(float);
}

extern "C" int mc_cache_attention(const mc_cache *cache, const void *q_dev, mc_type type, int64_t total_new, int heads, int64_t q_token_stride,
                                  int64_t q_head_stride, const int32_t *starts_dev, int batch, int max_new, const int32_t *lengths_dev,
                                  const int32_t *table_dev, int64_t table_stride, int table_pages, const uint64_t *tree_dev,
                                  float score_scale, void *o_dev, int64_t o_token_stride, int64_t o_head_stride, void *workspace_dev,
                                  size_t workspace_bytes, void *stream)
{
    if (const int rc = check(cache)) return rc;
    if (!valid_type((int)type)) return MC_EUNSUPPORTED;
    if (const int rc = check_shape(cache, heads, batch, max_new, table_pages)) return rc;
    if (total_new < 0 || total_new >= MOST_TOKENS || table_stride < table_pages || !std::isfinite(score_scale) || (tree_dev && max_new > 64)) return MC_EINVAL;
    if (!starts_dev && (int64_t)batch * max_new != total_new) return MC_EINVAL;
    if (total_new == 0 || batch == 0 || max_new == 0) return MC_OK;
    if (!q_dev || !o_dev || !lengths_dev || (!table_dev && table_pages > 0)) return MC_EINVAL;
    const int size = size_of(type);
    if (!aligned16(q_dev) || !aligned16(o_dev) || !whole_pieces(q_token_stride, q_head_stride, size) || !whole_pieces(o_token_stride, o_head_stride, size))
        return MC_EALIGN;
    const CacheAttnPlan p = plan_of(cache, heads, batch, max_new, table_pages);
    if (p.cut) {
        if (!workspace_dev || workspace_bytes < (size_t)p.lines * (p.width + 2) * sizeof(float)) return MC_ENOMEM;
        if ((reinterpret_cast<uintptr_t>(workspace_dev) & 255u) != 0) return MC_EALIGN;
    }
    CacheAttnArgs a = {};
    a.k_codes = static_cast<const uint8_t *>(cache->k_codes); a.v_codes = static_cast<const uint8_t *>(cache->v_codes);
    a.k_scales = cache->k_scales; a.v_scales = cache->v_scales;
    a.pages = cache->pages; a.page_shift = shift_of(cache->page_size); a.kv_heads = cache->kv_heads; a.dk = cache->dk; a.group = heads / cache->kv_heads;
    a.page_vectors = (unsigned)cache->kv_heads * (unsigned)cache->page_size;
    a.lengths = lengths_dev; a.starts = starts_dev; a.table = table_dev; a.table_stride = table_stride; a.table_pages = table_pages;
    a.batch = batch; a.max_new = max_new; a.total_new = total_new; a.tree = tree_dev;
    a.q = q_dev; a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride;
    a.o = o_dev; a.o_token_stride = o_token_stride; a.o_head_stride = o_head_stride;
    a.score_scale = (float)(score_scale * 1.4426950408889634); // (scores in base 2)
    a.pieces = p.pieces; a.row_tiles = p.row_tiles; a.rows_held = p.rows;
    a.partial = p.cut ? static_cast<float *>(workspace_dev) : nullptr;
    a.sums = p.cut ? a.partial + p.lines * p.width : nullptr;
    MC_HIP(launch_cache_attention(a, type, cache->bits, p.row_tile, static_cast<hipStream_t>(stream)));
    return MC_OK;
}
