// Internal declarations of the operators around decoding: rotary positions, the quantized cache, attention over it.
#pragma once

#include "internal.h"

// Real-valued element types in kernels (mc_type numbers them).
template <int TYPE> struct RealOf;
template <> struct RealOf<MC_F32> { typedef float type; };
template <> struct RealOf<MC_F16> { typedef _Float16 type; };
template <> struct RealOf<MC_BF16> { typedef __bf16 type; };

struct RopeArgs {
    const void *x;
    void *y;
    int64_t x_token_stride, x_head_stride, y_token_stride, y_head_stride; // elements
    const int64_t *positions;
    const double *inv_freq;
    int64_t tokens;
    int heads, dim, rot;
    int interleaved;
    double cos_scale, sin_scale; // magnitude, and with the sign of the direction
    int groups;                  // filled by the launcher: threads that share a token's heads
};

// K and V written into a cache (and read back): vectors of dk elements, one scale each.
struct CacheArgs {
    uint8_t *codes[2];           // K, V
    float *scales[2];
    int64_t slots_end;           // pages * page size
    int page_shift, kv_heads, dk, bits;
    void *x[2];                  // K, V: read by a write, written by a read
    int64_t token_stride[2], head_stride[2]; // elements
    const int64_t *slots;
    int64_t tokens;
    // rotation of K (rot 0: none)
    const int64_t *positions;
    const double *inv_freq;
    int rot, interleaved;
    double magnitude;
    int groups;                  // filled by the launcher, as in RopeArgs
};

// Attention of new tokens over a cache (cache_attention_kernels.hip).
struct CacheAttnArgs {
    const uint8_t *k_codes, *v_codes;
    const float *k_scales, *v_scales;
    int64_t pages;
    int page_shift, kv_heads, dk, group;
    unsigned page_vectors;       // kv_heads * page size
    const int32_t *lengths, *starts; // starts null: max_new rows per sequence
    const int32_t *table;
    int64_t table_stride;
    int table_pages;             // entries of a row of the table
    int batch, max_new;
    int64_t total_new;
    const uint64_t *tree;        // null: a chain
    const void *q;
    int64_t q_token_stride, q_head_stride, o_token_stride, o_head_stride; // elements
    void *o;
    float score_scale;           // times log2(e)
    int pieces;                  // pieces that the sequences' tokens are cut into, per head of the cache (see cache_attention_plan)
    int row_tiles, rows_held;    // tiles of rows (new token, query head of the group) at max_new tokens, and those rows
    float *partial, *sums;       // rows of pieces that are not a whole sequence, and their (maximum, l); null: no sequence is cut
    int units_per_head;          // filled by the launcher
};

hipError_t launch_rope(const RopeArgs &a, mc_type type, hipStream_t s);
hipError_t launch_cache_write(const CacheArgs &a, mc_type type, hipStream_t s);
hipError_t launch_cache_read(const CacheArgs &a, mc_type type, hipStream_t s);
// row_tile: 16, 64 or 128 rows
hipError_t launch_cache_attention(const CacheAttnArgs &a, mc_type type, int bits, int row_tile, hipStream_t s);

constexpr int CACHE_TILE = 32;         // tokens that a wave takes at a time
constexpr int CACHE_WAVES = 4;         // waves of a workgroup, which share a piece
// Tiles of the shortest piece: two a wave.  (Sixteen: one sequence of 1024 tokens, 8 heads of 128, 15.3 us instead of 13.1; from 32768 tokens on 3 % more to 3 % less.)
constexpr int CACHE_MIN_PIECE = 8;
// Pieces asked for, over all heads of the cache and row tiles: as many as run at once, two workgroups a compute unit.  256, 512 and 1024 at 8 heads of 128, four query heads each, bf16: one sequence of
// 65536 tokens 38.9, 37.9, 45.4 us; 8 of 4096 25.5, 24.8, 30.7; 32 of 4096 58.5, 58.6, 65.5; 64 of 8192 185.5, 192.7, 191.9.  Of 500 .. 8192 tokens each: 16 sequences 37.1, 30.4, 34.9;
// 32 60.5, 50.2, 51.7; 48 94.6, 79.1, 72.6; 64 115.9, 94.0, 88.5; 128 193.9, 180.8, 163.2 (there more pieces than run at once even out the end, which the rule does not know).
constexpr int CACHE_PIECES = 512;

// What the launch and its workspace are made for: pieces per head asked for, tiles of rows, whether a sequence can be cut at all, and the
// places for pieces' results: rows of `width` floats, and two floats for each.
struct CacheAttnPlan { int pieces, row_tile, row_tiles, rows, width; bool cut; int64_t slots, lines; };
inline CacheAttnPlan cache_attention_plan(int kv_heads, int dk, int group, int batch, int max_new, int64_t most_tokens)
{
    CacheAttnPlan p = {};
    const int64_t tiles = (most_tokens + CACHE_TILE - 1) / CACHE_TILE;
    p.rows = max_new * group;
    p.width = dk <= 64 ? 64 : dk <= 128 ? 128 : 256;
    // Tiles of 16, 64 and 128 rows for one another, 8 sequences of 4096 tokens, 8 heads of 128, bf16 (us): 16 rows 26.4, 30.9, 39.3; 20 35.1, 35.0, 40.3; 64 54.8, 42.0, 52.2;
    // 68 75.5, 57.1, 52.8; 128 78.1, 62.4, 61.3; 192 127, 99.6, 87.9
    p.row_tile = p.rows <= 16 ? 16 : p.rows <= 64 ? 64 : 128;
    p.row_tiles = (p.rows + p.row_tile - 1) / p.row_tile;
    const int64_t sharers = (int64_t)kv_heads * (p.row_tiles > 0 ? p.row_tiles : 1);
    p.pieces = (int)(CACHE_PIECES / sharers > 1 ? CACHE_PIECES / sharers : 1);
    p.cut = tiles > CACHE_MIN_PIECE && p.pieces > 1 && p.row_tiles > 0 && batch > 0; // (one piece to a head and tile of rows: all tokens together)
    // sequences that are cut have more than one piece, fewer than twice the pieces their share asks for; and every sequence adds one
    // that is not full
    p.slots = p.cut ? (2 * (int64_t)p.pieces < (int64_t)p.pieces + batch ? 2 * (int64_t)p.pieces : (int64_t)p.pieces + batch) : 0;
    p.lines = p.slots * kv_heads * p.rows;
    return p;
}

// How sequences are cut, for both sides: the kernels follow these from the lengths, and the plan above has to hold what comes of it.
#define CACHE_RULE __host__ __device__ __forceinline__
constexpr int CACHE_WHOLE = 0x40000000; // tiles of a piece where nothing is cut
// Tiles that a piece should have, for this many tiles in all
CACHE_RULE int cache_piece_tiles(int total, int pieces)
{
    const int t = (total + pieces - 1) / pieces;
    return t < CACHE_MIN_PIECE ? CACHE_MIN_PIECE : t;
}
// Pieces of a sequence: one while it has up to a quarter more than that (a remnant costs more than it relieves the others of)
CACHE_RULE int cache_pieces_of(int tiles, int each)
{
    if (tiles == 0) return 0;
    const int n = (tiles - 1 + each - each / 4) / each;
    return n < 1 ? 1 : n;
}
// Where the sequences' pieces are more than asked for: longer ones, some times at most, until they run at once (batches that one wave looks over)
constexpr int CACHE_LENGTHENINGS = 6;
CACHE_RULE bool cache_pieces_lengthened(int batch, int pieces) { return batch <= 64 && batch < pieces; }
CACHE_RULE int cache_longer_piece(int each, int n, int pieces) { return each + (int)((int64_t)each * (n - pieces) / (2 * pieces)) + 1; }
// Tiles of each of a sequence's pieces: equal ones, but for whole rounds of the waves
CACHE_RULE int cache_each_of(int tiles, int pieces) { return (tiles + pieces * CACHE_WAVES - 1) / (pieces * CACHE_WAVES) * CACHE_WAVES; }
