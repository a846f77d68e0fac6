// Attention of new tokens over a quantized cache: one token of each of many sequences, a chunk of a prompt, a tree of drafted tokens.
//   o_i = sum_t p_it s^v_t c^v_t / sum_t p_it,   p_it = exp(scale s^k_t (q_i . c^k_t) - max),   t over what row i may see.
// The rows of a tile are the new tokens' query heads that share a head of the cache.  A wave takes 32 tokens at a time, straight from memory into
// registers: S^T = K q^T, and with the probabilities where that product leaves them, o^T += V^T p^T (their places in a lane are the
// reduction's order of the second product, which V's rows follow).  Both products run on 16-bit floating MFMAs, in which codes are exact.
//
// Scales of V: with s^v = f 2^e, 1/2 <= f < 1, the running maximum is taken over x + e instead of x (x the score in base 2), so that the
// weights  w = 2^(x + e - max) f  of the second product are near 1 for the terms that count, whatever the scales; l = sum 2^(x + e - max) 2^-e.
//
// Sequences are cut into pieces of equal length, as many as fill the device: every workgroup works out its piece from the sequences' lengths,
// which the host does not know.  A piece that is not its whole sequence leaves (maximum, l, o) to a second kernel.
#include "decode.h"

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr float UP = 15.f;             // weights are held 2^15 times as large: f16 keeps what is 2^-24 of that
constexpr float NONE = -__builtin_inff();

__device__ __forceinline__ unsigned bits_of(h2 v) { return __builtin_bit_cast(unsigned, v); }
__device__ __forceinline__ h2 halves_of(unsigned v) { return __builtin_bit_cast(h2, v); }
__device__ __forceinline__ h8 operand(unsigned a, unsigned b, unsigned c, unsigned d) { return __builtin_bit_cast(h8, (v4u){a, b, c, d}); }

// max / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float max_of_groups(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_of_groups(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// ---- which piece ---------------------------------------------------------------------------------------
struct Sequence { int start, n, length; }; // first new token, new tokens, tokens in the cache with them
__device__ __forceinline__ Sequence sequence(const CacheAttnArgs &a, int b)
{
    Sequence s;
    const int64_t most = (int64_t)a.table_pages << a.page_shift;
    const int length = a.lengths[b];
    s.length = length < 0 ? 0 : length > most ? (int)most : length;
    if (a.starts) {
        s.start = a.starts[b];
        const int behind = a.starts[b + 1];
        s.n = s.start < 0 || behind <= s.start || behind > a.total_new ? 0 : behind - s.start < a.max_new ? behind - s.start : a.max_new;
    } else {
        s.start = b * a.max_new;
        s.n = a.max_new;
    }
    return s;
}
__device__ __forceinline__ int tiles_of(const Sequence &s) { return s.n == 0 ? 0 : s.length <= 0 ? 1 : (s.length - 1) / CACHE_TILE + 1; }
// Tiles of a piece, for this many tiles in all
__device__ __forceinline__ int piece_tiles(const CacheAttnArgs &a, int total)
{
    const int t = (total + a.pieces - 1) / a.pieces;
    return t <= CACHE_MIN_PIECE ? CACHE_MIN_PIECE : (t + CACHE_WAVES - 1) / CACHE_WAVES * CACHE_WAVES;
}

__device__ __forceinline__ int scan(int v) // inclusive, over the wave
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(v, o, 64);
        if (lane >= o) v += up;
    }
    return v;
}

// A sequence (b), the tiles of its pieces, how many there are and the number of its first among the pieces of sequences that are cut.
struct Cut { int b, each, pieces, slot, index; };
// The sequence that piece `number` belongs to (BY_PIECE, and its index there), or sequence `number` itself; b = -1: none.
template <bool BY_PIECE> __device__ __forceinline__ Cut cut_of(const CacheAttnArgs &a, int number)
{
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int b = 0; b < a.batch; b += 64) {
        const int t = b + lane < a.batch ? tiles_of(sequence(a, b + lane)) : 0;
        total += __shfl(scan(t), 63, 64);
    }
    Cut c = {-1, a.partial ? piece_tiles(a, total) : 0x7fffffff, 0, 0, 0};
    int before = 0, slots = 0;
    for (int b = 0; b < a.batch; b += 64) {
        const int t = b + lane < a.batch ? tiles_of(sequence(a, b + lane)) : 0;
        const int pieces = t == 0 ? 0 : (t - 1) / c.each + 1, up_to = scan(pieces), cut_up_to = scan(pieces > 1 ? pieces : 0);
        const bool here = BY_PIECE ? before + up_to - pieces <= number && number < before + up_to : b + lane == number;
        const unsigned long long who = __ballot(here);
        if (who) {
            const int l = __builtin_ctzll(who);
            c.b = b + l;
            c.pieces = __shfl(pieces, l, 64);
            c.slot = slots + __shfl(cut_up_to, l, 64) - (c.pieces > 1 ? c.pieces : 0);
            c.index = number - before - __shfl(up_to, l, 64) + c.pieces;
            break;
        }
        before += __shfl(up_to, 63, 64);
        slots += __shfl(cut_up_to, 63, 64);
    }
    c.b = __builtin_amdgcn_readfirstlane(c.b);
    c.each = __builtin_amdgcn_readfirstlane(c.each);
    c.pieces = __builtin_amdgcn_readfirstlane(c.pieces);
    c.slot = __builtin_amdgcn_readfirstlane(c.slot);
    c.index = __builtin_amdgcn_readfirstlane(c.index);
    return c;
}

// ---- codes to halves -----------------------------------------------------------------------------------
// 0x6400 | u is 1024 + u in half precision, and u - 128 (a signed byte with its top bit turned over) is exact
__device__ __forceinline__ unsigned minus(unsigned v, float bias) { return bits_of(halves_of(v) - (h2){(_Float16)bias, (_Float16)bias}); }
__device__ __forceinline__ unsigned nibble_high(unsigned v) // 1024 + 16 u -> u - 8
{
    const h2 k = {(_Float16)0.0625f, (_Float16)0.0625f}, m = {(_Float16)-72.f, (_Float16)-72.f};
    return bits_of(__builtin_elementwise_fma(halves_of(v), k, m));
}

// 8 codes of one token as an operand: bytes in their order, nibbles in the order 0 4 1 5 2 6 3 7
template <int BITS> __device__ __forceinline__ h8 row_operand(unsigned w0, unsigned w1)
{
    if constexpr (BITS == 8) {
        constexpr unsigned HI = 0x64646464u, P01 = 0x04010400u, P23 = 0x04030402u;
        w0 ^= 0x80808080u;
        w1 ^= 0x80808080u;
        return operand(minus(__builtin_amdgcn_perm(HI, w0, P01), 1152.f), minus(__builtin_amdgcn_perm(HI, w0, P23), 1152.f),
                       minus(__builtin_amdgcn_perm(HI, w1, P01), 1152.f), minus(__builtin_amdgcn_perm(HI, w1, P23), 1152.f));
    } else {
        const unsigned u = w0 ^ 0x88888888u, d = u >> 8;
        return operand(minus((u & 0x000F000Fu) | 0x64006400u, 1032.f), nibble_high((u & 0x00F000F0u) | 0x64006400u),
                       minus((d & 0x000F000Fu) | 0x64006400u, 1032.f), nibble_high((d & 0x00F000F0u) | 0x64006400u));
    }
}
__device__ __forceinline__ int nibble_order(int e) { return e / 2 + 4 * (e % 2); } // element of place e

// Column m of two tokens' words as a pair of halves (BITS 8: byte m of 4; BITS 4: nibble m of 8)
template <int BITS> __device__ __forceinline__ unsigned column_pair(unsigned first, unsigned second, int m)
{
    if constexpr (BITS == 8) {
        const unsigned sel = 0x0c000c00u | (unsigned)(4 + m) << 16 | (unsigned)m;
        return minus(__builtin_amdgcn_perm(second, first, sel) ^ 0x64806480u, 1152.f);
    } else {
        const unsigned sel = 0x0c000c00u | (unsigned)(4 + m / 2) << 16 | (unsigned)(m / 2);
        const unsigned pair = __builtin_amdgcn_perm(second, first, sel);
        if (m % 2 == 0) return minus((pair & 0x000F000Fu) ^ 0x64086408u, 1032.f);
        return nibble_high((pair & 0x00F000F0u) ^ 0x64806480u);
    }
}

// ---- the pieces ----------------------------------------------------------------------------------------
template <int N> struct Words { unsigned w[N]; };
template <int N> __device__ __forceinline__ Words<N> load_words(const uint8_t *p)
{
    Words<N> v;
    if constexpr (N >= 4) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            const v4u u = reinterpret_cast<const v4u *>(p)[q];
#pragma unroll
            for (int e = 0; e < 4; ++e) v.w[4 * q + e] = u[e];
        }
    } else if constexpr (N == 2) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        v.w[0] = u.x;
        v.w[1] = u.y;
    } else {
        v.w[0] = *reinterpret_cast<const unsigned *>(p);
    }
    return v;
}

template <int TYPE> __device__ __forceinline__ float real_at(const void *p, int64_t i) { return (float)static_cast<const typename RealOf<TYPE>::type *>(p)[i]; }

// D: head dimension's tile (64, 128, 256).  Lane l: row l % 16 of the products with q, group g = l / 16 of the reduction.
// FULL: q in one half each and rounded weights, else (fp32) both in two halves.
template <int D, int BITS, int TYPE> __global__ __launch_bounds__(CACHE_WAVES * 64, 1) void cache_attention_kernel(CacheAttnArgs a)
{
    constexpr int PLANES = TYPE == MC_F32 ? 2 : 1;
    constexpr int C = D / 16;                        // columns of V in a lane
    constexpr int STEPS = D / 32;                    // of the first product
    constexpr int KB = D * BITS / 32, PB = KB < 16 ? KB : 16, NK = KB / PB;  // bytes of a row of K in a lane, in pieces
    constexpr int VW = C * BITS / 32;                // words of a row of V in a lane (D = 64, 4 bits: half a word)
    constexpr int VN = VW ? VW : 1;
    __shared__ float shared_o[CACHE_WAVES][16][D + 4];
    __shared__ float shared_m[CACHE_WAVES][16], shared_l[CACHE_WAVES][16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int head = blockIdx.y, row0 = blockIdx.z * 16;
    const Cut cut = cut_of<true>(a, blockIdx.x);
    if (cut.b < 0) return;
    const Sequence s = sequence(a, cut.b);
    const int n = __builtin_amdgcn_readfirstlane(s.n), length = __builtin_amdgcn_readfirstlane(s.length), start = __builtin_amdgcn_readfirstlane(s.start);
    if (row0 >= n * a.group) return;

    // this lane's row (rows beyond the last repeat it), and what it may see: all tokens below `all`, and those of the tree's bits from `held` on
    const int row = row0 + i < n * a.group ? row0 + i : n * a.group - 1, token = row / a.group, q_head = head * a.group + row % a.group;
    const int held = length - n;
    const int all = a.tree ? held : held + token + 1;
    const uint64_t bits = a.tree ? a.tree[start + token] & (n < 64 ? (1ull << n) - 1 : ~0ull) : 0;
    const int last_row = row0 + 15 < n * a.group ? row0 + 15 : n * a.group - 1;
    const int end = a.tree ? length : held + last_row / a.group + 1; // no row of this tile sees more
    const int certain = a.tree ? held : held + row0 / a.group + 1;   // every row sees this many

    // q, times a power of two that brings the row's largest into [1, 2)
    const void *q = a.q;
    const int64_t q_at = (start + (int64_t)token) * a.q_token_stride + q_head * a.q_head_stride;
    auto element = [&](int step, int e) { // the code that place e of step `step` meets
        return BITS == 8 ? (PB == 16 ? 64 * (step / 2) + 16 * g + 8 * (step % 2) + e : 0) : NK > 0 && PB == 16 ? 128 * (step / 4) + 32 * g + 8 * (step % 4) + nibble_order(e)
                                                                                                              : 16 * g + 8 * step + nibble_order(e);
    };
    float top = 0;
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = element(st, e);
            if (d < a.dk) top = fmaxf(top, fabsf(real_at<TYPE>(q, q_at + d)));
        }
    top = max_of_groups(top);
    int up = top > 0 && top < __builtin_inff() ? __builtin_amdgcn_frexp_expf(top) - 1 : 0;
    h8 qo[PLANES][STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = element(st, e);
            const float v = d < a.dk ? __builtin_amdgcn_ldexpf(real_at<TYPE>(q, q_at + d), -up) : 0.f;
            qo[0][st][e] = (_Float16)v;
            if (PLANES == 2) qo[PLANES - 1][st][e] = (_Float16)((v - (float)(_Float16)v) * 2048.f);
        }
    const float row_scale = __builtin_amdgcn_ldexpf(a.score_scale, up);

    const int row_bytes = a.dk * BITS / 8;
    const int v_at = (i * C < a.dk ? i * C : 0) * BITS / 8;
    int k_at[NK];
#pragma unroll
    for (int p = 0; p < NK; ++p) {
        const int at = 64 * p + g * PB;
        k_at[p] = i * row_bytes + (at < row_bytes - PB ? at : row_bytes - PB);
    }

    struct Tile {
        Words<PB / 4> k[2][NK];
        Words<VN> v[2][4];
        v4f ks[2], vs[2];
        bool there[2];
    };
    const int last_page = length > 0 ? (length - 1) >> a.page_shift : 0;
    auto load = [&](Tile &t, int tile) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int at = tile * CACHE_TILE + half * 16;
            const int nth = at >> a.page_shift < last_page ? at >> a.page_shift : last_page;
            int64_t page = length > 0 ? a.table[cut.b * a.table_stride + nth] : -1;
            t.there[half] = page >= 0 && page < a.pages;
            if (!t.there[half]) page = 0;
            const int64_t first = ((page * a.kv_heads + head) << a.page_shift) + (at & ((1 << a.page_shift) - 1));
            const uint8_t *k = a.k_codes + first * row_bytes, *v = a.v_codes + first * row_bytes;
#pragma unroll
            for (int p = 0; p < NK; ++p) t.k[half][p] = load_words<PB / 4>(k + k_at[p]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint8_t *from = v + (4 * g + r) * row_bytes + v_at;
                if constexpr (VW == 0) t.v[half][r].w[0] = *reinterpret_cast<const unsigned short *>(from);
                else t.v[half][r] = load_words<VN>(from);
            }
            t.ks[half] = *reinterpret_cast<const v4f *>(a.k_scales + first + 4 * g);
            t.vs[half] = *reinterpret_cast<const v4f *>(a.v_scales + first + 4 * g);
        }
    };

    float m = NONE, l = 0;
    v4f o[PLANES][C];
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
#pragma unroll
        for (int c = 0; c < C; ++c) o[p][c] = (v4f){0, 0, 0, 0};

    auto take = [&](const Tile &t, int tile) {
        // scores in base 2, plus the exponents of V's scales
        float x[2][4], f[2][4], w[2][4];
        int ex[2][4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            v4f sc[PLANES];
#pragma unroll
            for (int p = 0; p < PLANES; ++p) sc[p] = (v4f){0, 0, 0, 0};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                constexpr int PER = PB * 8 / BITS / 8; // steps of a piece
                const auto &piece = t.k[half][st / PER];
                const int at = st % PER;
                const h8 k = BITS == 8 ? row_operand<BITS>(piece.w[2 * at], piece.w[2 * at + 1]) : row_operand<BITS>(piece.w[at], 0u);
#pragma unroll
                for (int p = 0; p < PLANES; ++p) sc[p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qo[p][st], sc[p], 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float vs = t.vs[half][r];
                int e = __builtin_amdgcn_frexp_expf(vs);
                e = e < -100 ? -100 : e;
                ex[half][r] = e;
                f[half][r] = __builtin_amdgcn_ldexpf(vs, -e);
                const float sum = PLANES == 2 ? __builtin_fmaf(sc[PLANES - 1][r], 1.f / 2048, sc[0][r]) : sc[0][r];
                x[half][r] = __builtin_fmaf(sum * row_scale, t.ks[half][r], (float)e);
            }
        }
        const int at = tile * CACHE_TILE;
        const bool masked = at + CACHE_TILE > certain || !t.there[0] || !t.there[1];
        if (masked) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int token = at + 16 * half + 4 * g + r, later = token - held;
                    const bool seen = t.there[half] && token < length && (token < all || (later >= 0 && later < 64 && (bits >> later & 1)));
                    if (!seen) {
                        x[half][r] = NONE;
                        f[half][r] = 0;
                    }
                }
        }
        float top = NONE;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, x[half][r]);
        top = max_of_groups(top);
        if (__any(top > m)) {
            const float to = fmaxf(top, m), by = to == NONE ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= by;
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int c = 0; c < C; ++c) o[p][c] *= by;
        }
        const float from = (m == NONE ? 0.f : m) - UP;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = __builtin_amdgcn_exp2f(x[half][r] - from);
                l += __builtin_amdgcn_ldexpf(p, -ex[half][r]);
                w[half][r] = p * f[half][r];
            }
        h8 wo[PLANES];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = w[e / 4][e % 4];
            if (PLANES == 2) asm("" : "+v"(v)); // (one product, rounded once: the first half by a fused rounding, and the second from another would differ at a tie)
            wo[0][e] = (_Float16)v;
            if (PLANES == 2) wo[PLANES - 1][e] = (_Float16)((v - (float)(_Float16)v) * 2048.f);
        }
        constexpr int PER_WORD = 32 / BITS; // columns of a word
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int q = c / PER_WORD, in = c % PER_WORD;
            const h8 v = operand(column_pair<BITS>(t.v[0][0].w[q], t.v[0][1].w[q], in), column_pair<BITS>(t.v[0][2].w[q], t.v[0][3].w[q], in),
                                 column_pair<BITS>(t.v[1][0].w[q], t.v[1][1].w[q], in), column_pair<BITS>(t.v[1][2].w[q], t.v[1][3].w[q], in));
#pragma unroll
            for (int p = 0; p < PLANES; ++p) o[p][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, wo[p], o[p][c], 0, 0, 0);
        }
    };

    // the waves take the piece's tiles in turn
    const int64_t from_tile = (int64_t)cut.index * cut.each;
    const int tiles = end > 0 ? (end - 1) / CACHE_TILE + 1 : 0, to_tile = tiles - from_tile < cut.each ? tiles : (int)from_tile + cut.each;
    for (int64_t tile = from_tile + wave; tile < to_tile; tile += CACHE_WAVES) {
        Tile t;
        load(t, (int)tile);
        take(t, (int)tile);
    }

    // the waves' results meet in LDS
    l = sum_of_groups(l);
    if (g == 0) {
        shared_m[wave][i] = m;
        shared_l[wave][i] = l;
    }
    __syncthreads();
    float top_m = NONE;
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) top_m = fmaxf(top_m, shared_m[w][i]);
    const float by = m == NONE ? 0.f : __builtin_amdgcn_exp2f(m - top_m);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float v = PLANES == 2 ? __builtin_fmaf(o[PLANES - 1][c][r], 1.f / 2048, o[0][c][r]) : o[0][c][r];
            shared_o[wave][i][(4 * g + r) * C + c] = m == NONE ? 0.f : v * by;
        }
    __syncthreads();
    const int out_row = threadIdx.x / 16, col = threadIdx.x % 16 * C;
    float sum[C] = {}, all_m = NONE, all_l = 0;
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) all_m = fmaxf(all_m, shared_m[w][out_row]);
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) {
        if (shared_m[w][out_row] != NONE) all_l += shared_l[w][out_row] * __builtin_amdgcn_exp2f(shared_m[w][out_row] - all_m);
#pragma unroll
        for (int c = 0; c < C; ++c) sum[c] += shared_o[w][out_row][col + c];
    }
    if (cut.pieces > 1) {
        const int64_t at = (((int64_t)(cut.slot + cut.index) * a.kv_heads + head) * a.row_tiles + blockIdx.z) * 16 + out_row;
        float *to = a.partial + at * (D + 2);
        if (threadIdx.x % 16 == 0) {
            to[D] = all_m;
            to[D + 1] = all_l;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) to[col + c] = sum[c];
        return;
    }
    if (row0 + out_row >= n * a.group || col >= a.dk) return;
    const int out_token = (row0 + out_row) / a.group, out_head = head * a.group + (row0 + out_row) % a.group;
    const float inv = all_l == 0 ? 0.f : 1.f / all_l; // (a row that sees nothing is zero)
    auto *to = static_cast<typename RealOf<TYPE>::type *>(a.o) + (start + (int64_t)out_token) * a.o_token_stride + out_head * a.o_head_stride + col;
#pragma unroll
    for (int c = 0; c < C; ++c) to[c] = (typename RealOf<TYPE>::type)(sum[c] * inv);
}

// Pieces of a sequence that was cut, joined in their order: one workgroup per sequence, head and row tile.
template <int D, int TYPE> __global__ __launch_bounds__(256) void cache_attention_join_kernel(CacheAttnArgs a)
{
    constexpr int C = D / 16;
    const Cut cut = cut_of<false>(a, blockIdx.x);
    if (cut.pieces <= 1) return;
    const Sequence s = sequence(a, cut.b);
    const int out_row = threadIdx.x / 16, col = threadIdx.x % 16 * C, row = blockIdx.z * 16 + out_row;
    if (row >= s.n * a.group) return;
    const int64_t step = (int64_t)a.kv_heads * a.row_tiles * 16 * (D + 2);
    const float *from = a.partial + ((((int64_t)cut.slot * a.kv_heads + blockIdx.y) * a.row_tiles + blockIdx.z) * 16 + out_row) * (D + 2);
    float m = NONE, l = 0, sum[C] = {};
    for (int p = 0; p < cut.pieces; ++p) m = fmaxf(m, from[p * step + D]);
    for (int p = 0; p < cut.pieces; ++p) {
        const float mp = from[p * step + D];
        if (mp == NONE) continue;
        const float by = __builtin_amdgcn_exp2f(mp - m);
        l += from[p * step + D + 1] * by;
#pragma unroll
        for (int c = 0; c < C; ++c) sum[c] += from[p * step + col + c] * by;
    }
    if (col >= a.dk) return;
    const int token = row / a.group, head = blockIdx.y * a.group + row % a.group;
    const float inv = l == 0 ? 0.f : 1.f / l;
    auto *to = static_cast<typename RealOf<TYPE>::type *>(a.o) + (s.start + (int64_t)token) * a.o_token_stride + head * a.o_head_stride + col;
#pragma unroll
    for (int c = 0; c < C; ++c) to[c] = (typename RealOf<TYPE>::type)(sum[c] * inv);
}

template <int D, int BITS, int TYPE> hipError_t launch(const CacheAttnArgs &a, hipStream_t s)
{
    const unsigned pieces = (unsigned)(a.partial ? a.pieces + a.batch : a.batch);
    const hipError_t e = launch_kernel((cache_attention_kernel<D, BITS, TYPE>), dim3(pieces, a.kv_heads, a.row_tiles), dim3(CACHE_WAVES * 64), 0, s, a);
    if (e != hipSuccess || !a.partial) return e;
    return launch_kernel((cache_attention_join_kernel<D, TYPE>), dim3(a.batch, a.kv_heads, a.row_tiles), dim3(256), 0, s, a);
}

template <int BITS, int TYPE> hipError_t launch_dim(const CacheAttnArgs &a, hipStream_t s)
{
    if (a.dk <= 64) return launch<64, BITS, TYPE>(a, s);
    if (a.dk <= 128) return launch<128, BITS, TYPE>(a, s);
    return launch<256, BITS, TYPE>(a, s);
}

template <int BITS> hipError_t launch_type(const CacheAttnArgs &a, mc_type type, hipStream_t s)
{
    if (type == MC_F32) return launch_dim<BITS, MC_F32>(a, s);
    if (type == MC_F16) return launch_dim<BITS, MC_F16>(a, s);
    return launch_dim<BITS, MC_BF16>(a, s);
}

} // namespace

hipError_t launch_cache_attention(const CacheAttnArgs &a, mc_type type, int bits, hipStream_t s)
{
    return bits == 8 ? launch_type<8>(a, type, s) : launch_type<4>(a, type, s);
}
