// Attention of new tokens over a quantized cache: one token of each of many sequences, a chunk of a prompt, a tree of drafted tokens.
//   o_i = sum_t p_it s^v_t c^v_t / sum_t p_it,   p_it = exp(scale s^k_t (q_i . c^k_t) - max),   t over what row i may see.
// The rows of a tile are the new tokens' query heads that share a head of the cache.  A wave takes 32 tokens at a time, straight from memory into
// registers: S^T = K q^T, and with the probabilities where that product leaves them, o^T += V^T p^T (their places in a lane are the
// reduction's order of the second product, which V's rows follow).  Both products run on 16-bit floating MFMAs, in which codes are exact.
//
// Weights of the second product are sums of two halves of w = 2^(x - r) s^v, x the score in base 2 and r a reference of the row that follows the largest of x + e, e the
// exponent of s^v: so they are of the size of 1 for the terms that count, whatever the scales.  The reference stays while no w is beyond 2^15, and is moved, with l and
// o, so that the largest is about 2^7; a half keeps what is 2^-24 of 1.  l = sum 2^(x - r) in fp32.
//
// Sequences are cut into pieces of equal length, as many as fill the device: every workgroup works out its piece from the sequences' lengths,
// which the host does not know.  A piece that is not its whole sequence leaves (reference, l, o) to a second kernel.
// (Pieces of the same length through sequences' borders, each workgroup with parts of two, were slower: short parts, and registers for two sequences.)
#include "decode.h"

namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr float UP = 7.f, MOST = 15.f; // binary logarithm of a row's largest weight when its reference is moved, and when it has to be
constexpr float NONE = -__builtin_inff();

__device__ __forceinline__ unsigned bits_of(h2 v) { return __builtin_bit_cast(unsigned, v); }
__device__ __forceinline__ h2 halves_of(unsigned v) { return __builtin_bit_cast(h2, v); }
__device__ __forceinline__ h8 operand(unsigned a, unsigned b, unsigned c, unsigned d) { return __builtin_bit_cast(h8, (v4u){a, b, c, d}); }

// max / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48 (a swap of a value with itself leaves the two lanes' values in both)
__device__ __forceinline__ float max_of_groups(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_groups(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ float max_of(v4f v) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }

// ---- which piece ---------------------------------------------------------------------------------------
struct Sequence { int start, n, length, held; }; // first new token, new tokens, tokens in the cache with them and before them
__device__ __forceinline__ Sequence sequence(const CacheAttnArgs &a, int b)
{
    Sequence s;
    const int64_t most = (int64_t)a.table_pages << a.page_shift;
    const int length = a.lengths[b];
    s.length = length < 0 ? 0 : length > most ? (int)most : length;
    int fresh = a.max_new;
    s.start = b * a.max_new;
    if (a.starts) {
        s.start = a.starts[b];
        const int behind = a.starts[b + 1];
        fresh = s.start < 0 || behind <= s.start || behind > a.total_new ? 0 : behind - s.start;
    }
    s.n = fresh < a.max_new ? fresh : a.max_new; // (rows beyond are not computed)
    s.held = s.length - fresh;
    return s;
}
__device__ __forceinline__ int tiles_of(const Sequence &s) { return s.n == 0 ? 0 : s.length <= 0 ? 1 : (s.length - 1) / CACHE_TILE + 1; }

__device__ __forceinline__ int scan(int v) // inclusive, over the wave: within rows of 16 lanes, then their last lanes' sums into the rows behind
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true); // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false); // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false); // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ int at_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// A sequence (b), the tiles of its pieces, how many there are, the number of its first among the pieces of sequences that are cut, and the index of
// the piece asked for.
struct Cut { int b, each, pieces, slot, index; Sequence of; };
// The sequence that piece `number` belongs to (BY_PIECE), or sequence `number` itself; b = -1: none.
template <bool BY_PIECE> __device__ __forceinline__ Cut cut_of(const CacheAttnArgs &a, int number)
{
    const int lane = threadIdx.x & 63;
    const Sequence none = {0, 0, 0, 0};
    Sequence s = lane < a.batch ? sequence(a, lane) : none;
    int t = tiles_of(s), total = 0;
    if (a.partial) {
        total = at_lane(scan(t), 63);
        for (int b = 64; b < a.batch; b += 64) total += at_lane(scan(tiles_of(b + lane < a.batch ? sequence(a, b + lane) : none)), 63);
    }
    int each = a.partial ? cache_piece_tiles(total, a.pieces) : CACHE_WHOLE;
    if (a.partial && cache_pieces_lengthened(a.batch, a.pieces)) {
        for (int i = 0; i < CACHE_LENGTHENINGS; ++i) {
            const int n = at_lane(scan(cache_pieces_of(t, each)), 63);
            if (n <= a.pieces) break;
            each = cache_longer_piece(each, n, a.pieces);
        }
    }
    Cut c = {-1, 0, 0, 0, 0, none};
    int before = 0, slots = 0;
    for (int b = 0; b < a.batch; b += 64) {
        if (b) {
            s = b + lane < a.batch ? sequence(a, b + lane) : none;
            t = tiles_of(s);
        }
        const int pieces = cache_pieces_of(t, each), up_to = scan(pieces), cut_up_to = scan(pieces > 1 ? pieces : 0);
        const bool here = BY_PIECE ? before + up_to - pieces <= number && number < before + up_to : b + lane == number;
        const unsigned long long who = __ballot(here);
        if (who) {
            const int l = __builtin_ctzll(who);
            c.b = b + l;
            c.pieces = at_lane(pieces, l);
            c.each = cache_each_of(at_lane(t, l), c.pieces);
            c.slot = slots + at_lane(cut_up_to, l) - (c.pieces > 1 ? c.pieces : 0);
            c.index = number - before - at_lane(up_to, l) + c.pieces;
            c.of = {at_lane(s.start, l), at_lane(s.n, l), at_lane(s.length, l), at_lane(s.held, l)};
            break;
        }
        before += at_lane(up_to, 63);
        slots += at_lane(cut_up_to, 63);
    }
    return c;
}

// ---- codes to halves -----------------------------------------------------------------------------------
// Codes enter the matrix unit as half-precision numbers, in which they are exact.  0x6400 | u is 1024 + u, and a signed code with its top bit turned over
// is u - 128 (u - 8).  In the first product the subtraction is left out where the type allows it (RAW): a half with the bits u is the subnormal number u 2^-24 (16 u 2^-24
// a nibble higher up), and the offset is the same for all tokens: offset * sum of the row's q, once a row.  That costs the sums one or two bits of fp32.  (In the
// second product the offset would be of the size of all weights together, which long contexts exceed their mean by far.)
__device__ __forceinline__ unsigned minus(unsigned v, float bias) { return bits_of(halves_of(v) - (h2){(_Float16)bias, (_Float16)bias}); }
__device__ __forceinline__ unsigned nibble_high(unsigned v) // 1024 + 16 u -> u - 8
{
    const h2 k = {(_Float16)0.0625f, (_Float16)0.0625f}, m = {(_Float16)-72.f, (_Float16)-72.f};
    return bits_of(__builtin_elementwise_fma(halves_of(v), k, m));
}
constexpr float RAW_SCALE = 0x1p24f;
template <int BITS> constexpr float raw_offset() { return BITS == 8 ? 128.f : 8.f; }
// what an element of q at place e of an operand is divided by for RAW codes
template <int BITS> constexpr float raw_share(int e) { return BITS == 4 && e / 2 % 2 == 1 ? 0.0625f : 1.f; }

// 8 codes of one token as an operand: bytes in their order, nibbles in the order 0 4 1 5 2 6 3 7
template <int BITS, bool RAW> __device__ __forceinline__ h8 row_operand(unsigned w0, unsigned w1)
{
    if constexpr (BITS == 8) {
        constexpr unsigned HI = RAW ? 0u : 0x64646464u, P01 = RAW ? 0x0c010c00u : 0x04010400u, P23 = RAW ? 0x0c030c02u : 0x04030402u;
        w0 ^= 0x80808080u;
        w1 ^= 0x80808080u;
        const unsigned a = __builtin_amdgcn_perm(HI, w0, P01), b = __builtin_amdgcn_perm(HI, w0, P23), c = __builtin_amdgcn_perm(HI, w1, P01),
                       d = __builtin_amdgcn_perm(HI, w1, P23);
        if constexpr (RAW) return operand(a, b, c, d);
        return operand(minus(a, 1152.f), minus(b, 1152.f), minus(c, 1152.f), minus(d, 1152.f));
    } else {
        constexpr unsigned LO = RAW ? 0x00080008u : 0x64086408u, HI = RAW ? 0x00800080u : 0x64806480u;
        const unsigned d = w0 >> 8;
        const unsigned a = (w0 & 0x000F000Fu) ^ LO, b = (w0 & 0x00F000F0u) ^ HI, c = (d & 0x000F000Fu) ^ LO, e = (d & 0x00F000F0u) ^ HI;
        if constexpr (RAW) return operand(a, b, c, e);
        return operand(minus(a, 1032.f), nibble_high(b), minus(c, 1032.f), nibble_high(e));
    }
}
constexpr int nibble_order(int e) { return e / 2 + 4 * (e % 2); } // element of place e

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
// `at` bytes behind a base that is the same for the whole wave (STREAM: that nobody reads again)
template <int BYTES, bool STREAM = false> __device__ __forceinline__ Words<(BYTES + 3) / 4> load_bytes(const uint8_t *base, unsigned at)
{
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    auto get = [&](auto *p) { return STREAM ? __builtin_nontemporal_load(p) : *p; };
    Words<(BYTES + 3) / 4> v;
    if constexpr (BYTES >= 16) {
        static_assert(BYTES == 16, "one request");
        const v4u u = get(reinterpret_cast<const v4u *>(base + at));
#pragma unroll
        for (int e = 0; e < 4; ++e) v.w[e] = u[e];
    } else if constexpr (BYTES == 8) {
        const v2u u = get(reinterpret_cast<const v2u *>(base + at));
        v.w[0] = u.x;
        v.w[1] = u.y;
    } else if constexpr (BYTES == 4) {
        v.w[0] = get(reinterpret_cast<const unsigned *>(base + at));
    } else {
        v.w[0] = get(reinterpret_cast<const unsigned short *>(base + at));
    }
    return v;
}

// 8 values of a row of q, and N results of a row of o (16-byte pieces, or 8 bytes)
template <int TYPE> __device__ __forceinline__ void load_real8(const void *p, int64_t at, float (&v)[8])
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int N = 16 / sizeof(T);
    typedef T Vec __attribute__((ext_vector_type(N)));
#pragma unroll
    for (int q = 0; q < 8 / N; ++q) {
        const Vec u = *reinterpret_cast<const Vec *>(static_cast<const T *>(p) + at + q * N);
#pragma unroll
        for (int e = 0; e < N; ++e) v[q * N + e] = (float)u[e];
    }
}
template <int TYPE, int N> __device__ __forceinline__ void store_real(void *p, int64_t at, const float *v)
{
    typedef typename RealOf<TYPE>::type T;
    constexpr int M = N * sizeof(T) < 16 ? N : 16 / sizeof(T);
    typedef T Vec __attribute__((ext_vector_type(M)));
#pragma unroll
    for (int q = 0; q < N / M; ++q) {
        Vec u;
#pragma unroll
        for (int e = 0; e < M; ++e) u[e] = (T)v[q * M + e];
        *reinterpret_cast<Vec *>(static_cast<T *>(p) + at + q * M) = u;
    }
}

// Where a row of results goes: row `row` (new token, query head of the group) of a sequence
__device__ __forceinline__ int64_t out_at(const CacheAttnArgs &a, const Sequence &s, int head, int row)
{
    return (s.start + (int64_t)(row / a.group)) * a.o_token_stride + (int64_t)(head * a.group + row % a.group) * a.o_head_stride;
}

// Sizes that follow from D (the head dimension's tile: 64, 128 or 256), the width of codes and the type.  Lane l of a wave: row i = l % 16 of a tile of rows in
// the products with q, group g = l / 16 of the reduction.
template <int D, int BITS, int TYPE> struct Shape {
    static constexpr int PLANES = TYPE == MC_F32 ? 2 : 1;  // halves that hold a value of q
    // Halves that hold a weight, for every type.  With one, results in fp16 were 1.4 - 1.55 times as far from the formula's as rounded ones are, and every eighth of those in bf16 was
    // not the rounded one (values that cancel lost up to 2^-12 of what they are summed from).
    static constexpr int PARTS = 2;
    static constexpr bool RAW = TYPE != MC_F32;           // K's codes enter with their offset
    static constexpr int C = D / 16;                      // columns of V in a lane
    static constexpr int STEPS = D / 32;                  // of the first product
    static constexpr int KB = D * BITS / 32, PB = KB < 16 ? KB : 16, NK = KB / PB, PER = PB / BITS; // bytes of a row of K in a lane, in pieces of PER steps
    static constexpr int VB = C * BITS / 8;               // bytes of a row of V in a lane
    // the first of the 8 elements that a lane's codes of a step are
    static __device__ __forceinline__ int element(int step, int g)
    {
        return BITS == 8 ? 64 * (step / 2) + 16 * g + 8 * (step % 2) : PB == 16 ? 128 * (step / 4) + 32 * g + 8 * (step % 4) : 16 * g + 8 * step;
    }
};

// A lane's row of q as operands of the first product, times a power of two that brings the row's largest into [2^14, 2^15), so that halves hold what is 2^-28 of it to their full
// width (a nibble higher up: 2^-24); a score is sum * scale + offset then
struct RowScale { float scale, offset; };
template <class S, int BITS, int TYPE> __device__ __forceinline__ RowScale load_q(const CacheAttnArgs &a, int64_t at, int g, h8 (&q)[S::PLANES][S::STEPS])
{
    float v[S::STEPS][8], top = 0;
#pragma unroll
    for (int st = 0; st < S::STEPS; ++st) {
        const int d = S::element(st, g);
        if (d < a.dk) load_real8<TYPE>(a.q, at + d, v[st]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[st][e] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[st][e]));
    }
    top = max_of_groups(top);
    const int up = top > 0 && top < __builtin_inff() ? __builtin_amdgcn_frexp_expf(top) - 15 : 0;
    float sum = 0;
#pragma unroll
    for (int st = 0; st < S::STEPS; ++st)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __builtin_amdgcn_ldexpf(v[st][BITS == 8 ? e : nibble_order(e)], -up) * (S::RAW ? raw_share<BITS>(e) : 1.f);
            q[0][st][e] = (_Float16)x;
            if (S::PLANES == 2) q[S::PLANES - 1][st][e] = (_Float16)(x - (float)(_Float16)x);
            if (S::RAW) sum += (float)q[0][st][e] / raw_share<BITS>(e); // (what the products are made with)
        }
    const float scale = __builtin_amdgcn_ldexpf(a.score_scale, up);
    if (!S::RAW) return {scale, 0.f};
    return {scale * RAW_SCALE, -scale * raw_offset<BITS>() * sum_of_groups(sum)};
}

// What a row may see: all tokens below `all`, and those of the bits from `held` on
struct Sight { int all; uint64_t bits; };
__device__ __forceinline__ Sight sight_of(const CacheAttnArgs &a, const Sequence &s, int token)
{
    if (!a.tree) return {s.held + token + 1, 0};
    const int fresh = s.length - s.held;
    return {s.held, a.tree[s.start + token] & (fresh < 64 ? (1ull << fresh) - 1 : ~0ull)};
}
// (no branches: as such the compiler lost some of the -infinities between them)
__device__ __forceinline__ unsigned sees(const Sight &s, int token, int held, bool there)
{
    const int later = token - held;
    const unsigned bit = (unsigned)(s.bits >> (later & 63)) & (unsigned)((unsigned)later < 64u);
    return (unsigned)there & ((unsigned)(token < s.all) | bit) & 1u;
}

// Offsets of this lane's pieces of a row of K, row i of 16, and of its part of a row of V
template <class S> __device__ __forceinline__ unsigned k_offset(int p, int i, int g, int row_bytes)
{
    const int at = 64 * p + g * S::PB;
    return i * row_bytes + (at < row_bytes - S::PB ? at : row_bytes - S::PB); // (what is beyond a row meets zeros of q)
}
template <class S> __device__ __forceinline__ unsigned v_offset(int i, int dk) { return i * S::C < dk ? i * S::VB : 0; }

// The page of the 16 tokens from `at` on (-1: none), and their place in the cache in vectors (where a page is none, some place)
__device__ __forceinline__ int page_at(const CacheAttnArgs &a, const int32_t *table, int last_page, int at)
{
    const int nth = at >> a.page_shift;
    return __builtin_amdgcn_readfirstlane(nth <= last_page ? table[nth] : -1);
}
__device__ __forceinline__ bool is_page(const CacheAttnArgs &a, int page) { return (unsigned)page < (unsigned)a.pages; } // (at most 2^31 of them)
__device__ __forceinline__ int64_t place_of(const CacheAttnArgs &a, int page, int head, int at)
{
    return (int64_t)((uint64_t)(is_page(a, page) ? (unsigned)page : 0u) * a.page_vectors + ((unsigned)head << a.page_shift) + ((unsigned)at & ((1u << a.page_shift) - 1)));
}

// The exponent of a scale: |scale| is below 2^exponent; at least -80, so that 2^(x - r) is at most 2^95 and 2^30 tokens' sum of it a number of fp32.  Zero has that lowest
// exponent, too: a value of zeros counts in l and must not raise the reference above the weights that are there.
__device__ __forceinline__ float exponent_of(float scale)
{
    return (float)__builtin_amdgcn_frexp_expf(fmaxf(fabsf(scale), 0x1p-81f));
}

// Two weights as sums of two halves each: what a half holds, cut off and not rounded, and the rest, which is exact in fp32 and whose half leaves 2^-22.  (Both are
// rounded to steps of 2^-24 where they are small: 2^-25 in the end, 2^-32 of a row's largest.)
__device__ __forceinline__ void put_parts(h8 (&w)[2], int e, float v0, float v1)
{
    const h2 first = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(v0, v1));
    w[0][e] = first[0];
    w[0][e + 1] = first[1];
    w[1][e] = (_Float16)__builtin_fmaf((float)first[0], -1.f, v0);
    w[1][e + 1] = (_Float16)__builtin_fmaf((float)first[1], -1.f, v1);
}

// A row's reference and sums
template <int C> struct Row {
    float m, l; // m: the reference, and 7 (NONE: nothing seen)
    v4f o[C];
    __device__ __forceinline__ float to_add() const { return m == NONE ? 0.f : UP - m; } // what scores become x - r by
    __device__ __forceinline__ void clear()
    {
        m = NONE;
        l = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = (v4f){0, 0, 0, 0};
    }
    // top: logarithm of the largest weight of some scores x - r, the same in the four lanes of a row.  Whether references move (of any row of the wave); by: what
    // these scores are less then
    __device__ __forceinline__ bool move(float top, float &by)
    {
        const bool must = top > MOST || (m == NONE && top > NONE);
        if (!__any(must)) return false;
        by = must ? top - UP : 0.f;
        const float factor = m == NONE ? 1.f : __builtin_amdgcn_exp2f(-by);
        m = must ? (m == NONE ? UP : m) + by : m;
        l *= factor;
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] *= factor;
        return true;
    }
};

// Which piece, head and rows a workgroup has.  Tiles of rows of the same piece and head follow each other on one XCD (workgroups go round the eight of
// them).
struct Unit { int piece, head, rows_at; };
__device__ __forceinline__ Unit unit_of(const CacheAttnArgs &a, int row_tile)
{
    int unit = blockIdx.x, tile = 0;
    if (a.row_tiles > 1) {
        const int turn = blockIdx.x / (8 * a.row_tiles), in = blockIdx.x - turn * 8 * a.row_tiles;
        tile = in / 8;
        unit = turn * 8 + in % 8;
    }
    const int piece = unit / a.kv_heads; // (numbers without a piece come last, so that no XCD has more of them than another)
    return {piece, unit - piece * a.kv_heads, tile * row_tile};
}

// C results of a row from column col on: to the output, or to a piece's place
template <int D, int TYPE, int C> __device__ __forceinline__ void put(const CacheAttnArgs &a, const Cut &cut, int head, int row, int col, float (&v)[C], float m, float l)
{
    if (cut.pieces > 1) {
        const int64_t line = ((int64_t)(cut.slot + cut.index) * a.kv_heads + head) * a.rows_held + row;
        store_real<MC_F32, C>(a.partial, line * D + col, v);
        if (col == 0) *reinterpret_cast<float2 *>(a.sums + line * 2) = make_float2(m, l);
    } else if (col < a.dk) {
        const float inv = l == 0 ? 0.f : 1.f / l; // (a row that sees nothing is zero)
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] *= inv;
        store_real<TYPE, C>(a.o, out_at(a, cut.of, head, row) + col, v);
    }
}

// Up to 16 rows: the waves of a workgroup take a piece's tiles of 32 tokens in turn, from memory through registers alone.
// Memory bounds it where there is much to read: 2216 MB (64 sequences of 16384, 8 heads of 128, 8 bits) in 341 us, 6.5 TB/s of 6.9 that reading alone reaches; with ordinary
// instead of streaming loads 375.  In 4 bits and fp16 (285 MB, two sequences of 131072) 59 us, 4.8 TB/s: there are twice as many conversions to a byte.  Unequal sequences (190 MB) take
// 44 us: 3 us until lengths and first pages are there, and workgroups of unequal work at the end.  Tried without gain: tiles three ahead, page ids a wave holds in its lanes, three waves
// of longer tiles, wave priorities.
template <int D, int BITS, int TYPE> __global__ __launch_bounds__(CACHE_WAVES * 64, D <= 128 ? 2 : 1) void cache_attention_kernel(CacheAttnArgs a)
{
    typedef Shape<D, BITS, TYPE> S;
    constexpr int PLANES = S::PLANES, PARTS = S::PARTS, C = S::C, PB = S::PB;
    __shared__ float shared_o[CACHE_WAVES][16][D + 4];
    __shared__ float shared_m[CACHE_WAVES][16], shared_l[CACHE_WAVES][16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const Unit unit = unit_of(a, 16);
    if (unit.piece >= a.units_per_head) return;
    const Cut cut = cut_of<true>(a, unit.piece);
    if (cut.b < 0) return;
    const Sequence s = cut.of;
    const int rows = s.n * a.group, head = unit.head, row0 = unit.rows_at;
    if (row0 >= rows) return;
    const int held = s.held;

    const int row = row0 + i < rows ? row0 + i : rows - 1; // (rows beyond the last repeat it)
    const Sight sight = sight_of(a, s, row / a.group);
    h8 q[PLANES][S::STEPS];
    const RowScale row_scale = load_q<S, BITS, TYPE>(a, (s.start + (int64_t)(row / a.group)) * a.q_token_stride + (int64_t)(head * a.group + row % a.group) * a.q_head_stride, g, q);
    const int last_row = row0 + 15 < rows ? row0 + 15 : rows - 1;
    const int end = a.tree ? s.length : held + last_row / a.group + 1; // no row sees more
    const int certain = a.tree ? held : held + row0 / a.group + 1;     // every row sees this many

    const int row_bytes = a.dk * BITS / 8;
    unsigned k_at[S::NK], v_at[4];
#pragma unroll
    for (int p = 0; p < S::NK; ++p) k_at[p] = k_offset<S>(p, i, g, row_bytes);
#pragma unroll
    for (int r = 0; r < 4; ++r) v_at[r] = (4 * g + r) * row_bytes + v_offset<S>(i, a.dk);

    struct Pages { int id[2]; };
    const int last_page = s.length > 0 ? (s.length - 1) >> a.page_shift : -1;
    const int32_t *table = a.table + cut.b * a.table_stride;
    auto pages_of = [&](int tile) {
        Pages p;
        p.id[0] = p.id[1] = page_at(a, table, last_page, tile * CACHE_TILE);
        if (a.page_shift < 5) p.id[1] = page_at(a, table, last_page, tile * CACHE_TILE + 16);
        return p;
    };
    struct Tile {
        Words<PB / 4> k[2][S::NK];
        Words<(S::VB + 3) / 4> v[2][4];
        v4f ks[2], vs[2];
        bool there[2];
    };
    auto load = [&](Tile &t, int tile, Pages pages) {
        const int64_t place = place_of(a, pages.id[0], head, tile * CACHE_TILE);
        int64_t other = place + 16;
        if (a.page_shift < 5) other = place_of(a, pages.id[1], head, tile * CACHE_TILE + 16);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            t.there[half] = is_page(a, pages.id[half]);
            const int64_t first = half ? other : place;
            const uint8_t *k = a.k_codes + first * row_bytes, *v = a.v_codes + first * row_bytes;
#pragma unroll
            for (int p = 0; p < S::NK; ++p) t.k[half][p] = load_bytes<PB, true>(k, k_at[p]);
#pragma unroll
            for (int r = 0; r < 4; ++r) t.v[half][r] = load_bytes<S::VB, true>(v, v_at[r]);
            t.ks[half] = *reinterpret_cast<const v4f *>(a.k_scales + first + 4 * g);
            t.vs[half] = *reinterpret_cast<const v4f *>(a.v_scales + first + 4 * g);
        }
    };

    Row<C> sums;
    sums.clear();

    auto take = [&](Tile &tile, int number) {
        v4f sc[2];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int st = 0; st < S::STEPS; ++st) {
                const auto &piece = tile.k[half][st / S::PER];
                const int at = st % S::PER;
                const h8 k = BITS == 8 ? row_operand<BITS, S::RAW>(piece.w[2 * at % (PB / 4)], piece.w[(2 * at + 1) % (PB / 4)]) : row_operand<BITS, S::RAW>(piece.w[at], 0u);
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
                    sc[half] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[p][st], st == 0 && p == 0 ? (v4f){0, 0, 0, 0} : sc[half], 0, 0, 0);
            }
        const int at = number * CACHE_TILE;
        const bool masked = at + CACHE_TILE > certain || !tile.there[0] || !tile.there[1];
        float vs[8];
        unsigned seen = 0xff;
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] = tile.vs[e / 4][e % 4];
        if (masked) {
            seen = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned yes = sees(sight, at + 16 * (e / 4) + 4 * g + e % 4, held, tile.there[e / 4]);
                seen |= yes << e;
                vs[e] = yes ? vs[e] : 0.f; // (whatever there is)
            }
        }
        float x[8];
        const float to_add = sums.to_add();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float score = S::RAW ? __builtin_fmaf(sc[e / 4][e % 4], row_scale.scale, row_scale.offset) : sc[e / 4][e % 4] * row_scale.scale;
            const float ks = tile.ks[e / 4][e % 4];
            x[e] = __builtin_fmaf(score, ks, __builtin_fmaf(ks, 0.f, to_add)); // (NaN, and not -infinity, where a scale is infinite)
        }
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = seen >> e & 1 ? x[e] : NONE;
        }
        // The largest weight: by each token's exponent (fp32), or by that of the largest scale of a lane's eight.
        float top, most = fabsf(vs[0]);
        if (PLANES == 2) {
            top = x[0] + exponent_of(vs[0]);
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e] + exponent_of(vs[e]));
        } else {
            top = x[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) {
                top = fmaxf(top, x[e]);
                most = fmaxf(most, fabsf(vs[e]));
            }
            top += exponent_of(most);
        }
        float by;
        if (sums.move(max_of_groups(top), by)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] -= by;
        }
        h8 w[PARTS];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(x[e]), p1 = __builtin_amdgcn_exp2f(x[e + 1]);
            sums.l += p0;
            sums.l += p1;
            put_parts(w, e, p0 * vs[e], p1 * vs[e + 1]);
        }
        constexpr int PER_WORD = 32 / BITS; // columns of a word
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int n = c / PER_WORD, in = c % PER_WORD;
            const h8 v = operand(column_pair<BITS>(tile.v[0][0].w[n], tile.v[0][1].w[n], in), column_pair<BITS>(tile.v[0][2].w[n], tile.v[0][3].w[n], in),
                                 column_pair<BITS>(tile.v[1][0].w[n], tile.v[1][1].w[n], in), column_pair<BITS>(tile.v[1][2].w[n], tile.v[1][3].w[n], in));
#pragma unroll
            for (int p = 0; p < PARTS; ++p) sums.o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[p], sums.o[c], 0, 0, 0);
        }
    };

    // A tile is asked for while the one before is worked on, and its pages one tile earlier.
    const int64_t from_tile = (int64_t)cut.index * cut.each;
    const int tiles = end > 0 ? (end - 1) / CACHE_TILE + 1 : 0, to_tile = tiles - from_tile < cut.each ? tiles : (int)from_tile + cut.each;
    int tile = (int)from_tile + wave;
    if (from_tile + wave < to_tile) {
        constexpr int STEP = CACHE_WAVES;
        Tile one, two;
        load(one, tile, pages_of(tile));
        Pages next = pages_of(tile + STEP);
        for (;;) {
            if (tile + STEP < to_tile) load(two, tile + STEP, next);
            next = pages_of(tile + 2 * STEP);
            take(one, tile);
            tile += STEP;
            if (tile >= to_tile) break;
            if (tile + STEP < to_tile) load(one, tile + STEP, next);
            next = pages_of(tile + 2 * STEP);
            take(two, tile);
            tile += STEP;
            if (tile >= to_tile) break;
        }
    }

    // the waves' results meet in LDS
    const float sum_l = sum_of_groups(sums.l);
    if (g == 0) {
        shared_m[wave][i] = sums.m;
        shared_l[wave][i] = sum_l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < C; c += 4)
            *reinterpret_cast<v4f *>(&shared_o[wave][i][(4 * g + r) * C + c]) = (v4f){sums.o[c][r], sums.o[c + 1][r], sums.o[c + 2][r], sums.o[c + 3][r]};
    __syncthreads();
    const int of = threadIdx.x / 16, col = threadIdx.x % 16 * C;
    float sum[C] = {}, all_m = NONE, all_l = 0;
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) all_m = fmaxf(all_m, shared_m[w][of]);
#pragma unroll
    for (int w = 0; w < CACHE_WAVES; ++w) {
        const float by = all_m == NONE ? 1.f : __builtin_amdgcn_exp2f(shared_m[w][of] - all_m);
        all_l += shared_l[w][of] * by;
#pragma unroll
        for (int c = 0; c < C; ++c) sum[c] += shared_o[w][of][col + c] * by;
    }
    if (row0 + of < rows) put<D, TYPE, C>(a, cut, head, row0 + of, col, sum, all_m, all_l);
}

// More rows: each wave has R tiles of 16 rows, and the workgroup converts a piece's tokens, 64 at a time (32 for D = 256), once for all of them.  The operands lie in LDS as
// the MFMAs take them, 16 bytes a lane side by side, two tiles of tokens in turn; beside them their scales.
// What bounds it is the issue of what is not a matrix product: 4 sequences of 512 new tokens over 4096, 32 heads of 128, bf16, 133 Gflop in 250 us (530 Tflop/s; a library's bf16 product of 8192^3 reaches
// 1200), the vector unit busy 50 % of the cycles and the matrix unit 31 %, a third of it with the weights' second halves (one half: 205 us), LDS conflicts 3 %.  A wave and tile (R = 2) counts 96 matrix and
// 446 other vector instructions: in the loop 82 convert, 74 make scores, 46 find the largest weight, 144, 32 of them exponentials at a quarter of the rate, make weights, and 47 are
// maxima over lanes, pages and scales; the others, 53 to each of a wave's 31 tiles, are masks, moved references, and what is before and behind the loop (the piece, q's operands, results).  Two
// registers of the instance spill, 12 bytes a lane.
// In fp16 251 us, fp32 295, 4 bits 238 (fp32 275), dk 64 182, dk 192 and 256 793 (one wave a SIMD, and a tile of 256 columns for both).  Before any of this, codes that each wave converted for itself took 595 us.
// Tried without gain: weights made first and the largest sought only where they do not fit (registers spill: 527 - 710 us), wave priorities, 32 tokens at a time.
template <int D, int BITS, int TYPE, int R> __global__ __launch_bounds__(CACHE_WAVES * 64, D <= 128 ? 2 : 1) void cache_attention_rows_kernel(CacheAttnArgs a)
{
    typedef Shape<D, BITS, TYPE> S;
    constexpr int PLANES = S::PLANES, PARTS = S::PARTS, C = S::C, PB = S::PB, STEPS = S::STEPS;
    constexpr int T = D <= 128 ? 64 : 32, BLOCKS = T / 16, PAIRS = T / 32;  // tokens of a tile, in blocks of 16 and 32
    constexpr int SHARE = CACHE_WAVES / BLOCKS, KU = S::NK / SHARE, VB = S::VB / SHARE, VC = C / SHARE; // waves that convert 16 tokens, each some pieces of K and columns of V
    static_assert(KU * SHARE == S::NK && VC * SHARE == C, "even shares");
    struct alignas(16) Stage {
        uint8_t k[BLOCKS * STEPS * 1024], v[PAIRS * C * 1024];
        float k_scale[T], v_scale[T], exponent[T / 4]; // (of the largest of four tokens' scales of V)
        uint8_t there[4];                              // whether a block's page is one
    };
    __shared__ Stage stages[2];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const Unit unit = unit_of(a, CACHE_WAVES * 16 * R);
    if (unit.piece >= a.units_per_head) return;
    const Cut cut = cut_of<true>(a, unit.piece);
    if (cut.b < 0) return;
    const Sequence s = cut.of;
    const int rows = s.n * a.group, head = unit.head;
    if (unit.rows_at >= rows) return;
    const int held = s.held;
    const int group_last = unit.rows_at + CACHE_WAVES * 16 * R - 1 < rows ? unit.rows_at + CACHE_WAVES * 16 * R - 1 : rows - 1;
    const int end = a.tree ? s.length : held + group_last / a.group + 1;   // no row of the workgroup sees more
    // this wave's rows (none: it converts for the others), the first token that none of them sees, and the first that not every one sees
    const int row0 = unit.rows_at + wave * 16 * R, wave_last = row0 + 16 * R - 1 < rows ? row0 + 16 * R - 1 : rows - 1;
    const int wave_end = row0 >= rows ? 0 : a.tree ? s.length : held + wave_last / a.group + 1;
    const int certain = a.tree ? held : held + row0 / a.group + 1;

    int token[R]; // of this lane's rows
    RowScale row_scale[R];
    h8 q[R][PLANES][STEPS];
    Row<C> sums[R];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int row = row0 + 16 * t + i < rows ? row0 + 16 * t + i : rows - 1; // (rows beyond the last repeat it)
        token[t] = row / a.group;
        row_scale[t] = load_q<S, BITS, TYPE>(a, (s.start + (int64_t)token[t]) * a.q_token_stride + (int64_t)(head * a.group + row % a.group) * a.q_head_stride, g, q[t]);
        sums[t].clear();
    }

    // What this wave converts: of a tile's tokens 16 (one page), and their scales, of K in lanes 0 .. 15 and of V in the next 16.  The page is asked for a tile's
    // turn ahead.
    const int row_bytes = a.dk * BITS / 8, block = wave / SHARE, share = wave % SHARE;
    unsigned k_at[KU];
#pragma unroll
    for (int u = 0; u < KU; ++u) k_at[u] = k_offset<S>(share * KU + u, i, g, row_bytes);
    const unsigned v_at = 4 * g * row_bytes + (i * C + share * VC < a.dk ? i * S::VB + share * VB : 0);
    const int last_page = s.length > 0 ? (s.length - 1) >> a.page_shift : -1;
    const int32_t *table = a.table + cut.b * a.table_stride;
    auto ask_page = [&](int at) { // (a load by lanes: as a scalar one it would hold up the waits for LDS, which share its counter)
        const int nth = (at + 16 * block) >> a.page_shift;
        return nth <= last_page ? table[nth + (lane & 0)] : -1;
    };
    struct Codes {
        Words<PB / 4> k[KU];
        Words<(VB + 3) / 4> v[4];
        float k_scale, v_scale;
        bool there;
    };
    auto load = [&](Codes &t, int at, int page) {
        page = __builtin_amdgcn_readfirstlane(page);
        t.there = is_page(a, page);
        const int64_t first = place_of(a, page, head, at + 16 * block);
        const uint8_t *k = a.k_codes + first * row_bytes, *v = a.v_codes + first * row_bytes;
#pragma unroll
        for (int u = 0; u < KU; ++u) t.k[u] = load_bytes<PB>(k, k_at[u]);
#pragma unroll
        for (int r = 0; r < 4; ++r) t.v[r] = load_bytes<VB>(v + r * row_bytes, v_at);
        t.k_scale = a.k_scales[first + i];
        t.v_scale = a.v_scales[first + i];
    };
    auto convert = [&](Codes &t, Stage &to) {
#pragma unroll
        for (int u = 0; u < KU; ++u)
#pragma unroll
            for (int e = 0; e < S::PER; ++e)
                *reinterpret_cast<h8 *>(&to.k[(block * STEPS + (share * KU + u) * S::PER + e) * 1024 + lane * 16]) =
                    BITS == 8 ? row_operand<BITS, S::RAW>(t.k[u].w[2 * e % (PB / 4)], t.k[u].w[(2 * e + 1) % (PB / 4)]) : row_operand<BITS, S::RAW>(t.k[u].w[e], 0u);
        constexpr int PER_WORD = 32 / BITS;
#pragma unroll
        for (int c = 0; c < VC; ++c) {
            const int n = c / PER_WORD, in = c % PER_WORD;
            *reinterpret_cast<uint2 *>(&to.v[(block / 2 * C + share * VC + c) * 1024 + lane * 16 + block % 2 * 8]) =
                make_uint2(column_pair<BITS>(t.v[0].w[n], t.v[1].w[n], in), column_pair<BITS>(t.v[2].w[n], t.v[3].w[n], in));
        }
        if (share == 0) {
            // scales that are not finite, V's too, go into the scores as NaN, from where they reach the rows that see the token and no other
            const bool finite = fabsf(t.v_scale) < __builtin_inff();
            const float v = finite ? t.v_scale : 0.f;
            float most = fabsf(v);
            most = fmaxf(most, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, most), 0xB1, 0xF, 0xF, true))); // quad_perm 1 0 3 2
            most = fmaxf(most, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, most), 0x4E, 0xF, 0xF, true))); // quad_perm 2 3 0 1
            if (g == 0) {
                to.k_scale[16 * block + i] = finite && fabsf(t.k_scale) < __builtin_inff() ? t.k_scale : __builtin_nanf("");
                to.v_scale[16 * block + i] = v;
                to.exponent[4 * block + i / 4] = exponent_of(most);
                to.there[block] = (uint8_t)t.there;
            }
        }
    };

    auto take = [&](const Stage &st, int at) {
        const unsigned there = *reinterpret_cast<const unsigned *>(st.there), all_there = BLOCKS == 4 ? 0x01010101u : 0x0101u;
        v4f sc[R][BLOCKS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) { // (sums that follow each other are of other blocks)
                const h8 op = *reinterpret_cast<const h8 *>(&st.k[(b * STEPS + k) * 1024 + lane * 16]);
#pragma unroll
                for (int t = 0; t < R; ++t)
#pragma unroll
                    for (int p = 0; p < PLANES; ++p)
                        sc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op, q[t][p][k], k == 0 && p == 0 ? (v4f){0, 0, 0, 0} : sc[t][b], 0, 0, 0);
            }
        float to_add[R];
#pragma unroll
        for (int t = 0; t < R; ++t) to_add[t] = sums[t].to_add();
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const v4f ks = *reinterpret_cast<const v4f *>(&st.k_scale[16 * b + 4 * g]);
#pragma unroll
            for (int t = 0; t < R; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float score = S::RAW ? __builtin_fmaf(sc[t][b][r], row_scale[t].scale, row_scale[t].offset) : sc[t][b][r] * row_scale[t].scale;
                    sc[t][b][r] = __builtin_fmaf(score, ks[r], to_add[t]);
                }
        }
        // the largest weight: by the exponent of four tokens, or of each where not all of them are seen
        float top[R];
#pragma unroll
        for (int t = 0; t < R; ++t) top[t] = NONE;
        if (at + T > certain || (__builtin_amdgcn_readfirstlane(there) & all_there) != all_there) {
            Sight sight[R];
#pragma unroll
            for (int t = 0; t < R; ++t) sight[t] = sight_of(a, s, token[t]);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const v4f vs = *reinterpret_cast<const v4f *>(&st.v_scale[16 * b + 4 * g]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float ex = exponent_of(vs[r]);
#pragma unroll
                    for (int t = 0; t < R; ++t) {
                        sc[t][b][r] = sees(sight[t], at + 16 * b + 4 * g + r, held, there >> 8 * b & 1) ? sc[t][b][r] : NONE;
                        top[t] = fmaxf(top[t], sc[t][b][r] + ex);
                    }
                }
            }
        } else {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const float ex = st.exponent[4 * b + g];
#pragma unroll
                for (int t = 0; t < R; ++t) top[t] = fmaxf(top[t], max_of(sc[t][b]) + ex);
            }
        }
#pragma unroll
        for (int t = 0; t < R; ++t) {
            float by;
            if (sums[t].move(max_of_groups(top[t]), by)) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) sc[t][b] -= by;
            }
        }
#pragma unroll
        for (int pair = 0; pair < PAIRS; ++pair) {
            h8 w[R][PARTS];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int b = 2 * pair + half;
                const v4f vs = *reinterpret_cast<const v4f *>(&st.v_scale[16 * b + 4 * g]);
#pragma unroll
                for (int t = 0; t < R; ++t)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const float p0 = __builtin_amdgcn_exp2f(sc[t][b][r]), p1 = __builtin_amdgcn_exp2f(sc[t][b][r + 1]);
                        sums[t].l += p0;
                        sums[t].l += p1;
                        put_parts(w[t], 4 * half + r, p0 * vs[r], p1 * vs[r + 1]);
                    }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const h8 v = *reinterpret_cast<const h8 *>(&st.v[(pair * C + c) * 1024 + lane * 16]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int t = 0; t < R; ++t) sums[t].o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[t][p], sums[t].o[c], 0, 0, 0);
            }
        }
    };

    const int64_t from = (int64_t)cut.index * cut.each * CACHE_TILE, most = from + (int64_t)cut.each * CACHE_TILE;
    const int to = end < most ? end : (int)most;
    if (from < to) {
        Codes codes;
        int at = (int)from;
        int page = ask_page(at + T);
        load(codes, at, ask_page(at));
        convert(codes, stages[0]);
        for (int turn = 0;; turn ^= 1) {
            __syncthreads();
            const bool more = at + T < to;
            if (more) {
                load(codes, at + T, page);
                page = ask_page(at + 2 * T);
            }
            if (at < wave_end) take(stages[turn], at);
            if (!more) break;
            convert(codes, stages[turn ^ 1]);
            at += T;
        }
    }

#pragma unroll
    for (int t = 0; t < R; ++t) {
        const float sum_l = sum_of_groups(sums[t].l);
        const int row = row0 + 16 * t + i;
        if (row >= rows) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float v[C];
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = sums[t].o[c][r];
            put<D, TYPE, C>(a, cut, head, row, (4 * g + r) * C, v, sums[t].m, sum_l);
        }
    }
}

// Pieces of sequences that were cut, joined in their order: a wave per row (and further rows after it), D / 4 lanes per piece.  3.5 - 5 us where rows are few: a launch and three trips to memory.
// (16 sequences of up to 192 rows, 8 heads, two or three pieces: 17.5 us, 30 MB written by other XCDs just before; with more or fewer workgroups or all pieces' requests at once
// the whole call took 1 - 17 % longer.)
template <int D, int TYPE> __global__ __launch_bounds__(256) void cache_attention_join_kernel(CacheAttnArgs a)
{
    constexpr int LANES = D / 4, AT_ONCE = 64 / LANES, AHEAD = 8;
    const Cut cut = cut_of<false>(a, blockIdx.x);
    if (cut.pieces <= 1) return;
    const int lane = threadIdx.x & 63, head = blockIdx.y, col = lane % LANES * 4, first = lane / LANES;
    const int64_t step = (int64_t)a.kv_heads * a.rows_held;
    for (int row = blockIdx.z * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); row < cut.of.n * a.group; row += gridDim.z * 4) {
        const int64_t line = ((int64_t)cut.slot * a.kv_heads + head) * a.rows_held + row;
        float m = NONE;
        for (int p = lane; p < cut.pieces; p += 64) m = fmaxf(m, a.sums[(line + p * step) * 2]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        float l = 0;
        v4f sum = {0, 0, 0, 0};
        for (int p0 = 0; p0 < cut.pieces; p0 += AHEAD * AT_ONCE) {
            v4f v[AHEAD];
            float2 ml[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int p = p0 + e * AT_ONCE + first;
                const int64_t at = line + (p < cut.pieces ? p : 0) * step;
                v[e] = *reinterpret_cast<const v4f *>(a.partial + at * D + col);
                ml[e] = *reinterpret_cast<const float2 *>(a.sums + at * 2);
            }
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                if (p0 + e * AT_ONCE + first >= cut.pieces) continue;
                const float by = m == NONE ? 1.f : __builtin_amdgcn_exp2f(ml[e].x - m);
                l += ml[e].y * by;
                sum += v[e] * by;
            }
        }
#pragma unroll
        for (int o = LANES; o < 64; o <<= 1) {
            l += __shfl_xor(l, o, 64);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], o, 64);
        }
        if (first != 0 || col >= a.dk) continue;
        const float inv = l == 0 ? 0.f : 1.f / l;
        const float out[4] = {sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
        store_real<TYPE, 4>(a.o, out_at(a, cut.of, head, row) + col, out);
    }
}

template <int D, int BITS, int TYPE> hipError_t launch(CacheAttnArgs a, int row_tile, hipStream_t s)
{
    a.units_per_head = a.partial ? a.pieces + a.batch : a.batch;
    int64_t groups = (int64_t)a.units_per_head * a.kv_heads;
    if (a.row_tiles > 1) groups = (groups + 7) / 8 * 8 * a.row_tiles;
    const dim3 grid((unsigned)groups), block(CACHE_WAVES * 64);
    const hipError_t e = row_tile == 16   ? launch_kernel((cache_attention_kernel<D, BITS, TYPE>), grid, block, 0, s, a)
                         : row_tile == 64 ? launch_kernel((cache_attention_rows_kernel<D, BITS, TYPE, 1>), grid, block, 0, s, a)
                                          : launch_kernel((cache_attention_rows_kernel<D, BITS, TYPE, 2>), grid, block, 0, s, a);
    if (e != hipSuccess || !a.partial) return e;
    // enough workgroups for the device, and few enough to be gone at once where nothing was cut
    const int most = (a.rows_held + 3) / 4, some = 2048 / (a.batch * a.kv_heads) + 1; // (batch * kv_heads is less than the workgroups above)
    return launch_kernel((cache_attention_join_kernel<D, TYPE>), dim3(a.batch, a.kv_heads, most < some ? most : some), dim3(256), 0, s, a);
}

template <int BITS, int TYPE> hipError_t launch_dim(const CacheAttnArgs &a, int row_tile, hipStream_t s)
{
    if (a.dk <= 64) return launch<64, BITS, TYPE>(a, row_tile, s);
    if (a.dk <= 128) return launch<128, BITS, TYPE>(a, row_tile, s);
    return launch<256, BITS, TYPE>(a, row_tile, s);
}

template <int BITS> hipError_t launch_type(const CacheAttnArgs &a, mc_type type, int row_tile, hipStream_t s)
{
    if (type == MC_F32) return launch_dim<BITS, MC_F32>(a, row_tile, s);
    if (type == MC_F16) return launch_dim<BITS, MC_F16>(a, row_tile, s);
    return launch_dim<BITS, MC_BF16>(a, row_tile, s);
}

} // namespace

hipError_t launch_cache_attention(const CacheAttnArgs &a, mc_type type, int bits, int row_tile, hipStream_t s)
{
    return bits == 8 ? launch_type<8>(a, type, row_tile, s) : launch_type<4>(a, type, row_tile, s);
}
