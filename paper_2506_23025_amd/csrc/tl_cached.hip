// Attention over the paged 8-bit cache.
//
// A wave takes 64 tokens of one key head at a time (a tile: four blocks of 16) against up to 16 * NR query rows, which are the query heads
// that share the key head times the tokens of the sequence.  The products are v_mfma_f32_16x16x32_f16: codes become fp16 in registers, exactly, and
// the blocks' scales go on the scores and on the weights in 32 bits.
//   scores  S^T = K Q^T: A = keys, B = queries.  The rows of A are taken so that lane (column q, group g = lane / 16) receives the scores of tokens
//           16 g .. 16 g + 15 of the tile, one block: a lane has one scale of each kind, and its 16 weights are the B operand of the second product as they stand
//   output  O^T = V^T P^T: A = values, dimension by token
// Both layouts of the cache are made for this: every load is 16 bytes a lane and 256 contiguous bytes for 16 lanes, and nothing passes through LDS.
// Softmax: weights p = 2^(x - m) are summed as they are, and reach the product as p * scale_v relative to a second running reference
// R = max(x + log2 scale_v) - kLift, so that their fp16 form (2^-11) is exact enough whatever the scales of the blocks are.  The references move only when a score
// is more than 2^8 beyond them, so a tile needs no exchange between lanes.
// Bound: memory.  Short caches: a workgroup takes a row tile, its waves deal the tiles among themselves and join their sums in LDS.  Otherwise the tiles of the whole
// call stand in one row, sequence after sequence, and every wave of a grid that fills the chip once takes an equal piece of it, whatever the sequences' lengths; they are
// read on the device, so one captured launch serves every step.  Pieces of row tiles that several waves share meet in a second kernel.
// Measured: 3 sequences of up to 131072 tokens, 32 heads of 128 on 8 key heads, int8 97 us (5.9 TB/s); 48 of up to 4096, e4m3 47.5 us (5.05 TB/s, 42 of them here and 5 in the second
// kernel); 16 of up to 2047 with 32 key heads 32 us (4.3 TB/s).  One sequence of 700 tokens with 16 heads 7.2 us, a chain of reads: lengths, pages, scales, codes.
#include "tl_attn.hpp"

#include <cmath>
#include <type_traits>

namespace tl {
namespace {

constexpr int kWaves = 4;
constexpr int kWavesAll = 2048;           // waves that share a call's tiles: two on each SIMD of 256 CUs, or one where a row tile is of 32 rows
constexpr int kFewRows = 1024;            // up to so many rows a workgroup joins the parts of each, of 8 waves up to a quarter of it; beyond a wave

constexpr float kInf = __builtin_inff();

struct Shape {
    int per;                              // tokens of a row tile
    int heads;                            // query heads of a row tile
    int subs;                             // row tiles that the query heads of a key head need
    int rows;                             // per * heads
    int nr;                               // blocks of 16 rows in a row tile
    int ys;                               // key heads * subs: what a token of the cache is read for
    int pieces;                           // that the row of all tiles is cut into, each for ys waves
    int64_t tiles;                        // row tiles of the call at most
};

inline Shape shape_of(int64_t seqs, int64_t tokens, bool one, int group, int kv_heads)
{
    Shape p;
    // Two blocks of 16 rows share the widened codes where the tokens of a sequence fill them.  One token each keeps to one, however many heads share its keys: 64 sequences of up to 800
    // with 32 heads on one of 128 9.8 us, with two 13.6 (over up to 9000, 64 heads on 2 of 64, 35.6 and 33.8).
    p.nr = tokens * group > 16 * seqs && tokens > seqs ? 2 : 1;
    const int most = 16 * p.nr;
    p.heads = group < most ? group : most;
    p.subs = (group + p.heads - 1) / p.heads;
    p.per = one ? 1 : most / p.heads;
    p.rows = p.per * p.heads;
    p.ys = kv_heads * p.subs;
    p.pieces = kWavesAll / p.nr / p.ys;
    if (p.pieces < 1) p.pieces = 1;
    p.tiles = one ? seqs : tokens / p.per + seqs;
    return p;
}

// About how many row tiles of all key heads there are: sequences of several tokens end anywhere in one.
inline double likely_tiles(int seqs, int tokens, const Shape& p)
{
    return (p.per == 1 ? double(tokens) : fmax(double(tokens) / p.per + 0.5 * seqs, fmin(tokens, seqs))) * p.ys;
}

constexpr int kExtra = 4;                 // floats beside a row's sums: m, l, R

// Eight codes as fp16, in order and exact: of whole numbers, code + 128 in the mantissa of 1024, less 1152.  (Scores of the codes + 1152, with what that adds taken off their sums at the start, spare the
// subtraction for keys, and round sums of numbers up to nine times as large: 0.125 of a code's step each where queries have a common part of 16.  One token of 16 sequences of up to 2047 with 32 key heads 32.9 us so,
// 32.4 with the subtraction; one token over 700 6.9 and 7.2; 300 tokens of 2 over 4000 with 32 heads on 8 113 and 114.)
template <bool FP8>
__device__ inline f16x8 widen(uint32_t a, uint32_t b)
{
    union { f16x8 v; f16x2 p[4]; uint32_t w[4]; } r;
    if constexpr (FP8) {
        r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
        r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
        r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
        r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    } else {
        a ^= 0x80808080u;
        b ^= 0x80808080u;
        r.w[0] = __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u);
        r.w[1] = __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u);
        r.w[2] = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
        r.w[3] = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
        const f16x2 c = {_Float16(1152.0f), _Float16(1152.0f)};
#pragma unroll
        for (int i = 0; i < 4; ++i) r.p[i] -= c;
    }
    return r.v;
}

// 16 bytes of codes; ONCE: that nobody else will ask for.
template <bool ONCE>
__device__ inline u32x4 fetch(const uint8_t* p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else return *reinterpret_cast<const u32x4*>(p);
}

__device__ inline float inverse(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }
__device__ inline float finite(float x) { return x == -kInf ? 0.0f : x; }
__device__ inline float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ inline float power(float x) { return __builtin_amdgcn_exp2f(x); }

// Positions that a sequence's pages hold.
__device__ inline int64_t room(const Cache& c) { return c.pages_per_seq << (c.page_shift + 4); }

// A sequence: its tokens in the call, those before them, and the tiles and row tiles that it needs.
struct Need {
    int first, n, past, tiles, rts;
    __device__ inline double share() const { return double(tiles) * double(rts); }
};

__device__ inline Need need_of(const CachedArgs& a, const Shape& p, int s)
{
    const Span sp = span(a.b, s);
    const int past = cached_of(a.b, s);
    Need need{sp.first, sp.n, past, 0, 0};
    if (sp.n == 0) return need;
    int64_t len = past < 0 ? 0 : int64_t(past) + sp.n;
    if (len > room(a.c)) len = room(a.c);
    need.tiles = int((len + 63) >> 6);
    need.rts = p.per == 1 ? sp.n : (sp.n + p.per - 1) / p.per;
    return need;
}

__device__ inline Need of_lane(const Need& x, int lane)
{
    return {__builtin_amdgcn_readlane(x.first, lane), __builtin_amdgcn_readlane(x.n, lane), __builtin_amdgcn_readlane(x.past, lane),
            __builtin_amdgcn_readlane(x.tiles, lane), __builtin_amdgcn_readlane(x.rts, lane)};
}

// Sums over the wave, exact: whole numbers below 2^53 in doubles.
template <int CTRL, int ROWS>
__device__ inline double moved(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = tl::moved<CTRL, ROWS>(int(uint32_t(b))), hi = tl::moved<CTRL, ROWS>(int(uint32_t(b >> 32)));
    return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}

__device__ inline double scanned(double x)
{
    x += moved<0x111, 15>(x);             // from the lane 1, 2, 4 and 8 before in the row of 16
    x += moved<0x112, 15>(x);
    x += moved<0x114, 15>(x);
    x += moved<0x118, 15>(x);
    x += moved<0x142, 10>(x);             // a row's last lane to the next row, rows 1 and 3
    x += moved<0x143, 12>(x);             // lane 31 to rows 2 and 3
    return x;
}

__device__ inline double of_lane(double x, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane(int(uint32_t(b)), lane), hi = __builtin_amdgcn_readlane(int(uint32_t(b >> 32)), lane);
    return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}

// The call's tiles in one row: sequence after sequence, of each its row tiles one after the other.
__device__ inline double all_tiles(const CachedArgs& a, const Shape& p)
{
    const int lane = threadIdx.x & 63, per = (a.b.seqs + 63) >> 6;
    double w = 0.0;
    for (int i = 0; i < per; ++i)
        if (lane * per + i < a.b.seqs) w += need_of(a, p, lane * per + i).share();
    return of_lane(scanned(w), 63);
}

// The sequence that holds tile x of the row, and how many tiles stand before it.
struct Found { int seq; double before; };
__device__ inline Found find_tile(const CachedArgs& a, const Shape& p, double x)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, count = a.b.seqs;
    double before = 0.0;
    while (true) {
        const int per = (count + 63) >> 6;
        double w = 0.0;
        for (int i = 0; i < per; ++i)
            if (lane * per + i < count) w += need_of(a, p, lo + lane * per + i).share();
        const double to = scanned(w);
        const uint64_t there = __ballot(before + to > x);
        if (!there) return {-1, 0.0};
        const int owner = __builtin_ctzll(there);
        before += of_lane(to, owner) - of_lane(w, owner);
        lo += owner * per;
        count = count - owner * per < per ? count - owner * per : per;
        if (per == 1) return {lo, before};
    }
}

// First tile of piece i, of `all` tiles: equal shares, or one each where there are fewer tiles than pieces.  Whole numbers below 2^52 with a
// divisor below 2^12: the quotient's rounding cannot reach the next whole number.
__device__ inline double piece_begin(const Shape& p, double all, int i)
{
    if (all <= p.pieces) return fmin(double(i), all);
    return floor(all * double(i) / double(p.pieces));
}

// The piece that holds tile x.
__device__ inline int piece_of(const Shape& p, double all, double x)
{
    if (all <= p.pieces) return int(x);
    int i = int((x + 1.0) * p.pieces / all);
    if (i > p.pieces - 1) i = p.pieces - 1;
    while (i > 0 && piece_begin(p, all, i) > x) --i;
    while (i < p.pieces - 1 && piece_begin(p, all, i + 1) <= x) ++i;
    return i;
}

struct Row { float m, l, R; };

// Where the parts of a row tile are: in the pieces from w0 on, so many of them.
struct Parts { int w0, n; };
__device__ inline Parts* parts_of(const CachedArgs& a, const Shape& p, int dp)
{
    return reinterpret_cast<Parts*>(a.part + int64_t(2 * p.pieces) * p.ys * p.rows * (dp + kExtra));
}

// A row's sums of a piece: its second place has a row tile that begins in it, its first the rest of one that an earlier piece began.
__device__ inline float* part_row(const CachedArgs& a, const Shape& p, int dp, int piece, bool begins, int y, int r)
{
    return a.part + (((int64_t(piece) * 2 + begins) * p.ys + y) * p.rows + r) * (dp + kExtra);
}

// One row tile of one key head: its queries, and its sums over tiles begin, begin + step, ... below end.
// A tile is in registers or on its way to them.  EXACT: the head has CH * 16 dimensions, else fewer.
template <bool FP8, int CH, bool EXACT, int NR>
struct Walk {
    static constexpr int J = (CH + 3) / 4;
    f16x8 q[NR][J][2];
    int64_t sees[NR], least, most;        // positions that this lane's rows see; the fewest of the tile, and the most, within the pages
    f32x4 o[NR][CH];
    float m[NR], l[NR], R[NR];
    int first, tokens, heads, rows;       // tokens of the sequence before the tile, tokens and heads in it

    __device__ inline void start(const CachedArgs& a, const Shape& p, const Span& sp, int past, int rt, int head, int sub)
    {
        const int m16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4, chunks = EXACT ? CH : a.c.dim >> 4;
        first = rt * p.per;
        tokens = sp.n - first < p.per ? sp.n - first : p.per;
        heads = a.group - sub * p.heads < p.heads ? a.group - sub * p.heads : p.heads;
        rows = tokens * p.heads;                             // those of heads beyond the group are computed and dropped
        least = past < 0 ? 0 : int64_t(past) + first + 1;
        most = past < 0 ? 0 : int64_t(past) + first + tokens;
        if (most > room(a.c)) most = room(a.c);              // a length beyond the pages asks for no tiles that cannot be there
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            // row r is token r / p.heads, head r % p.heads
            const int r = n * 16 + m16, tr = r / p.heads, hr = r - tr * p.heads;
            const bool there = r < rows && hr < heads;
            const int t = there ? tr : 0, h = there ? hr : 0;
            sees[n] = past < 0 ? 0 : int64_t(past) + first + t + 1;
            const _Float16* row = a.q.p + int64_t(sp.first + first + t) * a.q.token + int64_t(head * a.group + sub * p.heads + h) * a.q.head;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int c = 4 * j + g;
                    f16x8 x = *reinterpret_cast<const f16x8*>(row + (c < chunks ? c : 0) * 16 + i * 8);
                    if (c >= chunks) x = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
                    if (a.scale < 0.0f) x = -x;              // so that the largest sum is the largest score
                    q[n][j][i] = x;
                }
            m[n] = -kInf;
            R[n] = -kInf;
            l[n] = 0.0f;
#pragma unroll
            for (int d = 0; d < CH; ++d) o[n][d] = f32x4{0, 0, 0, 0};
        }
    }

    // A query with an infinity: its scores are infinities of both signs or NaN, and their softmax NaN.  All negative, they would look unseen: all of the query becomes NaN.
    __device__ inline void look_at_queries()
    {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            f16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};           // an infinity or a NaN leaves no 0
#pragma unroll
            for (int j = 0; j < J; ++j) zero += q[n][j][0] * _Float16(0.0f) + q[n][j][1] * _Float16(0.0f);
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) odd |= !(zero[e] == _Float16(0.0f));
            if (__any(odd)) {
                float x = odd ? __builtin_nanf("") : 0.0f;
                x += __shfl_xor(x, 16);
                x += __shfl_xor(x, 32);
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) q[n][j][i] += _Float16(x);
            }
        }
    }

    __device__ inline void walk(const CachedArgs& a, int seq, int head, int begin, int end, int step)
    {
        const int m16 = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4, chunks = EXACT ? CH : a.c.dim >> 4;
        const float scale = fabsf(a.scale);
        const int64_t block_bytes = int64_t(256) * chunks, blocks = int64_t(1) << a.c.page_shift;
        const int in_page = int(blocks - 1);
        auto page_at = [&](int64_t block) { return page_of(a.c, seq, block); };
        auto place = [&](int page, int64_t block) { return (int64_t(page < 0 ? 0 : page) * a.c.kv_heads + head) * blocks + (block & in_page); };
        u32x4 kw[4][J], vw[CH];
        float ks = 0.0f, vs = 0.0f;
        bool there = false;                                  // the lane's block has a page
        // Loads come back in order, so what is needed first is asked for first: the pages of the tile after, a tile's scales, its keys, its values.
        int next_k = 0, next_v = 0;
        int64_t value_block = 0;
        auto ask_pages = [&](int tile) {
            next_k = page_at(int64_t(tile) * 4 + (m16 >> 2));
            next_v = page_at(int64_t(tile) * 4 + g);
        };
        auto load_k = [&](int tile) {
            const int64_t key_block = place(next_k, int64_t(tile) * 4 + (m16 >> 2));
            value_block = place(next_v, int64_t(tile) * 4 + g);
            there = next_v >= 0;
            ask_pages(tile + step);
            ks = a.c.ks[value_block];
            vs = a.c.vs[value_block];
            const uint8_t* from = a.c.k + key_block * block_bytes + (m16 & 3) * 16;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int c = EXACT || 4 * j + g < chunks ? 4 * j + g : 0;
                    kw[b][j] = fetch<NR == 1>(from + (b * chunks + c) * 64);
                }
        };
        auto load_v = [&] {
            const uint8_t* from = a.c.v + value_block * block_bytes + m16 * 16;
#pragma unroll
            for (int d = 0; d < CH; ++d) vw[d] = fetch<NR == 1>(from + (EXACT || d < chunks ? d : 0) * 256);
        };
        begin = same(begin);
        end = same(end);
        if (begin >= end) return;
        ask_pages(begin);
        load_k(begin);
        look_at_queries();                                   // while the first keys are on their way
        load_v();
        for (int tile = begin; tile < end; tile += step) {
            const bool more = tile + step < end;
            const bool inside = there;
            const bool masked = int64_t(tile) * 64 + 64 > least || !__all(inside);
            const float ksc = ks * scale, vsc = vs;
            f32x4 s[NR][4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
#pragma unroll
                for (int n = 0; n < NR; ++n) s[n][b] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const f16x8 k0 = widen<FP8>(kw[b][j][0], kw[b][j][1]), k1 = widen<FP8>(kw[b][j][2], kw[b][j][3]);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[n][j][0], s[n][b], 0, 0, 0);
                        s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[n][j][1], s[n][b], 0, 0, 0);
                    }
                }
            }
            if (more) load_k(tile + step);
            const float lv = __builtin_amdgcn_logf(vsc);
            f16x8 w[NR][2];
            auto weigh = [&](auto some) {
                constexpr bool MASKED = decltype(some)::value;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    // of the lane's 16 tokens those before `seen` are there
                    int seen = 16;
                    if constexpr (MASKED) {
                        const int64_t x = sees[n] - int64_t(tile) * 64 - g * 16;
                        seen = !inside || x < 0 ? 0 : x > 16 ? 16 : int(x);
#pragma unroll
                        for (int i = 0; i < 16; ++i) if (i >= seen) s[n][i >> 2][i & 3] = -kInf;
                    }
                    float mx = -kInf;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) mx = max3(mx, s[n][i >> 2][i & 3], s[n][i >> 2][(i & 3) + 1]);
                    if (!MASKED || mx != -kInf) mx *= ksc;
                    const float top = MASKED && mx == -kInf ? -kInf : mx + (lv - kLift);
                    if (__any(mx > m[n] + kSlack || top > R[n] + kSlack)) {
                        // each row by itself: what one row sees does not change how another is rounded
                        float a1 = mx, a2 = top;
                        a1 = fmaxf(a1, __shfl_xor(a1, 16));
                        a2 = fmaxf(a2, __shfl_xor(a2, 16));
                        a1 = fmaxf(a1, __shfl_xor(a1, 32));
                        a2 = fmaxf(a2, __shfl_xor(a2, 32));
                        const bool moves = a1 > m[n] + kSlack || a2 > R[n] + kSlack;
                        a1 = moves ? fmaxf(a1, m[n]) : m[n];
                        a2 = moves ? fmaxf(a2, R[n]) : R[n];
                        l[n] *= power(m[n] - finite(a1));
                        const float f = power(R[n] - finite(a2));
#pragma unroll
                        for (int d = 0; d < CH; ++d) o[n][d] *= f;
                        m[n] = a1;
                        R[n] = a2;
                    }
                    const float mb = finite(m[n]);
                    // p * scale_v relative to R
                    float f = power(fminf(lv + mb - finite(R[n]), 126.0f));
                    if (!(vsc == vsc)) f = vsc;
                    union { f16x8 v[2]; _Float16 h[16]; } c;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float x = power(__builtin_fmaf(s[n][i >> 2][i & 3], ksc, -mb)), y = x * f;
                        if constexpr (MASKED) {
                            x = i < seen ? x : 0.0f;
                            y = i < seen ? y : 0.0f;
                        }
                        l[n] += x;
                        c.h[i] = _Float16(y);
                    }
                    w[n][0] = c.v[0];
                    w[n][1] = c.v[1];
                }
            };
            if (masked) {
                weigh(std::true_type{});
                // A weight of 0 does not take a NaN out of a sum, and bytes that no token of the sequence was written to, or those read in place of a page that is missing, may be codes
                // that stand for one (whole numbers have none): they become 0.
                if constexpr (FP8) {
                    const int64_t x = most - int64_t(tile) * 64 - g * 16;
                    const int held = !inside || x < 0 ? 0 : x > 16 ? 16 : int(x);
                    u32x4 keep;
#pragma unroll
                    for (int i = 0; i < 4; ++i) keep[i] = held >= 4 * i + 4 ? ~0u : held > 4 * i ? (1u << (held - 4 * i) * 8) - 1 : 0u;
#pragma unroll
                    for (int d = 0; d < CH; ++d) vw[d] &= keep;
                }
            } else {
                weigh(std::false_type{});
            }
#pragma unroll
            for (int d = 0; d < CH; ++d) {
                const f16x8 v0 = widen<FP8>(vw[d][0], vw[d][1]), v1 = widen<FP8>(vw[d][2], vw[d][3]);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[n][0], o[n][d], 0, 0, 0);
                    o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[n][1], o[n][d], 0, 0, 0);
                }
            }
            if (more) load_v();
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
        }
    }

    // This lane's quarter of its row in block n, where the wave has seen all of it.
    __device__ inline void write_row(const CachedArgs& a, _Float16* out, int n, int g) const
    {
        const float x = inverse(l[n]) * power(R[n] - finite(m[n]));
#pragma unroll
        for (int d = 0; d < CH; ++d) {
            if (!EXACT && d * 16 >= a.c.dim) continue;
            f16x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = _Float16(o[n][d][j] * x);
            *reinterpret_cast<f16x4*>(out + d * 16 + g * 4) = v;
        }
    }
};

__device__ inline _Float16* out_row(const CachedArgs& a, const Shape& p, int row, int head, int sub, int h)
{
    return a.out.p + int64_t(row) * a.out.token + int64_t(head * a.group + sub * p.heads + h) * a.out.head;
}

// A workgroup for each row tile of each key head.
template <bool FP8, int CH, bool EXACT, int NR, int W>
__global__ __launch_bounds__(64 * W, CH * NR > 8 ? 1 : 2) void short_kernel(CachedArgs a, Shape p)
{
    constexpr int DP = CH * 16;
    const int lane = threadIdx.x & 63, wave = same(threadIdx.x >> 6);
    const int m16 = lane & 15, g = lane >> 4;
    Item it{int(blockIdx.x), 0};
    if (a.b.start) it = find_item(a.b, int(blockIdx.x), p.per, 1);
    it = {same(it.seq), same(it.i)};
    if (it.seq < 0) return;
    Span sp = span(a.b, it.seq);
    sp = {same(sp.first), same(sp.n)};
    if (it.i * p.per >= sp.n) return;
    const int head = int(blockIdx.y) / p.subs, sub = int(blockIdx.y) - head * p.subs;
    Walk<FP8, CH, EXACT, NR> w;
    w.start(a, p, sp, same(cached_of(a.b, it.seq)), it.i, head, sub);
    w.walk(a, it.seq, head, wave, int((w.most + 63) >> 6), W);

    __shared__ float sums[W][16 * NR][DP + 4];
    __shared__ Row stats[W][16 * NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        if (g == 0) stats[wave][n * 16 + m16] = {w.m[n], w.l[n], w.R[n]};
#pragma unroll
        for (int d = 0; d < CH; ++d) *reinterpret_cast<f32x4*>(&sums[wave][n * 16 + m16][d * 16 + g * 4]) = w.o[n][d];
    }
    __syncthreads();
    constexpr int kQuads = DP / 4;
    for (int i = threadIdx.x; i < w.rows * kQuads; i += 64 * W) {
        const int r = i / kQuads, d = (i - r * kQuads) * 4, t = r / p.heads, h = r - t * p.heads;
        if (h >= w.heads || d >= a.c.dim) continue;
        float M = -kInf, L = 0.0f;
#pragma unroll
        for (int v = 0; v < W; ++v) M = fmaxf(M, stats[v][r].m);
        M = finite(M);
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < W; ++v) {
            L += stats[v][r].l * power(stats[v][r].m - M);
            sum += *reinterpret_cast<f32x4*>(&sums[v][r][d]) * power(stats[v][r].R - M);
        }
        sum *= inverse(L);
        f16x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = _Float16(sum[j]);
        *reinterpret_cast<f16x4*>(out_row(a, p, sp.first + w.first + t, head, sub, h) + d) = y;
    }
}

// A wave for each row tile of each key head.
template <bool FP8, int CH, bool EXACT, int NR>
__global__ __launch_bounds__(64 * kWaves, CH * NR > 8 ? 1 : 2) void wave_kernel(CachedArgs a, Shape p)
{
    const int lane = threadIdx.x & 63, m16 = lane & 15, g = lane >> 4;
    const int x = int(blockIdx.x) * kWaves + same(threadIdx.x >> 6);
    Item it{x < a.b.seqs ? x : -1, 0};
    if (a.b.start) it = find_item(a.b, x, p.per, 1);
    it = {same(it.seq), same(it.i)};
    if (it.seq < 0) return;
    Span sp = span(a.b, it.seq);
    sp = {same(sp.first), same(sp.n)};
    if (it.i * p.per >= sp.n) return;
    const int head = int(blockIdx.y) / p.subs, sub = int(blockIdx.y) - head * p.subs;
    Walk<FP8, CH, EXACT, NR> w;
    w.start(a, p, sp, same(cached_of(a.b, it.seq)), it.i, head, sub);
    w.walk(a, it.seq, head, 0, int((w.most + 63) >> 6), 1);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int r = n * 16 + m16, t = r / p.heads, h = r - t * p.heads;
        if (r < w.rows && h < w.heads) w.write_row(a, out_row(a, p, sp.first + w.first + t, head, sub, h), n, g);
    }
}

// A wave for each piece of the row of all tiles and each key head: neighbouring waves read the heads of the same tokens, which lie side by side in
// a page.  A row tile that a piece has whole is written out, of the others the sums go to the workspace.
template <bool FP8, int CH, bool EXACT, int NR>
__global__ __launch_bounds__(64 * kWaves, CH * NR > 8 ? 1 : 2) void piece_kernel(CachedArgs a, Shape p)
{
    constexpr int DP = CH * 16;
    const int lane = threadIdx.x & 63, m16 = lane & 15, g = lane >> 4;
    const int wave = int(blockIdx.x) * kWaves + same(threadIdx.x >> 6), piece = wave / p.ys, y = wave - piece * p.ys;
    if (piece >= p.pieces) return;
    const int head = y / p.subs, sub = y - head * p.subs;
    double all, at, stop;
    Found f;
    Need need;
    if (a.b.seqs <= 64) {
        // a lane for each sequence: one look at the lengths is all
        Need mine{0, 0, 0, 0, 0};
        if (lane < a.b.seqs) mine = need_of(a, p, lane);
        const double w = mine.share(), to = scanned(w);
        all = of_lane(to, 63);
        at = piece_begin(p, all, piece);
        stop = piece_begin(p, all, piece + 1);
        if (same(at < stop) == 0) return;
        const int owner = __builtin_ctzll(__ballot(to > at));
        f = {owner, of_lane(to, owner) - of_lane(w, owner)};
        need = of_lane(mine, owner);
    } else {
        all = all_tiles(a, p);
        at = piece_begin(p, all, piece);
        stop = piece_begin(p, all, piece + 1);
        if (same(at < stop) == 0) return;
        f = find_tile(a, p, at);
        if (same(f.seq) < 0) return;
        need = need_of(a, p, same(f.seq));
    }
    int seq = same(f.seq);
    // row tile, and tile in it
    const double inside = at - f.before;
    double u = need.rts == 1 ? 0.0 : floor(inside / double(need.tiles));
    if (u * need.tiles > inside) u -= 1.0;
    if ((u + 1.0) * need.tiles <= inside) u += 1.0;
    int rt = same(int(u)), tile = same(int(inside - u * need.tiles));
    while (true) {
        const int tiles = same(need.tiles), rts = same(need.rts);
        const double left = stop - at;
        const int to = same(double(tiles - tile) <= left ? tiles : tile + int(left));
        const Span sp = {same(need.first), same(need.n)};
        Walk<FP8, CH, EXACT, NR> w;
        w.start(a, p, sp, same(need.past), rt, head, sub);
        const int seen = int((w.most + 63) >> 6);
        w.walk(a, seq, head, tile, to < seen ? to : seen, 1);
        const bool whole = tile == 0 && to == tiles;
        if (tile == 0 && y == 0 && lane == 0)
            parts_of(a, p, DP)[a.b.start ? item_base(a.b, seq, p.per, 1) + rt : seq] = {piece, whole ? 1 : piece_of(p, all, at + tiles - 1.0) - piece + 1};
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int r = n * 16 + m16, t = r / p.heads, h = r - t * p.heads;
            if (r >= w.rows || h >= w.heads) continue;
            if (whole) {
                w.write_row(a, out_row(a, p, sp.first + w.first + t, head, sub, h), n, g);
            } else {
                float* row = part_row(a, p, DP, piece, tile == 0, y, r);
#pragma unroll
                for (int d = 0; d < CH; ++d) *reinterpret_cast<f32x4*>(row + d * 16 + g * 4) = w.o[n][d];
                if (g == 0) *reinterpret_cast<f32x4*>(row + DP) = f32x4{w.m[n], w.l[n], w.R[n], 0.0f};
            }
        }
        at += double(to - tile);
        if (same(at < stop) == 0) break;
        tile = 0;
        if (++rt == rts) {
            rt = 0;
            do {
                if (++seq >= a.b.seqs) return;
                need = need_of(a, p, seq);
            } while (same(need.tiles * (need.rts > 0)) == 0);
        }
    }
}

// Joins the pieces of row tiles that several waves share.  A row is a wave's, or of W = 4 or 8 of a workgroup where there are so few rows that the
// parts of each are worth dealing out.  Four dimensions are a lane's, and the parts go round among the lanes that have the same ones; the sums of the first
// are asked for before it is known how they weigh.
template <int CH, int W>
__global__ __launch_bounds__(64 * (W == 1 ? kWaves : W)) void join_kernel(CachedArgs a, Shape p)
{
    constexpr int DP = CH * 16, kQuads = DP / 4, kGroups = 64 * W / kQuads, kAhead = 8;
    const int lane = threadIdx.x & 63, wave = same(threadIdx.x >> 6);
    const int tid = W == 1 ? lane : int(threadIdx.x);
    Item it{int(blockIdx.x), 0};
    if (a.b.start) it = find_item(a.b, int(blockIdx.x), p.per, 1);
    it = {same(it.seq), same(it.i)};
    if (it.seq < 0) return;
    const Parts found = parts_of(a, p, DP)[blockIdx.x];      // of a sequence without tiles: anything
    const Need need = need_of(a, p, it.seq);
    const int w0 = same(found.w0), parts = same(found.n), n = same(need.n), first = it.i * p.per;
    const bool none = same(need.tiles) == 0;
    if (!none && parts == 1) return;
    const int r = W == 1 ? int(blockIdx.z) * kWaves + wave : int(blockIdx.z), t = r / p.heads, h = r - t * p.heads;
    const int head = int(blockIdx.y) / p.subs, sub = int(blockIdx.y) - head * p.subs;
    if (r >= p.rows || first + t >= n || sub * p.heads + h >= a.group) return;
    const int quad = tid % kQuads, d = quad * 4, mine = tid / kQuads;
    _Float16* out = out_row(a, p, same(need.first) + first + t, head, sub, h) + d;
    if (none) {
        if (mine == 0 && d < a.c.dim) *reinterpret_cast<f16x4*>(out) = f16x4{0, 0, 0, 0};
        return;
    }
    // part c is in piece w0 + c: the first in its second place, the others in their first
    auto row_of = [&](int c) { return part_row(a, p, DP, w0 + c, c == 0, int(blockIdx.y), r); };
    f32x4 ahead[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int c = mine + u * kGroups;
        ahead[u] = *reinterpret_cast<const f32x4*>(row_of(c < parts ? c : 0) + d);
    }
    // references first, over all parts
    f32x4 stat = {-kInf, 0, -kInf, 0};
    if (tid < parts) stat = *reinterpret_cast<const f32x4*>(row_of(tid) + DP);
    float M = stat[0];
    for (int c = tid + 64 * W; c < parts; c += 64 * W) M = fmaxf(M, row_of(c)[DP]);
    for (int k = 32; k; k >>= 1) M = fmaxf(M, __shfl_xor(M, k));
    __shared__ float most[W], total[W];
    __shared__ f32x4 sums[W][kQuads];
    if constexpr (W > 1) {
        if (lane == 0) most[wave] = M;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < W; ++v) M = fmaxf(M, most[v]);
    }
    M = finite(M);
    float L = 0.0f;
    f32x4 x = {0, 0, 0, 0};
    for (int c = tid; c < parts; c += 64 * W) {
        if (c != tid) stat = *reinterpret_cast<const f32x4*>(row_of(c) + DP);
        L += stat[1] * power(stat[0] - M);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int c = mine + u * kGroups;
        if (c < parts) x += ahead[u] * power(row_of(c)[DP + 2] - M);
    }
#pragma unroll 4
    for (int c = mine + kAhead * kGroups; c < parts; c += kGroups) {
        const float* row = row_of(c);
        x += *reinterpret_cast<const f32x4*>(row + d) * power(row[DP + 2] - M);
    }
    for (int k = 32; k; k >>= 1) L += __shfl_xor(L, k);
    for (int k = 32; k >= kQuads; k >>= 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += __shfl_xor(x[j], k);
    }
    if constexpr (W > 1) {
        if (lane == 0) total[wave] = L;
        if (lane < kQuads) sums[wave][lane] = x;
        __syncthreads();
        L = 0.0f;
        x = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < W; ++v) {
            L += total[v];
            x += sums[v][quad];
        }
    }
    if (mine == 0 && d < a.c.dim) {
        x *= inverse(L);
        f16x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = _Float16(x[j]);
        *reinterpret_cast<f16x4*>(out) = y;
    }
}

inline int padded(int64_t dim) { return dim <= 64 ? 64 : 128; }

template <bool FP8, int CH, bool EXACT, int NR>
hipError_t launch(const CachedArgs& a, const Shape& p, bool alone, int64_t longest, hipStream_t s)
{
    const unsigned y = unsigned(p.ys);
    if (alone) {
        // Tiles of the longest sequence to one wave or dealt to four: rounds of as many waves as the chip holds, each with 5 us before its first tile is there and `step` for each
        // further one.  Measured: 119 sequences of 5 tokens with 32 key heads of 128 32 us dealt to four, 16 with one wave each.
        const double tiles = double((longest + 63) / 64), units = likely_tiles(a.b.seqs, a.b.tokens, p), waves = CH * NR > 8 ? 1024.0 : 2048.0, step = NR == 1 ? 1.2 : CH > 4 ? 2.3 : 1.4;
        const double by_wave = fmax(units / waves, 1.0) * (5.0 + step * tiles), by_four = fmax(units * kWaves / waves, 1.0) * (5.0 + step * ceil(tiles / kWaves));
        if (by_wave < by_four) {
            wave_kernel<FP8, CH, EXACT, NR><<<dim3(unsigned((p.tiles + kWaves - 1) / kWaves), y), 64 * kWaves, 0, s>>>(a, p);
            return hipGetLastError();
        }
        if constexpr (CH * NR <= 8) {
            // eight waves where that leaves two on a SIMD: 45 tokens of 6 sequences over 3001 with 32 heads of 64 on 8 21.6 us with four, 18.7; one token of 64 over up to 900 with 8 key heads of 128
            // (512 row tiles) 18.6 and 21
            if (units <= (NR == 1 ? 256.0 : 512.0)) {
                short_kernel<FP8, CH, EXACT, NR, 2 * kWaves><<<dim3(unsigned(p.tiles), y), 64 * 2 * kWaves, 0, s>>>(a, p);
                return hipGetLastError();
            }
        }
        short_kernel<FP8, CH, EXACT, NR, kWaves><<<dim3(unsigned(p.tiles), y), 64 * kWaves, 0, s>>>(a, p);
        return hipGetLastError();
    }
    piece_kernel<FP8, CH, EXACT, NR><<<unsigned((p.pieces * p.ys + kWaves - 1) / kWaves), 64 * kWaves, 0, s>>>(a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Waves for a row: one token over 23827, 3 heads (up to 373 parts a row) 16.7 us with four, 14.4 with eight, 14.2 with sixteen; 3 over up to 131072, 32 heads 98.4, 96.9 and 97; 24 over
    // up to 2500, 16 heads on 2 10.8 and 11.7; 128 over up to 4000, 32 heads 116 with one and four
    const int64_t all_rows = p.tiles * p.ys * p.rows;
    if (all_rows <= kFewRows / 4) join_kernel<CH, 2 * kWaves><<<dim3(unsigned(p.tiles), y, unsigned(p.rows)), 64 * 2 * kWaves, 0, s>>>(a, p);
    else if (all_rows <= kFewRows) join_kernel<CH, kWaves><<<dim3(unsigned(p.tiles), y, unsigned(p.rows)), 64 * kWaves, 0, s>>>(a, p);
    else join_kernel<CH, 1><<<dim3(unsigned(p.tiles), y, unsigned((p.rows + kWaves - 1) / kWaves)), 64 * kWaves, 0, s>>>(a, p);
    return hipGetLastError();
}

template <bool FP8, int NR>
hipError_t launch_dim(const CachedArgs& a, const Shape& p, bool alone, int64_t longest, hipStream_t s)
{
    if (a.c.dim == 128) return launch<FP8, 8, true, NR>(a, p, alone, longest, s);
    if (a.c.dim == 64) return launch<FP8, 4, true, NR>(a, p, alone, longest, s);
    return a.c.dim < 64 ? launch<FP8, 4, false, NR>(a, p, alone, longest, s) : launch<FP8, 8, false, NR>(a, p, alone, longest, s);
}

template <bool FP8>
hipError_t launch_type(const CachedArgs& a, const Shape& p, bool alone, int64_t longest, hipStream_t s)
{
    return p.nr == 2 ? launch_dim<FP8, 2>(a, p, alone, longest, s) : launch_dim<FP8, 1>(a, p, alone, longest, s);
}

}  // namespace

size_t cached_workspace(int64_t seqs, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t dim)
{
    size_t most = 0;
    for (const bool one : {false, true}) {
        if (one && tokens != seqs) continue;
        const Shape p = shape_of(seqs, tokens, one, int(q_heads / kv_heads), int(kv_heads));
        const size_t n = size_t(2 * p.pieces) * p.ys * p.rows * (padded(dim) + kExtra) * sizeof(float) + size_t(p.tiles) * sizeof(Parts);
        if (n > most) most = n;
    }
    return (most + 15) / 16 * 16;
}

hipError_t launch_cached(const CachedArgs& a, int64_t longest, hipStream_t s)
{
    const Shape p = shape_of(a.b.seqs, a.b.tokens, !a.b.start, a.group, a.c.kv_heads);
    // Up to so many tiles a sequence is left to one workgroup: the partial sums and the second kernel would cost more than a finer split saves, and more so with many row tiles, or of 32
    // rows.  In us, so and with pieces, sequences of one length, int8, 32 query heads of 128: one token of 8, 8 key heads, 15 tiles 8.6 and 11.3, 30 tiles 14.2 and 14.2; of 24 with 8 heads of 96, 22
    // tiles 13 and 19; of 64 with 8, 32 tiles 42 and 48; of 16 with 32, 32 tiles 41 and 47; of 40 with 8, 47 tiles 44 and 47; 64 tokens of 2, 16 heads on 2, 32 tiles 23 and 26; 16 of 4, 16 heads
    // on 4, 32 tiles 23 and 24.  Heads of 64: 45 tokens of 6, 71 tiles 52 and 49 (e4m3 47 and 47); 5 of 3, 24 tiles 12 and 13; one token of 5, 32 tiles 10.3 and 10.8.  Where lengths differ a
    // workgroup has the longest to itself while others are done, which is why the limits lie below where the two meet here: one token of 40 with 8 key heads over up to 47 tiles 35 and 33.
    const bool many = likely_tiles(a.b.seqs, a.b.tokens, p) >= (p.nr == 2 ? 32.0 : 128.0);
    const int64_t alone_tiles = a.c.dim <= 64 ? (many && p.nr == 2 ? 80 : 24) : !many ? 16 : p.nr == 2 ? 32 : 36;
    const bool alone = longest > 0 && longest <= alone_tiles * 64;
    return a.c.fp8 ? launch_type<true>(a, p, alone, longest, s) : launch_type<false>(a, p, alone, longest, s);
}

}  // namespace tl
